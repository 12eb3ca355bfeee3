// kvx_ops.h -- launch parameters of the kernels that compute with a paged
// cache (append, attend, select, transfer of kept rows).  Not part of the
// public interface (include/kvx.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvx.h"
#include "kvx_internal.h"

namespace kvx {

// Most workgroups of one launch of these kernels: the work-items (up to 1024 a
// workgroup) stay below 2^32.  More take several launches.
#ifndef KVX_OPS_MAX_BLOCKS
#define KVX_OPS_MAX_BLOCKS (1 << 21)
#endif
constexpr int64_t kMaxBlocks = KVX_OPS_MAX_BLOCKS;

// One layer of a pool: row (c, page, slot, h) is at base + c * s_c + page *
// s_p + slot * s_t + h * s_h (bytes).
struct Layer {
    char *base;
    int64_t s_p, s_c, s_t, s_h;
    const int32_t *pt;
    int64_t pt_len;
    int32_t N, C, H, D;
    FastDiv fd_T;
};

// Rows of 16-bit values (kvx_rows) with a device base.
struct Rows {
    char *base;                  // nullptr: not given
    int64_t s_row, s_head;       // bytes
    int32_t heads;
};

struct AppendParams {
    Layer pool;
    const float *scales;         // e4m3 pools: [c][h], or nullptr
    Rows q, q_out, k, v;
    int64_t num_rows;
    const float *freq;
    int32_t half, rot_off, interleaved;   // half: rotated pairs of a head, 0: none
    float amplitude;
    const kvx_append_req *reqs;
    int32_t n_reqs, max_tokens;
    uint32_t *err;
    int32_t f16, e4m3;           // rows' and pool's types
    // launch
    int32_t tokens, blocks;      // tokens per workgroup, workgroups per record
    int32_t vec;                 // 8 elements at a time, else a pair
    int32_t partly;              // interleaved pairs end inside an eight
    int32_t items, items_v;      // of a q or k head, of a v head
    FastDiv fd_items, fd_items_v, fd_token, fd_half;
};

// kvx_norm with a device weight; dim 0: none.
struct HeadNorm {
    const float *weight;
    int32_t dim, off;
    float eps;
};

struct NormedParams : AppendParams {
    HeadNorm q_norm, k_norm;
    const int32_t *positions;    // [axis][pos_stride]: of rows; nullptr: the records'
    int64_t pos_stride;
    const int32_t *axis;         // of each pair, or nullptr
    int32_t num_axes;
    // launch (with AppendParams' but items_v, fd_items, fd_items_v): lanes of a
    // row, items of a lane; fd_token: heads
    int32_t lanes, per_lane;
};

struct AttendParams {
    Layer pool;
    const float *scales;
    Rows q, out;
    int32_t G, Dv;               // query heads per cache head; elements of a value
    float scale_log2;            // softmax scale times log2(e)
    float *lse;
    const kvx_attend_req *reqs;
    int32_t n_reqs, max_tokens;
    float *acc;
    int64_t acc_len, acc_stride;
    uint32_t *err;
    int32_t f16, e4m3;
    int32_t token_major;
    // launch: a workgroup's waves along cache heads and along blocks of 16 of their
    // query heads (the others along positions); head blocks (of `span` query heads)
    // per cache head, per record (per); positions of a step; whether every
    // unit has its own workgroup (whole), else the shares of the steps; query
    // heads of a part and cache head
    int32_t waves_k, waves_h, span, head_blocks, per, step, whole, shares, part_heads;
    // workspace
    int32_t *before;             // [record of the launch + 1]: steps before it
    float *lse2;                 // [record][q head]: m + log2 l, log2 units
    float *part_ml;              // [place][cache head][part head][2]
    float *part_o;               // [place][cache head][part head][Dv]
    float *scores;               // [record][q head][score_stride], log2 units
    float *spare;                // 64 floats
    int64_t score_stride;
};

// Records of one launch of kvx_attend.
#ifndef KVX_ATTEND_GROUP
#define KVX_ATTEND_GROUP 1024
#endif
constexpr int kAttendGroup = KVX_ATTEND_GROUP;

// The division of a call's work, from the sizes alone.
void plan_attend(AttendParams &p);
// The workspace of a planned call: its parts at `base`, or without one the bytes
// that serve it and every call of fewer records or positions.
int64_t attend_workspace(AttendParams &p, char *base);

struct SelectParams {
    const float *acc;
    int64_t acc_len, acc_stride;
    int32_t rows;
    const kvx_select_req *reqs;
    int32_t n_reqs, max_tokens;
    int32_t *kept;
    int64_t kept_len, kept_stride;
    float *out;
    int64_t out_len, out_stride;
    uint32_t *err;
};

struct KeptParams {
    Side src, dst;
    const kvx_req *reqs;
    int32_t n_reqs, max_tokens;
    int32_t L, C, H, vpr;
    const int32_t *kept;
    int64_t kept_len, kept_stride;
    uint32_t *err;
    int32_t rows;                // list entries of a workgroup
    int32_t blocks;              // workgroups per record, layer and head
    FastDiv fd_Ts, fd_Td, fd_vpr;
};

struct PathParams {
    Side pool;
    const kvx_path_req *reqs;
    int32_t n_reqs, max_tokens;
    const int32_t *path;
    int64_t path_len;
    int64_t vectors;             // 16-byte vectors of a token in all layers
    uint32_t *err;
    int32_t C, blocks;           // workgroups per record
    FastDiv fd_T, fd_H, fd_vpr;
};

// Each launches on `stream` and returns a hipError_t value.
int launch_append(const AppendParams &p, hipStream_t stream);
int launch_append_normed(const NormedParams &p, hipStream_t stream);
int launch_path(const PathParams &p, hipStream_t stream);
int launch_attend(const AttendParams &p, hipStream_t stream);
int launch_select(const SelectParams &p, hipStream_t stream);
int launch_kept(const KeptParams &p, hipStream_t stream);

}  // namespace kvx
