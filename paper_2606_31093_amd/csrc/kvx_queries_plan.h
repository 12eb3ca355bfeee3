// kvx_queries_plan.h -- attention of several queries of a request: launch parameters
// and the division of the work.  Not part of the public interface (include/kvx.h).
#pragma once

#include "kvx_ops.h"

namespace kvx {

// Records of one launch with shares.
#ifndef KVX_QUERIES_GROUP
#define KVX_QUERIES_GROUP 256
#endif
constexpr int kQueriesGroup = KVX_QUERIES_GROUP;

// So many units of one record, or of short ones, and more have a workgroup each (kvx_queries.hip).
constexpr int kWholeUnits = 1024;

// A unit that may lie in several shares: of all steps of a launch its first tile's and its
// last; record -1: none.
struct Cut {
    int64_t first, last;
    int32_t record, group, block, reserved;
};

struct QueriesParams {
    Layer pool;
    const float *scales;
    Rows q, out;
    int64_t num_rows;            // of q and out, the fewer
    int32_t Dv;
    float scale, cap;            // cap 0: none
    const float *slopes;
    int32_t window;              // 0: none
    float *lse;
    const kvx_queries_req *reqs;
    const uint64_t *tree;        // nullptr: prompts
    int32_t n_reqs, max_queries, max_tokens;
    uint32_t *err;
    int32_t f16, e4m3, token_major;
    FastDiv fd_G;
    // launch: wavefronts of a workgroup, and how many share a tile; cache heads of a
    // workgroup, and the groups of them; rows of a block, blocks of a record and cache
    // head at most; positions of a step; whether every unit has its own workgroup
    // (whole), else the shares of the steps; one: workgroups of one record whose queries say
    // which of the two, 0: not so
    int32_t waves, team, heads, groups, rows, blocks, step, whole, shares, by_share, one;
    // workspace
    Cut *cuts;                   // [record of the launch][group][block], or where there are more of them
                                 // than shares, [share]: the one that it begins inside
    int64_t *each;               // steps of a share; 0: every unit had its own workgroup
    float *part_ml;              // [place][head of the group][row][2]
    float *part_o;               // [place][head of the group][row / 32][value / 32][4][32][2][4]
};

// The division of a call's work, from the sizes alone; the workspace of a planned
// call: its parts at `base`, or without one the bytes that serve it.
void plan_queries(QueriesParams &p);
int64_t queries_workspace(QueriesParams &p, char *base);
// Bytes that serve every call of up to so many records, queries and positions.
int64_t queries_workspace_most(const QueriesParams &p);
int launch_queries(const QueriesParams &p, hipStream_t stream);

}  // namespace kvx
