// kvx_path.hip -- accepted drafts' rows moved to the front, in place (gfx950).
//
// A path ascends, so that entry i lies at i or behind, and every row is read before
// a later entry's is written in its place.  A thread moves one vector of 16 bytes
// of a layer, kv and head for all entries, in order, and so needs no other thread: eight are
// on their way at once, and written when all eight have been read.  A few rows in every
// layer are far less than the memory moves in the time of the launch and the reads
// in turn of record, path and table: 6 rows of one sequence in 36 layers of 8 heads of 128
// (1.8 MB) take 4.5 us on the device, 12 of 64 sequences in 8 bits (34 MB) 10, 3.4 TB/s.

#include "kvx_ops.h"
#include "kvx_values.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;

__global__ void __launch_bounds__(kThreads) kvx_path_kernel(PathParams p, int32_t r0) {
    __shared__ int64_t from[KVX_MAX_DRAFTS], to[KVX_MAX_DRAFTS];       // row offsets; to -1: left out
    const int32_t r = r0 + (int32_t)(blockIdx.x / (uint32_t)p.blocks);
    const uint32_t block = blockIdx.x % (uint32_t)p.blocks;
    const kvx_path_req q = p.reqs[r];
    const int i = threadIdx.x, n = q.n_tokens;
    bool bad = q.pt_off < 0 || q.path_off < 0 || q.start < 0 || n < 0 || n > p.max_tokens || q.path_off > p.path_len - n;
    int32_t k = 0;
    if (!bad && i < n) {
        k = p.path[q.path_off + i];
        bad = k < i || (int64_t)q.start + k > INT32_MAX || (i > 0 && p.path[q.path_off + i - 1] >= k);
    }
    if (__syncthreads_or(bad)) {
        if (i == 0 && block == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    if (i < n) {
        uint32_t raised = 0;
        const auto offset = [&](uint32_t at, uint32_t bit) {
            const uint32_t page_no = fd_div(p.fd_T, at);
            const uint64_t idx = (uint64_t)q.pt_off + page_no;
            const int32_t page = idx < (uint64_t)p.pool.pt_len ? p.pool.pt[idx] : -1;
            if (idx >= (uint64_t)p.pool.pt_len) raised |= KVX_DERR_PT_RANGE;
            else if (page < 0 || page >= p.pool.N) raised |= bit;
            return page * p.pool.s_p + (int64_t)(at - page_no * p.fd_T.d) * p.pool.s_t;
        };
        const int64_t z = offset((uint32_t)q.start + i, KVX_DERR_DST_PAGE), a = offset((uint32_t)q.start + k, KVX_DERR_SRC_PAGE);
        from[i] = a;
        to[i] = raised || k == i ? -1 : z;
        if (raised && block == 0 && p.err) atomicOr(p.err, raised);
    }
    __syncthreads();
    // vectors of a token: [layer][kv][head][vector of the row]
    for (uint64_t x = (uint64_t)block * kThreads + i; x < (uint64_t)p.vectors; x += (uint64_t)p.blocks * kThreads) {
        const uint32_t row = fd_div(p.fd_vpr, (uint32_t)x), v = (uint32_t)x - row * p.fd_vpr.d;
        const uint32_t lc = fd_div(p.fd_H, row), h = row - lc * p.fd_H.d, l = lc / (uint32_t)p.C, c = lc - l * p.C;
        char *base = p.pool.base + l * p.pool.s_l + c * p.pool.s_c + h * p.pool.s_h + 16 * (int64_t)v;
        for (int i0 = 0; i0 < n; i0 += 8) {
            u32x4 w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i0 + e < n && to[i0 + e] >= 0) w[e] = *reinterpret_cast<const u32x4 *>(base + from[i0 + e]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i0 + e < n && to[i0 + e] >= 0) *reinterpret_cast<u32x4 *>(base + to[i0 + e]) = w[e];
        }
    }
}

}  // namespace

int launch_path(const PathParams &p0, hipStream_t stream) {
    if (p0.n_reqs == 0) return hipSuccess;
    PathParams p = p0;
    const int64_t blocks = (p.vectors + kThreads - 1) / kThreads;      // at most 2^19: a token has up to 2 GiB
    p.blocks = (int32_t)(blocks < kMaxBlocks ? blocks : kMaxBlocks);
    const int64_t group = kMaxBlocks / p.blocks;
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
        const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
        hipLaunchKernelGGL(kvx_path_kernel, dim3((uint32_t)(n * p.blocks)), dim3(kThreads), 0, stream, p, (int32_t)r0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kvx
