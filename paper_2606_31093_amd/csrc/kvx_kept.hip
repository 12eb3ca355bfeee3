// kvx_kept.hip -- what a paged cache keeps of its requests (gfx950): the choice
// of positions by accumulated weight, and the move of the kept rows.

#include "kvx_ops.h"
#include "kvx_values.h"

namespace kvx {
namespace {

// ---------------------------------------------------------------------------
// choice
// ---------------------------------------------------------------------------

constexpr int kThreads = 256;

// Unsigned order of the weights: NaN lowest, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    if (x != x) return 0;
    const uint32_t u = bits<uint32_t>(x == 0.f ? 0.f : x);
    return u >> 31 ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ bool inside(int64_t off, int64_t stride, int rows, int64_t n, int64_t len) {
    return off >= 0 && off <= len && n <= len - off && (rows == 1 || stride <= (len - off - n) / (rows - 1));
}

// A workgroup per record and row.  The n_keep - sink - recent largest keys of
// the middle are found digit by digit from the top, 8 bits at a time: count
// the digits of the keys that share the digits found so far, and take the
// digit in which the last kept key lies.  Then all positions are walked in
// order and the kept ones listed.
__global__ void __launch_bounds__(kThreads) kvx_select_kernel(SelectParams p, int32_t r0) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t found[2];
    __shared__ uint32_t counts[2][kThreads / 64];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int r = r0 + (int)(blockIdx.x / (uint32_t)p.rows), j = (int)(blockIdx.x % (uint32_t)p.rows);
    const kvx_select_req q = p.reqs[r];
    const int64_t kept_n = q.n_tokens < q.n_keep ? q.n_tokens : q.n_keep;
    if (q.n_tokens < 0 || q.n_keep < 0 || q.sink < 0 || q.recent < 0 || q.n_tokens > p.max_tokens ||
        (int64_t)q.sink + q.recent > q.n_keep || !inside(q.acc_off, p.acc_stride, p.rows, q.n_tokens, p.acc_len) ||
        !inside(q.kept_off, p.kept_stride, p.rows, kept_n, p.kept_len) ||
        (p.out && !inside(q.out_off, p.out_stride, p.rows, kept_n, p.out_len))) {
        if (j == 0 && tid == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    const float *acc = p.acc + q.acc_off + j * p.acc_stride;
    int32_t *kept = p.kept + q.kept_off + j * p.kept_stride;
    float *out = p.out ? p.out + q.out_off + j * p.out_stride : nullptr;
    const int n = q.n_tokens;
    if (n <= q.n_keep) {
        for (int t = tid; t < n; t += kThreads) {
            kept[t] = t;
            if (out) out[t] = acc[t];
        }
        return;
    }
    const int lo = q.sink, hi = n - q.recent;
    uint32_t need = q.n_keep - q.sink - q.recent;       // < hi - lo
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0 && need > 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int t = lo + tid; t < hi; t += kThreads) {
            const uint32_t k = key_of(acc[t]);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        if (tid < 64) {
            // lane x: digits 255 - 4x .. 252 - 4x, from the largest down
            uint32_t part[4], sum = 0;
            for (int i = 0; i < 4; ++i) {
                part[i] = hist[255 - 4 * lane - i];
                sum += part[i];
            }
            uint32_t above = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t x = __shfl_up(above, d);
                if (lane >= d) above += x;
            }
            above -= sum;
            for (int i = 0; i < 4; ++i) {
                if (above < need && above + part[i] >= need) {
                    found[0] = 255 - 4 * lane - i;
                    found[1] = need - above;
                }
                above += part[i];
            }
        }
        __syncthreads();
        prefix |= found[0] << shift;
        need = found[1];
    }
    // `need` of the keys equal to prefix, the first ones, and all above
    const bool any = q.n_keep > q.sink + q.recent;
    uint32_t at = 0, ties = 0;
    for (int t0 = 0; t0 < n; t0 += kThreads) {
        const int t = t0 + tid;
        const bool mid = t >= lo && t < hi;
        const float x = t < n ? acc[t] : 0.f;
        const uint32_t k = key_of(x);
        const bool tie = any && mid && k == prefix;
        const uint64_t bt = __ballot(tie);
        if (lane == 0) counts[0][wave] = __popcll(bt);
        __syncthreads();
        uint32_t rank = ties + __popcll(bt & ((1ull << lane) - 1));
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) rank += counts[0][w];
            ties += counts[0][w];
        }
        const bool take = t < n && (!mid || (any && (k > prefix || (tie && rank < need))));
        const uint64_t bk = __ballot(take);
        if (lane == 0) counts[1][wave] = __popcll(bk);
        __syncthreads();
        uint32_t to = at + __popcll(bk & ((1ull << lane) - 1));
        for (int w = 0; w < kThreads / 64; ++w) {
            if (w < wave) to += counts[1][w];
            at += counts[1][w];
        }
        if (take) {
            kept[to] = t;
            if (out) out[to] = x;
        }
    }
}

// ---------------------------------------------------------------------------
// move
// ---------------------------------------------------------------------------

constexpr int kRows = 64;            // list entries of a workgroup

// A workgroup per 64 entries of one list (a record's layer and head): their
// source and destination rows are resolved once, then copied 16 bytes a lane,
// keys and values.
__global__ void __launch_bounds__(kThreads) kvx_kept_kernel(KeptParams p, int32_t r0, int32_t piece0) {
    __shared__ int64_t from[kRows], to[kRows];           // to < 0: left out
    uint32_t b = blockIdx.x;
    const int piece = piece0 + (int)(b % (uint32_t)p.blocks);
    b /= (uint32_t)p.blocks;
    const int h = (int)(b % (uint32_t)p.H);
    b /= (uint32_t)p.H;
    const int l = (int)(b % (uint32_t)p.L), r = r0 + (int)(b / (uint32_t)p.L);
    const kvx_req q = p.reqs[r];
    const int64_t n = q.n_tokens;
    if (n < 0 || q.src_start < 0 || q.dst_start < 0 || q.reserved != 0 || n > p.max_tokens ||
        q.src_start + n > INT32_MAX || q.dst_start + n > INT32_MAX ||
        !inside(q.buf_off, p.kept_stride, p.L * p.H, n, p.kept_len)) {
        if (piece == 0 && h == 0 && l == 0 && threadIdx.x == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    const int first = piece * kRows;
    if (first >= n) return;
    const int rows = (int)(n - first < kRows ? n - first : kRows);
    if ((int)threadIdx.x < rows) {
        const int i = first + threadIdx.x;
        const int64_t k = p.kept[q.buf_off + ((int64_t)l * p.H + h) * p.kept_stride + i];
        int64_t a = -1, z = -1;
        uint32_t bad = 0;
        const uint32_t dt = (uint32_t)(q.dst_start + i), dp = fd_div(p.fd_Td, dt);
        const uint64_t di = (uint64_t)q.dst_pt_off + dp;
        if (di >= (uint64_t)p.dst.pt_len) {
            bad = KVX_DERR_PT_RANGE;
        } else {
            const int32_t page = p.dst.pt[di];
            if (page < 0 || page >= p.dst.N) bad = KVX_DERR_DST_PAGE;
            else z = page * p.dst.s_p + (int64_t)(dt - dp * p.fd_Td.d) * p.dst.s_t;
        }
        if (!bad) {
            const int64_t st = q.src_start + k;
            if (k < 0 || st > INT32_MAX) {
                bad = KVX_DERR_PT_RANGE;
            } else {
                const uint32_t sp = fd_div(p.fd_Ts, (uint32_t)st);
                const uint64_t si = (uint64_t)q.src_pt_off + sp;
                if (si >= (uint64_t)p.src.pt_len) {
                    bad = KVX_DERR_PT_RANGE;
                } else {
                    const int32_t page = p.src.pt[si];
                    if (page < 0 || page >= p.src.N) bad = KVX_DERR_SRC_PAGE;
                    else a = page * p.src.s_p + (int64_t)((uint32_t)st - sp * p.fd_Ts.d) * p.src.s_t;
                }
            }
        }
        if (bad && p.err) atomicOr(p.err, bad);
        from[threadIdx.x] = bad ? 0 : a;
        to[threadIdx.x] = bad ? -1 : z;
    }
    __syncthreads();
    const char *src = p.src.base + l * p.src.s_l + h * p.src.s_h;
    char *dst = p.dst.base + l * p.dst.s_l + h * p.dst.s_h;
    const int per = rows * p.vpr;
    for (int c = 0; c < p.C; ++c) {
        for (int x = threadIdx.x; x < per; x += kThreads) {
            const int i = (int)fd_div(p.fd_vpr, x), v = x - i * p.vpr;
            if (to[i] < 0) continue;
            *reinterpret_cast<u32x4 *>(dst + to[i] + 16 * v) =
                *reinterpret_cast<const u32x4 *>(src + from[i] + 16 * v);
        }
        src += p.src.s_c;
        dst += p.dst.s_c;
    }
}

}  // namespace

int launch_select(const SelectParams &p, hipStream_t stream) {
    const int64_t group = kMaxBlocks / p.rows > 0 ? kMaxBlocks / p.rows : 1;
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
        const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
        hipLaunchKernelGGL(kvx_select_kernel, dim3((uint32_t)(n * p.rows)), dim3(kThreads), 0, stream, p, (int32_t)r0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int launch_kept(const KeptParams &p0, hipStream_t stream) {
    if (p0.n_reqs == 0 || p0.max_tokens == 0) return hipSuccess;
    KeptParams p = p0;
    const int32_t pieces = (p.max_tokens + kRows - 1) / kRows;
    const int64_t lists = (int64_t)p.L * p.H;             // at most 2^20
    p.blocks = (int32_t)(kMaxBlocks / lists < pieces ? kMaxBlocks / lists : pieces);
    const int64_t per = p.blocks * lists, group = kMaxBlocks / per;
    for (int32_t piece0 = 0; piece0 < pieces; piece0 += p.blocks) {
        for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
            const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
            hipLaunchKernelGGL(kvx_kept_kernel, dim3((uint32_t)(n * per)), dim3(kThreads), 0, stream, p, (int32_t)r0,
                               piece0);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace kvx
