// kvx_append_normed.hip -- new tokens into a paged cache, their queries and keys
// normed per head and rotated by positions of one axis or several (gfx950).
//
// As kvx_append.hip: every row is read and written once, and that is what takes
// the time.  A norm needs the whole head before the first element can be stored,
// so a head's row is held in the registers of a few neighbouring lanes (a power of
// two), 16 bytes an item, with halves the two eights that rotate together; their
// sums of squares meet by shuffles.  The sum is in 32 bits; norm, rotation and
// rounding to the stored type are one pass, so that there is one rounding.
// Cosines and sines of a token are made once into LDS for all its heads, the
// norms' weights lie there too.
//
// Four prompts of 1024 to 8192 tokens into an e4m3 cache (28 query heads of 128 on 4, all
// normed, positions on three axes, 260 MB) take 67 to 70 us, 3.9 TB/s, as much as kvx_append takes
// without norms, and 68 into a bfloat16 one (276 MB): about 42 us of them the vector instructions alone
// would take (915 a wavefront; a wavefront with a row of an e4m3 cache divides by its scale for all its
// rows), and 63% of a wavefront's time passes in waits.  The cosines' reads from LDS, 64 bytes apart from lane
// to lane, conflict in 59% of its cycles, which are few.  With the next row's loads asked for ahead fewer
// wavefronts fit and it is slower.  MLA's rows (16 heads of 576, 586 MB) take 224 us, 2.6 TB/s.  512
// drafted tokens take 12 to 13 us, 12.6 MB: 192 workgroups, each of which reads record, page ids and
// then five rows a group of lanes in turn.

#include "kvx_append.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 4096;       // rotated pairs x tokens a workgroup keeps in LDS (32 KiB)

// A norm's factor for a head whose normed elements' squares sum to ss.
__device__ __forceinline__ float inverse(float ss, const HeadNorm &n) {
    return 1.0f / sqrtf(ss / (float)n.dim + n.eps);
}

// Where the squares overflow, or are so small that some which vanish in 32 bits may count, the
// elements are scaled first.  Overflow: the largest lies in [2^59, 2^128), and scaled in [2^-21,
// 2^48).  A factor of 2^40 and more: eps is below 2^-80, the largest element in [2^-133,
// 2^-35], and scaled in [2^-40, 2^58]; what vanishes then is below 2^-40 of the sum.  1: neither, as
// nearly always: that it is looked for takes the e4m3 prompts above from 69.4 to 69.9 us, their interleaved pairs,
// with the weights' place in one register less, from 94 to 89.
__device__ __forceinline__ float scale_of(float f) { return f >= 0x1p40f ? 0x1p93f : f > 0.f ? 1.f : 0x1p-80f; }

__device__ __forceinline__ HeadNorm scaled(HeadNorm n, float by) {
    n.eps = n.eps * by * by;
    return n;
}

// VEC: eights of elements; K items a lane.  Else one element or pair at a time, a
// wavefront a row, which reads it twice.
template <bool F16, bool VEC, bool HALVES, int K>
__global__ void __launch_bounds__(kThreads) kvx_append_normed_kernel(NormedParams p, int32_t r0) {
    extern __shared__ float2 turn[];             // [token][pair]: cosine, sine; then the weights of q and k
    __shared__ int64_t slot_off[64];             // pool offset of a token, -1: none
    const int32_t r = r0 + (int32_t)(blockIdx.x / (uint32_t)p.blocks);
    const int32_t first = (int32_t)(blockIdx.x % (uint32_t)p.blocks) * p.tokens;
    const kvx_append_req q = p.reqs[r];
    const int64_t n = q.n_tokens;
    // with positions of their own the record's is not used
    if (n < 0 || q.reserved != 0 || q.pt_off < 0 || q.row_off < 0 || q.start < 0 || q.position < 0 || n > p.max_tokens ||
        q.start + n > INT32_MAX || (!p.positions && q.position + n > INT32_MAX) || q.row_off > p.num_rows - n) {
        if (threadIdx.x == 0 && first == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    if (first >= n) return;
    const int tokens = (int)(n - first < p.tokens ? n - first : p.tokens);

    bool bad_axis = false;
    for (int i = threadIdx.x; i < tokens * p.half; i += kThreads) {
        const uint32_t t = fd_div(p.fd_half, i), j = i - t * p.half;
        int32_t at;
        if (p.positions) {
            const int32_t axis = p.axis ? p.axis[j] : 0;
            const bool bad = axis < 0 || axis >= p.num_axes;
            bad_axis |= bad;
            at = p.positions[(bad ? 0 : axis) * p.pos_stride + q.row_off + first + t];
        } else {
            at = q.position + first + (int32_t)t;
        }
        const double turns = (double)at * (double)p.freq[j] * 0.15915494309189535;
        float s, c;
        sincospif(2.0f * (float)(turns - __builtin_rint(turns)), &s, &c);
        turn[i] = make_float2(c * p.amplitude, s * p.amplitude);
    }
    float *weights[2];
    weights[0] = reinterpret_cast<float *>(turn + p.tokens * p.half);
    weights[1] = weights[0] + p.q_norm.dim;
    for (int i = threadIdx.x; i < p.q_norm.dim; i += kThreads) weights[0][i] = p.q_norm.weight ? p.q_norm.weight[i] : 1.f;
    for (int i = threadIdx.x; i < p.k_norm.dim; i += kThreads) weights[1][i] = p.k_norm.weight ? p.k_norm.weight[i] : 1.f;
    if ((int)threadIdx.x < tokens) {
        const uint32_t at = (uint32_t)(q.start + first + threadIdx.x), page_no = fd_div(p.pool.fd_T, at);
        const uint64_t idx = (uint64_t)q.pt_off + page_no;
        int64_t off = -1;
        if (idx >= (uint64_t)p.pool.pt_len) {
            if (p.err) atomicOr(p.err, KVX_DERR_PT_RANGE);
        } else {
            const int32_t page = p.pool.pt[idx];
            if (page < 0 || page >= p.pool.N) {
                if (p.err) atomicOr(p.err, KVX_DERR_DST_PAGE);
            } else {
                off = page * p.pool.s_p + (int64_t)(at - page_no * p.pool.fd_T.d) * p.pool.s_t;
            }
        }
        slot_off[threadIdx.x] = off;
    }
    if (__syncthreads_or(bad_axis)) {            // every workgroup of the call sees it
        if (threadIdx.x == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }

    const int heads = p.q.heads + p.k.heads + p.v.heads, half = p.half, o = p.rot_off;
    const int lanes = VEC ? p.lanes : 64, groups = kThreads / lanes;
    const int lane = threadIdx.x & (lanes - 1);
    for (int row_no = threadIdx.x / lanes; row_no < tokens * heads; row_no += groups) {
        const uint32_t t = fd_div(p.fd_token, row_no);
        int head = row_no - t * heads;
        const bool is_q = head < p.q.heads, is_v = head >= p.q.heads + p.k.heads;
        if (!is_q) head -= p.q.heads + (is_v ? p.k.heads : 0);
        const Rows &in = is_v ? p.v : is_q ? p.q : p.k;
        const int64_t row = q.row_off + first + t;
        const char *src = in.base + row * in.s_row + head * in.s_head;
        Dest to;
        to.e4m3 = false;
        to.scale = 1.f;
        if (is_q) {
            to.row = p.q_out.base + row * p.q_out.s_row + head * p.q_out.s_head;
        } else {
            const int64_t off = slot_off[t];
            to.row = off < 0 ? nullptr : p.pool.base + off + (is_v ? p.pool.s_c : 0) + head * p.pool.s_h;
            to.e4m3 = p.e4m3;
            if (p.scales) to.scale = p.scales[(is_v ? p.pool.H : 0) + head];
        }
        const float2 *cs = turn + t * half;
        HeadNorm norm = is_q ? p.q_norm : p.k_norm;
        if (is_v) norm.dim = 0;
        const float *weight = weights[0] + ((is_q ? 0 : p.q_norm.dim) - norm.off);
        const auto normed = [&](int d) { return d >= norm.off && d < norm.off + norm.dim; };

        if (VEC) {
            // an item is an eight, or with halves the two eights that rotate together
            const int hv = half / 8, ov = o / 8;
            u32x4 w[K][HALVES ? 2 : 1];
            float x[K][HALVES ? 2 : 1][8];
            const auto eights = [&](int item) { return HALVES && item >= ov && item < ov + hv ? 2 : 1; };
            const auto dim = [&](int item, int e) { return 8 * (HALVES && (item >= ov + hv || e) ? item + hv : item); };
            float ss = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int item = lane + k * lanes;
#pragma unroll
                for (int e = 0; e < (HALVES ? 2 : 1); ++e)
                    if (item < p.items && e < eights(item)) w[k][e] = *reinterpret_cast<const u32x4 *>(src + 2 * dim(item, e));
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int item = lane + k * lanes;
#pragma unroll
                for (int e = 0; e < (HALVES ? 2 : 1); ++e) {
                    if (item >= p.items || e >= eights(item)) continue;
                    unpack8<F16>(w[k][e], x[k][e]);
                    if (!normed(dim(item, e))) continue;
#pragma unroll
                    for (int i = 0; i < 8; ++i) ss += x[k][e][i] * x[k][e][i];
                }
            }
            float f = 1.f;
            if (norm.dim) {                      // the same for all lanes of the row
                for (int d = 1; d < lanes; d <<= 1) ss += __shfl_xor(ss, d);
                f = inverse(ss, norm);
                const float by = scale_of(f);
                if (__builtin_expect_with_probability(by != 1.f, 0, 0.9999)) {
                    ss = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const int item = lane + k * lanes;
#pragma unroll
                        for (int e = 0; e < (HALVES ? 2 : 1); ++e) {
                            if (item >= p.items || e >= eights(item) || !normed(dim(item, e))) continue;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                x[k][e][i] *= by;
                                ss += x[k][e][i] * x[k][e][i];
                            }
                        }
                    }
                    for (int d = 1; d < lanes; d <<= 1) ss += __shfl_xor(ss, d);
                    f = inverse(ss, scaled(norm, by));
                }
            }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int item = lane + k * lanes;
                if (item >= p.items) continue;
                const int n_e = eights(item);
                bool changed[2];
#pragma unroll
                for (int e = 0; e < (HALVES ? 2 : 1); ++e) {
                    const int d = dim(item, e);
                    changed[e] = e < n_e && normed(d);
                    if (!changed[e]) continue;
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[k][e][i] *= f * weight[d + i];
                }
                if (HALVES) {
                    if (n_e == 2 && !is_v) {
                        const int j = (item - ov) * 8;
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float2 z = cs[j + i];
                            const float a = x[k][0][i], b = x[k][1][i];
                            x[k][0][i] = a * z.x - b * z.y;
                            x[k][1][i] = b * z.x + a * z.y;
                        }
                        changed[0] = changed[1] = true;
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (e < n_e) store8<F16>(to, dim(item, e), w[k][e], x[k][e], changed[e]);
                } else {
                    const int d = 8 * item;
                    if (half && !is_v && d + 8 > o && d < o + 2 * half) {
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            if (d + i < o || d + i >= o + 2 * half) continue;
                            const float2 z = cs[(d + i - o) / 2];
                            const float a = x[k][0][i], b = x[k][0][i + 1];
                            x[k][0][i] = a * z.x - b * z.y;
                            x[k][0][i + 1] = b * z.x + a * z.y;
                            // the eight's other elements keep their bits, also those of a NaN
                            if (!changed[0]) w[k][0][i / 2] = Half<F16>::pack(x[k][0][i], x[k][0][i + 1]);
                        }
                    }
                    store8<F16>(to, d, w[k][0], x[k][0], changed[0]);
                }
            }
        } else {
            // a rotated pair, or one element that stays
            const uint16_t *x = reinterpret_cast<const uint16_t *>(src);
            float f = 1.f, by = 1.f;
            if (norm.dim) {
                const auto squares = [&]() {
                    float ss = 0.f;
                    for (int d = norm.off + lane; d < norm.off + norm.dim; d += 64) {
                        const float y = Half<F16>::lo(x[d]) * by;
                        ss += y * y;
                    }
                    for (int d = 1; d < 64; d <<= 1) ss += __shfl_xor(ss, d);
                    return ss;
                };
                f = inverse(squares(), norm);
                by = scale_of(f);
                if (by != 1.f) f = inverse(squares(), scaled(norm, by));
            }
            const auto value = [&](int d) { return normed(d) ? Half<F16>::lo(x[d]) * by * (f * weight[d]) : Half<F16>::lo(x[d]); };
            // q_out may be q: nothing of the row is read after this, but by the lane that writes it
            for (int item = lane; item < (is_v ? p.pool.D : p.items); item += 64) {
                if (!is_v && item < half) {
                    const int da = p.interleaved ? o + 2 * item : o + item, db = p.interleaved ? da + 1 : da + half;
                    const float a = value(da), b = value(db);
                    const float2 z = cs[item];
                    store1<F16>(to, da, 0, a * z.x - b * z.y, true);
                    store1<F16>(to, db, 0, b * z.x + a * z.y, true);
                } else {
                    int d = is_v ? item : item - half;
                    if (!is_v && d >= o) d += 2 * half;
                    store1<F16>(to, d, x[d], value(d), normed(d));
                }
            }
        }
    }
}

template <bool F16>
auto pick(const NormedParams &p) {
    if (!p.vec) return kvx_append_normed_kernel<F16, false, false, 1>;
    if (p.half && !p.interleaved)
        return p.per_lane == 1 ? kvx_append_normed_kernel<F16, true, true, 1> : kvx_append_normed_kernel<F16, true, true, 2>;
    return p.per_lane == 1   ? kvx_append_normed_kernel<F16, true, false, 1>
           : p.per_lane == 2 ? kvx_append_normed_kernel<F16, true, false, 2>
                             : kvx_append_normed_kernel<F16, true, false, 3>;
}

}  // namespace

int launch_append_normed(const NormedParams &p0, hipStream_t stream) {
    if (p0.n_reqs == 0) return hipSuccess;
    NormedParams p = p0;
    const int D = p.pool.D, heads = p.q.heads + p.k.heads + p.v.heads;
    const bool halves = p.half && !p.interleaved;
    // eights where pairs never straddle one, as in kvx_append, and with the gain that it measured
    p.vec = p.half == 0 || (p.interleaved ? p.rot_off % 2 == 0 : p.rot_off % 8 == 0 && p.half % 8 == 0);
    p.items = p.vec ? D / 8 - (halves ? p.half / 8 : 0) : D - p.half;
    // the lanes of a row, of which the fewest idle; then the fewest items a lane
    p.lanes = 64;
    p.per_lane = (p.items + 63) / 64;
    for (int lanes = 32; p.vec && lanes >= 1; lanes >>= 1) {
        const int per = (p.items + lanes - 1) / lanes;
        if (per <= (halves ? 2 : 3) && per * lanes < p.per_lane * p.lanes) p.lanes = lanes, p.per_lane = per;
    }
    const int64_t per_token = (int64_t)heads * p.lanes * (p.vec ? 1 : 4);      // heads: up to 2^23
    int64_t tokens = (4 * kThreads + per_token - 1) / per_token;
    if (p.half && tokens > kMaxHalf / p.half) tokens = kMaxHalf / p.half;
    if (tokens > 64) tokens = 64;
    if (tokens > p.max_tokens) tokens = p.max_tokens > 0 ? p.max_tokens : 1;
    p.tokens = (int32_t)tokens;
    // with max_tokens 0 one: it looks whether the record is malformed
    p.blocks = p.max_tokens > 0 ? (int32_t)((p.max_tokens + tokens - 1) / tokens) : 1;
    p.fd_token = make_fastdiv(heads);
    p.fd_half = make_fastdiv(p.half ? p.half : 1);
    const size_t lds = sizeof(float2) * p.tokens * p.half + sizeof(float) * (p.q_norm.dim + p.k_norm.dim);
    const int64_t group = kMaxBlocks / p.blocks > 0 ? kMaxBlocks / p.blocks : 1;
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
        const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
        hipLaunchKernelGGL(p.f16 ? pick<true>(p) : pick<false>(p), dim3((uint32_t)(n * p.blocks)), dim3(kThreads), lds, stream,
                           p, (int32_t)r0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kvx
