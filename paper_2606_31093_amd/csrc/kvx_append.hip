// kvx_append.hip -- new tokens into a paged cache, rotated (gfx950).
//
// A token's q, k and v rows are read once, its q row and its pool rows are
// written once; the arithmetic (two products and a sum per element) is far
// below what the memory allows.  A workgroup takes some tokens of one record.
// The cosines and sines of a token are the same for all its heads, so the
// workgroup computes them once into LDS: the angle's whole turns are removed in
// 64 bits (position * freq reaches 2^31 turns of which only the fraction
// counts), cosine and sine are then taken in 32.
//
// Four prompts of 1024 to 8192 tokens into an e4m3 cache (28 query heads of 128 on
// 4, 245 MB) take 64 us, MLA's 824 MB (16 query heads, rows of 576) 175 us, 4.7
// TB/s; 64 new tokens 9.7 us, of which the data is under one.  Wavefronts hide
// the loads' latency: with the rows of two items a thread asked for ahead of the
// angles, or of four, fewer fit and the same cases took 84 and 261 us, or 95 and 292.

#include "kvx_ops.h"
#include "kvx_values.h"

namespace kvx {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 8192;       // rotated pairs x tokens a workgroup keeps in LDS (64 KiB)

// Where a row of the token goes.
struct Dest {
    char *row;         // nullptr: nowhere
    bool e4m3;
    float scale;
};

// Eight elements: w as they lie in the row, x their values, which have changed or not.
template <bool F16>
__device__ __forceinline__ void store8(const Dest &to, int d, u32x4 w, const float *x, bool changed) {
    if (!to.row) return;
    if (to.e4m3) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i] / to.scale;
        const u32x2 o = {pack_e4m3(y[0], y[1], y[2], y[3]), pack_e4m3(y[4], y[5], y[6], y[7])};
        *reinterpret_cast<u32x2 *>(to.row + d) = o;
        return;
    }
    if (changed) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = Half<F16>::pack(x[2 * i], x[2 * i + 1]);
    }
    *reinterpret_cast<u32x4 *>(to.row + 2 * d) = w;
}

template <bool F16>
__device__ __forceinline__ void store1(const Dest &to, int d, uint16_t w, float x, bool changed) {
    if (!to.row) return;
    if (to.e4m3) {
        const float y = changed ? x : Half<F16>::lo(w);
        to.row[d] = (char)pack_e4m3(y / to.scale, 0.f, 0.f, 0.f);
        return;
    }
    *reinterpret_cast<uint16_t *>(to.row + 2 * d) = changed ? (uint16_t)Half<F16>::pack(x, 0.f) : w;
}

template <bool F16>
__device__ __forceinline__ void unpack8(u32x4 w, float *x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = Half<F16>::lo(w[i]);
        x[2 * i + 1] = Half<F16>::hi(w[i]);
    }
}

template <bool F16, bool VEC>
__global__ void __launch_bounds__(kThreads) kvx_append_kernel(AppendParams p, int32_t r0) {
    extern __shared__ float2 turn[];             // [token][pair]: cosine, sine
    __shared__ int64_t slot_off[64];             // pool offset of a token, -1: none
    const int32_t r = r0 + (int32_t)(blockIdx.x / (uint32_t)p.blocks);
    const int32_t first = (int32_t)(blockIdx.x % (uint32_t)p.blocks) * p.tokens;
    const kvx_append_req q = p.reqs[r];
    const int64_t n = q.n_tokens;
    if (n < 0 || q.reserved != 0 || q.pt_off < 0 || q.row_off < 0 || q.start < 0 || q.position < 0 ||
        n > p.max_tokens || q.start + n > INT32_MAX || q.position + n > INT32_MAX || q.row_off > p.num_rows - n) {
        if (threadIdx.x == 0 && first == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    if (first >= n) return;
    const int tokens = (int)(n - first < p.tokens ? n - first : p.tokens);

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
    for (int i = threadIdx.x; i < tokens * p.half; i += kThreads) {
        const uint32_t t = fd_div(p.fd_half, i), j = i - t * p.half;
        const double turns = (double)(q.position + first + (int32_t)t) * (double)p.freq[j] * 0.15915494309189535;
        float s, c;
        sincospif(2.0f * (float)(turns - __builtin_rint(turns)), &s, &c);
        turn[i] = make_float2(c * p.amplitude, s * p.amplitude);
    }
    __syncthreads();

    const uint32_t heads_qk = p.q.heads + p.k.heads;
    const uint32_t qk_items = heads_qk * p.items;
    const int total = tokens * (int)p.fd_token.d;
    for (int i = threadIdx.x; i < total; i += kThreads) {
        const uint32_t t = fd_div(p.fd_token, i);
        uint32_t m = i - t * p.fd_token.d, head, item;
        const bool is_v = m >= qk_items;
        if (is_v) {
            m -= qk_items;
            head = fd_div(p.fd_items_v, m);
            item = m - head * p.items_v;
        } else {
            head = fd_div(p.fd_items, m);
            item = m - head * p.items;
        }
        const bool is_q = !is_v && head < (uint32_t)p.q.heads;
        if (!is_v && !is_q) head -= p.q.heads;
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
        const float2 *cs = turn + t * p.half;
        const int half = is_v ? 0 : p.half, o = p.rot_off;
        if (VEC) {
            // 8 elements, or with halves the two eights that rotate together
            const int hv = half / 8, ov = o / 8;
            if (half && !p.interleaved) {
                if ((int)item >= ov && (int)item < ov + hv) {
                    const int j = (item - ov) * 8;
                    const u32x4 wa = *reinterpret_cast<const u32x4 *>(src + 16 * item);
                    const u32x4 wb = *reinterpret_cast<const u32x4 *>(src + 16 * (item + hv));
                    float a[8], b[8];
                    unpack8<F16>(wa, a);
                    unpack8<F16>(wb, b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 z = cs[j + e];
                        const float x = a[e] * z.x - b[e] * z.y, y = b[e] * z.x + a[e] * z.y;
                        a[e] = x;
                        b[e] = y;
                    }
                    store8<F16>(to, 8 * item, wa, a, true);
                    store8<F16>(to, 8 * (item + hv), wb, b, true);
                    continue;
                }
                if ((int)item >= ov + hv) item += hv;      // behind the second half
            }
            u32x4 w = *reinterpret_cast<const u32x4 *>(src + 16 * item);
            float x[8];
            unpack8<F16>(w, x);
            const int d = 8 * item;
            // interleaved pairs of this eight that rotate: elements [o, o + 2 half)
            bool changed = half && p.interleaved && d + 8 > o && d < o + 2 * half;
            if (changed) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    if (d + e < o || d + e >= o + 2 * half) continue;
                    const float2 z = cs[(d + e - o) / 2];
                    const float a = x[e], b = x[e + 1];
                    x[e] = a * z.x - b * z.y;
                    x[e + 1] = b * z.x + a * z.y;
                }
                if (p.partly) {
                    // the eight's other elements keep their bits, also those of a NaN
#pragma unroll
                    for (int e = 0; e < 8; e += 2)
                        if (d + e >= o && d + e < o + 2 * half) w[e / 2] = Half<F16>::pack(x[e], x[e + 1]);
                    changed = false;
                }
            }
            store8<F16>(to, d, w, x, changed);
        } else {
            // a rotated pair, or one element that stays
            const uint16_t *x = reinterpret_cast<const uint16_t *>(src);
            if ((int)item < half) {
                const int da = p.interleaved ? o + 2 * item : o + item, db = p.interleaved ? da + 1 : da + half;
                const uint16_t wa = x[da], wb = x[db];
                const float a = Half<F16>::lo(wa), b = Half<F16>::lo(wb);
                const float2 z = cs[item];
                store1<F16>(to, da, wa, a * z.x - b * z.y, true);
                store1<F16>(to, db, wb, b * z.x + a * z.y, true);
            } else {
                int d = item - half;
                if (d >= o) d += 2 * half;
                store1<F16>(to, d, x[d], 0.f, false);
            }
        }
    }
}

}  // namespace

int launch_append(const AppendParams &p0, hipStream_t stream) {
    if (p0.n_reqs == 0) return hipSuccess;
    AppendParams p = p0;
    const int D = p.pool.D;
    // Eights where pairs never straddle one: halves that begin and end between
    // eights, interleaved pairs that begin at even elements.  4 prompts of 1024 to 8192
    // tokens, 32 query heads of 80 on 8 (216 MB), take 35 to 38 us in eights and 149 to 154
    // element by element, 40 to 46 and 158 to 165 into an e4m3 cache.
    p.vec = p.half == 0 || (p.interleaved ? p.rot_off % 2 == 0 : p.rot_off % 8 == 0 && p.half % 8 == 0);
    p.partly = p.interleaved && (p.rot_off % 8 || 2 * p.half % 8);
    p.items = p.vec ? D / 8 - (p.interleaved ? 0 : p.half / 8) : D - p.half;
    p.items_v = p.vec ? D / 8 : D;
    const int per_token = (p.q.heads + p.k.heads) * p.items + p.v.heads * p.items_v;
    // about four items a thread, within the LDS for the cosines and sines
    int64_t tokens = (4 * kThreads + per_token - 1) / per_token;
    if (p.half && tokens > kMaxHalf / p.half) tokens = kMaxHalf / p.half;
    if (tokens > 64) tokens = 64;
    if (tokens > p.max_tokens) tokens = p.max_tokens > 0 ? p.max_tokens : 1;
    p.tokens = (int32_t)tokens;
    // Each record has the workgroups of max_tokens: one of 8192 tokens among 256 of one takes 303
    // us, apart they take 33 and 4.  With max_tokens 0 one: it looks whether the record is malformed.
    p.blocks = p.max_tokens > 0 ? (int32_t)((p.max_tokens + tokens - 1) / tokens) : 1;
    p.fd_token = make_fastdiv(per_token);
    p.fd_items = make_fastdiv(p.items);
    p.fd_items_v = make_fastdiv(p.items_v);
    p.fd_half = make_fastdiv(p.half ? p.half : 1);
    const size_t lds = sizeof(float2) * p.tokens * p.half;
    const int64_t group = kMaxBlocks / p.blocks > 0 ? kMaxBlocks / p.blocks : 1;
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
        const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
        const dim3 grid((uint32_t)(n * p.blocks));
        const auto k = p.f16 ? (p.vec ? kvx_append_kernel<true, true> : kvx_append_kernel<true, false>)
                             : (p.vec ? kvx_append_kernel<false, true> : kvx_append_kernel<false, false>);
        hipLaunchKernelGGL(k, grid, dim3(kThreads), lds, stream, p, (int32_t)r0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace kvx
