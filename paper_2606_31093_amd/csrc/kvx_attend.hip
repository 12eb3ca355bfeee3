// kvx_attend.hip -- attention of one query per request over a paged cache
// (gfx950).
//
// Mathematics.  s = scale q.K, softmax over the positions, out = p V, in one
// pass over the cache with a running maximum m and sum l.  A workgroup takes
// `chunk` positions of one record and cache head; the chunks of a record are
// joined by a second launch: out = sum 2^(m_c - M) o_c / sum 2^(m_c - M) l_c.
// Scores are kept in units of log2, so that a weight is one exp2.
//
// Matrix products without a move between lanes.  A wavefront takes 32
// positions at a time against 16 query heads of one cache head (a group of
// fewer leaves columns unused: the product of 16 columns still costs far less
// than the memory does).  With c = lane % 16 and q = lane / 16:
// - scores: A = 16 rows of K (lane: row c, elements 8q..8q+7 of every 32), B =
//   the queries; the result gives lane (c, q) the scores of head c at positions
//   4q..4q+3, and two such products positions 16 + 4q..16 + 4q+3 as well;
// - those 8 weights are exactly one lane's part of the A operand of the second
//   product if its k index 8q + i stands for position 4q + i (i < 4) or
//   16 + 4q + i - 4.  Any order of k serves when B has the same one;
// - B = V: lane (c, q) loads W consecutive elements from c * W on of those 8
//   positions (16 lanes read a row as one run) and transposes its own 8 x W
//   block with byte permutes; product j then makes the outputs c * W + j.
// So neither scores, weights nor values pass through LDS or between lanes,
// except the row offsets that lanes resolve for each other, and the maxima.

#include "kvx_ops.h"
#include "kvx_values.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int kTile = 32;               // positions a wavefront takes at a time
// Weights are taken against a reference that follows the running maximum: it
// starts kLift below it and is raised when a tile's maximum is more than kSlack
// above where that leaves it, so that the sums are seldom rescaled.  Half has
// 2^-14 as smallest normal value and 65504 as largest: lifted by 7, weights up
// to 2^15, the small ones keep their digits 7 binades longer.
constexpr float kSlack = 8.0f;
template <bool F16>
constexpr float kLift = F16 ? 7.0f : 0.0f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// 2^(x - m), 0 where nothing has been seen (m = -inf).
__device__ __forceinline__ float weight(float x, float m) { return m == -INFINITY ? 0.f : exp2_fast(x - m); }

__device__ __forceinline__ bool valid(const kvx_attend_req &q, const AttendParams &p) {
    if (q.start < 0 || q.end < q.start || q.end - q.start > p.max_tokens) return false;
    if (!p.acc) return true;
    // accumulators [acc_off + start, acc_off + (H - 1) * stride + end) lie inside
    return q.acc_off >= 0 && q.acc_off <= p.acc_len && q.end <= p.acc_len - q.acc_off &&
           (p.pool.H == 1 || p.acc_stride <= (p.acc_len - q.acc_off - q.end) / (p.pool.H - 1));
}

// Chunks of a record that hold positions (at least one, for its zeros).
__device__ __forceinline__ int used_chunks(const kvx_attend_req &q, int chunk) {
    const int n = q.end - (q.start & -kTile);
    return q.end > q.start ? (n + chunk - 1) / chunk : 1;
}

template <bool F16, bool E4M3, int DC, int W, int NB>
__global__ void __launch_bounds__(64 * kWaves) kvx_attend_kernel(AttendParams p, int32_t r0) {
    typedef Half<F16> V;
    __shared__ int64_t row_off[kWaves][kTile];
    __shared__ float ml[kWaves][16][2];
    extern __shared__ float joined[];            // [waves_h][16][Dv], waves of the same heads only

    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane & 15, quad = lane >> 4;
    uint32_t b = blockIdx.x;
    const uint32_t hb = b % (uint32_t)(p.pool.H * p.head_blocks);
    b /= (uint32_t)(p.pool.H * p.head_blocks);
    const int chunk = (int)(b % (uint32_t)p.chunks);
    const int r = r0 + (int)(b / (uint32_t)p.chunks);
    const int h = (int)hb / p.head_blocks;
    const int wh = wave % p.waves_h, wt = wave / p.waves_h, waves_t = kWaves / p.waves_h;
    // first of this wave's 16 heads, within the group
    const int g0 = (((int)hb % p.head_blocks) * p.waves_h + wh) * 16;

    const kvx_attend_req rec = p.reqs[r];
    if (!valid(rec, p)) {
        if (blockIdx.x % (uint32_t)(p.pool.H * p.head_blocks * p.chunks) == 0 && threadIdx.x == 0 && p.err)
            atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    if (chunk >= used_chunks(rec, p.chunk)) return;
    const int begin = (rec.start & -kTile) + chunk * p.chunk;
    const int end = rec.end - begin < p.chunk ? rec.end : begin + p.chunk;

    // queries: head g0 + c, elements 8 quad.. of every 32
    u32x4 qv[DC];
    {
        const bool on = g0 + c < p.G;
        const char *src = p.q.base + r * p.q.s_row + (int64_t)(h * p.G + (on ? g0 + c : 0)) * p.q.s_head;
#pragma unroll
        for (int j = 0; j < DC; ++j) {
            const int d = j * 32 + quad * 8;
            qv[j] = u32x4{0, 0, 0, 0};
            if (on && d < p.pool.D) qv[j] = *reinterpret_cast<const u32x4 *>(src + 2 * d);
        }
    }
    const float k_scale = p.scales ? p.scales[h] : 1.f;
    const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
    const float unit = p.scale_log2 * k_scale;
    const char *kbase = p.pool.base + h * p.pool.s_h;
    const char *vbase = kbase + (p.pool.C - 1) * p.pool.s_c;

    f32x4 o[NB * W];
#pragma unroll
    for (int j = 0; j < NB * W; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    float *scores = p.scores ? p.scores + ((int64_t)r * p.pool.H * p.G + h * p.G + g0 + c) * p.score_stride -
                                   (rec.start & -kTile)
                             : nullptr;

    // unsigned: a tile may begin past 2^31 - 1, the last position there is
    for (uint32_t t0 = begin + wt * kTile; t0 < (uint32_t)end; t0 += waves_t * kTile) {
        // row offsets of the tile's positions, and which of them take part
        bool ok = false;
        if (lane < kTile) {
            const uint32_t t = t0 + lane;
            int64_t off = 0;
            ok = t >= (uint32_t)rec.start && t < (uint32_t)end;
            if (ok) {
                const uint32_t page_no = fd_div(p.pool.fd_T, t);
                const uint64_t idx = (uint64_t)rec.pt_off + page_no;
                if (idx >= (uint64_t)p.pool.pt_len) {
                    ok = false;
                    if (p.err) atomicOr(p.err, KVX_DERR_PT_RANGE);
                } else {
                    const int32_t page = p.pool.pt[idx];
                    if (page < 0 || page >= p.pool.N) {
                        ok = false;
                        if (p.err) atomicOr(p.err, KVX_DERR_SRC_PAGE);
                    } else {
                        off = page * p.pool.s_p + (int64_t)(t - page_no * p.pool.fd_T.d) * p.pool.s_t;
                    }
                }
            }
            row_off[wave][lane] = off;
        }
        const uint32_t mask = (uint32_t)__ballot(ok);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

        // scores of positions 4 quad + i and 16 + 4 quad + i
        f32x4 s[2];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char *row = kbase + row_off[wave][16 * half + c];
            s[half] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < DC; ++j) {
                const int d = j * 32 + quad * 8;
                u32x4 a = {0, 0, 0, 0};
                if (d < p.pool.D) {
                    if (E4M3) {
                        const u32x2 w = *reinterpret_cast<const u32x2 *>(row + d);
                        a = u32x4{V::template from_e4m3<false>(w[0]), V::template from_e4m3<true>(w[0]),
                                  V::template from_e4m3<false>(w[1]), V::template from_e4m3<true>(w[1])};
                    } else {
                        a = *reinterpret_cast<const u32x4 *>(row + 2 * d);
                    }
                }
                s[half] = V::mfma(a, qv[j], s[half]);
            }
        }
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = s[i / 4][i % 4] * unit;
        if (mask != 0xffffffffu) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (!((mask >> (16 * (i / 4) + 4 * quad + i % 4)) & 1)) x[i] = -INFINITY;
        }
        if (scores && g0 + c < p.G) {
            *reinterpret_cast<f32x4 *>(scores + t0 + 4 * quad) = f32x4{x[0], x[1], x[2], x[3]};
            *reinterpret_cast<f32x4 *>(scores + t0 + 16 + 4 * quad) = f32x4{x[4], x[5], x[6], x[7]};
        }

        // the maximum of head c over the tile
        float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top - kLift<F16> > m + kSlack)) {
            const float next = fmaxf(m, top - kLift<F16>), f = weight(m, next);
            m = next;
            l *= f;
            f32x4 fr;
#pragma unroll
            for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * quad + i);
#pragma unroll
            for (int j = 0; j < NB * W; ++j) o[j] *= fr;
        }
        float w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = weight(x[i], m);
            l += w[i];
        }
        const u32x4 a = {V::pack(w[0], w[1]), V::pack(w[2], w[3]), V::pack(w[4], w[5]), V::pack(w[6], w[7])};

        // values: 8 positions x W elements a lane
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            uint32_t v[8][W / 2];
            const int d = (nb * 16 + c) * W;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const char *row = vbase + row_off[wave][16 * (i / 4) + 4 * quad + i % 4];
#pragma unroll
                for (int e = 0; e < W / 2; ++e) v[i][e] = 0;
                // a position that takes no part must not bring its NaN
                const bool use = d < p.Dv && ((mask >> (16 * (i / 4) + 4 * quad + i % 4)) & 1);
                if (use) {
                    if (E4M3) {
#pragma unroll
                        for (int e = 0; e < W / 4; ++e) {
                            const uint32_t y = *reinterpret_cast<const uint32_t *>(row + d + 4 * e);
                            v[i][2 * e] = V::template from_e4m3<false>(y);
                            v[i][2 * e + 1] = V::template from_e4m3<true>(y);
                        }
                    } else {
                        __builtin_memcpy(v[i], __builtin_assume_aligned(row + 2 * d, 2 * W), 2 * W);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;
                u32x4 bv;
#pragma unroll
                for (int i = 0; i < 4; ++i) bv[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], pick);
                o[nb * W + j] = V::mfma(a, bv, o[nb * W + j]);
            }
        }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // Join the waves of the same heads: each scales to the common maximum, then
    // they add up in LDS, one after the other.
    if (waves_t > 1) {
        if (quad == 0) {
            ml[wave][c][0] = m;
            ml[wave][c][1] = l;
        }
        __syncthreads();
        float all = -INFINITY, sum = 0.f;
        for (int k = wh; k < kWaves; k += p.waves_h) all = fmaxf(all, ml[k][c][0]);
        for (int k = wh; k < kWaves; k += p.waves_h) sum += ml[k][c][1] * weight(ml[k][c][0], all);
        const float f = weight(m, all);
        m = all;
        l = sum;
        f32x4 fr;
#pragma unroll
        for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * quad + i);
#pragma unroll
        for (int j = 0; j < NB * W; ++j) o[j] *= fr;
        float *mine = joined + (int64_t)wh * 16 * (NB * 16 * W);
        for (int turn = 0; turn < waves_t; ++turn) {
            if (wt == turn) {
#pragma unroll
                for (int j = 0; j < NB * W; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float *at = mine + (4 * quad + i) * (NB * 16 * W) + (j / W * 16 + c) * W + j % W;
                        if (turn > 0) o[j][i] += *at;
                        if (turn < waves_t - 1) *at = o[j][i];
                    }
            }
            __syncthreads();
        }
        if (wt != waves_t - 1) return;
    }

    const int64_t head0 = (int64_t)r * p.pool.H * p.G + h * p.G + g0;      // of the wave's 16
    const bool last = used_chunks(rec, p.chunk) == 1;
    if (quad == 0 && g0 + c < p.G) {
        if (last) {
            const float x = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
            if (p.lse) p.lse[head0 + c] = x * kLn2;
            if (p.lse2) p.lse2[head0 + c] = x;
        } else {
            float *at = p.part_ml + ((head0 + c) * p.chunks + chunk) * 2;
            at[0] = m;
            at[1] = l;
        }
    }
    f32x4 lr;
#pragma unroll
    for (int i = 0; i < 4; ++i) lr[i] = __shfl(l, 4 * quad + i);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int g = g0 + 4 * quad + i;
        if (g >= p.G) continue;
        if (last) {
            const float f = lr[i] == 0.f ? 0.f : v_scale / lr[i];
            char *dst = p.out.base + r * p.out.s_row + (int64_t)(h * p.G + g) * p.out.s_head;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int d = (nb * 16 + c) * W;
                if (d >= p.Dv) continue;
                uint32_t w[W / 2];
#pragma unroll
                for (int e = 0; e < W / 2; ++e)
                    w[e] = V::pack(o[nb * W + 2 * e][i] * f, o[nb * W + 2 * e + 1][i] * f);
                __builtin_memcpy(__builtin_assume_aligned(dst + 2 * d, 2 * W), w, 2 * W);
            }
        } else {
            float *dst = p.part_o + ((head0 + 4 * quad + i) * p.chunks + chunk) * p.Dv;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int d = (nb * 16 + c) * W;
                if (d >= p.Dv) continue;
#pragma unroll
                for (int e = 0; e < W; e += 4)
                    *reinterpret_cast<f32x4 *>(dst + d + e) =
                        f32x4{o[nb * W + e][i], o[nb * W + e + 1][i], o[nb * W + e + 2][i], o[nb * W + e + 3][i]};
            }
        }
    }
}

// Joins the chunks of one record and query head: a wavefront per 64 outputs at
// a time, every lane its element over all chunks.
template <bool F16>
__global__ void __launch_bounds__(256) kvx_attend_join_kernel(AttendParams p, int64_t first) {
    const int64_t head = first + blockIdx.x;
    const int Hq = p.pool.H * p.G;
    const int r = (int)(head / Hq), hq = (int)(head % Hq);
    const kvx_attend_req rec = p.reqs[r];
    if (!valid(rec, p)) return;
    const int n = used_chunks(rec, p.chunk);
    if (n == 1) return;
    const float *ml = p.part_ml + head * p.chunks * 2;
    float m = -INFINITY, l = 0.f;
    for (int k = threadIdx.x % 64; k < n; k += 64) m = fmaxf(m, ml[2 * k]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    for (int k = threadIdx.x % 64; k < n; k += 64) l += ml[2 * k + 1] * weight(ml[2 * k], m);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
    if (threadIdx.x == 0) {
        const float x = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
        if (p.lse) p.lse[head] = x * kLn2;
        if (p.lse2) p.lse2[head] = x;
    }
    const int h = hq / p.G;
    const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
    const float f = l == 0.f ? 0.f : v_scale / l;
    const float *part = p.part_o + head * p.chunks * p.Dv;
    char *dst = p.out.base + r * p.out.s_row + hq * p.out.s_head;
    for (int d = threadIdx.x; d < p.Dv; d += 256) {
        float x = 0.f;
        for (int k = 0; k < n; ++k) x += part[(int64_t)k * p.Dv + d] * weight(ml[2 * k], m);
        reinterpret_cast<uint16_t *>(dst)[d] = (uint16_t)Half<F16>::pack(x * f, 0.f);
    }
}

// acc += sum over the group of 2^(score - lse): a thread per position.
__global__ void __launch_bounds__(256) kvx_attend_acc_kernel(AttendParams p, int32_t r0, int32_t piece0, int32_t blocks) {
    uint32_t b = blockIdx.x;
    const int piece = piece0 + (int)(b % (uint32_t)blocks);
    b /= (uint32_t)blocks;
    const int h = (int)(b % (uint32_t)p.pool.H), r = r0 + (int)(b / (uint32_t)p.pool.H);
    const kvx_attend_req rec = p.reqs[r];
    if (!valid(rec, p)) return;
    const int base = rec.start & -kTile;
    const int t = base + piece * 256 + (int)threadIdx.x;
    if (t < rec.start || t >= rec.end) return;
    const int64_t head0 = ((int64_t)r * p.pool.H + h) * p.G;
    float x = 0.f;
    for (int g = 0; g < p.G; ++g) {
        const float lse = p.lse2[head0 + g];
        if (lse != -INFINITY) x += exp2_fast(p.scores[(head0 + g) * p.score_stride + t - base] - lse);
    }
    p.acc[rec.acc_off + h * p.acc_stride + t] += x;
}

template <bool F16, bool E4M3>
auto pick(int D, int Dv) {
    if (D <= 64) return kvx_attend_kernel<F16, E4M3, 2, 4, 1>;
    if (D <= 128) return kvx_attend_kernel<F16, E4M3, 4, 8, 1>;
    if (D <= 192) return kvx_attend_kernel<F16, E4M3, 6, 4, 3>;
    if (D <= 256) return kvx_attend_kernel<F16, E4M3, 8, 8, 2>;
    return kvx_attend_kernel<F16, E4M3, 18, 8, 4>;
}

int padded(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : D <= 192 ? 192 : D <= 256 ? 256 : 512; }

}  // namespace

// Workgroups aimed at: 4 or more for each of the 256 compute units at equal
// lengths; half as many where a workgroup holds 64 heads of 512 values, whose
// partial sums would weigh against the cache read.
static int64_t target(const AttendParams &p) { return p.waves_h == kWaves ? 1024 : 2048; }

void plan_attend(AttendParams &p) {
    const int tiles = (p.G + 15) / 16;
    p.waves_h = tiles >= 4 ? 4 : tiles >= 2 ? 2 : 1;
    p.head_blocks = (tiles + p.waves_h - 1) / p.waves_h;
    const int step = kTile * (kWaves / p.waves_h);          // positions a workgroup takes at a time
    const int64_t units = (int64_t)p.n_reqs * p.pool.H * p.head_blocks;
    const int64_t span = (int64_t)p.max_tokens + kTile - 1;
    int64_t chunk = (span * units + target(p) - 1) / target(p);
    chunk = (chunk + step - 1) / step * step;
    if (chunk > span) chunk = (span + step - 1) / step * step;
    if (chunk < step) chunk = step;
    p.chunk = (int32_t)chunk;
    p.chunks = (int32_t)((span + chunk - 1) / chunk);
    p.score_stride = (span + kTile + 31) / 32 * 32;
}

// Partial results of a call with as many or fewer records and positions: units
// * chunks is at most target + units, and at most one chunk per step.
static int64_t most_parts(const AttendParams &p) {
    const int step = kTile * (kWaves / p.waves_h);
    const int64_t units = (int64_t)p.n_reqs * p.pool.H * p.head_blocks;
    const int64_t span = (int64_t)p.max_tokens + kTile - 1;
    const int64_t a = target(p) + units, b = units * ((span + step - 1) / step);
    return (p.G + p.head_blocks - 1) / p.head_blocks * (a < b ? a : b);
}

int64_t attend_workspace(AttendParams &p, char *base) {
    const int64_t heads = (int64_t)p.n_reqs * p.pool.H * p.G;
    int64_t at = 0;
    const auto take = [&](int64_t floats) {
        float *x = base ? reinterpret_cast<float *>(base + at) : nullptr;
        at += (floats * 4 + 15) / 16 * 16;
        return x;
    };
    const int64_t parts = base ? heads * p.chunks : most_parts(p);
    p.lse2 = take(heads);
    p.part_ml = take(parts * 2);
    p.part_o = take(parts * p.Dv);
    p.scores = p.acc ? take(heads * p.score_stride) : nullptr;
    return at;
}

int launch_attend(const AttendParams &p, hipStream_t stream) {
    if (p.n_reqs == 0) return hipSuccess;
    const auto kernel = p.f16 ? (p.e4m3 ? pick<true, true>(p.pool.D, p.Dv) : pick<true, false>(p.pool.D, p.Dv))
                              : (p.e4m3 ? pick<false, true>(p.pool.D, p.Dv) : pick<false, false>(p.pool.D, p.Dv));
    const size_t lds = p.waves_h == kWaves ? 0 : sizeof(float) * p.waves_h * 16 * padded(p.pool.D);
    const int64_t per = (int64_t)p.pool.H * p.head_blocks * p.chunks;
    int64_t group = kMaxBlocks / per > 0 ? kMaxBlocks / per : 1;
    hipError_t e;
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
        const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)(n * per)), dim3(64 * kWaves), lds, stream, p, (int32_t)r0);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.chunks > 1) {
        const int64_t heads = (int64_t)p.n_reqs * p.pool.H * p.G;
        for (int64_t at = 0; at < heads; at += kMaxBlocks) {
            const int64_t n = heads - at < kMaxBlocks ? heads - at : kMaxBlocks;
            hipLaunchKernelGGL(p.f16 ? kvx_attend_join_kernel<true> : kvx_attend_join_kernel<false>, dim3((uint32_t)n),
                               dim3(256), 0, stream, p, at);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (p.acc) {
        const int32_t pieces = (p.max_tokens + kTile - 1 + 255) / 256;
        const int32_t blocks = (int32_t)(kMaxBlocks / p.pool.H < pieces ? kMaxBlocks / p.pool.H : pieces);
        const int64_t per_r = (int64_t)blocks * p.pool.H;
        group = kMaxBlocks / per_r;
        for (int32_t piece0 = 0; piece0 < pieces; piece0 += blocks) {
            for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
                const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
                hipLaunchKernelGGL(kvx_attend_acc_kernel, dim3((uint32_t)(n * per_r)), dim3(256), 0, stream, p,
                                   (int32_t)r0, piece0, blocks);
                if ((e = hipGetLastError()) != hipSuccess) return e;
            }
        }
    }
    return hipSuccess;
}

}  // namespace kvx
