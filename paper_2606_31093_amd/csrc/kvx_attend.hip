// kvx_attend.hip -- attention of one query per request over a paged cache
// (gfx950).
//
// Mathematics.  s = scale q.K, softmax over the positions, out = p V, in one
// pass over the cache with a running maximum m and sum l.  Scores are kept in
// units of log2, so that a weight is one exp2.
//
// Division of the work.  A unit is a record and some of its cache heads (or a
// part of their query heads); it takes a step for every 32 to 256 positions.
// Only the device knows the lengths, so the workgroups, as many as the device
// holds at a time, add them up and take equal shares of all steps in order.  A
// unit that lies in one share is finished there; the parts of the others are
// joined by a second launch: out = sum 2^(m_c - M) o_c / sum 2^(m_c - M) l_c.
// Where no record takes more than a few steps, each unit has its own workgroup
// instead, and there is no second launch.
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
//   The weights are two parts in the rows' type, a product each; the second product
//   took no time with up to 16 query heads a cache head, and 1 to 3% with 32 and 64;
// - B = V: lane (c, q) loads W consecutive elements from c * W on of those 8
//   positions (16 lanes read a row as one run) and transposes its own 8 x W
//   block with byte permutes; product j then makes the outputs c * W + j.
// So neither scores, weights nor values pass through LDS or between lanes,
// except the row offsets that lanes resolve for each other, and the maxima.
//
// Bound by the cache's bytes, and where they are few by the second launch:
// bfloat16, 8 cache heads of 128, 32 query heads: one request of 32768
// positions (134 MB) takes 36 us, 29 of them the first launch; 32 requests of
// 1024 to 8192 with accumulated weights (663 MB) 152 us, 136 of them the first
// launch; e4m3, 4 cache heads, 28 query heads, 16 requests of 2048 to 16384
// (177 MB) 47 us, 42 of them the first launch.

#include "kvx_attend.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;

// A tile's rows while they are on their way: K in the shape of the first
// product's A operand, V as the second product's B operand before its
// transposition.
template <bool E4M3, int DC, int W, int NB, int TT>
struct Tile {
    static constexpr int KL = E4M3 ? DC / 2 : DC;    // 16-byte loads of a row's quarter
    static constexpr int VD = E4M3 ? W / 4 : W / 2;  // dwords of W elements
    uint32_t k[2 * TT][KL][4];
    uint32_t v[TT][NB][8][VD];
};

template <int N>
__device__ __forceinline__ void load_dwords(uint32_t *to, const char *from) {
    typedef __attribute__((ext_vector_type(N))) uint32_t vec;
    const vec v = __builtin_nontemporal_load(reinterpret_cast<const vec *>(from));
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = v[i];
}

template <>
__device__ __forceinline__ void load_dwords<1>(uint32_t *to, const char *from) {
    to[0] = *reinterpret_cast<const uint32_t *>(from);
}

// EXACT: head_dim and v_dim are 32 DC and 16 W NB; else the elements past them
// are read from the row's begin and taken as 0.  TT: 32 positions a wavefront
// takes at a time.
template <bool F16, bool E4M3, int DC, int W, int NB, int TT, bool EXACT, bool ACC>
__device__ __forceinline__ void attend_part(const AttendParams &p, const Part part, int64_t (*row_off)[64],
                                            float (*ml)[16][2], float *joined) {
    const kvx_attend_req rec = part.rec;
    const int r = part.r, hb = part.hb;
    const int64_t place = part.place;
    typedef Half<F16> V;
    constexpr int ES = E4M3 ? 1 : 2, TILE = 32 * TT;
    constexpr uint64_t ALL = TT == 2 ? ~0ull : 0xffffffffull;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int c = lane & 15, quad = lane >> 4;
    // waves along cache heads, blocks of 16 of their query heads, and positions
    const int waves_t = kWaves / (p.waves_h * p.waves_k);
    const int wt = wave % waves_t, wh = wave / waves_t % p.waves_h, wk = wave / (waves_t * p.waves_h);
    const int h = hb / p.head_blocks * p.waves_k + wk;
    // first of this wave's 16 heads, within the group
    const int g0 = ((hb % p.head_blocks) * p.waves_h + wh) * 16;

    // unsigned: a tile may begin past 2^31 - 1, the last position there is
    const uint32_t begin = part.begin, end = part.end, first = rec.start;
    const uint32_t step = waves_t * TILE;

    // A lane resolves position t0 + lane: its page id, and a tile later the row
    // offset.  The load is unconditional, so that nothing waits for it early.
    uint32_t bad = 0;
    const auto entry = [&](uint32_t t) { return (uint64_t)rec.pt_off + fd_div(p.pool.fd_T, t); };
    const auto look = [&](uint32_t t0) {
        const uint32_t t = t0 + lane;
        const uint64_t idx = entry(t < end ? t : end - 1);
        return p.pool.pt[idx < (uint64_t)p.pool.pt_len ? idx : 0];
    };
    // The row offsets of a tile to LDS; returns the positions that take part.
    const auto resolve = [&](uint32_t t0, int32_t page, int64_t *to) {
        const uint32_t t = t0 + lane;
        const bool in = lane < TILE && t >= first && t < end;
        const uint32_t at = t < end ? t : end - 1;
        const bool known = entry(at) < (uint64_t)p.pool.pt_len;
        const bool ok = in && known && (uint32_t)page < (uint32_t)p.pool.N;
        if (in && !ok) bad |= known ? KVX_DERR_SRC_PAGE : KVX_DERR_PT_RANGE;
        // every lane writes: a branch for some would split the loop's registers' lives
        const int64_t off = page * p.pool.s_p + (int64_t)(at - fd_div(p.pool.fd_T, at) * p.pool.fd_T.d) * p.pool.s_t;
        to[lane] = ok ? off : 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        return (uint64_t)__ballot(ok);
    };

    const char *kbase = p.pool.base + h * p.pool.s_h;
    const char *vbase = kbase + (p.pool.C - 1) * p.pool.s_c;
    Tile<E4M3, DC, W, NB, TT> tile;
    const auto load_k = [&](const int64_t *off) {
#pragma unroll
        for (int half = 0; half < 2 * TT; ++half) {
            const char *row = kbase + off[16 * half + c];
#pragma unroll
            for (int j = 0; j < tile.KL; ++j) {
                const int at = j * 64 + quad * 16;         // bytes
                load_dwords<4>(tile.k[half][j], row + (EXACT || at < ES * p.pool.D ? at : 0));
            }
        }
    };
    const auto load_v = [&](const int64_t *off) {
#pragma unroll
        for (int i = 0; i < 8 * TT; ++i) {
            const char *row = vbase + off[16 * (i / 4) + 4 * quad + i % 4];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                const int d = (nb * 16 + c) * W;
                load_dwords<tile.VD>(tile.v[i / 8][nb][i % 8], row + ES * (EXACT || d < p.Dv ? d : 0));
            }
        }
    };

    // Step j of the first product contracts 8 elements from dim(j) on: any order
    // serves that gives a lane 16 consecutive bytes of its row.
    const auto dim = [&](int j) { return E4M3 ? j / 2 * 64 + quad * 16 + j % 2 * 8 : j * 32 + quad * 8; };
    const int heads = p.G - g0 < 16 ? p.G - g0 : 16;     // of this wave
    // queries
    u32x4 qv[DC];
    {
        const bool on = c < heads;
        const char *src = p.q.base + r * p.q.s_row + (int64_t)(h * p.G + (on ? g0 + c : 0)) * p.q.s_head;
#pragma unroll
        for (int j = 0; j < DC; ++j) {
            const int d = dim(j);
            qv[j] = *reinterpret_cast<const u32x4 *>(src + 2 * (EXACT || d < p.pool.D ? d : 0));
        }
#pragma unroll
        for (int j = 0; j < DC; ++j)
            if (!on || (!EXACT && dim(j) >= p.pool.D)) qv[j] = u32x4{0, 0, 0, 0};
    }
    const float k_scale = p.scales ? p.scales[h] : 1.f;
    const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
    const float unit = p.scale_log2 * k_scale;

    f32x4 o[NB * W];
#pragma unroll
    for (int j = 0; j < NB * W; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    // Scores of head c from the position 4 quad on; the other columns' go to a
    // line of their own that nothing reads (64 spare floats a row of threads).
    float *scores = nullptr;
    if (ACC)
        scores = (c < heads ? p.scores + ((int64_t)r * p.pool.H * p.G + h * p.G + g0 + c) * p.score_stride - (rec.start & -kTile)
                            : p.spare) + 4 * quad;

    uint32_t t0 = begin + wt * TILE;
    if (t0 < end) {
        uint64_t mask = resolve(t0, look(t0), row_off[2 * wave]);
        int32_t page = look(t0 + step);
        // Page id, keys, values: asked for in the loop's order, which the loop's waits
        // count on (in another order the first turn's wait would be one for all).
        __builtin_amdgcn_sched_barrier(0);
        load_k(row_off[2 * wave]);
        __builtin_amdgcn_sched_barrier(0);
        load_v(row_off[2 * wave]);
        for (int turn = 0; t0 < end; t0 += step, turn ^= 1) {
            // Keys and values of this tile are on their way.  Those of the next are
            // asked for as soon as this tile's have been used, and its page ids were
            // a tile earlier, so that loads are in flight at all times.  Behind the
            // last tile they are asked for once more, from the layer's first row: a
            // branch around them would make the wait for this tile's loads one for all.
            int64_t *next = row_off[2 * wave + (turn ^ 1)];
            const uint64_t next_mask = resolve(t0 + step, page, next);
            page = look(t0 + 2 * step);

            // x[i]: the score of position 16 (i / 4) + 4 quad + i % 4
            float x[8 * TT];
#pragma unroll
            for (int half = 0; half < 2 * TT; ++half) {
                f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < DC; ++j) {
                    u32x4 a = widen<F16, E4M3>(E4M3 ? tile.k[half][j / 2] + j % 2 * 2 : tile.k[half][j]);
                    if (!EXACT && dim(j) >= p.pool.D) a = u32x4{0, 0, 0, 0};
                    s = V::mfma(a, qv[j], s);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) x[4 * half + i] = s[i] * unit;
            }
            load_k(next);

            if (mask != ALL) {
                // positions that take no part: no weight, and values that bring no NaN
                const uint64_t mine = mask >> (4 * quad);
#pragma unroll
                for (int i = 0; i < 8 * TT; ++i) {
                    if ((mine >> (16 * (i / 4) + i % 4)) & 1) continue;
                    x[i] = -INFINITY;
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                        for (int e = 0; e < tile.VD; ++e) tile.v[i / 8][nb][i % 8][e] = 0;
                }
            }

            // the maximum of head c over the tile
            float top = x[0];
#pragma unroll
            for (int i = 1; i < 8 * TT; ++i) top = fmaxf(top, x[i]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any(top - kLift<F16> > m + kSlack)) {
                const float raised = fmaxf(m, top - kLift<F16>), f = weight(m, raised);
                m = raised;
                l *= f;
                f32x4 fr;
#pragma unroll
                for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * quad + i);
#pragma unroll
                for (int j = 0; j < NB * W; ++j) o[j] *= fr;
            }
            const float from = m == -INFINITY ? 0.f : m;       // then every x is -inf
#pragma unroll
            for (int u = 0; u < TT; ++u) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = exp2_fast(x[8 * u + i] - from);
                    l += w[i];
                }
                u32x4 a, rest;
                split<F16>(w, a, rest);

                // values: 8 positions x W elements a lane, transposed
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    uint32_t v[8][W / 2];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
#pragma unroll
                        for (int e = 0; e < W / 2; ++e) {
                            if (E4M3)
                                v[i][e] = e % 2 ? V::template from_e4m3<true>(tile.v[u][nb][i][e / 2])
                                                : V::template from_e4m3<false>(tile.v[u][nb][i][e / 2]);
                            else
                                v[i][e] = tile.v[u][nb][i][e];
                            if (!EXACT && (nb * 16 + c) * W >= p.Dv) v[i][e] = 0;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < W; ++j) {
                        const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;
                        u32x4 bv;
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            bv[i] = __builtin_amdgcn_perm(v[2 * i + 1][j / 2], v[2 * i][j / 2], pick);
                        o[nb * W + j] = V::mfma(a, bv, o[nb * W + j]);
                        o[nb * W + j] = V::mfma(rest, bv, o[nb * W + j]);
                    }
                }
            }
            load_v(next);
            // Behind the loads, so that what waits for them does not wait for the
            // stores; by all lanes, so that the waits count on them.
            if (ACC) {
                float *to = scores + (c < heads ? t0 : 0);
#pragma unroll
                for (int i = 0; i < 2 * TT; ++i)
                    *reinterpret_cast<f32x4 *>(to + 16 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
            }
            mask = next_mask;
        }
    }
    if (bad && p.err) atomicOr(p.err, bad);
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
        const int w0 = wave - wt;
        for (int k = w0; k < w0 + waves_t; ++k) all = fmaxf(all, ml[k][c][0]);
        for (int k = w0; k < w0 + waves_t; ++k) sum += ml[k][c][1] * weight(ml[k][c][0], all);
        const float f = weight(m, all);
        m = all;
        l = sum;
        f32x4 fr;
#pragma unroll
        for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * quad + i);
#pragma unroll
        for (int j = 0; j < NB * W; ++j) o[j] *= fr;
        f32x4 *mine = reinterpret_cast<f32x4 *>(joined) + (int64_t)(wave / waves_t) * 64 * NB * W + lane;
        for (int turn = 0; turn < waves_t; ++turn) {
            if (wt == turn) {
#pragma unroll
                for (int j = 0; j < NB * W; ++j) {
                    if (turn > 0) o[j] += mine[64 * j];
                    if (turn < waves_t - 1) mine[64 * j] = o[j];
                }
            }
            __syncthreads();
        }
        if (wt != waves_t - 1) return;
    }

    const int64_t head0 = (int64_t)r * p.pool.H * p.G + h * p.G + g0;      // of the wave's 16
    // a part's heads: those of wave block wk, from wh * 16 on
    const int64_t part0 = place < 0 ? 0 : (place * p.waves_k + wk) * p.part_heads + wh * 16;
    if (quad == 0 && c < heads) {
        if (place < 0) {
            const float x = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
            if (p.lse) p.lse[head0 + c] = x * kLn2;
            p.lse2[head0 + c] = x;
        } else {
            p.part_ml[(part0 + c) * 2] = m;
            p.part_ml[(part0 + c) * 2 + 1] = l;
        }
    }
    f32x4 lr;
#pragma unroll
    for (int i = 0; i < 4; ++i) lr[i] = __shfl(l, 4 * quad + i);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int g = g0 + 4 * quad + i;
        if (4 * quad + i >= heads) continue;
        if (place < 0) {
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
            float *dst = p.part_o + (part0 + 4 * quad + i) * p.Dv;
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

// A workgroup's share, unit by unit.
template <bool F16, bool E4M3, int DC, int W, int NB, int TT, bool EXACT, bool ACC>
__global__ void __launch_bounds__(64 * kWaves) kvx_attend_kernel(AttendParams p, int32_t r0, int32_t n) {
    __shared__ int32_t before[kAttendGroup + 1];
    __shared__ __align__(16) int64_t row_off[2 * kWaves][64];
    __shared__ float ml[kWaves][16][2];
    extern __shared__ __align__(16) float joined[];   // [4 / waves along positions][W NB][lane][4]

    Walk walk(p, r0, n, before, blockIdx.x);
    Part part;
    while (walk.next(p, before, &part)) {
        attend_part<F16, E4M3, DC, W, NB, TT, EXACT, ACC>(p, part, row_off, ml, joined);
        __syncthreads();                         // the next unit uses the same LDS
    }
}

// The parts of a unit: shares first .. last, all or none of a unit in one.
struct Parts {
    int64_t first, last, unit0;
    Shares s;
    __device__ __forceinline__ Parts(const AttendParams &p, int32_t r, int hb, int32_t n) : s(p, p.before[n]) {
        const int32_t steps = p.before[r + 1] - p.before[r];
        unit0 = (int64_t)p.before[r] * p.per + (int64_t)hb * steps;
        first = quotient(unit0, s.each);
        last = steps > 0 ? quotient(unit0 + steps - 1, s.each) : first;
    }
    // a part's index of head g of the unit's cache head wk
    __device__ __forceinline__ int64_t head(const AttendParams &p, int64_t k, int wk, int g) const {
        return (s.place(p, unit0, k) * p.waves_k + wk) * p.part_heads + g;
    }
};

// log2 of a head's sum over its parts of 2^score, by a wavefront: maximum m and
// sum l of the parts' own.
__device__ __forceinline__ float joined_lse(const AttendParams &p, const Parts &u, int wk, int g) {
    float m = -INFINITY, l = 0.f;
#pragma unroll 4
    for (int64_t k = u.first + threadIdx.x % 64; k <= u.last; k += 64) {
        const float2 ml = *reinterpret_cast<const float2 *>(p.part_ml + 2 * u.head(p, k, wk, g));
        const float top = fmaxf(m, ml.x);
        l = l * weight(m, top) + ml.y * weight(ml.x, top);
        m = top;
    }
    const float mine = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
    l *= weight(mine, m);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
    return l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
}


// The second launch.  Its first `joins` workgroups join the parts of a record
// and query head each (Dv / 4 threads side by side, the parts dealt to as many
// such rows of threads as fit, added up in LDS); the others add the weights
// 2^(score - lse) of 4 positions a thread of a record and cache head to their
// accumulators.  They do not wait for the joins: each takes lse from the
// parts' maxima and sums itself.
template <bool F16>
__global__ void __launch_bounds__(1024) kvx_attend_finish_kernel(AttendParams p, int32_t r0, int32_t n, int64_t first,
                                                                int64_t joins, int32_t runs) {
    // partial outputs, maxima and sums of the rows of threads; a group's lse
    extern __shared__ __align__(16) float sums[];
    const int64_t at = first + blockIdx.x;
    const int Hq = p.pool.H * p.G, tid = threadIdx.x;
    const int span = p.span;
    if (at < joins) {
        const int r = (int)(at / Hq), hq = (int)(at % Hq), h = hq / p.G, g = hq % p.G;
        const Parts u(p, r, h / p.waves_k * p.head_blocks + g / span, n);
        if (u.first == u.last) return;           // written by the first launch, or malformed
        const int wk = h % p.waves_k, gp = g % span, parts = (int)(u.last - u.first) + 1;
        const int cols = p.Dv / 4, rows = blockDim.x / cols, col = tid % cols, row = tid / cols;
        float *row_m = sums + 4 * blockDim.x, *row_l = row_m + blockDim.x / 2;      // cols >= 2
        float m = -INFINITY, l = 0.f;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        if (row < rows) {
            for (int k0 = row; k0 < parts; k0 += 8 * rows) {
                f32x4 x[8];
                float2 y[8];
                // all on their way at once; past the end the last one, without weight
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int k = k0 + i * rows < parts ? k0 + i * rows : parts - 1;
                    const int64_t at = u.head(p, u.first + k, wk, gp);
                    y[i] = *reinterpret_cast<const float2 *>(p.part_ml + 2 * at);
                    x[i] = *reinterpret_cast<const f32x4 *>(p.part_o + at * p.Dv + 4 * col);
                }
                float top = m;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, y[i].x);
                const float f = weight(m, top);
                m = top;
                l *= f;
                sum *= f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (k0 + i * rows >= parts) continue;
                    const float w = weight(y[i].x, m);
                    l += y[i].y * w;
                    sum += x[i] * w;
                }
            }
            *reinterpret_cast<f32x4 *>(sums + 4 * tid) = sum;
            if (col == 0) {
                row_m[row] = m;
                row_l[row] = l;
            }
        }
        __syncthreads();
        if (row != 0) return;
        for (int k = 1; k < rows; ++k) m = fmaxf(m, row_m[k]);
        sum = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
        for (int k = 0; k < rows; ++k) {
            const float w = weight(row_m[k], m);
            l += row_l[k] * w;
            sum += *reinterpret_cast<const f32x4 *>(sums + 4 * (k * cols + col)) * w;
        }
        if (tid == 0 && p.lse)
            p.lse[(int64_t)(r0 + r) * Hq + hq] = (l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY) * kLn2;
        const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
        sum *= l == 0.f ? 0.f : v_scale / l;
        char *dst = p.out.base + (r0 + r) * p.out.s_row + hq * p.out.s_head;
        *reinterpret_cast<u32x2 *>(dst + 8 * col) =
            u32x2{Half<F16>::pack(sum[0], sum[1]), Half<F16>::pack(sum[2], sum[3])};
        return;
    }
    const int64_t b = at - joins;
    const int run = (int)(b % runs), h = (int)(b / runs % p.pool.H), r = (int)(b / runs / p.pool.H);
    const kvx_attend_req rec = p.reqs[r0 + r];
    if (!valid(rec, p)) return;
    const int base = rec.start & -kTile;
    if (rec.end - base <= run * 4 * (int)blockDim.x) return;
    const int64_t head0 = ((int64_t)(r0 + r) * p.pool.H + h) * p.G;
    // lse of the group's heads (at most 1024)
    for (int g = tid / 64; g < p.G; g += blockDim.x / 64) {
        float x = 0.f;
        bool split = false;
        if (!p.whole) {
            const Parts u(p, r, h / p.waves_k * p.head_blocks + g / span, n);
            split = u.first != u.last;
            if (split) x = joined_lse(p, u, h % p.waves_k, g % span);
        }
        if (!split) x = p.lse2[head0 + g];
        if (tid % 64 == 0) sums[g] = x;
    }
    __syncthreads();
    const int t = 4 * (run * (int)blockDim.x + tid);     // from base
    if (t >= rec.end - base) return;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    const float *scores = p.scores + head0 * p.score_stride + t;
    for (int g = 0; g < p.G; ++g) {
        const f32x4 s = *reinterpret_cast<const f32x4 *>(scores + g * p.score_stride);
        const float lse = sums[g];
        if (lse == -INFINITY) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] += exp2_fast(s[i] - lse);
    }
    float *acc = p.acc + rec.acc_off + h * p.acc_stride + base + t;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (base + t + i >= rec.start && t + i < rec.end - base) acc[i] += x[i];
}

// Tiles of 64 positions where rows are short (128 bytes and less): a wavefront
// then has 16 KiB on their way as with rows of 256, and units of up to 512 positions and
// more are whole (below).  8 cache heads of 64, 32 query heads: 64 requests of 300 took 15.5
// us, with tiles of 32 27.9 (e4m3: 11.3, 24.6); 32 of 4096 55.3 and 54.5 (37.8, 37.4); one
// of 16384 24.2 and 20.5 (20.3, 19.3).
int tile_of(int D) { return D <= 64 ? 2 : 1; }

template <bool F16, bool E4M3, bool ACC>
auto pick(int D, int Dv) {
    const bool exact = D == Dv;
    if (D == 64 && exact) return kvx_attend_kernel<F16, E4M3, 2, 4, 1, 2, true, ACC>;
    if (D <= 64) return kvx_attend_kernel<F16, E4M3, 2, 4, 1, 2, false, ACC>;
    if (D == 128 && exact) return kvx_attend_kernel<F16, E4M3, 4, 8, 1, 1, true, ACC>;
    if (D <= 128) return kvx_attend_kernel<F16, E4M3, 4, 8, 1, 1, false, ACC>;
    if (D <= 192) return kvx_attend_kernel<F16, E4M3, 6, 4, 3, 1, false, ACC>;
    if (D == 256 && exact) return kvx_attend_kernel<F16, E4M3, 8, 8, 2, 1, true, ACC>;
    return kvx_attend_kernel<F16, E4M3, 8, 8, 2, 1, false, ACC>;
}

template <bool ACC>
auto pick(const AttendParams &p) {
    return p.f16 ? (p.e4m3 ? pick<true, true, ACC>(p.pool.D, p.Dv) : pick<true, false, ACC>(p.pool.D, p.Dv))
                 : (p.e4m3 ? pick<false, true, ACC>(p.pool.D, p.Dv) : pick<false, false, ACC>(p.pool.D, p.Dv));
}

int padded(int D) { return D <= 64 ? 64 : D <= 128 ? 128 : D <= 192 ? 192 : 256; }

// Workgroups that the device holds at a time (its 256 compute units; a
// workgroup's registers leave room for 2 or 1 on each).
int resident(int D) { return D <= 128 ? 512 : 256; }

// A unit of up to this many steps is not worth a second launch.  8 cache heads of 128, 32
// query heads, 1 and 64 requests of 200 positions (8 steps): 13 and 18 us whole, 20 and 29
// split; of 300 (11): 17 and 25, 20 and 37; of 450 (16): 22 and 34, 20 and 40; of 700 (23):
// 30 and 48, 20 and 50.  Latents, 128 heads, one of 500 (9 steps): 50 whole, 33 split.
constexpr int kWholeSteps = 8;
// Fewer steps than this are not worth a share.  The same heads, 1, 8 and 64 requests of 4000,
// 4000 and 1000 positions: 21.7, 35.4 and 56.7 us; with shares of 1 step and more 17.7, 38.2 and
// 56.5, of 16 and more 40.0, 46.0 and 53.7.
constexpr int kLeastShare = 4;

}  // namespace

void plan_attend(AttendParams &p) {
    const int tiles = (p.G + 15) / 16;
    p.waves_h = tiles >= 4 ? 4 : tiles >= 2 ? 2 : 1;
    p.head_blocks = (tiles + p.waves_h - 1) / p.waves_h;
    p.waves_k = 1;
    if (p.pool.D > 256) {
        plan_attend_wide(p);
    } else {
    while (p.waves_h * p.waves_k < kWaves && p.pool.H % (2 * p.waves_k) == 0 && p.token_major) p.waves_k *= 2;
    p.span = p.waves_h * 16;
    p.step = 32 * tile_of(p.pool.D) * (kWaves / (p.waves_h * p.waves_k));
    p.shares = resident(p.pool.D);
    }
    p.part_heads = p.G < p.span ? p.G : p.span;
    p.per = p.pool.H / p.waves_k * p.head_blocks;
    const int64_t span = (int64_t)p.max_tokens + kTile - 1, steps = (span + p.step - 1) / p.step;
    p.whole = steps <= kWholeSteps;
    const int64_t n = p.n_reqs < kAttendGroup ? p.n_reqs : kAttendGroup;
    const int64_t most = (n * p.per * steps + kLeastShare - 1) / kLeastShare;
    if (p.shares > most) p.shares = (int32_t)most;
    p.score_stride = (span + 127) / 64 * 64;         // whole tiles
}

int64_t attend_workspace(AttendParams &p, char *base) {
    const int64_t heads = (int64_t)p.n_reqs * p.pool.H * p.G;
    int64_t at = 0;
    const auto take = [&](int64_t floats) {
        float *x = base ? reinterpret_cast<float *>(base + at) : nullptr;
        at += (floats * 4 + 15) / 16 * 16;
        return x;
    };
    // two parts a share, its first and its last
    const int64_t parts = 2 * (int64_t)p.shares * p.waves_k * p.part_heads;
    p.before = reinterpret_cast<int32_t *>(take(kAttendGroup + 1));
    p.lse2 = take(heads);
    p.part_ml = take(parts * 2);
    p.part_o = take(parts * p.Dv);
    p.scores = p.acc ? take(heads * p.score_stride) : nullptr;
    p.spare = p.acc ? take(64) : nullptr;
    return at;
}

int launch_attend_narrow(const AttendParams &p, int32_t r0, int32_t n, hipStream_t stream) {
    const auto kernel = p.acc ? pick<true>(p) : pick<false>(p);
    const int streams = p.waves_h * p.waves_k;
    const size_t lds = streams == kWaves ? 0 : sizeof(float) * streams * 16 * padded(p.pool.D);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.whole ? n * p.per : p.shares)), dim3(64 * kWaves), lds, stream, p, r0, n);
    return hipGetLastError();
}

int launch_attend(const AttendParams &p, hipStream_t stream) {
    // Threads of the second launch: many parts of few heads need many rows of them.
    const int threads = p.shares / (p.n_reqs < kAttendGroup ? p.n_reqs : kAttendGroup) / p.per >= 32 ? 1024 : 256;
    const int32_t runs = (p.max_tokens + kTile - 1 + 4 * threads - 1) / (4 * threads);
    for (int32_t r0 = 0; r0 < p.n_reqs; r0 += kAttendGroup) {
        const int32_t n = p.n_reqs - r0 < kAttendGroup ? p.n_reqs - r0 : kAttendGroup;
        int e = p.pool.D > 256 ? launch_attend_wide(p, r0, n, stream) : launch_attend_narrow(p, r0, n, stream);
        if (e != hipSuccess) return e;
        const int64_t joins = p.whole ? 0 : (int64_t)n * p.pool.H * p.G;
        const int64_t blocks = joins + (p.acc ? (int64_t)n * p.pool.H * runs : 0);
        for (int64_t at = 0; at < blocks; at += kMaxBlocks) {
            const int64_t some = blocks - at < kMaxBlocks ? blocks - at : kMaxBlocks;
            hipLaunchKernelGGL(p.f16 ? kvx_attend_finish_kernel<true> : kvx_attend_finish_kernel<false>,
                               dim3((uint32_t)some), dim3(threads), sizeof(float) * 5 * threads, stream, p, r0, n, at,
                               joins, runs);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace kvx
