// kvx_attend_wide.hip -- attention of one query per request over a paged cache
// whose rows have more than 256 elements (gfx950): MLA latents, with up to
// 128 query heads on one cache head.
//
// With 128 heads every byte of the cache takes part in 240 operations: the
// matrix units are as busy as the memory.  A wavefront takes 16 heads, so that
// a workgroup of eight reads a tile of positions once for 128; the tile lies
// in LDS, where the loads put it themselves (no register holds a row on its
// way), while the one before it is in use.  With c = lane % 16, e = lane / 16
// the products are those of the narrow kernel, of 16 x 16:
// - scores: A = 16 rows of K, B = the queries (registers, all their elements);
//   lane (c, e) gets the scores of head c at positions 4 e + i, i < 4;
// - those of 32 positions are the A operand of the second product, if its k
//   index 8 e + i stands for position 16 (i / 4) + 4 e + i % 4;
// - B = V: lane (c, e) reads 8 elements from (16 nb + c) * 8 on of those 8
//   positions and transposes its 8 x 8 block with byte permutes.
//
// LDS.  A row is cut into chunks of 16 bytes and padded to an odd multiple of 8 of
// them; chunk x of row r lies at place x ^ (r / 2 % 8), so that one chunk of 16
// rows (scores) and 16 chunks of a row (values) each lie in all 64 banks.
// The loads write LDS in order of lanes; the permutation is in the addresses
// they read.

#include "kvx_attend.h"

namespace kvx {
namespace {

constexpr int kSteps = 18;               // 32 elements each: rows of up to 576

constexpr int kBlocks = 2;                // values of a workgroup, 128 each

// Bytes of a row in LDS.
__host__ __device__ inline int pitch_of(int elems, bool e4m3) { return ((elems * (e4m3 ? 1 : 2) + 127) / 128 | 1) * 128; }

// Positions of a tile: two of them lie in a compute unit's LDS, once for eight
// wavefronts or twice for up to four.
constexpr int tile_of(int waves) { return waves == 8 ? 64 : 32; }

// 16 bytes a lane to LDS, in order of lanes from `to` on.
__device__ __forceinline__ void load_lds(const char *from, char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// This wavefront's memory operations are done, and the workgroup's other
// wavefronts are here too.
template <bool BARRIER>
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xf70);                   // vmcnt(0)
    if (BARRIER) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// WAVES: of a workgroup, 16 heads each.  LATENT: rows of 576 elements, values
// their first 512; else any head_dim up to 576, values up to 512, in rows of
// their own if num_kv is 2.
template <bool F16, bool E4M3, int WAVES, bool LATENT, bool ACC>
__global__ void __launch_bounds__(64 * WAVES, LATENT ? 2 : 1) kvx_attend_wide_kernel(AttendParams p, int32_t r0, int32_t n) {
    typedef Half<F16> V;
    constexpr int ES = E4M3 ? 1 : 2, TILE = tile_of(WAVES), HALVES = TILE / 32;
    __shared__ int32_t before[kAttendGroup + 1];
    __shared__ __align__(16) int64_t row_off[WAVES][2][TILE];
    extern __shared__ __align__(256) char tiles[];       // [2][rows of K, rows of V if num_kv is 2]

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int c = lane & 15, e = lane >> 4;
    const int D = LATENT ? 576 : p.pool.D, Dv = LATENT ? 512 : p.Dv;
    const bool two = !LATENT && p.pool.C == 2;
    const int pitch = LATENT ? (E4M3 ? 640 : 1152) : pitch_of(D, E4M3), row_chunks = pitch / 16, chunks = ES * D / 16;
    const int v_rows = two ? TILE * pitch : 0, tile_bytes = TILE * pitch + v_rows;
    constexpr int LATENT_LOADS = (E4M3 ? 640 : 1152) * TILE / 1024 / WAVES;
    const int loads = LATENT ? LATENT_LOADS : tile_bytes / 1024 / WAVES;      // a wavefront's, of a tile

    // Two workgroups share a unit's values where they are more than 256: one takes
    // the first 256, one the others.  They lie 8 apart, on one XCD, and the second
    // finds the rows in its cache.
    const int vb = p.v_blocks == 2 ? (int)(blockIdx.x / 8 % 2) : 0, v0 = 256 * vb;
    const int id = p.v_blocks == 2 ? (int)(blockIdx.x / 16 * 8 + blockIdx.x % 8) : (int)blockIdx.x;
    if (vb) p.err = nullptr;                             // the first one reports
    // Addresses in LDS from a tile's begin.  Scores: chunk 4 j + e of row c, for
    // j % 2 = i; values: this lane's first chunk of rows 4 e + 2 i and 4 e + 2 i + 1
    // (the second a pitch behind).
    int k_at[2], v_at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        k_at[i] = c * pitch + ((4 * i + e) ^ (c >> 1)) * 16;
        const int s = (2 * e + i) & 7;
        v_at[i] = v_rows + (4 * e + 2 * i) * pitch + v0 * ES + (E4M3 ? ((c >> 1) ^ s) * 16 + (c & 1) * 8 : (c ^ s) * 16);
    }

    Walk walk(p, r0, n, before, id);
    Part part;
    while (walk.next(p, before, &part)) {
        const kvx_attend_req rec = part.rec;
        const int h = part.hb / p.head_blocks, g0 = (part.hb % p.head_blocks * WAVES + wave) * 16;
        const uint32_t begin = __builtin_amdgcn_readfirstlane(part.begin), end = __builtin_amdgcn_readfirstlane(part.end);
        const uint32_t first = rec.start;
        const char *kbase = p.pool.base + h * p.pool.s_h;

        // A lane resolves position t0 + lane: its page id, and later the row offset.
        uint32_t bad = 0;
        const auto entry = [&](uint32_t t) { return (uint64_t)rec.pt_off + fd_div(p.pool.fd_T, t); };
        const auto look = [&](uint32_t t0) {
            const uint32_t t = t0 + lane;
            const uint64_t idx = entry(t < end ? t : end - 1);
            return p.pool.pt[idx < (uint64_t)p.pool.pt_len ? idx : 0];
        };
        const auto resolve = [&](uint32_t t0, int32_t page, int64_t *to) {
            const uint32_t t = t0 + lane;
            const bool in = lane < TILE && t >= first && t < end;
            const uint32_t at = t < end ? t : end - 1;
            const bool known = entry(at) < (uint64_t)p.pool.pt_len;
            const bool ok = in && known && (uint32_t)page < (uint32_t)p.pool.N;
            if (in && !ok) bad |= known ? KVX_DERR_SRC_PAGE : KVX_DERR_PT_RANGE;
            const int64_t off = page * p.pool.s_p + (int64_t)(at - fd_div(p.pool.fd_T, at) * p.pool.fd_T.d) * p.pool.s_t;
            if (TILE == 64 || lane < TILE) to[lane] = ok ? off : 0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            return (uint64_t)__ballot(ok);
        };
        // This wavefront's loads of a tile: 1 KiB of it each, row by row.
        const auto load_tile = [&](const int64_t *off, char *tile) {
            // Not known to be the same in every turn, so that what follows from it is
            // computed again instead of kept in registers.
            int ln = lane;
            asm volatile("" : "+v"(ln));
            const auto from = [&](int q) {
                const bool is_v = two && q >= TILE * row_chunks / 64;
                const uint32_t u = (is_v ? q - TILE * row_chunks / 64 : q) * 64 + ln;
                const uint32_t row = u / (uint32_t)row_chunks, x = (u - row * row_chunks) ^ (row / 2 & 7);
                return kbase + off[row] + 16 * ((int)x < chunks ? x : 0) + (is_v ? p.pool.s_c : 0);
            };
            if (LATENT) {
                // addresses first, some at a time: each load to LDS might write the offsets,
                // for all the compiler knows, and would wait for the reads of the next one's
                constexpr int SOME = LATENT_LOADS % 9 == 0 ? 9 : LATENT_LOADS % 5 == 0 ? 5 : 1;
#pragma unroll
                for (int t0 = 0; t0 < LATENT_LOADS; t0 += SOME) {
                    const char *at[SOME];
#pragma unroll
                    for (int t = 0; t < SOME; ++t) at[t] = from(wave * LATENT_LOADS + t0 + t);
#pragma unroll
                    for (int t = 0; t < SOME; ++t) load_lds(at[t], tile + (wave * LATENT_LOADS + t0 + t) * 1024);
                }
            } else {
                for (int t = 0; t < loads; ++t) load_lds(from(wave * loads + t), tile + (wave * loads + t) * 1024);
            }
        };

        // Heads of this wave.  Where they are 8 or fewer, bfloat16 weights take two
        // columns: head c in column c, and in column c + 8 what its rounding left.
        const int heads = p.G - g0 < 16 ? (p.G > g0 ? p.G - g0 : 0) : 16;
        const bool twice = !F16 && heads <= 8;
        u32x4 qv[kSteps];
        {
            const int g = twice ? c & 7 : c;
            const bool on = g < heads;
            const char *src = p.q.base + part.r * p.q.s_row + (int64_t)(h * p.G + (on ? g0 + g : 0)) * p.q.s_head;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int d = E4M3 ? (j / 2 * 4 + e) * 16 + j % 2 * 8 : j * 32 + e * 8;
                qv[j] = *reinterpret_cast<const u32x4 *>(src + 2 * (LATENT || d < D ? d : 0));
                if (!on || (!LATENT && d >= D)) qv[j] = u32x4{0, 0, 0, 0};
            }
        }
        const float k_scale = p.scales ? p.scales[h] : 1.f;
        const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
        const float unit = p.scale_log2 * k_scale;

        f32x4 o[kBlocks][8];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int j = 0; j < 8; ++j) o[b][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        float *scores = nullptr;
        if (ACC)
            scores = (c < heads ? p.scores + ((int64_t)part.r * p.pool.H * p.G + h * p.G + g0 + c) * p.score_stride -
                                      (rec.start & -kTile)
                                : p.spare) + 4 * e;

        uint64_t mask = resolve(begin, look(begin), row_off[wave][0]);
        load_tile(row_off[wave][0], tiles);
        int32_t page = look(begin + TILE);
        int buf = 0;
        for (uint32_t t0 = begin; t0 < end; t0 += TILE) {
            // this tile is here, and nobody reads the one before it any more
            arrive<(WAVES > 1)>();
            char *tile = tiles + buf * tile_bytes;
            buf ^= 1;
            const uint64_t next_mask = resolve(t0 + TILE, page, row_off[wave][buf]);
            page = look(t0 + 2 * TILE);
            load_tile(row_off[wave][buf], tiles + buf * tile_bytes);
            constexpr uint64_t ALL = TILE == 64 ? ~0ull : 0xffffffffull;
            if (mask != ALL) {
                // positions that take no part must not bring their NaN: zeros in their place
                int th = threadIdx.x * 16;
                asm volatile("" : "+v"(th));               // as above
#pragma unroll 1
                for (int at = th; at < tile_bytes; at += 1024 * WAVES) {
                    if (!((mask >> (at / pitch & (TILE - 1))) & 1)) *reinterpret_cast<u32x4 *>(tile + at) = u32x4{0, 0, 0, 0};
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (WAVES > 1) __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }

            // x[b][i]: the score of position 16 b + 4 e + i
            f32x4 x[2 * HALVES];
#pragma unroll
            for (int half = 0; half < HALVES; ++half) {
                f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
                // A pair of steps is read ahead of the one in use; left alone the
                // compiler would read all first, for which there are no registers.
                u32x4 k[2][2][2];
                const auto read_k = [&](int j0, u32x4 (*to)[2]) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const char *row = tile + (32 * half + 16 * b) * pitch;
                        if (E4M3) {
                            to[0][b] = *reinterpret_cast<const u32x4 *>(row + k_at[j0 / 2 % 2] + j0 / 4 * 128);
                        } else {
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                to[i][b] = *reinterpret_cast<const u32x4 *>(row + k_at[i] + j0 / 2 * 128);
                        }
                    }
                };
                read_k(0, k[0]);
#pragma unroll
                for (int j0 = 0; j0 < kSteps; j0 += 2) {
                    if (!LATENT && 32 * j0 >= D) continue;
                    if (j0 + 2 < kSteps && (LATENT || 32 * j0 + 64 < D)) read_k(j0 + 2, k[j0 / 2 % 2 ^ 1]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int j = j0 + i;
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            u32x4 a = k[j0 / 2 % 2][E4M3 ? 0 : i][b];
                            if (E4M3) {
                                const uint32_t w[2] = {a[2 * i], a[2 * i + 1]};
                                a = widen<F16, true>(w);
                            }
                            if (!LATENT && (E4M3 ? (j / 2 * 4 + e) * 16 : j * 32 + e * 8) >= D) a = u32x4{0, 0, 0, 0};
                            s[b] = V::mfma(a, qv[j], s[b]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int b = 0; b < 2; ++b) x[2 * half + b] = s[b] * unit;
            }
            if (mask != ALL) {
                const uint64_t mine = mask >> (4 * e);
#pragma unroll
                for (int b = 0; b < 2 * HALVES; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!((mine >> (16 * b + i)) & 1)) x[b][i] = -INFINITY;
            }
            mask = next_mask;
            if (ACC && vb == 0) {
                float *to = scores + (c < heads ? t0 : 0);
#pragma unroll
                for (int b = 0; b < 2 * HALVES; ++b) *reinterpret_cast<f32x4 *>(to + (c < heads ? 16 * b : 0)) = x[b];
            }
            float top = x[0][0];
#pragma unroll
            for (int i = 1; i < 8 * HALVES; ++i) top = fmaxf(top, x[i / 4][i % 4]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__builtin_amdgcn_ballot_w64(top - kLift<F16> > m + kSlack) != 0) {
                const float raised = fmaxf(m, top - kLift<F16>);
                const float f = weight(m, raised);
                m = raised;
                l *= f;
                f32x4 fr;
#pragma unroll
                for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * e + i);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[b][j] *= fr;
            }
            const float from = m == -INFINITY ? 0.f : m;       // then every x is -inf
            u32x4 a[HALVES];
#pragma unroll
            for (int half = 0; half < HALVES; ++half) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = exp2_fast(x[2 * half + i / 4][i % 4] - from);
                    l += w[i];
                }
                a[half] = u32x4{V::pack(w[0], w[1]), V::pack(w[2], w[3]), V::pack(w[4], w[5]), V::pack(w[6], w[7])};
                if (twice && c >= 8) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[half][i] = V::pack(w[2 * i] - V::lo(a[half][i]), w[2 * i + 1] - V::hi(a[half][i]));
                }
            }
#pragma unroll
            for (int half = 0; half < HALVES; ++half) {
#pragma unroll
                for (int nb = 0; nb < kBlocks; ++nb) {
                    uint32_t v[8][4];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const char *at = tile + v_at[i / 2 % 2] + (32 * half + 16 * (i / 4) + i % 2) * pitch + nb * 128 * ES;
                        u32x4 y;
                        if (E4M3) {
                            const u32x2 z = *reinterpret_cast<const u32x2 *>(at);
                            const uint32_t zw[2] = {z[0], z[1]};
                            y = widen<F16, true>(zw);
                        } else {
                            y = *reinterpret_cast<const u32x4 *>(at);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[i][k] = !LATENT && v0 + nb * 128 + c * 8 >= Dv ? 0 : y[k];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;
                        u32x4 bv;
#pragma unroll
                        for (int k = 0; k < 4; ++k) bv[k] = __builtin_amdgcn_perm(v[2 * k + 1][j / 2], v[2 * k][j / 2], pick);
                        o[nb][j] = V::mfma(a[half], bv, o[nb][j]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        if (bad && p.err) atomicOr(p.err, bad);
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        if (twice) {
            // row 4 e + i, its rest 8 rows on: of lane + 32; see the narrow kernel
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float rest = __shfl_xor(o[b][j][i], 32);
                        if (__builtin_fabsf(o[b][j][i]) < INFINITY) o[b][j][i] += rest;
                    }
        }

        const int64_t head0 = (int64_t)part.r * p.pool.H * p.G + h * p.G + g0;
        const int64_t part0 = part.place < 0 ? 0 : part.place * p.part_heads + wave * 16;
        if (vb == 0 && e == 0 && c < heads) {
            if (part.place < 0) {
                const float x = l > 0.f || l != l ? m + __builtin_amdgcn_logf(l) : -INFINITY;
                if (p.lse) p.lse[head0 + c] = x * kLn2;
                p.lse2[head0 + c] = x;
            } else {
                p.part_ml[(part0 + c) * 2] = m;
                p.part_ml[(part0 + c) * 2 + 1] = l;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 4 * e + i;
            const float lr = __shfl(l, row);
            if (row >= heads) continue;
            const float f = part.place >= 0 ? 1.f : lr == 0.f ? 0.f : v_scale / lr;
            char *dst = p.out.base + part.r * p.out.s_row + (int64_t)(h * p.G + g0 + row) * p.out.s_head;
            float *po = p.part_o + (part0 + row) * Dv;
#pragma unroll
            for (int nb = 0; nb < kBlocks; ++nb) {
                const int d = v0 + nb * 128 + c * 8;
                if (!LATENT && d >= Dv) continue;
                const f32x4 *y = o[nb];
                if (part.place < 0) {
                    *reinterpret_cast<u32x4 *>(dst + 2 * d) =
                        u32x4{V::pack(y[0][i] * f, y[1][i] * f), V::pack(y[2][i] * f, y[3][i] * f),
                              V::pack(y[4][i] * f, y[5][i] * f), V::pack(y[6][i] * f, y[7][i] * f)};
                } else {
                    *reinterpret_cast<f32x4 *>(po + d) = f32x4{y[0][i], y[1][i], y[2][i], y[3][i]};
                    *reinterpret_cast<f32x4 *>(po + d + 4) = f32x4{y[4][i], y[5][i], y[6][i], y[7][i]};
                }
            }
        }
        // the loads behind the last tile, before LDS is used again
        arrive<(WAVES > 1)>();
    }
}

bool latent(const AttendParams &p) { return p.pool.C == 1 && p.pool.D == 576 && p.Dv == 512; }

template <bool F16, bool E4M3, bool ACC>
auto pick(const AttendParams &p) {
    if (!latent(p))
        return p.waves_h == 1 ? kvx_attend_wide_kernel<F16, E4M3, 1, false, ACC> : kvx_attend_wide_kernel<F16, E4M3, 4, false, ACC>;
    if (p.waves_h == 1) return kvx_attend_wide_kernel<F16, E4M3, 1, true, ACC>;
    if (p.waves_h == 2) return kvx_attend_wide_kernel<F16, E4M3, 2, true, ACC>;
    if (p.waves_h == 4) return kvx_attend_wide_kernel<F16, E4M3, 4, true, ACC>;
    return kvx_attend_wide_kernel<F16, E4M3, 8, true, ACC>;
}

template <bool ACC>
auto pick(const AttendParams &p) {
    return p.f16 ? (p.e4m3 ? pick<true, true, ACC>(p) : pick<true, false, ACC>(p))
                 : (p.e4m3 ? pick<false, true, ACC>(p) : pick<false, false, ACC>(p));
}

int lds_of(const AttendParams &p) {
    return 2 * tile_of(p.waves_h) * pitch_of(p.pool.D, p.e4m3) * (p.pool.C == 2 ? 2 : 1);
}

}  // namespace

void plan_attend_wide(AttendParams &p) {
    const int tiles = (p.G + 15) / 16;
    p.waves_k = 1;
    if (latent(p)) p.waves_h = tiles <= 2 ? tiles : tiles <= 4 ? 4 : 8;
    else p.waves_h = tiles == 1 ? 1 : 4;
    p.span = 16 * p.waves_h;
    p.head_blocks = (tiles + p.waves_h - 1) / p.waves_h;
    p.step = tile_of(p.waves_h);
    p.v_blocks = p.Dv > 256 ? 2 : 1;
    // as many as a compute unit's LDS and registers hold
    const int fit = 150 * 1024 / lds_of(p), waves = 8 / p.waves_h;
    p.shares = 256 * (!latent(p) ? 1 : fit < waves ? fit : waves) / p.v_blocks;
}

int launch_attend_wide(const AttendParams &p, int32_t r0, int32_t n, hipStream_t stream) {
    const auto kernel = p.acc ? pick<true>(p) : pick<false>(p);
    const int64_t blocks = p.whole ? (int64_t)n * p.per : p.shares;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.v_blocks == 2 ? (blocks + 7) / 8 * 16 : blocks)), dim3(64 * p.waves_h), lds_of(p), stream, p, r0, n);
    return hipGetLastError();
}

}  // namespace kvx
