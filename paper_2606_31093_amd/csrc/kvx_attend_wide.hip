// kvx_attend_wide.hip -- attention of one query per request over a paged cache
// whose rows have more than 256 elements (gfx950): MLA latents, with up to
// 128 query heads on one cache head.
//
// With 128 heads every byte of the cache takes part in 240 operations: at the
// rates of a large product and a large copy the matrix units would be as busy as
// the memory.  A wavefront takes 16 heads, so that
// a workgroup of eight reads a tile of positions once for 128; the tile lies
// in LDS, where the loads put it themselves (no register holds a row on its
// way).  They are asked for when the tile before is taken up, and have arrived
// before its first values are read: the compiler waits for all loads there, as
// the reads of LDS that transpose might meet what the loads write.  With c = lane % 16, e = lane / 16
// the products are those of the narrow kernel, of 16 x 16:
// - scores: A = 16 rows of K, B = the queries (registers, all their elements);
//   row r of product b < 2 is position 8 (r / 4) + 4 b + r % 4, so that lane (c, e)
//   gets the scores of head c at positions 8 e + 4 b + i, i < 4;
// - they are the A operand of the second product, whose k index is the position;
// - B = V, from LDS by the loads that transpose: 16 lanes give the addresses of
//   4 rows x 16 elements of 16 bits (8 x 16 of 8), lane c gets column c.
//
// LDS.  A row is cut into chunks of 16 bytes and padded to an odd multiple of 8 of
// them; chunk x of row r lies at place x ^ turn(r).  One chunk of the rows of a
// product (scores), two of 4 and one of 8 successive rows (values) then lie in
// different banks.  The loads write LDS in order of lanes; the permutation is in
// the addresses they read.
//
// Weights are in two parts, as in the narrow kernel, but for eight wavefronts: there
// they are rounded once to the rows' type.  With 128 heads the second product took 185 us
// instead of 167, for an error against 64 bits of 0.0017 instead of 0.0019 of the
// outputs, 0.0017 of it their own rounding to bfloat16.  With 64 heads it took none (142 for
// 150), with 16 and 32 1 to 3%, in half 11% with 16.
//
// 16 requests of 4096 to 32768 positions, 128 heads on rows of 576 (409 MB, 98
// GFLOP): 171 us, 571 TFLOP/s.  Bound by waits:
// the matrix units are busy for a quarter of the first launch, a wavefront waits for 43%
// of its cycles (for the next tile's loads, and for rows of K, which are read one
// product ahead).  Registers for more reads ahead there are none: the kernels of four and
// eight wavefronts, and of one with 16-bit rows, spill 29 to 52 a lane, none of them
// among the products.

#include "kvx_attend.h"

namespace kvx {
namespace {

constexpr int kSteps = 18;               // 32 elements each: rows of up to 576
constexpr int kTiles = 32;               // 16 values each: up to 512
// Turns that reads of K and of V are ahead of their products, and one (a read of K is
// asked for behind the product before, so that of depth 2 is one product ahead).  With four
// wavefronts and more two lie on a SIMD: a query, its outputs and these fill the
// 256 registers of each, and a turn more of K took a wait for all loads per tile (170 us
// became 182).  Fewer have twice the registers.
constexpr int k_depth(int waves) { return waves >= 4 ? 2 : 6; }
constexpr int v_depth(int waves) { return waves >= 4 ? 4 : 8; }

// A row's permutation of its chunks, in each 8 of them.
template <bool E4M3>
__device__ __forceinline__ int turn(int r) {
    return (r & 2) | ((r >> 1 ^ r >> 2) & 4) | (((E4M3 ? r >> 2 : 0) ^ r >> 4) & 1);
}

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) int s32x2;

// The transposing loads: column c of the 4 (8) rows that a lane's group of 16 gives
// the addresses of, 8 bytes a lane.
__device__ __forceinline__ u32x2 columns16(const char *at) {
    return bits<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)at));
}
__device__ __forceinline__ u32x2 columns8(const char *at) {
    return bits<u32x2>(__builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) s32x2 *)at));
}

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

// The lane, computed where it is used: the registers are full, and what is known
// not to change would be kept in memory.  Reading it back waits for all loads.
__device__ __forceinline__ int lane_again() {
    int zero = 0;
    asm volatile("" : "+s"(zero));
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
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
__global__ void __launch_bounds__(64 * WAVES, LATENT && WAVES >= 4 ? 2 : 1) kvx_attend_wide_kernel(AttendParams p, int32_t r0, int32_t n) {
    typedef Half<F16> V;
    constexpr int ES = E4M3 ? 1 : 2, TILE = tile_of(WAVES), HALVES = TILE / 32;
    constexpr bool PARTS = WAVES < 8;                    // weights in two parts
    constexpr int kKDepth = LATENT ? k_depth(WAVES) : 2, kVDepth = LATENT ? v_depth(WAVES) : 4;
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

    Walk walk(p, r0, n, before, blockIdx.x);
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
        const auto look = [&](uint32_t t0, int ln) {
            const uint32_t t = t0 + ln;
            const uint64_t idx = entry(t < end ? t : end - 1);
            return p.pool.pt[idx < (uint64_t)p.pool.pt_len ? idx : 0];
        };
        const auto resolve = [&](uint32_t t0, int32_t page, int64_t *to, int ln) {
            const uint32_t t = t0 + ln;
            const bool in = ln < TILE && t >= first && t < end;
            const uint32_t at = t < end ? t : end - 1;
            const bool known = entry(at) < (uint64_t)p.pool.pt_len;
            const bool ok = in && known && (uint32_t)page < (uint32_t)p.pool.N;
            if (in && !ok) bad |= known ? KVX_DERR_SRC_PAGE : KVX_DERR_PT_RANGE;
            const int64_t off = page * p.pool.s_p + (int64_t)(at - fd_div(p.pool.fd_T, at) * p.pool.fd_T.d) * p.pool.s_t;
            if (TILE == 64 || ln < TILE) to[ln] = ok ? off : 0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            return (uint64_t)__ballot(ok);
        };
        // This wavefront's loads of a tile: 1 KiB of it each, row by row.
        const auto load_tile = [&](const int64_t *off, char *tile, int ln) {
            const auto from = [&](int q) {
                const bool is_v = two && q >= TILE * row_chunks / 64;
                const uint32_t u = (is_v ? q - TILE * row_chunks / 64 : q) * 64 + ln;
                const uint32_t row = u / (uint32_t)row_chunks, x = (u - row * row_chunks) ^ turn<E4M3>(row);
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

        const int heads = p.G - g0 < 16 ? (p.G > g0 ? p.G - g0 : 0) : 16;     // of this wave
        u32x4 qv[kSteps];
        {
            const bool on = c < heads;
            const char *src = p.q.base + part.r * p.q.s_row + (int64_t)(h * p.G + (on ? g0 + c : 0)) * p.q.s_head;
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

        f32x4 o[kTiles];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        float m = -INFINITY, l = 0.f;
        float *scores = nullptr;
        if (ACC)
            scores = (c < heads ? p.scores + ((int64_t)part.r * p.pool.H * p.G + h * p.G + g0 + c) * p.score_stride -
                                      (rec.start & -kTile)
                                : p.spare) + 8 * e;

        uint64_t mask = resolve(begin, look(begin, lane), row_off[wave][0], lane);
        load_tile(row_off[wave][0], tiles, lane);
        int32_t page = look(begin + TILE, lane);
        int buf = 0;
        for (uint32_t t0 = begin; t0 < end; t0 += TILE) {
            // this tile is here, and nobody reads the one before it any more
            arrive<(WAVES > 1)>();
            char *tile = tiles + buf * tile_bytes;
            const int ln = lane_again(), lc = ln & 15, le = ln >> 4;
            buf ^= 1;
            const uint64_t next_mask = resolve(t0 + TILE, page, row_off[wave][buf], ln);
            page = look(t0 + 2 * TILE, ln);
            load_tile(row_off[wave][buf], tiles + buf * tile_bytes, ln);
            constexpr uint64_t ALL = TILE == 64 ? ~0ull : 0xffffffffull;
            if (mask != ALL) {
                // positions that take no part must not bring their NaN: zeros in their place
                uint32_t zero = 0;
                asm volatile("" : "+v"(zero));             // as above
#pragma unroll 1
                for (int at = (wave * 64 + ln) * 16; at < tile_bytes; at += 1024 * WAVES) {
                    if (!((mask >> (at / pitch & (TILE - 1))) & 1))
                        *reinterpret_cast<u32x4 *>(tile + at) = u32x4{zero, zero, zero, zero};
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (WAVES > 1) __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }

            // Addresses in LDS from a tile's begin: a lane's first chunk of its row of product
            // 0, and of its first row of values.
            const int k_row = 8 * (lc / 4) + lc % 4, v_row = 8 * le + (E4M3 ? lc / 2 : lc / 4);
            const int k_at = k_row * pitch + (le ^ turn<E4M3>(k_row)) * 16;
            const int v_at = v_rows + v_row * pitch + ((E4M3 ? 0 : lc % 4 / 2) ^ turn<E4M3>(v_row)) * 16 + lc % 2 * 8;
            // not unrolled: twice the code took registers that there are not
#pragma unroll 1
            for (int half = 0; half < HALVES; ++half) {
                f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
                // Product b's rows are 4 on; turn() takes that into account for 8 bits.
                // Rows are read kKDepth - 1 turns ahead of the products; left alone the
                // compiler would read all first, for which there are no registers.
                constexpr int WIDE = E4M3 ? 2 : 1, TURNS = kSteps / WIDE;         // steps a turn
                u32x4 k[kKDepth][2];
                const auto read_k = [&](int u) {
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        k[u % kKDepth][b] = *reinterpret_cast<const u32x4 *>(
                            tile + (k_at ^ (u % 2 * 64 + (E4M3 ? 16 * b : 0))) + (32 * half + 4 * b) * pitch + u / 2 * 128);
                };
#pragma unroll
                for (int u = 0; u < kKDepth - 1; ++u) read_k(u);
#pragma unroll
                for (int u = 0; u < TURNS; ++u) {
                    if (!LATENT && 32 * WIDE * u >= D) continue;
                    if (u + kKDepth - 1 < TURNS && (LATENT || 32 * WIDE * (u + kKDepth - 1) < D)) read_k(u + kKDepth - 1);
#pragma unroll
                    for (int i = 0; i < WIDE; ++i) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            u32x4 a = k[u % kKDepth][b];
                            if (E4M3) {
                                const uint32_t w[2] = {a[2 * i], a[2 * i + 1]};
                                a = widen<F16, true>(w);
                            }
                            if (!LATENT && (E4M3 ? (4 * u + le) * 16 : u * 32 + le * 8) >= D) a = u32x4{0, 0, 0, 0};
                            s[b] = V::mfma(a, qv[WIDE * u + i], s[b]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                // x[b][i]: the score of position 32 half + 8 e + 4 b + i
                f32x4 x[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) x[b] = s[b] * unit;
                if (mask != ALL) {
                    const uint32_t mine = (uint32_t)(mask >> (32 * half)) >> (8 * le);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (!((mine >> i) & 1)) x[i / 4][i % 4] = -INFINITY;
                }
                if (ACC) {
                    float *to = scores + (lc < heads ? t0 + 32 * half : 0);
                    *reinterpret_cast<f32x4 *>(to) = x[0];
                    *reinterpret_cast<f32x4 *>(to + (lc < heads ? 4 : 0)) = x[1];
                }
                float top = x[0][0];
#pragma unroll
                for (int i = 1; i < 8; ++i) top = fmaxf(top, x[i / 4][i % 4]);
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                if (__builtin_amdgcn_ballot_w64(top - kLift<F16> > m + kSlack) != 0) {
                    const float raised = fmaxf(m, top - kLift<F16>);
                    const float f = weight(m, raised);
                    m = raised;
                    l *= f;
                    f32x4 fr;
#pragma unroll
                    for (int i = 0; i < 4; ++i) fr[i] = __shfl(f, 4 * le + i);
#pragma unroll
                    for (int j = 0; j < kTiles; ++j) o[j] *= fr;
                }
                const float from = m == -INFINITY ? 0.f : m;       // then every x is -inf
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = exp2_fast(x[i / 4][i % 4] - from);
                    l += w[i];
                }
                u32x4 a = {V::pack(w[0], w[1]), V::pack(w[2], w[3]), V::pack(w[4], w[5]), V::pack(w[6], w[7])}, rest;
                if (PARTS) split<F16>(w, a, rest);
                // Values are read kVDepth - 1 turns ahead.  Successive turns' chunks are 8 apart,
                // in the same place of theirs.
                constexpr int STRIDE = E4M3 ? 8 : 4;               // tiles of 128 bytes
                u32x4 v[kVDepth];
                const auto tile_of_turn = [&](int u) { return u % (kTiles / STRIDE) * STRIDE + u / (kTiles / STRIDE); };
                const auto read_v = [&](int u) {
                    const int j = tile_of_turn(u), far = 32 * half * pitch + j / STRIDE * 128;
                    if (!LATENT && 16 * j >= Dv) return;
                    if (E4M3) {
                        const u32x2 y = columns8(tile + (v_at ^ j % STRIDE * 16) + far);
                        v[u % kVDepth] = u32x4{y[0], y[1], 0, 0};
                    } else {
                        const u32x2 y = columns16(tile + (v_at ^ j % STRIDE * 32) + far);
                        const u32x2 z = columns16(tile + (v_at ^ j % STRIDE * 32) + far + 4 * pitch);
                        v[u % kVDepth] = u32x4{y[0], y[1], z[0], z[1]};
                    }
                };
#pragma unroll
                for (int u = 0; u < kVDepth - 1; ++u) read_v(u);
#pragma unroll
                for (int u = 0; u < kTiles; ++u) {
                    if (u + kVDepth - 1 < kTiles) read_v(u + kVDepth - 1);
                    if (!LATENT && 16 * tile_of_turn(u) >= Dv) continue;
                    u32x4 bv = v[u % kVDepth];
                    if (E4M3) {
                        const uint32_t w[2] = {bv[0], bv[1]};
                        bv = widen<F16, true>(w);
                    }
                    o[tile_of_turn(u)] = V::mfma(a, bv, o[tile_of_turn(u)]);
                    if (PARTS) o[tile_of_turn(u)] = V::mfma(rest, bv, o[tile_of_turn(u)]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            mask = next_mask;
        }
        if (bad && p.err) atomicOr(p.err, bad);
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);

        const int64_t head0 = (int64_t)part.r * p.pool.H * p.G + h * p.G + g0;
        const int64_t part0 = part.place < 0 ? 0 : part.place * p.part_heads + wave * 16;
        if (e == 0 && c < heads) {
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
            for (int j = 0; j < kTiles; ++j) {
                const int d = j * 16 + c;
                if (!LATENT && d >= Dv) continue;
                if (part.place < 0) reinterpret_cast<uint16_t *>(dst)[d] = V::pack(o[j][i] * f, 0.f);
                else po[d] = o[j][i];
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
    // For latents as many as a compute unit's LDS and registers hold, else one: for workgroups of
    // one wavefront more would serve (rows of 320, 4 heads, 110 MB: 164 us, 95 with all that fit;
    // of 448, 16 heads, 155 MB: 194, 127), for those of four not (rows of 320, 40 heads: 136, 162).
    // Latents by the kernel for any rows take 405 us instead of 130 with 16 heads, 560 instead
    // of 167 with 128.
    const int fit = 150 * 1024 / lds_of(p), waves = 8 / p.waves_h;
    p.shares = 256 * (!latent(p) ? 1 : fit < waves ? fit : waves);
}

int launch_attend_wide(const AttendParams &p, int32_t r0, int32_t n, hipStream_t stream) {
    const auto kernel = p.acc ? pick<true>(p) : pick<false>(p);
    const int64_t blocks = p.whole ? (int64_t)n * p.per : p.shares;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(64 * p.waves_h), lds_of(p), stream, p, r0, n);
    return hipGetLastError();
}

}  // namespace kvx
