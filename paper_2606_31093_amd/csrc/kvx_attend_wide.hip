// kvx_attend_wide.hip -- attention of one query per request over a paged cache
// whose rows have more than 256 elements (gfx950): MLA latents, with up to
// 128 query heads on one cache head.
//
// With 128 heads every byte of the cache takes part in 240 operations: the
// matrix units are as busy as the memory.  A wavefront takes 32 heads, so that
// a workgroup of four reads a tile of 32 positions once for 128; the tile lies
// in LDS, where the loads put it themselves (no register holds a row on its
// way), one or two tiles ahead of the one in use.  With c = lane % 32, e = lane /
// 32 the products are those of the narrow kernel, of 32 x 32:
// - scores: A = 32 rows of K, B = the queries (registers, all their elements);
//   lane (c, e) gets the scores of head c at positions 8 g + 4 e + i, i, g < 4;
// - these are the A operand of the second product, 16 positions at a time, if
//   its k index 8 e + i stands for position 16 s + 8 (i / 4) + 4 e + i % 4;
// - B = V: lane (c, e) reads 8 elements from (32 nb + c) * 8 on of those 8
//   positions and transposes its 8 x 8 block with byte permutes.
// Each wavefront reads the tile from LDS twice (once as K, once as V): with 32
// heads that takes LDS about as long as the products take (2200 cycles a tile);
// with 16 heads it would take twice that.  The outputs of 32 heads x 512 fill
// half of the registers, so a compute unit holds one workgroup of four waves.
//
// LDS.  A row is cut into chunks of 16 bytes and padded to a multiple of 8 of
// them; chunk x of row r lies at place x ^ (r % 8), so that 8 rows' chunk x
// (scores) and a row's 8 chunks (values) each lie in 8 different banks groups.
// The loads write LDS in order of lanes; the permutation is in the addresses
// they read.

#include "kvx_attend.h"

namespace kvx {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kSteps = 36;               // 16 elements each: rows of up to 576
constexpr int kOuts = 8;                 // outputs: 256 elements, 8 a lane

template <bool F16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(bits<f16x8>(a), bits<f16x8>(b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bits<bf16x8>(a), bits<bf16x8>(b), c, 0, 0, 0);
}

// Bytes of a row in LDS.
__host__ __device__ inline int pitch_of(int elems, bool e4m3) { return (elems * (e4m3 ? 1 : 2) + 127) / 128 * 128; }

// 16 bytes a lane to LDS, in order of lanes from `to` on.
__device__ __forceinline__ void load_lds(const char *from, char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// All but the NEWER newest of this wavefront's memory operations are done, and
// the workgroup's other wavefronts are here too.  (A barrier with its fence
// would wait for every load.)
template <int NEWER, bool BARRIER>
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xf70 | (NEWER & 15) | (NEWER >> 4 << 14));
    if (BARRIER) __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// WAVES: of a workgroup, 32 heads each.  BUFS: tiles in LDS.  LATENT: rows of 576
// elements, values their first 512; else any head_dim up to 576, values up to
// 512, in rows of their own if num_kv is 2.
template <bool F16, bool E4M3, int WAVES, int BUFS, bool LATENT, bool ACC>
__global__ void __launch_bounds__(64 * WAVES) kvx_attend_wide_kernel(AttendParams p, int32_t r0, int32_t n) {
    typedef Half<F16> V;
    constexpr int ES = E4M3 ? 1 : 2;
    __shared__ int32_t before[kAttendGroup + 1];
    __shared__ __align__(16) int64_t row_off[WAVES][2][64];
    extern __shared__ __align__(128) char tiles[];       // [BUFS][rows of K, rows of V if num_kv is 2]

    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int c = lane & 31, e = lane >> 5;
    const int D = LATENT ? 576 : p.pool.D, Dv = LATENT ? 512 : p.Dv;
    const bool two = !LATENT && p.pool.C == 2;
    const int pitch = pitch_of(D, E4M3), row_chunks = pitch / 16, chunks = ES * D / 16;
    const int v_rows = two ? 32 * pitch : 0, tile_bytes = 32 * pitch + v_rows;
    constexpr int LATENT_LOADS = (E4M3 ? 640 : 1152) / 32 / WAVES;
    const int loads = LATENT ? LATENT_LOADS : tile_bytes / 1024 / WAVES;      // a wavefront's, of a tile

    // Two workgroups share a unit's values where they are more than 256: one takes
    // the first 256, one the others.  They lie 8 apart, on one XCD, and the second
    // finds the rows in its cache.
    const int vb = p.v_blocks == 2 ? (int)(blockIdx.x / 8 % 2) : 0;
    const int id = p.v_blocks == 2 ? (int)(blockIdx.x / 16 * 8 + blockIdx.x % 8) : (int)blockIdx.x;
    if (vb) p.err = nullptr;                             // the first one reports
    // Addresses in LDS from a tile's begin.  Scores: chunk 2 j + e of row c, for
    // j % 4 = i; values: this lane's chunk of row 4 e + i.
    int k_at[4], v_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k_at[i] = c * pitch + ((2 * i + e) ^ (c & 7)) * 16;
        const int row = 4 * e + i;
        v_at[i] = v_rows + row * pitch + vb * 256 * ES + (E4M3 ? ((c >> 1) ^ row) * 16 + (c & 1) * 8 : (c ^ row) * 16);
    }

    Walk walk(p, r0, n, before, id);
    Part part;
    while (walk.next(p, before, &part)) {
        const kvx_attend_req rec = part.rec;
        const int h = part.hb / p.head_blocks, g0 = (part.hb % p.head_blocks * WAVES + wave) * 32;
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
            const bool in = lane < 32 && t >= first && t < end;
            const uint32_t at = t < end ? t : end - 1;
            const bool known = entry(at) < (uint64_t)p.pool.pt_len;
            const bool ok = in && known && (uint32_t)page < (uint32_t)p.pool.N;
            if (in && !ok) bad |= known ? KVX_DERR_SRC_PAGE : KVX_DERR_PT_RANGE;
            const int64_t off = page * p.pool.s_p + (int64_t)(at - fd_div(p.pool.fd_T, at) * p.pool.fd_T.d) * p.pool.s_t;
            to[lane] = ok ? off : 0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            return (uint32_t)__ballot(ok);
        };
        // This wavefront's loads of a tile: 1 KiB of it each, row by row.
        const auto load_tile = [&](const int64_t *off, char *tile) {
            // Not known to be the same in every turn, so that what follows from it is
            // computed again instead of kept in registers.
            int ln = lane;
            asm volatile("" : "+v"(ln));
            const auto from = [&](int q) {
                const bool is_v = two && q >= row_chunks / 2;
                const uint32_t u = (is_v ? q - row_chunks / 2 : q) * 64 + ln;
                const uint32_t row = u / (uint32_t)row_chunks, x = (u - row * row_chunks) ^ (row & 7);
                return kbase + off[row] + 16 * ((int)x < chunks ? x : 0) + (is_v ? p.pool.s_c : 0);
            };
            if (LATENT) {
                // addresses first: each load to LDS might write the offsets, for all the
                // compiler knows, and would wait for the reads of the next one's
                const char *at[LATENT_LOADS];
#pragma unroll
                for (int t = 0; t < LATENT_LOADS; ++t) at[t] = from(wave * LATENT_LOADS + t);
#pragma unroll
                for (int t = 0; t < LATENT_LOADS; ++t) load_lds(at[t], tile + (wave * LATENT_LOADS + t) * 1024);
            } else {
                for (int t = 0; t < loads; ++t) load_lds(from(wave * loads + t), tile + (wave * loads + t) * 1024);
            }
        };

        // Heads of this wave.  Where they are 16 or fewer, bfloat16 weights take two
        // columns: head c in column c, and in column c + 16 what its rounding left.
        const int heads = p.G - g0 < 32 ? (p.G > g0 ? p.G - g0 : 0) : 32;
        const bool twice = !F16 && heads <= 16;
        u32x4 qv[kSteps];
        {
            const int g = twice ? c & 15 : c;
            const bool on = g < heads;
            const char *src = p.q.base + part.r * p.q.s_row + (int64_t)(h * p.G + (on ? g0 + g : 0)) * p.q.s_head;
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
                const int d = E4M3 ? (j / 2 * 2 + e) * 16 + j % 2 * 8 : j * 16 + e * 8;
                qv[j] = *reinterpret_cast<const u32x4 *>(src + 2 * (LATENT || d < D ? d : 0));
                if (!on || (!LATENT && d >= D)) qv[j] = u32x4{0, 0, 0, 0};
            }
        }
        const float k_scale = p.scales ? p.scales[h] : 1.f;
        const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
        const float unit = p.scale_log2 * k_scale;

        f32x16 o[kOuts];
#pragma unroll
        for (int j = 0; j < kOuts; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
        float m = -INFINITY, l = 0.f;
        float *scores = nullptr;
        if (ACC)
            scores = (c < heads ? p.scores + ((int64_t)part.r * p.pool.H * p.G + h * p.G + g0 + c) * p.score_stride -
                                      (rec.start & -kTile)
                                : p.spare) + 4 * e;

        // Tiles in flight: the one in use and BUFS - 1 behind it.
        uint32_t masks[BUFS];
#pragma unroll
        for (int k = 0; k < BUFS - 1; ++k) {
            masks[k] = resolve(begin + 32 * k, look(begin + 32 * k), row_off[wave][k & 1]);
            load_tile(row_off[wave][k & 1], tiles + k * tile_bytes);
        }
        int32_t page = look(begin + 32 * (BUFS - 1));
        int buf = 0, turn = (BUFS - 1) & 1;
        for (uint32_t t0 = begin; t0 < end; t0 += 32) {
            // this tile is here, and nobody reads the one before it any more
            arrive<(BUFS - 2) * LATENT_LOADS, (WAVES > 1)>();
            {
                const uint32_t t = t0 + 32 * (BUFS - 1);
                const int free = buf == 0 ? BUFS - 1 : buf - 1;
                masks[BUFS - 1] = resolve(t, page, row_off[wave][turn]);
                page = look(t + 32);
                load_tile(row_off[wave][turn], tiles + free * tile_bytes);
                turn ^= 1;
            }
            const uint32_t mask = masks[0];
            char *tile = tiles + buf * tile_bytes;
            if (mask != 0xffffffffu) {
                // positions that take no part must not bring their NaN: zeros in their place
                const u32x4 zero = {0, 0, 0, 0};
                int th = threadIdx.x * 16;
                asm volatile("" : "+v"(th));               // as above
#pragma unroll 1
                for (int at = th; at < tile_bytes; at += 1024 * WAVES) {
                    if (!((mask >> (at / pitch & 31)) & 1)) *reinterpret_cast<u32x4 *>(tile + at) = zero;
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if (WAVES > 1) __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }

            // x[i]: the score of position 8 (i / 4) + 4 e + i % 4
            f32x16 s;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = 0.f;
            // Four steps' rows are read ahead of the four in use; left alone the
            // compiler would read all 36 first, for which there are no registers.
            u32x4 k[2][4];
            const auto read_k = [&](int j0, u32x4 *to) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + i;
                    if (E4M3) {
                        const uint32_t *w = reinterpret_cast<const uint32_t *>(tile + k_at[j / 2 % 4] + j / 8 * 128) + j % 2 * 2;
                        to[i] = u32x4{w[0], w[1], 0, 0};
                    } else {
                        to[i] = *reinterpret_cast<const u32x4 *>(tile + k_at[j % 4] + j / 4 * 128);
                    }
                }
            };
            read_k(0, k[0]);
#pragma unroll
            for (int j0 = 0; j0 < kSteps; j0 += 4) {
                if (!LATENT && 16 * j0 >= D) continue;
                if (j0 + 4 < kSteps) read_k(j0 + 4, k[j0 / 4 % 2 ^ 1]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = j0 + i;
                    u32x4 a = k[j0 / 4 % 2][i];
                    if (E4M3) {
                        const uint32_t w[2] = {a[0], a[1]};
                        a = widen<F16, true>(w);
                    }
                    if (!LATENT && (E4M3 ? (j / 2 * 2 + e) * 16 : j * 16 + e * 8) >= D) a = u32x4{0, 0, 0, 0};
                    s = mfma32<F16>(a, qv[j], s);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = s[i] * unit;
            if (mask != 0xffffffffu) {
                const uint32_t mine = mask >> (4 * e);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((mine >> (8 * (i / 4) + i % 4)) & 1)) x[i] = -INFINITY;
            }
            float top = x[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top = fmaxf(top, x[i]);
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any(top - kLift<F16> > m + kSlack)) {
                const float raised = fmaxf(m, top - kLift<F16>), f = weight(m, raised);
                m = raised;
                l *= f;
                f32x16 fr;
#pragma unroll
                for (int i = 0; i < 16; ++i) fr[i] = __shfl(f, 8 * (i / 4) + 4 * e + i % 4);
#pragma unroll
                for (int j = 0; j < kOuts; ++j) o[j] *= fr;
            }
            const float from = m == -INFINITY ? 0.f : m;       // then every x is -inf
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[i] = exp2_fast(x[8 * half + i] - from);
                    l += w[i];
                }
                u32x4 a = {V::pack(w[0], w[1]), V::pack(w[2], w[3]), V::pack(w[4], w[5]), V::pack(w[6], w[7])};
                if (twice && c >= 16) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) a[i] = V::pack(w[2 * i] - V::lo(a[i]), w[2 * i + 1] - V::hi(a[i]));
                }
                {
                    uint32_t v[8][4];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const char *at = tile + v_at[i % 4] + (16 * half + 8 * (i / 4)) * pitch;
                        u32x4 y;
                        if (E4M3) {
                            const u32x2 z = *reinterpret_cast<const u32x2 *>(at);
                            const uint32_t zw[2] = {z[0], z[1]};
                            y = widen<F16, true>(zw);
                        } else {
                            y = *reinterpret_cast<const u32x4 *>(at);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[i][k] = !LATENT && vb * 256 + c * 8 >= Dv ? 0 : y[k];
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint32_t pick = j % 2 ? 0x07060302u : 0x05040100u;
                        u32x4 bv;
#pragma unroll
                        for (int k = 0; k < 4; ++k) bv[k] = __builtin_amdgcn_perm(v[2 * k + 1][j / 2], v[2 * k][j / 2], pick);
                        o[j] = mfma32<F16>(a, bv, o[j]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (ACC && vb == 0) {
                float *to = scores + (c < heads ? t0 : 0);
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f32x4 *>(to + 8 * g) = f32x4{x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]};
            }
#pragma unroll
            for (int k = 0; k < BUFS - 1; ++k) masks[k] = masks[k + 1];
            buf = buf == BUFS - 1 ? 0 : buf + 1;
        }
        if (bad && p.err) atomicOr(p.err, bad);
        l += __shfl_xor(l, 32);
        if (twice) {
#pragma unroll
            for (int j = 0; j < kOuts; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i)        // row 8 (i / 4) + 4 e + i % 4, its rest 16 rows on; see the narrow kernel
                    if (__builtin_fabsf(o[j][i]) < INFINITY) o[j][i] += o[j][i + 8];
        }

        const int64_t head0 = (int64_t)part.r * p.pool.H * p.G + h * p.G + g0;
        const int64_t part0 = part.place < 0 ? 0 : part.place * p.part_heads + wave * 32;
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
        for (int i = 0; i < 16; ++i) {
            const int row = 8 * (i / 4) + 4 * e + i % 4;
            const float lr = __shfl(l, row);
            if (row >= heads) continue;
            const float f = part.place >= 0 ? 1.f : lr == 0.f ? 0.f : v_scale / lr;
            char *dst = p.out.base + part.r * p.out.s_row + (int64_t)(h * p.G + g0 + row) * p.out.s_head;
            float *po = p.part_o + (part0 + row) * Dv;
            {
                const int d = vb * 256 + c * 8;
                if (!LATENT && d >= Dv) continue;
                const f32x16 *y = o;
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
        arrive<0, (WAVES > 1)>();
    }
}

bool latent(const AttendParams &p) { return p.pool.C == 1 && p.pool.D == 576 && p.Dv == 512; }

template <bool F16, bool E4M3, bool ACC>
auto pick(const AttendParams &p) {
    if (!latent(p)) return kvx_attend_wide_kernel<F16, E4M3, 1, 2, false, ACC>;
    if (p.waves_h == 1) return kvx_attend_wide_kernel<F16, E4M3, 1, 2, true, ACC>;
    if (p.waves_h == 2) return kvx_attend_wide_kernel<F16, E4M3, 2, 2, true, ACC>;
    return kvx_attend_wide_kernel<F16, E4M3, 4, 3, true, ACC>;
}

template <bool ACC>
auto pick(const AttendParams &p) {
    return p.f16 ? (p.e4m3 ? pick<true, true, ACC>(p) : pick<true, false, ACC>(p))
                 : (p.e4m3 ? pick<false, true, ACC>(p) : pick<false, false, ACC>(p));
}

int lds_of(const AttendParams &p) {
    const int tile = 32 * pitch_of(p.pool.D, p.e4m3) * (p.pool.C == 2 ? 2 : 1);
    return tile * (latent(p) && p.waves_h == 4 ? 3 : 2);
}

}  // namespace

void plan_attend_wide(AttendParams &p) {
    const int tiles = (p.G + 31) / 32;
    p.waves_k = 1;
    p.waves_h = !latent(p) || tiles == 1 ? 1 : tiles == 2 ? 2 : 4;
    p.span = 32 * p.waves_h;
    p.head_blocks = (tiles + p.waves_h - 1) / p.waves_h;
    p.step = 32;
    p.v_blocks = p.Dv > 256 ? 2 : 1;
    // as many as a compute unit's registers and LDS hold
    p.shares = (p.waves_h == 4 || lds_of(p) > 72 * 1024 ? 256 : 512) / p.v_blocks;
}

int launch_attend_wide(const AttendParams &p, int32_t r0, int32_t n, hipStream_t stream) {
    const auto kernel = p.acc ? pick<true>(p) : pick<false>(p);
    const int64_t blocks = p.whole ? (int64_t)n * p.per : p.shares;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.v_blocks == 2 ? (blocks + 7) / 8 * 16 : blocks)), dim3(64 * p.waves_h),
                       lds_of(p), stream, p, r0, n);
    return hipGetLastError();
}

}  // namespace kvx
