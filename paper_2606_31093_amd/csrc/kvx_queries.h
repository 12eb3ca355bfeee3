// kvx_queries.h -- attention of several queries of a request over a paged cache
// (gfx950): the kernel.
//
// Mathematics.  Rows are pairs (query, query head of the group), row x = query x / G,
// head x % G: all rows of a cache head read the same keys.  s = q.K, capped and
// biased, softmax over the positions that a row sees, out = w V, in one pass with a
// running maximum m and sum l; scores are kept in units of log2.
//
// A workgroup's unit is a block of rows of one record and cache head; it goes over the
// tiles of the positions that some row of the block sees.  A tile's keys and values
// lie in LDS (16-bit; e4m3 is widened on the way, once for all wavefronts), twice, so
// that the next tile is on its way while this one is used.
//
// Bounds.  With many rows a tile's products take as long as its reads from LDS, each
// wavefront reading all of it for its 32 rows: 1.06 PFLOP/s for a prompt of 16384, 32 heads
// of 128 on 8 (2070 us; a large library product reaches 1.2 on this device), 1.02 for one of 8192,
// 0.74 with heads of 64 and 0.87 of 256; 80 and 192 elements take the time of 128 and 256; MLA's rows
// of 576 0.65 (16 heads, a prompt of 4096) to 0.79 (128).  Prompts of up to 2000 reach 0.6:
// a unit's first tile and its outputs take as long as three of its steps.  With few rows
// the cache's bytes bound it: 5 TB/s for a batch of single tokens.  A third and fourth tile
// on its way, or its lines asked for in the cache two tiles ahead, bring nothing (2150 and
// 2290 us), nor do barriers without a wait for stores.
//
// Matrix products of 32 x 32, without a move between lanes.  With c = lane % 32, e =
// lane / 32:
// - scores, transposed: A = 32 rows of K, B = 32 queries (registers); lane (c, e) gets
//   the scores of row c at positions 8 i + 4 e + j (i, j < 4): a row's maximum and sum
//   are taken within a lane and its partner in the other half;
// - these weights are one lane's part of the B operand of the second product, if its k
//   index 8 e + x stands for position 4 e + x (x < 4) or 8 + 4 e + x - 4 (of 16);
// - A = V transposed, by the loads from LDS that transpose: 16 lanes give the addresses
//   of 4 rows x 16 elements, and lane c gets column c;
// - out, transposed: lane (c, e) holds row c, so that a row's rescaling is its lane's.
//
// What a row does not see must not reach it, NaN and infinities too, and a product with
// weight 0 would bring them: where some row of a tile does not see all of it, the
// tile's values are looked over, and rows of V that are not finite are added by hand to
// the rows that see them, and replaced by zeros for the product.
#pragma once

#include "kvx_attend.h"
#include "kvx_queries_plan.h"

namespace kvx {

// Launches the first kernel, by the rows' and the pool's type, for units first ..
// first + n - 1 (whole), or for records first .. first + n - 1.
int launch_queries_bf16(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream);
int launch_queries_f16(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream);
int launch_queries_bf16_e4m3(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream);
int launch_queries_f16_e4m3(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream);

namespace {

constexpr float kLog2e = 1.4426950408889634f;

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;

__device__ __forceinline__ bool valid(const kvx_queries_req &q, const QueriesParams &p) {
    return q.pt_off >= 0 && q.row_off >= 0 && q.start >= 0 && q.end >= q.start && q.n_queries >= 0 && q.prefix >= 0 &&
           q.end >= q.n_queries && q.end - q.start <= p.max_tokens && q.n_queries <= p.max_queries &&
           q.row_off <= p.num_rows - q.n_queries && (!p.tree || (q.n_queries <= KVX_MAX_DRAFTS && q.prefix == 0));
}

// Positions [lo, hi) that some query of several sees, at most.
struct Span {
    uint32_t lo, hi;
};

// Queries i0 .. i1 of a well-formed record.
__device__ __forceinline__ Span span_of(const kvx_queries_req &q, const QueriesParams &p, int i0, int i1) {
    const int base = q.end - q.n_queries;
    const int near = (p.tree ? base : base + i0) - p.window + 1;
    const int seen = p.tree ? q.end : base + i1 + 1 > q.prefix ? base + i1 + 1 : q.prefix;
    return Span{(uint32_t)(p.window && near > q.start ? near : q.start), (uint32_t)(seen < q.end ? seen : q.end)};
}

__device__ __forceinline__ int blocks_of(const kvx_queries_req &q, const QueriesParams &p) {
    return (int)(((int64_t)q.n_queries * p.fd_G.d + p.rows - 1) / p.rows);
}

// Rows x0 .. x1 of a record, its queries' rows (x1: or the last one).
__device__ __forceinline__ Span span_of_rows(const kvx_queries_req &q, const QueriesParams &p, uint32_t x0, uint32_t x1) {
    const int i0 = fd_div(p.fd_G, x0), i1 = fd_div(p.fd_G, x1);
    return span_of(q, p, i0, i1 < q.n_queries ? i1 : q.n_queries - 1);
}

__device__ __forceinline__ int steps_of(const Span &s, const QueriesParams &p) {
    return s.hi > s.lo ? (int)((s.hi - (s.lo & -kTile) + p.step - 1) / p.step) : 1;
}

__device__ __forceinline__ Span span_of_block(const kvx_queries_req &q, const QueriesParams &p, int b) {
    return span_of_rows(q, p, (uint32_t)b * p.rows, (uint32_t)b * p.rows + p.rows - 1);
}

// What a unit costs beside its tiles (the way from its record to the first tile, and the
// outputs), in steps that come before its first: shares of equal steps are then done in
// about equal time.  Of a block of 256 rows 4.5 us pass before the first tile is there, of which 1.9
// until its page ids are, and 2.5 us in the outputs; a step takes 2.2.  With 2, 4 and 6 steps 16
// prompts of up to 2000 take 481, 442 and 458 us, four of 1500 61, 56 and 55.5.
constexpr int kUnitSteps = 4;

// Steps of the blocks of 64 from b0 on of a record and group, a block a lane.
__device__ __forceinline__ int steps_of_lane(const kvx_queries_req &q, const QueriesParams &p, int b0, int lane, int blocks) {
    const int b = b0 + lane;
    return b < blocks ? kUnitSteps + steps_of(span_of_block(q, p, b), p) : 0;
}

// Steps of one group of cache heads of a record, by a wavefront.
__device__ __forceinline__ int64_t steps_of_group(const kvx_queries_req &q, const QueriesParams &p, int lane) {
    if (!valid(q, p)) return 0;
    int64_t sum = 0;
    const int blocks = blocks_of(q, p);
    for (int b = 0; b < blocks; b += 64) sum += steps_of_lane(q, p, b, lane, blocks);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
    return sum;
}

__device__ __forceinline__ kvx_queries_req scalar(const kvx_queries_req &q) {
    uint32_t w[8];
    __builtin_memcpy(w, &q, sizeof w);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    kvx_queries_req s;
    __builtin_memcpy(&s, w, sizeof s);
    return s;
}

__device__ __forceinline__ int64_t scalar(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                     (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}

// Part of a unit: positions [begin, end) for block b of a group of cache heads.
struct Piece {
    kvx_queries_req rec;
    int32_t group, b;
    uint32_t begin, end;
    int64_t place;               // of its partial results; -1: it is the whole unit
};

// The place of share k's part of a unit whose first of all steps is `first`: its first
// part has the place k, one that begins inside the share place shares + k.
__device__ __forceinline__ int64_t place_of(int64_t first, int64_t k, int64_t each, int64_t shares) {
    return first > k * each ? shares + k : k;
}

// Partial results of 32 rows from `row` on, of values 32 d to 32 d + 31: [j][row c][half e][4], for the
// values 8 j + 4 e + x, as a lane has them.
__host__ __device__ constexpr int wide_blocks(int dv) { return (dv + 31) / 32; }
__device__ __forceinline__ float *part_of(const QueriesParams &p, int64_t row, int d) {
    return p.part_o + (row * wide_blocks(p.Dv) + 32 * d) * 32;
}

__device__ __forceinline__ int64_t share_of(int64_t total, int64_t shares) {
    const int64_t each = quotient(total + shares - 1, shares);
    return each < 1 ? 1 : each;
}

// bits below x
__device__ __forceinline__ uint64_t ones(int64_t x) { return x <= 0 ? 0 : x >= 64 ? ~0ull : (1ull << x) - 1; }

// 16 bytes a lane to LDS, in order of lanes from `to` on.  In assembly, since the compiler
// would wait for all of them before reads of LDS; nothing reads what they bring before
// the wait and the barrier of arrive().
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}

// The lane, computed where it is used, so that what follows from it is not kept in
// registers from tile to tile.
__device__ __forceinline__ int lane_again() {
    int zero = 0;
    asm volatile("" : "+s"(zero));
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, zero));
}

static __device__ const uint4 kvx_zeros = {0, 0, 0, 0};

template <bool F16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(bits<f16x8>(a), bits<f16x8>(b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(bits<bf16x8>(a), bits<bf16x8>(b), c, 0, 0, 0);
}

// Whether one of two 16-bit values is infinite or NaN.
template <bool F16>
__device__ __forceinline__ bool not_finite(uint32_t w) {
    const uint32_t e = F16 ? 0x7c00u : 0x7f80u;
    return (w & e) == e || (w >> 16 & e) == e;
}

// Whether LDS has room for one tile only.
__host__ __device__ constexpr bool one_tile(int dk, int kv) { return dk > 256 && kv == 2; }

// Caps above this, in units of log2: cap - 2 cap / (1 + e^2x) would lose the digits of scores
// far below the cap, up to 2^-22 of it.
constexpr float kWideCap = 256.f;

// tanh x to 2^-19 of it, z = 2 x log2 e: below 1/4 its series (the next term is 2^-27 of it), else
// 1 - 2 / (1 + e^2x).
__device__ __forceinline__ float tanh_of(float x, float z) {
    const float y = x * x;
    const float small = x + x * y * (-1.f / 3 + y * (2.f / 15 + y * (-17.f / 315 + y * (62.f / 2835))));
    return fabsf(x) < 0.25f ? small : 1.f + 2.f * __builtin_amdgcn_rcpf(-1.f - exp2_fast(z));
}

// The larger of three; what is not a number counts for nothing.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float x;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(x) : "v"(a), "v"(b), "v"(c));
    return x;
}

// x of this lane and of the lane in the other half.
__device__ __forceinline__ float max_of_halves(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(bits<uint32_t>(x), bits<uint32_t>(x), false, false);
    return fmaxf(bits<float>((uint32_t)y[0]), bits<float>((uint32_t)y[1]));
}

// A branch that is seldom taken: its code lies elsewhere.
__device__ __forceinline__ bool seldom(bool x) { return __builtin_expect_with_probability(x, 0, 0.9999); }

// The kernel's parameters, its first argument, read anew: kept from the kernel's begin to
// its end they would take more scalar registers than there are.
__device__ __forceinline__ QueriesParams again() {
    const auto *p = (const __attribute__((address_space(4))) QueriesParams *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const QueriesParams *)p;
}

// DK: elements of a row in LDS (head_dim is up to that), DV: of a value; TEAM: wavefronts
// that share a tile (all of the workgroup; or 1: each takes tiles of its own for the same
// 32 rows, and they join at the end); SPLIT: wavefronts that share 32 rows (wide rows: a
// query and its outputs would not leave registers for a second wavefront on the SIMD;
// each takes a part of the values, and for the scores half of the positions, whose weights
// they pass each other through LDS, or, where a query takes too many registers, half of
// the elements, and they add the scores up); TILE: positions; GENERAL: scores may be
// capped or biased.
template <bool F16, bool E4M3, int DK, int DV, int TEAM, int SPLIT, int TILE, bool GENERAL>
struct Queries {
    typedef Half<F16> V;
    // of a wavefront: steps of 16 elements of K, blocks of 32 values
    static constexpr bool HALVES = SPLIT > 1 && DK <= 256;
    static constexpr int KS = HALVES ? DK / 16 : DK / 16 / SPLIT, DB = DV / 32 / SPLIT;
    // blocks of 32 positions, those a wavefront scores and all that it takes values of
    static constexpr int PB = TILE / 32 / (HALVES ? SPLIT : 1), PV = TILE / 32, PITCH = 2 * DK;
    static constexpr int SRC = DK * (E4M3 ? 1 : 2) / 16;       // 16-byte chunks of a row in memory
    // loads of a wavefront for a tile's K or V, of them all a wavefront's at most
    static constexpr int ALL_LOADS = TILE * SRC / 64, LOADS = (ALL_LOADS + TEAM - 1) / TEAM;
    // Weights in two parts, as kvx_attend's, where few rows leave the matrix cores idle; with more rows the
    // second product would take half as long again, and a weight's rounding is one of many that average.
    static constexpr bool PARTS = TEAM == 1;
    // Reads of LDS are kept so many products ahead (left alone the compiler waits for each one
    // where registers are few, or reads more than there are registers for).  A prompt of 16384 takes
    // 2260, 2238 and 2236 us with 2, 4 and 6; rows of 576, whose registers are few, 190, 199 and 207
    // with 2, 3 and 4.
    static constexpr int AHEAD = SPLIT > 1 ? 2 : 4;
    // Tiles are taken from the last to the first where scores may have a bias: it is highest at the end
    // as a rule, and from the first on sums would be rescaled at nearly every tile.  A prompt of 16384, 32
    // heads of 128, takes 2290 us so and 2450 to 2520 forwards; 16 prompts of up to 2000, e4m3, 441 and
    // 452.  Without a bias it is the same (2098 and 2086).
    static constexpr bool BACK = GENERAL;
    static constexpr uint64_t ALL = TILE == 64 ? ~0ull : 0xffffffffull;
    static_assert(TILE * SRC % 64 == 0 && (TILE == 32 || TILE == 64), "tile");

    // Of TEAM tiles, and the next TEAM ones: row offsets (-1: none) and which are there.
    struct Rows {
        int64_t off[2][TEAM][TILE];
        uint64_t there[2][TEAM];
    };
    Rows &rows;                  // the team's
    float *depth;                // [64]
    // What a lane's row sees is needed at the edges only, and kept in LDS.
    struct Sight {
        uint64_t drafts;         // of the drafts
        uint32_t lo, hi;         // and of the positions before them [lo, hi)
    } *sight;                    // [32], the wavefront's rows
    char *lds;                   // [2][rows of K, rows of V if there are two], the team's
    float *ml;                   // [wavefronts][32][2]
    int32_t (*flags)[TEAM];      // [4]: of tiles in turns, of two questions
    char *all_lds;               // the workgroup's
    f32x4 *shared;               // [wavefront][4][64]: scores that wavefronts of the same rows add up, or
                                 // [wavefront][2][64]: weights that they pass each other
    float *tops;                 // [wavefront][32]: what they agree on, of each row
    int lane, wave, part, c, e;  // part: of the team
    bool two, once;              // V apart from K; LDS has room for one tile only
    int tile_bytes;
    // of the piece
    kvx_queries_req rec;
    const char *kbase;
    int64_t s_p, s_c, s_t, pt_len;
    const int32_t *pt;
    FastDiv fd_T;
    int32_t N, have;             // pages; 16-byte chunks of a row
    uint32_t first, end, bad;
    u32x4 staged[E4M3 ? LOADS : 1][2];

    __device__ __forceinline__ uint64_t entry(uint32_t t) const { return (uint64_t)rec.pt_off + fd_div(fd_T, t); }
    // the page id of position t0 + lane
    __device__ __forceinline__ int32_t look(uint32_t t0) const {
        const uint32_t t = t0 + lane_again();
        const uint64_t idx = entry(t < end ? t : end - 1);
        return pt[idx < (uint64_t)pt_len ? idx : 0];
    }
    // A tile's row offsets, to place `slot` of half `ring`.
    __device__ __forceinline__ void resolve(uint32_t t0, int32_t page, int ring, int slot) {
        const int lane = lane_again();
        const uint32_t t = t0 + lane;
        const bool in = lane < TILE && t >= first && t < end;
        const uint32_t at = t < end ? t : end - 1;
        const bool known = entry(at) < (uint64_t)pt_len;
        const bool ok = in && known && (uint32_t)page < (uint32_t)N;
        if (in && !ok) bad |= known ? KVX_DERR_SRC_PAGE : KVX_DERR_PT_RANGE;
        const int64_t off = page * s_p + (int64_t)(at - fd_div(fd_T, at) * fd_T.d) * s_t;
        if (TILE == 64 || lane < TILE) rows.off[ring][slot][lane] = ok ? off : -1;
        const uint64_t there = __ballot(ok);
        if (lane == 0) rows.there[ring][slot] = there;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    // Which row and 16-byte chunk of it a lane's load x takes.  Where rows have a power of two of
    // chunks, successive loads are R rows apart, and the permutation of a row is that of its
    // bits: only the first load's are kept.
    static constexpr bool REGULAR = (SRC & (SRC - 1)) == 0;
    static constexpr int R = 64 * TEAM / SRC;
    int row0, chunk0;
    __device__ __forceinline__ void place(int x, int &row, int &chunk) const {
        if constexpr (REGULAR) {
            row = row0 + x * R;
            chunk = E4M3 ? chunk0 : chunk0 ^ swirl(x * R);
        } else {
            const uint32_t u = (x * TEAM + part) * 64 + lane_again();
            row = u / SRC;
            chunk = u % SRC;
            if (!E4M3) chunk ^= swirl(row);
        }
    }
    // Asks for this wavefront's share of a tile's rows, zeros where there is none and behind head_dim.
    // WHOLE: all rows are there, and full.
    template <bool WHOLE>
    __device__ __forceinline__ void load_rows(int buf, const int64_t *off_of) {
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)(lds + buf * tile_bytes);
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int piece = x * TEAM + part;
            if (ALL_LOADS % TEAM && piece >= ALL_LOADS) continue;
            int row, chunk;
            place(x, row, chunk);
            const int64_t off = off_of[row];
            const bool ok = WHOLE || (off >= 0 && chunk < have);
            const char *k = ok ? kbase + off + (uint32_t)(16 * chunk) : reinterpret_cast<const char *>(&kvx_zeros);
            const char *v = ok ? k + s_c : k;
            if constexpr (E4M3) {
                staged[x][0] = *reinterpret_cast<const u32x4 *>(k);
                if (two) staged[x][1] = *reinterpret_cast<const u32x4 *>(v);
            } else {
                const uint32_t at = __builtin_amdgcn_readfirstlane(to + piece * 1024);
                load_to_lds(k, at);
                if (two) load_to_lds(v, at + TILE * PITCH);
            }
        }
    }
    __device__ __forceinline__ void load(int buf, const int64_t *off_of, uint64_t there) {
        if (seldom(there != ALL || have != SRC)) load_rows<false>(buf, off_of);
        else load_rows<true>(buf, off_of);
    }
    // e4m3: what load() has brought, widened, to LDS.
    __device__ __forceinline__ void put(int buf) {
        if constexpr (E4M3) {
            char *to = lds + buf * tile_bytes;
#pragma unroll
            for (int x = 0; x < LOADS; ++x) {
                if (ALL_LOADS % TEAM && x * TEAM + part >= ALL_LOADS) continue;
                int row, chunk;
                place(x, row, chunk);
                chunk *= 2;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (kv && !two) continue;
                    const u32x4 y = staged[x][kv];
                    const uint32_t w[4] = {y[0], y[1], y[2], y[3]};
                    char *at = to + (kv * TILE + row) * PITCH;
                    *reinterpret_cast<u32x4 *>(at + 16 * (chunk ^ swirl(row))) = widen<F16, true>(w);
                    *reinterpret_cast<u32x4 *>(at + 16 * ((chunk + 1) ^ swirl(row))) = widen<F16, true>(w + 2);
                }
            }
        }
    }
    // What this wavefront has asked for and put is in LDS, and the team's is.
    __device__ __forceinline__ void arrive() const {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (TEAM > 1) __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }

    // LDS.  Chunk x (16 bytes) of row r lies at place x ^ swirl(r) of the row, so that the
    // 64 banks are read without conflicts: one chunk of 16 rows (keys), and 64 bytes of 4
    // successive rows (values) lie in different banks.  Where rows begin 128 bytes apart
    // of 256, two rows lie side by side.
    static constexpr bool APART = PITCH % 256 != 0;
    static constexpr int TURNS = APART ? 8 : 16;               // chunks that a row's permutation moves
    static __device__ __forceinline__ int swirl(int r) {
        return APART ? (r >> 1 & 1) << 2 | (r >> 2 & 3) : (r & 3) << 2 | (r >> 2 & 3);
    }
    // Addresses, those that the permutation makes; the rest is in the instructions.
    // - K: the lane's row, chunks 2 k + e from the wavefront's first step on
    // - V, 32 columns from 32 db on: 16 lanes give the addresses of 4 rows x 16 elements,
    //   positions 32 pb + 16 s + 4 e + x, and 8 behind, x < 4
    // the first position of a tile that the wavefront scores
    __device__ __forceinline__ int own() const { return HALVES ? 32 * PB * (wave % SPLIT) : 0; }
    // Where a row has 16 places the others follow from one by an exclusive or, tiles lying at
    // multiples of 256 bytes.
    int k_at[APART ? TURNS / 2 : 1], v_at[APART ? TURNS / 4 : 1];
    __device__ __forceinline__ void address() {
        const int mine = wave % SPLIT, l = lane & 15, row = 4 * e + l / 4;
        row0 = (part * 64 + lane) / SRC;
        chunk0 = (part * 64 + lane) % SRC ^ (E4M3 ? 0 : swirl(row0));
#pragma unroll
        for (int k = 0; k < (APART ? TURNS / 2 : 1); ++k)
            k_at[k] = (c + own()) * PITCH + 16 * ((2 * ((HALVES ? 0 : mine * KS) + k) + e) ^ swirl(c));
#pragma unroll
        for (int d = 0; d < (APART ? TURNS / 4 : 1); ++d)
            v_at[d] = row * PITCH + 16 * ((4 * (mine * DB + d) + (lane >> 4 & 1) * 2 + (l >> 1 & 1)) ^ swirl(row)) + (l & 1) * 8;
    }
    // lowest addresses of a tile's reads
    __device__ __forceinline__ void at_tile(const char *k, const char *v, uint32_t *ka, uint32_t *va) const {
        const uint32_t kt = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)k;
        const uint32_t vt = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)v;
#pragma unroll
        for (int i = 0; i < (APART ? TURNS / 2 : 1); ++i) ka[i] = kt + k_at[i];
#pragma unroll
        for (int i = 0; i < (APART ? TURNS / 4 : 1); ++i) va[i] = vt + v_at[i];
    }
    typedef const __attribute__((address_space(3))) char *Lds;
    __device__ __forceinline__ u32x4 keys(const uint32_t *ka, int pb, int step) const {
        const int turn = step % (TURNS / 2), far = 32 * pb * PITCH + step / (TURNS / 2) * 16 * TURNS;
        const Lds at = (Lds)(APART ? ka[turn % (APART ? TURNS / 2 : 1)] : ka[0] ^ 32 * turn);
        return *(const __attribute__((address_space(3))) u32x4 *)(at + far);
    }
    __device__ __forceinline__ u32x4 columns(const uint32_t *va, int pb, int s, int db) const {
        const int turn = db % (TURNS / 4), far = (32 * pb + 16 * s) * PITCH + db / (TURNS / 4) * 16 * TURNS;
        const uint32_t at = APART ? va[turn % (APART ? TURNS / 4 : 1)] : va[0] ^ 64 * turn;
        // 8 rows on the permutation differs in its second bit
        const Lds a = (Lds)at + far, b = (Lds)(at ^ 32) + far + 8 * PITCH;
        const u32x2 x = bits<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)a));
        const u32x2 y = bits<u32x2>(__builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)b));
        return u32x4{x[0], x[1], y[0], y[1]};
    }

    // Whether x holds for one of the team's wavefronts; `turn` differs from call to call.  The
    // loads that are on their way are not waited for.
    __device__ __forceinline__ bool any_of_team(bool x, int turn) const {
        if (lane == 0) flags[turn][part] = x;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        return __any(flags[turn][lane & (TEAM - 1)]);
    }

    // Rows r0 .. r0 + n - 1 of V that hold values which are not finite.
    __device__ __forceinline__ uint64_t spoilt(const char *v, int r0, int n) const {
        uint64_t found_rows = 0;
        const int lane = lane_again();
        for (int r = r0; r < r0 + n; ++r) {
            bool found = false;
            if (lane < DV / 8) {
                const u32x4 w = *reinterpret_cast<const u32x4 *>(v + r * PITCH + 16 * (lane ^ swirl(r)));
                found = not_finite<F16>(w[0]) || not_finite<F16>(w[1]) || not_finite<F16>(w[2]) || not_finite<F16>(w[3]);
            }
            if (__any(found)) found_rows |= 1ull << r;
        }
        return found_rows;
    }
    __device__ __forceinline__ bool any_spoilt(const char *v, int r0, int n) const {
        bool found = false;
        const int lane = lane_again();
#pragma unroll 1
        for (int u = lane; u < n * (DV / 8); u += 64) {
            const int r = r0 + u / (DV / 8), chunk = u % (DV / 8);
            const u32x4 w = *reinterpret_cast<const u32x4 *>(v + r * PITCH + 16 * (chunk ^ swirl(r)));
            found |= not_finite<F16>(w[0]) || not_finite<F16>(w[1]) || not_finite<F16>(w[2]) || not_finite<F16>(w[3]);
        }
        return __any(found);
    }

    // The highest score of this lane's.
    static __device__ __forceinline__ float top_of(const f32x16 *s, float from, float shift) {
        float top[4] = {s[0][0], s[0][1], s[0][2], s[0][3]};
#pragma unroll
        for (int pb = 0; pb < PB; ++pb)
#pragma unroll
            for (int i = 0; i < 16; i += 8)
#pragma unroll
                for (int j = 0; j < 4; ++j) top[j] = max3(top[j], s[pb][i + 2 * j], s[pb][i + 2 * j + 1]);
        return __builtin_fmaf(max3(top[0], top[1], fmaxf(top[2], top[3])), from, shift);
    }
    static __device__ __forceinline__ void raise(float to, float &m, float &l, f32x16 *o) {
        const float f = weight(m, to);
        m = to;
        l *= f;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= f;
    }
    // Scores to weights against m; their sum.
    static __device__ __forceinline__ float weigh(f32x16 *s, float from, float shift, float m) {
        const float ref = shift - (m == -INFINITY ? 0.f : m);      // without any, every score is -inf
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int pb = 0; pb < PB; ++pb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[pb][i] = exp2_fast(__builtin_fmaf(s[pb][i], from, ref));
                sums[i % 2] += s[pb][i];
            }
        return sums[0] + sums[1];
    }
    static __device__ __forceinline__ void pack_weights(const f32x16 *s, u32x4 *w, u32x4 *rest) {
#pragma unroll
        for (int u = 0; u < 2 * PB; ++u) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = s[u / 2][8 * (u % 2) + i];
            if (PARTS) split<F16>(x, w[u], rest[u]);
            else w[u] = u32x4{V::pack(x[0], x[1]), V::pack(x[2], x[3]), V::pack(x[4], x[5]), V::pack(x[6], x[7])};
        }
    }

    __device__ __forceinline__ void run(const Piece &piece) {
        rec = piece.rec;
        const int base = rec.end - rec.n_queries;
        const uint32_t begin = piece.begin;
        end = piece.end;
        first = (uint32_t)rec.start > begin ? rec.start : begin;
        bad = 0;
        int x0, streams, h_rows, h, stream;       // the wavefront's cache head, its place among those of the head
        bool active;
        // This lane's row; past the last one, that one once more.
        int at;                          // its position
        float slope = 0.f, cap2 = 0.f, cap_unit = 0.f, unit;
        uint32_t slopes[2] = {0, 0};
        bool linear = false;
        bool is_tree, biased;
        uint32_t t0, step;               // this wavefront's tile, and from one to the next
        int32_t page0 = 0, page = 0;     // page ids of the first tiles to resolve, and the next
        uint32_t past;                   // positions below it are at or behind all rows of the wavefront
        u32x4 qv[KS];
        // Positions that all rows of the wavefront see, that some see, and that all of the
        // workgroup see.  In a tree depths differ within a block: the drafts and the last
        // position's window bound them.
        Span all, some, block_all;
        {
            const QueriesParams p = again();
            const int G = p.fd_G.d, n_rows = rec.n_queries * G;
            h_rows = n_rows;
            streams = TEAM > 1 ? 1 : p.waves / p.heads;
            stream = TEAM > 1 ? 0 : wave % streams;
            h = TEAM > 1 ? piece.group : piece.group * p.heads + wave / streams;
            kbase = p.pool.base + h * p.pool.s_h;
            s_p = p.pool.s_p;
            s_c = p.pool.s_c;
            s_t = p.pool.s_t;
            pt = p.pool.pt;
            pt_len = p.pool.pt_len;
            fd_T = p.pool.fd_T;
            N = p.pool.N;
            have = (E4M3 ? 1 : 2) * p.pool.D / 16;
            t0 = begin + stream * TILE;
            step = TILE * streams;
            if (BACK && t0 < end) {
                t0 += (end - 1 - t0) / step * step;
                step = 0u - step;
            }
            if (t0 < end) {
                page0 = look(t0 + part * step);
                page = look(t0 + (TEAM + part) * step);
            }
            is_tree = p.tree;
            biased = GENERAL && p.slopes;
            // Scores are taken times unit > 0: a sign goes into the queries.
            unit = p.scale * (p.scales ? p.scales[h] : 1.f) * kLog2e;
            const uint32_t flip = unit < 0.f ? 0x80008000u : 0;
            const bool none = unit == 0.f;
            unit = none ? 1.f : fabsf(unit);
            if (GENERAL && p.cap > 0.f) {
                cap2 = p.cap * kLog2e;
                cap_unit = 2.f * unit / p.cap;
                if (cap_unit > 3e38f) cap_unit = 3e38f;      // a score of 0 stays one
            }
            const int block0 = piece.b * p.rows;
            x0 = block0 + part / SPLIT * 32;
            active = x0 < n_rows;
            if (is_tree) {
                if (lane < rec.n_queries) {
                    const int k = __popcll(p.tree[rec.row_off + lane] & ones(rec.n_queries));
                    depth[lane] = k > 0 ? k - 1 : 0;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
            const int x = x0 + c, row = x < n_rows ? x : n_rows - 1;
            const int i = fd_div(p.fd_G, row), g = row - i * G;
            uint64_t drafts = 0;
            at = base + i;
            if (is_tree) {
                const int mine = (int)depth[i];
                at = base + mine;
                drafts = p.tree[rec.row_off + i] & ones(rec.n_queries) & ~ones((int64_t)rec.start - base);
                if (p.window)
                    for (int j = 0; j < rec.n_queries; ++j)
                        if (mine - (int)depth[j] >= p.window) drafts &= ~(1ull << j);
            }
            const int near = at - p.window + 1;
            const int seen = is_tree ? base : at + 1 > rec.prefix ? at + 1 : rec.prefix;
            sight[c] = Sight{drafts, (uint32_t)(p.window && near > rec.start ? near : rec.start),
                                (uint32_t)(seen < rec.end ? seen : rec.end)};
            if (biased) {
                slope = p.slopes[h * G + g] * kLog2e;
                // In three parts of the rows' type, for a product with whole numbers up to 63.  In half, whose
                // values are 2^-24 apart at least, up to 2^-25 is left, in the bias 2^-19 unit: with a large unit
                // it is added by hand.
                const float x = slope / unit, a = V::lo(V::pack(x, 0.f)), b = V::lo(V::pack(x - a, 0.f));
                slopes[0] = V::pack(a, b);
                slopes[1] = V::pack(x - a - b, 0.f);
                linear = cap_unit == 0.f && !__any(!(fabsf(x) < 1024.f)) && !(F16 && unit > 2.f);
            }
            const int d0 = 16 * (HALVES ? 0 : wave % SPLIT * KS) + 8 * (lane_again() >> 5), left = none ? 0 : p.pool.D - d0;
            const char *src = p.q.base + (rec.row_off + i) * p.q.s_row + (int64_t)(h * G + g) * p.q.s_head + 2 * d0;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                qv[k] = u32x4{0, 0, 0, 0};
                if (16 * k < left) qv[k] = *reinterpret_cast<const u32x4 *>(src + 32 * k);
#pragma unroll
                for (int w = 0; w < 4; ++w) qv[k][w] ^= flip;
            }
            const auto bounds = [&](int xa, int xz, Span &a, Span &s) {
                xa = xa < n_rows ? xa : n_rows - 1;
                xz = xz < n_rows ? xz : n_rows - 1;
                s = span_of_rows(rec, p, xa, xz);
                a.hi = is_tree ? (uint32_t)base : span_of_rows(rec, p, xa, xa).hi;
                const int last = rec.end - p.window;
                a.lo = !is_tree ? span_of_rows(rec, p, xz, xz).lo : (uint32_t)(p.window && last > rec.start ? last : rec.start);
            };
            Span unused;
            bounds(x0, x0 + 31, all, some);
            past = base + (is_tree ? 0 : (int)fd_div(p.fd_G, x0 < n_rows ? x0 : n_rows - 1) + 1);
            bounds(block0, block0 + p.rows - 1, block_all, unused);
        }

        f32x16 o[DB];
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
        float m = -INFINITY, l = 0.f;

        if (t0 < end) {
            // Tiles are resolved TEAM at a time, one by each wavefront, while the TEAM before are used;
            // their page ids are asked for as much earlier.
            const uint32_t mine = t0 + part * step;
            resolve(mine, page0, 0, part);
            if (TEAM > 1) __syncthreads();
            load(0, rows.off[0][0], scalar((int64_t)rows.there[0][0]));
            put(0);
            for (int k = 0; t0 - begin < end - begin; t0 += step, ++k) {
                const int buf = SPLIT > 1 && once ? 0 : k & 1, slot = k & (TEAM - 1), ring = k / TEAM & 1;
                if (SPLIT > 1 && once && k > 0) {
                    // the tile before has been used
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    load(0, rows.off[ring][slot], scalar((int64_t)rows.there[ring][slot]));
                    put(0);
                }
                arrive();
                if (TEAM > 1 ? seldom(slot == 0) : true) {
                    resolve(t0 + (TEAM + part) * step, page, ring ^ 1, part);
                    page = look(t0 + (2 * TEAM + part) * step);
                }
                const bool more = t0 + step - begin < end - begin && !(SPLIT > 1 && once);
                const int next = k + 1, next_ring = next / TEAM & 1, next_slot = next & (TEAM - 1);
                if (more) load(buf ^ 1, rows.off[next_ring][next_slot], scalar((int64_t)rows.there[next_ring][next_slot]));
                const uint64_t here = scalar((int64_t)rows.there[ring][slot]);
                const char *kt = lds + buf * tile_bytes, *vt = kt + (two ? TILE * PITCH : 0);
                uint32_t ka[APART ? TURNS / 2 : 1], va[APART ? TURNS / 4 : 1];
                at_tile(kt, vt, ka, va);
                const bool on = active && t0 < some.hi && t0 + TILE > some.lo;
                const bool edge = here != ALL || t0 < all.lo || t0 + TILE > all.hi;        // some row does not see all
                const bool team_edge = here != ALL || t0 < block_all.lo || t0 + TILE > block_all.hi;
                f32x16 s[PB];            // scores, then weights
                uint64_t sees = ALL;
                // all keys lie behind, and none of the bias has to follow a cap: it is linear in the position
                const bool straight = GENERAL && linear && t0 + TILE <= past;
#pragma unroll
                for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[pb][i] = 0.f;
                if (on) {
                    u32x4 a[AHEAD + 1];
#pragma unroll
                    for (int u = 0; u < AHEAD; ++u) a[u] = keys(ka, u % PB, u / PB);
                    if (GENERAL && straight && (HALVES || wave % SPLIT == 0)) {
                        // slope * (position within the tile) as one more step of the product
#pragma unroll
                        for (int pb = 0; pb < PB; ++pb) {
                            const int ln = lane_again();
                            const float row = own() + 32 * pb + (ln & 31);
                            const uint32_t off = V::pack(row, row);
                            s[pb] = mfma32<F16>(ln < 32 ? u32x4{off, off & 0xffff, 0, 0} : u32x4{0, 0, 0, 0}, u32x4{slopes[0], slopes[1], 0, 0}, s[pb]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int u = 0; u < KS * PB; ++u) {
                        if (u + AHEAD < KS * PB) a[(u + AHEAD) % (AHEAD + 1)] = keys(ka, (u + AHEAD) % PB, (u + AHEAD) / PB);
                        s[u % PB] = mfma32<F16>(a[u % (AHEAD + 1)], qv[u / PB], s[u % PB]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if constexpr (SPLIT > 1 && !HALVES) {
                    static_assert(PB == 1 && SPLIT == 2, "pairs");
                    f32x4 *mine = shared + wave * 256 + lane;
#pragma unroll
                    for (int i = 0; i < 4; ++i) mine[64 * i] = f32x4{s[0][4 * i], s[0][4 * i + 1], s[0][4 * i + 2], s[0][4 * i + 3]};
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    const f32x4 *other = shared + (wave ^ 1) * 256 + lane;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 x = other[64 * i];
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[0][4 * i + j] += x[j];
                    }
                }
                float from = unit, shift = 0.f;  // scores are s * from + shift
                if (on) {
                    if (GENERAL) {
                        if (seldom(cap_unit > 0.f)) {
                            if (seldom(cap2 > kWideCap)) {
                                const float near = 0.5f * kLn2 * cap_unit;
#pragma unroll
                                for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                                    for (int i = 0; i < 16; ++i) {
                                        if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                                        s[pb][i] = cap2 * tanh_of(s[pb][i] * near, s[pb][i] * cap_unit);
                                    }
                                from = 1.f;
                            } else {
                                // cap tanh(x) = cap - 2 cap / (1 + e^2x)
#pragma unroll
                                for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                                    for (int i = 0; i < 16; ++i) s[pb][i] = __builtin_amdgcn_rcpf(-1.f - exp2_fast(s[pb][i] * cap_unit));
                                from = 2.f * cap2;
                                shift = cap2;
                            }
                        }
                        if (straight) {
                            shift = -slope * (float)(at - (int)t0);      // the rest of the bias is in the product
                        } else if (seldom(biased)) {
                            const int e = lane_again() >> 5;
                            const int t = t0 + own() + 4 * e;
                            const float far = (float)(at - t);
                            const bool by_depth = is_tree && t0 + TILE > (uint32_t)base;
#pragma unroll
                            for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const int off = 32 * pb + 8 * (i / 4) + i % 4;
                                    float d = far - (float)off;
                                    if (by_depth) {
                                        if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                                        const int j = t + off - base;
                                        const bool draft = j >= 0 && j < rec.n_queries;
                                        if (draft) d = (float)(at - base) - depth[j];
                                    }
                                    s[pb][i] = __builtin_fmaf(-slope, fabsf(d), __builtin_fmaf(s[pb][i], from, shift));
                                }
                            from = 1.f;
                            shift = 0.f;
                        }
                    }
                    if (seldom(edge)) {
                        const int ln = lane_again();
                        const Sight mine = sight[ln & 31];
                        uint64_t v = ones((int64_t)mine.hi - t0) & ~ones((int64_t)mine.lo - t0);
                        const int64_t to = (int64_t)base - t0;
                        if (is_tree && to < 64 && to > -64) v |= to >= 0 ? mine.drafts << to : mine.drafts >> -to;
                        sees = v & here;
                        const uint64_t shown = sees >> (own() + 4 * (ln >> 5));
#pragma unroll
                        for (int pb = 0; pb < PB; ++pb)
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (!((uint32_t)(shown >> (32 * pb)) >> (8 * (i / 4) + i % 4) & 1)) s[pb][i] = -INFINITY;
                    }
                    if constexpr (!HALVES) {
                        float top = top_of(s, from, shift);
                        if (seldom(__any(top - kLift<F16> > m + kSlack))) {
                            top = max_of_halves(top);
                            raise(fmaxf(m, top - kLift<F16>), m, l, o);
                        }
                        l += weigh(s, from, shift, m);
                    }
                }
                u32x4 w[2 * PV], rest[2 * PV];   // weights of 8 positions, in one part or two
                if constexpr (HALVES) {
                    // Weights against the reference that both wavefronts of the rows have; where one of the
                    // team's finds scores too far above, both raise theirs, and weigh once more.
                    static_assert(PB == 1 && SPLIT == 2, "pairs");
                    u32x4 *mine = reinterpret_cast<u32x4 *>(shared) + wave * 128 + lane;
                    const u32x4 *others = reinterpret_cast<const u32x4 *>(shared) + (wave ^ 1) * 128 + lane;
                    const f32x16 raw = s[0];
                    float sum = 0.f;
                    const auto pass = [&]() __attribute__((always_inline)) {
                        s[0] = raw;
                        sum = weigh(s, from, shift, m);
                        pack_weights(s, w, rest);
                        mine[0] = w[0];
                        mine[64] = w[1];
                    };
                    bool far_above = false;
                    if (on) {
                        const float top = max_of_halves(top_of(s, from, shift));
                        far_above = __any(top - kLift<F16> > m + kSlack);
                        if (lane < 32) tops[wave * 32 + lane] = top;
                        pass();
                    }
                    if (seldom(any_of_team(far_above, k & 1))) {
                        if (on) {
                            const float top = fmaxf(tops[wave * 32 + c], tops[(wave ^ 1) * 32 + c]);
                            raise(fmaxf(m, top - kLift<F16> > m + kSlack ? top - kLift<F16> : m), m, l, o);
                            pass();
                        }
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                    }
                    l += sum;
                    if (on) {
                        const bool second = wave & 1;
                        const u32x4 a = others[0], b = others[64], x = w[0], y = w[1];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            w[0][i] = second ? a[i] : x[i];
                            w[1][i] = second ? b[i] : y[i];
                            w[2][i] = second ? x[i] : a[i];
                            w[3][i] = second ? y[i] : b[i];
                        }
                    }
                }
                if (seldom(team_edge)) {
                    // The tile is the team's: it looks over its values together.
                    constexpr int MINE = TILE / TEAM;
                    char *v = const_cast<char *>(vt);
                    const int lane = lane_again(), c = lane & 31, e = lane >> 5;
                    bool found = any_spoilt(v, part * MINE, MINE);
                    if (TEAM > 1) found = any_of_team(found, 2 + (k & 1));
                    if (seldom(found)) {
                        const uint64_t spoilt_rows = spoilt(v, 0, TILE);
                        for (uint64_t left = spoilt_rows; left && on; left &= left - 1) {
                            const int r = __ffsll((unsigned long long)left) - 1;
                            const int owner = c + 32 * (r / 4 % 2);
                            float x = 0.f;
                            if constexpr (HALVES) {
                                uint32_t two = 0;            // as they are held for the product
#pragma unroll
                                for (int i = 0; i < 8 * PV; ++i) two = i == r / 16 * 4 + r / 8 % 2 * 2 + r / 2 % 2 ? w[i / 4][i % 4] : two;
                                two = __shfl(two, owner);
                                x = r % 2 ? V::hi(two) : V::lo(two);
                            } else {
                                const int held = r / 32 * 16 + r % 32 / 8 * 4 + r % 4;
#pragma unroll
                                for (int i = 0; i < 16 * PB; ++i) x = i == held ? s[i / 16][i % 16] : x;
                                x = __shfl(x, owner);
                            }
                            if (!(sees >> r & 1)) continue;
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                __builtin_amdgcn_sched_barrier(0);       // seldom run: few registers
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const u32x2 y = *reinterpret_cast<const u32x2 *>(v + r * PITCH + 16 * ((4 * (wave % SPLIT * DB + d) + i) ^ swirl(r)) + 8 * e);
                                    o[d][4 * i] += x * V::lo(y[0]);
                                    o[d][4 * i + 1] += x * V::hi(y[0]);
                                    o[d][4 * i + 2] += x * V::lo(y[1]);
                                    o[d][4 * i + 3] += x * V::hi(y[1]);
                                }
                            }
                        }
                        if (TEAM > 1) __syncthreads();
                        for (int r = part * MINE; r < (part + 1) * MINE; ++r)
                            if (spoilt_rows >> r & 1)
                                for (int x = lane; x < DK / 8; x += 64) *reinterpret_cast<u32x4 *>(v + r * PITCH + 16 * x) = u32x4{0, 0, 0, 0};
                        if (TEAM > 1) __syncthreads();
                        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    }
                }
                if (on) {
                    if constexpr (!HALVES) pack_weights(s, w, rest);
                    u32x4 v[AHEAD + 1];
#pragma unroll
                    for (int x = 0; x < AHEAD; ++x) v[x] = columns(va, x / DB / 2, x / DB % 2, x % DB);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int x = 0; x < 2 * PV * DB; ++x) {
                        const int y = x + AHEAD;
                        if (y < 2 * PV * DB) v[y % (AHEAD + 1)] = columns(va, y / DB / 2, y / DB % 2, y % DB);
                        o[x % DB] = mfma32<F16>(v[x % (AHEAD + 1)], w[x / DB], o[x % DB]);
                        if (PARTS) o[x % DB] = mfma32<F16>(v[x % (AHEAD + 1)], rest[x / DB], o[x % DB]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                if (more) put(buf ^ 1);
            }
        }
        const QueriesParams p = again();
        const int G = p.fd_G.d, block0 = piece.b * p.rows;
        if (bad && p.err) atomicOr(p.err, bad);
        l += __shfl_xor(l, 32);
        if constexpr (HALVES) {
            // each has the sum of its half of the positions
            __syncthreads();
            if (lane < 32) tops[wave * 32 + lane] = l;
            __syncthreads();
            l += tops[(wave ^ 1) * 32 + c];
        }

        // Join the wavefronts of the same rows: each scales to the common maximum, then they
        // add up in LDS, one after the other.
        if (TEAM == 1 && streams > 1) {
            if (e == 0) {
                ml[(wave * 32 + c) * 2] = m;
                ml[(wave * 32 + c) * 2 + 1] = l;
            }
            __syncthreads();
            const int w0 = wave - stream;
            float top = -INFINITY, sum = 0.f;
            for (int k = w0; k < w0 + streams; ++k) top = fmaxf(top, ml[(k * 32 + c) * 2]);
            for (int k = w0; k < w0 + streams; ++k) sum += ml[(k * 32 + c) * 2 + 1] * weight(ml[(k * 32 + c) * 2], top);
            const float f = weight(m, top);
            m = top;
            l = sum;
            // [head of the group][value / 4][lane]
            f32x4 *joined = reinterpret_cast<f32x4 *>(all_lds) + wave / streams * (64 * 4 * DB) + lane;
            for (int turn = 0; turn < streams; ++turn) {
                if (stream == turn) {
#pragma unroll
                    for (int d = 0; d < DB; ++d) {
                        o[d] *= f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            f32x4 x = {o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
                            if (turn > 0) x += joined[64 * (4 * d + i)];
                            if (turn < streams - 1) joined[64 * (4 * d + i)] = x;
#pragma unroll
                            for (int j = 0; j < 4; ++j) o[d][4 * i + j] = x[j];
                        }
                    }
                }
                __syncthreads();
            }
            if (stream != streams - 1) return;
        }
        const int ln = lane_again(), half = ln >> 5, x = x0 + (ln & 31);
        if (x >= h_rows) return;
        const int i = fd_div(p.fd_G, x), head = h * G + x - i * G;
        const int mine = 32 * DB * (wave % SPLIT);           // this wavefront's first value; a lane has 4 of every 8
        if (piece.place < 0) {
            const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * p.pool.H + h] : 1.f;
            const float f = l == 0.f ? 0.f : v_scale / l;
            if (p.lse && half == 0 && mine == 0)
                p.lse[(rec.row_off + i) * p.pool.H * G + head] =
                    l > 0.f || l != l ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
            // Values 0 .. 3 of an eight lie in one half of the wavefront, 4 .. 7 in the other: they swap
            // them, so that a lane stores whole eights, every second one: 256 rows of 128 take 2.5 us, 4.4 in
            // fours.
            char *dst = p.out.base + (rec.row_off + i) * p.out.s_row + head * p.out.s_head + 2 * (mine + 8 * half);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    u32x4 y;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const auto z = __builtin_amdgcn_permlane32_swap(
                            V::pack(o[d][4 * j + 2 * u] * f, o[d][4 * j + 2 * u + 1] * f),
                            V::pack(o[d][4 * j + 4 + 2 * u] * f, o[d][4 * j + 5 + 2 * u] * f), false, false);
                        y[u] = z[0];
                        y[2 + u] = z[1];
                    }
                    if (mine + 32 * d + 8 * (j + half) < p.Dv) *reinterpret_cast<u32x4 *>(dst + 64 * d + 16 * j) = y;
                }
        } else {
            const int64_t row = (piece.place * p.heads + (TEAM > 1 ? 0 : wave / streams)) * p.rows + x - block0;
            if (half == 0 && mine == 0) *reinterpret_cast<float2 *>(p.part_ml + 2 * row) = make_float2(m, l);
            // a wavefront's 1024 bytes side by side
            const int64_t block = row - (ln & 31);
            const int at = 4 * (2 * (ln & 31) + half);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (mine + 32 * d + 8 * j < p.Dv)
                        *reinterpret_cast<f32x4 *>(part_of(p, block, mine / 32 + d) + 256 * j + at) =
                            f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
        }
    }
};

// Two wavefronts lie on a SIMD.
template <bool F16, bool E4M3, int DK, int DV, int WAVES, int TEAM, int SPLIT, int TILE, bool GENERAL>
__global__ void __launch_bounds__(64 * WAVES, DK <= 128 || SPLIT > 1 ? 2 : 1) kvx_queries_kernel(QueriesParams p, int64_t first, int32_t n) {
    typedef Queries<F16, E4M3, DK, DV, TEAM, SPLIT, TILE, GENERAL> Work;
    __shared__ int64_t before[kQueriesGroup + 1];        // steps of one cache head of the records before
    __shared__ __align__(16) typename Work::Rows rows[WAVES / TEAM];
    __shared__ float depth[KVX_MAX_DRAFTS];              // every wavefront writes the same
    __shared__ typename Work::Sight sight[WAVES / SPLIT][32];
    __shared__ float tops[SPLIT > 1 ? WAVES * 32 : 1];
    __shared__ float ml[TEAM == 1 ? WAVES * 32 * 2 : 1];
    __shared__ int32_t flags[4][TEAM];
    __shared__ __align__(16) f32x4 shared[SPLIT == 1 ? 1 : DK <= 256 ? WAVES * 128 : WAVES * 256];
    extern __shared__ __align__(256) char lds[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int tile_bytes = TILE * 2 * DK * p.pool.C;
    Work work{rows[TEAM > 1 ? 0 : wave], depth, sight[wave / SPLIT], lds + (TEAM > 1 ? 0 : wave * 2 * tile_bytes), ml, flags, lds, shared, tops, lane, wave,
              TEAM > 1 ? wave : 0, lane & 31, lane >> 5, p.pool.C == 2, one_tile(DK, p.pool.C), tile_bytes};
    work.address();
    // Two wavefronts of a workgroup lie on a SIMD: with one of them preferred, their products and
    // the other's exponentials fall together, not products and products.
    if (WAVES == 8 && wave < 4) __builtin_amdgcn_s_setprio(1);
    const kvx_queries_req *reqs = p.whole ? p.reqs : p.reqs + first;
    int64_t at = first + blockIdx.x, stop = at + 1, each = 0;        // of units (whole), else of steps
    int share = 0;
    bool whole = p.whole;
    if (p.one) {
        const kvx_queries_req q = scalar(p.reqs[0]);
        stop = valid(q, p) ? (int64_t)blocks_of(q, p) * p.groups : 0;
        whole = stop >= kWholeUnits;
        if (whole && at == 0 && threadIdx.x == 0) *p.each = 0;
        if (!whole && at >= p.shares) return;
    }
    if (!whole) {
        // steps of a group of cache heads of the records before each
        if (p.blocks <= 8) {
            // few blocks a record: a thread each, whose reads are on their way together
            for (int r = threadIdx.x; r < n; r += 64 * WAVES) {
                const kvx_queries_req q = reqs[r];
                int64_t sum = 0;
                const int count = valid(q, p) ? blocks_of(q, p) : 0;
                for (int b = 0; b < count; ++b) sum += kUnitSteps + steps_of(span_of_block(q, p, b), p);
                before[r] = sum;
            }
        } else {
            for (int r = wave; r < n; r += WAVES) {
                const int64_t x = steps_of_group(scalar(reqs[r]), p, lane);
                if (lane == 0) before[r] = x;
            }
        }
        __syncthreads();
        if (wave == 0) {
            int64_t upto = 0;
            for (int r0 = 0; r0 < n; r0 += 64) {
                const int64_t x = r0 + lane < n ? before[r0 + lane] : 0;
                int64_t sum = x;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int64_t y = __shfl_up(sum, d);
                    if (lane >= d) sum += y;
                }
                if (r0 + lane < n) before[r0 + lane] = upto + sum - x;
                upto += __shfl(sum, 63);
            }
            if (lane == 0) before[n] = upto;
        }
        __syncthreads();
        // successive shares on one die
        share = p.shares % 8 == 0 ? blockIdx.x % 8 * (p.shares / 8) + blockIdx.x / 8 : blockIdx.x;
        const int64_t total = scalar(before[n]) * p.groups;
        each = share_of(total, p.shares);
        if (share == 0) {
            if (threadIdx.x == 0) *p.each = each;
            for (int r = threadIdx.x; r < n; r += blockDim.x)
                if (p.err && !valid(reqs[r], p)) atomicOr(p.err, KVX_DERR_BAD_REQ);
        }
        at = share * each;
        stop = at + each < total ? at + each : total;
        if (p.by_share && threadIdx.x == 0) p.cuts[share] = Cut{0, 0, -1, 0, 0, 0};
    }
    // the unit that was taken last, of a record that is kept
    Piece piece;
    int r = -1, blocks = 0;
    while (at < stop) {
        const QueriesParams p = again();
        const kvx_queries_req *reqs = p.whole ? p.reqs : p.reqs + first;
        Span s;
        int64_t here = gridDim.x;
        bool some = true;
        if (whole) {
            // Longest first: a record's last blocks see most.  Blocks of a record and group are n_reqs x groups
            // workgroups apart: with a multiple of 8 of them on one die, whose cache holds their keys.
            const int64_t lists = (int64_t)p.n_reqs * p.groups, rank = quotient(at, lists);
            // Of several records each die takes every eighth block, so that long ones are no die's alone.
            const int list = (int)((at - rank * lists + (p.n_reqs > 1 ? rank : 0)) % lists);
            r = list / p.groups;
            piece.group = list - r * p.groups;
            piece.rec = scalar(reqs[r]);
            if (!valid(piece.rec, p)) {
                if (rank == 0 && piece.group == 0 && threadIdx.x == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
                return;
            }
            blocks = blocks_of(piece.rec, p);
            if (rank >= blocks) return;
            piece.b = blocks - 1 - (int)rank;
            s = span_of_block(piece.rec, p, piece.b);
            piece.place = -1;
            piece.begin = s.lo & -kTile;
            piece.end = s.hi;
        } else {
            int64_t in = 0;              // steps of the unit before `at`
            if (r >= 0 && piece.b + 1 < blocks) {
                ++piece.b;
            } else {
                int lo = 0, hi = n;      // the record: the last one whose steps begin at or before `at`
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (before[mid] * p.groups <= at) lo = mid;
                    else hi = mid;
                }
                r = __builtin_amdgcn_readfirstlane(lo);
                const int64_t base = scalar(before[r]) * p.groups, per = scalar(before[r + 1]) - scalar(before[r]);
                piece.rec = scalar(reqs[r]);
                piece.group = (int)quotient(at - base, per);
                in = at - base - piece.group * per;
                blocks = blocks_of(piece.rec, p);
                for (int b0 = 0;; b0 += 64) {        // the block, of 64 at a time
                    const int mine = steps_of_lane(piece.rec, p, b0, lane, blocks);
                    int64_t upto = mine;
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) {
                        const int64_t y = __shfl_up(upto, d);
                        if (lane >= d) upto += y;
                    }
                    const uint64_t past = __ballot(upto > in);
                    if (past) {
                        const int lane_of = __ffsll((unsigned long long)past) - 1;
                        piece.b = b0 + lane_of;
                        in -= scalar(__shfl(upto - mine, lane_of));
                        break;
                    }
                    in -= scalar(__shfl(upto, 63));
                }
            }
            s = span_of_block(piece.rec, p, piece.b);
            const int steps = kUnitSteps + steps_of(s, p);
            here = stop - at < steps - in ? stop - at : steps - in;
            const int64_t first_tile = at - in + kUnitSteps;
            const int64_t from = in > kUnitSteps ? in - kUnitSteps : 0, to = in + here - kUnitSteps;     // tiles
            some = to > from;
            piece.place = from > 0 || to < steps - kUnitSteps ? place_of(first_tile, share, each, p.shares) : -1;
            piece.begin = (s.lo & -kTile) + (uint32_t)from * p.step;
            const uint32_t end = (s.lo & -kTile) + (uint32_t)to * p.step;
            piece.end = end < s.hi ? end : s.hi;
            if (threadIdx.x == 0 && (p.by_share ? in > kUnitSteps : some && from == 0))
                p.cuts[p.by_share ? share : (r * p.groups + piece.group) * p.blocks + piece.b] =
                    Cut{first_tile, at - in + steps - 1, r, piece.group, piece.b, 0};
        }
        if (s.hi <= s.lo) piece.end = piece.begin;
        if (some) work.run(piece);
        at += here;
        __syncthreads();                 // the next piece uses the same LDS
    }
}

template <bool F16, bool E4M3, int DK, int DV, int WAVES, int TEAM, int SPLIT, int TILE>
int launch_form(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream) {
    // few rows are bound by memory, and take one kernel for all scores
    const bool general = TEAM == 1 || p.cap > 0.f || p.slopes;
    const auto kernel = general ? kvx_queries_kernel<F16, E4M3, DK, DV, WAVES, TEAM, SPLIT, TILE, true>
                                : kvx_queries_kernel<F16, E4M3, DK, DV, WAVES, TEAM, SPLIT, TILE, TEAM == 1>;
    const size_t lds = (size_t)(one_tile(DK, p.pool.C) ? 1 : 2) * TILE * 2 * DK * p.pool.C * (p.waves / TEAM);
    hipLaunchKernelGGL(kernel, dim3((uint32_t)(p.whole ? n : p.one ? p.one : p.shares)), dim3(64 * p.waves), lds, stream, p, first, (int32_t)n);
    return hipGetLastError();
}

template <bool F16, bool E4M3>
int launch_type(const QueriesParams &p, int64_t first, int64_t n, hipStream_t stream) {
    const int D = p.pool.D;
    if (D > 256) return launch_form<F16, E4M3, 576, 512, 8, 8, 2, 32>(p, first, n, stream);
    if (p.team == 1) {
        if (D <= 64) return launch_form<F16, E4M3, 64, 64, 4, 1, 1, 32>(p, first, n, stream);
        if (D <= 128) return launch_form<F16, E4M3, 128, 128, 4, 1, 1, 32>(p, first, n, stream);
        return launch_form<F16, E4M3, 256, 256, 2, 1, 1, 32>(p, first, n, stream);
    }
    if (D <= 64) return launch_form<F16, E4M3, 64, 64, 8, 8, 1, 64>(p, first, n, stream);
    if (D <= 128)
        return p.team == 4 ? launch_form<F16, E4M3, 128, 128, 4, 4, 1, 64>(p, first, n, stream)
                           : launch_form<F16, E4M3, 128, 128, 8, 8, 1, 64>(p, first, n, stream);
    return launch_form<F16, E4M3, 256, 256, 8, 8, 2, 64>(p, first, n, stream);
}

}  // namespace

}  // namespace kvx
