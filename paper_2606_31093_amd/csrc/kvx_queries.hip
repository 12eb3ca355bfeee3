// kvx_queries.hip -- attention of several queries of a request over a paged cache
// (gfx950): the division of the work, the launches, and the second kernel, which
// joins the parts of units that lie in several shares.
//
// A unit is a block of rows of one record and group of cache heads, and its steps are
// the tiles that some row of it sees.  Either every unit has a workgroup of its own, or
// the launch's steps are dealt out in equal shares, one to each workgroup that the device
// holds at a time, and a unit that lies in several shares leaves a part (maximum, sum,
// values, in 32 bits) in each.  Which, is a rule on sizes alone, and of one long record on what
// it holds, so that a captured launch serves other lengths; the shares themselves come from the
// records, on the device.

#include "kvx_queries.h"

namespace kvx {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// A wavefront joins 32 rows x 32 values of a unit, or fewer rows and more values: out = sum 2^(m_c - M) o_c / sum 2^(m_c - M) l_c.
// `split` wavefronts share the parts and add up in LDS.  Of 32 values lane 2 c + e has 8 j + 4 e .. + 3
// (j < 4) of row c, as the first kernel's lane (c, e) stored them, a kilobyte side by side: one
// tree of 60 drafts behind 32768 positions, 256 shares, takes 63 us so, and 67 with parts that lie
// row by row, 32 trees of 16 96 and 105, MLA's 149 and 160; a batch of single tokens 127 and 126.
template <bool F16>
__global__ void __launch_bounds__(kThreads) kvx_queries_join_kernel(QueriesParams p, int64_t r0, int32_t runs, int32_t split,
                                                                    int32_t lines, int32_t row_blocks) {
    __shared__ f32x4 sums[kWaves][4][64];
    __shared__ float2 tops[kWaves][64];
    const int64_t each = *p.each;
    if (each == 0) return;
    const int id = blockIdx.x / (uint32_t)runs, run = blockIdx.x - id * runs, H = p.pool.H, G = p.fd_G.d;
    const Cut u = p.cuts[id];                            // by units, of no meaning where there is no such unit
    const int list = id / p.blocks, of = p.by_share ? u.record : list / p.groups;
    if (of < 0) return;
    const kvx_queries_req rec = p.reqs[r0 + of];
    const int b = p.by_share ? u.block : id - list * p.blocks, group = p.by_share ? u.group : list - of * p.groups;
    if (!valid(rec, p) || b >= blocks_of(rec, p)) return;
    // Parts in shares k0 .. k1; of those that begin inside the unit the first is its own.
    const int64_t k0 = quotient(u.first, each), k1 = quotient(u.last, each);
    if (k0 == k1 || (p.by_share && id != k0 + 1)) return;        // one part: written by the first launch
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, c = lane / 2 % lines, e = lane % 2;
    const int item = (run * kWaves + wave) / split, mine = wave % split, side = 32 / lines;
    const int wide = wide_blocks(p.Dv), turns = (wide + side - 1) / side;
    const int d = item % turns * side + lane / 2 / lines, rb = item / turns % row_blocks, head_of = item / turns / row_blocks;
    const int64_t row = (int64_t)b * p.rows + rb * 32 + c;
    const bool on = head_of < p.heads && d < wide && row < (int64_t)rec.n_queries * G;
    float m = -INFINITY, l = 0.f;
    f32x4 sum[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (on) {
        const int64_t slots = p.heads * p.rows, slot = head_of * p.rows + rb * 32;
        for (int64_t k = k0 + mine; k <= k1; k += 2 * split) {
            f32x4 y[2][4];
            float2 ml[2];
            // all on their way at once
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                ml[i] = make_float2(-INFINITY, 0.f);
#pragma unroll
                for (int j = 0; j < 4; ++j) y[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (k + i * split > k1) continue;
                const int64_t at = place_of(u.first, k + i * split, each, p.shares) * slots + slot;
                ml[i] = *reinterpret_cast<const float2 *>(p.part_ml + 2 * (at + c));
                const float *from = part_of(p, at, d) + 4 * (2 * c + e);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (32 * d + 8 * j < p.Dv) y[i][j] = __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(from + 256 * j));
            }
            const float top = fmaxf(m, fmaxf(ml[0].x, ml[1].x)), f = weight(m, top), w0 = weight(ml[0].x, top), w1 = weight(ml[1].x, top);
            m = top;
            l = l * f + ml[0].y * w0 + ml[1].y * w1;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = sum[j] * f + y[0][j] * w0 + y[1][j] * w1;
        }
    }
    if (split > 1) {
        tops[wave][lane] = make_float2(m, l);
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[wave][j][lane] = sum[j];
        __syncthreads();
        if (mine != 0) return;
        float top = m;
        for (int k = 1; k < split; ++k) top = fmaxf(top, tops[wave + k][lane].x);
        const float f = weight(m, top);
        l *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] *= f;
        for (int k = 1; k < split; ++k) {
            const float w = weight(tops[wave + k][lane].x, top);
            l += tops[wave + k][lane].y * w;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] += sums[wave + k][j][lane] * w;
        }
        m = top;
    }
    if (!on) return;
    const int h = group * p.heads + head_of, i = (int)fd_div(p.fd_G, (uint32_t)row), head = h * G + (int)(row - (int64_t)i * G);
    if (p.lse && d == 0 && e == 0)
        p.lse[(rec.row_off + i) * H * G + head] =
            l > 0.f || l != l ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
    const float v_scale = p.scales ? p.scales[(p.pool.C - 1) * H + h] : 1.f;
    const float f = l == 0.f ? 0.f : v_scale / l;
    char *dst = p.out.base + (rec.row_off + i) * p.out.s_row + head * p.out.s_head + 2 * (32 * d + 8 * e);
#pragma unroll
    for (int j = 0; j < 4; j += 2) {                     // whole eights, every second one a lane's
        u32x2 x[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const f32x4 y = sum[j + k] * f;
            x[k] = u32x2{Half<F16>::pack(y[0], y[1]), Half<F16>::pack(y[2], y[3])};
        }
        const u32x2 own = e ? x[1] : x[0], give = e ? x[0] : x[1];
        const u32x2 got = {(uint32_t)__shfl_xor((int)give[0], 1), (uint32_t)__shfl_xor((int)give[1], 1)};
        if (32 * d + 8 * (j + e) < p.Dv)
            *reinterpret_cast<u32x4 *>(dst + 16 * j) = e ? u32x4{got[0], got[1], own[0], own[1]} : u32x4{own[0], own[1], got[0], got[1]};
    }
}

// Workgroups that the device holds at a time, by their LDS and registers: its 256 compute
// units have room for one, or for two of four wavefronts.
int resident(const QueriesParams &p) { return (p.team == 4 && p.pool.D <= 128) || (p.team == 1 && p.pool.D <= 64) ? 512 : 256; }
// Units of up to this many steps are not split: a share's search and the join would cost more.
constexpr int kWholeSteps = 8;
// Nor are kWholeUnits and more of one record, or of short ones: the device deals them out as it
// gets free, and those of one cache head, that run at the same time on one die, find their keys in
// its cache.  A prompt of 8192 (32 heads of 128 on 8: 1024 units) takes 547 us so and 575 in shares,
// one of 16384 2150 and 2250, 32 of 512 164 and 181.  Fewer units are uneven among the compute units
// where all see about as much: 288 behind 60000 positions take 3710 so and 2400 in shares, though a
// prompt of 4096 152 and 177, whose last blocks are short.  Longer ragged records leave compute units
// without work at the end: 16 of 333 to 2000, e4m3 and biased, take 495 so and 387 in shares, four
// of 1500 81 and 57.
//
// The units counted here are those of the limits, records may hold fewer.  A workgroup without a
// unit takes 3 ns, so that short records have at most so many of them beside each record's first
// block, and shares beyond: under limits of 2^20 queries 32 prompts of 256 take 70 us, 26900 otherwise.
// With that many units shares are as fast: 64 prompts of 1000 971 us, whole 984.
constexpr int kWholeMore = 8192;
// One record's kernel looks how many units there are, and takes one or the other: at most so many
// workgroups, which go on to a further unit.  One query behind 131072 positions takes 138 us under limits
// of 16384 (2450 with a workgroup a unit), a chunk of 512 behind 100000 800 (2540); a prompt of 16384
// 2057, and 2042 without the look and the second launch, in which nothing is left to do (5 us).
constexpr int kOneBlocks = 2048;
static_assert(kOneBlocks >= 512, "as many as shares");
// Records of up to this many positions: four wavefronts a workgroup, two of which begin and
// end at different times, so that one computes while the other waits for its first tile.  16
// prompts of 512 take 94 us, 102 in eights; one of 300 16.2 and 18.6.  Longer ones share a tile
// among eight: uniform ones of 2000 642 us and 672 in fours, one of 16384 2163 and 2273.
constexpr int kShort = 1024;
// Fewer steps than this are not worth a share: its way to the first tile takes as long.
constexpr int kLeastShare = 4;

int tile_of(const QueriesParams &p) { return p.team == 1 || p.pool.D > 256 ? 32 : 64; }

// The kernel for records of up to `most` rows a cache head, and its shape.
void shape(QueriesParams &p, int64_t most) {
    const int D = p.pool.D;
    // Up to 32 rows: wavefronts take positions of their own; as many as LDS holds tiles for.  Up to
    // 128: four share a tile.  Rows wider than 256 always have eight, in pairs.
    p.team = D > 256 ? 8 : most <= 32 ? 1 : D > 64 && D <= 128 && (most <= 128 || p.max_tokens <= kShort) ? 4 : 8;
    p.waves = p.team > 1 ? p.team : D <= 128 ? 4 : 2;
    p.rows = D > 128 && p.team > 1 ? 128 : 32 * p.team;      // two wavefronts for 32 wide rows
    // Rows of the cache that lie side by side, several heads of a position, are read by one workgroup.
    p.heads = 1;
    while (p.team == 1 && p.token_major && 2 * p.heads <= p.waves && p.pool.H % (2 * p.heads) == 0) p.heads *= 2;
    p.groups = p.pool.H / p.heads;
    p.step = tile_of(p) * (p.team > 1 ? 1 : p.waves / p.heads);
    p.blocks = (int32_t)((most + p.rows - 1) / p.rows);
    if (p.blocks < 1) p.blocks = 1;
}

int64_t most_steps(const QueriesParams &p) { return ((int64_t)p.max_tokens + kTile - 1 + p.step - 1) / p.step; }

// Shares for so many units of the longest records.
int32_t shares_for(const QueriesParams &p, int64_t units) {
    const int64_t steps = most_steps(p), n = (units * (steps > 0 ? steps : 1) + kLeastShare - 1) / kLeastShare;
    return (int32_t)(n < resident(p) ? (n > 0 ? n : 1) : resident(p));
}

// Workspace of the shares.
int64_t split_bytes(const QueriesParams &p) {
    // two parts a share, its first and its last
    const int64_t rows = 2 * (int64_t)p.shares * p.heads * p.rows;
    return 64 + (int64_t)p.shares * (int64_t)sizeof(Cut) + rows * 8 + rows * wide_blocks(p.Dv) * 128;
}

int64_t units_of(const QueriesParams &p) {
    return (p.n_reqs < kQueriesGroup ? p.n_reqs : (int64_t)kQueriesGroup) * p.groups * p.blocks;
}

}  // namespace

void plan_queries(QueriesParams &p) {
    shape(p, (int64_t)p.max_queries * p.fd_G.d);
    const int64_t units = (int64_t)p.n_reqs * p.groups * p.blocks;
    const bool many = units >= kWholeUnits;
    p.whole = (most_steps(p) <= kWholeSteps || (many && p.max_tokens <= kShort)) &&
              units - (int64_t)p.n_reqs * p.groups <= kWholeMore;
    const int64_t most = kOneBlocks < kMaxBlocks ? kOneBlocks : kMaxBlocks;
    p.one = !p.whole && many && p.n_reqs == 1 ? (int32_t)(units < most ? units : most) : 0;
    p.shares = shares_for(p, units_of(p));
    p.by_share = units_of(p) > p.shares;
}

int64_t queries_workspace_most(const QueriesParams &p0) {
    // Fewer queries may take another kernel, fewer records or positions fewer shares.
    const int64_t most = (int64_t)p0.max_queries * p0.fd_G.d;
    int64_t bytes = 0;
    for (const int64_t rows : {most < 32 ? most : 32, most < 128 ? most : 128, most})
        for (const int32_t tokens : {p0.max_tokens, p0.max_tokens < kShort ? p0.max_tokens : kShort}) {
            QueriesParams p = p0;
            p.max_tokens = tokens;
            shape(p, rows);
            p.shares = shares_for(p, units_of(p));
            const int64_t need = split_bytes(p);
            if (need > bytes) bytes = need;
        }
    return bytes;
}

int64_t queries_workspace(QueriesParams &p, char *base) {
    int64_t at = 0;
    const auto take = [&](int64_t bytes) {
        char *x = base ? base + at : nullptr;
        at += (bytes + 15) / 16 * 16;
        return x;
    };
    const int64_t rows = 2 * (int64_t)p.shares * p.heads * p.rows;
    if (p.whole) return at;
    p.each = reinterpret_cast<int64_t *>(take(16));
    p.cuts = reinterpret_cast<Cut *>(take(p.shares * (int64_t)sizeof(Cut)));
    p.part_ml = reinterpret_cast<float *>(take(rows * 8));
    p.part_o = reinterpret_cast<float *>(take(rows * wide_blocks(p.Dv) * 128));
    return at;
}

int launch_queries(const QueriesParams &p, hipStream_t stream) {
    const auto launch = p.f16 ? (p.e4m3 ? launch_queries_f16_e4m3 : launch_queries_f16)
                              : (p.e4m3 ? launch_queries_bf16_e4m3 : launch_queries_bf16);
    int e;
    if (p.whole) {
        const int64_t units = (int64_t)p.n_reqs * p.groups * p.blocks;
        for (int64_t at = 0; at < units; at += kMaxBlocks) {
            const int64_t n = units - at < kMaxBlocks ? units - at : kMaxBlocks;
            if ((e = launch(p, at, n, stream)) != hipSuccess) return e;
        }
        return hipSuccess;
    }
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += kQueriesGroup) {
        const int64_t n = p.n_reqs - r0 < kQueriesGroup ? p.n_reqs - r0 : kQueriesGroup;
        if ((e = launch(p, r0, n, stream)) != hipSuccess) return e;
        const int64_t units = n * p.groups * p.blocks;
        if (p.shares > 1) {
            // Wavefronts that share the parts: as many as there are pairs of them, on average.
            int split = 1;
            while (split < kWaves && units * 2 * split < p.shares) split *= 2;
            const int64_t most = (int64_t)p.max_queries * p.fd_G.d;
            const int32_t row_blocks = ((most < p.rows ? (int)most : p.rows) + 31) / 32;
            int32_t lines = 1;
            while (lines < 32 && lines < most) lines *= 2;
            const int32_t turns = (wide_blocks(p.Dv) * lines + 31) / 32;
            const int32_t runs = (p.heads * row_blocks * turns * split + kWaves - 1) / kWaves;
            hipLaunchKernelGGL(p.f16 ? kvx_queries_join_kernel<true> : kvx_queries_join_kernel<false>,
                               dim3((uint32_t)((p.by_share ? p.shares : units) * runs)), dim3(kThreads), 0, stream, p, r0, runs, split,
                               lines, row_blocks);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace kvx
