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

// Unsigned order of the weights, -0 as 0, with a key below and above all of
// them: 0 for what is not there, 1 for NaN, the largest for what is kept in any case.
constexpr uint32_t kAbsent = 0, kAlways = 0xffffffffu;
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = bits<uint32_t>(x + 0.f);          // -0 + 0 is 0
    return x != x ? 1 : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ bool inside(int64_t off, int64_t stride, int rows, int64_t n, int64_t len) {
    return off >= 0 && off <= len && n <= len - off && (rows == 1 || stride <= (len - off - n) / (rows - 1));
}

// Lanes below this one in a ballot.
__device__ __forceinline__ uint32_t below(uint64_t ballot) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(ballot >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)ballot, 0));
}

// Sum over this lane and those below it, by the moves of lanes within and across
// rows of 16.
__device__ __forceinline__ uint32_t sum_upto(uint32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);        // 1 lane up
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);        // 2
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);        // 4
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);        // 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);        // lane 15 of rows 0 and 2 to the next row
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);        // lane 31 to the upper half
    return x;
}

// A workgroup per record and row.  The keys lie in LDS, so that the choice reads the row
// once (KEEP; else they are made again in every pass, for rows too long for that).  A
// wavefront has a run of successive positions, four a lane.  The first and last
// positions have the largest key there is; then the n_keep largest are found
// digit by digit from the top, 11, 11 and 10 bits: count the digits of the keys that
// share the digits found so far, and take the digit in which the last kept key
// lies; when all of its keys are kept, the rest needs no look.  Then each
// wavefront counts what it keeps, and lists it behind what the ones before it keep;
// for acc_out it reads the row's weights a second time there, those not kept too.
// Bound by its instructions and the waits between its up to six passes: 1792 rows of 2048
// to 16384 positions (77 MB of weights, 29 MB of lists), 2048 kept of each, take 72 us;
// 77 vector instructions a key are half of that, and 114 to 125 MB are read from memory.
template <int THREADS, bool KEEP>
__global__ void __launch_bounds__(THREADS) kvx_select_kernel(SelectParams p, int32_t r0) {
    constexpr int WAVES = THREADS / 64, BINS = 2048, MINE = BINS / THREADS;
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ uint32_t hist[BINS];
    __shared__ uint32_t found[3], sums[WAVES], ties[WAVES];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
    const int r = r0 + (int)(blockIdx.x / (uint32_t)p.rows), j = (int)(blockIdx.x % (uint32_t)p.rows);
    const kvx_select_req q = p.reqs[r];
    const int64_t kept_n = q.n_tokens < q.n_keep ? q.n_tokens : q.n_keep;
    if (q.n_tokens < 0 || q.n_keep < 0 || q.sink < 0 || q.recent < 0 || q.n_tokens > p.max_tokens ||
        (int64_t)q.sink + q.recent > q.n_keep || !inside(q.acc_off, p.acc_stride, p.rows, q.n_tokens, p.acc_len) ||
        !inside(q.kept_off, p.kept_stride, p.rows, kept_n, p.kept_len) ||
        (p.out && !inside(q.out_off, p.out_stride, p.rows, kept_n, p.out_len)) ||
        (p.rows > 1 && (p.kept_stride < kept_n || (p.out && p.out_stride < kept_n)))) {      // rows would meet
        if (j == 0 && tid == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        return;
    }
    const float *acc = p.acc + q.acc_off + j * p.acc_stride;
    int32_t *kept = p.kept + q.kept_off + j * p.kept_stride;
    float *out = p.out ? p.out + q.out_off + j * p.out_stride : nullptr;
    const int n = q.n_tokens;
    if (n <= q.n_keep) {
        for (int t = tid; t < n; t += THREADS) {
            kept[t] = t;
            if (out) out[t] = acc[t];
        }
        return;
    }
    const int turns = (n + 4 * THREADS - 1) / (4 * THREADS);        // of 256 positions a wavefront
    const int t0 = wave * turns * 256 + 4 * lane;
    const auto key_at = [&](int t) {
        if (t >= n) return kAbsent;
        return t < q.sink || t >= n - q.recent ? kAlways : key_of(acc[t]);
    };
    if (KEEP) {
        const int padded = turns * 4 * THREADS;
#pragma unroll 4
        for (int t = tid; t < padded; t += THREADS) keys[t] = key_of(acc[t < n ? t : n - 1]);
        __syncthreads();
        for (int t = tid; t < q.sink; t += THREADS) keys[t] = kAlways;
        for (int t = n - q.recent + tid; t < n; t += THREADS) keys[t] = kAlways;
        for (int t = n + tid; t < padded; t += THREADS) keys[t] = kAbsent;
    }
    // f(first position, keys) for this lane's positions, in order
    const auto each = [&](const auto &f) {
        for (int i = 0; i < turns; ++i) {
            if ((wave * turns + i) * 256 >= n) break;
            const int t = t0 + 256 * i;
            u32x4 k;
            if (KEEP) k = *reinterpret_cast<const u32x4 *>(keys + t);
            else k = u32x4{key_at(t), key_at(t + 1), key_at(t + 2), key_at(t + 3)};
            f(t, k);
        }
    };

    // kept: keys above `prefix`, and the first `need` equal to it
    uint32_t need = q.n_keep, prefix = 0;                // < n
    if (need == 0) return;
    bool crowded = true;                                 // many keys share the digits found
    for (int shift = 21, width = 11;;) {
        for (int i = tid; i < BINS; i += THREADS) hist[i] = 0;
        __syncthreads();
        if (crowded) {
            // Lanes with the digit of the first one are counted together: equal weights
            // (zeros, say) would be added one after the other.
            each([&](int, u32x4 k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool on = shift == 21 || k[i] >> (shift + width) == prefix >> (shift + width);
                    const uint64_t all = __ballot(on);
                    if (all == 0) continue;
                    const uint32_t d = k[i] >> shift & ((1u << width) - 1);
                    const int leader = __builtin_ctzll(all);
                    const uint32_t d0 = __builtin_amdgcn_readlane(d, leader);
                    const uint64_t same = __ballot(on && d == d0);
                    if (on && (d != d0 || lane == leader))
                        atomicAdd(&hist[d], lane == leader ? (uint32_t)__popcll(same) : 1u);
                }
            });
        } else {
            each([&](int, u32x4 k) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k[i] >> (shift + width) == prefix >> (shift + width))
                        atomicAdd(&hist[k[i] >> shift & ((1u << width) - 1)], 1u);
            });
        }
        __syncthreads();
        // thread x: MINE digits, the larger ones before the smaller ones
        uint32_t part[MINE], sum = 0;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            part[i] = hist[BINS - 1 - MINE * tid - i];
            sum += part[i];
        }
        uint32_t above = sum_upto(sum);
        if (lane == 63) sums[wave] = above;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES - 1; ++w) above += w < wave ? sums[w] : 0;       // all read at once
        above -= sum;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            if (above < need && above + part[i] >= need) {
                found[0] = BINS - 1 - MINE * tid - i;
                found[1] = above + part[i] == need ? 0 : need - above;
                found[2] = part[i];
            }
            above += part[i];
        }
        __syncthreads();
        prefix |= found[0] << shift;
        need = found[1];
        crowded = found[2] > 4 * THREADS;
        if (need == 0) --prefix;                         // all of them; not 0, the key of none that is there
        if (need == 0 || shift == 0) break;
        width = shift == 21 ? 11 : 10;
        shift -= width;
    }

    uint32_t mine = 0, equal = 0;
    each([&](int, u32x4 k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            mine += __popcll(__ballot(k[i] > prefix));
            equal += __popcll(__ballot(k[i] == prefix));
        }
    });
    if (lane == 0) {
        sums[wave] = mine;
        ties[wave] = equal;
    }
    __syncthreads();
    uint32_t at = 0, rank = 0;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w) {
        at += w < wave ? sums[w] : 0;
        rank += w < wave ? ties[w] : 0;
    }
    at += rank < need ? rank : need;
    each([&](int t, u32x4 k) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = out ? acc[t + i < n ? t + i : n - 1] : 0.f;
        bool take[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) take[i] = k[i] > prefix;
        if (rank < need) {                               // ties are left: the first ones in order
            uint32_t mine = rank, all = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t b = __ballot(k[i] == prefix);
                mine += below(b);
                all += __popcll(b);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool tie = k[i] == prefix;
                take[i] = take[i] || (tie && mine < need);
                mine += tie;
            }
            rank += all;
        }
        uint32_t to = at;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t b = __ballot(take[i]);
            to += below(b);
            at += __popcll(b);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!take[i]) continue;
            *reinterpret_cast<int32_t *>(reinterpret_cast<char *>(kept) + 4 * to) = t + i;
            if (out) *reinterpret_cast<float *>(reinterpret_cast<char *>(out) + 4 * to) = x[i];
            ++to;
        }
    });
}

// ---------------------------------------------------------------------------
// move
// ---------------------------------------------------------------------------

constexpr int kRows = 64;            // list entries of a workgroup at most

// A workgroup per p.rows entries of one list (a record's layer and head): their
// source and destination rows are resolved once, then copied 16 bytes a lane,
// keys and values.  Bound by the memory: 1792 lists of up to 2048 rows of 256 bytes, 3.8 GB
// read and written, take 715 us, 5.2 TB/s (750 us through the caches; four rows a
// lane on their way at a time 719, eight 814).  Copies in the order of pages reach
// 6.1 to 6.4 TB/s.
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
    const int first = piece * p.rows;
    if (first >= n) return;
    const int rows = (int)(n - first < p.rows ? n - first : p.rows);
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
            const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(src + from[i] + 16 * v));
            __builtin_nontemporal_store(w, reinterpret_cast<u32x4 *>(dst + to[i] + 16 * v));
        }
        src += p.src.s_c;
        dst += p.dst.s_c;
    }
}

}  // namespace

// Threads of a workgroup, by the longest row there may be: 288 rows of 1500 took 8.5 us
// with 512 (9.0 with 256, and 10 with 1024), 1792 rows of 2048 to 16384 71 us with 1024
// (81 with 512).  1792 and 288 rows of 8192 took 46.8 and 16.1 us with 512, 51.5 and 16.3
// with 1024; of 12000 80.7 and 21.7 with 512, 67.2 and 21.0 with 1024.
int select_threads(int max_tokens) { return max_tokens <= 8192 ? 512 : 1024; }

// The longest row whose keys lie in LDS (128 KiB): 1792 and 288 rows of 32768 took 234 and
// 60 us, and without it 370 and 97.  1792 of 40000 take 428 us, of 131072 1308.
constexpr int kMostKeys = 32768;

auto pick_select(int threads, bool keep) {
    if (threads == 512) return kvx_select_kernel<512, true>;
    return keep ? kvx_select_kernel<1024, true> : kvx_select_kernel<1024, false>;
}

int launch_select(const SelectParams &p, hipStream_t stream) {
    const int threads = select_threads(p.max_tokens);
    const bool keep = p.max_tokens <= kMostKeys;
    const auto kernel = pick_select(threads, keep);
    const int lds = keep ? (p.max_tokens + 4 * threads - 1) / (4 * threads) * 16 * threads : 0;
    const int64_t group = kMaxBlocks / p.rows > 0 ? kMaxBlocks / p.rows : 1;
    for (int64_t r0 = 0; r0 < p.n_reqs; r0 += group) {
        const int64_t n = p.n_reqs - r0 < group ? p.n_reqs - r0 : group;
        hipLaunchKernelGGL(kernel, dim3((uint32_t)(n * p.rows)), dim3(threads), lds, stream, p, (int32_t)r0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

int launch_kept(const KeptParams &p0, hipStream_t stream) {
    if (p0.n_reqs == 0) return hipSuccess;
    KeptParams p = p0;
    // The longest list shapes the launch: one of 8192 entries among 256 of one (4 layers of 8
    // heads) takes 1035 us, alone it takes 50.  The vectors of a workgroup's entries are counted
    // in 31 bits: fewer entries where rows have 512 MiB and more.
    const int32_t fit = (INT32_MAX - kThreads) / p.vpr;
    p.rows = fit < kRows ? fit : kRows;
    // with max_tokens 0 one too: it looks whether the record is malformed
    const int32_t pieces = p.max_tokens > 0 ? (p.max_tokens + p.rows - 1) / p.rows : 1;
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
