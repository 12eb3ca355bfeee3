// kvx_attend.h -- what the attention kernels share: weights, the checks of a
// record, and the division of all records' steps among the workgroups.
#pragma once

#include "kvx_ops.h"
#include "kvx_values.h"

namespace kvx {
namespace {

constexpr int kTile = 32;               // tiles begin at multiples of this
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
    // one accumulator for each head and position: heads that shared one would add to it at the same time
    if (p.pool.H > 1 && p.acc_stride < q.end - q.start) return false;
    // accumulators [acc_off + start, acc_off + (H - 1) * stride + end) lie inside
    return q.acc_off >= 0 && q.acc_off <= p.acc_len && q.end <= p.acc_len - q.acc_off &&
           (p.pool.H == 1 || p.acc_stride <= (p.acc_len - q.acc_off - q.end) / (p.pool.H - 1));
}

// Steps of a record: one for every `step` positions from the tile in which it
// begins; one for a record without positions (for its zeros), none if malformed.
__device__ __forceinline__ int steps_of(const kvx_attend_req &q, const AttendParams &p) {
    if (!valid(q, p)) return 0;
    const int n = q.end - (q.start & -kTile);
    return q.end > q.start ? (n + p.step - 1) / p.step : 1;
}

// before[r] = steps of the launch's records 0 .. r-1, one cache head block's;
// the last entry is the total.  All threads, 64 to 512.
__device__ __forceinline__ void add_up(const AttendParams &p, int32_t r0, int32_t n, int32_t *before) {
    __shared__ int32_t waves[8];
    const int tid = threadIdx.x, lane = tid % 64;
    const int threads = blockDim.x, each = (n + threads - 1) / threads;      // records a thread
    int32_t sum = 0;
    for (int r = tid * each; r < (tid + 1) * each && r < n; ++r) {
        before[r] = steps_of(p.reqs[r0 + r], p);
        sum += before[r];
    }
    int32_t upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int32_t x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 63) waves[tid / 64] = upto;
    __syncthreads();
    for (int w = 0; w < tid / 64; ++w) upto += waves[w];
    upto -= sum;
    for (int r = tid * each; r < (tid + 1) * each && r < n; ++r) {
        const int32_t x = before[r];
        before[r] = upto;
        upto += x;
    }
    if (tid == threads - 1) before[n] = upto;
    __syncthreads();
}

// a / b for a >= 0, b > 0; 32 bits nearly always do, in a fraction of the time.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// A share of the steps of all units (unit: record r of the launch, block hb of
// its `per` head blocks; in order of r, then hb).
struct Shares {
    int64_t total, each;
    __device__ __forceinline__ Shares(const AttendParams &p, int32_t steps) : total((int64_t)steps * p.per) {
        each = quotient(total + p.shares - 1, p.shares);
        if (each < 1) each = 1;
    }
    // Where the part of a unit that begins at step `first` of all lies among the
    // partial results when share k holds it: a share's first part has the
    // place k, one that begins inside it place shares + k.
    __device__ __forceinline__ int64_t place(const AttendParams &p, int64_t first, int64_t k) const {
        return first > k * each ? p.shares + k : k;
    }
};

// A workgroup's part of a unit: positions [begin, end) of a record's head block,
// and the place of its partial results (-1: it is the whole unit).
struct Part {
    kvx_attend_req rec;          // by value: read where it is, it would be read again after every store
    int32_t r, hb;
    uint32_t begin, end;         // unsigned: a step may end past 2^31 - 1, the last position there is
    int64_t place;
};

// The same record in scalar registers (loaded, it comes in vector registers).
__device__ __forceinline__ kvx_attend_req scalar(const kvx_attend_req &q) {
    uint32_t w[6];
    __builtin_memcpy(w, &q, sizeof w);
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = __builtin_amdgcn_readfirstlane(w[i]);
    kvx_attend_req s;
    __builtin_memcpy(&s, w, sizeof w);
    return s;
}

// The parts of a workgroup's share, in order.  Uniform over the workgroup.
struct Walk {
    int64_t at, stop;            // units (p.whole), or steps of all units in order
    int32_t r0, n, share;
    // `id`: the unit (p.whole) or the share.  All threads, 64 to 512.
    __device__ __forceinline__ Walk(const AttendParams &p, int32_t r0_, int32_t n_, int32_t *before, int32_t id)
        : at(id), stop(at + 1), r0(r0_), n(n_), share(id) {
        if (p.whole) {
            if (at >= (int64_t)n * p.per) stop = at;
            return;
        }
        add_up(p, r0, n, before);
        if (share == 0) {
            for (int r = threadIdx.x; r <= n; r += blockDim.x) p.before[r] = before[r];
            for (int r = threadIdx.x; r < n; r += blockDim.x)
                if (before[r] == before[r + 1] && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
        }
        const Shares s(p, before[n]);
        at *= s.each;
        stop = share >= p.shares ? at : at + s.each < s.total ? at + s.each : s.total;
    }
    __device__ __forceinline__ bool next(const AttendParams &p, const int32_t *before, Part *part) {
        if (at >= stop) return false;
        int step0 = 0, here;
        part->place = -1;
        if (p.whole) {
            part->r = r0 + (int)(at / p.per);
            part->hb = (int)(at % p.per);
            part->rec = scalar(p.reqs[part->r]);
            at = stop;
            here = steps_of(part->rec, p);
            if (here == 0) {
                if (part->hb == 0 && threadIdx.x == 0 && p.err) atomicOr(p.err, KVX_DERR_BAD_REQ);
                return false;
            }
        } else {
            // the record: the last one whose steps begin at or before `at`
            int lo = 0, hi = n;
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if ((int64_t)before[mid] * p.per <= at) lo = mid;
                else hi = mid;
            }
            const int r = __builtin_amdgcn_readfirstlane(lo);
            const int base = __builtin_amdgcn_readfirstlane(before[r]);
            const int steps = __builtin_amdgcn_readfirstlane(before[r + 1]) - base;
            const int64_t in = at - (int64_t)base * p.per;
            part->r = r0 + r;
            part->rec = scalar(p.reqs[part->r]);
            part->hb = (int)quotient(in, steps);
            step0 = (int)(in - (int64_t)part->hb * steps);
            here = stop - at < steps - step0 ? (int)(stop - at) : steps - step0;
            if (here < steps)
                part->place = Shares(p, before[n]).place(p, (int64_t)base * p.per + (int64_t)part->hb * steps, share);
            at += here;
        }
        part->begin = (part->rec.start & -kTile) + (uint32_t)step0 * p.step;
        const uint32_t to = part->begin + (uint32_t)here * p.step;
        part->end = to < (uint32_t)part->rec.end ? to : part->rec.end;
        return true;
    }
};

// Eight weights in two parts of the rows' type, for a product each, so that their
// rounding is kRest of one to the type: rounded once, weights cost an output as
// much as its own rounding does.  `a` is less than w by about kRest of it: the rest
// is then not zero where w is not, and an infinite value times it is not NaN.  (In
// half, whose smallest value is 2^-24, that holds from 2^-21 on, 2^-28 of the
// largest weight.)
template <bool F16>
constexpr float kRest = F16 ? 1.0f / 16 : 1.0f / 256;
template <bool F16>
__device__ __forceinline__ void split(const float *w, u32x4 &a, u32x4 &rest) {
    typedef Half<F16> V;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = V::pack(w[2 * i] * (1 - kRest<F16>), w[2 * i + 1] * (1 - kRest<F16>));
        rest[i] = V::pack(w[2 * i] - V::lo(a[i]), w[2 * i + 1] - V::hi(a[i]));
    }
}

template <bool F16, bool E4M3>
__device__ __forceinline__ u32x4 widen(const uint32_t *w) {
    if (E4M3)
        return u32x4{Half<F16>::template from_e4m3<false>(w[0]), Half<F16>::template from_e4m3<true>(w[0]),
                     Half<F16>::template from_e4m3<false>(w[1]), Half<F16>::template from_e4m3<true>(w[1])};
    return u32x4{w[0], w[1], w[2], w[3]};
}

}  // namespace

// Launches the first kernel of kvx_attend for records r0 .. r0 + n - 1 of heads
// of up to 256, or of more.
int launch_attend_narrow(const AttendParams &p, int32_t r0, int32_t n, hipStream_t stream);
int launch_attend_wide(const AttendParams &p, int32_t r0, int32_t n, hipStream_t stream);
void plan_attend_wide(AttendParams &p);

}  // namespace kvx
