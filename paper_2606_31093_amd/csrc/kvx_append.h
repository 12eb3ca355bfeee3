// kvx_append.h -- what the kernels that put new tokens into a paged cache share:
// the stores of a row's elements, and where a token's slot lies.
#pragma once

#include "kvx_ops.h"
#include "kvx_values.h"

namespace kvx {
namespace {

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

}  // namespace
}  // namespace kvx
