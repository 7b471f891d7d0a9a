// Reductions over a wavefront's lanes that stay in registers: a row of 16 lanes turns by data-parallel moves, rows change places by
// permlane16_swap and permlane32_swap.  (A step through LDS, as __shfl_xor takes, waits about a hundred clocks for its result.)
#pragma once
#include "common.h"

#define RS_LANES __device__ __forceinline__

struct larger_of { template <typename T> RS_LANES T operator()(T a, T b) const { return a > b ? a : b; } };
struct smaller_of { template <typename T> RS_LANES T operator()(T a, T b) const { return a < b ? a : b; } };
struct sum_of { template <typename T> RS_LANES T operator()(T a, T b) const { return a + b; } };
template <> RS_LANES float larger_of::operator()(float a, float b) const { return fmaxf(a, b); }
template <> RS_LANES float smaller_of::operator()(float a, float b) const { return fminf(a, b); }

// Of lanes i, i + 16, i + 32 and i + 48, in all of them.
template <typename Op, typename T>
RS_LANES T of_quarters(T x, Op op) {
    // (the halves by name: __builtin_bit_cast of a vector's element takes its first)
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const uint32_t a0 = a[0], a1 = a[1];
    const uint32_t v = __builtin_bit_cast(uint32_t, op(__builtin_bit_cast(T, a0), __builtin_bit_cast(T, a1)));
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t b0 = b[0], b1 = b[1];
    return op(__builtin_bit_cast(T, b0), __builtin_bit_cast(T, b1));
}
template <int N, typename T>
RS_LANES T row_turned(T x) {   // lane i of a row: what lane i - N, around the row, has
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + N, 0xf, 0xf, false));
}
// Of the row's lanes i, i + STRIDE, i + 2 STRIDE ..., in all of them (for operations that do not mind the order).
template <int STRIDE, typename Op, typename T>
RS_LANES T of_row(T x, Op op) {
    if constexpr (STRIDE <= 1) x = op(x, row_turned<1>(x));
    if constexpr (STRIDE <= 2) x = op(x, row_turned<2>(x));
    if constexpr (STRIDE <= 4) x = op(x, row_turned<4>(x));
    if constexpr (STRIDE <= 8) x = op(x, row_turned<8>(x));
    return x;
}
template <typename Op, typename T>
RS_LANES T of_wave(T x, Op op) { return of_quarters(of_row<1>(x, op), op); }

// The sum over this lane and all later ones.
template <int N>
RS_LANES uint32_t row_later(uint32_t x) {   // what lane i + N of the row has; 0 past its end
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x100 + N, 0xf, 0xf, true);
}
RS_LANES uint32_t sum_from_lane(uint32_t x) {
    x += row_later<1>(x);
    x += row_later<2>(x);
    x += row_later<4>(x);
    x += row_later<8>(x);
    const uint32_t t1 = __builtin_amdgcn_readlane(x, 16), t2 = __builtin_amdgcn_readlane(x, 32), t3 = __builtin_amdgcn_readlane(x, 48);
    const int row = (threadIdx.x & 63) >> 4;
    return x + (row < 1 ? t1 : 0u) + (row < 2 ? t2 : 0u) + (row < 3 ? t3 : 0u);
}
