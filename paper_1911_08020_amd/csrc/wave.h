// Wave-wide (64 lanes) sums, maxima and scans of the training operators, in a fixed order.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace darb {

// The value of another lane by a DPP pattern; lanes outside the row mask get `other`.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float x, float other) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(other), __float_as_int(x),
                                                      CTRL, ROWS, 0xf, false));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t dpp(uint32_t x, uint32_t other) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(other), int(x), CTRL, ROWS, 0xf, false));
}

// Patterns in which every lane has a source: the move folds into the operation that uses it.
template <int CTRL> __device__ __forceinline__ float dpp_all(float x) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ uint32_t dpp_all(uint32_t x) {
    return uint32_t(__builtin_amdgcn_mov_dpp(int(x), CTRL, 0xf, 0xf, true));
}

constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;
constexpr int kDppBcast15 = 0x142, kDppBcast31 = 0x143;

struct AddOp {
    __device__ static float of(float a, float b) { return a + b; }
    __device__ static float none() { return 0.0f; }
};
struct MaxOp {  // a NaN is left out
    __device__ static float of(float a, float b) { return fmaxf(a, b); }
    __device__ static float none() { return -__builtin_inff(); }
};

// Over each aligned group of LANES (1 ... 64, a power of two) lanes; every lane of a group of
// up to 16 gets the result (where x is a product its first addition may be fused, and lanes
// differ in the last bit: take one lane's), lane 63 that of 64.
template <int LANES, typename Op> __device__ __forceinline__ float group_reduce(float x) {
    if (LANES >= 2) x = Op::of(x, dpp_all<kDppXor1>(x));
    if (LANES >= 4) x = Op::of(x, dpp_all<kDppXor2>(x));
    if (LANES >= 8) x = Op::of(x, dpp_all<kDppHalfMirror>(x));
    if (LANES >= 16) x = Op::of(x, dpp_all<kDppMirror>(x));
    if (LANES >= 32) x = Op::of(x, dpp<kDppBcast15, 0xa>(x, Op::none()));
    if (LANES >= 64) x = Op::of(x, dpp<kDppBcast31, 0xc>(x, Op::none()));
    return x;
}

__device__ __forceinline__ float lane_of(float x, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), lane));
}

// The whole wave's result, the same in every lane (in a scalar register).
__device__ __forceinline__ float wave_sum(float x) { return lane_of(group_reduce<64, AddOp>(x), 63); }
__device__ __forceinline__ float wave_max(float x) { return lane_of(group_reduce<64, MaxOp>(x), 63); }

// x summed over the lanes that hold the same place in their rows of 16, in each of them.
__device__ __forceinline__ float sum_rows(float x) {
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
}

__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) {
    auto of = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    x = of(x, dpp_all<kDppXor1>(x));
    x = of(x, dpp_all<kDppXor2>(x));
    x = of(x, dpp_all<kDppHalfMirror>(x));
    x = of(x, dpp_all<kDppMirror>(x));
    x = of(x, dpp<kDppBcast15, 0xa>(x, 0u));
    x = of(x, dpp<kDppBcast31, 0xc>(x, 0u));
    return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}

// The wave's place in its workgroup, known to be the same in all lanes.
__device__ __forceinline__ int wave_id() {
    return __builtin_amdgcn_readfirstlane(int(threadIdx.x) / 64);
}

__device__ __forceinline__ int lane_id() {
    return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));
}

}  // namespace darb
