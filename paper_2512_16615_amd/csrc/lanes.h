// Sums over neighbouring lanes by vector instructions alone; a shuffle waits for LDS in every step (norms, 2 x 30000 rows of 320: forward 45 -> 40 us, backward 59 -> 56;
// 2048 rows of 1024 backward 20.6 -> 17.9; glue gradient, 16 heads x 4096 tokens, d = 64: 15.0 -> 14.6).
#pragma once
#include <hip/hip_runtime.h>

namespace llsa {

// a lane's value from the lane that a step within 16 lanes names: its neighbour (1), the other pair of four (2), the other four of eight (4), the other eight (8)
template <int STEP> __device__ __forceinline__ float lane_step(float x) {
    constexpr int ctrl = STEP == 1 ? 0xb1 : STEP == 2 ? 0x4e : STEP == 4 ? 0x141 : 0x140;      // quads permuted; eight, sixteen lanes mirrored
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), ctrl, 0xf, 0xf, true));
}
// The sum over N lanes (2 to 64, a power of two), in each of them and the same bits
template <int N> __device__ __forceinline__ float lanes_sum(float x) {
    x += lane_step<1>(x);
    if constexpr (N >= 4) x += lane_step<2>(x);
    if constexpr (N >= 8) x += lane_step<4>(x);
    if constexpr (N >= 16) x += lane_step<8>(x);
    if constexpr (N >= 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if constexpr (N >= 64) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    return x;
}

// The sum of the lanes that are N apart (4 or 16), over the whole wave; lanes 0 .. N - 1 have it
template <int N> __device__ __forceinline__ float rows_sum(float x) {
    static_assert(N == 4 || N == 16, "");
    if constexpr (N == 4) {                                  // 16 lanes turned by 4 and 8
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x124, 0xf, 0xf, true));
        x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, true));
    }
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

}  // namespace llsa
