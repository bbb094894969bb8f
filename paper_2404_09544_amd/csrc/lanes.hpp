// A lane's values: from another lane of its wavefront, without LDS, and in and out of its words.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace gnnav {

// The value of lane ^ S, S = 1, 2, 4 or 8.
template <int S>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
    static_assert(S == 1 || S == 2 || S == 4 || S == 8, "within 16 lanes");
    if constexpr (S == 1) return __builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, true);        // quad_perm 1 0 3 2
    else if constexpr (S == 2) return __builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, true);   // quad_perm 2 3 0 1
    else if constexpr (S == 4)   // reversed within 8 lanes, then within 4
        return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, true), 0x1b, 0xf, 0xf, true);
    else return __builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true);                        // row_ror 8
}

struct LanePair {
    uint32_t low, high;
};
// The values of the lane of each pair l, l ^ S whose bit S is clear, and of the one whose bit is set; S = 16 or 32.
template <int S>
__device__ __forceinline__ LanePair lane_pair(uint32_t x) {
    static_assert(S == 16 || S == 32, "rows of 16 lanes, or halves");
    if constexpr (S == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return {r[0], r[1]};
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return {r[0], r[1]};
    }
}

// Sum or max over groups of N lanes (16, 32 or 64; a power of two), in every lane: the same bits in each.
template <int N, bool MAX>
__device__ __forceinline__ float lanes_reduce(float x) {
    auto join = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    auto f = [](uint32_t u) { return __uint_as_float(u); };
    if constexpr (N >= 2) x = join(x, f(lane_xor<1>(__float_as_uint(x))));
    if constexpr (N >= 4) x = join(x, f(lane_xor<2>(__float_as_uint(x))));
    if constexpr (N >= 8) x = join(x, f(lane_xor<4>(__float_as_uint(x))));
    if constexpr (N >= 16) x = join(x, f(lane_xor<8>(__float_as_uint(x))));
    if constexpr (N >= 32) {
        const LanePair p = lane_pair<16>(__float_as_uint(x));
        x = join(f(p.low), f(p.high));
    }
    if constexpr (N >= 64) {
        const LanePair p = lane_pair<32>(__float_as_uint(x));
        x = join(f(p.low), f(p.high));
    }
    return x;
}

// Two values in one conversion: the bits of bf16_rne.
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
// Entry e of a vector of 32-bit words that hold fp32 values, or pairs of bf16 ones.
template <bool BF, class V>
__device__ __forceinline__ float element(const V &v, int e) {
    if constexpr (BF) return __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    else return __uint_as_float(v[e]);
}

}  // namespace gnnav
