// The two 16-bit element types of the operators that take either (projections, rotary positions, attention over packed
// sequences).  Internal.
#pragma once
#include "common.h"

namespace chipmunk {

typedef __attribute__((ext_vector_type(8))) _Float16 fp16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 fp16x2;

// x8: eight elements, an operand of a lane for the matrix products (16x16x32, 32x32x16); pack: two floats rounded to nearest even, lo in bits
// 0..15; low, high: the two elements of a word
struct Bf16 {
    typedef bf16x8 x8;
    static constexpr uint32_t kOnes = 0x3f803f80u, kExponent = 0x7f807f80u, kExponentStep = 0x00800080u;
    static __device__ __forceinline__ f32x4 product(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 product(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
    static __device__ __forceinline__ float low(uint32_t word) { return __uint_as_float(word << 16); }
    static __device__ __forceinline__ float high(uint32_t word) { return __uint_as_float(word & 0xffff0000u); }
};
struct Fp16 {
    typedef fp16x8 x8;
    static constexpr uint32_t kOnes = 0x3c003c00u, kExponent = 0x7c007c00u, kExponentStep = 0x04000400u;
    static __device__ __forceinline__ f32x4 product(x8 a, x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 product(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return __builtin_bit_cast(uint32_t, fp16x2{(_Float16)lo, (_Float16)hi}); }
    static __device__ __forceinline__ float low(uint32_t word) { return (float)__builtin_bit_cast(fp16x2, word)[0]; }
    static __device__ __forceinline__ float high(uint32_t word) { return (float)__builtin_bit_cast(fp16x2, word)[1]; }
};

// A lane of a 16x16 product holds four consecutive columns (4 g ..) of one row of each block of 16 columns, g = lane / 16.
// Lanes 16 apart exchange halves of two neighbouring blocks, after which each holds eight consecutive columns, those from
// columns_of_lane(g) on of the 32; from_columns is the way back.
__device__ __forceinline__ int columns_of_lane(int g) { return (g & 1) * 16 + (g >> 1) * 8; }
__device__ __forceinline__ u32x4 to_columns(u32x2 first, u32x2 second) {
    const auto lo = __builtin_amdgcn_permlane16_swap(first[0], second[0], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(first[1], second[1], false, false);
    return u32x4{lo[0], hi[0], lo[1], hi[1]};
}
__device__ __forceinline__ void from_columns(u32x4 columns, u32x2 (&block)[2]) {
    const auto lo = __builtin_amdgcn_permlane16_swap(columns[0], columns[2], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(columns[1], columns[3], false, false);
    block[0] = u32x2{lo[0], hi[0]};
    block[1] = u32x2{lo[1], hi[1]};
}
// The same of a 32x32 product: a lane holds columns 4 h .. of each run of eight, h = lane / 32; of two neighbouring runs lanes 32
// apart exchange halves, after which each holds the eight of one, those from 8 h on.
__device__ __forceinline__ u32x4 to_columns_32(u32x2 first, u32x2 second) {
    const auto lo = __builtin_amdgcn_permlane32_swap(first[0], second[0], false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(first[1], second[1], false, false);
    return u32x4{lo[0], hi[0], lo[1], hi[1]};
}
__device__ __forceinline__ void from_columns_32(u32x4 columns, u32x2 (&run)[2]) {
    const auto lo = __builtin_amdgcn_permlane32_swap(columns[0], columns[2], false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(columns[1], columns[3], false, false);
    run[0] = u32x2{lo[0], hi[0]};
    run[1] = u32x2{lo[1], hi[1]};
}
// Lanes 8 apart in a row of 16 exchange: `first` then holds both of the lower lane, side by side, `second` both of the upper one.
// (row_ror:8; the banks of four lanes that are written are 2 and 3, then 0 and 1.)
__device__ __forceinline__ void exchange_8_apart(u32x4& first, u32x4& second) {
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const uint32_t a = first[w], b = second[w];
        first[w] = (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128, 0xf, 0xc, false);
        second[w] = (uint32_t)__builtin_amdgcn_update_dpp((int)b, (int)a, 0x128, 0xf, 0x3, false);
    }
}
// The same of lanes 16 apart in a half of 32.
__device__ __forceinline__ void exchange_16_apart(u32x4& first, u32x4& second) {
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const auto both = __builtin_amdgcn_permlane16_swap(first[w], second[w], false, false);
        first[w] = both[0];
        second[w] = both[1];
    }
}

}  // namespace chipmunk
