// Keys and values in pages (chipmunk_pages): where a row lies, and e4m3 under a power of two for each row of a head.  Internal.
#pragma once
#include "element.h"

#include <algorithm>

namespace chipmunk {

constexpr int kLeastPage = 16, kMostPage = 1 << 16;   // tokens of a page, a power of two

// A row of a head in e4m3 is code * 2^(byte - 127).  A power of two costs the type nothing but range: a value keeps its four significant
// bits whatever the power is, and the products with it and their way back are exact.  k = byte - 127 is the least at which the row's largest
// finite magnitude stays within 448 = 1.75 * 2^8, and -126 at least, so that 2^-k is a normal number.  `bits`: of that magnitude, 32 bits.
__device__ __forceinline__ int e4m3_exponent(uint32_t bits) {
    const int k = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return bits == 0 ? 0 : max(k, -126);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }   // -126 .. 127

// Magnitudes of the element types, as 15-bit numbers: the largest that e4m3 rows stand for (1.875 * 2^emax, four significant bits, so that nothing
// is rounded to infinity on the way back), and the first that is not finite.
template <class T> struct Magnitudes;
template <> struct Magnitudes<Bf16> { static constexpr uint32_t kMost = 0x7f70u, kNotFinite = 0x7f80u; };
template <> struct Magnitudes<Fp16> { static constexpr uint32_t kMost = 0x7b80u, kNotFinite = 0x7c00u; };

// Four codes and their power of two as four elements; the conversions take the power along and are exact, below the normal numbers of fp16 rounded.
template <class T> __device__ __forceinline__ u32x2 elements_of_codes(uint32_t codes, float scale);
template <> __device__ __forceinline__ u32x2 elements_of_codes<Bf16>(uint32_t codes, float scale) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true))};
}
template <> __device__ __forceinline__ u32x2 elements_of_codes<Fp16>(uint32_t codes, float scale) {
    return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes, scale, true))};
}

// Two elements under a power of two as codes, in half `upper` of a word: exact up to the one rounding, to nearest even.  (Of magnitudes above 448 times the
// power it makes NaN.)
typedef __attribute__((ext_vector_type(2))) short s16x2;
template <class T, bool upper> __device__ __forceinline__ uint32_t codes_of_elements(uint32_t word, uint32_t into, float scale) {
    if constexpr (T::kOnes == Bf16::kOnes)
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(__builtin_bit_cast(s16x2, into), __builtin_bit_cast(bf16x2, word), scale, upper));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(__builtin_bit_cast(s16x2, into), __builtin_bit_cast(fp16x2, word), scale, upper));
}

// ---- host side ---------------------------------------------------------------

// What is wrong with the pages of a call whose elements are of type dtype.  A stride along a size of one becomes zero.
inline int32_t check_pages(chipmunk_pages& pages, int dtype) {
    if (!pages.k || !pages.v) return CHIPMUNK_ERR_NULL;
    if (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16) return CHIPMUNK_ERR_UNSUPPORTED;
    const bool codes = pages.format == CHIPMUNK_DTYPE_E4M3;
    if (!codes && pages.format != dtype) return CHIPMUNK_ERR_UNSUPPORTED;
    if (codes && (!pages.k_scales || !pages.v_scales)) return CHIPMUNK_ERR_NULL;
    if (pages.pages <= 0 || pages.page_size <= 0 || pages.heads <= 0) return CHIPMUNK_ERR_SHAPE;
    if ((pages.E != 64 && pages.E != 128) || pages.page_size < kLeastPage || pages.page_size > kMostPage || (pages.page_size & (pages.page_size - 1)) != 0) return CHIPMUNK_ERR_UNSUPPORTED;
    if ((int64_t)pages.pages * pages.page_size > INT32_MAX) return CHIPMUNK_ERR_SHAPE;
    if (pages.pages == 1) pages.page_stride = pages.scale_page_stride = 0;
    if (pages.heads == 1) pages.head_stride = pages.scale_head_stride = 0;
    // no two rows overlap: of the three sizes, from the least stride on, each passes over all that the ones before it span
    auto apart = [&](int64_t page, int64_t token, int64_t head, int64_t row) {
        struct Size { int64_t stride; int count; } d[3] = {{page, pages.pages}, {token, pages.page_size}, {head, pages.heads}};
        std::sort(d, d + 3, [](const Size& a, const Size& b) { return a.stride < b.stride; });
        __int128 span = row;
        for (const Size& n : d) {
            if (n.count == 1) continue;
            if (n.stride < span) return false;
            span += (__int128)n.stride * (n.count - 1);
        }
        return span < ((__int128)1 << 60);
    };
    if (!apart(pages.page_stride, pages.token_stride, pages.head_stride, pages.E) || pages.token_stride >= (1 << 24)) return CHIPMUNK_ERR_SHAPE;
    if (codes && (!apart(pages.scale_page_stride, pages.scale_token_stride, pages.scale_head_stride, 1) || pages.scale_token_stride >= (1 << 24))) return CHIPMUNK_ERR_SHAPE;
    const int64_t unit = codes ? 16 : 8;   // elements of 16 bytes
    if (!aligned16(pages.k) || !aligned16(pages.v) || (pages.page_stride | pages.token_stride | pages.head_stride) % unit != 0) return CHIPMUNK_ERR_ALIGN;
    return CHIPMUNK_OK;
}

}  // namespace chipmunk
