// Keys and values of new tokens into pages, and rows of pages back: in the element type, copied, or in e4m3 with a power of two for each row of a
// head (pages.h has the numbers).
//
// Bound: memory; a row of a head in e4m3 is 2 E bytes on one side and E + 1 on the other.
#include "pages.h"
#include "rope.h"

namespace chipmunk {

struct CacheParams {
    chipmunk_pages pages;
    const int64_t* rows;                             // [tokens]
    const uint16_t* from_k;                          // writing
    const uint16_t* from_v;
    uint16_t* to_k;                                  // reading
    uint16_t* to_v;
    int64_t k_token, k_head, v_token, v_head;
    int tokens;
    int shift;                                       // log2 of the page's tokens
};

constexpr int kCacheThreads = 256;

// A thread's 16 elements of a row of a head of K or V: E / 16 threads to a row; the rows of a token's heads and of K and V side by side.
struct CacheItem {
    int64_t token;
    int head, chunk;
    bool value;
};
__device__ __forceinline__ CacheItem cache_item(const CacheParams& p) {
    const uint32_t per_row = p.pages.E / 16, per_token = per_row * 2 * p.pages.heads;
    const int64_t id = (int64_t)blockIdx.x * kCacheThreads + threadIdx.x;
    const int64_t token = id / per_token;
    const uint32_t in_token = (uint32_t)(id - token * per_token), row = in_token / per_row;
    return CacheItem{token, (int)(row % p.pages.heads), (int)(in_token % per_row), row >= (uint32_t)p.pages.heads};
}

// Where a row of the pages lies, in elements of the values or of the scales.
__device__ __forceinline__ int64_t place_of(const CacheParams& p, int64_t row, int head, int64_t page_stride, int64_t token_stride, int64_t head_stride) {
    return (row >> p.shift) * page_stride + (row & (p.pages.page_size - 1)) * token_stride + head * head_stride;
}

template <class T, bool CODES>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheParams p) {
    const CacheItem at = cache_item(p);
    if (at.token >= p.tokens) return;                // (with all threads of its row)
    const int64_t row = p.rows[at.token];
    if (row < 0 || row >= (int64_t)p.pages.pages * p.pages.page_size) return;
    const uint16_t* from = at.value ? p.from_v + at.token * p.v_token + at.head * p.v_head : p.from_k + at.token * p.k_token + at.head * p.k_head;
    u32x4 x[2];
#pragma unroll
    for (int i = 0; i < 2; i++) x[i] = reinterpret_cast<const u32x4*>(from + at.chunk * 16)[i];
    const int64_t to = place_of(p, row, at.head, p.pages.page_stride, p.pages.token_stride, p.pages.head_stride) + at.chunk * 16;
    void* held = at.value ? p.pages.v : p.pages.k;
    if constexpr (!CODES) {
#pragma unroll
        for (int i = 0; i < 2; i++) reinterpret_cast<u32x4*>(static_cast<uint16_t*>(held) + to)[i] = x[i];
        return;
    }
    typedef Magnitudes<T> M;
    // By the bits: the order of the magnitudes is that of their 15 bits, and these files are compiled as if NaN did not exist.
    uint32_t most = 0;
    uint32_t mag[16], sign[16];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const uint32_t bits = i % 2 ? x[i / 8][i % 8 / 2] >> 16 : x[i / 8][i % 8 / 2] & 0xffffu;
        mag[i] = bits & 0x7fffu;
        sign[i] = bits & 0x8000u;
        const bool finite = mag[i] < M::kNotFinite;
        if (finite) mag[i] = min(mag[i], M::kMost);
        most = max(most, finite ? mag[i] : 0u);
    }
    // over the row's threads: 4 (E = 64) or 8 side by side
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xb1, 0xf, 0xf, false));        // quad_perm 1 0 3 2
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4e, 0xf, 0xf, false));        // quad_perm 2 3 0 1
    if (p.pages.E == 128) most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x141, 0xf, 0xf, false));   // row_half_mirror
    const int k = e4m3_exponent(__float_as_uint(T::low(most)));
    const float down = power_of_two(-k);
    u32x4 codes;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const uint32_t m = mag[4 * i + j];
            // no finite value passes 448; the others become NaN, which the conversion leaves NaN
            f[j] = __uint_as_float(m < M::kNotFinite ? __float_as_uint(T::low(m | sign[4 * i + j]) * down) : 0x7fc00000u);
        }
        const int half = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
        codes[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], half, true);
    }
    *reinterpret_cast<u32x4*>(static_cast<uint8_t*>(held) + to) = codes;
    if (at.chunk == 0)
        (at.value ? p.pages.v_scales : p.pages.k_scales)[place_of(p, row, at.head, p.pages.scale_page_stride, p.pages.scale_token_stride, p.pages.scale_head_stride)] = (uint8_t)(k + 127);
}

template <class T, bool CODES>
__global__ __launch_bounds__(kCacheThreads) void cache_read_kernel(CacheParams p) {
    const CacheItem at = cache_item(p);
    if (at.token >= p.tokens) return;
    const int64_t row = p.rows[at.token];
    if (row < 0 || row >= (int64_t)p.pages.pages * p.pages.page_size) return;
    const int64_t from = place_of(p, row, at.head, p.pages.page_stride, p.pages.token_stride, p.pages.head_stride) + at.chunk * 16;
    const void* held = at.value ? p.pages.v : p.pages.k;
    u32x4 x[2];
    if constexpr (CODES) {
        const uint8_t byte = (at.value ? p.pages.v_scales : p.pages.k_scales)[place_of(p, row, at.head, p.pages.scale_page_stride, p.pages.scale_token_stride, p.pages.scale_head_stride)];
        const u32x4 codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(held) + from);
        const float scale = __uint_as_float((uint32_t)byte << 23);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const u32x2 four = elements_of_codes<T>(codes[i], scale);
            x[i / 2][i % 2 * 2] = four[0];
            x[i / 2][i % 2 * 2 + 1] = four[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; i++) x[i] = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(held) + from)[i];
    }
    uint16_t* to = (at.value ? p.to_v + at.token * p.v_token + at.head * p.v_head : p.to_k + at.token * p.k_token + at.head * p.k_head) + at.chunk * 16;
#pragma unroll
    for (int i = 0; i < 2; i++) reinterpret_cast<u32x4*>(to)[i] = x[i];
}

// The checks that writing and reading share.
static int32_t check_rows(CacheParams& p, const void* k, const void* v, int dtype) {
    if (!k || !v || !p.rows) return CHIPMUNK_ERR_NULL;
    if (p.tokens <= 0) return CHIPMUNK_ERR_SHAPE;
    const int32_t status = check_pages(p.pages, dtype);
    if (status != CHIPMUNK_OK) return status;
    const int E = p.pages.E, heads = p.pages.heads;
    if (p.tokens == 1) p.k_token = p.v_token = 0;    // of one row alone a stride means nothing
    if (heads == 1) p.k_head = p.v_head = 0;
    if (rope_rows_overlap(p.k_token, p.k_head, p.tokens, heads, E) || rope_rows_overlap(p.v_token, p.v_head, p.tokens, heads, E)) return CHIPMUNK_ERR_SHAPE;
    if (!aligned16(k) || !aligned16(v) || (reinterpret_cast<uintptr_t>(p.rows) & 7) || (p.k_token | p.k_head | p.v_token | p.v_head) % 8 != 0) return CHIPMUNK_ERR_ALIGN;
    p.shift = __builtin_ctz((uint32_t)p.pages.page_size);
    if ((int64_t)p.tokens * heads * (E / 8) / kCacheThreads >= (1 << 24) - 1) return CHIPMUNK_ERR_SHAPE;   // a launch has fewer than 2^32 threads
    return CHIPMUNK_OK;
}
static uint32_t cache_workgroups(const CacheParams& p) {
    return (uint32_t)(((int64_t)p.tokens * p.pages.heads * (p.pages.E / 8) + kCacheThreads - 1) / kCacheThreads);
}

}  // namespace chipmunk

using namespace chipmunk;

extern "C" int32_t chipmunk_cache_write(const uint16_t* k, int64_t k_token_stride, int64_t k_head_stride, const uint16_t* v, int64_t v_token_stride,
                                        int64_t v_head_stride, const int64_t* rows, const chipmunk_pages* pages, int tokens, int dtype, void* stream) {
    if (!pages) return CHIPMUNK_ERR_NULL;
    CacheParams p{*pages, rows, k, v, nullptr, nullptr, k_token_stride, k_head_stride, v_token_stride, v_head_stride, tokens, 0};
    const int32_t status = check_rows(p, k, v, dtype);
    if (status != CHIPMUNK_OK) return status;
    const auto s = static_cast<hipStream_t>(stream);
    const uint32_t grid = cache_workgroups(p);
    if (pages->format != CHIPMUNK_DTYPE_E4M3) cache_write_kernel<Bf16, false><<<grid, kCacheThreads, 0, s>>>(p);   // (a copy is a copy)
    else if (dtype == CHIPMUNK_DTYPE_BF16) cache_write_kernel<Bf16, true><<<grid, kCacheThreads, 0, s>>>(p);
    else cache_write_kernel<Fp16, true><<<grid, kCacheThreads, 0, s>>>(p);
    return launch_status();
}

extern "C" int32_t chipmunk_cache_read(const chipmunk_pages* pages, const int64_t* rows, uint16_t* k, int64_t k_token_stride, int64_t k_head_stride, uint16_t* v,
                                       int64_t v_token_stride, int64_t v_head_stride, int tokens, int dtype, void* stream) {
    if (!pages) return CHIPMUNK_ERR_NULL;
    CacheParams p{*pages, rows, nullptr, nullptr, k, v, k_token_stride, k_head_stride, v_token_stride, v_head_stride, tokens, 0};
    const int32_t status = check_rows(p, k, v, dtype);
    if (status != CHIPMUNK_OK) return status;
    const auto s = static_cast<hipStream_t>(stream);
    const uint32_t grid = cache_workgroups(p);
    if (pages->format != CHIPMUNK_DTYPE_E4M3) cache_read_kernel<Bf16, false><<<grid, kCacheThreads, 0, s>>>(p);
    else if (dtype == CHIPMUNK_DTYPE_BF16) cache_read_kernel<Bf16, true><<<grid, kCacheThreads, 0, s>>>(p);
    else cache_read_kernel<Fp16, true><<<grid, kCacheThreads, 0, s>>>(p);
    return launch_status();
}
