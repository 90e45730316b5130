// Keys and values of new tokens into pages, and rows of pages back: in the element type, copied, or in e4m3 with a power of two for each row of a
// head (pages.h has the numbers).
//
// Bound: memory; a row of a head in e4m3 is 2 E bytes on one side and E + 1 on the other.  16 383 tokens of 8 heads x 128 written in 21 us and read in 17 (4.8
// and 6.1 TB/s), 75 600 of 24 heads read in 257 (5.4 TB/s); 16 tokens 3.0 and 2.8 us.
#include "pages.h"
#include "rope.h"

#include <type_traits>

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
    // Workgroups go to the eight XCDs in turn: each XCD takes one run of the tokens, so that the scales of neighbouring tokens, bytes of one line,
    // meet in one L2
    const uint32_t run = gridDim.x / 8, more = gridDim.x % 8, xcd = blockIdx.x % 8;
    const uint32_t block = xcd * run + min(xcd, more) + blockIdx.x / 8;
    const int64_t id = (int64_t)block * kCacheThreads + threadIdx.x;
    const int64_t token = id / per_token;
    const uint32_t in_token = (uint32_t)(id - token * per_token), row = in_token / per_row;
    return CacheItem{token, (int)(row % p.pages.heads), (int)(in_token % per_row), row >= (uint32_t)p.pages.heads};
}

// Where a row of the pages lies, in elements of the values or of the scales.
__device__ __forceinline__ int64_t place_of(const CacheParams& p, int64_t row, int head, int64_t page_stride, int64_t token_stride, int64_t head_stride) {
    return (row >> p.shift) * page_stride + (row & (p.pages.page_size - 1)) * token_stride + head * head_stride;
}

// FAR: new tokens beyond the L2s pass them by (rope.h; 67 MB 45 -> 39 us with the way back).
template <class T, bool CODES, bool FAR>
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheParams p) {
    const CacheItem at = cache_item(p);
    if (at.token >= p.tokens) return;                // (with all threads of its row)
    const int64_t row = p.rows[at.token];
    if (row < 0 || row >= (int64_t)p.pages.pages * p.pages.page_size) return;
    const uint16_t* from = at.value ? p.from_v + at.token * p.v_token + at.head * p.v_head : p.from_k + at.token * p.k_token + at.head * p.k_head;
    u32x4 x[2];
#pragma unroll
    for (int i = 0; i < 2; i++) x[i] = rope_load<FAR ? kPastL2 : kThroughCaches>(from + at.chunk * 16 + i * 8);
    const int64_t to = place_of(p, row, at.head, p.pages.page_stride, p.pages.token_stride, p.pages.head_stride) + at.chunk * 16;
    void* held = at.value ? p.pages.v : p.pages.k;
    if constexpr (!CODES) {
#pragma unroll
        for (int i = 0; i < 2; i++) reinterpret_cast<u32x4*>(static_cast<uint16_t*>(held) + to)[i] = x[i];
        return;
    }
    typedef Magnitudes<T> M;
    // The order of the magnitudes is that of their 15 bits, two to a word; over the row's threads: 4 (E = 64) or 8 side by side.
    typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
    const bool eight = p.pages.E == 128;
    auto row_most = [&]() {
        u16x2 most = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; i++) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[i / 4][i % 4] & 0x7fff7fffu));
        uint32_t m = max((uint32_t)most[0], (uint32_t)most[1]);
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));         // quad_perm 1 0 3 2
        m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));         // quad_perm 2 3 0 1
        if (eight) m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, false));   // row_half_mirror
        return m;
    };
    uint32_t most = row_most();
    uint32_t special = 0;                            // a bit for each element that is infinite or NaN
    if (most > M::kMost) {                           // (a row's threads alike) those out of the way, and magnitudes beyond the most cut
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int at = i % 2 * 16;
            const uint32_t bits = x[i / 8][i % 8 / 2] >> at & 0xffffu, magnitude = bits & 0x7fffu;
            if (magnitude <= M::kMost) continue;
            const bool finite = magnitude < M::kNotFinite;
            if (!finite) special |= 1u << i;
            x[i / 8][i % 8 / 2] = (x[i / 8][i % 8 / 2] & ~(0xffffu << at)) | (finite ? (bits & 0x8000u) | M::kMost : 0u) << at;
        }
        most = row_most();
    }
    const int k = e4m3_exponent(__float_as_uint(T::low(most)));
    const float power = power_of_two(k);
    u32x4 codes;
#pragma unroll
    for (int i = 0; i < 4; i++) codes[i] = codes_of_elements<T, true>(x[i / 2][i % 2 * 2 + 1], codes_of_elements<T, false>(x[i / 2][i % 2 * 2], 0u, power), power);
    if (special) {
#pragma unroll
        for (int i = 0; i < 16; i++)
            if (special >> i & 1) codes[i / 4] |= 0x7fu << i % 4 * 8;
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
    for (int i = 0; i < 2; i++) reinterpret_cast<u32x4*>(to)[i] = x[i];   // (past the last-level cache 1.4 GB take 268 us for 254)
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
    auto go = [&](auto far) {
        constexpr bool FAR = decltype(far)::value;
        if (pages->format != CHIPMUNK_DTYPE_E4M3) cache_write_kernel<Bf16, false, FAR><<<grid, kCacheThreads, 0, s>>>(p);   // (a copy is a copy)
        else if (dtype == CHIPMUNK_DTYPE_BF16) cache_write_kernel<Bf16, true, FAR><<<grid, kCacheThreads, 0, s>>>(p);
        else cache_write_kernel<Fp16, true, FAR><<<grid, kCacheThreads, 0, s>>>(p);
    };
    (int64_t)tokens * p.pages.heads * p.pages.E * 4 > kRopeL2 ? go(std::true_type{}) : go(std::false_type{});
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
