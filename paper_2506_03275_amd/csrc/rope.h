// What the rotary positions (rope.hip) and the norm with them (norm_rope.hip) share.  Internal.
#pragma once
#include "element.h"

namespace chipmunk {

constexpr int kRopeMostHeads = 1 << 16;

// A source beyond the L2s passes them by, and a result beyond the last-level cache passes that by as well.  Measured with the kernel that reads
// the result: 113 MB 43.9 us, sources past 38.6, results too 43.3; 737 MB 267, 262, 253; 28 MB 19.3, 21.4, 23.5.  A smaller result of
// whole lines of 128 bytes is written through the L2s as it comes (12 MB 6.0 us, so 5.2; 57 MB 21.4 and 19.4, in place 21.0 and 17.8, with its
// reader 38.4 and 36.5; 184 MB 65.3 and 60.3; only 111 MB in place lose, 36.7 and 41.8).
constexpr int64_t kRopeL2 = 32 << 20, kRopeLastLevel = 256 << 20;
enum RopeSource { kThroughCaches, kPastL2 };
enum RopeResult { kKept, kWrittenThrough, kPastLastLevel };

// A row's 16 bytes from and to memory, by the ways above.  result: the whole of what is written through (no further than 32 bits reach).
template <int SOURCE>
__device__ __forceinline__ u32x4 rope_load(const uint16_t* at) {
    const u32x4* words = reinterpret_cast<const u32x4*>(at);
    return SOURCE == kPastL2 ? __builtin_nontemporal_load(words) : *words;
}
template <int RESULT>
__device__ __forceinline__ void rope_store(__amdgpu_buffer_rsrc_t result, const uint16_t* base, uint16_t* at, u32x4 value) {
    u32x4* words = reinterpret_cast<u32x4*>(at);
    if (RESULT == kWrittenThrough) __builtin_amdgcn_raw_buffer_store_b128(value, result, (int)((at - base) * 2), 0, 16);   // sc1
    else if (RESULT == kPastLastLevel) __builtin_nontemporal_store(value, words);
    else *words = value;
}

// Cosine and sine of pos * freq, in 64 bits up to the whole turns.
__device__ __forceinline__ void rope_turn(int pos, double freq, float& c, float& s) {
    double turns = (double)pos * freq * 0.15915494309189533577;
    turns -= __builtin_rint(turns);
    c = __builtin_amdgcn_cosf((float)turns);
    s = __builtin_amdgcn_sinf((float)turns);
}

// Rows of heads (or heads of rows) that do not overlap: one of the two strides is a row's length at least, and the other the rows it spans.
inline bool rope_rows_overlap(int64_t token, int64_t head, int tokens, int heads, int E) {
    return !((tokens == 1 || token >= (__int128)(heads - 1) * head + E) && (heads == 1 || head >= E)) &&
           !((heads == 1 || head >= (__int128)(tokens - 1) * token + E) && (tokens == 1 || token >= E));
}

}  // namespace chipmunk
