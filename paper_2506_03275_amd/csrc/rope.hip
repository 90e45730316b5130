// Rotary positions with several axes: pair j of a head's elements is turned by the angle
//     pos[t][axis(j)] * freqs[j],        (a, b) -> (a cos - b sin, a sin + b cos)
// where the first pairs belong to axis 0 (time), the next to axis 1 (height), the last to axis 2 (width).  The inverse, by the
// opposite angle, is the gradient of the turn.
//
// Bound: memory, 2 E bytes read and 2 E written per row of a head: 4608 tokens x 48 heads x 128 take 19.5 us (5.8 TB/s), 18 000 x 80 126 us
// (5.8 TB/s; a large copy reaches 5.2 to 5.8).  An angle belongs to a token and a pair and serves every head,
// so a thread keeps the sines of its four (or eight) pairs and walks heads.  An angle is formed in 64 bits: positions go to 2^31, and
// in 32 bits the angle of position 100 000 is off by 4e-3.  What is left of it after the whole turns, rounded to 32 bits, goes to
// the sine and cosine instructions, which take turns.
#include "rope.h"

#include <algorithm>
#include <type_traits>

namespace chipmunk {

struct RopeParams {
    const uint16_t* x;
    uint16_t* out;
    const int32_t* pos;      // [tokens][3]
    const double* freqs;     // [pairs]
    int64_t x_token, x_head, out_token, out_head;   // strides in elements
    int tokens, heads, E;
    int end0, end1, pairs;   // pairs of axis 0; of axes 0 and 1; of all
    int items;               // threads per row of a head
    int side, per, at_once;  // heads that threads of a workgroup walk side by side, heads per thread, tokens per workgroup
    float sign;
};

constexpr int kRopeThreads = 256;
constexpr int kRopeAhead = 4;    // heads of a thread in flight

// A thread's item of a row: ADJACENT pairs (elements 2j, 2j + 1), eight elements that hold four pairs; HALVES (elements j, j +
// pairs), the eight elements of eight pairs in either half.  Items behind the pairs are copied.
template <class T, bool HALVES, int SOURCE, int RESULT>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeParams p) {
    constexpr int NP = HALVES ? 8 : 4;
    const int slot = threadIdx.x / p.items, item = threadIdx.x - slot * p.items;
    const int in_group = slot / p.side, first_head = (int)blockIdx.y * p.side * p.per + slot - in_group * p.side;
    if (in_group >= p.at_once) return;
    const int turned = p.pairs / NP;                     // items that hold pairs
    const bool turn = item < turned;
    const int64_t e0 = HALVES && !turn ? 2 * p.pairs + (item - turned) * 8 : item * 8, e1 = HALVES && turn ? e0 + p.pairs : e0;
    auto load = [](const uint16_t* at) { return rope_load<SOURCE>(at); };
    const __amdgpu_buffer_rsrc_t result = raw_buffer(p.out, INT32_MAX);   // (a result that is written through reaches no further)
    auto store = [&](uint16_t* at, u32x4 value) { rope_store<RESULT>(result, p.out, at, value); };
    const int last_head = min(p.heads, ((int)blockIdx.y + 1) * p.side * p.per);
    for (int64_t t = (int64_t)blockIdx.x * p.at_once + in_group; t < p.tokens; t += (int64_t)gridDim.x * p.at_once) {
        float c[NP], s[NP];
        if (turn) {
            const int at[3] = {p.pos[3 * t], p.pos[3 * t + 1], p.pos[3 * t + 2]};
#pragma unroll
            for (int i = 0; i < NP; i++) {
                const int j = item * NP + i;
                rope_turn(j < p.end0 ? at[0] : j < p.end1 ? at[1] : at[2], p.freqs[j], c[i], s[i]);
                s[i] *= p.sign;
            }
        }
        const uint16_t* from = p.x + t * p.x_token;
        uint16_t* to = p.out + t * p.out_token;
        for (int h = first_head; h < last_head; h += kRopeAhead * p.side) {
            u32x4 a[kRopeAhead], b[kRopeAhead];
#pragma unroll
            for (int n = 0; n < kRopeAhead; n++) {
                const int64_t row = (int64_t)min(h + n * p.side, last_head - 1) * p.x_head;
                a[n] = load(from + row + e0);
                if (HALVES) b[n] = load(from + row + e1);
            }
#pragma unroll
            for (int n = 0; n < kRopeAhead; n++) {
                if (h + n * p.side >= last_head) break;
                if (turn) {
#pragma unroll
                    for (int w = 0; w < 4; w++) {
                        if constexpr (HALVES) {
                            const float x0 = T::low(a[n][w]), x1 = T::high(a[n][w]), y0 = T::low(b[n][w]), y1 = T::high(b[n][w]);
                            a[n][w] = T::pack(x0 * c[2 * w] - y0 * s[2 * w], x1 * c[2 * w + 1] - y1 * s[2 * w + 1]);
                            b[n][w] = T::pack(x0 * s[2 * w] + y0 * c[2 * w], x1 * s[2 * w + 1] + y1 * c[2 * w + 1]);
                        } else {
                            const float x0 = T::low(a[n][w]), y0 = T::high(a[n][w]);
                            a[n][w] = T::pack(x0 * c[w] - y0 * s[w], x0 * s[w] + y0 * c[w]);
                        }
                    }
                }
                const int64_t row = (int64_t)(h + n * p.side) * p.out_head;
                store(to + row + e0, a[n]);
                if (HALVES && turn) store(to + row + e1, b[n]);
            }
        }
    }
}

template <class T, bool HALVES>
static void rope_launch(const RopeParams& p, dim3 grid, int source, int result, hipStream_t s) {
    auto go = [&](auto source_c, auto result_c) { rope_kernel<T, HALVES, decltype(source_c)::value, decltype(result_c)::value><<<grid, kRopeThreads, 0, s>>>(p); };
    typedef std::integral_constant<int, kThroughCaches> Near;
    typedef std::integral_constant<int, kPastL2> Far;
    typedef std::integral_constant<int, kKept> Kept;
    typedef std::integral_constant<int, kWrittenThrough> Through;
    if (result == kPastLastLevel) go(Far{}, std::integral_constant<int, kPastLastLevel>{});   // (then the source is as large)
    else if (source == kPastL2) result == kKept ? go(Far{}, Kept{}) : go(Far{}, Through{});
    else result == kKept ? go(Near{}, Kept{}) : go(Near{}, Through{});
}

}  // namespace chipmunk

using namespace chipmunk;

extern "C" int32_t chipmunk_rope(const uint16_t* x, int64_t x_token_stride, int64_t x_head_stride, const int32_t* pos, const double* freqs,
                                 uint16_t* out, int64_t out_token_stride, int64_t out_head_stride, int tokens, int heads, int E,
                                 int pairs_t, int pairs_h, int pairs_w, int halves, int inverse, int dtype, void* stream) {
    if (!x || !pos || !freqs || !out) return CHIPMUNK_ERR_NULL;
    if (tokens <= 0 || heads <= 0 || heads > kRopeMostHeads || E <= 0 || pairs_t < 0 || pairs_h < 0 || pairs_w < 0) return CHIPMUNK_ERR_SHAPE;
    const int64_t pairs = (int64_t)pairs_t + pairs_h + pairs_w;
    if (pairs <= 0 || 2 * pairs > E) return CHIPMUNK_ERR_SHAPE;
    if (E % 8 != 0 || E > 512 || pairs % (halves ? 8 : 4) != 0 || (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16)) return CHIPMUNK_ERR_UNSUPPORTED;
    if (tokens == 1) x_token_stride = out_token_stride = 0;   // of one row alone a stride means nothing
    if (heads == 1) x_head_stride = out_head_stride = 0;
    if (rope_rows_overlap(x_token_stride, x_head_stride, tokens, heads, E) || rope_rows_overlap(out_token_stride, out_head_stride, tokens, heads, E)) return CHIPMUNK_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(out) || (reinterpret_cast<uintptr_t>(pos) & 3) || (reinterpret_cast<uintptr_t>(freqs) & 7) ||
        (x_token_stride | x_head_stride | out_token_stride | out_head_stride) % 8 != 0)
        return CHIPMUNK_ERR_ALIGN;
    RopeParams p{x, out, pos, freqs, x_token_stride, x_head_stride, out_token_stride, out_head_stride, tokens, heads, E,
                 pairs_t, pairs_t + pairs_h, (int)pairs, 0, 0, 0, 0, inverse ? -1.f : 1.f};
    p.items = halves ? (int)(pairs / 8 + (E - 2 * pairs) / 8) : E / 8;
    const int slots = kRopeThreads / p.items;
    p.per = kRopeAhead;
    // Side by side stand heads, whose rows lie behind one another; heads of rows get four tokens' rows in one run (18 000 x 80 heads
    // 144 -> 131 us, 75 600: 636 -> 568)
    p.side = std::min(out_head_stride > out_token_stride ? std::min(4, slots) : slots, (heads + p.per - 1) / p.per);
    p.at_once = slots / p.side;
    const int64_t groups = ((int64_t)tokens + p.at_once - 1) / p.at_once;
    const int parts = (heads + p.side * p.per - 1) / (p.side * p.per);
    const dim3 grid((uint32_t)std::min<int64_t>(groups, (1 << 22) / parts), parts);   // a launch has fewer than 2^32 threads
    const auto s = static_cast<hipStream_t>(stream);
    const int64_t bytes = (int64_t)tokens * heads * E * 2;
    const bool whole_lines = (reinterpret_cast<uintptr_t>(out) & 127) == 0 && ((halves ? pairs | (E - 2 * pairs) : E) | out_token_stride | out_head_stride) % 64 == 0;
    const bool near = (__int128)(tokens - 1) * out_token_stride + (__int128)(heads - 1) * out_head_stride + E <= INT32_MAX / 2;   // a 32-bit offset reaches it all
    const int source = bytes > kRopeL2 ? kPastL2 : kThroughCaches, result = bytes > kRopeLastLevel ? kPastLastLevel : whole_lines && near ? kWrittenThrough : kKept;
    if (dtype == CHIPMUNK_DTYPE_BF16) halves ? rope_launch<Bf16, true>(p, grid, source, result, s) : rope_launch<Bf16, false>(p, grid, source, result, s);
    else halves ? rope_launch<Fp16, true>(p, grid, source, result, s) : rope_launch<Fp16, false>(p, grid, source, result, s);
    return launch_status();
}
