// The RMS norm of every head of queries and keys, and the rotary positions behind it, in one pass: with n = x r, r = 1 / sqrt(mean_e x_e^2 + eps),
//     out = turn(n w)           (w: the queries' heads have one weight, the keys' another; turn: rope.hip)
// and the gradient: with g = turn^-1(grad), c = mean_e(g_e w_e n_e),
//     dx = r (g w - n c),       dw_e = sum over rows of g_e n_e.
//
// Bound: memory; 4 E bytes per row of a head, the gradient 6 E.  18 000 tokens of 80 heads x 128: 130 us (5.7 TB/s), the gradient 220 (5.0 TB/s);
// 4608 tokens of 48 heads 20.2 us (5.6 TB/s); 8 tokens of 40 heads 3.7 to 4.0.
#include "rope.h"

#include <algorithm>
#include <type_traits>

namespace chipmunk {

struct NormParams {
    const uint16_t* x;
    const uint16_t* grad;    // of the result; the gradient only
    uint16_t* out;           // the result, or dx
    const uint16_t* weight[2];   // of queries, of keys: [E]
    const int32_t* pos;      // [tokens][3]
    const double* freqs;     // [pairs]
    float* partial;          // [workgroups][2][E]; the gradient only
    int64_t x_token, x_head, grad_token, grad_head, out_token, out_head;   // strides in elements
    int tokens, heads, q_heads, E;
    int end0, end1, pairs;   // pairs of axis 0; of axes 0 and 1; of all
    int items, lanes;        // items of a row; threads that a row takes, a power of two
    int side, per, at_once;  // heads that threads of a workgroup walk side by side, heads per thread, tokens per workgroup
    float eps, inv_E;
};

constexpr int kNormThreads = 256;
constexpr int kNormAhead = 4;        // heads of a thread in flight
constexpr int kNormGradAhead = 2;

// Sum over a row's threads, side by side in a wave; in every one of them.
__device__ __forceinline__ float row_sum(float x, int lanes) {
    auto add = [&](int moved) { x += __builtin_bit_cast(float, moved); };
    if (lanes > 1) add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0xb1, 0xf, 0xf, false));    // quad_perm 1 0 3 2
    if (lanes > 2) add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x4e, 0xf, 0xf, false));    // quad_perm 2 3 0 1
    if (lanes > 4) add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x141, 0xf, 0xf, false));   // row_half_mirror
    if (lanes > 8) add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x140, 0xf, 0xf, false));   // row_mirror
    if (lanes > 16) {
        const uint32_t u = __float_as_uint(x);
        const auto s = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if (lanes > 32) {
        const uint32_t u = __float_as_uint(x);
        const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return x;
}

// A thread's item of a row: ADJACENT pairs (elements 2j, 2j + 1), eight elements that hold four pairs; HALVES (elements j, j +
// pairs), the eight elements of eight pairs in either half.  Items behind the pairs are not turned.
template <class T, bool HALVES>
struct NormItem {
    static constexpr int NP = HALVES ? 8 : 4, NE = HALVES ? 16 : 8;
    int64_t e0, e1;          // its first elements
    bool present, turn;

    __device__ __forceinline__ NormItem(const NormParams& p, int item) {
        const int turned = p.pairs / NP;
        present = item < p.items;
        turn = item < turned;
        e0 = !present ? 0 : HALVES && !turn ? 2 * p.pairs + (item - turned) * 8 : item * 8;
        e1 = HALVES && turn ? e0 + p.pairs : e0;
    }
    // words as numbers; what the thread has not is zero
    __device__ __forceinline__ void numbers(const u32x4& a, const u32x4& b, float (&f)[NE]) const {
#pragma unroll
        for (int w = 0; w < 4; w++) {
            f[2 * w] = present ? T::low(a[w]) : 0.f;
            f[2 * w + 1] = present ? T::high(a[w]) : 0.f;
            if constexpr (HALVES) {
                f[8 + 2 * w] = turn ? T::low(b[w]) : 0.f;
                f[8 + 2 * w + 1] = turn ? T::high(b[w]) : 0.f;
            }
        }
    }
    __device__ __forceinline__ static void words(const float (&f)[NE], u32x4& a, u32x4& b) {
#pragma unroll
        for (int w = 0; w < 4; w++) {
            a[w] = T::pack(f[2 * w], f[2 * w + 1]);
            if constexpr (HALVES) b[w] = T::pack(f[8 + 2 * w], f[8 + 2 * w + 1]);
        }
    }
    __device__ __forceinline__ void angles(const NormParams& p, int64_t t, int item, float (&c)[NP], float (&s)[NP]) const {
        if (!turn) return;
        const int at[3] = {p.pos[3 * t], p.pos[3 * t + 1], p.pos[3 * t + 2]};
#pragma unroll
        for (int i = 0; i < NP; i++) {
            const int j = item * NP + i;
            rope_turn(j < p.end0 ? at[0] : j < p.end1 ? at[1] : at[2], p.freqs[j], c[i], s[i]);
        }
    }
    // sign -1: back
    __device__ __forceinline__ void rotate(float (&f)[NE], const float (&c)[NP], const float (&s)[NP], float sign) const {
        if (!turn) return;
#pragma unroll
        for (int i = 0; i < NP; i++) {
            const int a = HALVES ? i : 2 * i, b = HALVES ? 8 + i : 2 * i + 1;
            const float u = f[a], v = f[b], sn = s[i] * sign;
            f[a] = u * c[i] - v * sn;
            f[b] = u * sn + v * c[i];
        }
    }
    // A row's x becomes n = x r; r.  Squares of bf16, and their mean with eps, may pass 32 bits' range: then n is formed of values 2^-72 times as large,
    // and so is the root (eps counts there too: beside a mean of 2^119 or more, which a sum of 2^128 leaves, any up to 2^128 may stand).
    __device__ __forceinline__ static float normalize(const NormParams& p, float (&f)[NE]) {
        float sum = 0.f, down = 1.f;
#pragma unroll
        for (int i = 0; i < NE; i++) sum += f[i] * f[i];
        float mean = row_sum(sum, p.lanes) * p.inv_E + p.eps;
        if ((__float_as_uint(mean) & 0x7f800000u) == 0x7f800000u) {
            down = 0x1p-72f;
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < NE; i++) {
                f[i] *= down;
                sum += f[i] * f[i];
            }
            mean = row_sum(sum, p.lanes) * p.inv_E + p.eps * down * down;
        }
        const float r = __builtin_amdgcn_rsqf(mean);
#pragma unroll
        for (int i = 0; i < NE; i++) f[i] *= r;
        return r * down;
    }
};

template <class T, bool HALVES, int SOURCE, int RESULT>
__global__ __launch_bounds__(kNormThreads) void norm_rope_kernel(NormParams p) {
    typedef NormItem<T, HALVES> Item;
    const int slot = threadIdx.x / p.lanes, item = threadIdx.x & (p.lanes - 1);
    const int in_group = slot / p.side, first_head = (int)blockIdx.y * p.side * p.per + slot - in_group * p.side;
    if (in_group >= p.at_once) return;                   // (all threads of a row)
    const Item it(p, item);
    const __amdgpu_buffer_rsrc_t result = raw_buffer(p.out, INT32_MAX);   // (a result that is written through reaches no further)
    u32x4 w[2][2];                                       // of queries, of keys
#pragma unroll
    for (int i = 0; i < 2; i++) {
        w[i][0] = *reinterpret_cast<const u32x4*>(p.weight[i] + it.e0);
        w[i][1] = *reinterpret_cast<const u32x4*>(p.weight[i] + it.e1);
    }
    const int last_head = min(p.heads, ((int)blockIdx.y + 1) * p.side * p.per);
    for (int64_t t = (int64_t)blockIdx.x * p.at_once + in_group; t < p.tokens; t += (int64_t)gridDim.x * p.at_once) {
        const uint16_t* from = p.x + t * p.x_token;
        uint16_t* to = p.out + t * p.out_token;
        float c[Item::NP], s[Item::NP];
        for (int h = first_head; h < last_head; h += kNormAhead * p.side) {
            u32x4 a[kNormAhead], b[kNormAhead];
#pragma unroll
            for (int n = 0; n < kNormAhead; n++) {
                if (h + n * p.side >= last_head) break;
                const int64_t row = (int64_t)(h + n * p.side) * p.x_head;
                a[n] = rope_load<SOURCE>(from + row + it.e0);
                if (HALVES) b[n] = rope_load<SOURCE>(from + row + it.e1);
            }
            if (h == first_head) it.angles(p, t, item, c, s);   // while the first rows are under way
#pragma unroll
            for (int n = 0; n < kNormAhead; n++) {
                const int head = h + n * p.side;
                if (head >= last_head) break;
                const int which = head >= p.q_heads;
                float f[Item::NE], weight[Item::NE];
                it.numbers(a[n], b[n], f);
                it.numbers(which ? w[1][0] : w[0][0], which ? w[1][1] : w[0][1], weight);
                Item::normalize(p, f);
#pragma unroll
                for (int i = 0; i < Item::NE; i++) f[i] *= weight[i];
                it.rotate(f, c, s, 1.f);
                Item::words(f, a[n], b[n]);
                const int64_t row = (int64_t)head * p.out_head;
                if (it.present) rope_store<RESULT>(result, p.out, to + row + it.e0, a[n]);
                if (HALVES && it.turn) rope_store<RESULT>(result, p.out, to + row + it.e1, b[n]);
            }
        }
    }
}

// The weights' gradients are summed in 32 bits in an order that the launch's layout decides, and that goes by the sizes, HALVES and whether dx is heads of
// rows alone: a thread's rows, the rows that a workgroup's threads have side by side, then the workgroups (norm_weights_kernel).  (One layout for
// either dx would make it one order: 18 000 x 80 heads x 128 as rows 200 -> 227 us, or as heads of rows 218 -> 232, of 64 126 -> 159.)
template <class T, bool HALVES, int SOURCE, int RESULT>
__global__ __launch_bounds__(kNormThreads) void norm_rope_grad_kernel(NormParams p) {
    typedef NormItem<T, HALVES> Item;
    __shared__ float sums[2][kNormThreads * Item::NE];   // of either weight, [slot][element]
    const int slot = threadIdx.x / p.lanes, item = threadIdx.x & (p.lanes - 1);
    const int in_group = slot / p.side, first_head = (int)blockIdx.y * p.side * p.per + slot - in_group * p.side;
    const Item it(p, item);
    const __amdgpu_buffer_rsrc_t result = raw_buffer(p.out, INT32_MAX);
    u32x4 w[2][2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        w[i][0] = *reinterpret_cast<const u32x4*>(p.weight[i] + it.e0);
        w[i][1] = *reinterpret_cast<const u32x4*>(p.weight[i] + it.e1);
    }
    float dw[2][Item::NE];
#pragma unroll
    for (int i = 0; i < Item::NE; i++) dw[0][i] = dw[1][i] = 0.f;
    const int last_head = in_group < p.at_once ? min(p.heads, ((int)blockIdx.y + 1) * p.side * p.per) : 0;   // (a row's threads alike)
    for (int64_t t = (int64_t)blockIdx.x * p.at_once + in_group; t < p.tokens && first_head < last_head; t += (int64_t)gridDim.x * p.at_once) {
        const uint16_t* from = p.x + t * p.x_token;
        const uint16_t* grad = p.grad + t * p.grad_token;
        uint16_t* to = p.out + t * p.out_token;
        float c[Item::NP], s[Item::NP];
        for (int h = first_head; h < last_head; h += kNormGradAhead * p.side) {
            u32x4 a[kNormGradAhead], b[kNormGradAhead], ga[kNormGradAhead], gb[kNormGradAhead];
#pragma unroll
            for (int n = 0; n < kNormGradAhead; n++) {
                const int head = h + n * p.side;
                if (head >= last_head) break;
                const uint16_t* row = from + head * p.x_head;
                const uint16_t* grad_row = grad + head * p.grad_head;
                a[n] = rope_load<SOURCE>(row + it.e0);
                ga[n] = rope_load<SOURCE>(grad_row + it.e0);
                if (HALVES) {
                    b[n] = rope_load<SOURCE>(row + it.e1);
                    gb[n] = rope_load<SOURCE>(grad_row + it.e1);
                }
            }
            if (h == first_head) it.angles(p, t, item, c, s);
#pragma unroll
            for (int n = 0; n < kNormGradAhead; n++) {
                const int head = h + n * p.side;
                if (head >= last_head) break;
                const int which = head >= p.q_heads;
                float f[Item::NE], g[Item::NE], weight[Item::NE];
                it.numbers(a[n], b[n], f);
                it.numbers(ga[n], gb[n], g);
                it.numbers(which ? w[1][0] : w[0][0], which ? w[1][1] : w[0][1], weight);
                it.rotate(g, c, s, -1.f);
                const float r = Item::normalize(p, f);
                float along = 0.f;
#pragma unroll
                for (int i = 0; i < Item::NE; i++) {
                    dw[0][i] += which ? 0.f : g[i] * f[i];
                    dw[1][i] += which ? g[i] * f[i] : 0.f;
                    g[i] *= weight[i];
                    along += g[i] * f[i];
                }
                along = row_sum(along, p.lanes) * p.inv_E;
#pragma unroll
                for (int i = 0; i < Item::NE; i++) f[i] = r * (g[i] - f[i] * along);
                Item::words(f, a[n], b[n]);
                const int64_t row = (int64_t)head * p.out_head;
                if (it.present) rope_store<RESULT>(result, p.out, to + row + it.e0, a[n]);
                if (HALVES && it.turn) rope_store<RESULT>(result, p.out, to + row + it.e1, b[n]);
            }
        }
    }
    // the rows that the workgroup's threads have side by side
#pragma unroll
    for (int i = 0; i < 2; i++)
        if (it.present) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                sums[i][slot * p.E + it.e0 + e] = dw[i][e];
                if (HALVES && it.turn) sums[i][slot * p.E + it.e1 + e] = dw[i][Item::NE - 8 + e];
            }
        }
    __syncthreads();
    float* mine = p.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.E;
    const int slots = kNormThreads / p.lanes;
    for (int e = threadIdx.x; e < 2 * p.E; e += kNormThreads) {
        const float* column = e < p.E ? sums[0] + e : sums[1] + e - p.E;
        float sum = 0.f;
#pragma unroll 8
        for (int n = 0; n < slots; n++) sum += column[n * p.E];
        mine[e] = sum;
    }
}

// The workgroups' sums joined: 16 columns to a workgroup, 64 threads to a column with eight sums each under way.
__global__ __launch_bounds__(1024) void norm_weights_kernel(const float* partial, int workgroups, int E, float* dq, float* dk) {
    __shared__ float sums[64][16];
    const int column = threadIdx.x & 15, lane = threadIdx.x >> 4, at = min((int)blockIdx.x * 16 + column, 2 * E - 1);
    float sum = 0.f;
    for (int n0 = lane; n0 < workgroups; n0 += 512) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = partial[(int64_t)min(n0 + i * 64, workgroups - 1) * 2 * E + at];
#pragma unroll
        for (int i = 0; i < 8; i++) sum += n0 + i * 64 < workgroups ? v[i] : 0.f;
    }
    sums[lane][column] = sum;
    __syncthreads();
    if (lane > 0 || (int)blockIdx.x * 16 + column >= 2 * E) return;
#pragma unroll
    for (int n = 1; n < 64; n++) sum += sums[n][column];
    float* to = at < E ? dq : dk;
    if (to) to[at < E ? at : at - E] = sum;
}

// Workgroups of the gradient at most: as many sums of weights are joined.
constexpr int64_t kNormGradWorkgroups = 2048;
constexpr int kNormGradMost = 12;    // heads of a thread

// How a launch's threads are laid out: rows of a token side by side; a result in heads of rows gets four tokens' rows in one run (rope.hip).
constexpr int64_t kNormSmall = 1 << 17;   // threads
static int lanes_of(int items) {
    int lanes = 1;
    while (lanes < items) lanes *= 2;
    return lanes;
}
struct NormGrid {
    int items, lanes, side, per, at_once, parts;
    int64_t groups;          // of tokens
};
static NormGrid norm_grid(int tokens, int heads, int E, int64_t pairs, bool halves, bool heads_of_rows, bool grad) {
    NormGrid g;
    // Few rows: a head to a thread (8 tokens x 40 heads 5.1 -> 3.8 us; the gradient, whose workgroups have more to begin and end, loses)
    const bool small = !grad && (int64_t)tokens * heads * lanes_of(halves ? (int)(pairs / 8 + (E - 2 * pairs) / 8) : E / 8) <= kNormSmall;
    int per = small ? 1 : grad ? kNormGradAhead : kNormAhead;
    g.items = halves ? (int)(pairs / 8 + (E - 2 * pairs) / 8) : E / 8;
    g.lanes = lanes_of(g.items);
    const int slots = kNormThreads / g.lanes;
    g.side = std::min(heads_of_rows ? std::min(4, slots) : slots, (heads + per - 1) / per);
    // The gradient's angles serve more heads of a thread where there are workgroups enough: as many as divide the heads best
    if (grad && (int64_t)tokens * heads / (slots * kNormGradMost) >= kNormGradWorkgroups) {
        auto over = [&](int n) { return (heads + g.side * n - 1) / (g.side * n) * g.side * n; };
        for (int n = per; n <= kNormGradMost; n += kNormGradAhead)
            if (over(n) <= over(per)) per = n;
    }
    g.per = per;
    g.at_once = slots / g.side;
    g.parts = (heads + g.side * per - 1) / (g.side * per);
    g.groups = ((int64_t)tokens + g.at_once - 1) / g.at_once;
    return g;
}

template <class T, bool HALVES>
static void norm_launch(const NormParams& p, bool grad, dim3 grid, int source, int result, hipStream_t s) {
    auto go = [&](auto source_c, auto result_c) {
        constexpr int SOURCE = decltype(source_c)::value, RESULT = decltype(result_c)::value;
        if (grad) norm_rope_grad_kernel<T, HALVES, SOURCE, RESULT><<<grid, kNormThreads, 0, s>>>(p);
        else norm_rope_kernel<T, HALVES, SOURCE, RESULT><<<grid, kNormThreads, 0, s>>>(p);
    };
    typedef std::integral_constant<int, kThroughCaches> Near;
    typedef std::integral_constant<int, kPastL2> Far;
    typedef std::integral_constant<int, kKept> Kept;
    typedef std::integral_constant<int, kWrittenThrough> Through;
    if (result == kPastLastLevel) go(Far{}, std::integral_constant<int, kPastLastLevel>{});   // (then the source is as large)
    else if (source == kPastL2) result == kKept ? go(Far{}, Kept{}) : go(Far{}, Through{});
    else result == kKept ? go(Near{}, Kept{}) : go(Near{}, Through{});
}

// The checks and the launch that both share.
static int32_t norm_call(NormParams& p, bool grad, int64_t pairs_t, int64_t pairs_h, int64_t pairs_w, int halves, int dtype, dim3& grid, int* workgroups, hipStream_t s) {
    const int64_t pairs = pairs_t + pairs_h + pairs_w;
    if (!p.x || !p.out || (grad && !p.grad)) return CHIPMUNK_ERR_NULL;
    if (p.tokens <= 0 || p.heads <= 0 || p.heads > kRopeMostHeads || p.q_heads < 0 || p.q_heads > p.heads || p.E <= 0 || pairs_t < 0 || pairs_h < 0 || pairs_w < 0)
        return CHIPMUNK_ERR_SHAPE;
    if ((p.q_heads > 0 && !p.weight[0]) || (p.q_heads < p.heads && !p.weight[1]) || (pairs > 0 && (!p.pos || !p.freqs))) return CHIPMUNK_ERR_NULL;
    if (2 * pairs > p.E || !is_positive_finite_scalar(p.eps) || float_bits(p.eps) < 0x00800000u) return CHIPMUNK_ERR_SHAPE;
    if (p.E % 8 != 0 || p.E > 512 || pairs % (halves ? 8 : 4) != 0 || (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16)) return CHIPMUNK_ERR_UNSUPPORTED;
    if (p.tokens == 1) p.x_token = p.grad_token = p.out_token = 0;   // of one row alone a stride means nothing
    if (p.heads == 1) p.x_head = p.grad_head = p.out_head = 0;
    auto overlap = [&](int64_t token, int64_t head) { return rope_rows_overlap(token, head, p.tokens, p.heads, p.E); };
    if (overlap(p.x_token, p.x_head) || overlap(p.out_token, p.out_head) || (grad && overlap(p.grad_token, p.grad_head))) return CHIPMUNK_ERR_SHAPE;
    if (!aligned16(p.x) || !aligned16(p.out) || !aligned16(p.grad) || !aligned16(p.weight[0]) || !aligned16(p.weight[1]) || (reinterpret_cast<uintptr_t>(p.pos) & 3) ||
        (reinterpret_cast<uintptr_t>(p.freqs) & 7) || (p.x_token | p.x_head | p.out_token | p.out_head | (grad ? p.grad_token | p.grad_head : 0)) % 8 != 0)
        return CHIPMUNK_ERR_ALIGN;
    if (!p.weight[0]) p.weight[0] = p.weight[1];             // (no head has it)
    if (!p.weight[1]) p.weight[1] = p.weight[0];
    p.end0 = (int)pairs_t;
    p.end1 = (int)(pairs_t + pairs_h);
    p.pairs = (int)pairs;
    p.inv_E = 1.f / (float)p.E;
    const NormGrid g = norm_grid(p.tokens, p.heads, p.E, pairs, halves != 0, p.tokens > 1 && p.out_head > p.out_token, grad);
    p.items = g.items;
    p.lanes = g.lanes;
    p.side = g.side;
    p.per = g.per;
    p.at_once = g.at_once;
    const int64_t most = grad ? std::max<int64_t>(1, kNormGradWorkgroups / g.parts) : (1 << 22) / g.parts;   // (a launch has fewer than 2^32 threads)
    grid = dim3((uint32_t)std::min(g.groups, most), g.parts);
    if (workgroups) {
        *workgroups = (int)(grid.x * grid.y);
        return CHIPMUNK_OK;
    }
    const int64_t bytes = (int64_t)p.tokens * p.heads * p.E * 2;
    const bool whole_lines = (reinterpret_cast<uintptr_t>(p.out) & 127) == 0 && ((halves ? pairs | (p.E - 2 * pairs) : p.E) | p.out_token | p.out_head) % 64 == 0;
    const bool near = (__int128)(p.tokens - 1) * p.out_token + (__int128)(p.heads - 1) * p.out_head + p.E <= INT32_MAX / 2;   // a 32-bit offset reaches it all
    const int source = bytes > kRopeL2 ? kPastL2 : kThroughCaches, result = bytes > kRopeLastLevel ? kPastLastLevel : whole_lines && near ? kWrittenThrough : kKept;
    if (dtype == CHIPMUNK_DTYPE_BF16) halves ? norm_launch<Bf16, true>(p, grad, grid, source, result, s) : norm_launch<Bf16, false>(p, grad, grid, source, result, s);
    else halves ? norm_launch<Fp16, true>(p, grad, grid, source, result, s) : norm_launch<Fp16, false>(p, grad, grid, source, result, s);
    return launch_status();
}

}  // namespace chipmunk

using namespace chipmunk;

extern "C" int32_t chipmunk_norm_rope(const uint16_t* x, int64_t x_token_stride, int64_t x_head_stride, const uint16_t* q_weight, const uint16_t* k_weight, int q_heads,
                                      const int32_t* pos, const double* freqs, uint16_t* out, int64_t out_token_stride, int64_t out_head_stride, int tokens, int heads,
                                      int E, int pairs_t, int pairs_h, int pairs_w, float eps, int halves, int dtype, void* stream) {
    NormParams p{x, nullptr, out, {q_weight, k_weight}, pos, freqs, nullptr, x_token_stride, x_head_stride, 0, 0, out_token_stride, out_head_stride, tokens, heads, q_heads, E};
    p.eps = eps;
    dim3 grid;
    return norm_call(p, false, pairs_t, pairs_h, pairs_w, halves, dtype, grid, nullptr, static_cast<hipStream_t>(stream));
}

extern "C" size_t chipmunk_norm_rope_grad_workspace_bytes(int tokens, int heads, int E) {
    if (tokens <= 0 || heads <= 0 || heads > kRopeMostHeads || E <= 0 || E % 8 != 0 || E > 512) return 0;
    // at most so many workgroups, and never more than rows of heads or parts of the heads
    const int64_t rows = (int64_t)tokens * heads;
    return (size_t)std::min<int64_t>(rows, std::max<int64_t>(kNormGradWorkgroups, heads)) * 2 * E * sizeof(float);
}

extern "C" int32_t chipmunk_norm_rope_grad(const uint16_t* grad, int64_t grad_token_stride, int64_t grad_head_stride, const uint16_t* x, int64_t x_token_stride,
                                           int64_t x_head_stride, const uint16_t* q_weight, const uint16_t* k_weight, int q_heads, const int32_t* pos,
                                           const double* freqs, uint16_t* dx, int64_t dx_token_stride, int64_t dx_head_stride, float* dq_weight, float* dk_weight,
                                           int tokens, int heads, int E, int pairs_t, int pairs_h, int pairs_w, float eps, int halves, int dtype, void* ws,
                                           size_t ws_bytes, void* stream) {
    NormParams p{x, grad, dx, {q_weight, k_weight}, pos, freqs, static_cast<float*>(ws), x_token_stride, x_head_stride, grad_token_stride, grad_head_stride, dx_token_stride,
                 dx_head_stride, tokens, heads, q_heads, E};
    p.eps = eps;
    if ((q_heads > 0 && !dq_weight) || (q_heads < heads && !dk_weight)) return CHIPMUNK_ERR_NULL;
    if ((reinterpret_cast<uintptr_t>(dq_weight) | reinterpret_cast<uintptr_t>(dk_weight)) & 3 || !aligned16(ws)) return CHIPMUNK_ERR_ALIGN;
    dim3 grid;
    int workgroups = 0;
    NormParams checked = p;
    int32_t status = norm_call(checked, true, pairs_t, pairs_h, pairs_w, halves, dtype, grid, &workgroups, nullptr);
    if (status != CHIPMUNK_OK) return status;
    if (!ws || ws_bytes < (size_t)workgroups * 2 * E * sizeof(float)) return CHIPMUNK_ERR_WORKSPACE;
    const auto s = static_cast<hipStream_t>(stream);
    status = norm_call(p, true, pairs_t, pairs_h, pairs_w, halves, dtype, grid, nullptr, s);
    if (status != CHIPMUNK_OK) return status;
    norm_weights_kernel<<<(2 * E + 15) / 16, 1024, 0, s>>>(p.partial, workgroups, E, dq_weight, dk_weight);
    return launch_status();
}
