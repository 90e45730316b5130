// Linear layers: out = act(x w^T + bias) + residual, x [N, D], w [F, D], out [N, F].
//
// The product is formed as w x^T, so that a lane holds consecutive output columns of one row (P: rows of w = output columns, Q:
// rows of x = output rows), and everything behind it happens on the accumulators: bias, activation and residual in 32 bits,
// one rounding.
#include "element.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace chipmunk {

struct LinearParams {
    const uint16_t* x;
    const uint16_t* w;
    const uint16_t* bias;
    const uint16_t* residual;
    uint16_t* out;
    int64_t ldx, ldr, ldo;
    int N, D, F, act;
    int past;                // LinearPast
    int tiles_p, tiles_q;
};

template <int ACT>
__device__ __forceinline__ float activation(float y) {
    // x (1 + erf(x / sqrt 2)) / 2 = max(x, 0) - |x| h(|x|), h(z) = erfc(z / sqrt 2) / 2 = exp(-z^2 / 2) t P(t) with t = 1 / (1 + 0.362 z).
    // P was fitted here to the least relative error, 7.9e-7 for z up to 14 (2.4e-6 at 15, where the exponential leaves 32 bits: zero);
    // with the rounding of 32 bits the result is off by 2.4e-7 at most.  With erff, two branches that a wave mostly takes both, the
    // results cost more than the product: 2148 rows, 256 -> 8192, 53.6 us, now 31.7 (no activation: 22.8).  The bound on x keeps infinity
    // from 0 times infinity; minus infinity is to have it, as in the formula, which gives NaN there, and the other activations' too.
    if constexpr (ACT == CHIPMUNK_ACT_GELU_ERF) {
        const float z = fmaxf(fminf(y, 30.f), -y), t = __builtin_amdgcn_rcpf(__builtin_fmaf(z, 0.362f, 1.f));
        float h = 0.047938276f;
        h = __builtin_fmaf(h, t, -0.18000965f);
        h = __builtin_fmaf(h, t, 0.17661723f);
        h = __builtin_fmaf(h, t, 0.0288315f);
        h = __builtin_fmaf(h, t, 0.13942969f);
        h = __builtin_fmaf(h, t, 0.14268932f);
        h = __builtin_fmaf(h, t, 0.1445039f) * t * __builtin_amdgcn_exp2f(y * y * -0.72134752f);
        return __builtin_fmaf(-z, h, fmaxf(y, 0.f));
    }
    // x (1 + tanh(u)) / 2 = x / (1 + exp(-2 u)), u = sqrt(2 / pi) (x + 0.044715 x^3);  -2 u log2(e) = x (A + B x^2).  The reciprocal
    // and the exponential are an ulp of 32 bits off, and the result has 8 or 11 bits.
    if constexpr (ACT == CHIPMUNK_ACT_GELU_TANH)
        return y * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y * __builtin_fmaf(y * y, -0.10294324f, -2.3022082f)));
    if constexpr (ACT == CHIPMUNK_ACT_SILU) return y * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y * -1.4426950408889634f));
    return y;
}

// f(std::integral_constant<int, ACT>): the activation's form is chosen once per tile
template <typename F>
__device__ __forceinline__ void with_activation(int act, F&& f) {
    if (act == CHIPMUNK_ACT_NONE) f(std::integral_constant<int, CHIPMUNK_ACT_NONE>{});
    else if (act == CHIPMUNK_ACT_GELU_TANH) f(std::integral_constant<int, CHIPMUNK_ACT_GELU_TANH>{});
    else if (act == CHIPMUNK_ACT_SILU) f(std::integral_constant<int, CHIPMUNK_ACT_SILU>{});
    else f(std::integral_constant<int, CHIPMUNK_ACT_GELU_ERF>{});
}

// Rows of an operand from row0 on, `rows` of them at most, of `length` elements `ld` apart: what lies behind the last one reads
// as zero.
__device__ __forceinline__ i32x4 operand_rows(const uint16_t* base, int64_t ld, int64_t row0, int rows, int length) {
    return raw_buffer_words(base + row0 * ld, (uint32_t)((rows - 1) * ld + length) * 2u);
}
constexpr uint32_t kNowhere = 0x80000000u;   // an offset behind every such buffer: the load gives zeros

// Asynchronous 16-byte load to LDS through a buffer, with a wave-uniform part of the offset, which lies inside the buffer.  Not a memory access to the compiler,
// so LDS reads of other stages may be scheduled across it; waits and barriers order it against those of its own.
__device__ __forceinline__ void load_rows_to_lds_16B(i32x4 buffer, uint32_t byte_offset, uint32_t uniform_offset, uint32_t lds_wave_base) {
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds_wave_base), "v"(byte_offset), "s"(buffer), "s"(uniform_offset));
}

// The tile of a workgroup: each XCD takes one run of the tiles, in bands of eight column tiles, so that what its CUs work on at a
// time shares operands in its L2.
__device__ __forceinline__ bool linear_tile(int tiles_p, int tiles_q, int* tp, int* tq) {
    const int tiles = tiles_p * tiles_q, each = tiles >> 3, more = tiles & 7;
    const int xcd = (int)blockIdx.x & 7, slot = (int)blockIdx.x >> 3;
    if (slot >= each + (xcd < more ? 1 : 0)) return false;
    const int tile = xcd * each + min(xcd, more) + slot;
    const int band = tile / (8 * tiles_q), in_band = tile - band * 8 * tiles_q;
    const int height = min(8, tiles_p - 8 * band);
    *tq = in_band / height;
    *tp = 8 * band + (in_band - *tq * height);
    return true;
}

// The result or the residual from (row0, col0) on, for 16-byte accesses to `rows` rows at most; nothing is read or stored at kNowhere.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const LinearParams& p, const uint16_t* base, int64_t ld, int row0, int col0, int rows) {
    const int there = col0 < p.F ? max(min(rows, p.N - row0), 0) : 0;
    return raw_buffer(base + (int64_t)row0 * ld + col0, there > 0 ? (uint32_t)((there - 1) * ld + p.F - col0) * 2u : 0u);
}
__device__ __forceinline__ u32x4 load_16B(__amdgpu_buffer_rsrc_t from, uint32_t offset) { return __builtin_amdgcn_raw_buffer_load_b128(from, (int)offset, 0, 0); }
// A result whose rows are whole lines of 128 bytes is written through the L2s as it comes, and past the last-level cache where it is larger
// than that; other lines come in parts, which meet in an L2 (64 columns of a row at a time; us with a kernel that reads the result,
// kept in the L2s / written through / past the last-level cache: 8000 x 4096 60.3, 56.2, 64.2; 32 768 x 2048 105, 99, 103; 75 600 x 5120
// 696, 673, 633; 16 000 x 3000 78, 98, 86).
enum LinearPast { kKept, kThrough, kPastLastLevel };
constexpr int64_t kLinearLastLevel = 256 << 20;
template <int N>
__device__ __forceinline__ void store_16B(const u32x4 (&values)[N], __amdgpu_buffer_rsrc_t to, const uint32_t (&offsets)[N], int past) {
    auto store = [&](auto bits) {
#pragma unroll
        for (int n = 0; n < N; n++) __builtin_amdgcn_raw_buffer_store_b128(values[n], to, (int)offsets[n], 0, decltype(bits)::value);
    };
    if (past == kKept) store(std::integral_constant<int, 0>{});
    else if (past == kThrough) store(std::integral_constant<int, 16>{});   // sc1
    else store(std::integral_constant<int, 2>{});                          // nt
}

// Results of a wave: PB x QB blocks of 16 columns x 16 rows from (col0, row0) on.  The residual's values there come ahead of them: loaded
// block by block, one latency behind the other: 18 000 rows, 5120 -> 5120 706 us, so 696; 8000, 512 -> 4096 58 and 54.6.
template <int PB, int QB>
struct Residual {
    u32x4 of[PB / 2][QB];                                 // a lane's eight columns of each pair of blocks
};
template <int PB, int QB>
__device__ __forceinline__ void load_residual(Residual<PB, QB>& old, const LinearParams& p, int col0, int row0, int g, int l16) {
#pragma unroll
    for (int pair = 0; pair < PB / 2; pair++)
#pragma unroll
        for (int c = 0; c < QB; c++) old.of[pair][c] = u32x4{0, 0, 0, 0};
    if (!p.residual) return;
    const __amdgpu_buffer_rsrc_t from = rows_from(p, p.residual, p.ldr, row0, col0, QB * 16);
#pragma unroll
    for (int pair = 0; pair < PB / 2; pair++)
#pragma unroll
        for (int c = 0; c < QB; c++) {
            const int row = c * 16 + l16, at = pair * 32 + columns_of_lane(g);
            old.of[pair][c] = load_16B(from, row0 + row < p.N && col0 + at < p.F ? (uint32_t)(row * (uint32_t)p.ldr + at) * 2u : kNowhere);
        }
}
template <class T, int ACT, int PB, int QB>
__device__ __forceinline__ void store_blocks(const LinearParams& p, const f32x4 (&acc)[PB][QB], const Residual<PB, QB>& residual, int col0, int row0, int g, int l16) {
    static_assert(PB % 2 == 0, "blocks of columns go in pairs");
    // the lane's eight columns of block c of rows and of one pair of blocks of columns
    auto eight_columns = [&](int pair, int c, const u32x2 (&bias)[2]) {
        u32x2 old[2];
        from_columns(residual.of[pair][c], old);
        u32x2 result[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            f32x4 v = acc[2 * pair + i][c];
            // (the widest tiles' sums stay in their accumulation registers up to here: copied ahead of the activations' branches they would spill)
            if (PB * QB == 8) asm volatile("" : "+a"(v));
            result[i] = u32x2{T::pack(activation<ACT>(v[0] + T::low(bias[i][0])) + T::low(old[i][0]), activation<ACT>(v[1] + T::high(bias[i][0])) + T::high(old[i][0])),
                              T::pack(activation<ACT>(v[2] + T::low(bias[i][1])) + T::low(old[i][1]), activation<ACT>(v[3] + T::high(bias[i][1])) + T::high(old[i][1]))};
        }
        return to_columns(result[0], result[1]);
    };
    const __amdgpu_buffer_rsrc_t to = rows_from(p, p.out, p.ldo, row0, col0, QB * 16);
    constexpr int PAIRS = PB % 4 == 0 ? 2 : 1;            // at a time: 64 columns are 128 bytes, and rows of whole lines are stored
#pragma unroll
    for (int pair = 0; pair < PB / 2; pair += PAIRS) {
        const int col = col0 + pair * 32;
        u32x2 bias[PAIRS][2];
#pragma unroll
        for (int n = 0; n < PAIRS; n++)
#pragma unroll
            for (int i = 0; i < 2; i++) bias[n][i] = p.bias ? *reinterpret_cast<const u32x2*>(p.bias + min(col + n * 32 + i * 16 + 4 * g, p.F - 4)) : u32x2{0, 0};
#pragma unroll
        for (int c = 0; c < QB; c++) {
            u32x4 columns[PAIRS];
#pragma unroll
            for (int n = 0; n < PAIRS; n++) columns[n] = eight_columns(pair + n, c, bias[n]);
            if constexpr (PAIRS == 2) exchange_8_apart(columns[0], columns[1]);
            uint32_t offset[PAIRS];
#pragma unroll
            for (int n = 0; n < PAIRS; n++) {
                const int at = pair * 32 + columns_of_lane(g) + (PAIRS == 2 ? (l16 >> 3) * 32 : 0), row = c * 16 + (PAIRS == 2 ? n * 8 + (l16 & 7) : l16);
                offset[n] = row0 + row < p.N && col0 + at < p.F ? (uint32_t)(row * (uint32_t)p.ldo + at) * 2u : kNowhere;
            }
            store_16B(columns, to, offset, PAIRS == 2 ? p.past : kKept);
            if (PB * QB == 8) __builtin_amdgcn_sched_barrier(0);
        }
    }
}
template <class T, int PB, int QB>
__device__ __forceinline__ void linear_store(const LinearParams& p, const f32x4 (&acc)[PB][QB], int col0, int row0, int g, int l16) {
    if constexpr (PB > 1) {
        Residual<PB, QB> residual;
        load_residual(residual, p, col0, row0, g, l16);
        with_activation(p.act, [&](auto form) { store_blocks<T, decltype(form)::value, PB, QB>(p, acc, residual, col0, row0, g, l16); });
    } else {
        with_activation(p.act, [&](auto form) {           // four columns of a lane at a time
            constexpr int ACT = decltype(form)::value;
            const int at = col0 + 4 * g;
            const u32x2 bias = p.bias ? *reinterpret_cast<const u32x2*>(p.bias + min(at, p.F - 4)) : u32x2{0, 0};
#pragma unroll
            for (int c = 0; c < QB; c++) {
                const int row = row0 + c * 16 + l16;
                if (row >= p.N || at >= p.F) continue;
                const u32x2 old = p.residual ? *reinterpret_cast<const u32x2*>(p.residual + (int64_t)row * p.ldr + at) : u32x2{0, 0};
                const f32x4 v = acc[0][c];
                *reinterpret_cast<u32x2*>(p.out + (int64_t)row * p.ldo + at) =
                    u32x2{T::pack(activation<ACT>(v[0] + T::low(bias[0])) + T::low(old[0]), activation<ACT>(v[1] + T::high(bias[0])) + T::high(old[0])),
                          T::pack(activation<ACT>(v[2] + T::low(bias[1])) + T::low(old[1]), activation<ACT>(v[3] + T::high(bias[1])) + T::high(old[1]))};
            }
        });
    }
}

// The same for blocks of 32 x 32: a lane holds, of its row (lane % 32), four runs of four columns, 8 i + 4 (lane / 32) on.
template <class T, int PN, int QN>
__device__ __forceinline__ void linear_store_32(const LinearParams& p, const f32x16 (&acc)[PN][QN], int col0, int row0, int lane) {
    const int high = lane >> 5;
    u32x4 residual[4][QN];                               // by 16 columns
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
        for (int c = 0; c < QN; c++) residual[m][c] = u32x4{0, 0, 0, 0};
    if (p.residual) {
        const __amdgpu_buffer_rsrc_t from = rows_from(p, p.residual, p.ldr, row0, col0, QN * 32);
#pragma unroll
        for (int m = 0; m < 4; m++)
#pragma unroll
            for (int c = 0; c < QN; c++) {
                const int row = c * 32 + (lane & 31), at = m * 16 + 8 * high;
                residual[m][c] = load_16B(from, row0 + row < p.N && col0 + at < p.F ? (uint32_t)(row * (uint32_t)p.ldr + at) * 2u : kNowhere);
            }
    }
    with_activation(p.act, [&](auto form) {
        constexpr int ACT = decltype(form)::value;
        static_assert(PN == 2, "64 columns: rows of whole lines of 128 bytes are stored");
        const __amdgpu_buffer_rsrc_t to = rows_from(p, p.out, p.ldo, row0, col0, QN * 32);
        u32x2 bias[4][2];                                // of the lane's first run and its second of each 16 columns
#pragma unroll
        for (int m = 0; m < 4; m++)
#pragma unroll
            for (int i = 0; i < 2; i++) bias[m][i] = p.bias ? *reinterpret_cast<const u32x2*>(p.bias + min(col0 + m * 16 + i * 8 + 4 * high, p.F - 4)) : u32x2{0, 0};
#pragma unroll
        for (int c = 0; c < QN; c++) {
            u32x4 columns[4];
#pragma unroll
            for (int m = 0; m < 4; m++) {
                u32x2 old[2], result[2];
                from_columns_32(residual[m][c], old);
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const int e = 8 * (m & 1) + 4 * i + 2 * h;
                        result[i][h] = T::pack(activation<ACT>(acc[m >> 1][c][e] + T::low(bias[m][i][h])) + T::low(old[i][h]),
                                               activation<ACT>(acc[m >> 1][c][e + 1] + T::high(bias[m][i][h])) + T::high(old[i][h]));
                    }
                columns[m] = to_columns_32(result[0], result[1]);
            }
            // rows of the 32 by their bits 4 and 3: columns[2 * bit 4 + bit 3] afterwards, the 16 columns by the lane's
            exchange_8_apart(columns[0], columns[1]);
            exchange_8_apart(columns[2], columns[3]);
            exchange_16_apart(columns[0], columns[2]);
            exchange_16_apart(columns[1], columns[3]);
            uint32_t offset[4];
#pragma unroll
            for (int m = 0; m < 4; m++) {
                const int row = c * 32 + m * 8 + (lane & 7), at = (lane >> 3 & 3) * 16 + 8 * high;
                offset[m] = row0 + row < p.N && col0 + at < p.F ? (uint32_t)(row * (uint32_t)p.ldo + at) * 2u : kNowhere;
            }
            store_16B(columns, to, offset, p.past);
        }
    });
}

// Waits until at most `left` steps of N transfers each are outstanding; there are MOST of them at most.
template <int N, int MOST>
__device__ __forceinline__ void wait_steps(int left) {
    if constexpr (MOST == 0) {
        wait_vmem_at_most<0>();
    } else {
        if (left >= MOST) wait_vmem_at_most<N * MOST>();
        else wait_steps<N, MOST - 1>(left);
    }
}

// Tiles of 32 PB columns x 32 QB rows.  The contraction goes in steps of 64; TEAMS of four waves (each wave half the columns and
// half the rows) take the steps in turn, each team through a ring of STAGES stages of its own in LDS, and their sums meet at the
// end.  A wave holds the operands of a slice (32 of the contraction) ahead, so a stage is free again halfway through its step.
//
// Bound: for few tiles the latency of a step, of which STAGES - 1 are on their way; with every CU busy what the CUs can fetch (see
// linear_block_kernel): 2000 rows, 4096 -> 4096 by 128 x 128 56 us (1.2 PFLOP/s).
template <class T, int PB, int QB, int STAGES, int TEAMS>
__global__ __launch_bounds__(256 * TEAMS, 2) void linear_ring_kernel(LinearParams p) {
    constexpr int BP = 32 * PB, BQ = 32 * QB, STAGE = (BP + BQ) * 128;
    constexpr int NP = BP / 32, NQ = BQ / 32;            // transfers of a wave per step: eight rows of 128 bytes each
    constexpr int NT = NP + NQ;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), team = wave >> 2, w = wave & 3;
    const int wp = w >> 1, wq = w & 1, g = lane >> 4, l16 = lane & 15;
    int tp, tq;
    if (!linear_tile(p.tiles_p, p.tiles_q, &tp, &tq)) return;
    const int p0 = tp * BP, q0 = tq * BQ;
    const i32x4 wbuf = operand_rows(p.w, p.D, p0, min(BP, p.F - p0), p.D);
    const i32x4 xbuf = operand_rows(p.x, p.ldx, q0, min(BQ, p.N - q0), p.D);

    // 16-byte chunks XOR-swizzled by the row: the same chunk in all transfers of a lane
    const int first_row = w * 8 + (lane >> 3), chunk = (lane & 7) ^ ((first_row >> 1) & 7);
    uint32_t woff[NP], xoff[NQ];
#pragma unroll
    for (int n = 0; n < NP; n++) woff[n] = (uint32_t)(n * 32 + first_row) * (uint32_t)(p.D * 2) + chunk * 16u;
#pragma unroll
    for (int n = 0; n < NQ; n++) xoff[n] = (uint32_t)(n * 32 + first_row) * (uint32_t)(p.ldx * 2) + chunk * 16u;
    const int all_chunks = p.D / 8, all_steps = (p.D + 63) / 64, steps = (all_steps + TEAMS - 1) / TEAMS;
    const uint32_t lds0 = lds_address(smem) + (uint32_t)(team * STAGES * STAGE);
    // transfer n of the team's step t, zeros where the contraction ends.  (A team may have one step less than the other; in its place the last
    // step's offset stands, which is inside even a single row: the hardware takes the uniform offset from the buffer's size.)
    auto request = [&](int t, int n) {
        const int step = t * TEAMS + team, inside = TEAMS == 1 ? step : min(step, all_steps - 1);
        const uint32_t to = lds0 + (uint32_t)(t % STAGES * STAGE + (n < NP ? n : n - NP) * 4096 + (n < NP ? 0 : BP * 128) + w * 1024);
        const uint32_t off = step * 8 + chunk < all_chunks ? (n < NP ? woff[n < NP ? n : 0] : xoff[n < NP ? 0 : n - NP]) : kNowhere;
        load_rows_to_lds_16B(n < NP ? wbuf : xbuf, off, (uint32_t)inside * 128u, to);
    };
    auto request_all = [&](int t) {
#pragma unroll
        for (int n = 0; n < NT; n++) request(t, n);
    };
    static_assert((STAGES - 1) * NT < 64, "what a wave's counter counts");

    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem) + (uint32_t)(team * STAGES * STAGE);
    typedef typename T::x8 x8;
    const uint32_t in_row = (uint32_t)((g ^ ((l16 >> 1) & 7)) * 16);
    uint32_t pat[2], qat[2];                             // by slice of 32; opaque, so that what is added stays in the reads' offset field
#pragma unroll
    for (int ks = 0; ks < 2; ks++) {
        pat[ks] = smem_at + (uint32_t)((wp * PB * 16 + l16) * 128) + (in_row ^ (64u * ks));
        qat[ks] = smem_at + (uint32_t)(BP * 128 + (wq * QB * 16 + l16) * 128) + (in_row ^ (64u * ks));
        asm volatile("" : "+v"(pat[ks]), "+v"(qat[ks]));
    }
    struct Operands {
        x8 P[PB], Q[QB];
    } first, second;                                     // of a step's two slices
    constexpr int READS = PB + QB, PRODUCTS = PB * QB;
    auto read = [&](Operands& op, uint32_t stage, int ks, int n) {   // read n of a slice: P's blocks, then Q's
        if (n < PB) op.P[n < PB ? n : 0] = __builtin_bit_cast(x8, lds_read_b128(pat[ks] + stage + n * 2048));
        else op.Q[n < PB ? 0 : n - PB] = __builtin_bit_cast(x8, lds_read_b128(qat[ks] + stage + (n - PB) * 2048));
    };
    f32x4 acc[PB][QB] = {};
    // A slice's products; `beside(i)` puts what is read and requested meanwhile in front of product i: in one go ahead of the
    // products, all waves of the CU would read at a time and then multiply at a time.
    auto multiply = [&](const Operands& op, auto&& beside) {
#pragma unroll
        for (int i = 0; i < PRODUCTS; i++) {
            beside(i);
            acc[i / QB][i % QB] = T::product(op.P[i / QB], op.Q[i % QB], acc[i / QB][i % QB]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int t = 0; t < min(STAGES, steps); t++) request_all(t);
    wait_steps<NT, STAGES - 1>(min(STAGES, steps) - 1);
    lds_accesses_then_barrier();
#pragma unroll
    for (int n = 0; n < READS; n++) read(first, 0, 0, n);
    auto step = [&](auto more_c, int t) {
        constexpr bool more = decltype(more_c)::value;   // t + STAGES < steps
        const uint32_t here = (uint32_t)(t % STAGES * STAGE), there = (uint32_t)((t + 1) % STAGES * STAGE);
        multiply(first, [&](int i) {
#pragma unroll
            for (int n = i * READS / PRODUCTS; n < (i + 1) * READS / PRODUCTS; n++) read(second, here, 1, n);
        });
        if (more) wait_vmem_at_most<(STAGES - 2) * NT>();   // step t + 1 has landed
        else wait_steps<NT, STAGES - 2>(steps - 2 - t);
        lds_accesses_then_barrier();                     // for every wave; and every wave holds what is left of step t
        multiply(second, [&](int i) {
            // (behind the last step the reads find what an earlier one left)
#pragma unroll
            for (int n = i * READS / PRODUCTS; n < (i + 1) * READS / PRODUCTS; n++) read(first, there, 0, n);
            if (more) {
#pragma unroll
                for (int n = i * NT / PRODUCTS; n < (i + 1) * NT / PRODUCTS; n++) request(t + STAGES, n);
            }
        });
    };
    int t = 0;
#pragma unroll 1
    for (; t + STAGES < steps; t++) step(std::true_type{}, t);
#pragma unroll 1
    for (; t < steps; t++) step(std::false_type{}, t);
    const int col0 = p0 + wp * PB * 16, row0 = q0 + wq * QB * 16;
    if constexpr (TEAMS == 1) {
        linear_store<T, PB, QB>(p, acc, col0, row0, g, l16);
    } else {
        // every team's sums to LDS, then each team takes some blocks of rows and adds in the order of the teams
        lds_accesses_then_barrier();
        f32x4* sums = reinterpret_cast<f32x4*>(smem);
#pragma unroll
        for (int a = 0; a < PB; a++)
#pragma unroll
            for (int c = 0; c < QB; c++) sums[((wave * PB + a) * QB + c) * 64 + lane] = acc[a][c];
        lds_accesses_then_barrier();
        for (int c = team; c < QB; c += TEAMS) {
            f32x4 total[PB][1] = {};
#pragma unroll
            for (int v = 0; v < TEAMS; v++)
#pragma unroll
                for (int a = 0; a < PB; a++) total[a][0] += sums[(((v * 4 + w) * PB + a) * QB + c) * 64 + lane];
            linear_store<T, PB, 1>(p, total, col0, row0 + c * 16, g, l16);
        }
    }
}

// Tiles of 64 PN columns x 64 QN rows, four waves of half of either, one workgroup to a CU: where that makes one round of tiles, or
// little more.  One wave per SIMD keeps the matrix pipe full only with products of 32 x 32 (2.01 PFLOP/s; of 16 x 16: 1.52).
//
// Bound: a step of 128 x 128 takes 0.36 us on a few CUs, of which its products are 0.25, and 0.55 us where all of them fetch: a CU has 60
// lines of 128 bytes in flight in the mean, for 340 cycles each, which is 23 bytes a clock, a third of them from beyond the L2 (333 rows, 4096 -> 10 880:
// 41 us; more stages, or waves that fetch nothing but weights or rows, changed nothing).
template <class T, int PN, int QN, int STAGES>
__global__ __launch_bounds__(256, 1) void linear_block_kernel(LinearParams p) {
    typedef typename T::x8 x8;
    constexpr int BP = 64 * PN, BQ = 64 * QN, STAGE = (BP + BQ) * 128;
    constexpr int NP = BP / 32, NQ = BQ / 32, NT = NP + NQ;                   // transfers per step of a wave
    static_assert((STAGES - 1) * NT < 64, "what a wave's counter counts");
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = w >> 1, wq = w & 1, l32 = lane & 31, high = lane >> 5;
    int tp, tq;
    if (!linear_tile(p.tiles_p, p.tiles_q, &tp, &tq)) return;
    const int p0 = tp * BP, q0 = tq * BQ;
    const i32x4 wbuf = operand_rows(p.w, p.D, p0, min(BP, p.F - p0), p.D);
    const i32x4 xbuf = operand_rows(p.x, p.ldx, q0, min(BQ, p.N - q0), p.D);
    const int first_row = w * 8 + (lane >> 3), chunk = (lane & 7) ^ ((first_row >> 1) & 7);
    uint32_t off[NT];
#pragma unroll
    for (int n = 0; n < NT; n++)
        off[n] = (n < NP ? (uint32_t)(n * 32 + first_row) * (uint32_t)(p.D * 2) : (uint32_t)((n - NP) * 32 + first_row) * (uint32_t)(p.ldx * 2)) + chunk * 16u;
    const int all_chunks = p.D / 8, steps = (p.D + 63) / 64;
    const uint32_t lds0 = lds_address(smem) + w * 1024;
    uint32_t put = lds0;                                 // the stage that the next request fills
    auto request = [&](int t, int n) {                   // zeros where the contraction ends
        load_rows_to_lds_16B(n < NP ? wbuf : xbuf, t * 8 + chunk < all_chunks ? off[n] : kNowhere, (uint32_t)t * 128u, put + n * 4096);
    };
    auto filled = [&]() { put = put == lds0 + (STAGES - 1) * STAGE ? lds0 : put + STAGE; };

    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem);
    const uint32_t in_row = (uint32_t)((high ^ ((l32 >> 1) & 7)) * 16);
    uint32_t pat[4], qat[4];                             // by slice of 16
#pragma unroll
    for (int ks = 0; ks < 4; ks++) {
        pat[ks] = smem_at + (uint32_t)((wp * PN * 32 + l32) * 128) + (in_row ^ (32u * ks));
        qat[ks] = smem_at + (uint32_t)(BP * 128 + (wq * QN * 32 + l32) * 128) + (in_row ^ (32u * ks));
        asm volatile("" : "+v"(pat[ks]), "+v"(qat[ks]));
    }
    struct Operands {
        x8 P[2][PN], Q[2][QN];
    } first, second;                                     // of a step's two halves
    constexpr int READS = 2 * (PN + QN), PRODUCTS = 2 * PN * QN;
    auto read = [&](Operands& op, uint32_t stage, int half, int n) {
        const int ks = n / (PN + QN), i = n % (PN + QN);
        if (i < PN) op.P[ks][i < PN ? i : 0] = __builtin_bit_cast(x8, lds_read_b128(pat[half * 2 + ks] + stage + i * 4096));
        else op.Q[ks][i < PN ? 0 : i - PN] = __builtin_bit_cast(x8, lds_read_b128(qat[half * 2 + ks] + stage + (i - PN) * 4096));
    };
    f32x16 acc[PN][QN] = {};
    auto multiply = [&](const Operands& op, auto&& beside) {
#pragma unroll
        for (int i = 0; i < PRODUCTS; i++) {
            beside(i);
            const int ks = i / (PN * QN), a = i / QN % PN, c = i % QN;
            acc[a][c] = T::product(op.P[ks][a], op.Q[ks][c], acc[a][c]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int t = 0; t < min(STAGES, steps); t++) {
#pragma unroll
        for (int n = 0; n < NT; n++) request(t, n);
        filled();
    }
    wait_steps<NT, STAGES - 1>(min(STAGES, steps) - 1);
    lds_accesses_then_barrier();
    uint32_t here = 0;                                   // where the step's operands stand
#pragma unroll
    for (int n = 0; n < READS; n++) read(first, 0, 0, n);
    auto step = [&](auto more_c, int t) {
        constexpr bool more = decltype(more_c)::value;   // t + STAGES < steps
        multiply(first, [&](int i) {
#pragma unroll
            for (int n = i * READS / PRODUCTS; n < (i + 1) * READS / PRODUCTS; n++) read(second, here, 1, n);
        });
        if (more) wait_vmem_at_most<(STAGES - 2) * NT>();   // step t + 1 has landed
        else wait_steps<NT, STAGES - 2>(steps - 2 - t);
        lds_accesses_then_barrier();                     // for every wave; and every wave holds what is left of step t
        here = here == (STAGES - 1) * STAGE ? 0 : here + STAGE;
        multiply(second, [&](int i) {
            // (behind the last step the reads find what an earlier one left)
#pragma unroll
            for (int n = i * READS / PRODUCTS; n < (i + 1) * READS / PRODUCTS; n++) read(first, here, 0, n);
            if (more) {
#pragma unroll
                for (int n = i * NT / PRODUCTS; n < (i + 1) * NT / PRODUCTS; n++) request(t + STAGES, n);
            }
        });
        if (more) filled();
    };
    int t = 0;
#pragma unroll 1
    for (; t + STAGES < steps; t++) step(std::true_type{}, t);
#pragma unroll 1
    for (; t < steps; t++) step(std::false_type{}, t);
    linear_store_32<T, PN, QN>(p, acc, p0 + wp * PN * 32, q0 + wq * QN * 32, lane);
}

// C += A B with C in accumulation registers, where the compiler would move 128 accumulators among the others and spill.  It does
// not know when such a product has landed: whatever else reads C waits first (finish_products), and no accumulator may be
// moved inside a loop (a test looks at the compiled kernels).
template <class T>
__device__ __forceinline__ void product_in_place(f32x4& c, typename T::x8 a, typename T::x8 b) {
    if constexpr (std::is_same_v<T, Bf16>) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
__device__ __forceinline__ void finish_products() { asm volatile("s_nop 15\n\ts_nop 15" ::: "memory"); }

// Tiles of 256 x 256, eight waves, contraction steps of 64.  A step's operands are four half tiles of 16 KB in LDS (P0, P1, Q0,
// Q1: 128 rows each), two steps deep; each wave multiplies 128 columns x 64 rows as four quadrants P_i x Q_j of 64 x 32.
//
// Bound: the matrix cores.  Waves 0-3 and 4-7 take turns: while one group runs 32 products the other reads the operands of its
// next ones from LDS and requests half tiles that both groups have read:
//     slot    reads                        requests                       then multiplies
//     0       P0 and Q1 (step t)           Q0 (step t + 2), P1 (t + 1)    P0 x Q0, P0 x Q1
//     1       P1 (t) and Q0 (step t + 1)   P0 and Q1 (t + 2)              P1 x Q1, P1 x Q0
// A slot ends with its LDS reads complete and with the wave's share of what the next slot reads landed: all but the eight
// transfers of the last two slots.  CUT: the contraction's last step is not whole.
// 75 600 rows, 5120 -> 15 360: 8.44 ms (1.41 PFLOP/s, matrix pipes 78 % busy at 1.79 GHz, the power limit's clock).
constexpr int kWideHalf = 128 * 128;               // bytes of a half tile
constexpr int kWideStage = 4 * kWideHalf;
template <class T, bool CUT>
__global__ __launch_bounds__(512, 2) void linear_wide_kernel(LinearParams p) {
    typedef typename T::x8 x8;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = w >> 2, wq = w & 3, g = lane >> 4, l16 = lane & 15;
    int tp, tq;
    if (!linear_tile(p.tiles_p, p.tiles_q, &tp, &tq)) return;
    const int p0 = tp * 256, q0 = tq * 256;
    const i32x4 pbuf = operand_rows(p.w, p.D, p0, min(256, p.F - p0), p.D);
    const i32x4 qbuf = operand_rows(p.x, p.ldx, q0, min(256, p.N - q0), p.D);

    // a transfer: eight rows of 128 bytes, 16-byte chunks XOR-swizzled by the row
    uint32_t poff[2][2], qoff[2][2];               // [half][transfer]
    bool beyond[2];                                // the lane's chunk of the wave's transfers lies behind a cut step's end
    const int rest = CUT ? p.D % 64 / 8 : 8;
#pragma unroll
    for (int n = 0; n < 2; n++) {
        const int row = (w * 2 + n) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
        beyond[n] = chunk >= rest;
#pragma unroll
        for (int hf = 0; hf < 2; hf++) {
            poff[hf][n] = (uint32_t)(hf * 128 + row) * (uint32_t)(p.D * 2) + chunk * 16u;
            qoff[hf][n] = (uint32_t)(hf * 128 + row) * (uint32_t)(p.ldx * 2) + chunk * 16u;
        }
    }
    const int steps = (p.D + 63) / 64;
    const uint32_t lds0 = lds_address(smem);
    // half tile `hf` of P or Q of step t (past the end the last step again, into a place nobody reads)
    auto request = [&](bool is_q, int hf, int t) {
        const uint32_t to = lds0 + (uint32_t)((t & 1) * kWideStage + (is_q ? 2 : 0) * kWideHalf + hf * kWideHalf);
        const int from = min(t, steps - 1);
#pragma unroll
        for (int n = 0; n < 2; n++) {
            uint32_t off = is_q ? qoff[hf][n] : poff[hf][n];
            if (CUT) off = from == steps - 1 && beyond[n] ? kNowhere : off;
            load_rows_to_lds_16B(is_q ? qbuf : pbuf, off, (uint32_t)from * 128u, to + (w * 2 + n) * 1024);
        }
    };

    // LDS read addresses in the first stage; the second lies at the XOR of kWideStage
    static_assert((kWideStage & (kWideStage - 1)) == 0, "stages are told apart by one address bit");
    uint32_t pat[2], qat[2];                       // by slice of 32
    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem);
    const uint32_t in_row = (uint32_t)((g ^ ((l16 >> 1) & 7)) * 16);
#pragma unroll
    for (int ks = 0; ks < 2; ks++) {
        pat[ks] = smem_at + (uint32_t)((wp * 64 + l16) * 128) + (in_row ^ (64u * ks));
        qat[ks] = smem_at + (uint32_t)(2 * kWideHalf + (wq * 32 + l16) * 128) + (in_row ^ (64u * ks));
    }
    f32x4 acc[2][2][4][2];                         // [half of P][half of Q][block of columns][block of rows]
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int a = 0; a < 4; a++)
#pragma unroll
                for (int c = 0; c < 2; c++) acc[i][j][a][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    x8 P[4][2], Q0[2][2], Q1[2][2], Q0next[2][2];  // [block][slice]
    auto read_p = [&](int hf) {
#pragma unroll
        for (int ks = 0; ks < 2; ks++)
#pragma unroll
            for (int a = 0; a < 4; a++) P[a][ks] = __builtin_bit_cast(x8, lds_read_b128(pat[ks] + (uint32_t)(hf * kWideHalf + a * 2048)));
    };
    auto read_q = [&](x8 (&Q)[2][2], int hf) {
#pragma unroll
        for (int ks = 0; ks < 2; ks++)
#pragma unroll
            for (int c = 0; c < 2; c++) Q[c][ks] = __builtin_bit_cast(x8, lds_read_b128(qat[ks] + (uint32_t)(hf * kWideHalf + c * 2048)));
    };
    auto other_stage = [&](uint32_t (&at)[2]) {
        at[0] ^= kWideStage;
        at[1] ^= kWideStage;
    };
    auto turn = [&]() {                            // the end of a slot
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto ready = [&]() {                           // the slot's LDS reads are complete, the next slot's operands have landed
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
        turn();
    };
    auto multiply = [&](f32x4 (&C)[4][2], const x8 (&Q)[2][2]) {
#pragma unroll
        for (int ks = 0; ks < 2; ks++)
#pragma unroll
            for (int a = 0; a < 4; a++)
#pragma unroll
                for (int c = 0; c < 2; c++) product_in_place<T>(C[a][c], P[a][ks], Q[c][ks]);
    };
    request(true, 0, 0);
    request(false, 0, 0);
    request(true, 1, 0);
    request(true, 0, 1);
    request(false, 1, 0);
    request(false, 0, 1);
    request(true, 1, 1);
    ready();                                       // Q0, P0 and Q1 of the first step
    read_q(Q0, 0);
    lds_accesses_then_barrier();                   // read by every wave before the first step requests Q0 again
    if (wp == 1) turn();                           // waves 4-7 run one slot behind from here
#pragma unroll 1
    for (int t = 0; t < steps; t++) {
        read_p(0);
        read_q(Q1, 1);
        request(true, 0, t + 2);
        request(false, 1, t + 1);
        ready();
        __builtin_amdgcn_s_setprio(1);
        multiply(acc[0][0], Q0);
        multiply(acc[0][1], Q1);
        __builtin_amdgcn_s_setprio(0);
        turn();
        read_p(1);
        other_stage(pat);
        other_stage(qat);
        read_q(Q0next, 0);
        request(false, 0, t + 2);
        request(true, 1, t + 2);
        ready();
        __builtin_amdgcn_s_setprio(1);
        multiply(acc[1][1], Q1);
        multiply(acc[1][0], Q0);
        __builtin_amdgcn_s_setprio(0);
        if (t + 1 == steps) finish_products();     // in the loop: behind it the compiler may move accumulators at once
        turn();
#pragma unroll
        for (int ks = 0; ks < 2; ks++)
#pragma unroll
            for (int c = 0; c < 2; c++) Q0[c][ks] = Q0next[c][ks];
    }
    if (wp == 0) turn();
    Residual<4, 2> residual[2];                    // of this quadrant and the next
    auto column = [&](int n) { return p0 + n % 2 * 128 + wp * 64; };
    auto row = [&](int n) { return q0 + n / 2 * 128 + wq * 32; };
    load_residual(residual[0], p, column(0), row(0), g, l16);
    wait_all_memory();                             // the transfers past the end have landed before the wave may end
    with_activation(p.act, [&](auto form) {
#pragma unroll
        for (int n = 0; n < 4; n++) {
            if (n < 3) load_residual(residual[(n + 1) % 2], p, column(n + 1), row(n + 1), g, l16);
            asm volatile("" ::: "memory");         // one quadrant behind the other: beside the accumulators there is no room for more
            store_blocks<T, decltype(form)::value, 4, 2>(p, acc[n % 2][n / 2], residual[n % 2], column(n), row(n), g, l16);
            asm volatile("" ::: "memory");
        }
    });
}

// Tiles of 16 CB columns x 8 NX rows, whose contraction the waves of a workgroup divide, in steps of 64 dealt out in turn.  Each wave has a
// ring of its own, so none waits for another before their sums meet in LDS.
//
// Bound: memory, the weights read once.  They pass through LDS because a transfer then fetches whole lines of 128 bytes (eight
// rows); straight to registers in the product's layout a load fetches 64 bytes of sixteen rows, and a CU got half the rate.  2 rows, 5120
// -> 30 720: 52.6 us, 6.0 TB/s.
template <class T, int CB, int NX, int STAGES>
__global__ __launch_bounds__(512) void linear_patch_kernel(LinearParams p) {
    typedef typename T::x8 x8;
    constexpr int QB = (NX + 1) / 2, NT = 2 * CB + NX, STAGE = NT * 1024;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, l16 = lane & 15;
    int tp, tq;
    if (!linear_tile(p.tiles_p, p.tiles_q, &tp, &tq)) return;
    const int col0 = tp * 16 * CB, row0 = tq * 8 * NX;
    const i32x4 wbuf = operand_rows(p.w, p.D, col0, min(16 * CB, p.F - col0), p.D);
    const i32x4 xbuf = operand_rows(p.x, p.ldx, row0, min(8 * NX, p.N - row0), p.D);
    const int all_chunks = p.D / 8, steps = ((p.D + 63) / 64 - w + waves - 1) / waves;   // the wave's: w, w + waves, ...
    uint32_t off[NT];
    int chunk[NT];
#pragma unroll
    for (int n = 0; n < NT; n++) {
        const int row = (n < 2 * CB ? n : n - 2 * CB) * 8 + (lane >> 3);
        chunk[n] = (lane & 7) ^ ((row >> 1) & 7);
        off[n] = (uint32_t)row * (uint32_t)((n < 2 * CB ? p.D : p.ldx) * 2) + chunk[n] * 16u;
    }
    const uint32_t lds0 = lds_address(smem) + (uint32_t)(w * STAGES * STAGE);
    auto request = [&](int t) {
        const int step = t * waves + w;
#pragma unroll
        for (int n = 0; n < NT; n++)
            load_rows_to_lds_16B(n < 2 * CB ? wbuf : xbuf, step * 8 + chunk[n] < all_chunks ? off[n] : kNowhere, (uint32_t)step * 128u,
                                 lds0 + (uint32_t)(t % STAGES * STAGE + n * 1024));
    };
    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem) + (uint32_t)(w * STAGES * STAGE + l16 * 128);
    const uint32_t in_row = (uint32_t)((g ^ ((l16 >> 1) & 7)) * 16);
    f32x4 acc[CB][QB] = {};
    for (int t = 0; t < min(STAGES, steps); t++) request(t);
    for (int t = 0; t < steps; t++) {
        if (t + STAGES <= steps) wait_vmem_at_most<(STAGES - 1) * NT>();
        else if (t + 2 == steps && STAGES > 2) wait_vmem_at_most<NT>();
        else wait_vmem_at_most<0>();
        asm volatile("" ::: "memory");
        const uint32_t stage = (uint32_t)(t % STAGES * STAGE);
        x8 W[CB][2], X[QB][2];
#pragma unroll
        for (int ks = 0; ks < 2; ks++) {
#pragma unroll
            for (int a = 0; a < CB; a++) W[a][ks] = __builtin_bit_cast(x8, lds_read_b128(smem_at + stage + (in_row ^ (64u * ks)) + a * 2048));
#pragma unroll
            for (int c = 0; c < QB; c++) X[c][ks] = __builtin_bit_cast(x8, lds_read_b128(smem_at + stage + (in_row ^ (64u * ks)) + (CB + c) * 2048));
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read: the stage is free
        if (t + STAGES < steps) request(t + STAGES);
#pragma unroll
        for (int ks = 0; ks < 2; ks++)
#pragma unroll
            for (int a = 0; a < CB; a++)
#pragma unroll
                for (int c = 0; c < QB; c++) acc[a][c] = T::product(W[a][ks], X[c][ks], acc[a][c]);
    }
    lds_accesses_then_barrier();                             // every wave is done with its stages
    f32x4* sums = reinterpret_cast<f32x4*>(smem);
#pragma unroll
    for (int a = 0; a < CB; a++)
#pragma unroll
        for (int c = 0; c < QB; c++) sums[((w * CB + a) * QB + c) * 64 + lane] = acc[a][c];
    lds_accesses_then_barrier();
    // a wave takes a block of 16 rows at a time, in the order of the waves' sums
    for (int c = w; c < QB; c += waves) {
        f32x4 total[CB][1] = {};
        for (int v = 0; v < waves; v++)
#pragma unroll
            for (int a = 0; a < CB; a++) total[a][0] += sums[((v * CB + a) * QB + c) * 64 + lane];
        linear_store<T, CB, 1>(p, total, col0, row0 + c * 16, g, l16);
    }
}

static uint32_t grid_of(LinearParams& p, int columns, int rows) {
    p.tiles_p = (p.F + columns - 1) / columns;
    p.tiles_q = (int)(((int64_t)p.N + rows - 1) / rows);
    return (uint32_t)(((int64_t)p.tiles_p * p.tiles_q + 7) / 8 * 8);
}

template <class T, int PB, int QB, int STAGES, int TEAMS>
static int32_t launch_ring(LinearParams p, hipStream_t stream) {
    constexpr int LDS = std::max(STAGES * 32 * (PB + QB) * 128, TEAMS == 1 ? 0 : 4096 * PB * QB) * TEAMS;
    const auto kernel = linear_ring_kernel<T, PB, QB, STAGES, TEAMS>;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    kernel<<<grid_of(p, 32 * PB, 32 * QB), 256 * TEAMS, LDS, stream>>>(p);
    return launch_status();
}

template <class T, int PN, int QN, int STAGES>
static int32_t launch_block(LinearParams p, hipStream_t stream) {
    constexpr int LDS = STAGES * (PN + QN) * 64 * 128;
    const auto kernel = linear_block_kernel<T, PN, QN, STAGES>;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    kernel<<<grid_of(p, 64 * PN, 64 * QN), 256, LDS, stream>>>(p);
    return launch_status();
}

template <class T, bool CUT>
static int32_t launch_wide(LinearParams p, hipStream_t stream) {
    const auto kernel = linear_wide_kernel<T, CUT>;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * kWideStage) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    kernel<<<grid_of(p, 256, 256), 512, 2 * kWideStage, stream>>>(p);
    return launch_status();
}

template <class T, int CB, int NX, int STAGES>
static int32_t launch_patch(LinearParams p, int waves, hipStream_t stream) {
    const int lds = (waves * STAGES * (2 * CB + NX) + NX % 2) * 1024;   // (the sums take less; an odd number of rows is read with what lies behind)
    const auto kernel = linear_patch_kernel<T, CB, NX, STAGES>;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    kernel<<<grid_of(p, 16 * CB, 8 * NX), 64 * waves, lds, stream>>>(p);
    return launch_status();
}

// The forms of tiles.  A launch is priced in us as rounds of as many tiles as the CUs hold: each round has its start and end, and
// for every contraction step what it takes alone and what the tiles beside it add; the last, partly filled round counts by its
// share.  Fitted to 5901 random sizes, 17 to 30 000 rows, contractions of 256 to 8192, 256 to 30 720 columns: the form taken is 1.005
// times the quickest's time in the mean, 1.25 at most; of 1019 others 1.004 and 1.18.  The small forms whose
// waves divide the contraction are for few tiles: 190 rows, 4992 -> 520: 8.3 us by 16 x 32, 16.2 by the quickest other; 4032 -> 464
// with 21 rows 4.7 and 12.9; 236 rows, 5440 -> 3480 29.4 and 20.4.
enum Form { kSmall, kSmallTeams, kMiddleTeams, kTwoPerCu, kBlock, kTallBlock, kWide, kPatch16, kPatch16x32, kPatch32, kPatch64x32, kForms, kFewRows = kForms };
struct FormPrice {
    int columns, rows, per_round, parts;                  // parts: of the contraction, a wave's each
    float round, step, beside;
};
static const FormPrice kFormPrices[kForms] = {{64, 64, 512, 1, 1.65f, 0.24f, 0.20f},  {64, 64, 256, 1, 2.78f, 0.18f, 0.09f},  {64, 128, 256, 1, 2.4f, 0.26f, 0.075f},
                                              {128, 128, 512, 1, 2.47f, 0.56f, 0.44f}, {128, 128, 256, 1, 2.62f, 0.36f, 0.20f}, {128, 192, 256, 1, 3.6f, 0.51f, 0.31f},
                                              {256, 256, 256, 1, 7.15f, 1.02f, 0.42f}, {16, 16, 256, 8, 2.05f, 0.385f, 0.0f},  {16, 32, 256, 8, 1.98f, 0.50f, 0.057f},
                                              {32, 32, 256, 4, 2.3f, 0.246f, 0.07f},   {64, 32, 256, 4, 3.44f, 0.364f, 0.20f}};
constexpr int64_t kMostTiles = 1 << 22;                   // a launch has fewer than 2^32 threads
static double price_of(Form form, int64_t N, int64_t D, int64_t F) {
    const FormPrice& f = kFormPrices[form];
    const int64_t tiles = (N + f.rows - 1) / f.rows * ((F + f.columns - 1) / f.columns), steps = ((D + 63) / 64 + f.parts - 1) / f.parts;
    const int64_t whole = tiles / f.per_round, rest = tiles % f.per_round;
    if (tiles >= kMostTiles) return HUGE_VAL;
    return whole * (f.round + steps * (double)(f.step + f.beside)) + (rest ? f.round + steps * (f.step + f.beside * (double)rest / f.per_round) : 0.0);
}

// Up to 16 rows there is nothing to choose: a patch of all rows reads the weights once, at the memory's rate (4096 x 4096, one row:
// 7.4 us, tiles 13.5).
static Form linear_form(int N, int D, int F) {
    if (N <= 16 && F / 16 < kMostTiles) return kFewRows;
    Form best = kSmall;
    double least = price_of(best, N, D, F);
    for (int f = 1; f < kForms; f++) {
        const double price = price_of((Form)f, N, D, F);
        if (price < least) {
            best = (Form)f;
            least = price;
        }
    }
    return best;
}

template <class T>
static int32_t linear_launch(const LinearParams& p, hipStream_t stream) {
    const Form form = linear_form(p.N, p.D, p.F);
    if (form == kFewRows) {
        // 16 columns to a workgroup while those find a CU each with few to spare (10 880 columns: 15.6 us, by 32 19.4; 15 360: 27.7 and
        // 27.4, with 16 rows 35 and 29.5); more waves where there are fewer workgroups
        const int steps = (p.D + 63) / 64;
        const bool narrow = p.F <= 12288;
        const int waves = p.F <= 4096 && steps >= 16 ? 8 : steps >= 32 ? 4 : 2;
        if (p.N <= 8) return narrow ? launch_patch<T, 1, 1, 4>(p, waves, stream) : launch_patch<T, 2, 1, 3>(p, waves, stream);
        return narrow ? launch_patch<T, 1, 2, 4>(p, waves, stream) : launch_patch<T, 2, 2, 3>(p, waves, stream);
    }
    if (price_of(form, p.N, p.D, p.F) == HUGE_VAL) return CHIPMUNK_ERR_SHAPE;
    switch (form) {
        case kSmall: return launch_ring<T, 2, 2, 4, 1>(p, stream);
        case kSmallTeams: return launch_ring<T, 2, 2, 4, 2>(p, stream);
        case kMiddleTeams: return launch_ring<T, 2, 4, 3, 2>(p, stream);
        case kTwoPerCu: return launch_ring<T, 4, 4, 2, 1>(p, stream);
        case kBlock: return launch_block<T, 2, 2, 4>(p, stream);
        case kTallBlock: return launch_block<T, 2, 3, 4>(p, stream);
        case kPatch16: return launch_patch<T, 1, 2, 4>(p, 8, stream);
        case kPatch16x32: return launch_patch<T, 1, 4, 3>(p, 8, stream);
        case kPatch32: return launch_patch<T, 2, 4, 3>(p, 4, stream);
        case kPatch64x32: return launch_patch<T, 4, 4, 3>(p, 4, stream);
        default: return p.D % 64 ? launch_wide<T, true>(p, stream) : launch_wide<T, false>(p, stream);
    }
}

}  // namespace chipmunk

using namespace chipmunk;

// The form that a call takes, for the tests.
extern "C" int chipmunk_internal_linear_form(int N, int D, int F) { return linear_form(N, D, F); }

extern "C" int32_t chipmunk_linear(const uint16_t* x, int64_t ldx, const uint16_t* w, const uint16_t* bias, const uint16_t* residual, int64_t ldr,
                                   uint16_t* out, int64_t ldo, int N, int D, int F, int act, int dtype, void* stream) {
    if (!x || !w || !out) return CHIPMUNK_ERR_NULL;
    constexpr int64_t kMostStride = 1 << 22;
    if (N == 1) {                                             // of one row alone a stride means nothing
        ldx = D;
        ldo = ldr = F;
    }
    if (N <= 0 || D <= 0 || F <= 0 || D >= 1 << 20) return CHIPMUNK_ERR_SHAPE;
    if (ldx < D || ldo < F || (residual && ldr < F) || ldx >= kMostStride || ldo >= kMostStride || (residual && ldr >= kMostStride)) return CHIPMUNK_ERR_SHAPE;
    if (D % 8 != 0 || F % 8 != 0 || act < CHIPMUNK_ACT_GELU_ERF || act > CHIPMUNK_ACT_SILU || (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16))
        return CHIPMUNK_ERR_UNSUPPORTED;
    if (!aligned16(x) || !aligned16(w) || !aligned16(bias) || !aligned16(residual) || !aligned16(out) || (ldx | ldo | (residual ? ldr : 0)) % 8 != 0)
        return CHIPMUNK_ERR_ALIGN;
    const bool whole_lines = ldo % 64 == 0 && (reinterpret_cast<uintptr_t>(out) & 127) == 0;
    const int past = !whole_lines ? kKept : (int64_t)N * F * 2 > kLinearLastLevel ? kPastLastLevel : kThrough;
    const LinearParams p{x, w, bias, residual, out, ldx, ldr, ldo, N, D, F, act, past, 0, 0};
    return dtype == CHIPMUNK_DTYPE_BF16 ? linear_launch<Bf16>(p, static_cast<hipStream_t>(stream)) : linear_launch<Fp16>(p, static_cast<hipStream_t>(stream));
}
