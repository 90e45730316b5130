// Linear layers: out = act(x w^T + bias) + residual, x [N, D], w [F, D], out [N, F].
//
// The product is formed as w x^T, so that a lane holds consecutive output columns of one row (P: rows of w = output columns, Q:
// rows of x = output rows), and everything behind it happens on the accumulators: bias, activation and residual in 32 bits,
// one rounding.
#include "element.h"

#include <algorithm>
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
    int tiles_p, tiles_q;
};

template <int ACT>
__device__ __forceinline__ float activation(float y) {
    if constexpr (ACT == CHIPMUNK_ACT_GELU_ERF) return 0.5f * y * (1.f + erff(y * 0.70710678118654752f));
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

// Asynchronous 16-byte load to LDS through a buffer, with a wave-uniform part of the offset.
__device__ __forceinline__ void load_rows_to_lds_16B(i32x4 buffer, uint32_t byte_offset, uint32_t uniform_offset, uint32_t lds_wave_base) {
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds_wave_base), "v"(byte_offset), "s"(buffer), "s"(uniform_offset)
                 : "memory");
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

// Results of a wave: PB x QB blocks of 16 columns x 16 rows from (col0, row0) on.
template <class T, int PB, int QB>
__device__ __forceinline__ void linear_store(const LinearParams& p, const f32x4 (&acc)[PB][QB], int col0, int row0, int g, int l16) {
    static_assert(PB % 2 == 0, "blocks of columns go in pairs");
    with_activation(p.act, [&](auto form) {
        constexpr int ACT = decltype(form)::value;
#pragma unroll
        for (int pair = 0; pair < PB / 2; pair++) {
            const int col = col0 + pair * 32;
            u32x2 bias[2] = {u32x2{0, 0}, u32x2{0, 0}};
            if (p.bias) {
#pragma unroll
                for (int i = 0; i < 2; i++) bias[i] = *reinterpret_cast<const u32x2*>(p.bias + min(col + i * 16 + 4 * g, p.F - 4));
            }
            const int at = col + columns_of_lane(g);
#pragma unroll
            for (int c = 0; c < QB; c++) {
                const int row = row0 + c * 16 + l16;
                const bool there = row < p.N && at < p.F;
                u32x2 old[2] = {u32x2{0, 0}, u32x2{0, 0}};
                if (p.residual) {
                    u32x4 r = {0, 0, 0, 0};
                    if (there) r = *reinterpret_cast<const u32x4*>(p.residual + (int64_t)row * p.ldr + at);
                    from_columns(r, old);
                }
                u32x2 result[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const f32x4 v = acc[2 * pair + i][c];
                    result[i] = u32x2{T::pack(activation<ACT>(v[0] + T::low(bias[i][0])) + T::low(old[i][0]), activation<ACT>(v[1] + T::high(bias[i][0])) + T::high(old[i][0])),
                                      T::pack(activation<ACT>(v[2] + T::low(bias[i][1])) + T::low(old[i][1]), activation<ACT>(v[3] + T::high(bias[i][1])) + T::high(old[i][1]))};
                }
                const u32x4 columns = to_columns(result[0], result[1]);
                if (there) *reinterpret_cast<u32x4*>(p.out + (int64_t)row * p.ldo + at) = columns;
            }
        }
    });
}

// Tiles of 32 PB columns x 32 QB rows, four waves of half of either.  The contraction goes in steps of 64 through a ring of
// STAGES stages in LDS; the operands of the step behind the one that is multiplied are in registers already, so a stage is free
// again as soon as it has been read.
template <class T, int PB, int QB, int STAGES>
__global__ __launch_bounds__(256, 2) void linear_ring_kernel(LinearParams p) {
    constexpr int BP = 32 * PB, BQ = 32 * QB, STAGE = (BP + BQ) * 128;
    constexpr int NP = BP / 32, NQ = BQ / 32;            // transfers of a wave per step: eight rows of 128 bytes each
    constexpr int NT = NP + NQ;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wp = w >> 1, wq = w & 1, g = lane >> 4, l16 = lane & 15;
    int tp, tq;
    if (!linear_tile(p.tiles_p, p.tiles_q, &tp, &tq)) return;
    const int p0 = tp * BP, q0 = tq * BQ;
    const i32x4 wbuf = operand_rows(p.w, p.D, p0, min(BP, p.F - p0), p.D);
    const i32x4 xbuf = operand_rows(p.x, p.ldx, q0, min(BQ, p.N - q0), p.D);

    // 16-byte chunks XOR-swizzled by the row
    uint32_t woff[NP], xoff[NQ];
    int chunk_w[NP], chunk_x[NQ];
#pragma unroll
    for (int n = 0; n < NP; n++) {
        const int row = (n * 4 + w) * 8 + (lane >> 3);
        chunk_w[n] = (lane & 7) ^ ((row >> 1) & 7);
        woff[n] = (uint32_t)row * (uint32_t)(p.D * 2) + chunk_w[n] * 16u;
    }
#pragma unroll
    for (int n = 0; n < NQ; n++) {
        const int row = (n * 4 + w) * 8 + (lane >> 3);
        chunk_x[n] = (lane & 7) ^ ((row >> 1) & 7);
        xoff[n] = (uint32_t)row * (uint32_t)(p.ldx * 2) + chunk_x[n] * 16u;
    }
    const int steps = (p.D + 63) / 64, rest = p.D % 64 / 8;   // chunks of the last step, 0: all eight
    const uint32_t lds0 = lds_address(smem);
    auto request = [&](int t) {
        const uint32_t stage = lds0 + (uint32_t)(t % STAGES * STAGE), from = (uint32_t)t * 128u;
        const bool cut = rest != 0 && t == steps - 1;
#pragma unroll
        for (int n = 0; n < NP; n++) load_rows_to_lds_16B(wbuf, cut && chunk_w[n] >= rest ? kNowhere : woff[n], from, stage + (n * 4 + w) * 1024);
#pragma unroll
        for (int n = 0; n < NQ; n++)
            load_rows_to_lds_16B(xbuf, cut && chunk_x[n] >= rest ? kNowhere : xoff[n], from, stage + BP * 128 + (n * 4 + w) * 1024);
    };
    auto wait_steps = [&](int left) {   // at most `left` steps' transfers outstanding
        if (left >= 3) wait_vmem_at_most<3 * NT>();
        else if (left == 2) wait_vmem_at_most<2 * NT>();
        else if (left == 1) wait_vmem_at_most<NT>();
        else wait_vmem_at_most<0>();
    };
    static_assert(STAGES <= 4 && 3 * NT < 64, "the cases above");

    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem);
    const uint32_t in_row = (uint32_t)((g ^ ((l16 >> 1) & 7)) * 16);
    uint32_t pat[2], qat[2];                             // by slice of 32; opaque, so that what is added stays in the reads' offset field
#pragma unroll
    for (int ks = 0; ks < 2; ks++) {
        pat[ks] = smem_at + (uint32_t)((wp * PB * 16 + l16) * 128) + (in_row ^ (64u * ks));
        qat[ks] = smem_at + (uint32_t)(BP * 128 + (wq * QB * 16 + l16) * 128) + (in_row ^ (64u * ks));
        asm volatile("" : "+v"(pat[ks]), "+v"(qat[ks]));
    }
    typedef typename T::x8 x8;
    struct Operands {
        x8 P[PB][2], Q[QB][2];
    } even, odd;
    auto read = [&](Operands& op, int t) {
        const uint32_t stage = (uint32_t)(t % STAGES * STAGE);
#pragma unroll
        for (int ks = 0; ks < 2; ks++) {
#pragma unroll
            for (int a = 0; a < PB; a++) op.P[a][ks] = __builtin_bit_cast(x8, lds_read_b128(pat[ks] + stage + a * 2048));
#pragma unroll
            for (int c = 0; c < QB; c++) op.Q[c][ks] = __builtin_bit_cast(x8, lds_read_b128(qat[ks] + stage + c * 2048));
        }
    };
    f32x4 acc[PB][QB] = {};
    for (int t = 0; t < min(STAGES, steps); t++) request(t);
    wait_steps(min(STAGES, steps) - 1);
    lds_accesses_then_barrier();
    read(even, 0);
    auto step = [&](int t, Operands& now, Operands& next) {
        if (t + STAGES <= steps) wait_vmem_at_most<(STAGES - 2) * NT>();   // step t + 1 has landed
        else wait_steps(max(0, steps - 2 - t));
        lds_accesses_then_barrier();                     // for every wave; and every wave holds its operands of step t
        if (t + 1 < steps) read(next, t + 1);
        __builtin_amdgcn_sched_barrier(0);               // the reads lead: they land behind this step's products
        if (t + STAGES < steps) request(t + STAGES);
#pragma unroll
        for (int ks = 0; ks < 2; ks++)
#pragma unroll
            for (int a = 0; a < PB; a++)
#pragma unroll
                for (int c = 0; c < QB; c++) acc[a][c] = T::product(now.P[a][ks], now.Q[c][ks], acc[a][c]);
    };
#pragma unroll 1
    for (int t = 0; t < steps; t += 2) {
        step(t, even, odd);
        if (t + 1 < steps) step(t + 1, odd, even);
    }
    linear_store<T, PB, QB>(p, acc, p0 + wp * PB * 16, q0 + wq * QB * 16, g, l16);
}

template <class T>
static int32_t linear_launch(LinearParams p, hipStream_t stream) {
    constexpr int STAGES = 4, STAGE = 128 * 128;
    p.tiles_p = (int)(((int64_t)p.F + 63) / 64);
    p.tiles_q = (int)(((int64_t)p.N + 63) / 64);
    const int64_t tiles = (int64_t)p.tiles_p * p.tiles_q;
    if (tiles >= (INT64_C(1) << 24) - 8) return CHIPMUNK_ERR_SHAPE;   // a launch has fewer than 2^32 threads
    linear_ring_kernel<T, 2, 2, STAGES><<<(uint32_t)((tiles + 7) / 8 * 8), 256, STAGES * STAGE, stream>>>(p);
    return launch_status();
}

}  // namespace chipmunk

using namespace chipmunk;

extern "C" int32_t chipmunk_linear(const uint16_t* x, int64_t ldx, const uint16_t* w, const uint16_t* bias, const uint16_t* residual, int64_t ldr,
                                   uint16_t* out, int64_t ldo, int N, int D, int F, int act, int dtype, void* stream) {
    if (!x || !w || !out) return CHIPMUNK_ERR_NULL;
    constexpr int64_t kMostStride = 1 << 22;
    if (N <= 0 || D <= 0 || F <= 0 || D >= 1 << 20) return CHIPMUNK_ERR_SHAPE;
    if (ldx < D || ldo < F || (residual && ldr < F) || ldx >= kMostStride || ldo >= kMostStride || (residual && ldr >= kMostStride)) return CHIPMUNK_ERR_SHAPE;
    if (D % 8 != 0 || F % 8 != 0 || act < CHIPMUNK_ACT_GELU_ERF || act > CHIPMUNK_ACT_SILU || (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16))
        return CHIPMUNK_ERR_UNSUPPORTED;
    if (!aligned16(x) || !aligned16(w) || !aligned16(bias) || !aligned16(residual) || !aligned16(out) || (ldx | ldo | (residual ? ldr : 0)) % 8 != 0)
        return CHIPMUNK_ERR_ALIGN;
    const LinearParams p{x, w, bias, residual, out, ldx, ldr, ldo, N, D, F, act, 0, 0};
    return dtype == CHIPMUNK_DTYPE_BF16 ? linear_launch<Bf16>(p, static_cast<hipStream_t>(stream)) : linear_launch<Fp16>(p, static_cast<hipStream_t>(stream));
}
