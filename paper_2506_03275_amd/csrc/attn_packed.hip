// Attention over packed sequences of different lengths: causal or not, heads grouped over the keys' heads.
//
// attn_packed_rows_kernel: one workgroup of four waves owns 64 NQB consecutive queries of one sequence and head and walks the
// sequence's keys in steps of two tiles of 32.  K and V tiles go from memory to LDS by asynchronous 16-byte loads, double
// buffered by step; scores are formed transposed, S^T = K Q^T, so that a lane holds, for one query (lane % 16), four keys of each
// block of 16, which are the contraction entries that it supplies to O^T += V^T P^T: probabilities go from the softmax into the
// second product without leaving registers.  One pass with a running maximum and sum.
// Bound: the matrix cores and, beside them, the softmax's vector instructions, two waves to a SIMD: 40 heads x 128 over 12 000 and 9041
// tokens 3.80 ms (1.22 PFLOP/s, matrix pipes 71 % busy at 1.86 GHz); causal, 32 heads over 8, 574 to 8190 tokens 0.64 ms (1.18, 62 %).  With 192
// rows a wave reads a K and V tile from LDS once for three blocks of 16; fewer rows give more workgroups, which counts where there are
// few (the prices below).
#include "element.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace chipmunk {

struct PackedParams {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    uint16_t* out;
    const int32_t* cu_q;
    const int32_t* cu_k;
    const int32_t* k_len;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, out_token, out_head;
    int S, Tq, Tk, Hq, Hk, G;
    int max_q, max_k, causal;
    int tiles;     // of one head: as many as there can be
    int part_keys, parts;   // few queries: keys that a workgroup walks, and how many such parts the longest sequence can have
    int few_rows;  // rows of a key head: max_q * G
    float* partial;         // [S][Hk][parts][few_rows][E] sums, then [S][Hk][parts][few_rows][2]: reference (units of <q, k>), sum of weights
    float sl2;     // softmax_scale * log2(e)
};

constexpr int kTile = 32;             // keys per LDS tile = one step of the running softmax
constexpr int kStepTiles = 2;         // tiles between two workgroup barriers
constexpr int kStepKeys = kTile * kStepTiles;
constexpr float kSlack = 8.f;         // the reference may lag the row's maximum by 2^8 before a rescale

// XOR swizzle of the 16-byte chunk position inside a row of the LDS tile
template <int E>
__device__ __forceinline__ int tile_swizzle(int row) {
    return E == 128 ? swizzle_rows16(row) : (row >> 1) & 7;
}

// A sequence's rows, clamped into the tensors.
struct Rows {
    int first, count;
};
__device__ __forceinline__ Rows queries_of(const PackedParams& p, int s) {
    const int first = min(max(p.cu_q[s], 0), p.Tq), end = min(max(p.cu_q[s + 1], 0), p.Tq);
    return Rows{first, min(max(end - first, 0), p.max_q)};
}
__device__ __forceinline__ Rows keys_of(const PackedParams& p, int s) {
    const int first = min(max(p.cu_k[s], 0), p.Tk);
    const int count = p.k_len ? p.k_len[s] : min(max(p.cu_k[s + 1], 0), p.Tk) - first;
    return Rows{first, min(min(max(count, 0), p.max_k), p.Tk - first)};
}

// Tile `tile` of all sequences' tiles of ROWS queries, the last rows of a sequence first (with a causal mask they have the most
// keys).  Every wave works it out by itself.  False: there are fewer tiles.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const PackedParams& p, int tile, int lane, int* sequence, int* in_sequence) {
    if (p.max_q <= ROWS) {            // a tile per sequence
        *sequence = tile;
        *in_sequence = 0;
        return true;
    }
    for (int s0 = 0; s0 < p.S; s0 += 64) {
        const int s = s0 + lane;
        const int mine = s < p.S ? (queries_of(p, s).count + ROWS - 1) / ROWS : 0;
        int upto = mine;              // tiles of this group of sequences up to the lane's
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int below = __shfl_up(upto, d);
            if (lane >= d) upto += below;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (tile < all) {
            const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > tile));
            *sequence = s0 + at;
            *in_sequence = __builtin_amdgcn_readlane(upto, at) - 1 - tile;
            return true;
        }
        tile -= all;
    }
    return false;
}

// The keys of a tile that a query does not see.  `first`: the number of the lane's first key, limit: the first key that its
// query does not see.
template <int NQB>
__device__ __forceinline__ void hide_keys(f32x4 (&S)[2][NQB], int first, const int (&limit)[NQB]) {
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        const int left = limit[qb] - first;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                S[u][qb][r] = u * 16 + r < left ? S[u][qb][r] : -INFINITY;
                asm volatile("" : "+v"(S[u][qb][r]));   // one behind the other: all comparisons' masks at a time do not fit the scalar registers
            }
    }
}

template <class T, int E, int NQB>
struct RowState {
    f32x4 O[E / 16][NQB];
    f32x4 L[NQB];       // sum of the probabilities, by the product with a row of ones: of the very values that weight V
    f32x4 negm[NQB];    // minus the reference of the exponentials, in units of <q, k>: starts every score's accumulation
    typename T::x8 Q[E / 32][NQB];
};

// Raises the reference where a row's scores exceed it by more than the slack; as long as a row has no weight at all, the reference
// is set, up or down, to the tile's maximum (if it has one).
template <class T, int E, int NQB>
__device__ __forceinline__ void raise_reference(RowState<T, E, NQB>& st, f32x4 (&S)[2][NQB], float sl2, float slack) {
    float most[NQB];
    bool need = false;
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        const float a = fmaxf(fmaxf(S[0][qb][0], S[0][qb][1]), S[0][qb][2]);
        const float b = fmaxf(fmaxf(a, S[0][qb][3]), S[1][qb][0]);
        const float c = fmaxf(fmaxf(b, S[1][qb][1]), S[1][qb][2]);
        most[qb] = fmaxf(c, S[1][qb][3]);
        need |= most[qb] > slack || st.L[qb][0] == 0.f;
    }
    if (__builtin_amdgcn_ballot_w64(need) != 0) {
#pragma unroll
        for (int qb = 0; qb < NQB; qb++) {
            const float d = rows4_max(most[qb]);
            float up = st.L[qb][0] == 0.f || d > slack ? d : 0.f;   // a row goes by its own scores alone
            if (d == -INFINITY) up = 0.f;                 // every key hidden
            const float alpha = st.L[qb][0] == 0.f ? 1.f : __builtin_amdgcn_exp2f(-up * sl2);
            const float nm = st.negm[qb][0] - up;
            st.negm[qb] = f32x4{nm, nm, nm, nm};
            st.L[qb] *= alpha;
#pragma unroll
            for (int eb = 0; eb < E / 16; eb++) st.O[eb][qb] *= alpha;
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int r = 0; r < 4; r++) S[u][qb][r] -= up;
        }
    }
}

// S^T = K Q^T - reference for one tile.  between(j), j = 0 .. E/16 - 1, is called behind the j-th group of products: the next
// step's transfers are spread over them.
template <class T, int E, int NQB, typename Between>
__device__ __forceinline__ void tile_scores(f32x4 (&S)[2][NQB], const RowState<T, E, NQB>& st, const uint32_t (&kaddr)[E / 32], int tile_off,
                                            Between&& between) {
    typedef typename T::x8 x8;
    constexpr int ROWB = E * 2, NG = E / 16;
    x8 kop[NG];
    kop[0] = __builtin_bit_cast(x8, lds_read_b128(kaddr[0] + tile_off));
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
    for (int j = 0; j < NG; j++) {
        if (j + 1 < NG) {
            kop[j + 1] = __builtin_bit_cast(x8, lds_read_b128(kaddr[(j + 1) / 2] + tile_off + ((j + 1) % 2) * 16 * ROWB));
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
#pragma unroll
        for (int qb = 0; qb < NQB; qb++) S[j % 2][qb] = T::product(kop[j], st.Q[j / 2][qb], j < 2 ? st.negm[qb] : S[j % 2][qb]);
        __builtin_amdgcn_sched_group_barrier(0x008, NQB, 0);
        between(j);
    }
}

// The top bit of either element of a word that is infinite or NaN: one more in the last place of an exponent of all ones carries into it.
// (On the bits: these files are compiled as if NaN did not exist, and a comparison of values is folded accordingly.)
template <class T>
__device__ __forceinline__ uint32_t not_finite(uint32_t word) { return ((word & T::kExponent) + T::kExponentStep) & 0x80008000u; }

// One word of two elements without those that are infinite or NaN; they are noted in `found`.
template <class T>
__device__ __forceinline__ uint32_t finite_elements(uint32_t word, uint32_t& found) {
    const uint32_t tops = not_finite<T>(word);
    found |= tops;
    return word & ~((tops - (tops >> 15)) | tops);
}

// P = exp2(S sl2) rounded to the element type (to 8 or 11 bits, like the values that it weights), its sum, and O^T += V^T P^T.
// A matrix product takes both operands in 16 bits; what is rounded off would be a second product with V, half as many matrix instructions
// again in kernels that these bound.  So each weight is off by half a step at most, in the product and in the sum alike, and a row by
// half a step of sum w |v| + |out| at most: against 64 bits the results of prompts of 574 to 8190 tokens are off by 2.1e-3 of their
// size in bf16 (exact results, rounded: 1.6e-3), of clips of 12 000 and 9041 by 2.9e-4 in fp16 (2.1e-4), root mean squares.
// HIDDEN: some keys are hidden from some of the queries, and a hidden key's zero probability times an infinite or NaN value would
// be a NaN: such values are left out and noted.
template <class T, int E, int NQB, bool HIDDEN>
__device__ __forceinline__ void tile_values(RowState<T, E, NQB>& st, const f32x4 (&S)[2][NQB], const uint32_t (&vaddr)[E / 16], int tile_off, float sl2,
                                            uint32_t& found) {
    typedef typename T::x8 x8;
    typedef __attribute__((ext_vector_type(8))) short short8v;
    constexpr int ROWB = E * 2, NEB = E / 16, AHEAD = 2;
    short4v lo[NEB], hi[NEB];
#pragma unroll
    for (int eb = 0; eb < AHEAD; eb++) {
        lo[eb] = lds_read_tr16_at(vaddr[eb] + tile_off);
        hi[eb] = lds_read_tr16_at(vaddr[eb] + tile_off + 16 * ROWB);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
    x8 pop[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; i++) e[i] = __builtin_amdgcn_exp2f(S[i / 4][qb][i % 4] * sl2);
        pop[qb] = __builtin_bit_cast(x8, u32x4{T::pack(e[0], e[1]), T::pack(e[2], e[3]), T::pack(e[4], e[5]), T::pack(e[6], e[7])});
    }
    const x8 ones = __builtin_bit_cast(x8, u32x4{T::kOnes, T::kOnes, T::kOnes, T::kOnes});
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) st.L[qb] = T::product(ones, pop[qb], st.L[qb]);
    __builtin_amdgcn_sched_group_barrier(0x008, NQB, 0);
#pragma unroll
    for (int eb = 0; eb < NEB; eb++) {
        if (eb + AHEAD < NEB) {
            lo[eb + AHEAD] = lds_read_tr16_at(vaddr[eb + AHEAD] + tile_off);
            hi[eb + AHEAD] = lds_read_tr16_at(vaddr[eb + AHEAD] + tile_off + 16 * ROWB);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        x8 vop = __builtin_bit_cast(x8, (short8v)__builtin_shufflevector(lo[eb], hi[eb], 0, 1, 2, 3, 4, 5, 6, 7));
        if constexpr (HIDDEN) {
            u32x4 words = __builtin_bit_cast(u32x4, vop);
#pragma unroll
            for (int i = 0; i < 4; i++) words[i] = finite_elements<T>(words[i], found);
            vop = __builtin_bit_cast(x8, words);
        }
#pragma unroll
        for (int qb = 0; qb < NQB; qb++) st.O[eb][qb] = T::product(vop, pop[qb], st.O[eb][qb]);
        __builtin_amdgcn_sched_group_barrier(0x008, NQB, 0);
    }
}

// Adds the infinite and NaN values of keys first .. last - 1 to the queries that see them (tile_values leaves them out where
// something is hidden).
template <class T, int E, int NQB>
__device__ __forceinline__ void add_special_values(RowState<T, E, NQB>& st, const uint16_t* vh, int64_t v_token, int first, int last, const int (&limit)[NQB], int g) {
#pragma unroll 1
    for (int key = first; key < last; key++) {
        const uint16_t* from = vh + key * v_token + 4 * g;
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) {
            const u32x2 words = *reinterpret_cast<const u32x2*>(from + eb * 16);
#pragma unroll
            for (int r = 0; r < 4; r++) {
                float value = r % 2 ? T::high(words[r / 2]) : T::low(words[r / 2]);
                const bool special = not_finite<T>(words[r / 2]) & (r % 2 ? 0x80000000u : 0x8000u);
                asm volatile("" : "+v"(value));           // nothing is known of it, not even that it is none of the two
#pragma unroll
                for (int qb = 0; qb < NQB; qb++)
                    if (special && key < limit[qb]) st.O[eb][qb][r] += value;
            }
        }
    }
}

// Tile and head of a workgroup.  Workgroups go to the eight XCDs in turn (id modulo 8), each with an L2 of its own: a key head's
// workgroups stay on as few XCDs as there are heads for, and every XCD gets as many of the long tiles.
__device__ __forceinline__ void tile_and_head(const PackedParams& p, uint32_t id, int* tile, int* head) {
    const uint32_t x = id & 7, slot = id >> 3;
    uint32_t kv, within;                                  // within: tile * G + head of the group
    if (p.Hk % 8 == 0) {
        const uint32_t each = (uint32_t)p.tiles * p.G;
        kv = slot / each * 8 + x;
        within = slot % each;
    } else if (8 % p.Hk == 0) {
        const uint32_t sides = 8 / p.Hk;                  // XCDs of a key head: every so many-th tile is an XCD's
        kv = x % p.Hk;
        const uint32_t t = slot / p.G * sides + x / p.Hk;
        within = t * p.G + slot % p.G;
    } else {
        within = id / p.Hk;
        kv = id % p.Hk;
    }
    *tile = within / p.G;
    *head = kv * p.G + within % p.G;
}

template <class T, int E, int NQB>
__global__ __launch_bounds__(256, 2) void attn_packed_rows_kernel(PackedParams p) {
    typedef typename T::x8 x8;
    constexpr int NWAVES = 4, ROWS = 16 * NQB * NWAVES;
    constexpr int ROWB = E * 2;                           // bytes per K/V row
    constexpr int CH = ROWB / 16, RPI = 64 / CH;          // 16-byte chunks per row; rows covered by one wave-wide load
    constexpr int NI = kTile / (RPI * NWAVES);            // such loads per wave, tile and matrix
    constexpr int TILE = kTile * ROWB, STAGE = 2 * TILE;  // K tile then V tile
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, l16 = lane & 15;

    int tile, head, s, part;
    tile_and_head(p, blockIdx.x, &tile, &head);
    if (tile >= p.tiles || !find_tile<ROWS>(p, tile, lane, &s, &part)) return;
    s = __builtin_amdgcn_readfirstlane(s);
    part = __builtin_amdgcn_readfirstlane(part);
    const Rows qs = queries_of(p, s), ks = keys_of(p, s);
    const int row0 = part * ROWS, rows = min(ROWS, qs.count - row0);
    if (rows <= 0) return;
    const int past = ks.count - qs.count;                 // query i sees the keys up to i + past
    const uint16_t* qh = p.q + head * p.q_head + (int64_t)(qs.first + row0) * p.q_token;
    const uint16_t* kh = p.k + head / p.G * p.k_head + (int64_t)ks.first * p.k_token;
    const uint16_t* vh = p.v + head / p.G * p.v_head + (int64_t)ks.first * p.v_token;
    uint16_t* oh = p.out + head * p.out_head + (int64_t)(qs.first + row0) * p.out_token;

    RowState<T, E, NQB> st;
    int limit[NQB];                                       // the first key that the lane's query does not see
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        st.negm[qb] = st.L[qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) st.O[eb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int row = (w * NQB + qb) * 16 + l16;
        limit[qb] = p.causal ? min(ks.count, row0 + min(row, rows - 1) + 1 + past) : ks.count;   // (rows that are not there: the last one's)
#pragma unroll
        for (int es = 0; es < E / 32; es++) {
            u32x4 val = u32x4{0, 0, 0, 0};
            if (row < rows) val = *reinterpret_cast<const u32x4*>(qh + row * p.q_token + 32 * es + 8 * g);
            st.Q[es][qb] = __builtin_bit_cast(x8, val);
        }
    }
    // keys that the workgroup walks, that all of a wave's rows see, and that any of them sees
    const int keys = p.causal ? max(0, min(ks.count, row0 + rows + past)) : ks.count;
    const int wave_row = w * NQB * 16, wave_rows = min(rows - wave_row, NQB * 16);
    const int seen = wave_rows <= 0 ? 0 : p.causal ? min(ks.count, row0 + wave_row + wave_rows + past) : ks.count;
    const int seen_by_all = p.causal ? min(seen, row0 + wave_row + 1 + past) : seen;
    const float slack = kSlack / p.sl2;

    const int koff = l16 * ROWB + ((g ^ tile_swizzle<E>(l16)) * 16);
    const int vrow = 4 * g + (l16 >> 2);
    const int voff = vrow * ROWB + ((((l16 & 3) >> 1) ^ tile_swizzle<E>(vrow)) * 16) + 8 * (l16 & 1);
    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem);
    uint32_t kaddr[E / 32], vaddr[E / 16];                // opaque, so that what is added stays in the reads' offset field
#pragma unroll
    for (int es = 0; es < E / 32; es++) {
        kaddr[es] = smem_at + (uint32_t)(koff ^ (64 * es));
        asm volatile("" : "+v"(kaddr[es]));
    }
#pragma unroll
    for (int eb = 0; eb < E / 16; eb++) {
        vaddr[eb] = smem_at + (uint32_t)(voff ^ (32 * eb));
        asm volatile("" : "+v"(vaddr[eb]));
    }

    // Load i of a wave fills rows (i * NWAVES + w) * RPI .. of a tile; a lane's offsets into a step's keys stay the same from
    // step to step, the buffer's base moves on (so that a head may be larger than 32-bit offsets reach).
    uint32_t from_k[kStepTiles][NI], from_v[kStepTiles][NI];
#pragma unroll
    for (int n = 0; n < kStepTiles; n++)
#pragma unroll
        for (int i = 0; i < NI; i++) {
            const int row = (i * NWAVES + w) * RPI + lane / CH;
            const uint32_t chunk = (uint32_t)(((lane % CH) ^ tile_swizzle<E>(row)) * 16);
            from_k[n][i] = (uint32_t)(n * kTile + row) * (uint32_t)(p.k_token * 2) + chunk;
            from_v[n][i] = (uint32_t)(n * kTile + row) * (uint32_t)(p.v_token * 2) + chunk;
        }
    const uint32_t lds0 = lds_address(smem) + (uint32_t)w * 1024u;
    i32x4 kbuf, vbuf;                                     // the next step's keys, none behind the sequence's last: those read as zero
    auto next_step = [&](int first) {
        const int left = min(max(ks.count - first, 0), kStepKeys);
        kbuf = raw_buffer_words(kh + first * p.k_token, left > 0 ? (uint32_t)((left - 1) * p.k_token + E) * 2u : 0u);
        vbuf = raw_buffer_words(vh + first * p.v_token, left > 0 ? (uint32_t)((left - 1) * p.v_token + E) * 2u : 0u);
    };
    auto request = [&](int half, int j) {
        const int n = j / (2 * NI), i = (j / 2) % NI;
        const uint32_t to = lds0 + (uint32_t)((half * kStepTiles + n) * STAGE + i * NWAVES * 1024);
        if (j & 1) load_buffer_to_lds_16B(vbuf, from_v[n][i], to + TILE);
        else load_buffer_to_lds_16B(kbuf, from_k[n][i], to);
    };
    static_assert(kStepTiles * NI * 2 == E / 16, "one transfer per group of score products");

    if (keys > 0) {
        wait_all_memory();                                // no wait for the queries inside the loop
        next_step(0);
#pragma unroll
        for (int j = 0; j < E / 16; j++) request(0, j);
    }
    auto arrived = [&](int first) {
        wait_all_memory();
        __syncthreads();                                  // this step's tiles have landed for every wave; the other half is free
        next_step(first + kStepKeys);
    };
    // The steps whose keys all of the wave's rows see, in two copies, whose LDS offsets are constants; then those with hidden keys.
    // Waves may stand in different loops: each step of each is one barrier.
    uint32_t found = 0;
    auto step = [&](auto half_c, int first) {
        constexpr int half = decltype(half_c)::value;
        arrived(first);
#pragma unroll
        for (int n = 0; n < kStepTiles; n++) {
            const int tile_off = (half * kStepTiles + n) * STAGE;
            f32x4 S[2][NQB];
            if (n == 0) tile_scores<T, E, NQB>(S, st, kaddr, tile_off, [&](int j) { request(half ^ 1, j); });
            else tile_scores<T, E, NQB>(S, st, kaddr, tile_off, [](int) {});
            raise_reference<T, E, NQB>(st, S, p.sl2, slack);
            tile_values<T, E, NQB, false>(st, S, vaddr, tile_off + TILE, p.sl2, found);
        }
    };
    int first = 0;
#pragma unroll 1
    while (first + kStepKeys <= seen_by_all) {
        step(std::integral_constant<int, 0>{}, first);
        first += kStepKeys;
        if (first + kStepKeys > seen_by_all) break;
        step(std::integral_constant<int, 1>{}, first);
        first += kStepKeys;
    }
    const int first_hidden = first;
    int half = first / kStepKeys & 1;
    auto move = [&](int bytes) {                          // the addresses to the other half
#pragma unroll
        for (int es = 0; es < E / 32; es++) kaddr[es] += bytes;
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) vaddr[eb] += bytes;
    };
    move(half * kStepTiles * STAGE);
#pragma unroll 1
    for (; first < keys; first += kStepKeys, half ^= 1) {
        arrived(first);
#pragma unroll
        for (int j = 0; j < E / 16; j++) request(half ^ 1, j);
        if (first < seen) {                               // else nothing to see for this wave
#pragma unroll
            for (int n = 0; n < kStepTiles; n++) {
                f32x4 S[2][NQB];
                tile_scores<T, E, NQB>(S, st, kaddr, n * STAGE, [](int) {});
                hide_keys<NQB>(S, first + n * kTile + 4 * g, limit);
                raise_reference<T, E, NQB>(st, S, p.sl2, slack);
                tile_values<T, E, NQB, true>(st, S, vaddr, n * STAGE + TILE, p.sl2, found);
            }
        }
        move(half ? -kStepTiles * STAGE : kStepTiles * STAGE);
    }
    wait_all_memory();                                    // the transfers behind the last step

    // Infinite and NaN values among the steps with hidden keys go to the queries that see them.
    if (__builtin_amdgcn_ballot_w64(found != 0) != 0) add_special_values<T, E, NQB>(st, vh, p.v_token, first_hidden, seen, limit, g);

#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        const int row = (w * NQB + qb) * 16 + l16;
        if (row >= rows) continue;
        const float f = limit[qb] > 0 ? 1.f / st.L[qb][0] : 0.f;   // no key to see: zero
        uint16_t* to = oh + row * p.out_token;
#pragma unroll
        for (int pair = 0; pair < E / 32; pair++) {
            u32x2 r[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const f32x4 o = st.O[2 * pair + i][qb] * f;
                r[i] = u32x2{T::pack(o[0], o[1]), T::pack(o[2], o[3])};
            }
            *reinterpret_cast<u32x4*>(to + pair * 32 + columns_of_lane(g)) = to_columns(r[0], r[1]);
        }
    }
}

// Few queries over many keys: a workgroup owns one key head of one sequence and walks part_keys of its keys for all rows of the head
// (query i, head g of the group: row i * G + g), so the keys and values are read once for the whole group.  Its waves take the tiles of 32 keys in
// turn, each with a K and a V tile of its own in LDS and a reference, sum and accumulator of its own: no wave waits for another before
// they meet at the end.  A longer sequence's parts are joined by attn_packed_join_kernel.
//
// Bound: memory, K and V read once: 16 tokens over 210 551 keys, 32 heads over 8, 167 us (5.1 TB/s) and 6 us of joining.  A K tile is
// requested again as soon as its scores have been formed, a V tile when it has been weighted: of the eight waves on a CU at most one
// is without a request.
template <class T, int E, int NQB>
__global__ __launch_bounds__(256, NQB == 4 ? 1 : 2) void attn_packed_few_kernel(PackedParams p) {
    typedef typename T::x8 x8;
    constexpr int ROWB = E * 2, CH = ROWB / 16, RPI = 64 / CH, NI = kTile / RPI;   // NI: transfers of a tile
    constexpr int TILE = kTile * ROWB;
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, l16 = lane & 15;
    // Workgroups go to the XCDs in turn, and an XCD's to its groups of CUs: a sequence's heads, whose rows lie side by side, to all XCDs; then its
    // parts and rows, the last ones, which may see the most, first; then the next sequence.  (Sequences side by side give every fourth workgroup
    // of an XCD to the longest of four, which one group of CUs then walks: 1179 and three of 201 tokens, 8 heads 28.7 us.)
    int id = (int)(blockIdx.x / p.Hk);
    const int head = (int)blockIdx.x % p.Hk, part = id % p.parts;
    id /= p.parts;
    const int row0 = (p.tiles - 1 - id % p.tiles) * 16 * NQB, s = id / p.tiles;
    const Rows qs = queries_of(p, s), ks = keys_of(p, s);
    const int rows = min(16 * NQB, qs.count * p.G - row0);
    if (rows <= 0) return;
    const int past = ks.count - qs.count;
    // the first keys that the first and the last row do not see
    const int seen_by_all = p.causal ? min(ks.count, row0 / p.G + 1 + past) : ks.count;
    const int seen = p.causal ? min(ks.count, (row0 + rows - 1) / p.G + 1 + past) : ks.count;
    const int start = part * p.part_keys, end = start + min((p.parts == 1 ? seen : ks.count) - start, p.part_keys);   // (no sum passes 31 bits)
    if (start >= end && part > 0) return;                 // (without any key the first part writes zeros)
    const uint16_t* kh = p.k + head * p.k_head + (int64_t)ks.first * p.k_token;
    const uint16_t* vh = p.v + head * p.v_head + (int64_t)ks.first * p.v_token;

    RowState<T, E, NQB> st;
    int limit[NQB];                                       // the first key that the lane's row does not see
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        st.negm[qb] = st.L[qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) st.O[eb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int row = row0 + min(qb * 16 + l16, rows - 1), i = row / p.G;   // (rows that are not there: the last one's limit)
        limit[qb] = p.causal ? min(ks.count, i + 1 + past) : ks.count;
        const uint16_t* from = p.q + (int64_t)(qs.first + i) * p.q_token + (head * p.G + row % p.G) * p.q_head + 8 * g;
#pragma unroll
        for (int es = 0; es < E / 32; es++) {
            u32x4 val = u32x4{0, 0, 0, 0};
            if (qb * 16 + l16 < rows) val = *reinterpret_cast<const u32x4*>(from + 32 * es);
            st.Q[es][qb] = __builtin_bit_cast(x8, val);
        }
    }
    const float slack = kSlack / p.sl2;

    const int koff = l16 * ROWB + ((g ^ tile_swizzle<E>(l16)) * 16);
    const int vrow = 4 * g + (l16 >> 2);
    const int voff = vrow * ROWB + ((((l16 & 3) >> 1) ^ tile_swizzle<E>(vrow)) * 16) + 8 * (l16 & 1);
    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem) + w * 2 * TILE;
    uint32_t kaddr[E / 32], vaddr[E / 16];
#pragma unroll
    for (int es = 0; es < E / 32; es++) kaddr[es] = smem_at + (uint32_t)(koff ^ (64 * es));
#pragma unroll
    for (int eb = 0; eb < E / 16; eb++) vaddr[eb] = smem_at + (uint32_t)(voff ^ (32 * eb));
    uint32_t from_k[NI], from_v[NI];
#pragma unroll
    for (int i = 0; i < NI; i++) {
        const int row = i * RPI + lane / CH;
        const uint32_t chunk = (uint32_t)(((lane % CH) ^ tile_swizzle<E>(row)) * 16);
        from_k[i] = (uint32_t)row * (uint32_t)(p.k_token * 2) + chunk;
        from_v[i] = (uint32_t)row * (uint32_t)(p.v_token * 2) + chunk;
    }
    const uint32_t lds0 = lds_address(smem) + (uint32_t)(w * 2 * TILE);
    // the tile from key `first` on; what lies behind the part's end reads as zero
    auto request = [&](const uint16_t* rows_at, int64_t token, const uint32_t (&from)[NI], int first, uint32_t to) {
        const int left = min(max(end - first, 0), kTile);
        const i32x4 buf = raw_buffer_words(rows_at + first * token, left > 0 ? (uint32_t)((left - 1) * token + E) * 2u : 0u);
#pragma unroll
        for (int i = 0; i < NI; i++) load_buffer_to_lds_16B(buf, from[i], to + i * 1024);
    };
    constexpr int TURN = 4 * kTile;                       // keys from one tile of a wave to its next
    int first = start + w * kTile;
    wait_all_memory();                                    // the queries
    if (first < end) {
        request(kh, p.k_token, from_k, first, lds0);
        request(vh, p.v_token, from_v, first, lds0 + TILE);
    }
    uint32_t found = 0;
    auto tile = [&](auto hidden_c) {
        constexpr bool HIDDEN = decltype(hidden_c)::value;
        f32x4 S[2][NQB];
        wait_vmem_at_most<NI>();                          // K has landed
        asm volatile("" ::: "memory");
        tile_scores<T, E, NQB>(S, st, kaddr, 0, [](int) {});
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // and has been read
        request(kh, p.k_token, from_k, first + TURN, lds0);
        if (HIDDEN) {
            int within[NQB];                              // the part's end hides the keys behind it as well
#pragma unroll
            for (int qb = 0; qb < NQB; qb++) within[qb] = min(limit[qb], end);
            hide_keys<NQB>(S, first + 4 * g, within);
        }
        raise_reference<T, E, NQB>(st, S, p.sl2, slack);
        wait_vmem_at_most<NI>();                          // V
        asm volatile("" ::: "memory");
        tile_values<T, E, NQB, HIDDEN>(st, S, vaddr, TILE, p.sl2, found);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        request(vh, p.v_token, from_v, first + TURN, lds0 + TILE);
    };
    const int plain_end = min(end, seen_by_all);
#pragma unroll 1
    for (; first + kTile <= plain_end; first += TURN) tile(std::false_type{});
    const int first_hidden = first;
#pragma unroll 1
    for (; first < end; first += TURN) tile(std::true_type{});
    wait_all_memory();
    if (__builtin_amdgcn_ballot_w64(found != 0) != 0)
        for (int at = first_hidden; at < end; at += TURN) add_special_values<T, E, NQB>(st, vh, p.v_token, at, min(end, at + kTile), limit, g);
    lds_accesses_then_barrier();                          // every wave is done with its tiles

    // The waves' sums meet in LDS, two blocks of rows at a time; each wave joins a quarter of the columns.
    constexpr int TOGETHER = NQB < 2 ? NQB : 2, COLUMNS = E / 16 / 4;
    f32x4* sums = reinterpret_cast<f32x4*>(smem);         // [wave][block of rows][block of columns][lane]
    f32x2* stats = reinterpret_cast<f32x2*>(smem + 4 * TOGETHER * E * 64);   // [wave][block of rows][lane]
    const bool alone = p.parts == 1 || ks.count <= p.part_keys;
#pragma unroll
    for (int qb0 = 0; qb0 < NQB; qb0 += TOGETHER) {
        if (qb0 > 0) lds_accesses_then_barrier();
#pragma unroll
        for (int b = 0; b < TOGETHER; b++) {
            const int qb = qb0 + b;
#pragma unroll
            for (int eb = 0; eb < E / 16; eb++) sums[((w * TOGETHER + b) * (E / 16) + eb) * 64 + lane] = st.O[eb][qb];
            // (not yet times the scale: a difference of two references times the scale may overflow to a weight of zero, either alone to a NaN)
            const float m = st.L[qb][0] == 0.f ? -INFINITY : -st.negm[qb][0];   // no weight: no reference
            stats[(w * TOGETHER + b) * 64 + lane] = f32x2{m, st.L[qb][0]};
        }
        lds_accesses_then_barrier();
#pragma unroll
        for (int b = 0; b < TOGETHER; b++) {
            const int row = row0 + (qb0 + b) * 16 + l16;
            float m[4], l[4], top = -INFINITY;
#pragma unroll
            for (int v = 0; v < 4; v++) {
                const f32x2 x = stats[(v * TOGETHER + b) * 64 + lane];
                m[v] = x[0];
                l[v] = x[1];
                top = fmaxf(top, m[v]);
            }
            float total = 0.f;
#pragma unroll
            for (int v = 0; v < 4; v++) {
                m[v] = m[v] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[v] - top) * p.sl2);
                total += l[v] * m[v];
            }
            f32x4 o[COLUMNS];
#pragma unroll
            for (int i = 0; i < COLUMNS; i++) {
                o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int v = 0; v < 4; v++) o[i] += sums[((v * TOGETHER + b) * (E / 16) + w * COLUMNS + i) * 64 + lane] * m[v];
            }
            if (row >= row0 + rows) continue;
            const int column = w * COLUMNS * 16 + 4 * g;
            if (alone) {
                const float f = limit[qb0 + b] > 0 ? 1.f / total : 0.f;          // no key to see: zero
                uint16_t* to = p.out + (int64_t)(qs.first + row / p.G) * p.out_token + (head * p.G + row % p.G) * p.out_head + column;
#pragma unroll
                for (int i = 0; i < COLUMNS; i++) *reinterpret_cast<u32x2*>(to + i * 16) = u32x2{T::pack(o[i][0] * f, o[i][1] * f), T::pack(o[i][2] * f, o[i][3] * f)};
            } else {
                const int64_t at = (((int64_t)s * p.Hk + head) * p.parts + part) * p.few_rows + row;
#pragma unroll
                for (int i = 0; i < COLUMNS; i++) *reinterpret_cast<f32x4*>(p.partial + at * E + column + i * 16) = o[i];
                if (w == 0 && g == 0)
                    *reinterpret_cast<f32x2*>(p.partial + (int64_t)p.S * p.Hk * p.parts * p.few_rows * E + at * 2) = f32x2{top, total};
            }
        }
    }
}

// Joins the parts of the sequences that have more than one: a wave per row.
template <class T, int E>
__global__ __launch_bounds__(256) void attn_packed_join_kernel(PackedParams p) {
    const int lane = threadIdx.x & 63;
    const int64_t id = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (id >= (int64_t)p.S * p.Hk * p.few_rows) return;
    const int row = (int)(id % p.few_rows), head = (int)(id / p.few_rows % p.Hk), s = (int)(id / p.few_rows / p.Hk);
    const Rows qs = queries_of(p, s), ks = keys_of(p, s);
    if (row >= qs.count * p.G || ks.count <= p.part_keys) return;
    const int parts = (ks.count - 1) / p.part_keys + 1;
    const float* sums = p.partial + (((int64_t)s * p.Hk + head) * p.parts * p.few_rows + row) * E;
    const float* stats = p.partial + (int64_t)p.S * p.Hk * p.parts * p.few_rows * E + (((int64_t)s * p.Hk + head) * p.parts * p.few_rows + row) * 2;
    constexpr int PER = E / 64;                           // columns of a lane
    float top = -INFINITY, total = 0.f, o[PER] = {};
    for (int part0 = 0; part0 < parts; part0 += 64) {     // 64 parts' references and sums at a time
        f32x2 mine = f32x2{-INFINITY, 0.f};
        if (part0 + lane < parts) mine = *reinterpret_cast<const f32x2*>(stats + (int64_t)(part0 + lane) * p.few_rows * 2);
        float most = mine[0];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        most = fmaxf(most, top);
        const float before = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - most) * p.sl2);
        const float weight = mine[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mine[0] - most) * p.sl2);
        float add = mine[1] * weight;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) add += __shfl_xor(add, d);
        total = total * before + add;
        top = most;
#pragma unroll
        for (int i = 0; i < PER; i++) o[i] *= before;
        const int here = min(64, parts - part0);
        auto load = [&](int n, float (&v)[PER]) {
            const float* from = sums + (int64_t)(part0 + n) * p.few_rows * E + lane * PER;
            if constexpr (PER == 2) {
                const f32x2 x = *reinterpret_cast<const f32x2*>(from);
                v[0] = x[0];
                v[PER - 1] = x[1];
            } else {
                v[0] = *from;
            }
        };
        constexpr int AHEAD = 8;
        for (int n0 = 0; n0 < here; n0 += AHEAD) {
            float v[AHEAD][PER];
#pragma unroll
            for (int n = 0; n < AHEAD; n++) load(min(n0 + n, here - 1), v[n]);
#pragma unroll
            for (int n = 0; n < AHEAD; n++) {
                const float f = n0 + n < here ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), min(n0 + n, here - 1))) : 0.f;
                if (n0 + n < here) {
#pragma unroll
                    for (int i = 0; i < PER; i++) o[i] += v[n][i] * f;
                }
            }
        }
    }
    // a row that sees no key has no weight anywhere
    const int i = row / p.G;
    const float f = p.causal && i + 1 + ks.count - qs.count <= 0 ? 0.f : 1.f / total;
    uint16_t* to = p.out + (int64_t)(qs.first + i) * p.out_token + (head * p.G + row % p.G) * p.out_head + lane * PER;
    if constexpr (PER == 2) {
        *reinterpret_cast<uint32_t*>(to) = T::pack(o[0] * f, o[PER - 1] * f);
    } else {
        *to = (uint16_t)T::pack(o[0] * f, 0.f);
    }
}

// Tiles (of a head, or of a sequence and key head) and workgroups of a launch: in double precision, for sizes that no launch covers.
constexpr double kMostWorkgroups = 1 << 24;               // a launch has fewer than 2^32 threads
struct PackedGrid {
    double tiles, workgroups;
};
static PackedGrid rows_grid(int rows, int S, int64_t Tq, int Hq, int Hk, int max_q) {
    const int64_t tiles = max_q <= rows ? S : Tq / rows + std::min<int64_t>(S, Tq);
    // (whole turns over the XCDs: tiles of every XCD's heads, or of a head's XCDs)
    const int64_t whole = Hk % 8 != 0 && 8 % Hk == 0 ? (tiles + 8 / Hk - 1) / (8 / Hk) * (8 / Hk) : tiles;
    return PackedGrid{(double)tiles, (double)whole * Hq};
}
static PackedGrid few_grid(int rows, int S, int Hk, int64_t few_rows, int parts) {
    const double tiles = (double)((few_rows + rows - 1) / rows);
    return PackedGrid{tiles, tiles * S * Hk * parts};
}

template <class T, int E, int NQB>
static int32_t launch_rows(PackedParams p, hipStream_t stream) {
    constexpr int ROWS = 64 * NQB, LDS = 2 * kStepTiles * 2 * kTile * E * 2;
    const PackedGrid grid = rows_grid(ROWS, p.S, p.Tq, p.Hq, p.Hk, p.max_q);
    p.tiles = (int)grid.tiles;
    attn_packed_rows_kernel<T, E, NQB><<<(uint32_t)grid.workgroups, 256, LDS, stream>>>(p);
    return launch_status();
}

// A few queries over many keys are walked in parts: rows of a key head, keys of a workgroup, parts of the longest sequence.
// rows 0: in whole sequences, where parts and their joining take longer; over 264 batches, all sequences as long, the choice takes 1.018 times
// the quicker's time in the mean (us by parts and whole: 8 heads x 4 rows, 1000 keys 8.3 8.0, 1500 8.5
// 9.7, 4000 10.8 27.6; 128 heads, 1500 24.2 22.8, 2000 29.5 31.5; 8 heads x 64 rows, 2000 15.8 11.5, 8000 19.0 47.0; 128 heads 45 33 and 125 113;
// 1 head x 512 rows, 2000 15.4 11.3, 8000 19.4 39.5; 8 heads 22.4 15.8, 4000 35 27, 8000 41 47; 32 heads 47 29 and 125 129).  However many the
// heads, parts begin at 3000 or 5000 keys: whole, the one long sequence of a ragged batch would take one CU a head.
struct FewPlan {
    int rows, part_keys, parts;
};
// A part's length: a workgroup walks its keys, a row's parts are joined one behind the other, every part costs its start and end, and between
// one and two workgroups to a CU some CUs have twice the work.  Measured on 112 batches, ragged and not, 1 to 512 heads of 1300 to 38 000
// keys: the length taken is 1.022 times the quickest's time in the mean, 1.21 at most (us by 256, 512, 1024, 2048, 4096 keys: 136 heads of up
// to 4125 keys 42.4 42.9 44.1 62.1 86.4; 16 of 36 258 63.8 58.6 52.1 49.2 64.3; 512 of 10 000, all as long, 514 478 455 444 463).
// A limit may be far above the lengths: beyond 2^17 workgroups the parts grow with it, so that neither the workspace (4.4 GB at most) nor the
// launch does, and the call goes by the rows that there are (few_plan_within).
constexpr int64_t kMostPartWorkgroups = 1 << 17;
static int parts_of(int max_k, int keys) { return (int)(((int64_t)max_k + keys - 1) / keys); }
static FewPlan few_plan(int S, int Hq, int Hk, int max_q, int max_k) {
    const int64_t rows = (int64_t)max_q * (Hq / Hk), heads = (int64_t)S * Hk;
    if (rows > 1024 || heads > kMostPartWorkgroups / 2) return FewPlan{0, 0, 0};
    const int64_t blocks = heads * ((rows + 63) / 64);
    const int64_t least_keys = rows <= 32 ? std::min<int64_t>(1000 + 15 * heads, 3000) : std::min<int64_t>(2800 + 30 * blocks, 5000);
    if (max_k <= least_keys || (rows > 32 && blocks >= 128)) return FewPlan{0, 0, 0};
    int keys = 0;
    double least = 0.0;
    for (int length = 256; length <= 4096; length *= 2) {
        const int64_t workgroups = blocks * parts_of(max_k, length);
        const double price = length * (workgroups > 256 && workgroups < 512 ? 1.3 : 1.0) + (double)max_k / length * (30.0 + (double)blocks);
        if (keys == 0 || price < least) {
            keys = length;
            least = price;
        }
    }
    while (blocks * parts_of(max_k, keys) > kMostPartWorkgroups) keys *= 2;   // (two parts of 2^30 keys at the latest)
    return FewPlan{(int)rows, keys, parts_of(max_k, keys)};
}
// The plan for no more than Tk keys, with no more parts than the workspace of the limits as given has room for.
static FewPlan few_plan_within(int S, int Hq, int Hk, int max_q, int max_k, int Tk) {
    const FewPlan given = few_plan(S, Hq, Hk, max_q, max_k);
    if (given.rows == 0 || max_k <= Tk) return given;
    FewPlan plan = few_plan(S, Hq, Hk, max_q, Tk);
    while (plan.parts > given.parts) {
        plan.part_keys *= 2;
        plan.parts = parts_of(Tk, plan.part_keys);
    }
    return plan;
}
static size_t few_bytes(const FewPlan& f, int S, int Hk, int E) {
    return f.parts <= 1 ? 0 : (size_t)S * Hk * f.parts * f.rows * (E + 2) * sizeof(float);
}

// Everything else has a form by its price in us: how many workgroups there are, each with its start and end, 512 of them side by side; what
// 64 keys take the workgroup that has the most of them, which bounds a small launch; what 64 rows x 64 keys take where the CUs are full, and a share
// of the last workgroup.  Fitted to 2567 random batches of 1 to 32 sequences of up to 10 000 tokens, 1 to 120 heads, causal or not: the form
// taken is 1.010 times the quickest's time in the mean.  The lengths are on the device: one sequence of the given limits is assumed, and the
// rest of the rows evenly spread over the others.  Workgroups beyond those find nothing to do, which takes 0.8 us for a thousand of them: the
// rows of a key head are cut as often for every sequence as for the longest (over 1365 batches of one or two prompts of 100 to 8000 tokens and up to
// 2000 of 1 to 40 1.031 times the quickest's time in the mean; without this term 1.40, and 14.6 at most: 6430 tokens and 483 single ones, 8
// heads over 1, 64 rows 88 us, 32 rows of the key head 582).
enum PackedForm { kKeys16, kKeys32, kRows64, kRows128, kRows192, kPackedForms };
struct PackedPrice {
    int rows;
    float start, alone, full;
};
static const PackedPrice kPackedPrices[2][kPackedForms] = {{{16, 3.8f, 0.17f, 0.81f}, {32, 6.6f, 0.21f, 0.37f}, {64, 3.2f, 0.80f, 0.36f}, {128, 4.4f, 1.26f, 0.29f}, {192, 9.2f, 1.22f, 0.275f}},
                                                           {{16, 5.5f, 0.165f, 1.78f}, {32, 8.3f, 0.43f, 0.70f}, {64, 5.1f, 0.94f, 0.64f}, {128, 5.1f, 1.49f, 0.50f}, {192, 13.8f, 2.34f, 0.41f}}};
static const float kPackedLast[2][2] = {{0.35f, 0.25f}, {0.49f, 0.53f}};   // of E = 64, 128; all keys, causal
static const double kPackedEmpty = 0.0008;               // us
static double packed_price(PackedForm form, int S, int64_t Tq, int Hq, int Hk, int E, int max_q, int max_k, int causal) {
    const PackedPrice& f = kPackedPrices[E == 128][form];
    const bool grouped = form <= kKeys32;                 // rows of a key head, of all its queries' heads
    const double launched = (grouped ? few_grid(f.rows, S, Hk, (int64_t)max_q * (Hq / Hk), 1) : rows_grid(f.rows, S, Tq, Hq, Hk, max_q)).workgroups;
    if (launched >= kMostWorkgroups) return HUGE_VAL;
    const double per_query = grouped ? (double)Hq / Hk : 1.0, heads = grouped ? Hk : Hq;
    double workgroups = 0, units = 0;
    const double rest = S > 1 ? std::max(0.0, (double)(Tq - max_q) / (S - 1)) : 0.0;
    auto add = [&](double sequences, double nq, double nk) {
        const double blocks = std::max(1.0, (double)(int64_t)((nq * per_query + f.rows - 1) / f.rows));
        const double keys = causal ? std::max(nk - nq / 2 + f.rows / per_query / 2, std::min(nk, 64.0)) : nk;
        workgroups += sequences * blocks * heads;
        units += sequences * blocks * heads * (f.rows / 64.0) * (std::min(keys, nk) / 64);
    };
    add(1, max_q, max_k);
    if (S > 1) add(S - 1, rest, rest * max_k / max_q);
    const double longest = max_k / 64.0, last = kPackedLast[E == 128][causal != 0] * longest * (f.rows / 64.0) * f.full;
    return f.start * std::max(1.0, workgroups / 512) + std::max(longest * f.alone, units / 256 * f.full + last) + kPackedEmpty * std::max(0.0, launched - workgroups);
}
static PackedForm packed_form(int S, int64_t Tq, int Hq, int Hk, int E, int max_q, int max_k, int causal) {
    PackedForm best = kKeys16;
    double least = packed_price(best, S, Tq, Hq, Hk, E, max_q, max_k, causal);
    for (int f = 1; f < kPackedForms; f++) {
        const double price = packed_price((PackedForm)f, S, Tq, Hq, Hk, E, max_q, max_k, causal);
        if (price < least) {
            best = (PackedForm)f;
            least = price;
        }
    }
    return best;
}

template <class T, int E, int NQB>
static int32_t launch_few(PackedParams p, hipStream_t stream) {
    constexpr int TOGETHER = NQB < 2 ? NQB : 2;
    constexpr int LDS = std::max(4 * 2 * kTile * E * 2, 4 * TOGETHER * (E * 64 + 512));
    const auto kernel = attn_packed_few_kernel<T, E, NQB>;
    const PackedGrid grid = few_grid(16 * NQB, p.S, p.Hk, p.few_rows, p.parts);
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    p.tiles = (int)grid.tiles;
    kernel<<<(uint32_t)grid.workgroups, 256, LDS, stream>>>(p);
    if (p.parts > 1) attn_packed_join_kernel<T, E><<<(uint32_t)(((int64_t)p.S * p.Hk * p.few_rows + 3) / 4), 256, 0, stream>>>(p);
    return launch_status();
}

template <class T, int E>
static int32_t launch_packed(PackedParams p, const FewPlan& few, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (few.rows > 0) {
        if (few_bytes(few, p.S, p.Hk, E) > (ws ? ws_bytes : 0)) return CHIPMUNK_ERR_WORKSPACE;
        p.few_rows = few.rows;
        p.part_keys = few.part_keys;
        p.parts = few.parts;
        p.partial = static_cast<float*>(ws);
        return few.rows <= 16 ? launch_few<T, E, 1>(p, stream) : few.rows <= 32 ? launch_few<T, E, 2>(p, stream) : launch_few<T, E, 4>(p, stream);
    }
    const PackedForm form = packed_form(p.S, p.Tq, p.Hq, p.Hk, E, p.max_q, p.max_k, p.causal);
    if (packed_price(form, p.S, p.Tq, p.Hq, p.Hk, E, p.max_q, p.max_k, p.causal) == HUGE_VAL) return CHIPMUNK_ERR_SHAPE;   // no form's launch covers it
    if (form <= kKeys32) {
        p.few_rows = p.max_q * p.G;
        p.part_keys = INT32_MAX;
        p.parts = 1;
    }
    switch (form) {
        case kKeys16: return launch_few<T, E, 1>(p, stream);
        case kKeys32: return launch_few<T, E, 2>(p, stream);
        case kRows64: return launch_rows<T, E, 1>(p, stream);
        case kRows128: return launch_rows<T, E, 2>(p, stream);
        default: return launch_rows<T, E, 3>(p, stream);
    }
}

}  // namespace chipmunk

using namespace chipmunk;

// The form that a call takes and, for parts, their keys, for the tests.
extern "C" int chipmunk_internal_attn_packed_form(int S, int Tq, int Hq, int Hk, int E, int max_q, int max_k, int causal) {
    const FewPlan few = few_plan(S, Hq, Hk, max_q, max_k);
    return few.rows > 0 ? few.part_keys : packed_form(S, Tq, Hq, Hk, E, std::min(max_q, Tq), max_k, causal);
}

extern "C" size_t chipmunk_attn_packed_workspace_bytes(int S, int Hq, int Hk, int E, int max_q, int max_k) {
    if (S <= 0 || Hq <= 0 || Hk <= 0 || Hq % Hk != 0 || (E != 64 && E != 128) || max_q <= 0 || max_k <= 0) return 0;
    return few_bytes(few_plan(S, Hq, Hk, max_q, max_k), S, Hk, E);
}

extern "C" int32_t chipmunk_attn_packed(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const uint16_t* k, int64_t k_token_stride,
                                        int64_t k_head_stride, const uint16_t* v, int64_t v_token_stride, int64_t v_head_stride, uint16_t* out,
                                        int64_t out_token_stride, int64_t out_head_stride, const int32_t* cu_q, const int32_t* cu_k, const int32_t* k_len,
                                        int S, int Tq, int Tk, int Hq, int Hk, int E, int max_q, int max_k, int causal, float softmax_scale, int dtype,
                                        void* ws, size_t ws_bytes, void* stream) {
    if (!q || !k || !v || !out || !cu_q || !cu_k) return CHIPMUNK_ERR_NULL;
    if (S <= 0 || Tq <= 0 || Tk <= 0 || Hq <= 0 || Hk <= 0 || Hq % Hk != 0 || max_q <= 0 || max_k <= 0) return CHIPMUNK_ERR_SHAPE;
    const float sl2 = softmax_scale * 1.4426950408889634f;
    if (!is_positive_finite_scalar(softmax_scale) || !is_finite_scalar(sl2)) return CHIPMUNK_ERR_SHAPE;
    if ((E != 64 && E != 128) || (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16)) return CHIPMUNK_ERR_UNSUPPORTED;
    constexpr int64_t kMostStride = 1 << 24;
    if (Tq == 1) q_token_stride = out_token_stride = E;   // of one row alone a stride means nothing
    if (Tk == 1) k_token_stride = v_token_stride = E;
    for (int64_t token : {q_token_stride, k_token_stride, v_token_stride, out_token_stride})
        if (token < E || token >= kMostStride) return CHIPMUNK_ERR_SHAPE;
    if ((Hq > 1 && (q_head_stride < E || out_head_stride < E)) || (Hk > 1 && (k_head_stride < E || v_head_stride < E))) return CHIPMUNK_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) ||
        !aligned16(ws) || ((reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(cu_k) | reinterpret_cast<uintptr_t>(k_len)) & 3) ||
        (q_token_stride | k_token_stride | v_token_stride | out_token_stride) % 8 != 0 || (Hq > 1 && (q_head_stride | out_head_stride) % 8 != 0) ||
        (Hk > 1 && (k_head_stride | v_head_stride) % 8 != 0))
        return CHIPMUNK_ERR_ALIGN;
    const PackedParams p{q, k, v, out, cu_q, cu_k, k_len, q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
                         out_token_stride, out_head_stride, S, Tq, Tk, Hq, Hk, Hq / Hk, std::min(max_q, Tq), std::min(max_k, Tk), causal != 0, 0, 0, 0, 0, nullptr,
                         sl2};
    const FewPlan few = few_plan_within(S, Hq, Hk, max_q, max_k, Tk);
    const auto st = static_cast<hipStream_t>(stream);
    if (dtype == CHIPMUNK_DTYPE_BF16) return E == 128 ? launch_packed<Bf16, 128>(p, few, ws, ws_bytes, st) : launch_packed<Bf16, 64>(p, few, ws, ws_bytes, st);
    return E == 128 ? launch_packed<Fp16, 128>(p, few, ws, ws_bytes, st) : launch_packed<Fp16, 64>(p, few, ws, ws_bytes, st);
}
