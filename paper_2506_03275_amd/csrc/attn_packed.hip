// Attention over packed sequences of different lengths: causal or not, heads grouped over the keys' heads.
//
// attn_packed_rows_kernel: one workgroup of four waves owns 64 NQB consecutive queries of one sequence and head and walks the
// sequence's keys in steps of two tiles of 32.  K and V tiles go from memory to LDS by asynchronous 16-byte loads, double
// buffered by step; scores are formed transposed, S^T = K Q^T, so that a lane holds, for one query (lane % 16), four keys of each
// block of 16, which are the contraction entries that it supplies to O^T += V^T P^T: probabilities go from the softmax into the
// second product without leaving registers.  One pass with a running maximum and sum.
#include "element.h"

#include <algorithm>
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
    for (int u = 0; u < 2; u++)
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int qb = 0; qb < NQB; qb++)
                if (first + u * 16 + r >= limit[qb]) S[u][qb][r] = -INFINITY;
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

// Whether the lower or the upper element of a word is infinite or NaN.  (On the bits: these files are compiled as if NaN did not
// exist, and a comparison of values is folded accordingly.)
template <class T>
__device__ __forceinline__ bool low_not_finite(uint32_t word) { return (~word & T::kExponent & 0xffffu) == 0; }
template <class T>
__device__ __forceinline__ bool high_not_finite(uint32_t word) { return (~word & T::kExponent & 0xffff0000u) == 0; }

// One word of two elements without those that are infinite or NaN; they are noted in `found`.
template <class T>
__device__ __forceinline__ uint32_t finite_elements(uint32_t word, bool& found) {
    const bool low = low_not_finite<T>(word), high = high_not_finite<T>(word);
    found |= low || high;
    return word & ((low ? 0u : 0xffffu) | (high ? 0u : 0xffff0000u));
}

// P = exp2(S sl2) rounded to the element type (to 8 or 11 bits, like the values that it weights), its sum, and O^T += V^T P^T.
// HIDDEN: some keys are hidden from some of the queries, and a hidden key's zero probability times an infinite or NaN value would
// be a NaN: such values are left out and noted.
template <class T, int E, int NQB, bool HIDDEN>
__device__ __forceinline__ void tile_values(RowState<T, E, NQB>& st, const f32x4 (&S)[2][NQB], const uint32_t (&vaddr)[E / 16], int tile_off, float sl2,
                                            bool& found) {
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
    bool found = false;
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
#pragma unroll 1
    for (; first < keys; first += kStepKeys) {
        const int half = first / kStepKeys & 1;
        arrived(first);
#pragma unroll
        for (int j = 0; j < E / 16; j++) request(half ^ 1, j);
        if (first >= seen) continue;                      // nothing to see for this wave
        uint32_t kat[E / 32], vat[E / 16];
#pragma unroll
        for (int es = 0; es < E / 32; es++) kat[es] = kaddr[es] + half * kStepTiles * STAGE;
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) vat[eb] = vaddr[eb] + half * kStepTiles * STAGE;
#pragma unroll
        for (int n = 0; n < kStepTiles; n++) {
            f32x4 S[2][NQB];
            tile_scores<T, E, NQB>(S, st, kat, n * STAGE, [](int) {});
            hide_keys<NQB>(S, first + n * kTile + 4 * g, limit);
            raise_reference<T, E, NQB>(st, S, p.sl2, slack);
            tile_values<T, E, NQB, true>(st, S, vat, n * STAGE + TILE, p.sl2, found);
        }
    }
    wait_all_memory();                                    // the transfers behind the last step

    // Infinite and NaN values among the steps with hidden keys go to the queries that see them.
    if (__builtin_amdgcn_ballot_w64(found) != 0) {
#pragma unroll 1
        for (int key = first_hidden; key < seen; key++) {
            const uint16_t* from = vh + key * p.v_token + 4 * g;
#pragma unroll
            for (int eb = 0; eb < E / 16; eb++) {
                const u32x2 words = *reinterpret_cast<const u32x2*>(from + eb * 16);
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    float value = r % 2 ? T::high(words[r / 2]) : T::low(words[r / 2]);
                    const bool special = r % 2 ? high_not_finite<T>(words[r / 2]) : low_not_finite<T>(words[r / 2]);
                    asm volatile("" : "+v"(value));       // nothing is known of it, not even that it is none of the two
#pragma unroll
                    for (int qb = 0; qb < NQB; qb++)
                        if (special && key < limit[qb]) st.O[eb][qb][r] += value;
                }
            }
        }
    }

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

template <class T, int E, int NQB>
static int32_t launch_rows(PackedParams p, hipStream_t stream) {
    constexpr int ROWS = 64 * NQB, LDS = 2 * kStepTiles * 2 * kTile * E * 2;
    const int64_t tiles = p.max_q <= ROWS ? p.S : (int64_t)p.Tq / ROWS + std::min(p.S, p.Tq);
    // (a grid of whole turns over the XCDs: tiles of every XCD's heads, or of a head's XCDs)
    const int64_t whole = p.Hk % 8 == 0 ? tiles * p.Hq : 8 % p.Hk == 0 ? (tiles + 8 / p.Hk - 1) / (8 / p.Hk) * 8 * p.G : tiles * p.Hq;
    if (whole >= INT64_C(1) << 24) return CHIPMUNK_ERR_SHAPE;
    p.tiles = (int)tiles;
    attn_packed_rows_kernel<T, E, NQB><<<(uint32_t)whole, 256, LDS, stream>>>(p);
    return launch_status();
}

template <class T>
static int32_t launch_packed(const PackedParams& p, int E, hipStream_t stream) {
    return E == 128 ? launch_rows<T, 128, 2>(p, stream) : launch_rows<T, 64, 2>(p, stream);
}

}  // namespace chipmunk

using namespace chipmunk;

extern "C" size_t chipmunk_attn_packed_workspace_bytes(int S, int Hq, int Hk, int E, int max_q, int max_k) {
    return 0;
}

extern "C" int32_t chipmunk_attn_packed(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const uint16_t* k, int64_t k_token_stride,
                                        int64_t k_head_stride, const uint16_t* v, int64_t v_token_stride, int64_t v_head_stride, uint16_t* out,
                                        int64_t out_token_stride, int64_t out_head_stride, const int32_t* cu_q, const int32_t* cu_k, const int32_t* k_len,
                                        int S, int Tq, int Tk, int Hq, int Hk, int E, int max_q, int max_k, int causal, float softmax_scale, int dtype,
                                        void* ws, size_t ws_bytes, void* stream) {
    if (!q || !k || !v || !out || !cu_q || !cu_k) return CHIPMUNK_ERR_NULL;
    if (S <= 0 || Tq <= 0 || Tk <= 0 || Hq <= 0 || Hk <= 0 || Hq % Hk != 0 || max_q <= 0 || max_k <= 0) return CHIPMUNK_ERR_SHAPE;
    if (!is_positive_finite_scalar(softmax_scale)) return CHIPMUNK_ERR_SHAPE;
    if ((E != 64 && E != 128) || (dtype != CHIPMUNK_DTYPE_BF16 && dtype != CHIPMUNK_DTYPE_FP16)) return CHIPMUNK_ERR_UNSUPPORTED;
    constexpr int64_t kMostStride = 1 << 24;
    for (int64_t token : {q_token_stride, k_token_stride, v_token_stride, out_token_stride})
        if (token < E || token >= kMostStride) return CHIPMUNK_ERR_SHAPE;
    if ((Hq > 1 && (q_head_stride < E || out_head_stride < E)) || (Hk > 1 && (k_head_stride < E || v_head_stride < E))) return CHIPMUNK_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) ||
        ((reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(cu_k) | reinterpret_cast<uintptr_t>(k_len)) & 3) ||
        (q_token_stride | k_token_stride | v_token_stride | out_token_stride) % 8 != 0 || (Hq > 1 && (q_head_stride | out_head_stride) % 8 != 0) ||
        (Hk > 1 && (k_head_stride | v_head_stride) % 8 != 0))
        return CHIPMUNK_ERR_ALIGN;
    const PackedParams p{q, k, v, out, cu_q, cu_k, k_len, q_token_stride, q_head_stride, k_token_stride, k_head_stride, v_token_stride, v_head_stride,
                         out_token_stride, out_head_stride, S, Tq, Tk, Hq, Hk, Hq / Hk, std::min(max_q, Tq), std::min(max_k, Tk), causal != 0, 0,
                         softmax_scale * 1.4426950408889634f};
    return dtype == CHIPMUNK_DTYPE_BF16 ? launch_packed<Bf16>(p, E, static_cast<hipStream_t>(stream)) : launch_packed<Fp16>(p, E, static_cast<hipStream_t>(stream));
}
