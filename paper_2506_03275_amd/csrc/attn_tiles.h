// What the kernels of attention over sequences of different lengths share (packed, attn_packed.hip; paged, attn_paged.hip): a tile
// of 32 keys against blocks of 16 rows, and the plans of their launches.  Internal.
#pragma once
#include "element.h"

#include <algorithm>
#include <cmath>

namespace chipmunk {

struct AttnParams {
    const uint16_t* q;
    uint16_t* out;
    const int32_t* cu_q;
    int64_t q_token, q_head, out_token, out_head;
    int S, Tq, Hq, Hk, G;
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
__device__ __forceinline__ Rows queries_of(const AttnParams& p, int s) {
    const int first = min(max(p.cu_q[s], 0), p.Tq), end = min(max(p.cu_q[s + 1], 0), p.Tq);
    return Rows{first, min(max(end - first, 0), p.max_q)};
}

// Tile `tile` of all sequences' tiles of ROWS queries, the last rows of a sequence first (with a causal mask they have the most
// keys).  Every wave works it out by itself.  False: there are fewer tiles.
template <int ROWS>
__device__ __forceinline__ bool find_tile(const AttnParams& p, int tile, int lane, int* sequence, int* in_sequence) {
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
    auto read = [&](int eb) {
        if (eb >= NEB) return;
        lo[eb] = lds_read_tr16_at(vaddr[eb] + tile_off);
        hi[eb] = lds_read_tr16_at(vaddr[eb] + tile_off + 16 * ROWB);
    };
    auto operand = [&](int eb) { return __builtin_bit_cast(u32x4, (short8v)__builtin_shufflevector(lo[eb], hi[eb], 0, 1, 2, 3, 4, 5, 6, 7)); };
    auto weigh = [&](int eb, u32x4 words) {
#pragma unroll
        for (int qb = 0; qb < NQB; qb++) st.O[eb][qb] = T::product(__builtin_bit_cast(x8, words), pop[qb], st.O[eb][qb]);
    };
    if constexpr (!HIDDEN) {
#pragma unroll
        for (int eb = 0; eb < NEB; eb++) {
            if (eb + AHEAD < NEB) {
                read(eb + AHEAD);
                __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            }
            weigh(eb, operand(eb));
            __builtin_amdgcn_sched_group_barrier(0x008, NQB, 0);
        }
    } else {
        // (looked for first: to take them out of every word would cost three times as much as to find that there is none)
#pragma unroll
        for (int eb = 0; eb < NEB; eb++) {
            read(eb + AHEAD);
            u32x4 words = operand(eb);
            uint32_t tops = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) tops |= not_finite<T>(words[i]);
            if (__builtin_amdgcn_ballot_w64(tops != 0) != 0) {
#pragma unroll
                for (int i = 0; i < 4; i++) words[i] = finite_elements<T>(words[i], found);
            }
            weigh(eb, words);
        }
    }
}

// Tile and head of a workgroup.  Workgroups go to the eight XCDs in turn (id modulo 8), each with an L2 of its own: a key head's
// workgroups stay on as few XCDs as there are heads for, and every XCD gets as many of the long tiles.
__device__ __forceinline__ void tile_and_head(const AttnParams& p, uint32_t id, int* tile, int* head) {
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

// A wave's NQB blocks of rows from `row0` on of `rows` go to their places.
template <class T, int E, int NQB>
__device__ __forceinline__ void store_rows(const RowState<T, E, NQB>& st, const int (&limit)[NQB], uint16_t* oh, int64_t out_token, int row0, int rows, int g, int l16) {
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        const int row = row0 + qb * 16 + l16;
        if (row >= rows) continue;
        const float f = limit[qb] > 0 ? 1.f / st.L[qb][0] : 0.f;   // no key to see: zero
        uint16_t* to = oh + row * out_token;
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

// The sums of four waves over different keys meet in LDS (4 * min(NQB, 2) * (E * 64 + 512) bytes at smem, whose earlier contents every wave
// must be done with), two blocks of rows at a time; each wave joins a quarter of the columns, E / 64 blocks of 16 from block w * E / 64 on, and
// hands them to store(block of rows, its lane's columns, reference, sum of weights).
template <class T, int E, int NQB, class Store>
__device__ __forceinline__ void join_waves(const RowState<T, E, NQB>& st, uint8_t* smem, int w, int lane, float sl2, Store&& store) {
    constexpr int TOGETHER = NQB < 2 ? NQB : 2, COLUMNS = E / 16 / 4;
    f32x4* sums = reinterpret_cast<f32x4*>(smem);         // [wave][block of rows][block of columns][lane]
    f32x2* stats = reinterpret_cast<f32x2*>(smem + 4 * TOGETHER * E * 64);   // [wave][block of rows][lane]
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
                m[v] = m[v] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[v] - top) * sl2);
                total += l[v] * m[v];
            }
            f32x4 o[COLUMNS];
#pragma unroll
            for (int i = 0; i < COLUMNS; i++) {
                o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int v = 0; v < 4; v++) o[i] += sums[((v * TOGETHER + b) * (E / 16) + w * COLUMNS + i) * 64 + lane] * m[v];
            }
            store(qb0 + b, o, top, total);
        }
    }
}

// What a workgroup's waves have joined goes to its place, or, of one part of several, to the workspace.  Row `row` of the key head; sees: it sees a key.
template <class T, int E>
__device__ __forceinline__ void store_joined(const AttnParams& p, int s, int head, int part, int first_query, int row, bool alone, bool sees, int w, int g,
                                             const f32x4 (&o)[E / 64], float top, float total) {
    constexpr int COLUMNS = E / 64;
    const int column = w * COLUMNS * 16 + 4 * g;
    if (alone) {
        const float f = sees ? 1.f / total : 0.f;         // no key to see: zero
        uint16_t* to = p.out + (int64_t)(first_query + row / p.G) * p.out_token + (head * p.G + row % p.G) * p.out_head + column;
#pragma unroll
        for (int i = 0; i < COLUMNS; i++) *reinterpret_cast<u32x2*>(to + i * 16) = u32x2{T::pack(o[i][0] * f, o[i][1] * f), T::pack(o[i][2] * f, o[i][3] * f)};
    } else {
        const int64_t at = (((int64_t)s * p.Hk + head) * p.parts + part) * p.few_rows + row;
#pragma unroll
        for (int i = 0; i < COLUMNS; i++) *reinterpret_cast<f32x4*>(p.partial + at * E + column + i * 16) = o[i];
        if (w == 0 && g == 0) *reinterpret_cast<f32x2*>(p.partial + (int64_t)p.S * p.Hk * p.parts * p.few_rows * E + at * 2) = f32x2{top, total};
    }
}

// Joins the `parts` parts of a row, one wave's work: sums, stats: those of the first part, `apart`: rows from one part's to the next's; to: its place.
template <class T, int E>
__device__ __forceinline__ void join_parts(const float* sums, const float* stats, int64_t apart, int parts, float sl2, bool sees, uint16_t* to, int lane) {
    constexpr int PER = E / 64;                           // columns of a lane
    constexpr int AHEAD = 8;
    float top = -INFINITY, total = 0.f, o[PER] = {};
    auto load = [&](int part, float (&v)[PER]) {
        const float* from = sums + part * apart * E + lane * PER;
        if constexpr (PER == 2) {
            const f32x2 x = *reinterpret_cast<const f32x2*>(from);
            v[0] = x[0];
            v[PER - 1] = x[1];
        } else {
            v[0] = *from;
        }
    };
    for (int part0 = 0; part0 < parts; part0 += 64) {     // 64 parts' references and sums at a time
        const int here = min(64, parts - part0);
        f32x2 mine = f32x2{-INFINITY, 0.f};
        if (part0 + lane < parts) mine = *reinterpret_cast<const f32x2*>(stats + (part0 + lane) * apart * 2);
        float v[AHEAD][PER];                              // under way together with those
#pragma unroll
        for (int n = 0; n < AHEAD; n++) load(part0 + min(n, here - 1), v[n]);
        float most = mine[0];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        most = fmaxf(most, top);
        const float before = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((top - most) * sl2);
        const float weight = mine[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mine[0] - most) * sl2);
        float add = mine[1] * weight;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) add += __shfl_xor(add, d);
        total = total * before + add;
        top = most;
#pragma unroll
        for (int i = 0; i < PER; i++) o[i] *= before;
        for (int n0 = 0; n0 < here; n0 += AHEAD) {
            float next[AHEAD][PER];
#pragma unroll
            for (int n = 0; n < AHEAD; n++) load(part0 + min(n0 + AHEAD + n, here - 1), next[n]);
#pragma unroll
            for (int n = 0; n < AHEAD; n++) {
                const float f = n0 + n < here ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, weight), min(n0 + n, here - 1))) : 0.f;
                if (n0 + n < here) {
#pragma unroll
                    for (int i = 0; i < PER; i++) o[i] += v[n][i] * f;
                }
#pragma unroll
                for (int i = 0; i < PER; i++) v[n][i] = next[n][i];
            }
        }
    }
    // a row that sees no key has no weight anywhere
    const float f = sees ? 1.f / total : 0.f;
    to += lane * PER;
    if constexpr (PER == 2) {
        *reinterpret_cast<uint32_t*>(to) = T::pack(o[0] * f, o[PER - 1] * f);
    } else {
        *to = (uint16_t)T::pack(o[0] * f, 0.f);
    }
}

// The same of a row of a key head, where store_joined left its parts.
template <class T, int E>
__device__ __forceinline__ void join_parts(const AttnParams& p, int s, int head, int row, int first_query, int parts, bool sees, int lane) {
    const int64_t first = ((int64_t)s * p.Hk + head) * p.parts * p.few_rows + row;
    join_parts<T, E>(p.partial + first * E, p.partial + (int64_t)p.S * p.Hk * p.parts * p.few_rows * E + first * 2, p.few_rows, parts, p.sl2, sees,
                     p.out + (int64_t)(first_query + row / p.G) * p.out_token + (head * p.G + row % p.G) * p.out_head, lane);
}

// Tiles (of a head, or of a sequence and key head) and workgroups of a launch: in double precision, for sizes that no launch covers.
constexpr double kMostWorkgroups = 1 << 24;               // a launch has fewer than 2^32 threads
struct PackedGrid {
    double tiles, workgroups;
};
inline PackedGrid rows_grid(int rows, int S, int64_t Tq, int Hq, int Hk, int max_q) {
    const int64_t tiles = max_q <= rows ? S : Tq / rows + std::min<int64_t>(S, Tq);
    // (whole turns over the XCDs: tiles of every XCD's heads, or of a head's XCDs)
    const int64_t whole = Hk % 8 != 0 && 8 % Hk == 0 ? (tiles + 8 / Hk - 1) / (8 / Hk) * (8 / Hk) : tiles;
    return PackedGrid{(double)tiles, (double)whole * Hq};
}
inline PackedGrid few_grid(int rows, int S, int Hk, int64_t few_rows, int parts) {
    const double tiles = (double)((few_rows + rows - 1) / rows);
    return PackedGrid{tiles, tiles * S * Hk * parts};
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
inline int parts_of(int max_k, int keys) { return (int)(((int64_t)max_k + keys - 1) / keys); }
inline FewPlan few_plan(int S, int Hq, int Hk, int max_q, int max_k) {
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
inline FewPlan few_plan_within(int S, int Hq, int Hk, int max_q, int max_k, int Tk) {
    const FewPlan given = few_plan(S, Hq, Hk, max_q, max_k);
    if (given.rows == 0 || max_k <= Tk) return given;
    FewPlan plan = few_plan(S, Hq, Hk, max_q, Tk);
    while (plan.parts > given.parts) {
        plan.part_keys *= 2;
        plan.parts = parts_of(Tk, plan.part_keys);
    }
    return plan;
}
inline size_t few_bytes(const FewPlan& f, int S, int Hk, int E) {
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
constexpr PackedPrice kPackedPrices[2][kPackedForms] = {{{16, 3.8f, 0.17f, 0.81f}, {32, 6.6f, 0.21f, 0.37f}, {64, 3.2f, 0.80f, 0.36f}, {128, 4.4f, 1.26f, 0.29f}, {192, 9.2f, 1.22f, 0.275f}},
                                                           {{16, 5.5f, 0.165f, 1.78f}, {32, 8.3f, 0.43f, 0.70f}, {64, 5.1f, 0.94f, 0.64f}, {128, 5.1f, 1.49f, 0.50f}, {192, 13.8f, 2.34f, 0.41f}}};
constexpr float kPackedLast[2][2] = {{0.35f, 0.25f}, {0.49f, 0.53f}};   // of E = 64, 128; all keys, causal
constexpr double kPackedEmpty = 0.0008;               // us
// last_share: of the last workgroup; parts: in which every workgroup's keys are divided
inline double form_price(PackedForm form, const PackedPrice& f, double last_share, int S, int64_t Tq, int Hq, int Hk, int max_q, int max_k, int causal, int parts = 1) {
    const bool grouped = form <= kKeys32;                 // rows of a key head, of all its queries' heads
    const double launched = (grouped ? few_grid(f.rows, S, Hk, (int64_t)max_q * (Hq / Hk), 1) : rows_grid(f.rows, S, Tq, Hq, Hk, max_q)).workgroups;
    if (launched * parts >= kMostWorkgroups) return HUGE_VAL;
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
    const double longest = max_k / 64.0 / parts, last = last_share * longest * (f.rows / 64.0) * f.full;
    workgroups *= parts;
    return f.start * std::max(1.0, workgroups / 512) + std::max(longest * f.alone, units / 256 * f.full + last) + kPackedEmpty * std::max(0.0, launched * parts - workgroups);
}
inline double packed_price(PackedForm form, int S, int64_t Tq, int Hq, int Hk, int E, int max_q, int max_k, int causal) {
    return form_price(form, kPackedPrices[E == 128][form], kPackedLast[E == 128][causal != 0], S, Tq, Hq, Hk, max_q, max_k, causal);
}
inline PackedForm packed_form(int S, int64_t Tq, int Hq, int Hk, int E, int max_q, int max_k, int causal) {
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


}  // namespace chipmunk
