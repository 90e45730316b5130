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

#include "attn_tiles.h"

#include <type_traits>

namespace chipmunk {

struct PackedParams : AttnParams {
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* cu_k;
    const int32_t* k_len;
    int64_t k_token, k_head, v_token, v_head;
    int Tk;
};

__device__ __forceinline__ Rows keys_of(const PackedParams& p, int s) {
    const int first = min(max(p.cu_k[s], 0), p.Tk);
    const int count = p.k_len ? p.k_len[s] : min(max(p.cu_k[s + 1], 0), p.Tk) - first;
    return Rows{first, min(min(max(count, 0), p.max_k), p.Tk - first)};
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

    store_rows<T, E, NQB>(st, limit, oh, p.out_token, w * NQB * 16, rows, g, l16);
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

    const bool alone = p.parts == 1 || ks.count <= p.part_keys;
    join_waves<T, E, NQB>(st, smem, w, lane, p.sl2, [&](int qb, const f32x4 (&o)[E / 64], float top, float total) {
        const int row = row0 + qb * 16 + l16;
        if (row < row0 + rows) store_joined<T, E>(p, s, head, part, qs.first, row, alone, limit[qb] > 0, w, g, o, top, total);
    });
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
    const bool sees = !p.causal || row / p.G + 1 + ks.count - qs.count > 0;
    join_parts<T, E>(p, s, head, row, qs.first, (ks.count - 1) / p.part_keys + 1, sees, lane);
}

template <class T, int E, int NQB>
static int32_t launch_rows(PackedParams p, hipStream_t stream) {
    constexpr int ROWS = 64 * NQB, LDS = 2 * kStepTiles * 2 * kTile * E * 2;
    const PackedGrid grid = rows_grid(ROWS, p.S, p.Tq, p.Hq, p.Hk, p.max_q);
    p.tiles = (int)grid.tiles;
    attn_packed_rows_kernel<T, E, NQB><<<(uint32_t)grid.workgroups, 256, LDS, stream>>>(p);
    return launch_status();
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
    const PackedParams p{{q, out, cu_q, q_token_stride, q_head_stride, out_token_stride, out_head_stride, S, Tq, Hq, Hk, Hq / Hk, std::min(max_q, Tq), std::min(max_k, Tk),
                          causal != 0, 0, 0, 0, 0, nullptr, sl2},
                         k, v, cu_k, k_len, k_token_stride, k_head_stride, v_token_stride, v_head_stride, Tk};
    const FewPlan few = few_plan_within(S, Hq, Hk, max_q, max_k, Tk);
    const auto st = static_cast<hipStream_t>(stream);
    if (dtype == CHIPMUNK_DTYPE_BF16) return E == 128 ? launch_packed<Bf16, 128>(p, few, ws, ws_bytes, st) : launch_packed<Bf16, 64>(p, few, ws, ws_bytes, st);
    return E == 128 ? launch_packed<Fp16, 128>(p, few, ws, ws_bytes, st) : launch_packed<Fp16, 64>(p, few, ws, ws_bytes, st);
}
