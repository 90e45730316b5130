// Attention of new tokens over sequences in pages (chipmunk_pages): one token of a sequence, a few or a chunk of them, causal or not, every key or
// a sliding window and the sequence's first keys; pages of 16 bits, or e4m3 whose rows are brought to the element type on their way to LDS, so that
// a form gives over codes bit by bit what it gives over the elements that they stand for (the prices of either may choose another form, whose sums
// are rounded elsewhere: 1 query over 900 keys, 32 heads over 8).
//
// The kernels are those of attention over packed sequences (attn_packed.hip, attn_tiles.h) with other keys: a workgroup walks a row of "numbered" keys,
// those that some of its rows may see, those first that all of them may (an online softmax has no order).  Where groups of 16 numbered keys
// begin is worked out from the table for 4096 of them at a time, and lies in LDS: a group is in one page, so a transfer's base is in scalar
// registers and its lanes' offsets never change.
#include "attn_tiles.h"
#include "pages.h"

#include <type_traits>

namespace chipmunk {

struct PagedParams : AttnParams {
    chipmunk_pages pages;
    const int32_t* table;
    const int32_t* k_len;
    int64_t table_row;       // stride of the table's rows
    int most_keys;           // of a sequence: by the limit and by the table
    int window, sinks;       // window 0: every key
    int shift;               // log2 of the page's tokens
    int block_rows;          // few queries: rows of a workgroup
};

constexpr int kGroup = 16;                    // keys that lie in one page, side by side
constexpr int kTableKeys = 4096;              // keys of a part of the table in LDS
constexpr int kTableGroups = kTableKeys / kGroup;

__device__ __forceinline__ int keys_held(const PagedParams& p, int s) { return min(max(p.k_len[s], 0), p.most_keys); }

// The first key that query i does not see, and the first of its window.
__device__ __forceinline__ int limit_of(const PagedParams& p, int i, int keys, int past) { return p.causal ? min(keys, i + 1 + past) : keys; }
__device__ __forceinline__ int low_of(const PagedParams& p, int i, int past) { return p.window ? max(max(i + 1 + past, 0) - p.window, 0) : 0; }

// The keys that the rows of queries first .. last walk, numbered from 0 in whole steps: from the first that is in every row's window (`high`) to the
// last; then the sequence's first ones, up to `sinks`; then from the first that is in any row's window (`low`) to `high`.
struct Walk {
    int sinks, end;                           // end: the first key that none of the rows sees
    int high, low, upto, edge, count;         // numbers below upto, below edge, of all
    __device__ __forceinline__ int key(int n) const { return n < upto ? high + n : n < edge ? n - upto : n - edge + low; }
};
template <int STEP>
__device__ __forceinline__ Walk walk_of(const PagedParams& p, int first, int last, int keys, int past) {
    auto whole = [](int n) { return (n + STEP - 1) / STEP * STEP; };
    Walk k;
    k.sinks = p.window ? min(p.sinks, keys) : 0;
    k.end = max(limit_of(p, last, keys, past), 0);
    k.high = min(whole(low_of(p, last, past)), whole(k.end));
    k.low = low_of(p, first, past) / STEP * STEP;
    int shown = whole(k.sinks);
    if (shown >= k.low) k.low = shown = 0;    // no gap behind the first ones
    k.upto = whole(k.end) - k.high;
    k.edge = k.upto + shown;
    k.count = k.edge + k.high - k.low;
    return k;
}

// Where a group of keys begins: bytes from the pages' first, bytes of its rows up to the last key (0: none), its keys; and its scales.
struct Place {
    u32x4 rows;
    u32x2 scales;
};
template <int E, bool CODES>
__device__ __forceinline__ Place place_of_group(const PagedParams& p, const Walk& walk, int s, int head, int n) {
    Place to{u32x4{0, 0, 0, 0}, u32x2{0, 0}};
    const int key = walk.key(n), rows = min(walk.end - key, kGroup);
    if (n >= walk.count || rows <= 0) return to;
    const int page = p.table[s * p.table_row + (key >> p.shift)], place = key & (p.pages.page_size - 1);
    if (page < 0 || page >= p.pages.pages) return to;
    constexpr int WIDTH = CODES ? 1 : 2;
    const uint64_t at = (page * p.pages.page_stride + place * p.pages.token_stride + head * p.pages.head_stride) * WIDTH;
    const uint64_t scales = page * p.pages.scale_page_stride + place * p.pages.scale_token_stride + head * p.pages.scale_head_stride;
    to.rows = u32x4{(uint32_t)at, (uint32_t)(at >> 32), (uint32_t)((rows - 1) * (int)p.pages.token_stride + E) * WIDTH, (uint32_t)rows};
    if (CODES) to.scales = u32x2{(uint32_t)scales, (uint32_t)(scales >> 32)};
    return to;
}
// The same in scalar registers; buffers over the rows: what lies behind them reads as zero.
struct Group {
    uint64_t at, scales;
    uint32_t bytes;
    int rows;
};
template <bool CODES>
__device__ __forceinline__ Group group_of(const u32x4* rows, const u32x2* scales, int i, bool there) {
    auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
    const u32x4 r = rows[i];
    Group g{(uint64_t)scalar(r[1]) << 32 | scalar(r[0]), 0, there ? scalar(r[2]) : 0u, 0};
    if (CODES) {
        const u32x2 c = scales[i];
        g.scales = (uint64_t)scalar(c[1]) << 32 | scalar(c[0]);
        g.rows = there ? (int)scalar(r[3]) : 0;
    }
    return g;
}

// Rows of codes in registers, on their way to a tile: NL loads of 16 codes a lane, ROWS_A_LOAD rows each.
template <int E, int NL>
struct Codes {
    static constexpr int LANES = E / 16, ROWS_A_LOAD = 64 / LANES;
    u32x4 code[NL];
    uint32_t scale[NL];
    // load i: rows first .. first + ROWS_A_LOAD of a group
    __device__ __forceinline__ void request(int i, const PagedParams& p, const void* base, const uint8_t* scales, const Group& g, int first, int lane) {
        const int row = first + lane / LANES;
        const int token = (int)p.pages.token_stride, scale_token = (int)p.pages.scale_token_stride;
        const auto rows = raw_buffer(static_cast<const uint8_t*>(base) + g.at, g.bytes);
        const auto bytes = raw_buffer(scales + g.scales, g.rows > 0 ? (uint32_t)((g.rows - 1) * scale_token + 1) : 0u);
        code[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, row * token + lane % LANES * 16, 0, 0));
        scale[i] = __builtin_amdgcn_raw_buffer_load_b8(bytes, row * scale_token, 0, 0);
    }
    // to row `row` of the tile at LDS address `tile`, as elements
    template <class T>
    __device__ __forceinline__ void put(int i, uint32_t tile, int row, int lane) const {
        const float power = __uint_as_float(scale[i] << 23);
        const int swizzle = tile_swizzle<E>(row);
#pragma unroll
        for (int c = 0; c < 2; c++) {
            const u32x2 a = elements_of_codes<T>(code[i][2 * c], power), b = elements_of_codes<T>(code[i][2 * c + 1], power);
            const uint32_t to = tile + (uint32_t)(row * E * 2 + (((lane % LANES * 2 + c) ^ swizzle) * 16));
            *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((uintptr_t)to) = u32x4{a[0], a[1], b[0], b[1]};
        }
    }
};

// The keys of a tile that a query does not see: from its limit on, and between the first ones and its window.
template <int NQB>
__device__ __forceinline__ void hide_far_keys(f32x4 (&S)[2][NQB], int first, const int (&low)[NQB], int sinks) {
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        const int from = low[qb] - first, shown = sinks - first;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                S[u][qb][r] = u * 16 + r < from && u * 16 + r >= shown ? -INFINITY : S[u][qb][r];
                asm volatile("" : "+v"(S[u][qb][r]));
            }
    }
}

// Adds the infinite and NaN values of 32 keys from key `first` on to the queries that see them (tile_values leaves them out where something
// is hidden).  Rare: the table is read from memory.
template <class T, int E, int NQB, bool CODES>
__device__ __forceinline__ void add_special_values(RowState<T, E, NQB>& st, const PagedParams& p, int s, int head, int first, int end, int sinks, const int (&limit)[NQB],
                                                   const int (&low)[NQB], int g) {
#pragma unroll 1
    for (int key = first; key < min(first + kTile, end); key++) {
        const int page = p.table[s * p.table_row + (key >> p.shift)];
        if (page < 0 || page >= p.pages.pages) continue;
        const int place = key & (p.pages.page_size - 1);
        const int64_t at = page * p.pages.page_stride + place * p.pages.token_stride + head * p.pages.head_stride + 4 * g;
        float power = 0.f;
        if (CODES) power = __uint_as_float((uint32_t)p.pages.v_scales[page * p.pages.scale_page_stride + place * p.pages.scale_token_stride + head * p.pages.scale_head_stride] << 23);
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) {
            u32x2 words;
            if constexpr (CODES) words = elements_of_codes<T>(*reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(p.pages.v) + at + eb * 16), power);
            else words = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(p.pages.v) + at + eb * 16);
#pragma unroll
            for (int r = 0; r < 4; r++) {
                float value = r % 2 ? T::high(words[r / 2]) : T::low(words[r / 2]);
                const bool special = not_finite<T>(words[r / 2]) & (r % 2 ? 0x80000000u : 0x8000u);
                asm volatile("" : "+v"(value));           // nothing is known of it, not even that it is none of the two
#pragma unroll
                for (int qb = 0; qb < NQB; qb++)
                    if (special && key < limit[qb] && (key >= low[qb] || key < sinks)) st.O[eb][qb][r] += value;
            }
        }
    }
}

// Few queries over many keys, as attn_packed_few_kernel: a workgroup owns one key head of one sequence and walks part_keys of its numbered keys for
// block_rows rows of the head; its waves take the tiles of 32 keys in turn and meet at the end.  Bound by the pages' bytes: 16 tokens over 1 to 32 011 keys
// each, 32 heads over 8 x 128, e4m3: 98 us (4.4 TB/s), where a launch's round trips (lengths, table, first tiles) and its parts' ends are some 10 of them;
// joining takes 6 us.  (64 rows of codes at E = 128 keep 22 registers in scratch memory: 64 queries over 2000 keys 26 us, of elements, in whole walks, 16.6.)
template <class T, int E, int NQB, bool CODES>
__global__ __launch_bounds__(256, NQB == 4 ? 1 : NQB == 1 && CODES ? 3 : 2) void attn_paged_few_kernel(PagedParams p) {
    typedef typename T::x8 x8;
    constexpr int ROWB = E * 2, CH = ROWB / 16, RPI = 64 / CH, NI = kTile / RPI;   // NI: transfers of a tile
    constexpr int NL = kTile * E / 1024;                  // loads of a tile's codes
    constexpr int TILE = kTile * ROWB, TILES = CODES ? 1 : 2, V_TILE = (TILES - 1) * TILE;   // of codes K and V go through one tile by turns
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    __shared__ u32x4 places[4][kWave];                    // of each wave's next 32 tiles' groups
    __shared__ u32x2 scale_places[CODES ? 4 : 1][kWave];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, l16 = lane & 15;
    int id = (int)(blockIdx.x / p.Hk);
    const int head = (int)blockIdx.x % p.Hk, part = id % p.parts;
    id /= p.parts;
    const int row0 = (p.tiles - 1 - id % p.tiles) * 16 * NQB, s = id / p.tiles;
    const Rows qs = queries_of(p, s);
    const int rows = min(16 * NQB, qs.count * p.G - row0);
    if (rows <= 0) return;
    const int keys = keys_held(p, s), past = keys - qs.count;
    const int i0 = row0 / p.G, i1 = (row0 + rows - 1) / p.G;
    const Walk walk = walk_of<kTile>(p, i0, i1, keys, past);
    const int low_of_all = low_of(p, i1, past);
    const int64_t start64 = (int64_t)part * p.part_keys;
    if (start64 >= walk.count && part > 0) return;        // (without any key the first part writes zeros)
    const int start = (int)start64, end = (int)std::min<int64_t>(walk.count, start64 + p.part_keys);

    constexpr int TURN = 4 * kTile;                       // keys from one tile of a wave to its next
    const int first = start + w * kTile;
    auto fill_table = [&](int n) {                        // the wave's tiles from numbered key n on
        const Place at = place_of_group<E, CODES>(p, walk, s, head, n + (lane >> 1) * TURN + (lane & 1) * kGroup);
        places[w][lane] = at.rows;
        if (CODES) scale_places[CODES ? w : 0][lane] = at.scales;
    };
    if (first < end) fill_table(first);                   // under way together with the queries

    RowState<T, E, NQB> st;
    int limit[NQB], low[NQB];                             // the first key that the lane's row does not see; the first of its window
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        st.negm[qb] = st.L[qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) st.O[eb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int row = row0 + min(qb * 16 + l16, rows - 1), i = row / p.G;   // (rows that are not there: the last one's)
        limit[qb] = limit_of(p, i, keys, past);
        low[qb] = low_of(p, i, past);
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
    const uint32_t smem_at = (uint32_t)(uintptr_t)CHIPMUNK_LDS_PTR(smem) + w * TILES * TILE;
    uint32_t kaddr[E / 32], vaddr[E / 16];
#pragma unroll
    for (int es = 0; es < E / 32; es++) kaddr[es] = smem_at + (uint32_t)(koff ^ (64 * es));
#pragma unroll
    for (int eb = 0; eb < E / 16; eb++) vaddr[eb] = smem_at + (uint32_t)(voff ^ (32 * eb));
    const uint32_t lds0 = lds_address(smem) + (uint32_t)(w * TILES * TILE);
    const int64_t token = p.pages.token_stride;
    constexpr int NIG = NI / 2;                           // transfers of a group: a lane's offsets into it stay the same
    uint32_t from[NIG];
#pragma unroll
    for (int i = 0; i < NIG; i++) {
        const int row = i * RPI + lane / CH;
        from[i] = (uint32_t)row * (uint32_t)(token * 2) + (uint32_t)(((lane % CH) ^ tile_swizzle<E>(row)) * 16);
    }
    auto group = [&](int n, int u) {                      // group u of the tile from numbered key n on; nothing behind the part's end
        return group_of<CODES>(places[w], scale_places[CODES ? w : 0], ((uint32_t)(n - first) / TURN % (kWave / 2)) * 2 + u, n < end);
    };
    Codes<E, NL> k_codes, v_codes;
    auto request = [&](const void* base, const uint8_t* scales, Codes<E, NL>& codes, int n, uint32_t to) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const Group at = group(n, u);
            if constexpr (CODES) {
                constexpr int ROWS = Codes<E, NL>::ROWS_A_LOAD;
#pragma unroll
                for (int i = u * NL / 2; i < (u + 1) * NL / 2; i++) codes.request(i, p, base, scales, at, i * ROWS % kGroup, lane);
            } else {
                const i32x4 buf = raw_buffer_words(static_cast<const uint8_t*>(base) + at.at, at.bytes);
#pragma unroll
                for (int i = 0; i < NIG; i++) load_buffer_to_lds_16B(buf, from[i], to + (u * NIG + i) * 1024);
            }
        }
    };
    auto put = [&](const Codes<E, NL>& codes, uint32_t tile) {
        constexpr int ROWS = Codes<E, NL>::ROWS_A_LOAD;
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < NL; i++) codes.template put<T>(i, tile, i * ROWS + lane / Codes<E, NL>::LANES, lane);
        asm volatile("" ::: "memory");                    // (a wave's LDS accesses are done in order)
    };
    auto request_k = [&](int n) {
        if ((uint32_t)(n - first) % (kWave / 2 * TURN) == 0 && n > first && n < end) fill_table(n);
        request(p.pages.k, p.pages.k_scales, k_codes, n, lds0);
    };
    auto request_v = [&](int n) { request(p.pages.v, p.pages.v_scales, v_codes, n, lds0 + V_TILE); };
    uint32_t found = 0;
    int n = first;
    auto tile = [&](auto hidden_c) {
        constexpr bool HIDDEN = decltype(hidden_c)::value;
        f32x4 S[2][NQB];
        if constexpr (CODES) {
            put(k_codes, lds0);
            request_k(n + TURN);
        } else {
            wait_vmem_at_most<NI>();                      // K has landed
            asm volatile("" ::: "memory");
        }
        tile_scores<T, E, NQB>(S, st, kaddr, 0, [](int) {});
        if constexpr (!CODES) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // and has been read
            request_k(n + TURN);
        }
        if (HIDDEN) {
            const int key = walk.key(n);
            hide_keys<NQB>(S, key + 4 * g, limit);
            if (key < low_of_all) hide_far_keys<NQB>(S, key + 4 * g, low, walk.sinks);
        }
        raise_reference<T, E, NQB>(st, S, p.sl2, slack);
        if constexpr (CODES) {
            put(v_codes, lds0 + V_TILE);
            request_v(n + TURN);
        } else {
            wait_vmem_at_most<NI>();                      // V
            asm volatile("" ::: "memory");
        }
        tile_values<T, E, NQB, HIDDEN>(st, S, vaddr, V_TILE, p.sl2, found);
        if constexpr (!CODES) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            request_v(n + TURN);
        }
    };
    if (n < end) {
        request_k(n);
        request_v(n);
    }
    // The queries, in registers now: no wait for them inside the loop
#pragma unroll
    for (int qb = 0; qb < NQB; qb++)
#pragma unroll
        for (int es = 0; es < E / 32; es++) asm volatile("" : "+v"(st.Q[es][qb]));
    const int plain_end = min(min(end, walk.upto), limit_of(p, i0, keys, past) - walk.high);
#pragma unroll 1
    for (; n + kTile <= plain_end; n += TURN) tile(std::false_type{});
    const int first_hidden = n;
#pragma unroll 1
    for (; n < end; n += TURN) tile(std::true_type{});
    wait_all_memory();
    if (__builtin_amdgcn_ballot_w64(found != 0) != 0)
        for (int at = first_hidden; at < end; at += TURN) add_special_values<T, E, NQB, CODES>(st, p, s, head, walk.key(at), walk.end, walk.sinks, limit, low, g);
    lds_accesses_then_barrier();                          // every wave is done with its tiles
    const bool alone = walk.count <= p.part_keys;
    join_waves<T, E, NQB>(st, smem, w, lane, p.sl2, [&](int qb, const f32x4 (&o)[E / 64], float top, float total) {
        const int row = row0 + qb * 16 + l16;
        if (row < row0 + rows) store_joined<T, E>(p, s, head, part, qs.first, row, alone, limit[qb] > 0, w, g, o, top, total);
    });
}

// Of rows in parts: the workspace's row of query i of sequence s and a head, [parts][Hq][S][max_q] rows of E sums, then as many references and sums.
__device__ __forceinline__ int64_t partial_row(const PagedParams& p, int part, int head, int s, int i) { return (((int64_t)part * p.Hq + head) * p.S + s) * p.max_q + i; }
template <int E>
__device__ __forceinline__ float* partial_stats(const PagedParams& p) { return p.partial + (int64_t)p.parts * p.Hq * p.S * p.max_q * E; }

// Rows, as attn_packed_rows_kernel: a workgroup of four waves owns 64 NQB consecutive queries of one sequence and head and walks its numbered keys in steps of
// two tiles of 32.  Elements go from the pages to LDS by asynchronous loads, double buffered by step; codes are in registers a step before, and go to LDS
// as elements while the step before theirs is computed.  Of few rows over many keys a workgroup walks part_keys of them (gridDim.y parts), and
// attn_paged_join_rows_kernel joins the parts.  Bound by the matrix pipes and the softmax beside them, as attn_packed_rows_kernel: chunks of 33 to 1024
// tokens over 1000 to 16 384 keys, 32 heads over 8 x 128: 386 to 408 us a pass; in passes of 437 us under the counters the matrix pipes are busy 51 % and
// the vector units 45 % of the time at 2.04 GHz.
template <class T, int E, int NQB, bool CODES>
__global__ __launch_bounds__(256, E == 64 ? 3 : 2) void attn_paged_rows_kernel(PagedParams p) {
    typedef typename T::x8 x8;
    constexpr int NWAVES = 4, ROWS = 16 * NQB * NWAVES;
    constexpr int ROWB = E * 2;                           // bytes per K/V row of a tile
    constexpr int CH = ROWB / 16, RPI = 64 / CH;          // 16-byte chunks per row; rows covered by one wave-wide load
    constexpr int NI = kTile / (RPI * NWAVES);            // such loads per wave, tile and matrix
    constexpr int TILE = kTile * ROWB, STAGE = 2 * TILE;  // K tile then V tile
    constexpr int NL = kStepKeys * E / 4096;              // loads of a step's codes per wave and matrix
    constexpr int NG = CODES ? NL : kStepTiles * NI;      // groups of a step that a wave fills rows of
    extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
    __shared__ u32x4 places[2 * kTableGroups];            // of two parts of the keys by turns
    __shared__ u32x2 scale_places[CODES ? 2 * kTableGroups : 1];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, l16 = lane & 15;

    int tile, head, s, part;
    tile_and_head(p, blockIdx.x, &tile, &head);
    if (tile >= p.tiles || !find_tile<ROWS>(p, tile, lane, &s, &part)) return;
    s = __builtin_amdgcn_readfirstlane(s);
    part = __builtin_amdgcn_readfirstlane(part);
    const Rows qs = queries_of(p, s);
    const int row0 = part * ROWS, rows = min(ROWS, qs.count - row0);
    if (rows <= 0) return;
    const int keys = keys_held(p, s), past = keys - qs.count;
    const Walk walk = walk_of<kStepKeys>(p, row0, row0 + rows - 1, keys, past);
    const int64_t begin64 = (int64_t)blockIdx.y * p.part_keys;
    if (begin64 >= walk.count && blockIdx.y > 0) return;  // (without any key the first part writes zeros)
    // The part's keys are numbered from 0 anew.
    const int begin = (int)begin64, count = (int)std::min<int64_t>(walk.count - begin, p.part_keys);
    const uint16_t* qh = p.q + head * p.q_head + (int64_t)(qs.first + row0) * p.q_token;
    uint16_t* oh = p.out + head * p.out_head + (int64_t)(qs.first + row0) * p.out_token;
    const int kv_head = head / p.G;

    RowState<T, E, NQB> st;
    int limit[NQB], low[NQB];
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        st.negm[qb] = st.L[qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) st.O[eb][qb] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int row = (w * NQB + qb) * 16 + l16, i = row0 + min(row, rows - 1);   // (rows that are not there: the last one's)
        limit[qb] = limit_of(p, i, keys, past);
        low[qb] = low_of(p, i, past);
#pragma unroll
        for (int es = 0; es < E / 32; es++) {
            u32x4 val = u32x4{0, 0, 0, 0};
            if (row < rows) val = *reinterpret_cast<const u32x4*>(qh + row * p.q_token + 32 * es + 8 * g);
            st.Q[es][qb] = __builtin_bit_cast(x8, val);
        }
    }
    // what all of a wave's rows see, and what any of them sees
    const int wave_row = w * NQB * 16, wave_rows = min(rows - wave_row, NQB * 16);
    const int first_row = row0 + wave_row, last_row = first_row + max(wave_rows, 1) - 1;
    const int seen = wave_rows <= 0 ? 0 : limit_of(p, last_row, keys, past), low_of_any = low_of(p, first_row, past);
    const int seen_by_all = wave_rows <= 0 ? 0 : limit_of(p, first_row, keys, past), low_of_all = low_of(p, last_row, past);
    const int plain_end = min(count, min(walk.upto, seen_by_all - walk.high) - begin);
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
    const uint32_t lds0 = lds_address(smem);
    const int64_t token = p.pages.token_stride;

    // Elements: load (n, i) of a wave fills rows (i * NWAVES + w) * RPI .. of tile n, which are in group 2 n + i (E = 128) or 2 n + w / 2 of the step.
    // Codes: load i fills rows of group 2 i + w / 2 (E = 128), or of group w.
    auto group_at = [&](int n) { return E == 128 ? (CODES ? 2 * n + (w >> 1) : n) : (CODES ? w : 2 * n + (w >> 1)); };
    constexpr int ROWS_A_LOAD = CODES ? Codes<E, NL>::ROWS_A_LOAD : RPI;
    const int in_group = w * ROWS_A_LOAD % kGroup;        // of the load's first row
    const int row_of_lane = in_group + lane / CH;
    const uint32_t from = (uint32_t)row_of_lane * (uint32_t)(token * 2) + (uint32_t)(((lane % CH) ^ tile_swizzle<E>(row_of_lane)) * 16);   // (elements)
    Group at[NG];                                         // of the step that is requested next
    auto next_step = [&](int n) {
#pragma unroll
        for (int i = 0; i < NG; i++) at[i] = group_of<CODES>(places, scale_places, ((uint32_t)n / kGroup + group_at(i)) % (2 * kTableGroups), n < count);
    };
    auto fill_table = [&](int n) {                        // the part of the keys from n on
        const int i = (uint32_t)n / kGroup % (2 * kTableGroups) + tid;
        const Place to = place_of_group<E, CODES>(p, walk, s, kv_head, begin + n + tid * kGroup);
        places[i] = to.rows;
        if (CODES) scale_places[CODES ? i : 0] = to.scales;
    };
    static_assert(kTableGroups == 256, "one group to a thread");
    // Codes of the next SETS steps are under way: a step of narrow heads is shorter than memory takes; wide ones have no registers for two.
    constexpr int SETS = CODES && E == 64 ? 2 : 1;
    Codes<E, CODES ? NL : 1> k_codes[SETS], v_codes[SETS];
    auto request = [&](int half, int j) {
        const int n = j / (2 * NI), i = (j / 2) % NI;
        const uint32_t to = lds0 + (uint32_t)((half * kStepTiles + n) * STAGE + (i * NWAVES + w) * 1024);
        const Group& from_group = at[CODES ? 0 : n * NI + i];
        if (j & 1) load_buffer_to_lds_16B(raw_buffer_words(static_cast<const uint8_t*>(p.pages.v) + from_group.at, from_group.bytes), from, to + TILE);
        else load_buffer_to_lds_16B(raw_buffer_words(static_cast<const uint8_t*>(p.pages.k) + from_group.at, from_group.bytes), from, to);
    };
    static_assert(kStepTiles * NI * 2 == E / 16, "one transfer per group of score products");
    auto request_codes = [&](auto set_c) {
        if constexpr (CODES) {
            constexpr int set = decltype(set_c)::value % SETS;
#pragma unroll
            for (int i = 0; i < NL; i++) {
                k_codes[set].request(i, p, p.pages.k, p.pages.k_scales, at[i], in_group, lane);
                v_codes[set].request(i, p, p.pages.v, p.pages.v_scales, at[i], in_group, lane);
            }
        }
    };
    auto put_codes = [&](auto set_c, int half) {
        if constexpr (CODES) {
            constexpr int set = decltype(set_c)::value % SETS;
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < NL; i++) {
                const int row = group_at(i) * kGroup + in_group + lane / Codes<E, NL>::LANES;   // of the step
                const uint32_t to = lds0 + (uint32_t)((half * kStepTiles + group_at(i) / 2) * STAGE);
                k_codes[set].template put<T>(i, to, row % kTile, lane);
                v_codes[set].template put<T>(i, to + TILE, row % kTile, lane);
            }
            asm volatile("" ::: "memory");
        }
    };
    typedef std::integral_constant<int, 0> Even;
    typedef std::integral_constant<int, 1> Odd;

    if (count > 0) {
        fill_table(0);
        if (count > kTableKeys) fill_table(kTableKeys);
        wait_all_memory();                                // no wait for the queries inside the loop
        __syncthreads();
        next_step(0);
        if constexpr (CODES) {
            request_codes(Even{});
            if (SETS == 2) {
                next_step(kStepKeys);
                request_codes(Odd{});
            }
            put_codes(Even{}, 0);
            next_step(SETS * kStepKeys);
            request_codes(std::integral_constant<int, SETS>{});
        } else {
#pragma unroll
            for (int j = 0; j < E / 16; j++) request(0, j);
        }
    }
    // Begins the step from numbered key n on, whose tiles are in half `half`.  (set: of the step behind it, whose parity is the other half's)
    auto arrived = [&](auto set_c, int half, int n) {
        if constexpr (CODES) lds_accesses_then_barrier();  // the codes stay under way
        else wait_all_memory(), __syncthreads();          // this step's tiles have landed for every wave; the other half is free
        if ((uint32_t)n % kTableKeys == 0 && n > 0 && n + kTableKeys < count) fill_table(n + kTableKeys);   // (many barriers before its first use)
        if constexpr (CODES) {
            put_codes(set_c, half ^ 1);
            next_step(n + (SETS + 1) * kStepKeys);
            request_codes(set_c);
        } else {
            next_step(n + kStepKeys);
        }
    };
    // The steps whose keys all of the wave's rows see, in two copies, whose LDS offsets are constants; then those with hidden keys.
    // Waves may stand in different loops: each step of each is one barrier.
    uint32_t found = 0;
    auto step = [&](auto half_c, int n) {
        constexpr int half = decltype(half_c)::value;
        arrived(std::integral_constant<int, half ^ 1>{}, half, n);
#pragma unroll
        for (int t = 0; t < kStepTiles; t++) {
            const int tile_off = (half * kStepTiles + t) * STAGE;
            f32x4 S[2][NQB];
            if (t == 0 && !CODES) tile_scores<T, E, NQB>(S, st, kaddr, tile_off, [&](int j) { request(half ^ 1, j); });
            else tile_scores<T, E, NQB>(S, st, kaddr, tile_off, [](int) {});
            raise_reference<T, E, NQB>(st, S, p.sl2, slack);
            tile_values<T, E, NQB, false>(st, S, vaddr, tile_off + TILE, p.sl2, found);
        }
    };
    auto nothing_seen = [&](int key) { return key >= seen || (key + kStepKeys <= low_of_any && key >= walk.sinks); };   // by this wave's rows
    auto hidden_step = [&](auto set_c, int half, int n, int base) {   // base: what the addresses lack
        arrived(set_c, half, n);
        if constexpr (!CODES) {
#pragma unroll
            for (int j = 0; j < E / 16; j++) request(half ^ 1, j);
        }
        const int key = walk.key(begin + n);
        if (nothing_seen(key)) return;
#pragma unroll
        for (int t = 0; t < kStepTiles; t++) {
            f32x4 S[2][NQB];
            tile_scores<T, E, NQB>(S, st, kaddr, base + t * STAGE, [](int) {});
            if (key + kStepKeys > seen_by_all) hide_keys<NQB>(S, key + t * kTile + 4 * g, limit);
            if (key < low_of_all) hide_far_keys<NQB>(S, key + t * kTile + 4 * g, low, walk.sinks);
            raise_reference<T, E, NQB>(st, S, p.sl2, slack);
            tile_values<T, E, NQB, true>(st, S, vaddr, base + t * STAGE + TILE, p.sl2, found);
        }
    };
    // (codes: an even number, so that the steps behind them are in pairs as well, which takes fewer registers)
    const int plain_keys = CODES ? plain_end / (2 * kStepKeys) * (2 * kStepKeys) : plain_end;
    int n = 0;
#pragma unroll 1
    while (n + kStepKeys <= plain_keys) {
        step(Even{}, n);
        n += kStepKeys;
        if (n + kStepKeys > plain_keys) break;
        step(Odd{}, n);
        n += kStepKeys;
    }
    const int first_hidden = n;
    if constexpr (CODES) {
#pragma unroll 1
        while (n < count) {
            hidden_step(Odd{}, 0, n, 0);
            n += kStepKeys;
            if (n >= count) break;
            hidden_step(Even{}, 1, n, kStepTiles * STAGE);
            n += kStepKeys;
        }
    } else {
        auto move = [&](int bytes) {                      // the addresses to the other half
#pragma unroll
            for (int es = 0; es < E / 32; es++) kaddr[es] += bytes;
#pragma unroll
            for (int eb = 0; eb < E / 16; eb++) vaddr[eb] += bytes;
        };
        int half = n / kStepKeys & 1;
        move(half * kStepTiles * STAGE);
#pragma unroll 1
        for (; n < count; n += kStepKeys, half ^= 1) {
            hidden_step(Even{}, half, n, 0);
            move(half ? -kStepTiles * STAGE : kStepTiles * STAGE);
        }
    }
    wait_all_memory();                                    // the transfers behind the last step

    // Infinite and NaN values among the steps with hidden keys go to the queries that see them.
    if (__builtin_amdgcn_ballot_w64(found != 0) != 0)
#pragma unroll 1
        for (int at = first_hidden; at < count; at += kTile) {
            const int key = walk.key(begin + at);
            if (!nothing_seen(key / kStepKeys * kStepKeys)) add_special_values<T, E, NQB, CODES>(st, p, s, kv_head, key, walk.end, walk.sinks, limit, low, g);
        }
    if (walk.count <= p.part_keys) {
        store_rows<T, E, NQB>(st, limit, oh, p.out_token, w * NQB * 16, rows, g, l16);
        return;
    }
#pragma unroll
    for (int qb = 0; qb < NQB; qb++) {
        const int row = (w * NQB + qb) * 16 + l16;
        if (row >= rows) continue;
        const int64_t to = partial_row(p, blockIdx.y, head, s, row0 + row);
#pragma unroll
        for (int eb = 0; eb < E / 16; eb++) *reinterpret_cast<f32x4*>(p.partial + to * E + eb * 16 + 4 * g) = st.O[eb][qb];
        if (g == 0) *reinterpret_cast<f32x2*>(partial_stats<E>(p) + to * 2) = f32x2{st.L[qb][0] == 0.f ? -INFINITY : -st.negm[qb][0], st.L[qb][0]};
    }
}

// Joins the parts of the rows that have more than one: a wave per row.
template <class T, int E>
__global__ __launch_bounds__(256) void attn_paged_join_kernel(PagedParams p) {
    const int lane = threadIdx.x & 63, row = (int)blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s = blockIdx.x / p.Hk, head = blockIdx.x % p.Hk;
    if (row >= p.few_rows) return;
    const Rows qs = queries_of(p, s);
    if (row >= qs.count * p.G) return;
    const int keys = keys_held(p, s), past = keys - qs.count;
    const int row0 = row / p.block_rows * p.block_rows, rows = min(p.block_rows, qs.count * p.G - row0);   // the workgroup's that had it
    const Walk walk = walk_of<kTile>(p, row0 / p.G, (row0 + rows - 1) / p.G, keys, past);
    if (walk.count <= p.part_keys) return;
    join_parts<T, E>(p, s, head, row, qs.first, min((walk.count - 1) / p.part_keys + 1, p.parts), limit_of(p, row / p.G, keys, past) > 0, lane);
}

// The same of the rows kernel's parts: a wave per query and head.  block_rows: the rows that walked together.
template <class T, int E>
__global__ __launch_bounds__(256) void attn_paged_join_rows_kernel(PagedParams p) {
    const int lane = threadIdx.x & 63, id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.y;
    const int i = id % p.max_q, s = id / p.max_q;
    if (s >= p.S) return;
    const Rows qs = queries_of(p, s);
    if (i >= qs.count) return;
    const int keys = keys_held(p, s), past = keys - qs.count, first = i / p.block_rows * p.block_rows;
    const Walk walk = walk_of<kStepKeys>(p, first, min(first + p.block_rows, qs.count) - 1, keys, past);
    if (walk.count <= p.part_keys) return;
    const int64_t at = partial_row(p, 0, head, s, i);
    join_parts<T, E>(p.partial + at * E, partial_stats<E>(p) + at * 2, (int64_t)p.Hq * p.S * p.max_q, min((walk.count - 1) / p.part_keys + 1, p.parts), p.sl2,
                     limit_of(p, i, keys, past) > 0, p.out + (int64_t)(qs.first + i) * p.out_token + head * p.out_head, lane);
}

// The numbered keys that a workgroup has at most: its rows' queries, at most max_q of them, see as many more than a window, in whole steps.
static int most_numbered(int max_q, int max_k, int window, int sinks) {
    if (window == 0) return max_k;
    const int64_t most = (int64_t)window + max_q + sinks + 3 * kStepKeys;   // (the window, the first keys and the last in whole steps)
    return (int)std::min<int64_t>(most, max_k);
}

// Up to 1024 rows of a key head may walk their n numbered keys in parts, whose length goes by its price.  A part of codes takes half the time to begin and end
// that one of elements does.  Measured on 4009 batches of up to 32 rows (1 to 128 sequences of 300 to 40 000 keys, ragged and not): parts or whole, and
// their length, take 1.03 times the quickest's time in the mean, of codes and of elements (by the rules of packed attention 1.06 and 1.04).  More rows
// have their price beside whole_plan's.
struct PartsPlan {
    FewPlan few;              // rows 0: none
    double price;             // us; of more than 32 rows
};
struct PartsPrice {
    float start, keys, join, join_block, share;   // of a launch; 64 keys of 64 rows; a part's joining, for each block of 64 rows; workgroups that have work
};
constexpr PartsPrice kPartsPrices[2][2] = {{{6.5f, 0.615f, 0.074f, 0.0074f, 1.47f}, {16.3f, 0.567f, 0.167f, 0.0035f, 1.65f}},   // elements: E = 64, 128
                                           {{8.8f, 0.423f, 0.092f, 0.006f, 1.4f}, {8.1f, 0.8f, 0.17f, 0.004f, 1.59f}}};         // codes
constexpr int64_t kMostPartRows = 1 << 19;    // rows of all parts in the workspace, of more than 32 rows (272 MB at E = 128)
static PartsPlan parts_plan(int S, int Hq, int Hk, int E, int max_q, int n, bool codes) {
    const PartsPlan none{FewPlan{0, 0, 0}, HUGE_VAL};
    const int64_t rows = (int64_t)max_q * (Hq / Hk), heads = (int64_t)S * Hk;
    if (rows > 1024 || heads > kMostPartWorkgroups / 2) return none;
    const bool few = rows <= 32;
    if (few && n <= (codes ? std::min<int64_t>(700 + 4 * heads, 3000) : std::min<int64_t>(1000 + 15 * heads, 3000))) return none;
    const int64_t blocks = heads * ((rows + 63) / 64);
    const PartsPrice& f = kPartsPrices[codes][E == 128];
    PartsPlan best = none;
    for (int length : {256, 512, 768, 1024, 1536, 2048, 4096}) {
        const int64_t workgroups = blocks * parts_of(n, length);
        const double parts = (double)n / length;
        double price;
        if (few) price = codes ? length + parts * (17.0 + 0.3 * (double)heads)
                               : length * (workgroups > 256 && workgroups < 2048 ? 2.0 : 1.0) + parts * (30.0 + 0.7 * (double)heads);
        else price = f.start + length / 64.0 * f.keys * std::max(1.0, (double)workgroups * f.share / 256) + parts * (f.join + f.join_block * (double)blocks);
        if (!few && (length < 512 || heads * parts_of(n, length) * rows > kMostPartRows)) continue;
        if (best.few.rows == 0 || price < best.price) best = PartsPlan{FewPlan{(int)rows, length, parts_of(n, length)}, price};
    }
    // (a limit may be far above the lengths: the parts grow with it)
    while (best.few.rows > 0 && blocks * best.few.parts > kMostPartWorkgroups) {
        best.few.part_keys *= 2;
        best.few.parts = parts_of(n, best.few.part_keys);
    }
    return best;
}
// The plan for `there` of n keys, with no more parts than the workspace of n has room for.
static PartsPlan parts_plan_within(int S, int Hq, int Hk, int E, int max_q, int n, int there, bool codes) {
    const PartsPlan given = parts_plan(S, Hq, Hk, E, max_q, n, codes);
    if (given.few.rows == 0 || n <= there) return given;
    PartsPlan plan = parts_plan(S, Hq, Hk, E, max_q, there, codes);
    while (plan.few.parts > given.few.parts) {
        plan.few.part_keys *= 2;
        plan.few.parts = parts_of(there, plan.few.part_keys);
    }
    return plan;
}

// Whole sequences, as packed_price has it, fitted to the 5294 batches.  (192 rows were the quickest in 22 of them, and twice as slow as 128 of codes at
// E = 128, whose registers they pass; there are none here.)
constexpr int kPagedForms = kRows192;
constexpr PackedPrice kPagedPrices[2][2][kPagedForms] = {
    {{{16, 3.7f, 0.17f, 0.58f}, {32, 6.1f, 0.25f, 0.29f}, {64, 3.1f, 0.9f, 0.32f}, {128, 5.9f, 1.31f, 0.246f}},
     {{16, 5.f, 0.165f, 1.72f}, {32, 8.f, 0.45f, 0.58f}, {64, 5.1f, 0.85f, 0.64f}, {128, 7.f, 1.32f, 0.18f}}},
    {{{16, 3.5f, 0.31f, 0.745f}, {32, 6.1f, 0.33f, 0.37f}, {64, 3.1f, 1.01f, 0.45f}, {128, 4.8f, 1.04f, 0.24f}},
     {{16, 2.7f, 0.36f, 1.78f}, {32, 6.9f, 0.39f, 0.72f}, {64, 5.9f, 0.84f, 0.61f}, {128, 5.85f, 1.18f, 0.38f}}}};
constexpr float kPagedLast[2][2] = {{0.25f, 0.53f}, {0.235f, 0.56f}};
// Rows of a head in parts of their keys: few of them over many keys leave CUs without work (one chunk of 512 tokens, 32 heads, over 32 768 keys: 430 us whole).
// Joined are Tq Hq rows, from 1 MB of sums on by their size.  Over 1581 batches of 40 to 2048 queries of 1 to 4 sequences over 1500 to 60 000 keys what
// is taken, whole, rows or a key head's rows in parts, takes 1.05 (E = 64) and 1.07 times the quickest's time in the mean; without rows in parts 1.17 to 1.22.
struct RowPartsPrice {
    PackedPrice forms[2];     // 64 and 128 rows
    float last, join, join_mb;
};
constexpr RowPartsPrice kRowPartsPrices[2][2] = {{{{{64, 1.96f, 0.9f, 0.295f}, {128, 3.63f, 2.08f, 0.141f}}, 0.124f, 4.2f, 0.116f},     // elements: E = 64, 128
                                                  {{{64, 8.4f, 0.86f, 0.61f}, {128, 7.8f, 1.97f, 0.242f}}, 0.66f, 6.f, 0.25f}},
                                                 {{{{64, 2.4f, 0.84f, 0.33f}, {128, 2.f, 1.3f, 0.242f}}, 0.089f, 2.8f, 0.26f},          // codes
                                                  {{{64, 5.9f, 0.84f, 0.61f}, {128, 3.9f, 1.49f, 0.387f}}, 0.63f, 4.8f, 0.165f}}};
constexpr int64_t kMostRowPartBytes = 64 << 20;
// (By S * max_q, whether or not the sequences have so many: the workspace is asked for without the number of queries that there are, and a part's rows are
// found by their sequence.  So a chunk beside other sequences' single tokens has room for fewer parts than alone, or for none: 512 queries over 32 768
// keys 296 us, with one token over as many beside it 323, with three 784, where the three by themselves take 86.)
constexpr int kLeastRowPart = 512, kMostRowParts = 16;   // keys; parts
static int64_t row_part_bytes(int S, int Hq, int E, int max_q) { return (int64_t)S * Hq * max_q * (E + 2) * (int64_t)sizeof(float); }
// The parts that there may be, by the room for their sums, by the keys and by the CUs, of any number of queries within the limits.
static int most_row_parts(int S, int Hq, int E, int max_q, int n) {
    if ((int64_t)S * max_q > (1 << 20) || Hq > (1 << 12) || max_q < 32) return 1;
    const int64_t workgroups = (int64_t)((max_q + 127) / 128) * Hq;   // of one sequence
    return (int)std::max<int64_t>(1, std::min<int64_t>({kMostRowParts, n / kLeastRowPart, 1024 / workgroups, kMostRowPartBytes / row_part_bytes(S, Hq, E, max_q)}));
}
struct WholePlan {
    PackedForm form;
    int parts;                // of the rows' forms
    double price;             // HUGE_VAL: no form's launch covers it
};
static WholePlan whole_plan(int S, int64_t Tq, int Hq, int Hk, int E, int max_q, int n, int causal, bool codes, int most_parts) {
    WholePlan best{kKeys16, 1, HUGE_VAL};
    for (int f = 0; f < kPagedForms; f++) {
        const double price = form_price((PackedForm)f, kPagedPrices[codes][E == 128][f], kPagedLast[codes][E == 128], S, Tq, Hq, Hk, max_q, n, causal);
        if (price < best.price) best = WholePlan{(PackedForm)f, 1, price};
    }
    const RowPartsPrice& r = kRowPartsPrices[codes][E == 128];
    for (int f = kRows64; f < kPagedForms; f++)
        for (int parts : {2, 3, 4, 6, 8, 12, 16}) {
            if (parts > most_parts) break;
            const double price = form_price((PackedForm)f, r.forms[f - kRows64], r.last, S, Tq, Hq, Hk, max_q, n, causal, parts) + r.join +
                                 (double)Tq * Hq * parts * E * 8 / 1e6 * r.join_mb;
            if (price < best.price) best = WholePlan{(PackedForm)f, parts, price};
        }
    return best;
}
static bool in_parts(const PartsPlan& parts, const WholePlan& whole) { return parts.few.rows > 0 && (parts.few.rows <= 32 || parts.price < whole.price); }

template <class T, int E, int NQB, bool CODES>
static int32_t launch_paged_rows(PagedParams p, hipStream_t stream) {
    constexpr int ROWS = 64 * NQB, LDS = 2 * kStepTiles * 2 * kTile * E * 2;
    const auto kernel = attn_paged_rows_kernel<T, E, NQB, CODES>;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    const PackedGrid grid = rows_grid(ROWS, p.S, p.Tq, p.Hq, p.Hk, p.max_q);
    p.tiles = (int)grid.tiles;
    p.block_rows = ROWS;
    kernel<<<dim3((uint32_t)grid.workgroups, (uint32_t)p.parts), 256, LDS, stream>>>(p);
    if (p.parts > 1) attn_paged_join_rows_kernel<T, E><<<dim3((uint32_t)(((int64_t)p.S * p.max_q + 3) / 4), (uint32_t)p.Hq), 256, 0, stream>>>(p);
    return launch_status();
}

template <class T, int E, int NQB, bool CODES>
static int32_t launch_paged_few(PagedParams p, hipStream_t stream) {
    constexpr int TOGETHER = NQB < 2 ? NQB : 2;
    constexpr int LDS = std::max(4 * (CODES ? 1 : 2) * kTile * E * 2, 4 * TOGETHER * (E * 64 + 512));
    const auto kernel = attn_paged_few_kernel<T, E, NQB, CODES>;
    const PackedGrid grid = few_grid(16 * NQB, p.S, p.Hk, p.few_rows, p.parts);
    if (grid.workgroups >= kMostWorkgroups) return CHIPMUNK_ERR_SHAPE;
    if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return CHIPMUNK_ERR_LAUNCH;
    p.tiles = (int)grid.tiles;
    p.block_rows = 16 * NQB;
    kernel<<<(uint32_t)grid.workgroups, 256, LDS, stream>>>(p);
    if (p.parts > 1) attn_paged_join_kernel<T, E><<<dim3((uint32_t)(p.S * p.Hk), (uint32_t)(p.few_rows + 3) / 4), 256, 0, stream>>>(p);
    return launch_status();
}

template <class T, int E, bool CODES>
static int32_t launch_paged(PagedParams p, const PartsPlan& parts, int most_parts, int n, void* ws, size_t ws_bytes, hipStream_t stream) {
    const WholePlan whole = whole_plan(p.S, p.Tq, p.Hq, p.Hk, E, p.max_q, n, p.causal, CODES, most_parts);
    if (in_parts(parts, whole)) {
        const FewPlan& few = parts.few;
        if (few_bytes(few, p.S, p.Hk, E) > (ws ? ws_bytes : 0)) return CHIPMUNK_ERR_WORKSPACE;
        p.few_rows = few.rows;
        p.part_keys = few.part_keys;
        p.parts = few.parts;
        p.partial = static_cast<float*>(ws);
        return few.rows <= 16   ? launch_paged_few<T, E, 1, CODES>(p, stream)
               : few.rows <= 32 ? launch_paged_few<T, E, 2, CODES>(p, stream)
                                : launch_paged_few<T, E, 4, CODES>(p, stream);
    }
    if (whole.price == HUGE_VAL) return CHIPMUNK_ERR_SHAPE;
    p.few_rows = p.max_q * p.G;
    p.part_keys = INT32_MAX;
    p.parts = whole.parts;
    if (p.parts > 1) {
        if ((size_t)(row_part_bytes(p.S, p.Hq, E, p.max_q) * p.parts) > (ws ? ws_bytes : 0)) return CHIPMUNK_ERR_WORKSPACE;
        p.part_keys = (int)(((int64_t)n + (int64_t)p.parts * kStepKeys - 1) / ((int64_t)p.parts * kStepKeys) * kStepKeys);   // (whole steps)
        p.partial = static_cast<float*>(ws);
    }
    switch (whole.form) {
        case kKeys16: return launch_paged_few<T, E, 1, CODES>(p, stream);
        case kKeys32: return launch_paged_few<T, E, 2, CODES>(p, stream);
        case kRows64: return launch_paged_rows<T, E, 1, CODES>(p, stream);
        default: return launch_paged_rows<T, E, 2, CODES>(p, stream);
    }
}

}  // namespace chipmunk

using namespace chipmunk;


// The form that a call takes, with ten times its further parts, or the keys of a key head's parts, for the tests.
extern "C" int chipmunk_internal_attn_paged_form(int S, int Tq, int Hq, int Hk, int E, int max_q, int max_k, int causal, int window, int sinks, int codes) {
    const int n = most_numbered(max_q, max_k, window, sinks);
    const PartsPlan parts = parts_plan(S, Hq, Hk, E, max_q, n, codes != 0);
    const WholePlan whole = whole_plan(S, Tq, Hq, Hk, E, std::min(max_q, Tq), n, causal, codes != 0, most_row_parts(S, Hq, E, max_q, n));
    return in_parts(parts, whole) ? parts.few.part_keys : whole.form + 10 * (whole.parts - 1);
}

extern "C" size_t chipmunk_attn_paged_workspace_bytes(int S, int Hq, int Hk, int E, int max_q, int max_k, int window, int sinks) {
    if (S <= 0 || Hq <= 0 || Hk <= 0 || Hq % Hk != 0 || (E != 64 && E != 128) || max_q <= 0 || max_k <= 0 || window < 0 || sinks < 0) return 0;
    const int n = most_numbered(max_q, max_k, window, sinks);   // (of either format)
    const int rows = most_row_parts(S, Hq, E, max_q, n);
    return std::max({few_bytes(parts_plan(S, Hq, Hk, E, max_q, n, false).few, S, Hk, E), few_bytes(parts_plan(S, Hq, Hk, E, max_q, n, true).few, S, Hk, E),
                     rows > 1 ? (size_t)(row_part_bytes(S, Hq, E, max_q) * rows) : 0});
}

extern "C" int32_t chipmunk_attn_paged(const uint16_t* q, int64_t q_token_stride, int64_t q_head_stride, const chipmunk_pages* pages, const int32_t* table,
                                       int64_t table_stride, int table_pages, uint16_t* out, int64_t out_token_stride, int64_t out_head_stride, const int32_t* cu_q,
                                       const int32_t* k_len, int S, int Tq, int Hq, int max_q, int max_k, int causal, int window, int sinks, float softmax_scale,
                                       int dtype, void* ws, size_t ws_bytes, void* stream) {
    if (!q || !pages || !table || !out || !cu_q || !k_len) return CHIPMUNK_ERR_NULL;
    chipmunk_pages held = *pages;
    const int32_t status = check_pages(held, dtype);
    if (status != CHIPMUNK_OK) return status;
    const int Hk = held.heads, E = held.E;
    if (S <= 0 || Tq <= 0 || Hq <= 0 || Hq % Hk != 0 || max_q <= 0 || max_k <= 0 || table_pages <= 0 || window < 0 || sinks < 0 || (window > 0 && !causal)) return CHIPMUNK_ERR_SHAPE;
    if ((int64_t)table_pages * held.page_size > (1 << 30)) return CHIPMUNK_ERR_SHAPE;
    const float sl2 = softmax_scale * 1.4426950408889634f;
    if (!is_positive_finite_scalar(softmax_scale) || !is_finite_scalar(sl2)) return CHIPMUNK_ERR_SHAPE;
    constexpr int64_t kMostStride = 1 << 24;
    if (Tq == 1) q_token_stride = out_token_stride = E;   // of one row alone a stride means nothing
    if (S == 1) table_stride = table_pages;
    for (int64_t token : {q_token_stride, out_token_stride})
        if (token < E || token >= kMostStride) return CHIPMUNK_ERR_SHAPE;
    if (table_stride < table_pages || (Hq > 1 && (q_head_stride < E || out_head_stride < E))) return CHIPMUNK_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(out) || !aligned16(ws) ||
        ((reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(k_len) | reinterpret_cast<uintptr_t>(table)) & 3) ||
        (q_token_stride | out_token_stride) % 8 != 0 || (Hq > 1 && (q_head_stride | out_head_stride) % 8 != 0))
        return CHIPMUNK_ERR_ALIGN;
    const int most_keys = std::min(max_k, table_pages * held.page_size);
    const int given = most_numbered(max_q, max_k, window, sinks);   // as the workspace was asked for
    if (window >= most_keys) window = 0;                  // (which every query sees whole)
    PagedParams p{{q, out, cu_q, q_token_stride, q_head_stride, out_token_stride, out_head_stride, S, Tq, Hq, Hk, Hq / Hk, std::min(max_q, Tq), most_keys, causal != 0, 0, 0, 0, 0,
                   nullptr, sl2},
                  held, table, k_len, table_stride, most_keys, window, window ? sinks : 0, __builtin_ctz((uint32_t)held.page_size), 0};
    const int planned = most_numbered(max_q, most_keys, window, sinks);
    const PartsPlan parts = parts_plan_within(S, Hq, Hk, E, max_q, given, planned, held.format == CHIPMUNK_DTYPE_E4M3);
    const int most_parts = std::min(most_row_parts(S, Hq, E, max_q, given), std::max(1, planned / kLeastRowPart));
    const auto st = static_cast<hipStream_t>(stream);
    auto go = [&](auto type, auto width) {
        typedef decltype(type) T;
        constexpr int W = decltype(width)::value;
        return held.format == CHIPMUNK_DTYPE_E4M3 ? launch_paged<T, W, true>(p, parts, most_parts, planned, ws, ws_bytes, st) : launch_paged<T, W, false>(p, parts, most_parts, planned, ws, ws_bytes, st);
    };
    typedef std::integral_constant<int, 64> Narrow;
    typedef std::integral_constant<int, 128> Wide;
    if (dtype == CHIPMUNK_DTYPE_BF16) return E == 128 ? go(Bf16{}, Wide{}) : go(Bf16{}, Narrow{});
    return E == 128 ? go(Fp16{}, Wide{}) : go(Fp16{}, Narrow{});
}
