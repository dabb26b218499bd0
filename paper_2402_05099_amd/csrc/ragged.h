// Attention of packed tokens of several sequences, each with its own number of new tokens and of keys: whole prompts
// (hg_prompt_attn) and chunks behind a paged cache (hg_chunk_attn_paged).  Arguments and what the kernels share (gfx950 only).
#pragma once
#include "hg_internal.h"

namespace hg {

// Sequence b owns the tokens [q_off[b], q_off[b + 1]) of Q and O; the query rows of one of its KV heads are numbered r = t * G + g
// (token t, head g of the group).  Token t of n sees keys [0, len - (n - 1 - t)), len = lengths[b], or n where lengths is null: the keys
// are then the sequence's own tokens' rows of K and V.
struct RaggedArgs {
    const uint16_t* Q;
    const unsigned char* K;   // packed rows, or the page pool
    const unsigned char* V;
    int64_t q_stride;         // bytes between consecutive tokens of Q
    int64_t kv_stride;        // bytes between consecutive rows of K and of V
    const int32_t* q_off;     // [B + 1], non-decreasing
    const int32_t* lengths;   // [B], or null
    PagedDev pg;              // pg.table != null where lengths is
    int rows;                 // tokens in Q and O
    int B, Hq, Hkv, G;
    int max_new;              // tokens of a sequence from here on are not computed
    int max_len;              // keys of a sequence from here on are ignored
    Divider by_group, by_heads;      // division by G and by Hkv
    float scale;              // of the scores, the K scale of codes included
    float v_scale;            // of the values (1 for bf16 rows)
    OutDev out;               // packed rows t * Hq + h

    // Paged cache: a sequence's n G rows to a KV head are cut into tiles of kTile for the matrix pipes (ragged_wide_impl.h), and what remains, where it
    // is no more than few_rows, goes to ragged_rows_impl.h, which is bound by the reads of the cache: all rows of a decode step, the last ones of a chunk.
    int few_rows;             // 0: packed rows, where the tiles take everything
    int few_most;             // rows that remain of a sequence, at most
    int nsplit, chunk;        // key ranges they are split into, and their length (a multiple of 128)
    int tiles;                // tiles of 32 rows in few_most
    int both_tiles;           // 0: few_most <= 16
    int wavefronts;           // of a workgroup: 4 or 8
    Divider by_seqs;          // division by B
    int paired;               // neighbouring KV heads share lines of the cache: their workgroups have ids that differ by 8
    Divider by_pairs;         // division by Hkv / 2 where they do
    unsigned row_wgs;         // workgroups
    float* part_O;            // nsplit > 1: partial results [nsplit][part_rows][D], [nsplit][part_rows], part_rows = B * Hkv * few_most
    float* part_L;
    int64_t part_rows;
    Divider by_most;          // division by few_most

    // Tiles.
    int tiles_all;            // numbers of tiles (ragged_tile)
    Divider by_heads8;        // division by Hkv / 8 where Hkv is a multiple of 8
    int tile_nsplit, tile_chunk;        // key ranges of a tile and their length (a multiple of 64)
    float* tile_part_O;       // tile_nsplit > 1: partial results [tile_nsplit][rows * Hq][D], [tile_nsplit][rows * Hq]
    float* tile_part_L;
};
constexpr int kTile = 128;        // rows of a tile
constexpr int kFewRows = 32;      // a remainder of more rows is a tile: beside tiles, and wherever a read of the cache for every 32 rows is what costs
constexpr int kFewRowsAlone = 64; // ... in small calls of no more rows than these, where a launch without tiles is over sooner (plan_few_rows)
// Of a sequence's n G rows, those that tiles take.
__host__ __device__ inline int rows_in_tiles(int nrows, int few_rows) { return nrows % kTile <= few_rows ? nrows - nrows % kTile : nrows; }

// Workgroups that take what remains (whole groups of sixteen where they come in pairs)
inline int64_t rows_grid(const RaggedArgs& a) {
    const int64_t n = (int64_t)a.B * a.tiles * a.nsplit * a.Hkv;
    return a.paired ? (n + 15) / 16 * 16 : n;
}

// Workgroups that take tiles
inline int64_t tiles_grid(const RaggedArgs& a) { return (int64_t)a.tiles_all * a.Hkv * a.tile_nsplit; }
// ... and of a launch that has tiles: over a paged cache both kinds by turns, 256 of each
inline int64_t ragged_grid(const RaggedArgs& a) { return a.few_rows == 0 ? tiles_grid(a) : ((tiles_grid(a) + 255) / 256 + (rows_grid(a) + 255) / 256) * 256; }
// Workgroups of the join of parts: groups of D / 8 lanes to a row, and of a token's heads
inline int join_groups(const RaggedArgs& a) { return a.nsplit > 8 || a.tile_nsplit > 8 ? 8 : 1; }
inline int join_per_token(const RaggedArgs& a, int D) { const int rows = 2048 / D / join_groups(a); return a.tile_nsplit > 1 ? (a.Hq + rows - 1) / rows : 0; }
inline int64_t join_grid(const RaggedArgs& a, int D) {
    const int rows = 2048 / D / join_groups(a);
    return (int64_t)a.rows * join_per_token(a, D) + (a.nsplit > 1 ? (a.part_rows + rows - 1) / rows : 0);
}

// ---- launchers ----
hipError_t launch_ragged_rows(const RaggedArgs& a, int D, bool codes, hipStream_t s);       // ragged_rows.hip: what remains, or all there is
hipError_t launch_ragged_wide(const RaggedArgs& a, bool codes, hipStream_t s);           // ragged_wide.hip, D = 128: tiles, and what remains in the same launch
hipError_t launch_ragged_wide_d64(const RaggedArgs& a, bool codes, hipStream_t s);          // ragged_wide_d64.hip
hipError_t launch_ragged_join(const RaggedArgs& a, int D, hipStream_t s);                   // ragged_rows.hip: the parts of either (nsplit > 1, tile_nsplit > 1)

// ---- block tables, slots and the write into a paged cache (pages.hip) ----
struct SlotArgs {
    const int32_t* lengths;
    const int32_t* counts;
    const int32_t* free_pages;
    int n_free;
    int32_t* table;           // [B, stride]
    int stride, shift;        // log2(rows per page)
    int B, rows;
    int32_t* q_off;
    int32_t* slots;
    int32_t* new_lengths;
    int32_t* pages_used;
};
hipError_t launch_page_slots(const SlotArgs& a, hipStream_t s);

struct WriteArgs {
    const uint16_t* Knew;     // rows of Hkv * D elements, `stride` elements apart
    const uint16_t* Vnew;
    int64_t stride;
    const int32_t* slots;
    uint16_t* K;              // the pool
    uint16_t* V;
    int64_t pool_rows;
    int rows, vec;            // vec: pieces of eight elements per row
    Divider by_vec;
    int codes;
    float k_scale, v_scale;
};
hipError_t launch_kv_write(const WriteArgs& a, hipStream_t s);

#ifdef __HIPCC__
// LSE of a part whose row is NaN: infinity, which no maximum passes over, and with which every sum of parts becomes NaN.
__device__ __forceinline__ float part_lse(float lse) { return lse != lse ? INFINITY : lse; }

// A value that is infinite or NaN would reach the rows of a tile that do not see its key: 0 times it is NaN.  So in stages that some row does not see as a whole such values are
// 0 in LDS (take_out), and the rows that do see them have them added at the end, from memory (value_if_not_finite).
template <bool CODES>      // the top bit of every element of the word that is not finite
__device__ __forceinline__ unsigned not_finite(unsigned v) {
    return CODES ? ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u : ((v & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
}
// Of N pieces of 16 bytes at `at`, `step` bytes apart; true: some lane had one.
template <bool CODES, int N>
__device__ __forceinline__ bool take_out(unsigned char* at, int step) {
    typedef unsigned V4 __attribute__((ext_vector_type(4)));
    V4 v[N];
    unsigned bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const V4*>(at + i * step);
    if constexpr (CODES) {
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) bad |= not_finite<CODES>(v[i / 4][i % 4]);
    } else {      // two instructions a word: the largest magnitude
        typedef unsigned short Pair __attribute__((ext_vector_type(2)));
        Pair most = {0, 0};
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) most = __builtin_elementwise_max(most, __builtin_bit_cast(Pair, v[i / 4][i % 4] & 0x7fff7fffu));
        bad = not_finite<CODES>(__builtin_bit_cast(unsigned, most));
    }
    if (__builtin_expect(!__any(bad != 0u), 1)) return false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned x = not_finite<CODES>(v[i][k]);
            v[i][k] &= ~(CODES ? (x >> 7) * 0xffu : (x >> 15) * 0xffffu);
        }
        *reinterpret_cast<V4*>(at + i * step) = v[i];
    }
    return true;
}
template <bool CODES>
__device__ __forceinline__ float value_if_not_finite(const unsigned char* e) {
    if constexpr (CODES) {
        return (*e & 0x7f) == 0x7f ? __builtin_nanf("") : 0.f;
    } else {
        const unsigned x = *reinterpret_cast<const uint16_t*>(e);
        return (x & 0x7f80u) == 0x7f80u ? __builtin_bit_cast(float, x << 16) : 0.f;
    }
}

// What a tile's kernel knows of its sequence; uniform over the workgroup.
struct RaggedSeq {
    int b;
    int q0, n;        // first token, tokens
    int take;         // tokens that are computed (n, or max_new)
    int len;          // keys
    __device__ __forceinline__ int seen(int t) const { return len - (n - 1 - t); }      // keys that token t sees (none if <= 0)
};
__device__ __forceinline__ RaggedSeq ragged_seq(const RaggedArgs& a, int b) {
    RaggedSeq s;
    s.b = b;
    s.q0 = min(max(a.q_off[b], 0), a.rows);      // (offsets out of order or range give wrong numbers, never an access outside Q or O)
    s.n = min(max(a.q_off[b + 1], s.q0), a.rows) - s.q0;
    s.take = min(s.n, a.max_new);
    s.len = a.lengths ? max(min(a.lengths[b], a.max_len), 0) : s.n;
    return s;
}

// The `rank`-th of all sequences' tiles, and its sequence; false: nobody's.  Every lane of a wavefront must call this.  Tiles come sequence after sequence, so that
// the rows of few sequences at a time are in the L2s (by size alone, whatever their sequence: 16 prompts up to 2048 tokens, 40 heads 329 -> 371 us), the last
// tiles, which see the most keys, first, so that the last workgroups to start have little to do.
// Tiles of sequence b are numbered from floor(q_off[b] * G / kTile) + b on, which leaves room for each of its at most ceil(n * G / kTile) tiles before the next
// sequence's: no table is needed, and the sequence is found with a look at 64 at a time.  Up to eight sequences are taken in the order of their largest tiles
// instead (lane i holds sequence i and adds up the tiles of those before it: 0.09 us a sequence, 5 us of the 16 that a workgroup had with 45 short prompts).
__device__ __forceinline__ bool tile_of_rank(const RaggedArgs& a, int rank, RaggedSeq& seq, int& tile) {
    const int lane = threadIdx.x & 63;
    if (a.B <= 8) {
        const RaggedSeq own = ragged_seq(a, min(lane, a.B - 1));
        const int tiles = lane < a.B ? (rows_in_tiles(own.take * a.G, a.few_rows) + kTile - 1) / kTile : 0;
        const int size = (max(own.seen(0), 0) / kTile) * a.G + tiles;      // of the largest tile, in units of a tile's tokens
        int start = 0;
        for (int i = 0; i < a.B; ++i) {
            const int other = __builtin_amdgcn_readlane(size, i);
            start += other > size || (other == size && i < lane) ? __builtin_amdgcn_readlane(tiles, i) : 0;
        }
        const unsigned long long at = __ballot(rank >= start && rank < start + tiles);
        if (at == 0) return false;
        const int b = __builtin_ctzll(at);
        seq = RaggedSeq{b, __builtin_amdgcn_readlane(own.q0, b), __builtin_amdgcn_readlane(own.n, b), __builtin_amdgcn_readlane(own.take, b),
                        __builtin_amdgcn_readlane(own.len, b)};
        tile = __builtin_amdgcn_readlane(start + tiles - 1, b) - rank;
        return true;
    }
    const int number = a.tiles_all - 1 - rank;
    const auto first = [&](int q0, int i) { return (int)(((unsigned)q0 * (unsigned)a.G) / kTile) + i; };
    int lo = 0, n = a.B;
    while (n > 64) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const int c = __builtin_popcountll(__ballot(lane * step < n && first(min(max(a.q_off[i], 0), a.rows), i) <= number));
        if (c == 0) return false;
        lo += (c - 1) * step;
        n = min(step, n - (c - 1) * step);
    }
    const RaggedSeq own = ragged_seq(a, min(lo + lane, a.B - 1));
    const int c = __builtin_popcountll(__ballot(lane < n && first(own.q0, lo + lane) <= number));
    if (c == 0) return false;
    const int at = __builtin_amdgcn_readfirstlane(c - 1);
    seq = RaggedSeq{lo + at, __builtin_amdgcn_readlane(own.q0, at), __builtin_amdgcn_readlane(own.n, at), __builtin_amdgcn_readlane(own.take, at),
                    __builtin_amdgcn_readlane(own.len, at)};
    tile = number - first(seq.q0, seq.b);
    return tile >= 0 && tile * kTile < rows_in_tiles(seq.take * a.G, a.few_rows);      // (tile < 0: offsets out of order)
}
#endif
// Tile numbers of a call.
inline int64_t ragged_tiles(int64_t rows, int G, int B) { return rows * G / kTile + B; }

}  // namespace hg
