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

    // Sequences of at most few_rows query rows to a KV head (paged cache): ragged_rows.hip.  The tiles' kernel takes the others.
    int few_rows;             // 0: none
    int few_tokens;           // tokens that such a sequence has at most
    int nsplit, chunk;        // key ranges a tile is split into, and their length (a multiple of 128)
    int tiles;                // tiles of few_tokens tokens
    int both_tiles;           // 0: no sequence has more than 16 rows
    int wavefronts;           // of a workgroup: 4 or 8
    Divider by_seqs;          // division by B
    float* part_O;            // nsplit > 1: partial results [nsplit][part_rows][D], [nsplit][part_rows], part_rows = B * few_tokens * Hq
    float* part_L;
    int64_t part_rows;
    Divider by_q_heads, by_tokens;      // division by Hq and by few_tokens

    // The others, and prompts: ragged_wide_impl.h, tiles of kTile rows.
    int tiles_all;            // numbers of tiles (ragged_tile)
    Divider by_heads8;        // division by Hkv / 8 where Hkv is a multiple of 8
    int tile_nsplit, tile_chunk;        // key ranges of a tile and their length (a multiple of 64)
    float* tile_part_O;       // tile_nsplit > 1: partial results [tile_nsplit][rows * Hq][D], [tile_nsplit][rows * Hq]
    float* tile_part_L;
};
constexpr int kTile = 128;
constexpr int kFewRows = 64;

// Workgroups that take the sequences of few rows
inline int64_t rows_grid(const RaggedArgs& a) { return (int64_t)a.B * a.tiles * a.nsplit * a.Hkv; }

// ---- launchers ----
hipError_t launch_ragged_rows(const RaggedArgs& a, int D, bool codes, hipStream_t s);       // ragged_rows.hip: sequences of few rows
hipError_t launch_ragged_merge(const RaggedArgs& a, int D, hipStream_t s);                  // ... their parts (nsplit > 1)
hipError_t launch_ragged_wide(const RaggedArgs& a, bool codes, bool with_rows, hipStream_t s);           // ragged_wide.hip, D = 128: the others' tiles; with_rows: sequences of few rows in the same launch
hipError_t launch_ragged_wide_d64(const RaggedArgs& a, bool codes, bool with_rows, hipStream_t s);          // ragged_wide_d64.hip
hipError_t launch_ragged_join(const RaggedArgs& a, int D, hipStream_t s);                   // the parts of the others' rows (tile_nsplit > 1)

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

// Tiles of ROWS query rows are numbered so that no table is needed: those of sequence b start at floor(q_off[b] * G / ROWS) + b, which
// leaves room for each of its ceil(n * G / ROWS) tiles before the next sequence's; a number between two sequences' tiles is nobody's.
// Found with one look at 64 sequences at a time.  Every lane of a wavefront must call this; false: nobody's.
template <int ROWS>
__device__ __forceinline__ bool ragged_tile(const RaggedArgs& a, int number, int& b, int& tile) {
    const int lane = threadIdx.x & 63;
    const auto first = [&](int i) { return (int)(((unsigned)min(max(a.q_off[i], 0), a.rows) * (unsigned)a.G) / ROWS) + i; };
    int lo = 0, n = a.B;
    for (;;) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const bool at_or_before = lane * step < n && first(i) <= number;
        const int c = __builtin_popcountll(__ballot(at_or_before));
        if (c == 0) return false;
        lo += (c - 1) * step;
        n = min(step, n - (c - 1) * step);
        if (n == 1) break;
    }
    b = __builtin_amdgcn_readfirstlane(lo);
    tile = __builtin_amdgcn_readfirstlane(number - first(b));
    return tile >= 0;
}
#endif
// Tile numbers of a call.
inline int64_t ragged_tiles(int64_t rows, int G, int B, int tile_rows) { return rows * G / tile_rows + B; }

}  // namespace hg
