// Host side of the calls between a prompt and its first decode step: argument checks and the choice of kernels for hg_prompt_attn,
// hg_chunk_attn_paged, hg_page_slots and hg_kv_write_paged.  As in api.hip: no device allocation, no host synchronisation, no copies.
#include <math.h>
#include <algorithm>

#include "context.h"
#include "hydragen.h"
#include "hydragen_debug.h"
#include "ragged.h"

namespace {

using namespace hg;

constexpr int kAllKeys = 0x3fffffff;      // longer than any key range
constexpr int64_t kMostWorkgroups = (1LL << 24) - 1024;      // of 256 threads: a launch has fewer than 2^32, and either kind of workgroup is rounded up to whole 256

int rc_of(hipError_t e) { return e == hipSuccess ? HG_OK : HG_ERR_HIP; }

bool positive_scale(float s) { return s > 0.f && s <= 3.0e38f; }

// log2 of the rows per page; -1: not a power of two in [16, 1024]
int page_shift(int page_size) {
    for (int s = 4; s <= 10; ++s)
        if (1 << s == page_size) return s;
    return -1;
}

// Sizes that both attention calls have.
int check_sizes(int rows, int max_new, int B, int Hq, int Hkv, int D) {
    if (rows < 0 || max_new < 0 || B < 0 || Hq <= 0 || Hkv <= 0) return HG_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return HG_ERR_UNSUPPORTED;
    if (Hq % Hkv != 0) return HG_ERR_UNSUPPORTED;
    if ((int64_t)Hq * D > (1LL << 30)) return HG_ERR_UNSUPPORTED;      // (a head lies within 32 bits of its token's first)
    // (the last: with one range of keys to each, tiles and what remains are fewer than kMostWorkgroups)
    if ((int64_t)rows * Hq >= (1LL << 31) || B >= (1 << 24) || ((int64_t)rows * (Hq / Hkv) + 256LL * B) * Hkv >= 128 * kMostWorkgroups) return HG_ERR_UNSUPPORTED;
    return HG_OK;
}
// ... and those of keys in a cache.
int check_cache_sizes(int max_len, int Hkv, int D) { return max_len >= kAllKeys || (int64_t)Hkv * D * 32 >= (1LL << 31) ? HG_ERR_UNSUPPORTED : HG_OK; }

// Shapes and row distances that both attention calls have.
int check_ragged(const hg_ctx* c, const void* Q, int64_t q_stride, const int32_t* q_off, int rows, int max_new, int B, int Hq, int Hkv, int D,
                 const void* O, int o_dtype) {
    if (!c || (o_dtype != HG_F32 && o_dtype != HG_BF16)) return HG_ERR_INVALID_ARG;
    const int rc = check_sizes(rows, max_new, B, Hq, Hkv, D);
    if (rc) return rc;
    if (rows > 0 && B > 0 && max_new > 0) {
        if (!Q || !q_off || !O) return HG_ERR_INVALID_ARG;
        if (q_stride < (int64_t)Hq * D || q_stride % 8 != 0 ||
            (reinterpret_cast<uintptr_t>(Q) | reinterpret_cast<uintptr_t>(O)) % 16 != 0)
            return HG_ERR_INVALID_ARG;
    }
    return HG_OK;
}

// What is the same for both attention calls, from checked arguments.
RaggedArgs ragged_args(const void* Q, int64_t q_stride, const int32_t* q_off, int rows, int max_new, int B, int Hq, int Hkv, int D, float scale,
                       void* O, int o_dtype, float* LSE) {
    RaggedArgs a{};
    a.Q = static_cast<const uint16_t*>(Q);
    a.q_stride = 2 * q_stride;
    a.q_off = q_off;
    a.rows = rows;
    a.B = B; a.Hq = Hq; a.Hkv = Hkv; a.G = Hq / Hkv;
    a.max_new = max_new;
    a.by_group = divider((unsigned)a.G);
    a.by_heads = divider((unsigned)Hkv);
    a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)D);
    a.v_scale = 1.f;
    a.out.O = O;
    a.out.LSE = LSE;
    a.out.bf16 = o_dtype == HG_BF16;
    a.nsplit = a.tile_nsplit = 1;
    a.chunk = a.tile_chunk = kAllKeys;
    a.tiles_all = (int)ragged_tiles(rows, a.G, B);
    a.by_heads8 = divider((unsigned)std::max(Hkv / 8, 1));
    return a;
}

// Workspace that is left: partial results are taken from it in turn.
struct Room {
    float* p;
    size_t floats;
    float* take(size_t n) {
        float* const at = p;
        p += n;
        floats -= n;
        return at;
    }
};
Room room_of(const hg_ctx* c) { return Room{reinterpret_cast<float*>(c->ws), c->ws ? c->ws_bytes / sizeof(float) : 0}; }

// Ranges of at least `least` keys, a multiple of `step` long, for `want` of them, and where their parts go.
void split_keys(int64_t want, int max_len, int least, int step, int64_t rows, int D, Room& room, int& nsplit, int& chunk, float*& O, float*& L) {
    const size_t per = (size_t)rows * (D + 1);
    const int64_t most = std::min<int64_t>({want, max_len / least, (int64_t)(per ? room.floats / per : 0), 256});
    if (most <= 1 || rows >= (1LL << 31)) return;
    chunk = (int)(((max_len + most - 1) / most + step - 1) / step * step);
    nsplit = (int)(((int64_t)max_len + chunk - 1) / chunk);
    O = room.take((size_t)nsplit * rows * D);
    L = room.take((size_t)nsplit * rows);
}

// What remains behind the tiles, or all there is: how many rows that may be, and how the keys are split.
//
// 33 .. 64 rows are two tiles of the few rows, which each read the cache, or one of 128, which reads it once and multiplies for nothing what is not there.  The latter is
// slower to start and end, and has at most a range for every 1024 keys.  us by the first / by the second, 64 rows at most of B sequences, bf16, 32/8 heads, D = 128: B = 4, up to 1200 keys
// 12.5 / 23.5, up to 2400 20.9 / 28.1, up to 8000 35.1 / 29.7; B = 16, up to 600 11.6 / 16.8, 1200 19.1 / 24.3, 2400 40.8 / 35.8, 8000 113 / 73; B = 32 (two workgroups to a
// CU by the first), up to 300 17.0 / 13.9, 8000 209 / 134; codes, B = 16, up to 2400 31.5 / 40.1, 8000 77.8 / 57.0; D = 64, B = 16, up to 2400 25.2 / 27.8, 8000 59.9 / 41.5.  Behind tiles (that
// is, in calls of more rows) the second is as good or better: 64 x 32/8, 8 chunks up to 256 tokens among single ones, up to 4096 keys 130 / 125, chunks of 1 .. 64 tokens 198 / 179.
void plan_few_rows(RaggedArgs& a, int D, bool codes, Room& room) {
    const double cache = (double)a.B * a.Hkv * a.max_len * D * (codes ? 2 : 4);      // bytes, at most
    const bool alone = (int64_t)a.max_new * a.G <= kFewRowsAlone && (int64_t)a.B * a.Hkv <= 128 && cache <= 1e8;
    a.few_rows = alone ? kFewRowsAlone : kFewRows;
    a.few_most = (int)std::min<int64_t>((int64_t)a.max_new * a.G, a.few_rows);
    a.both_tiles = a.few_most > 16;
    a.tiles = (a.few_most + 31) / 32;
    // Four times the workgroups that fit the chip, so that contexts of different lengths even out, of at least 256 keys each.  Up to 1280 keys the join costs more than
    // it saves.  us with 1 / 512 / 1024 / 2048 / 4096 workgroups wanted: 64 x 32/8 heads, up to 4096 rows 113 / 114 / 109 / 105 / 101, all of 4096 rows 173.6 / 173.7 / 178.8 /
    // 182.7 / 188.6; 16 x 32/8, up to 8192 103.6 / 69.8 / 55.0 / 56.2 / 55.9; 32 x 64/8, up to 8192 122.1 / 127.5 / 111.5 / 103.8 / 105.4, codes 75.9 / 78.2 / 73.4 / 68.6 / 66.2; 16 x 40,
    // up to 4096 140.0 / 138.6 / 130.2 / 122.2 / 120.2; one sequence of 65536 rows, 64/8 696 / 53.0 / 58.0 / 58.7 / 58.9; 256 x 8/1, up to 1024 17.7 / 20.4 / 21.5 / 21.3 / 21.3.
    const int64_t wgs = (int64_t)a.B * a.Hkv;
    a.part_rows = wgs * a.few_most;
    split_keys(a.max_len <= 1280 ? 1 : (2048 + wgs - 1) / wgs, a.max_len, 256, 128, a.part_rows, D, room, a.nsplit, a.chunk, a.part_O, a.part_L);
    a.wavefronts = wgs * a.nsplit <= 256 ? 8 : 4;
    a.by_seqs = divider((unsigned)a.B);
    a.paired = codes && D == 64 && a.Hkv % 2 == 0;
    a.by_pairs = divider((unsigned)std::max(a.Hkv / 2, 1));
    a.row_wgs = (unsigned)std::min<int64_t>(rows_grid(a), 0xffffffffLL);      // (the launch refuses what does not fit a grid)
    a.by_most = divider((unsigned)a.few_most);
}

// Tiles.  A call of few tiles splits their keys; what that saves is weighed against the parts' way through memory and the join, from the host's bounds (tokens and
// longest context; contexts are taken to be three quarters of that on average).  512 workgroups run at a time, so their number is made to go into whole rounds; a
// stage of 32 keys takes 0.95 us, 0.6 where a workgroup has its CU to itself, a workgroup 8 us beside its stages; parts are written and read at 4.5 TB/s.
void plan_tiles(RaggedArgs& a, int D, Room& room) {
    const double wgs = (double)(((int64_t)a.rows * a.G + kTile - 1) / kTile) * a.Hkv, stages = a.max_len * (D == 128 ? 1.0 : 0.5) / 32.0;
    const double part = 8.0 * a.rows * a.Hq * (D + 1) / 4.5e6;
    int best = 1;
    double least = 1e300;
    const int most = std::max(1, (int)std::min<int64_t>({64, a.max_len / 1024, (kMostWorkgroups - (int64_t)a.row_wgs) / std::max<int64_t>(1, (int64_t)a.tiles_all * a.Hkv)}));
    for (int s = 1; s <= most; ++s) {
        const double n = 0.75 * wgs * s, us = std::max(1.0, ceil(n / 512.0)) * (stages / s * (n <= 256.0 ? 0.6 : 0.95) + 8.0) + (s > 1 ? part * s + (a.nsplit > 1 ? 1.0 : 6.0) : 0.0);
        if (us < (best == 1 ? 0.9 : 1.0) * least) { least = us; best = s; }      // (a tenth at least, or there is nothing to join)
        if (wgs >= 512.0) break;
    }
    split_keys(best, a.max_len, 1024, 64, (int64_t)a.rows * a.Hq, D, room, a.tile_nsplit, a.tile_chunk, a.tile_part_O, a.tile_part_L);
}

// Choices of a call over packed rows, whose sequences have no more keys than there are tokens, whatever the caller's bound ...
void plan_prompt(RaggedArgs& a, int max_len, int D, Room room) {
    a.max_len = std::min(max_len, a.rows);
    plan_tiles(a, D, room);
}
// ... and of one over a paged cache.  true: it has tiles
bool plan_chunk(RaggedArgs& a, int max_len, int D, bool codes, Room room) {
    a.max_len = max_len;
    plan_few_rows(a, D, codes, room);
    const bool tiles = (int64_t)std::min(a.max_new, a.rows) * a.G > a.few_rows;
    if (tiles) plan_tiles(a, D, room);
    return tiles;
}

// tiles: the call has any; what remains behind them, or is all there is, goes along
int run(const hg_ctx* c, const RaggedArgs& a, int D, bool codes, bool tiles) {
    const int rc = rc_of(!tiles ? launch_ragged_rows(a, D, codes, c->stream) : D == 128 ? launch_ragged_wide(a, codes, c->stream) : launch_ragged_wide_d64(a, codes, c->stream));
    if (rc || (a.nsplit == 1 && a.tile_nsplit == 1)) return rc;
    return rc_of(launch_ragged_join(a, D, c->stream));
}

}  // namespace

extern "C" {

int hg_prompt_attn(hg_ctx* c, const void* Q, const void* K, const void* V, int64_t q_stride, int64_t kv_stride, const int32_t* q_off, int rows,
                   int max_len, int B, int Hq, int Hkv, int D, float scale, void* O, int o_dtype, float* LSE) {
    const int rc = check_ragged(c, Q, q_stride, q_off, rows, max_len, B, Hq, Hkv, D, O, o_dtype);
    if (rc) return rc;
    if (rows == 0 || B == 0 || max_len == 0) return HG_OK;
    if (!K || !V || kv_stride < (int64_t)Hkv * D || kv_stride % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) % 16 != 0) return HG_ERR_INVALID_ARG;
    if (kv_stride >= (1LL << 26)) return HG_ERR_UNSUPPORTED;      // (a copy's rows lie within 32 bits of each other)
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    RaggedArgs a = ragged_args(Q, q_stride, q_off, rows, max_len, B, Hq, Hkv, D, scale, O, o_dtype, LSE);
    a.K = static_cast<const unsigned char*>(K);
    a.V = static_cast<const unsigned char*>(V);
    a.kv_stride = 2 * kv_stride;
    plan_prompt(a, max_len, D, room_of(c));
    return run(c, a, D, false, true);
}

int hg_chunk_attn_paged(hg_ctx* c, const void* Q, int64_t q_stride, const int32_t* q_off, int rows, const hg_paged_kv* kv, const int32_t* lengths,
                        int max_new, int max_len, int B, int Hq, int Hkv, int D, float scale, void* O, int o_dtype, float* LSE) {
    const int rc = check_ragged(c, Q, q_stride, q_off, rows, max_new, B, Hq, Hkv, D, O, o_dtype);
    if (rc) return rc;
    if (!kv || max_len < 0) return HG_ERR_INVALID_ARG;
    const bool codes = kv->kv_format == HG_KV_E4M3;
    if (!codes && kv->kv_format != HG_KV_BF16) return HG_ERR_INVALID_ARG;
    if (codes && (!positive_scale(kv->k_scale) || !positive_scale(kv->v_scale))) return HG_ERR_INVALID_ARG;
    const int shift = page_shift(kv->page_size);
    if (shift < 0 || kv->n_pages < 0 || kv->table_stride < 0) return HG_ERR_INVALID_ARG;
    if ((int64_t)kv->n_pages * kv->page_size >= (1LL << 31) || (int64_t)kv->table_stride * kv->page_size >= (1LL << 31) || check_cache_sizes(max_len, Hkv, D))
        return HG_ERR_UNSUPPORTED;
    if (rows == 0 || B == 0 || max_new == 0) return HG_OK;
    if (!lengths || !kv->K || !kv->V || !kv->page_table || kv->n_pages < 1 || (int64_t)kv->table_stride * kv->page_size < std::max(max_len, 1) ||
        (reinterpret_cast<uintptr_t>(kv->K) | reinterpret_cast<uintptr_t>(kv->V)) % 16 != 0) return HG_ERR_INVALID_ARG;
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    RaggedArgs a = ragged_args(Q, q_stride, q_off, rows, max_new, B, Hq, Hkv, D, scale, O, o_dtype, LSE);
    a.K = static_cast<const unsigned char*>(kv->K);
    a.V = static_cast<const unsigned char*>(kv->V);
    a.kv_stride = (int64_t)Hkv * D * (codes ? 1 : 2);
    a.lengths = lengths;
    a.pg.table = kv->page_table;
    a.pg.shift = shift;
    a.pg.stride = kv->table_stride;
    a.pg.n_pages = kv->n_pages;
    if (codes) {
        a.scale *= kv->k_scale;
        a.v_scale = kv->v_scale;
    }
    const bool tiles = plan_chunk(a, max_len, D, codes, room_of(c));
    return run(c, a, D, codes, tiles);
}

int hg_page_slots(hg_ctx* c, const int32_t* lengths, const int32_t* counts, const int32_t* free_pages, int n_free, int page_size, int B, int rows,
                  int32_t* page_table, int table_stride, int32_t* q_off, int32_t* slots, int32_t* new_lengths, int32_t* pages_used) {
    const int shift = page_shift(page_size);
    if (!c || shift < 0 || n_free < 0 || B < 0 || rows < 0 || table_stride < 0 || !q_off || !pages_used) return HG_ERR_INVALID_ARG;
    if ((int64_t)table_stride * page_size >= (1LL << 31) || (int64_t)B * table_stride >= (1LL << 31)) return HG_ERR_UNSUPPORTED;
    if (B > 0 && (!lengths || !counts || !new_lengths || (table_stride > 0 && !page_table))) return HG_ERR_INVALID_ARG;
    if ((rows > 0 && !slots) || (n_free > 0 && !free_pages)) return HG_ERR_INVALID_ARG;
    // every workgroup reads the lengths and the counts: none may write over them
    if (B > 0 && (new_lengths == lengths || new_lengths == counts || q_off == lengths || q_off == counts)) return HG_ERR_INVALID_ARG;
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    SlotArgs a{};
    a.lengths = lengths; a.counts = counts; a.free_pages = free_pages; a.n_free = n_free;
    a.table = page_table; a.stride = table_stride; a.shift = shift;
    a.B = B; a.rows = rows;
    a.q_off = q_off; a.slots = slots; a.new_lengths = new_lengths; a.pages_used = pages_used;
    return rc_of(launch_page_slots(a, c->stream));
}

int hg_kv_write_paged(hg_ctx* c, const void* Knew, const void* Vnew, int64_t stride, const int32_t* slots, int rows, const hg_paged_kv* kv, int Hkv,
                      int D) {
    if (!c || !kv || rows < 0 || Hkv <= 0) return HG_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return HG_ERR_UNSUPPORTED;
    const bool codes = kv->kv_format == HG_KV_E4M3;
    if (!codes && kv->kv_format != HG_KV_BF16) return HG_ERR_INVALID_ARG;
    if (codes && (!positive_scale(kv->k_scale) || !positive_scale(kv->v_scale))) return HG_ERR_INVALID_ARG;
    if (page_shift(kv->page_size) < 0 || kv->n_pages < 0) return HG_ERR_INVALID_ARG;
    if ((int64_t)kv->n_pages * kv->page_size >= (1LL << 31) || (int64_t)rows * Hkv * D >= (1LL << 33) || (int64_t)Hkv * D >= (1LL << 31))
        return HG_ERR_UNSUPPORTED;
    if (rows == 0) return HG_OK;
    if (!Knew || !Vnew || !slots || stride < (int64_t)Hkv * D || stride % 8 != 0 ||
        (reinterpret_cast<uintptr_t>(Knew) | reinterpret_cast<uintptr_t>(Vnew)) % 16 != 0) return HG_ERR_INVALID_ARG;
    if (kv->n_pages > 0 && (!kv->K || !kv->V || (reinterpret_cast<uintptr_t>(kv->K) | reinterpret_cast<uintptr_t>(kv->V)) % 16 != 0))
        return HG_ERR_INVALID_ARG;
    if (kv->n_pages == 0) return HG_OK;      // no row has a place
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    WriteArgs a{};
    a.Knew = static_cast<const uint16_t*>(Knew);
    a.Vnew = static_cast<const uint16_t*>(Vnew);
    a.stride = stride;
    a.slots = slots;
    a.K = static_cast<uint16_t*>(kv->K);
    a.V = static_cast<uint16_t*>(kv->V);
    a.pool_rows = (int64_t)kv->n_pages * kv->page_size;
    a.rows = rows;
    a.vec = Hkv * D / 8;
    a.by_vec = divider((unsigned)a.vec);
    a.codes = codes;
    a.k_scale = kv->k_scale;
    a.v_scale = kv->v_scale;
    return rc_of(launch_kv_write(a, c->stream));
}

int hg_debug_ragged_plan(int paged, int codes, int rows, int max_new, int max_len, int B, int Hq, int Hkv, int D, size_t workspace_bytes, int64_t out[14]) {
    if (!out || max_len < 0) return HG_ERR_INVALID_ARG;
    int rc = check_sizes(rows, paged ? max_new : max_len, B, Hq, Hkv, D);
    if (!rc && paged) rc = check_cache_sizes(max_len, Hkv, D);
    if (rc) return rc;
    std::fill(out, out + 14, (int64_t)0);
    if (rows == 0 || B == 0 || (paged ? max_new : max_len) == 0) return HG_OK;      // nothing is launched
    RaggedArgs a = ragged_args(nullptr, 0, nullptr, rows, paged ? max_new : max_len, B, Hq, Hkv, D, 0.f, nullptr, HG_F32, nullptr);
    float* const ws = reinterpret_cast<float*>(256);      // (only distances from it are looked at)
    const Room room{ws, workspace_bytes / sizeof(float)};
    bool tiles = true;
    if (paged) tiles = plan_chunk(a, max_len, D, codes != 0, room);
    else plan_prompt(a, max_len, D, room);
    const auto at = [&](const float* p) { return p ? (int64_t)((reinterpret_cast<intptr_t>(p) - reinterpret_cast<intptr_t>(ws)) / (int64_t)sizeof(float)) : -1; };
    const bool join = a.nsplit > 1 || a.tile_nsplit > 1;
    const int64_t got[14] = {tiles, a.few_rows, a.few_most, a.nsplit, a.chunk, a.tile_nsplit, a.tile_chunk, at(a.part_O), at(a.part_L), at(a.tile_part_O), at(a.tile_part_L),
                             tiles ? ragged_grid(a) : rows_grid(a), tiles ? 256 : 64 * a.wavefronts, join ? join_grid(a, D) : 0};
    std::copy(got, got + 14, out);
    return HG_OK;
}

}  // extern "C"
