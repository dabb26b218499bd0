// Host side of the bookkeeping of drafted trees: argument checks and launches of hg_tree_masks, hg_tree_verify and hg_tree_keep_paged.  As in api.hip: no device
// allocation, no host synchronisation, no copies.
#include <algorithm>

#include "context.h"
#include "hydragen.h"
#include "tree.h"

namespace {

using namespace hg;

int rc_of(hipError_t e) { return e == hipSuccess ? HG_OK : HG_ERR_HIP; }

// Sizes that the three calls have.  (A launch has fewer than 2^32 threads.)
int check_tree(const hg_ctx* c, const int32_t* q_off, int rows, int max_new, int B) {
    if (!c || rows < 0 || max_new < 0 || B < 0) return HG_ERR_INVALID_ARG;
    if (max_new > HG_MAX_TREE || B >= (1 << 22)) return HG_ERR_UNSUPPORTED;
    return B > 0 && !q_off ? HG_ERR_INVALID_ARG : HG_OK;
}

// Workgroups that share a sequence's first sum over the vocabulary: 8192 elements each, as far as all of them run at once.  The second launch costs 2.5 to 3 us, so vocabularies are large that
// do.  us with / without: 8 sequences, 131072 tokens, chains with drafts in fp32 12.6 / 17.1, trees 29.0 / 31.8, without drafts 11.7 / 12.9; 65536 tokens, 4 trees in bf16 20.0 / 20.4; 50000
// tokens, 64 trees 24.6 / 22.6; 32000 tokens, 32 chains 12.3 / 9.1.
int verify_splits(const hg_ctx* c, int B, int V) {
    const int n = (int)std::min<int64_t>({(V + 8191) / 8192, 1024 / B, kVerifySplits});
    return V >= 98304 && n > 1 && c->ws && c->ws_bytes >= verify_bytes(B, n) ? n : 1;
}

bool among(const void* p, std::initializer_list<const void*> others) { return p && std::find(others.begin(), others.end(), p) != others.end(); }

}  // namespace

extern "C" {

int hg_tree_masks(hg_ctx* c, const int32_t* parents, const int32_t* q_off, int rows, int max_new, int B, uint32_t* masks, int mask_words, int32_t* depth) {
    const int rc = check_tree(c, q_off, rows, max_new, B);
    if (rc) return rc;
    if (mask_words < 0) return HG_ERR_INVALID_ARG;
    if (rows == 0 || B == 0 || max_new == 0) return HG_OK;
    if (!parents || !masks || 32LL * mask_words < std::min(max_new, rows)) return HG_ERR_INVALID_ARG;
    if ((int64_t)HG_MAX_TREE * mask_words >= (1LL << 31)) return HG_ERR_UNSUPPORTED;      // (a sequence's words are counted in 32 bits)
    if (among(masks, {parents, q_off, depth}) || among(depth, {parents, q_off})) return HG_ERR_INVALID_ARG;
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    return rc_of(launch_tree_masks(TreeMaskArgs{parents, q_off, rows, max_new, B, masks, mask_words, depth}, c->stream));
}

int hg_tree_verify(hg_ctx* c, const int32_t* tokens, const int32_t* parents, const int32_t* q_off, int rows, int max_new, int B, int V,
                   const void* target, int64_t target_stride, const void* draft, int64_t draft_stride, int p_dtype,
                   const float* u, const float* u_next, int32_t* path, int32_t* accepted, int32_t* next_tokens) {
    const int rc = check_tree(c, q_off, rows, max_new, B);
    if (rc) return rc;
    if (p_dtype != HG_F32 && p_dtype != HG_BF16 && p_dtype != HG_TOKENS) return HG_ERR_INVALID_ARG;
    const bool probs = p_dtype != HG_TOKENS;
    if (probs && (V < 1 || target_stride < V || (draft && draft_stride < V))) return HG_ERR_INVALID_ARG;
    if (probs && V >= (1 << 30)) return HG_ERR_UNSUPPORTED;
    if (B == 0) return HG_OK;
    if (!accepted || !next_tokens || (probs && !u_next)) return HG_ERR_INVALID_ARG;
    if (rows > 0 && max_new > 0 && (!tokens || !parents || !target || !path || (probs && !u))) return HG_ERR_INVALID_ARG;
    const size_t align = p_dtype == HG_BF16 ? 2 : 4;
    if ((reinterpret_cast<uintptr_t>(target) | (probs ? reinterpret_cast<uintptr_t>(draft) : 0)) % align != 0) return HG_ERR_INVALID_ARG;
    for (const void* out : {static_cast<const void*>(path), static_cast<const void*>(accepted), static_cast<const void*>(next_tokens)})
        if (among(out, {tokens, parents, q_off, target, probs ? draft : nullptr, probs ? u : nullptr, probs ? u_next : nullptr})) return HG_ERR_INVALID_ARG;
    if (among(path, {accepted, next_tokens}) || accepted == next_tokens) return HG_ERR_INVALID_ARG;
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    TreeVerifyArgs a{tokens, parents, q_off, rows, max_new, B, V, target, probs ? draft : nullptr, target_stride, draft_stride, u, u_next, path, accepted, next_tokens};
    a.nsplit = probs ? verify_splits(c, B, V) : 1;
    a.state = reinterpret_cast<TreeVerifyState*>(c->ws);
    a.parts = reinterpret_cast<double*>(c->ws + (a.nsplit > 1 ? (size_t)B * sizeof(TreeVerifyState) : 0));
    return rc_of(launch_tree_verify(a, p_dtype, c->stream));
}

int hg_tree_keep_paged(hg_ctx* c, int n_layers, const hg_paged_kv* kv, const int32_t* q_off, int rows, const int32_t* path, const int32_t* accepted,
                       const int32_t* lengths, int max_new, int B, int Hkv, int D, int32_t* new_lengths) {
    int rc = check_tree(c, q_off, rows, max_new, B);
    if (rc) return rc;
    if (n_layers < 0 || Hkv <= 0 || (n_layers > 0 && !kv)) return HG_ERR_INVALID_ARG;
    if (n_layers > HG_MAX_LAYERS || (D != 64 && D != 128) || (int64_t)Hkv * D >= (1LL << 24)) return HG_ERR_UNSUPPORTED;
    TreeKeepArgs a{};
    for (int i = 0; i < n_layers; ++i) {
        const hg_paged_kv &l = kv[i], &first = kv[0];
        if (l.page_table != first.page_table || l.page_size != first.page_size || l.table_stride != first.table_stride || l.n_pages != first.n_pages || l.kv_format != first.kv_format)
            return HG_ERR_INVALID_ARG;
        a.pool[2 * i] = static_cast<unsigned char*>(l.K);
        a.pool[2 * i + 1] = static_cast<unsigned char*>(l.V);
    }
    if (n_layers > 0) {
        const bool codes = kv->kv_format == HG_KV_E4M3;
        if (!codes && kv->kv_format != HG_KV_BF16) return HG_ERR_INVALID_ARG;
        while (a.shift < 11 && (1 << a.shift) != kv->page_size) ++a.shift;
        if (a.shift < 4 || a.shift > 10 || kv->n_pages < 0 || kv->table_stride < 0) return HG_ERR_INVALID_ARG;
        if ((int64_t)kv->n_pages * kv->page_size >= (1LL << 31) || (int64_t)kv->table_stride * kv->page_size >= (1LL << 31)) return HG_ERR_UNSUPPORTED;
        a.pieces = Hkv * D * (codes ? 1 : 2) / 16;
        if ((int64_t)B * 2 * n_layers * ((a.pieces + 255) / 256) * 256 >= (1LL << 32)) return HG_ERR_UNSUPPORTED;
    }
    if (B == 0) return HG_OK;
    if (!accepted || !lengths || !new_lengths || (rows > 0 && max_new > 0 && !path)) return HG_ERR_INVALID_ARG;
    if (among(new_lengths, {lengths, accepted, q_off, path, n_layers > 0 ? kv->page_table : nullptr})) return HG_ERR_INVALID_ARG;      // (every workgroup reads those)
    if (n_layers > 0 && kv->n_pages > 0 && kv->table_stride > 0) {
        if (!kv->page_table) return HG_ERR_INVALID_ARG;
        void* pools[2 * HG_MAX_LAYERS];
        const int n = 2 * n_layers;
        for (int i = 0; i < n; ++i) {
            if (!a.pool[i] || reinterpret_cast<uintptr_t>(a.pool[i]) % 16 != 0) return HG_ERR_INVALID_ARG;
            pools[i] = a.pool[i];
        }
        std::sort(pools, pools + n);
        if (std::adjacent_find(pools, pools + n) != pools + n) return HG_ERR_INVALID_ARG;      // (a pool that is there twice would be moved twice at once)
        a.layers = n_layers;
        a.table = kv->page_table;
        a.stride = kv->table_stride;
        a.n_pages = kv->n_pages;
    }
    a.q_off = q_off; a.path = path; a.accepted = accepted; a.lengths = lengths; a.new_lengths = new_lengths;
    a.rows = rows; a.max_new = max_new; a.B = B;
    if (hipSetDevice(c->device) != hipSuccess) return HG_ERR_HIP;
    return rc_of(launch_tree_keep(a, c->stream));
}

}  // extern "C"
