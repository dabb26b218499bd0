// Trees of drafted tokens: what each token follows from, which tokens stand, and the accepted rows' move in a paged cache (gfx950 only).
#pragma once
#include "hg_internal.h"

namespace hg {

// Sequence b owns the tokens [q_off[b], q_off[b + 1]) of `rows`; of them the first max_new are looked at.
struct TreeMaskArgs {
    const int32_t* parents;
    const int32_t* q_off;
    int rows, max_new, B;
    uint32_t* masks;      // [rows][words]
    int words;
    int32_t* depth;       // may be null
};
hipError_t launch_tree_masks(const TreeMaskArgs& a, hipStream_t s);

constexpr int kVerifySplits = 64;      // workgroups that share the first sum of a sequence, at most
struct TreeVerifyState {               // where the walk stands when that sum is needed
    int cur, t, kept, more;            // more: for the next sibling; else for the next token
    double c;
};
struct TreeVerifyArgs {
    const int32_t* tokens;
    const int32_t* parents;
    const int32_t* q_off;
    int rows, max_new, B, V;
    const void* target;       // [rows, V], or int32 [rows]
    const void* draft;        // or null
    int64_t target_stride, draft_stride;      // elements
    const float* u;
    const float* u_next;
    int32_t* path;
    int32_t* accepted;
    int32_t* next;
    int nsplit;               // > 1: so many workgroups to a sequence for the first sum
    TreeVerifyState* state;   // [B]
    double* parts;            // [B][4 nsplit]
};
// Bytes that it takes
inline size_t verify_bytes(int B, int nsplit) { return (size_t)B * (sizeof(TreeVerifyState) + (size_t)nsplit * 4 * sizeof(double)); }
hipError_t launch_tree_verify(const TreeVerifyArgs& a, int p_dtype, hipStream_t s);

struct TreeKeepArgs {
    unsigned char* pool[2 * HG_MAX_LAYERS];      // K and V of each layer
    const int32_t* table;
    int stride, shift, n_pages;
    const int32_t* q_off;
    const int32_t* path;
    const int32_t* accepted;
    const int32_t* lengths;
    int32_t* new_lengths;
    int layers, rows, max_new, B;
    int pieces;               // 16 bytes each, of a row of K or of V
};
hipError_t launch_tree_keep(const TreeKeepArgs& a, hipStream_t s);

#ifdef __HIPCC__
struct TreeSeq { int q0, n; };
__device__ __forceinline__ TreeSeq tree_seq(const int32_t* q_off, int rows, int b) {
    TreeSeq s;
    s.q0 = min(max(q_off[b], 0), rows);      // (offsets out of order or range give wrong numbers, never an access outside the tensors)
    s.n = min(max(q_off[b + 1], s.q0), rows) - s.q0;
    return s;
}
#endif

}  // namespace hg
