// Bookkeeping of drafted trees: bit masks of ancestors, verification against the target's probabilities, and the accepted rows' move in the pages.
#include <algorithm>
#include <type_traits>

#include "tree.h"

namespace hg {

namespace {

// ---- masks -----------------------------------------------------------------------------------------------------------------------

// Of 64 tokens, a lane's each, that name their parents by lane (-1: none among them): bits of the lanes that each follows from, itself included, and the topmost of those.
// Doubling: what a token follows from within 2^k steps, and where that many steps lead.
__device__ __forceinline__ void ancestors64(int up, int lane, unsigned long long& bits, int& top) {
    bits = 1ull << lane;
    top = lane;
    int to = up;
    while (__any(to >= 0)) {
        const int src = to < 0 ? lane : to;
        const unsigned lo = __shfl((unsigned)bits, src), hi = __shfl((unsigned)(bits >> 32), src);
        const int t = __shfl(top, src), next = __shfl(to, src);
        if (to >= 0) {
            bits |= (unsigned long long)hi << 32 | lo;
            top = t;
            to = next;
        }
    }
}

// At most 64 tokens to a sequence: a wavefront each, all in registers.
__global__ __launch_bounds__(256) void tree_masks_kernel(TreeMaskArgs a) {
    const int lane = threadIdx.x & 63, b = (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    if (b >= a.B) return;
    const TreeSeq s = tree_seq(a.q_off, a.rows, b);
    const int take = min(s.n, a.max_new);
    const bool here = lane < take;
    int up = here ? a.parents[s.q0 + lane] : -1;
    if (up < 0 || up >= lane) up = -1;
    unsigned long long bits;
    int top;
    ancestors64(up, lane, bits, top);
    if (!here) return;
    uint32_t* const row = a.masks + (int64_t)(s.q0 + lane) * a.words;
    for (int w = 0; w < a.words; ++w) row[w] = w == 0 ? (uint32_t)bits : w == 1 ? (uint32_t)(bits >> 32) : 0u;
    if (a.depth) a.depth[s.q0 + lane] = __builtin_popcountll(bits) - 1;
}

// More: a workgroup to a sequence.  Its 64-token blocks find their own bits side by side; then block after block takes over the row of the token that its topmost one
// follows, which is complete by then.  The rows lie in LDS, a block's only as long as they can have bits: 64 x 2 (k + 1) words, 64 x 272 in all.
constexpr int kMaskThreads = 1024, kMaskWords = 64 * (HG_MAX_TREE / 64) * (HG_MAX_TREE / 64 + 1);
__device__ __forceinline__ int mask_row(int t) { const int k = t >> 6; return 64 * k * (k + 1) + (t & 63) * 2 * (k + 1); }
__global__ __launch_bounds__(kMaskThreads) void tree_masks_long_kernel(TreeMaskArgs a) {
    extern __shared__ uint32_t rows[];      // [kMaskWords], then [HG_MAX_TREE] tokens that lead out of a block
    int* const out = reinterpret_cast<int*>(rows + kMaskWords);
    const int tid = threadIdx.x, lane = tid & 63;
    const TreeSeq s = tree_seq(a.q_off, a.rows, (int)blockIdx.x);
    const int take = min(s.n, a.max_new);
    {
        const bool here = tid < take;
        int up = here ? a.parents[s.q0 + tid] : -1;
        if (up < 0 || up >= tid) up = -1;
        unsigned long long bits;
        int top;
        ancestors64(up >= (tid & ~63) ? up & 63 : -1, lane, bits, top);
        const int leaves = __shfl(up, top);      // (the topmost one's parent lies in an earlier block, or it has none)
        if (here) {
            const int at = mask_row(tid) + 2 * (tid >> 6);
            rows[at] = (uint32_t)bits;
            rows[at + 1] = (uint32_t)(bits >> 32);
            out[tid] = leaves;
        }
    }
    __syncthreads();
    for (int k = 1; 64 * k < take; ++k) {
        for (int i = tid; i < 128 * k; i += kMaskThreads) {
            const int t = 64 * k + i / (2 * k), w = i % (2 * k);
            if (t < take) {
                const int from = out[t];
                rows[mask_row(t) + w] = from >= 0 && w < 2 * ((from >> 6) + 1) ? rows[mask_row(from) + w] : 0u;
            }
        }
        __syncthreads();
    }
    const int64_t first = (int64_t)s.q0 * a.words;
    for (int i = tid; i < take * a.words; i += kMaskThreads) {
        const int t = i / a.words, w = i - t * a.words;
        a.masks[first + i] = w < 2 * ((t >> 6) + 1) ? rows[mask_row(t) + w] : 0u;
    }
    if (a.depth && tid < take) {
        int n = -1;
        for (int w = 0; w < 2 * ((tid >> 6) + 1); ++w) n += __builtin_popcount(rows[mask_row(tid) + w]);
        a.depth[s.q0 + tid] = n;
    }
}

// ---- verification ----------------------------------------------------------------------------------------------------------------

constexpr int kGroup = 8;          // elements that a lane takes at a time

__device__ __forceinline__ float counted(float x) { return x > 0.f && x < INFINITY ? x : 0.f; }      // what is no positive finite number counts as 0
__device__ __forceinline__ float element(const float* row, int64_t i) { return row[i]; }
__device__ __forceinline__ float element(const uint16_t* row, int64_t i) { return __builtin_bit_cast(float, (unsigned)row[i] << 16); }

// Elements 8 g .. 8 g + 7 of a row of V; those behind its end are 0.  Rows begin anywhere, so the loads are of unaligned pieces.
__device__ __forceinline__ void load8(const float* row, int g, int V, float (&x)[kGroup]) {
    struct __attribute__((packed, aligned(4))) Piece { float v[4]; };
    if (kGroup * g + kGroup <= V) {
        const Piece lo = *reinterpret_cast<const Piece*>(row + kGroup * g), hi = *reinterpret_cast<const Piece*>(row + kGroup * g + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = lo.v[i]; x[4 + i] = hi.v[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) x[i] = kGroup * g + i < V ? row[kGroup * g + i] : 0.f;
    }
}
__device__ __forceinline__ void load8(const uint16_t* row, int g, int V, float (&x)[kGroup]) {
    struct __attribute__((packed, aligned(2))) Piece { uint16_t v[8]; };
    if (kGroup * g + kGroup <= V) {
        const Piece p = *reinterpret_cast<const Piece*>(row + kGroup * g);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) x[i] = __builtin_bit_cast(float, (unsigned)p.v[i] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) x[i] = kGroup * g + i < V ? element(row, kGroup * g + i) : 0.f;
    }
}

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// A workgroup to a sequence.  The first wavefront walks along the tree: the numbers that decide about a token (its probabilities in its parent's rows, its random number) are
// fetched for all tokens at once, so a step is a search for the next child in LDS.  The vocabulary is read only where a sum over it is needed: for S_k, where another sibling follows a refused
// one, and for the next token.  That one is found by halving the row in steps of the number of wavefronts: every wavefront sums one piece of the row, the piece in which the running sum
// passes the random number is cut again, and the last is searched by one wavefront.
// What bounds it is latency, and for large vocabularies the one CU that reads a row.
template <class T, bool DRAFT, int NT>
__global__ __launch_bounds__(NT) void tree_verify_kernel(TreeVerifyArgs a) {
    constexpr int NW = NT / 64;
    __shared__ int s_up[HG_MAX_TREE], s_tok[HG_MAX_TREE];
    __shared__ float s_u[HG_MAX_TREE], s_p[HG_MAX_TREE], s_q[DRAFT ? HG_MAX_TREE : 1];
    __shared__ double s_sum[NW], s_c;
    __shared__ int s_cur, s_more, s_kept;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = (int)blockIdx.x;
    const TreeSeq sq = tree_seq(a.q_off, a.rows, b);
    const int take = min(sq.n, a.max_new), V = a.V;
    if (take == 0) {
        if (tid == 0) { a.accepted[b] = 0; a.next[b] = -1; }
        return;
    }
    const T* const target = static_cast<const T*>(a.target);
    const T* const draft = static_cast<const T*>(a.draft);
    for (int t = tid; t < take; t += NT) {
        int up = a.parents[sq.q0 + t];
        const int x = a.tokens[sq.q0 + t];
        if (up < 0 || up >= t) up = -1;
        float p = 0.f, q = 0.f;
        if (up >= 0 && x >= 0 && x < V) {
            p = element(target + (int64_t)(sq.q0 + up) * a.target_stride, x);
            if constexpr (DRAFT) q = element(draft + (int64_t)(sq.q0 + up) * a.draft_stride, x);
        }
        s_up[t] = up;
        s_tok[t] = x;
        s_u[t] = a.u[sq.q0 + t];
        s_p[t] = counted(p);
        if constexpr (DRAFT) s_q[t] = counted(q);
    }
    __syncthreads();

    // ---- the walk ----
    const auto find = [&](int from, int to, auto what) -> int {      // the first t in [from, to) with what(t), or `to`; of one wavefront
        for (int t0 = from; t0 < to; t0 += 64) {
            const int t = t0 + lane;
            const unsigned long long hit = __ballot(t < to && what(t));
            if (hit) return t0 + __builtin_ctzll(hit);
        }
        return to;
    };
    // Sum over the vocabulary of what is left: max(0, p - c q), or p but for the refused tokens (those of `cur`'s children).  Groups [from, to) to this wavefront.
    int cur = 0;
    double c = 0.0;
    bool without = false;      // (no draft) refused tokens count as 0
    const auto weights = [&](int g, double (&x)[kGroup]) {
        float p[kGroup];
        load8(target + (int64_t)(sq.q0 + cur) * a.target_stride, g, V, p);
        if constexpr (DRAFT) {
            float q[kGroup];
            load8(draft + (int64_t)(sq.q0 + cur) * a.draft_stride, g, V, q);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) x[i] = fmax(0.0, (double)counted(p[i]) - c * (double)counted(q[i]));
        } else {
            if (without)
                for (int t = cur + 1; t < take; ++t) {
                    const unsigned at = (unsigned)(s_tok[t] - kGroup * g);
                    if (at < (unsigned)kGroup && s_up[t] == cur) {
#pragma unroll
                        for (int i = 0; i < kGroup; ++i)
                            if ((unsigned)i == at) p[i] = 0.f;
                    }
                }
#pragma unroll
            for (int i = 0; i < kGroup; ++i) x[i] = (double)counted(p[i]);
        }
    };
    const auto sum_of = [&](int from, int to) -> double {
        double s = 0.0;
        for (int g = from + lane; g < to; g += 64) {
            double x[kGroup];
            weights(g, x);
#pragma unroll
            for (int i = 0; i < kGroup; ++i) s += x[i];
        }
        return wave_sum(s);
    };
    const int groups = (V + kGroup - 1) / kGroup;
    const auto piece_of = [&](int n) { return (n + NW - 1) / NW; };

    int t = 1, kept = 1;
    double S = 1.0;
    bool stale = false;      // S has to be taken before the next test
    while (true) {
        if (w == 0) {
            bool more = false;
            while (true) {
                t = find(t, take, [&](int i) { return s_up[i] == cur; });
                if (t >= take) break;
                if (DRAFT && stale) { more = true; break; }
                const double u = s_u[t];
                double p = s_p[t];
                bool yes;
                if constexpr (DRAFT) {
                    const double q = s_q[t];
                    yes = u * q * S < fmax(0.0, p - c * q);
                } else {
                    const int x = s_tok[t], first = find(cur + 1, t, [&](int i) { return s_up[i] == cur && s_tok[i] == x; });
                    if (first < t) p = 0.0;      // a sibling had the token
                    yes = p > 0.0 && u * S < p;
                }
                if (yes) {
                    if (lane == 0) a.path[sq.q0 + kept] = t;
                    ++kept;
                    cur = t;
                    c = 0.0;
                    S = 1.0;
                } else if constexpr (DRAFT) {
                    c += S;
                    stale = true;
                } else {
                    S -= p;
                }
                ++t;
            }
            if (lane == 0) { s_cur = cur; s_c = c; s_more = more; s_kept = kept; }
        }
        __syncthreads();
        cur = __builtin_amdgcn_readfirstlane(s_cur);
        c = s_c;
        if (!s_more) break;
        const int piece = piece_of(groups);
        const double part = sum_of(min(w * piece, groups), min((w + 1) * piece, groups));
        if (lane == 0) s_sum[w] = part;
        __syncthreads();
        S = 0.0;
        for (int i = 0; i < NW; ++i) S += s_sum[i];
        stale = false;
    }
    kept = s_kept;
    for (int i = tid; i < take; i += NT)
        if (i == 0 || i >= kept) a.path[sq.q0 + i] = i == 0 ? 0 : -1;

    // ---- the next token ----
    without = true;
    const double un = a.u_next[b];
    double before = 0.0, aim = 0.0;      // sum of the pieces before the one in hand; what the running sum has to pass
    int from = 0, to = groups;
    for (int level = 0; level < 16; ++level) {
        const int piece = piece_of(to - from);
        const double part = sum_of(min(from + w * piece, to), min(from + (w + 1) * piece, to));
        __syncthreads();      // (the sums of the level before have been read)
        if (lane == 0) s_sum[w] = part;
        __syncthreads();
        if (level == 0) {
            double all = 0.0;
            for (int i = 0; i < NW; ++i) all += s_sum[i];
            if (!(all > 0.0)) {      // nothing is left: the draw is from p itself, if that has anything
                if (c == 0.0 && !without) {
                    if (tid == 0) { a.accepted[b] = kept; a.next[b] = -1; }
                    return;
                }
                c = 0.0;
                without = false;
                level = -1;
                continue;
            }
            aim = un * all;
        }
        // the first piece in which the running sum passes; none (rounding, or a number above the range): the last that has anything
        double run = before, base = before;
        int at = -1;
        for (int i = 0; i < NW; ++i) {
            if (s_sum[i] > 0.0) {
                at = i;
                base = run;
                run += s_sum[i];
                if (run > aim) break;
            }
        }
        before = base;
        const int f = from;
        from = min(f + at * piece, to);
        to = min(f + (at + 1) * piece, to);
        if (to - from <= 64) break;
    }
    if (w > 0) return;
    {
        const int g = from + lane;
        double x[kGroup] = {};
        if (g < to) weights(g, x);
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) s += x[i];
        double run = s;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double o = __shfl_up(run, d);
            if (lane >= d) run += o;
        }
        run += before;
        const unsigned long long some = __ballot(s > 0.0), passes = __ballot(s > 0.0 && run > aim);
        const int pick = passes ? __builtin_ctzll(passes) : 63 - __builtin_clzll(some);
        if (lane == pick) {
            run -= s;
            int y = -1;
            bool done = false;
#pragma unroll
            for (int i = 0; i < kGroup; ++i) {
                run += x[i];
                if (!done && x[i] > 0.0) {
                    y = kGroup * g + i;
                    done = run > aim;
                }
            }
            a.accepted[b] = kept;
            a.next[b] = y;
        }
    }
}

// Greedy decoding: the target's tokens are there already.  A wavefront to a sequence.
__global__ __launch_bounds__(64) void tree_match_kernel(TreeVerifyArgs a) {
    __shared__ int s_up[HG_MAX_TREE], s_tok[HG_MAX_TREE], s_says[HG_MAX_TREE];
    const int lane = threadIdx.x, b = (int)blockIdx.x;
    const TreeSeq sq = tree_seq(a.q_off, a.rows, b);
    const int take = min(sq.n, a.max_new);
    if (take == 0) {
        if (lane == 0) { a.accepted[b] = 0; a.next[b] = -1; }
        return;
    }
    for (int t = lane; t < take; t += 64) {
        const int up = a.parents[sq.q0 + t];
        s_up[t] = up < t ? up : -1;
        s_tok[t] = a.tokens[sq.q0 + t];
        s_says[t] = static_cast<const int32_t*>(a.target)[sq.q0 + t];
    }
    __syncthreads();
    int cur = 0, kept = 1;
    for (int t0 = 0; t0 < take;) {
        const int t = t0 + lane;
        const unsigned long long hit = __ballot(t > cur && t < take && s_up[t] == cur && s_tok[t] == s_says[cur]);
        if (hit == 0) { t0 += 64; continue; }
        cur = t0 + __builtin_ctzll(hit);      // (its children lie behind it: the search goes on in the same 64)
        if (lane == 0) a.path[sq.q0 + kept] = cur;
        ++kept;
    }
    for (int i = lane; i < take; i += 64)
        if (i == 0 || i >= kept) a.path[sq.q0 + i] = i == 0 ? 0 : -1;
    if (lane == 0) { a.accepted[b] = kept; a.next[b] = s_says[cur]; }
}

// ---- the accepted rows' move -----------------------------------------------------------------------------------------------------

// A thread moves one 16-byte piece of every accepted row, in order: row i comes from row path[i] >= i, so a place has been read, by the thread that writes it, before it is written.
// Bound by HBM where there are many layers, by latency (lengths, path, table, rows) where there are few.
constexpr int kMoves = 256;        // rows whose places are looked up at a time
constexpr int kAtOnce = 8;         // rows that are in flight
__global__ __launch_bounds__(256) void tree_keep_kernel(TreeKeepArgs a) {
    __shared__ int s_src[kMoves], s_dst[kMoves];
    const int b = (int)blockIdx.x, tid = threadIdx.x;
    const TreeSeq sq = tree_seq(a.q_off, a.rows, b);
    const int take = min(sq.n, a.max_new), kept = min(max(a.accepted[b], 0), take);
    const int before = max(a.lengths[b], 0) - sq.n;      // rows of the context (below 0: some of the tree's rows have no place)
    if (blockIdx.y == 0 && blockIdx.z == 0 && tid == 0) a.new_lengths[b] = max(before + kept, 0);
    if (a.layers == 0) return;
    unsigned char* const pool = a.pool[blockIdx.y];
    const int piece = (int)blockIdx.z * (int)blockDim.x + tid;
    const int64_t rowb = 16LL * a.pieces;
    const auto place = [&](int64_t j) -> int {      // pool row of the sequence's row j, -1: none
        if (j < 0 || (j >> a.shift) >= a.stride) return -1;
        const int page = a.table[(int64_t)b * a.stride + (j >> a.shift)];
        return page < 0 || page >= a.n_pages ? -1 : (page << a.shift) + (int)(j & ((1 << a.shift) - 1));
    };
    for (int i0 = 0; i0 < kept; i0 += kMoves) {
        const int m = min(kept - i0, kMoves);
        __syncthreads();
        for (int i = tid; i < m; i += (int)blockDim.x) {
            const int from = a.path[sq.q0 + i0 + i];
            int src = -1, dst = -1;
            if (from > i0 + i && from < sq.n) {      // (its own place already, or none of the tree's: nothing moves)
                src = place((int64_t)before + from);
                dst = place((int64_t)before + i0 + i);
            }
            s_src[i] = dst < 0 ? -1 : src;
            s_dst[i] = dst;
        }
        __syncthreads();
        if (piece < a.pieces) {
            for (int i = 0; i < m; i += kAtOnce) {
                uint4 v[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int src = i + k < m ? s_src[i + k] : -1;
                    if (src >= 0) v[k] = *reinterpret_cast<const uint4*>(pool + src * rowb + 16 * piece);
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
                    if (i + k < m && s_src[i + k] >= 0) *reinterpret_cast<uint4*>(pool + s_dst[i + k] * rowb + 16 * piece) = v[k];
            }
        }
    }
}

}  // namespace

hipError_t launch_tree_masks(const TreeMaskArgs& a, hipStream_t s) {
    if (a.max_new <= 64) {
        tree_masks_kernel<<<(unsigned)((a.B + 3) / 4), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    constexpr int bytes = (kMaskWords + HG_MAX_TREE) * 4;
    static bool attr_set[64] = {};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&tree_masks_long_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    tree_masks_long_kernel<<<(unsigned)a.B, kMaskThreads, bytes, s>>>(a);
    return hipGetLastError();
}

template <class T, bool DRAFT>
static hipError_t launch_verify_t(const TreeVerifyArgs& a, hipStream_t s) {
    if (a.V <= 8192) tree_verify_kernel<T, DRAFT, 256><<<(unsigned)a.B, 256, 0, s>>>(a);
    else tree_verify_kernel<T, DRAFT, 1024><<<(unsigned)a.B, 1024, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_tree_verify(const TreeVerifyArgs& a, int p_dtype, hipStream_t s) {
    if (p_dtype == HG_TOKENS) {
        tree_match_kernel<<<(unsigned)a.B, 64, 0, s>>>(a);
        return hipGetLastError();
    }
    if (p_dtype == HG_F32) return a.draft ? launch_verify_t<float, true>(a, s) : launch_verify_t<float, false>(a, s);
    return a.draft ? launch_verify_t<uint16_t, true>(a, s) : launch_verify_t<uint16_t, false>(a, s);
}

hipError_t launch_tree_keep(const TreeKeepArgs& a, hipStream_t s) {
    const int threads = std::min(256, (std::max(a.pieces, 1) + 63) / 64 * 64);
    const dim3 grid((unsigned)a.B, (unsigned)std::max(2 * a.layers, 1), (unsigned)std::max((a.pieces + threads - 1) / threads, 1));
    tree_keep_kernel<<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace hg
