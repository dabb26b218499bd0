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

// More: a workgroup to 64 tokens of a sequence.  It finds the bits of the blocks of 64 up to its own, each for itself; a token's row is then what its own bits say of its block, of the
// block that its topmost ancestor there leads to what the bits of that one say, and so on: at most one token of every block is looked at, 8 lanes to a row, which is written as it goes.
// What bounds it is latency: offsets, parents, the doubling, up to 16 looks into LDS.  64 trees of 64 to 1024 tokens, 4.7 MB out, 6.4 us (a workgroup to a sequence, whose blocks took over each
// other's rows one after another, 14.5).
constexpr int kMaskThreads = 512;
__global__ __launch_bounds__(kMaskThreads) void tree_masks_long_kernel(TreeMaskArgs a) {
    __shared__ unsigned long long s_bits[HG_MAX_TREE];
    __shared__ int s_out[HG_MAX_TREE];      // the parent of the topmost token that one follows from in its block, which lies in an earlier one, or -1
    const int tid = threadIdx.x, lane = tid & 63, own = (int)blockIdx.y;
    const TreeSeq s = tree_seq(a.q_off, a.rows, (int)blockIdx.x);
    const int take = min(s.n, a.max_new);
    if (64 * own >= take) return;
    for (int k = tid >> 6; k <= own; k += kMaskThreads / 64) {
        const int t = 64 * k + lane;
        int up = t < take ? a.parents[s.q0 + t] : -1;
        if (up < 0 || up >= t) up = -1;
        unsigned long long bits;
        int top;
        ancestors64(up >= 64 * k ? up & 63 : -1, lane, bits, top);
        s_bits[t] = bits;
        s_out[t] = __shfl(up, top);
    }
    __syncthreads();
    const int t = 64 * own + (tid >> 3), l = tid & 7;
    if (t >= take) return;
    unsigned long long mine[2] = {0, 0};      // of blocks l and l + 8
    int n = -1;
    for (int e = t; e >= 0; e = s_out[e]) {
        const unsigned long long bits = s_bits[e];
        n += __builtin_popcountll(bits);
        if ((e >> 6) == l) mine[0] = bits;
        if ((e >> 6) == l + 8) mine[1] = bits;
    }
    uint32_t* const row = a.masks + (int64_t)(s.q0 + t) * a.words;
    const bool pairs = a.words % 2 == 0 && reinterpret_cast<uintptr_t>(a.masks) % 8 == 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = 2 * l + 16 * i;
        if (pairs) {
            if (w < a.words) *reinterpret_cast<unsigned long long*>(row + w) = mine[i];
        } else {
            if (w < a.words) row[w] = (uint32_t)mine[i];
            if (w + 1 < a.words) row[w + 1] = (uint32_t)(mine[i] >> 32);
        }
    }
    for (int w = 32 + l; w < a.words; w += 8) row[w] = 0u;
    if (a.depth && l == 0) a.depth[s.q0 + t] = n;
}

// ---- verification ----------------------------------------------------------------------------------------------------------------

constexpr int kGroup = 8;          // elements that a lane takes at a time

// What is no positive finite number counts as 0.  Such numbers, and zero, are those whose bits are at most kMost as an unsigned number.
constexpr unsigned kMost = 0x7f7fffffu;
__device__ __forceinline__ unsigned bits_of(float x) { return __builtin_bit_cast(unsigned, x); }
__device__ __forceinline__ float counted(float x) { return bits_of(x) <= kMost ? x : 0.f; }
__device__ __forceinline__ float element(const float* row, int64_t i) { return row[i]; }
__device__ __forceinline__ float element(const uint16_t* row, int64_t i) { return __builtin_bit_cast(float, (unsigned)row[i] << 16); }

// Elements 8 g .. 8 g + 7 of a row of V, as they are or as pairs; those behind its end are 0.  Rows begin anywhere, so the loads are of unaligned pieces.
template <class T>
struct Group;
template <>
struct Group<float> {
    unsigned v[8];
    __device__ __forceinline__ void load_full(const float* row, int g) {
        struct __attribute__((packed, aligned(4))) Piece { unsigned v[4]; };
        const Piece lo = *reinterpret_cast<const Piece*>(row + kGroup * g), hi = *reinterpret_cast<const Piece*>(row + kGroup * g + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = lo.v[i]; v[4 + i] = hi.v[i]; }
    }
    __device__ __forceinline__ void load(const float* row, int g, int V) {
        if (kGroup * g + kGroup <= V) {
            load_full(row, g);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = kGroup * g + i < V ? bits_of(row[kGroup * g + i]) : 0u;
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0u;
    }
    __device__ __forceinline__ unsigned get(int i) const { return v[i]; }
};
template <>
struct Group<uint16_t> {
    unsigned v[4];
    __device__ __forceinline__ void load_full(const uint16_t* row, int g) {
        struct __attribute__((packed, aligned(2))) Piece { unsigned v[4]; };
        const Piece p = *reinterpret_cast<const Piece*>(row + kGroup * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = p.v[i];
    }
    __device__ __forceinline__ void load(const uint16_t* row, int g, int V) {
        if (kGroup * g + kGroup <= V) {
            load_full(row, g);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = kGroup * g + 2 * i;
                v[i] = (e < V ? (unsigned)row[e] : 0u) | (e + 1 < V ? (unsigned)row[e + 1] : 0u) << 16;
            }
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0u;
    }
    __device__ __forceinline__ unsigned get(int i) const { return i & 1 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16; }
};

__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// A workgroup to a sequence.  The first wavefront walks along the tree: the numbers that decide about a token (its probabilities in its parent's rows, its random number) are
// fetched for all tokens at once, so a step is a search for the next child among 64 tokens in registers.  The vocabulary is read only where a sum over it is needed: for S_k, where another
// sibling follows a refused one, and once for the next token: every wavefront sums one piece of the row, and the piece in which the running sum passes the random number is read once more, a few
// elements by every thread.
// What bounds it is latency, and for large vocabularies the one CU that reads a row.
//
// One CU takes in some 40 GB/s of a row and converts as much, so where rows are long and sequences few the first of these sums, which for chains and without drafts is the only one, is
// shared out: kFirst, `nsplit` workgroups of four wavefronts to a sequence, walk as far as that sum, each for itself, and take a piece of it per wavefront; kRest goes on from there.
enum { kWhole, kFirst, kRest };
constexpr int kFirstWaves = 4;
template <class T, bool DRAFT, int NT, int PART>
__global__ __launch_bounds__(NT) void tree_verify_kernel(TreeVerifyArgs a) {
    constexpr int NW = NT / 64;
    static_assert(PART != kFirst || NW == kFirstWaves, "");
    constexpr int U = 64 / (sizeof(Group<T>) / 4 * (DRAFT ? 2 : 1));      // groups of a lane that are in flight: 64 registers of them
    constexpr int kFilter = 1 << 14;      // places that say whether a group of elements may have a refused token
    __shared__ int s_up[HG_MAX_TREE], s_tok[HG_MAX_TREE];
    __shared__ float s_u[HG_MAX_TREE], s_p[HG_MAX_TREE], s_q[DRAFT ? HG_MAX_TREE : 1];
    __shared__ unsigned s_filter[DRAFT ? 1 : kFilter / 32];
    __shared__ double s_sum[NW], s_cut[NW], s_c;
    __shared__ double s_part[PART == kRest ? kVerifySplits * kFirstWaves : 1];
    __shared__ int s_cur, s_more, s_kept, s_refused;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = PART == kFirst ? (int)blockIdx.x / a.nsplit : (int)blockIdx.x, slice = PART == kFirst ? (int)blockIdx.x - b * a.nsplit : 0;
    const int parts = PART == kWhole ? NW : a.nsplit * kFirstWaves;
    const TreeSeq sq = tree_seq(a.q_off, a.rows, b);
    const int take = min(sq.n, a.max_new), V = a.V;
    if (take == 0) {
        if (PART != kFirst && tid == 0) { a.accepted[b] = 0; a.next[b] = -1; }
        return;
    }
    TreeVerifyState from_first{0, 1, 1, 1, 0.0};
    if constexpr (PART == kRest) {
        from_first = a.state[b];
        for (int i = tid; i < parts; i += NT) s_part[i] = a.parts[(int64_t)b * parts + i];
    }
    const bool walk_on = from_first.more != 0;
    const T* const target = static_cast<const T*>(a.target);
    const T* const draft = static_cast<const T*>(a.draft);
    for (int t = tid; t < (DRAFT && !walk_on ? 0 : take); t += NT) {
        int up = a.parents[sq.q0 + t];
        const int x = a.tokens[sq.q0 + t];
        if (up < 0 || up >= t) up = -1;
        float p = 0.f, q = 0.f;
        if (walk_on && up >= 0 && x >= 0 && x < V) {
            p = element(target + (int64_t)(sq.q0 + up) * a.target_stride, x);
            if constexpr (DRAFT) q = element(draft + (int64_t)(sq.q0 + up) * a.draft_stride, x);
        }
        s_up[t] = up;
        s_tok[t] = x;
        s_u[t] = a.u[sq.q0 + t];
        s_p[t] = counted(p);
        if constexpr (DRAFT) s_q[t] = counted(q);
    }
    const double un = a.u_next[b];
    if constexpr (!DRAFT)
        for (int i = tid; i < kFilter / 32; i += NT) s_filter[i] = 0;
    __syncthreads();

    int cur = 0;
    double c = 0.0;
    bool without = false;      // (no draft) refused tokens count as 0
    // What is left of a group's elements: max(0, p - c q), or p but for the refused tokens, which are s_tok[0 .. s_refused) when they are asked for.
    const auto weights = [&](int g, const Group<T>& p, const Group<T>& q, double (&x)[kGroup]) {
        unsigned most = p.get(0);
#pragma unroll
        for (int i = 1; i < kGroup; ++i) most = max(most, p.get(i));
        if constexpr (DRAFT) {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) most = max(most, q.get(i));
        }
        const bool plain = most <= kMost;
        if constexpr (DRAFT) {
            if (__builtin_expect(plain, 1)) {
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                    x[i] = fmax(0.0, fma(-c, (double)__builtin_bit_cast(float, q.get(i)), (double)__builtin_bit_cast(float, p.get(i))));
            } else {
#pragma unroll
                for (int i = 0; i < kGroup; ++i)
                    x[i] = fmax(0.0, fma(-c, (double)counted(__builtin_bit_cast(float, q.get(i))), (double)counted(__builtin_bit_cast(float, p.get(i)))));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kGroup; ++i) x[i] = (double)__builtin_bit_cast(float, p.get(i));
            if (__builtin_expect(!plain, 0)) {
#pragma unroll
                for (int i = 0; i < kGroup; ++i) x[i] = (double)counted(__builtin_bit_cast(float, p.get(i)));
            }
            const unsigned place = (unsigned)g & (kFilter - 1);
            if (without && (s_filter[place >> 5] >> (place & 31) & 1u)) {
                for (int k = 0; k < s_refused; ++k) {
                    const unsigned at = (unsigned)(s_tok[k] - kGroup * g);
#pragma unroll
                    for (int i = 0; i < kGroup; ++i)
                        if ((unsigned)i == at) x[i] = 0.0;
                }
            }
        }
    };
    const auto load = [&](int g, Group<T>& p, Group<T>& q) {
        p.load(target + (int64_t)(sq.q0 + cur) * a.target_stride, g, V);
        if constexpr (DRAFT) {
            if (c != 0.0) q.load(draft + (int64_t)(sq.q0 + cur) * a.draft_stride, g, V);
            else q.clear();
        }
    };
    const auto total = [](const double (&x)[kGroup]) -> double { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); };
    const int groups = (V + kGroup - 1) / kGroup, piece = (groups + NW - 1) / NW;
    const int full = V / kGroup;      // groups without an end of the row in them
    const auto sum_up = [&](int which, int piece) -> double {      // of one piece of the row, by a wavefront
        const T* const prow = target + (int64_t)(sq.q0 + cur) * a.target_stride;
        const T* const qrow = DRAFT ? draft + (int64_t)(sq.q0 + cur) * a.draft_stride : nullptr;
        const int to = min((which + 1) * piece, full);
        double all = 0.0;
        for (int first = which * piece; first < to; first += 64 * U) {
            Group<T> p[U], q[U];
            // (every lane loads, those past the end the last group once more: a load under a condition of a lane's own is waited for before the next)
#pragma unroll
            for (int k = 0; k < U; ++k) p[k].load_full(prow, min(first + 64 * k + lane, to - 1));
            if constexpr (DRAFT) {
                if (c != 0.0) {
#pragma unroll
                    for (int k = 0; k < U; ++k) q[k].load_full(qrow, min(first + 64 * k + lane, to - 1));
                } else {
#pragma unroll
                    for (int k = 0; k < U; ++k) q[k].clear();
                }
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (first + 64 * k >= to) break;
                double x[kGroup];
                weights(min(first + 64 * k + lane, to - 1), p[k], q[k], x);
                all += first + 64 * k + lane < to ? total(x) : 0.0;
            }
        }
        if (full < groups && full / piece == which && lane == 0) {      // what is left behind them
            Group<T> p, q;
            double x[kGroup];
            load(full, p, q);
            weights(full, p, q, x);
            all += total(x);
        }
        return wave_sum(all);
    };
    // ... of NW or of `parts` pieces
    const auto sum_whole = [&]() {
        const double x = sum_up(w, piece);
        if (lane == 0) s_sum[w] = x;
    };

    // ---- the walk ----
    int t = from_first.t, kept = from_first.kept;
    double S = 1.0;
    bool stale = false;      // S has to be taken before the next test
    if constexpr (PART == kRest) {
        cur = from_first.cur;
        c = from_first.c;
        S = 0.0;
        for (int i = lane; i < parts; i += 64) S += s_part[i];
        S = wave_sum(S);
    }
    const double first_sum = S;
    while (true) {
        if (w == 0) {
            bool more = false;
            while (walk_on && t < take) {
                // 64 tokens, those before t among them that no one asks for any more
                const int t0 = t & ~63, at = min(t0 + lane, take - 1);
                const int up = t0 + lane < take ? s_up[at] : -1, x = s_tok[at];
                const float u = s_u[at], p = s_p[at], q = DRAFT ? s_q[at] : 0.f;
                while (true) {
                    const unsigned long long children = t - t0 < 64 ? __ballot(up == cur) & (~0ull << (t - t0)) : 0ull;
                    if (children == 0) {
                        t = t0 + 64;
                        break;
                    }
                    const int i = __builtin_ctzll(children);
                    t = t0 + i;
                    if (DRAFT && stale) {
                        more = true;
                        break;
                    }
                    const auto of_lane = [&](float v) -> double { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), i)); };
                    const double ut = of_lane(u);
                    double pt = of_lane(p);
                    bool yes;
                    if constexpr (DRAFT) {
                        yes = ut * of_lane(q) * S < fmax(0.0, pt - c * of_lane(q));
                    } else {
                        const int xt = __builtin_amdgcn_readlane(x, i);
                        bool had = (__ballot(up == cur && x == xt) & ((1ull << i) - 1)) != 0;      // a sibling has had the token
                        for (int e0 = cur & ~63; e0 < t0; e0 += 64) had |= __any(s_up[e0 + lane] == cur && s_tok[e0 + lane] == xt) != 0;
                        if (had) pt = 0.0;
                        yes = pt > 0.0 && ut * S < pt;
                    }
                    if (yes) {
                        if (lane == 0 && slice == 0) a.path[sq.q0 + kept] = t;
                        ++kept;
                        cur = t;
                        c = 0.0;
                        S = 1.0;
                    } else if constexpr (DRAFT) {
                        c += S;
                        stale = true;
                    } else {
                        S -= pt;
                    }
                    ++t;
                }
                if (more) break;
            }
            if constexpr (!DRAFT) {      // the refused tokens, packed (none moves behind one that has yet to be read), and their groups
                int n = 0;
                for (int t0 = cur & ~63; t0 < take; t0 += 64) {
                    const bool mine = t0 + lane < take && s_up[t0 + lane] == cur;
                    const int x = mine ? s_tok[t0 + lane] : -1;
                    const unsigned long long some = __ballot(mine);
                    if (mine) {
                        s_tok[n + __builtin_popcountll(some & ((1ull << lane) - 1))] = x;
                        if (x >= 0) atomicOr(&s_filter[(x / kGroup & (kFilter - 1)) >> 5], 1u << (x / kGroup & 31));
                    }
                    n += __builtin_popcountll(some);
                }
                if (lane == 0) s_refused = n;
            }
            if (lane == 0) { s_cur = cur; s_c = c; s_more = more; s_kept = kept; }
            if (PART == kFirst && slice == 0 && lane == 0) a.state[b] = TreeVerifyState{cur, t, kept, more, c};
        }
        __syncthreads();
        cur = __builtin_amdgcn_readfirstlane(s_cur);
        c = s_c;
        if (PART == kFirst || !s_more) break;
        sum_whole();
        __syncthreads();
        S = 0.0;
        for (int i = 0; i < NW; ++i) S += s_sum[i];
        stale = false;
    }
    without = !DRAFT && s_refused > 0;
    if constexpr (PART == kFirst) {
        const int which = slice * NW + w;
        const double x = sum_up(which, (groups + parts - 1) / parts);
        if (lane == 0) a.parts[(int64_t)b * parts + which] = x;
        return;
    }
    kept = s_kept;
    for (int i = tid; i < take; i += NT)
        if (i == 0 || i >= kept) a.path[sq.q0 + i] = i == 0 ? 0 : -1;

    // ---- the next token ----
    bool whole = DRAFT ? c == 0.0 : !without;      // the draw is from p as it is
    bool shared_out = PART == kRest && !walk_on && first_sum > 0.0;      // the sums of the row's pieces are there
    double all = first_sum;
    while (!shared_out) {
        sum_whole();
        __syncthreads();
        all = 0.0;
        for (int i = 0; i < NW; ++i) all += s_sum[i];
        if (all > 0.0 || whole) break;
        c = 0.0;      // nothing is left: the draw is from p itself
        without = false;
        whole = true;
        __syncthreads();      // (everyone has read the sums)
    }
    if (!(all > 0.0)) {
        if (tid == 0) { a.accepted[b] = kept; a.next[b] = -1; }
        return;
    }
    // Everywhere below: the first in which the running sum passes `aim`; if there is none (rounding, or a random number that is none), the last that has anything.
    const double aim = un * all;
    const auto scan = [&](double x) -> double {      // the running sum over the lanes, this one's included
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double o = __shfl_up(x, d);
            if (lane >= d) x += o;
        }
        return x;
    };
    const auto pick = [&](bool some, bool passes) -> int {      // a lane, or -1
        const unsigned long long p = __ballot(some && passes), s = __ballot(some);
        return p ? __builtin_ctzll(p) : s ? 63 - __builtin_clzll(s) : -1;
    };
    const auto cut = [&](const double* sums, int n, double before, double& base) -> int {      // which of n sums, and the sum of those before it
        int at = 0;
        base = before;
        for (int i0 = 0; i0 < n; i0 += 64) {
            const double own = i0 + lane < n ? sums[i0 + lane] : 0.0, run = before + scan(own);
            const int i = pick(own > 0.0, run > aim);
            if (i >= 0) {
                at = i0 + i;
                base = __shfl(run - own, i);
            }
            if (__any(own > 0.0 && run > aim)) break;
            before = __shfl(run, 63);
        }
        return at;
    };
    double before;
    const int size = shared_out ? (groups + parts - 1) / parts : piece, first = (shared_out ? cut(s_part, parts, 0.0, before) : cut(s_sum, NW, 0.0, before)) * size;
    const int each = (size + NT - 1) / NT, from = min(first + tid * each, groups), to = min(min(from + each, first + size), groups);      // the piece is cut into as many groups to a thread
    double own = 0.0;
    for (int g = from; g < to; ++g) {
        Group<T> p, q;
        double x[kGroup];
        load(g, p, q);
        weights(g, p, q, x);
        own += total(x);
    }
    double run = scan(own);
    if (lane == 63) s_cut[w] = run;
    __syncthreads();
    double base;
    if (cut(s_cut, NW, before, base) != w) return;
    run += base;
    if (lane != max(pick(own > 0.0, run > aim), 0)) return;
    run -= own;
    int y = -1;
    for (int g = from; g < to; ++g) {
        Group<T> p, q;
        double x[kGroup];
        load(g, p, q);
        weights(g, p, q, x);
        bool done = false;
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            run += x[i];
            if (!done && x[i] > 0.0) {
                y = kGroup * g + i;
                done = run > aim;
            }
        }
        if (done) break;
    }
    a.accepted[b] = kept;
    a.next[b] = y;
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
// Bound by HBM where there are many layers, by latency (lengths, path, table, rows) where there are few.  Stores go past the caches: 64 sequences with 7 rows to move, 32 layers of 8 heads
// of 128, 21.0 us so, 5.0 TB/s, and 45.6 the ordinary way.
constexpr int kMoves = 256;        // rows whose places are looked up at a time
constexpr int kAtOnce = 8;         // rows that are in flight
typedef unsigned Piece __attribute__((ext_vector_type(4)));
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
                Piece v[kAtOnce];
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int src = i + k < m ? s_src[i + k] : -1;
                    if (src >= 0) v[k] = *reinterpret_cast<const Piece*>(pool + src * rowb + 16 * piece);
                }
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k)
                    if (i + k < m && s_src[i + k] >= 0) __builtin_nontemporal_store(v[k], reinterpret_cast<Piece*>(pool + s_dst[i + k] * rowb + 16 * piece));
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
    const int blocks = (a.max_new + 63) / 64, most = (int)(0xffffffffu / (unsigned)(kMaskThreads * blocks));      // sequences of a launch, which has fewer than 2^32 threads
    for (int first = 0; first < a.B; first += most) {
        TreeMaskArgs some = a;
        some.q_off += first;
        some.B = std::min(most, a.B - first);
        tree_masks_long_kernel<<<dim3((unsigned)some.B, (unsigned)blocks), kMaskThreads, 0, s>>>(some);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class T, bool DRAFT>
static hipError_t launch_verify_t(const TreeVerifyArgs& a, hipStream_t s) {
    if (a.nsplit > 1) {
        tree_verify_kernel<T, DRAFT, 64 * kFirstWaves, kFirst><<<(unsigned)(a.B * a.nsplit), 64 * kFirstWaves, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        tree_verify_kernel<T, DRAFT, 1024, kRest><<<(unsigned)a.B, 1024, 0, s>>>(a);
    } else if (a.V <= 8192) {
        tree_verify_kernel<T, DRAFT, 256, kWhole><<<(unsigned)a.B, 256, 0, s>>>(a);
    } else {
        tree_verify_kernel<T, DRAFT, 1024, kWhole><<<(unsigned)a.B, 1024, 0, s>>>(a);
    }
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
