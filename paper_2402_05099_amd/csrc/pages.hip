// Bookkeeping of a paged cache on the GPU: block tables and slots from the requests' lengths, and the write of new K/V rows to their slots.
#include <algorithm>
#include <type_traits>

#include "ragged.h"

namespace hg {

namespace {
constexpr int kThreads = 256;
constexpr int kPer = 4;                          // sequences that a thread looks at
constexpr int kSeqs = kThreads * kPer;           // ... and a workgroup at a time
constexpr int kTokens = 1024;                    // tokens that a workgroup finds the slots of
}

// With have = ceil(len / ps) pages in use and want = ceil(min(len + n, capacity) / ps) needed, sequence b's new pages are the entries
// [first, first + want - have) of the list of free ones, first = the new pages of the sequences before it; token t of it becomes row
// len + t.  Two prefix sums over the sequences (tokens, new pages) are all that ties the sequences to each other; every workgroup takes them
// for itself, so that one launch does: 8 bytes per sequence out of L2 instead of a second launch.  A new page begins with a new token, so the
// page's entry in the table is written where that token's slot is found.
// What bounds it is latency: loads, two scans, the search of a token's sequence (ten looks into LDS), its page, 4.1 us for four sequences with 125 tokens, of which
// the launch is most (3.5 to 4.4 on different boxes); 512 sequences with 131 thousand tokens 6.1 us, 0.6 MB in and out.  (256 sequences at a time, the pages of a sequence entered by the one
// workgroup that has it, 20.5 us.)
__global__ __launch_bounds__(kThreads) void page_slots_kernel(SlotArgs a) {
    __shared__ int s_q0[kSeqs], s_len[kSeqs], s_have[kSeqs], s_first[kSeqs], s_sum[2][kThreads / 64];
    const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
    const int ps_mask = (1 << a.shift) - 1, cap = a.stride << a.shift;
    const int tok0 = (int)blockIdx.x * kTokens, tok1 = min(tok0 + kTokens, a.rows);
    int base_q = 0, base_p = 0;
    for (int b0 = 0; b0 < a.B; b0 += kSeqs) {
        const int b = b0 + kPer * tid;
        int len[kPer], n[kPer], have[kPer], fresh[kPer], end[kPer];
        int q = 0, p = 0;      // inclusive sums over this thread's sequences, then over all before
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            len[i] = b + i < a.B ? a.lengths[b + i] : 0;
            n[i] = b + i < a.B ? a.counts[b + i] : 0;
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            len[i] = max(len[i], 0);
            n[i] = max(n[i], 0);
            have[i] = (int)(((int64_t)len[i] + ps_mask) >> a.shift);
            end[i] = max((int)min((int64_t)len[i] + n[i], (int64_t)cap), len[i]);      // rows with a place in the table (what is there already stays)
            fresh[i] = max((int)(((int64_t)end[i] + ps_mask) >> a.shift) - have[i], 0);
            q += n[i];
            p += fresh[i];
        }
        const int own_q = q, own_p = p;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int qo = __shfl_up(q, d), po = __shfl_up(p, d);
            if (l >= d) { q += qo; p += po; }
        }
        if (l == 63) { s_sum[0][w] = q; s_sum[1][w] = p; }
        __syncthreads();
        int all_q = 0, all_p = 0;
#pragma unroll
        for (int i = 0; i < kThreads / 64; ++i) {
            if (i < w) { q += s_sum[0][i]; p += s_sum[1][i]; }
            all_q += s_sum[0][i];
            all_p += s_sum[1][i];
        }
        int q0 = base_q + q - own_q, first = base_p + p - own_p;
        const bool owner = (b0 / kSeqs) % (int)gridDim.x == (int)blockIdx.x;      // of these sequences' own results
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int at = kPer * tid + i;
            s_q0[at] = q0;
            s_len[at] = len[i];
            s_have[at] = have[i];
            s_first[at] = first;
            if (owner && b + i < a.B) {
                a.q_off[b + i] = q0;
                const int granted = min(max(a.n_free - first, 0), fresh[i]);
                a.new_lengths[b + i] = max(len[i], (int)min((int64_t)end[i], (int64_t)(have[i] + granted) << a.shift));
            }
            q0 += n[i];
            first += fresh[i];
        }
        if (owner && b0 + kSeqs >= a.B && tid == 0) {
            a.q_off[a.B] = base_q + all_q;
            *a.pages_used = base_p + all_p;
        }
        __syncthreads();
        if (blockIdx.x == gridDim.x - 1 && base_q + all_q > a.rows) {      // pages that begin with a token that has no place in `slots`
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int at = kPer * tid + i, from = max(a.rows - s_q0[at], 0);      // the first such token of the sequence
                const int e0 = max((int)(((int64_t)s_len[at] + from + ps_mask) >> a.shift), s_have[at]);
                for (int e = e0; b + i < a.B && e < s_have[at] + fresh[i]; ++e) {
                    const int f = s_first[at] + e - s_have[at];
                    a.table[(int64_t)(b + i) * a.stride + e] = f < a.n_free ? a.free_pages[f] : -1;
                }
            }
        }
        // the tokens of this workgroup that belong to these sequences
        const int t_end = min(tok1, base_q + all_q);
        for (int i = max(tok0, base_q) + tid; i < t_end; i += kThreads) {
            int lo = 0;      // the last sequence that starts at or before i
#pragma unroll
            for (int d = kSeqs / 2; d > 0; d /= 2)
                if (s_q0[lo + d] <= i) lo += d;
            const int64_t j = (int64_t)s_len[lo] + (i - s_q0[lo]);
            int slot = -1;
            if (j >= 0 && j < cap && b0 + lo < a.B) {      // (j < 0, or a sequence behind the last: the counts' sum has left 32 bits)
                const int e = (int)j >> a.shift;
                int32_t* const entry = a.table + (int64_t)(b0 + lo) * a.stride + e;
                int page;
                if (e < s_have[lo]) {
                    page = *entry;
                } else {
                    const int f = s_first[lo] + e - s_have[lo];
                    page = f < a.n_free ? a.free_pages[f] : -1;
                    if (((int)j & ps_mask) == 0) *entry = page;
                }
                if (page >= 0 && page <= 0x7fffffff >> a.shift) slot = (page << a.shift) + ((int)j & ps_mask);
            }
            a.slots[i] = slot;
        }
        base_q += all_q;
        base_p += all_p;
        __syncthreads();
    }
    if (a.B == 0 && blockIdx.x == 0 && tid == 0) {
        a.q_off[0] = 0;
        *a.pages_used = 0;
    }
    for (int i = max(tok0, base_q) + tid; i < tok1; i += kThreads) a.slots[i] = -1;      // behind the last token
}

hipError_t launch_page_slots(const SlotArgs& a, hipStream_t s) {
    const int grid = std::max((a.rows + kTokens - 1) / kTokens, 1);
    page_slots_kernel<<<(unsigned)grid, kThreads, 0, s>>>(a);
    return hipGetLastError();
}

// A thread takes a piece of eight elements of K and of V.  Bound by HBM: 16.8 thousand tokens, 40 heads of 128, as codes 91 us, 5.5 TB/s of 503 MB, two thirds of
// them reads (an addition of the same bytes, two reads to a write, 85); a decode step's rows 4.1 us, a launch.
template <bool CODES>
__global__ __launch_bounds__(256) void kv_write_kernel(WriteArgs a) {
    using Piece = std::conditional_t<CODES, uint2, uint4>;
    const unsigned n = (unsigned)a.rows * (unsigned)a.vec;
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    if (i >= n) return;
    const unsigned row = a.by_vec.of(i), c = i - row * (unsigned)a.vec;
    const int64_t src = (int64_t)row * a.stride + 8 * c;
    const int slot = a.slots[row];
    const uint4 k = *reinterpret_cast<const uint4*>(a.Knew + src), v = *reinterpret_cast<const uint4*>(a.Vnew + src);
    if (slot < 0 || slot >= a.pool_rows) return;      // a token without a place
    const int64_t dst = (int64_t)slot * a.vec + c;
    if constexpr (CODES) {
        reinterpret_cast<Piece*>(a.K)[dst] = quantize8(k, a.k_scale);
        reinterpret_cast<Piece*>(a.V)[dst] = quantize8(v, a.v_scale);
    } else {
        reinterpret_cast<Piece*>(a.K)[dst] = k;
        reinterpret_cast<Piece*>(a.V)[dst] = v;
    }
}

hipError_t launch_kv_write(const WriteArgs& a, hipStream_t s) {
    const int64_t n = (int64_t)a.rows * a.vec;
    if (n == 0) return hipSuccess;
    const unsigned grid = (unsigned)((n + 255) / 256);
    if (a.codes) kv_write_kernel<true><<<grid, 256, 0, s>>>(a);
    else kv_write_kernel<false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace hg
