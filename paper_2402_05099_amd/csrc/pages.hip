// Bookkeeping of a paged cache on the GPU: block tables and slots from the requests' lengths, and the write of new K/V rows to their slots.
#include <algorithm>
#include <type_traits>

#include "ragged.h"

namespace hg {

namespace {
constexpr int kThreads = 256;        // also: sequences that a workgroup looks at together
constexpr int kTokens = 1024;        // tokens that a workgroup finds the slots of
}

// With have = ceil(len / ps) pages in use and want = ceil(min(len + n, capacity) / ps) needed, sequence b's new pages are the entries
// [first, first + want - have) of the list of free ones, first = the new pages of the sequences before it; token t of it becomes row
// len + t.  Two prefix sums over the sequences (tokens, new pages) are all that ties the sequences to each other; every workgroup takes them
// for itself, so that one launch does: 4 bytes twice per sequence out of L2 instead of a second launch.
__global__ __launch_bounds__(kThreads) void page_slots_kernel(SlotArgs a) {
    __shared__ int s_q0[kThreads + 1], s_len[kThreads], s_have[kThreads], s_first[kThreads], s_sum[2][kThreads / 64];
    const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
    const int ps_mask = (1 << a.shift) - 1, cap = a.stride << a.shift;
    const int tok0 = (int)blockIdx.x * kTokens, tok1 = min(tok0 + kTokens, a.rows);
    int base_q = 0, base_p = 0;
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        int len = 0, n = 0;
        if (b < a.B) {
            len = max(a.lengths[b], 0);
            n = max(a.counts[b], 0);
        }
        const int have = (int)(((int64_t)len + ps_mask) >> a.shift);
        const int end = max((int)min((int64_t)len + n, (int64_t)cap), len);      // rows with a place in the table (what is there already stays)
        const int fresh = max((int)(((int64_t)end + ps_mask) >> a.shift) - have, 0);
        int q = n, p = fresh;      // inclusive sums
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
        const int q0 = base_q + q - n, first = base_p + p - fresh;
        s_q0[tid] = q0;
        s_len[tid] = len;
        s_have[tid] = have;
        s_first[tid] = first;
        if (tid == 0) s_q0[kThreads] = base_q + all_q;
        __syncthreads();
        if ((b0 / kThreads) % (int)gridDim.x == (int)blockIdx.x) {      // these sequences' own results
            if (b < a.B) {
                a.q_off[b] = q0;
                const int granted = min(max(a.n_free - first, 0), fresh);
                a.new_lengths[b] = max(len, (int)min((int64_t)end, (int64_t)(have + granted) << a.shift));
            }
            if (b0 + kThreads >= a.B && tid == 0) {
                a.q_off[a.B] = base_q + all_q;
                *a.pages_used = base_p + all_p;
            }
            // table entries: a wavefront goes through its own sequences, a lane per entry
            for (unsigned long long todo = __ballot(fresh > 0); todo; todo &= todo - 1) {
                const int from = __builtin_ctzll(todo);
                const int nf = __shfl(fresh, from), f0 = __shfl(first, from), h = __shfl(have, from);
                int32_t* const row = a.table + (int64_t)(b0 + 64 * w + from) * a.stride + h;
                for (int i = l; i < nf; i += 64) row[i] = f0 + i < a.n_free ? a.free_pages[f0 + i] : -1;
            }
        }
        // slots of the tokens of this workgroup that belong to these sequences
        const int t_end = min(tok1, base_q + all_q);
        for (int i = max(tok0, base_q) + tid; i < t_end; i += kThreads) {
            int lo = 0;      // the last sequence that starts at or before i
#pragma unroll
            for (int d = kThreads / 2; d > 0; d /= 2)
                if (s_q0[lo + d] <= i) lo += d;
            const int j = s_len[lo] + (i - s_q0[lo]);
            int slot = -1;
            if (j < cap && j >= 0) {
                const int e = j >> a.shift;
                int page;
                if (e < s_have[lo]) {
                    page = a.table[(int64_t)(b0 + lo) * a.stride + e];
                } else {
                    const int f = s_first[lo] + e - s_have[lo];
                    page = f < a.n_free ? a.free_pages[f] : -1;
                }
                if (page >= 0) slot = (page << a.shift) + (j & ps_mask);
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

namespace {
// As in kvcache.hip: code = nearest E4M3 value to the fp32 quotient, ties to even, magnitudes above 448 saturated, NaN stays NaN.
__device__ __forceinline__ uint2 codes8(const uint4& r, float scale) {
    const float f[8] = {bf16_lo(r.x), bf16_hi(r.x), bf16_lo(r.y), bf16_hi(r.y), bf16_lo(r.z), bf16_hi(r.z), bf16_lo(r.w), bf16_hi(r.w)};
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = f[i] / scale;
        q[i] = x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f);
    }
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    return make_uint2((unsigned)lo, (unsigned)hi);
}
}

// A thread takes a piece of eight elements of K and of V.
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
        reinterpret_cast<Piece*>(a.K)[dst] = codes8(k, a.k_scale);
        reinterpret_cast<Piece*>(a.V)[dst] = codes8(v, a.v_scale);
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
