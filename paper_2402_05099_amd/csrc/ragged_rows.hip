// Kernels over ragged_rows_impl.h, and the joins of partial results.
#include <algorithm>

#include "ragged_rows_impl.h"

namespace hg {

using namespace rr;

template <int D, bool CODES, bool BOTH, int NW>
__global__ __launch_bounds__(64 * NW) void ragged_rows_kernel(RaggedArgs a) { rows_workgroup<D, CODES, BOTH, NW>(a, blockIdx.x); }

// Parts first, first + step, .. of a row's `parts` joined by Eq. 5 into (m, den, o): D / 8 lanes of eight columns.  Part p of row `at` is O[p * part_rows + at],
// L[p * part_rows + at].
template <int D>
__device__ __forceinline__ void join_parts(const float* O, const float* L, int64_t part_rows, int64_t at, int first, int step, int parts, int c8, float& m, float& den,
                                           float (&o)[8]) {
    constexpr int U = 4;
    for (int p0 = first; p0 < parts; p0 += U * step) {
        float li[U];
        float4 x[U][2];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t i = (int64_t)min(p0 + k * step, parts - 1) * part_rows + at;
            li[k] = L[i];
            const float4* const src = reinterpret_cast<const float4*>(O + i * D + 8 * c8);
            x[k][0] = src[0];
            x[k][1] = src[1];
            if (p0 + k * step >= parts) li[k] = -INFINITY;
        }
        float gm = m;
#pragma unroll
        for (int k = 0; k < U; ++k) gm = fmaxf(gm, li[k]);
        if (gm == -INFINITY) continue;      // (parts without a key have O = 0 and LSE = -inf)
        const float old = __builtin_amdgcn_exp2f((m - gm) * kLog2e);
        m = gm;
        den *= old;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= old;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const float e = __builtin_amdgcn_exp2f((li[k] - m) * kLog2e);
            den += e;
            o[0] = fmaf(e, x[k][0].x, o[0]); o[1] = fmaf(e, x[k][0].y, o[1]); o[2] = fmaf(e, x[k][0].z, o[2]); o[3] = fmaf(e, x[k][0].w, o[3]);
            o[4] = fmaf(e, x[k][1].x, o[4]); o[5] = fmaf(e, x[k][1].y, o[5]); o[6] = fmaf(e, x[k][1].z, o[6]); o[7] = fmaf(e, x[k][1].w, o[7]);
        }
    }
}
template <int D>
__device__ __forceinline__ void store_joined(const OutDev& out, int64_t row, int c8, float m, float den, float (&o)[8]) {
    const float inv = den > 0.f ? 1.0f / den : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= inv;
    store_row8<D>(out, row, c8, o, den > 0.f ? m + __logf(den) : -INFINITY);
}

// The rows of ragged_rows_impl.h, PG groups of D / 8 lanes to a row, each with every PG-th of its parts (a row of many parts would be a chain of loads
// otherwise); a workgroup takes 2048 / D / PG of the places for few_most rows of every sequence and KV head.  Part p holds the keys from p * chunk on, so those
// of a row are its first ceil(seen / chunk).
template <int D, int PG>
__global__ __launch_bounds__(256) void ragged_merge_kernel(RaggedArgs a) {
    constexpr int LPR = D / 8, RPW = 256 / LPR / PG;
    __shared__ float s_o[PG > 1 ? 256 : 1][8], s_m[256 / LPR], s_l[256 / LPR];
    const int group = threadIdx.x / LPR, c8 = threadIdx.x % LPR, pg = group / RPW;
    const int64_t at = (int64_t)blockIdx.x * RPW + group % RPW;
    int parts = 0;
    int64_t row = 0;
    bool mine = false;
    if (at < a.part_rows) {
        const int bh = (int)a.by_most.of((unsigned)at), b = (int)a.by_heads.of((unsigned)bh), kvh = bh - b * a.Hkv;
        const RaggedSeq sq = ragged_seq(a, b);
        const int r = rows_in_tiles(sq.take * a.G, a.few_rows) + ((int)at - bh * a.few_most), tok = (int)a.by_group.of((unsigned)r);
        mine = r < sq.take * a.G;
        const int seen = mine ? sq.seen(tok) : 0;
        parts = seen > 0 ? min((seen + a.chunk - 1) / a.chunk, a.nsplit) : 0;
        row = (int64_t)(sq.q0 + tok) * a.Hq + kvh * a.G + (r - tok * a.G);
    }
    float m = -INFINITY, den = 0.f, o[8] = {};
    join_parts<D>(a.part_O, a.part_L, a.part_rows, at, pg, PG, parts, c8, m, den, o);
    if constexpr (PG > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) s_o[threadIdx.x][i] = o[i];
        if (c8 == 0) { s_m[group] = m; s_l[group] = den; }
        __syncthreads();
        if (pg > 0) return;
#pragma unroll 1
        for (int k = 1; k < PG; ++k) {
            const int other = group + k * RPW;
            const float gm = fmaxf(m, s_m[other]);
            if (gm == -INFINITY) continue;
            const float x = __builtin_amdgcn_exp2f((m - gm) * kLog2e), y = __builtin_amdgcn_exp2f((s_m[other] - gm) * kLog2e);
            m = gm;
            den = den * x + s_l[other] * y;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = o[i] * x + s_o[threadIdx.x + k * RPW * LPR][i] * y;
        }
    }
    if (mine) store_joined<D>(a.out, row, c8, m, den, o);
}

// The rows of tiles: a workgroup takes one token's rows from blockIdx.y * 2048 / D on.
template <int D>
__global__ __launch_bounds__(256) void ragged_join_kernel(RaggedArgs a) {
    constexpr int LPR = D / 8;
    const int token = blockIdx.x;
    // the sequence that owns the token: the last that begins at or before it 
    int lo = 0, n = a.B;
    const int lane = threadIdx.x & 63;
    while (true) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const int c = __builtin_popcountll(__ballot(lane * step < n && a.q_off[i] <= token));
        if (c == 0) return;
        lo += (c - 1) * step;
        n = min(step, n - (c - 1) * step);
        if (n == 1) break;
    }
    const RaggedSeq sq = ragged_seq(a, __builtin_amdgcn_readfirstlane(lo));
    const int tok = token - sq.q0, h = (int)blockIdx.y * (256 / LPR) + (int)threadIdx.x / LPR;
    if (tok < 0 || tok >= sq.take || h >= a.Hq) return;
    if (tok * a.G + (h - (h / a.G) * a.G) >= rows_in_tiles(sq.take * a.G, a.few_rows)) return;
    const int seen = sq.seen(tok);
    float m = -INFINITY, den = 0.f, o[8] = {};
    join_parts<D>(a.tile_part_O, a.tile_part_L, (int64_t)a.rows * a.Hq, (int64_t)token * a.Hq + h, 0, 1,
                  seen > 0 ? min((seen + a.tile_chunk - 1) / a.tile_chunk, a.tile_nsplit) : 0, threadIdx.x % LPR, m, den, o);
    store_joined<D>(a.out, (int64_t)token * a.Hq + h, threadIdx.x % LPR, m, den, o);
}

template <int D, bool CODES, bool BOTH, int NW>
static hipError_t launch_rows_t(const RaggedArgs& a, unsigned grid, hipStream_t s) {
    constexpr int bytes = rows_lds<D, CODES, BOTH>(NW);
    static bool attr_set[64] = {};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (bytes > 65536 && (dev < 0 || dev >= 64 || !attr_set[dev])) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&ragged_rows_kernel<D, CODES, BOTH, NW>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    ragged_rows_kernel<D, CODES, BOTH, NW><<<grid, 64 * NW, bytes, s>>>(a);
    return hipGetLastError();
}

template <int D, bool CODES>
static hipError_t launch_rows_d(const RaggedArgs& a, unsigned grid, hipStream_t s) {
    if (!a.both_tiles) return a.wavefronts == 8 ? launch_rows_t<D, CODES, false, 8>(a, grid, s) : launch_rows_t<D, CODES, false, 4>(a, grid, s);
    return a.wavefronts == 8 ? launch_rows_t<D, CODES, true, 8>(a, grid, s) : launch_rows_t<D, CODES, true, 4>(a, grid, s);
}

hipError_t launch_ragged_rows(const RaggedArgs& a, int D, bool codes, hipStream_t s) {
    const int64_t grid = rows_grid(a);
    if (grid >= (1LL << 31)) return hipErrorInvalidValue;
    if (D == 128) return codes ? launch_rows_d<128, true>(a, (unsigned)grid, s) : launch_rows_d<128, false>(a, (unsigned)grid, s);
    return codes ? launch_rows_d<64, true>(a, (unsigned)grid, s) : launch_rows_d<64, false>(a, (unsigned)grid, s);
}

template <int D>
static hipError_t launch_merge_d(const RaggedArgs& a, hipStream_t s) {
    if (a.nsplit > 8) ragged_merge_kernel<D, 8><<<(unsigned)((a.part_rows + 256 / D - 1) / (256 / D)), 256, 0, s>>>(a);
    else ragged_merge_kernel<D, 1><<<(unsigned)((a.part_rows + 2048 / D - 1) / (2048 / D)), 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_ragged_merge(const RaggedArgs& a, int D, hipStream_t s) { return D == 128 ? launch_merge_d<128>(a, s) : launch_merge_d<64>(a, s); }

hipError_t launch_ragged_join(const RaggedArgs& a, int D, hipStream_t s) {
    const dim3 grid((unsigned)a.rows, (unsigned)((a.Hq * D / 8 + 255) / 256));
    if (grid.y > 65535) return hipErrorInvalidValue;
    if (D == 128) ragged_join_kernel<128><<<grid, 256, 0, s>>>(a);
    else ragged_join_kernel<64><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace hg
