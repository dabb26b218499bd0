// Kernels over ragged_rows_impl.h, and the joins of partial results.
#include <algorithm>

#include "ragged_rows_impl.h"

namespace hg {

using namespace rr;

template <int D, bool CODES, bool BOTH, int NW>
__global__ __launch_bounds__(64 * NW, 2) void ragged_rows_kernel(RaggedArgs a) { rows_workgroup<D, CODES, BOTH, NW>(a, blockIdx.x); }

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
    const float inv = den == 0.f ? 0.f : 1.0f / den;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= inv;
    store_row8<D>(out, row, c8, o, den == 0.f ? -INFINITY : m + __logf(den));
}

// Joins the parts of both kinds of rows, PG groups of D / 8 lanes to a row, each with every PG-th of its parts (a row of many parts would be a chain of loads
// otherwise), so a workgroup takes 2048 / D / PG rows.  Part p holds the keys from p * chunk on: those of a row are its first ceil(seen / chunk).  Where
// a tile, or what remains of a sequence, has one range, its rows are there already.
// The first a.rows * per_token workgroups (tile_nsplit > 1) take the rows of tiles, per_token of them one token's heads; the others (nsplit > 1) the places for
// few_most rows of every sequence and KV head.
// What bounds it is that the parts, which the kernels before have just written, are read once: 11 us for 37 MB of up to 86 parts a row (3 x 64/8 heads, up to 33 tokens behind 64K
// keys), 4 to 6 us where few rows have any.
template <int D, int PG>
__global__ __launch_bounds__(256) void ragged_join_kernel(RaggedArgs a, int per_token) {
    constexpr int LPR = D / 8, RPW = 256 / LPR / PG;
    __shared__ float s_o[PG > 1 ? 256 : 1][8], s_m[256 / LPR], s_l[256 / LPR];
    const int group = threadIdx.x / LPR, c8 = threadIdx.x % LPR, pg = group / RPW;
    const unsigned of_tiles = (unsigned)a.rows * (unsigned)per_token;
    const float *O, *L;
    int64_t stride, at, row = 0;
    int parts = 0;
    bool mine = false;
    if (blockIdx.x < of_tiles) {
        const int token = (int)(blockIdx.x / (unsigned)per_token), h = (int)(blockIdx.x - (unsigned)token * (unsigned)per_token) * RPW + group % RPW;
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
        const int tok = token - sq.q0, g = h - (int)a.by_group.of((unsigned)h) * a.G;
        if (tok < 0 || tok >= sq.take) return;
        const int in_tiles = rows_in_tiles(sq.take * a.G, a.few_rows), r = tok * a.G + g;
        mine = h < a.Hq && r < in_tiles && sq.seen((int)a.by_group.of((unsigned)(min(r / kTile * kTile + kTile, in_tiles) - 1))) > a.tile_chunk;
        const int seen = mine ? sq.seen(tok) : 0;
        parts = seen > 0 ? min((seen + a.tile_chunk - 1) / a.tile_chunk, a.tile_nsplit) : 0;
        O = a.tile_part_O;
        L = a.tile_part_L;
        stride = (int64_t)a.rows * a.Hq;
        row = at = (int64_t)token * a.Hq + h;
    } else {
        at = (int64_t)(blockIdx.x - of_tiles) * RPW + group % RPW;
        if (at < a.part_rows) {
            const int bh = (int)a.by_most.of((unsigned)at), b = (int)a.by_heads.of((unsigned)bh), kvh = bh - b * a.Hkv;
            const RaggedSeq sq = ragged_seq(a, b);
            const int r = rows_in_tiles(sq.take * a.G, a.few_rows) + ((int)at - bh * a.few_most), tok = (int)a.by_group.of((unsigned)r);
            mine = r < sq.take * a.G && sq.seen(sq.take - 1) > a.chunk;
            const int seen = mine ? sq.seen(tok) : 0;
            parts = seen > 0 ? min((seen + a.chunk - 1) / a.chunk, a.nsplit) : 0;
            row = (int64_t)(sq.q0 + tok) * a.Hq + kvh * a.G + (r - tok * a.G);
        }
        O = a.part_O;
        L = a.part_L;
        stride = a.part_rows;
    }
    float m = -INFINITY, den = 0.f, o[8] = {};
    join_parts<D>(O, L, stride, at, pg, PG, parts, c8, m, den, o);
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

template <int D, int PG>
static hipError_t launch_join_t(const RaggedArgs& a, hipStream_t s) {
    const int64_t grid = join_grid(a, D);
    if (grid >= (1LL << 31)) return hipErrorInvalidValue;
    ragged_join_kernel<D, PG><<<(unsigned)grid, 256, 0, s>>>(a, join_per_token(a, D));
    return hipGetLastError();
}

hipError_t launch_ragged_join(const RaggedArgs& a, int D, hipStream_t s) {
    const bool many = join_groups(a) > 1;
    if (D == 128) return many ? launch_join_t<128, 8>(a, s) : launch_join_t<128, 1>(a, s);
    return many ? launch_join_t<64, 8>(a, s) : launch_join_t<64, 1>(a, s);
}

}  // namespace hg
