// Causal attention of packed tokens, 128 query rows to a workgroup: four wavefronts with 32 rows each, multiplied with stages of 32 keys in
// LDS as in decode_mfma_core.h (S^T = K Q^T, O^T += V^T P^T, a lane owns one query row).  Any head dimension, packed or paged rows, bf16
// or codes: rows go through registers, where codes become bf16, into one stage of LDS.
#include "decode_mfma_core.h"
#include "ragged.h"

namespace hg {

using namespace dm;

namespace {

constexpr int kRows = 128;      // query rows of a workgroup

// (O, LSE) of this lane's row to part `part`; rv: the row exists
template <int D, bool CODES, int TR>
__device__ __forceinline__ void store_row(const MfmaTile<D, CODES, TR>& t, const OutDev& out, int part, int64_t row, bool rv, float v_scale) {
    using Tile = MfmaTile<D, CODES, TR>;
    float lsub = t.lsum;
    if constexpr (TR == 16) lsub += __shfl_xor(lsub, 16);
    const float ltot = half_sum(lsub);
    if (!rv) return;
    const float inv = ltot > 0.f ? v_scale / ltot : 0.f;      // a row that sees no key: O = 0, LSE = -inf
    const int64_t at = (int64_t)part * out.part_stride_O + row * D;
    const auto put = [&](int d, float o0, float o1, float o2, float o3) {
        if (out.bf16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out.O) + at + d) = make_uint2(pack_pair(o0, o1), pack_pair(o2, o3));
        else *reinterpret_cast<float4*>(static_cast<float*>(out.O) + at + d) = make_float4(o0, o1, o2, o3);
    };
    if constexpr (TR == 16) {
#pragma unroll
        for (int db = 0; db < Tile::DB16; ++db)
            put(16 * db + 4 * t.lg, t.Oacc16[db][0] * inv, t.Oacc16[db][1] * inv, t.Oacc16[db][2] * inv, t.Oacc16[db][3] * inv);
    } else {
#pragma unroll
        for (int db = 0; db < Tile::DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                put(32 * db + 8 * q4 + 4 * t.hl, t.Oacc[db][4 * q4] * inv, t.Oacc[db][4 * q4 + 1] * inv, t.Oacc[db][4 * q4 + 2] * inv,
                    t.Oacc[db][4 * q4 + 3] * inv);
    }
    if (out.LSE && (TR == 16 ? t.lg : t.hl) == 0)
        out.LSE[(int64_t)part * out.part_stride_L + row] = ltot > 0.f ? t.m_used * t.kscale + __logf(ltot) : -INFINITY;
}

}  // namespace

template <int D, bool PAGED, bool CODES>
__global__ __launch_bounds__(256) void ragged_tiles_kernel(RaggedArgs a) {
    using Tile = MfmaTile<D, false, 32>;
    using G_ = Geo<D>;
    constexpr int CPR = G_::CPR, ROWB = G_::ROWB, STB = G_::STB, PER = KT * CPR / 256;      // 16-byte pieces of a stage per thread and tensor
    __shared__ __attribute__((aligned(1024))) unsigned char sK[STB], sV[STB], sQ[4 * STB];

    const unsigned per_split = gridDim.x / (unsigned)a.nsplit;
    const int sp = (int)(blockIdx.x / per_split);
    const int u = (int)(blockIdx.x - (unsigned)sp * per_split);
    const int number = (int)a.by_heads.of((unsigned)u), kvh = u - number * a.Hkv;
    int b, tile;
    if (!ragged_tile<kRows>(a, number, b, tile)) return;
    const RaggedSeq sq = ragged_seq(a, b);
    const int nrows = sq.take * a.G, row0 = tile * kRows;
    if (row0 >= nrows || nrows <= a.few_rows) return;

    const int tid = threadIdx.x, l = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int last_t = (int)a.by_group.of((unsigned)(min(row0 + kRows, nrows) - 1));      // the tile's last token
    const int k0 = sp * a.chunk, ke = min(max(sq.seen(last_t), 0), k0 + a.chunk);

    // ---- Q: this wavefront's 32 rows (rows past the sequence's read its first) ----
    const int wrow0 = row0 + 32 * w;
    Tile t(a.scale, l);
    t.tau_raw = 0.f;      // sums follow every maximum: the largest weight of a row is 1, which bf16 holds exactly (with scores of many nats it is nearly the only one)
    {
        unsigned char* const qs = sQ + w * STB;
        const int sch = l % CPR;
#pragma unroll
        for (int i = 0; i < 32 * CPR / 64; ++i) {
            const int row = i * (64 / CPR) + l / CPR, r = wrow0 + row < nrows ? wrow0 + row : 0;
            const int tok = (int)a.by_group.of((unsigned)r), g = r - tok * a.G;
            const unsigned char* const src = reinterpret_cast<const unsigned char*>(a.Q) + (int64_t)(sq.q0 + tok) * a.q_stride + (kvh * a.G + g) * ROWB;
            *reinterpret_cast<uintx4*>(qs + row * ROWB + ((sch ^ G_::kswz(row)) * 16)) = *reinterpret_cast<const uintx4*>(src + sch * 16);
        }
        __syncthreads();
        t.load_q(qs);
    }
    const int r = wrow0 + t.row();
    const bool rv = r < nrows;
    const int tok = (int)a.by_group.of((unsigned)(rv ? r : 0)), g = (rv ? r : 0) - tok * a.G;
    const int seen = rv ? sq.seen(tok) : 0;
    const int wave_last = wrow0 < nrows ? sq.seen((int)a.by_group.of((unsigned)(min(wrow0 + 32, nrows) - 1))) : 0;      // the most any row of the wavefront sees
    const int wave_first = wrow0 < nrows ? sq.seen((int)a.by_group.of((unsigned)wrow0)) : 0;                           // ... and the least

    const int es = CODES ? 1 : 2;
    const unsigned char* const Kh = a.K + (int64_t)kvh * (D * es);
    const unsigned char* const Vh = a.V + (int64_t)kvh * (D * es);
    for (int key0 = k0; key0 < ke; key0 += KT) {
        uintx4 kr[PER], vr[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int piece = i * 256 + tid, row = piece / CPR, ch = piece % CPR, j = min(key0 + row, ke - 1);
            int64_t prow;
            if (PAGED) {
                const int e = min(j >> a.pg.shift, a.pg.stride - 1);
                const int page = min(max(a.pg.table[(int64_t)b * a.pg.stride + e], 0), a.pg.n_pages - 1);
                prow = ((int64_t)page << a.pg.shift) + (j & ((1 << a.pg.shift) - 1));
            } else {
                prow = sq.q0 + j;
            }
            const int64_t at = prow * a.kv_stride + ch * (8 * es);
            if (CODES) {
                const uint2 kc = *reinterpret_cast<const uint2*>(Kh + at), vc = *reinterpret_cast<const uint2*>(Vh + at);
                kr[i] = Tile::expand8(kc.x, kc.y);
                vr[i] = Tile::expand8(vc.x, vc.y);
            } else {
                kr[i] = *reinterpret_cast<const uintx4*>(Kh + at);
                vr[i] = *reinterpret_cast<const uintx4*>(Vh + at);
            }
            if (key0 + row >= ke) vr[i] = uintx4{0u, 0u, 0u, 0u};
        }
        __syncthreads();      // everyone has multiplied the stage before
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int piece = i * 256 + tid, row = piece / CPR, ch = piece % CPR;
            *reinterpret_cast<uintx4*>(sK + row * ROWB + ((ch ^ G_::kswz(row)) * 16)) = kr[i];
            *reinterpret_cast<uintx4*>(sV + row * ROWB + ((ch ^ G_::vswz(row)) * 16)) = vr[i];
        }
        __syncthreads();
        if (key0 < wave_last) {
            typename Tile::Scores S;
            uintx4 pb[2];
            t.scores(sK, S);
            if (key0 + KT > min(wave_first, ke)) t.mask(S, 0, min(seen, ke) - key0);
            t.softmax(S, pb);
            t.values(sV, pb);
        }
    }
    store_row<D, false, 32>(t, a.out, sp, (int64_t)(sq.q0 + tok) * a.Hq + kvh * a.G + g, rv, a.v_scale);
}

template <int D>
static hipError_t launch_tiles_d(const RaggedArgs& a, bool codes, hipStream_t s) {
    const int64_t grid = ragged_tiles(a.rows, a.G, a.B, kRows) * a.Hkv * a.nsplit;
    if (grid >= (1LL << 31)) return hipErrorInvalidValue;
    if (!a.pg.table) ragged_tiles_kernel<D, false, false><<<(unsigned)grid, 256, 0, s>>>(a);
    else if (codes) ragged_tiles_kernel<D, true, true><<<(unsigned)grid, 256, 0, s>>>(a);
    else ragged_tiles_kernel<D, true, false><<<(unsigned)grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_ragged_tiles(const RaggedArgs& a, int D, bool codes, hipStream_t s) {
    return D == 128 ? launch_tiles_d<128>(a, codes, s) : launch_tiles_d<64>(a, codes, s);
}

}  // namespace hg
