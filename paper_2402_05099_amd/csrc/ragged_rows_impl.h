// Attention over a paged cache of what remains of a sequence's query rows behind its tiles, at most 32 (64 in small calls) to a KV head: all rows of decode steps and drafted
// tokens, the last ones of a chunk.
// What bounds it is the cache that is read, once for every KV head whatever the rows, so the rows of a head's group and of all
// new tokens form one tile of 16 or 32 rows (v_mfma_f32_16x16x32_bf16, v_mfma_f32_32x32x16_bf16; decode_mfma_core.h has the products and the softmax).
//
// A workgroup of NW wavefronts takes one tile and one range of its keys; its 32-key stages go to the wavefronts in turn, each with a K and a V slot
// in LDS that is filled again by global_load_lds_dwordx4 as soon as its rows have been multiplied.  The wavefronts never wait for each other until their
// (m, l, O) meet in LDS.  So a call of short contexts is one launch that needs no workspace, and one of long contexts splits the
// keys over workgroups as well: partial results by Eq. 5, joined by the kernel of ragged_rows_kernels.h.
//
// Single tokens, all of one length: 32 x 64/8 heads, 8192 keys 179 us, 6.0 TB/s, codes 106 us, 5.1 (at D = 64 102 and 69 us); 32 x 40/40, 2048 keys 213 us, 6.3 TB/s, codes 132, 5.1;
// 32 rows instead of 8 cost 14 % more, over codes 22.  45 x 16/2 heads, up to 515 keys 8.8 us, a chain of loads: lengths, table, rows, the join.
#pragma once
#include "decode_mfma_core.h"
#include "ragged.h"

#pragma clang diagnostic ignored "-Winline-asm"

namespace hg {
namespace rr {

using namespace dm;

extern __shared__ __attribute__((aligned(1024))) unsigned char rr_smem[];

template <int D, bool CODES, int TR>
struct RowsGeo {
    static constexpr int RPI = CODES ? 8 : Geo<D>::RPI;          // rows one copy instruction covers (codes of either D lie 128 bytes apart in LDS)
    static constexpr int CPS = KT / RPI;                         // copy instructions per stage and tensor
    static constexpr int TENSOR = CPS * 1024;                    // bytes of a stage's K or V in LDS
    static constexpr int JOIN = TR * D * 4;                      // bytes of a wavefront's O where they meet
    static constexpr int SLOT = 2 * TENSOR > JOIN ? 2 * TENSOR : JOIN;
    static constexpr int bytes(int nw) { return nw * (SLOT + 2 * TR * 4); }
};
template <int D, bool CODES, bool BOTH>
constexpr int rows_lds(int nw) { return BOTH ? RowsGeo<D, CODES, 32>::bytes(nw) : RowsGeo<D, CODES, 16>::bytes(nw); }

// Columns 8 c8 .. + 7 of a row's result
template <int D>
__device__ __forceinline__ void store_row8(const OutDev& out, int64_t row, int c8, const float (&o)[8], float lse) {
    if (out.bf16) {
        *reinterpret_cast<uintx4*>(static_cast<uint16_t*>(out.O) + row * D + 8 * c8) =
            uintx4{pack_pair(o[0], o[1]), pack_pair(o[2], o[3]), pack_pair(o[4], o[5]), pack_pair(o[6], o[7])};
    } else {
        float* const O = static_cast<float*>(out.O) + row * D + 8 * c8;
        *reinterpret_cast<float4*>(O) = make_float4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<float4*>(O + 4) = make_float4(o[4], o[5], o[6], o[7]);
    }
    if (out.LSE && c8 == 0) out.LSE[row] = lse;
}

// What workgroup `id` does for a sequence whose tiles have TR rows; everything up to the tile is known to the caller.
template <int D, bool CODES, int TR, int NW, bool TREE>
__device__ __forceinline__ void rows_tile(const RaggedArgs& a, int b, int rt, int sp, int kvh, int q0, int n, int len, int row0, int nrows) {
    using Tile = MfmaTile<D, CODES, TR>;
    using G_ = Geo<D>;
    using R_ = RowsGeo<D, CODES, TR>;
    constexpr int RPI = R_::RPI, CPS = R_::CPS, ES = CODES ? 1 : 2;
    const int l = threadIdx.x & 63;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);

    const int r0 = row0 + rt * TR;      // the tile's first row; the sequence's rows are [0, nrows), those from row0 on are taken here
    if (r0 >= nrows) return;
    const auto seen_by = [&](int t) { return TREE ? len : len - (n - 1 - t); };
    const int t_first = (int)a.by_group.of((unsigned)r0), t_last = (int)a.by_group.of((unsigned)(min(r0 + TR, nrows) - 1));
    const int k0 = sp * a.chunk, ke = min(seen_by(t_last), k0 + a.chunk);      // keys [k0, ke)
    if (sp > 0 && k0 >= ke) return;      // (the join looks at no part that starts behind a row's keys)
    const int all_see = TREE ? len - n : seen_by(t_first);       // every row of the tile sees the keys below
    const bool in_parts = seen_by((int)a.by_group.of((unsigned)(nrows - 1))) > a.chunk;      // the sequence has several ranges
    const int nst = ke > k0 ? (ke - k0 + KT - 1) / KT : 0;

    // ---- this lane's query row ----
    Tile t(a.scale, l);
    t.tau_raw = 0.f;      // sums follow every maximum: the largest weight of a row is 1, which bf16 holds exactly (with scores of many nats it is nearly the only one)
    const int r = r0 + t.row();
    const bool rv = r < nrows;
    const int tok = (int)a.by_group.of((unsigned)(rv ? r : r0)), g = (rv ? r : r0) - tok * a.G;
    const int seen = rv ? seen_by(tok) : 0;
    const uint32_t* const words = TREE ? a.masks + (int64_t)(q0 + tok) * a.mask_words : nullptr;
    const auto bits_from = [&](int key0) { return tree_bits(words, a.mask_words, key0 - all_see); };      // (TREE) of 32 keys from key0 on
    {
        const unsigned char* const qp = reinterpret_cast<const unsigned char*>(a.Q) + (int64_t)(q0 + tok) * a.q_stride + (kvh * a.G + g) * (D * 2);
        if constexpr (TR == 16) {
#pragma unroll
            for (int s = 0; s < Tile::KS16; ++s) t.qf16[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uintx4*>(qp + 64 * s + 16 * t.lg));
        } else {
#pragma unroll
            for (int s = 0; s < Tile::KS; ++s) t.qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uintx4*>(qp + 32 * s + 16 * t.hl));
        }
    }

    // ---- copies: stage i of this wavefront is stage w + i NW of the range ----
    unsigned char* const slot = rr_smem + w * R_::SLOT;
    const unsigned dst = (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)HG_LDS(slot));
    unsigned voffK[CPS], voffV[CPS];      // lane offsets within the rows of one copy instruction
    {
        constexpr int LPR = 64 / RPI;
        const int lr = l / LPR, sl = l % LPR;
#pragma unroll
        for (int i = 0; i < CPS; ++i) {
            const int row = i * RPI + lr;
            int ck, cv;
            if (CODES) {      // slots of 16 codes, swizzled as MfmaTile reads them; at D = 64 the other four of eight hold a row once more, which nothing reads
                ck = (sl ^ ((row >> 1) & 7)) & (D / 16 - 1);
                cv = (sl ^ (((row >> 1) & 1) | (((row >> (TR == 16 ? 4 : 3)) & 1) << 1))) & (D / 16 - 1);
            } else {
                ck = sl ^ G_::kswz(row);
                cv = sl ^ G_::vswz(row);
            }
            voffK[i] = (unsigned)lr * (unsigned)a.kv_stride + (unsigned)ck * 16u;
            voffV[i] = (unsigned)lr * (unsigned)a.kv_stride + (unsigned)cv * 16u;
        }
    }
    // page of half a stage (16 rows): lane 2 i + h holds that of half h of this wavefront's stage i0 + i, 32 stages at a time
    int pages = 0;
    const int shift = a.pg.shift;
    const auto look_up = [&](int i0) {
        const int j = k0 + (w + (i0 + (l >> 1)) * NW) * KT + (l & 1) * 16;
        const int e = min(j >> shift, a.pg.stride - 1);
        pages = min(max(a.pg.table[(int64_t)b * a.pg.stride + e], 0), a.pg.n_pages - 1);
    };
    const auto base_of = [&](int i, int h) -> int64_t {      // byte offset of the first row of half h of stage i
        const int page = __builtin_amdgcn_readlane(pages, (2 * i + h) & 63);
        const int j = k0 + (w + i * NW) * KT + h * 16;
        return (((int64_t)page << shift) + (j & ((1 << shift) - 1))) * a.kv_stride + (int64_t)kvh * (D * ES);
    };
    const auto scalar = [](const unsigned char* p) {
        const uint64_t v = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
        return reinterpret_cast<const unsigned char*>(((uint64_t)hi << 32) | lo);
    };
    const auto copy = [&](const unsigned char* tensor, const unsigned (&voff)[CPS], int i, unsigned to) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned char* const first = scalar(tensor + base_of(i, h));
#pragma unroll
            for (int k = 0; k < CPS / 2; ++k) {
                const unsigned char* const base = first + (int64_t)(k * RPI) * a.kv_stride;
                const int c = h * (CPS / 2) + k;
                const unsigned at = to + (unsigned)c * 1024u;
                // a line is used once, unless it has rows of two heads (32 x 64/8 heads, 8192 keys, bf16 179 us so, 199 without the hint; codes at D = 64 75 and 69)
                if constexpr (CODES && D == 64) asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff[c]), "s"(scalar(base)), "s"(at) : "memory", "m0");
                else asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1 nt" ::"v"(voff[c]), "s"(scalar(base)), "s"(at) : "memory", "m0");
            }
        }
    };
    const int mine = nst > w ? (nst - w + NW - 1) / NW : 0;
    int spoiled = mine;      // the first stage of this wavefront with values that were taken out: infinite or NaN, and not seen by every row
    if (mine > 0) {
        look_up(0);
        copy(a.K, voffK, 0, dst);
        copy(a.V, voffV, 0, dst + R_::TENSOR);
    }
    for (int i = 0; i < mine; ++i) {
        const bool more = i + 1 < mine;
        const int key0 = k0 + (w + i * NW) * KT;
        typename Tile::Scores S;
        uintx4 pb[2];
        wait_vm<CPS>();      // K has landed; V may be in flight
        asm volatile("" ::: "memory");
        t.scores(slot, S);
        if (more) {
            if (((i + 1) & 31) == 0) look_up(i + 1);
            copy(a.K, voffK, i + 1, dst);
        }
        if (key0 + KT > min(ke, all_see)) {
            if constexpr (TREE) t.mask_bits(S, bits_from(key0) & first_bits(min(seen, ke) - key0));
            else t.mask(S, 0, min(seen, ke) - key0);
        }
        t.softmax(S, pb);
        if (more) wait_vm<CPS>();      // V has landed; the next K may be in flight
        else wait_vm<0>();
        asm volatile("" ::: "memory");
        if (key0 + KT > ke) {      // rows past the range may hold anything, and 0 * NaN would be NaN
#pragma unroll
            for (int c = 0; c < CPS; ++c)
                if (c * RPI + l / (64 / RPI) >= ke - key0) *reinterpret_cast<uintx4*>(slot + R_::TENSOR + c * 1024 + l * 16) = uintx4{0u, 0u, 0u, 0u};
        }
        if (key0 + KT > all_see && all_see < ke) {      // some row does not see the stage as a whole
            if (take_out<CODES, CPS>(slot + R_::TENSOR + l * 16, 1024)) spoiled = min(spoiled, i);
        }
        t.values(slot + R_::TENSOR, pb);
        if (more) copy(a.V, voffV, i + 1, dst + R_::TENSOR);
    }

    if (__builtin_expect(spoiled < mine, 0)) {      // the rows that see them get them from memory
#pragma unroll 1
        for (int i = spoiled; i < mine; ++i)
#pragma unroll 1
            for (int key = k0 + (w + i * NW) * KT, end = min(key + KT, min(ke, seen)); key < end; ++key) {
                if (TREE && !(bits_from(key) & 1u)) continue;
                const int page = min(max(a.pg.table[(int64_t)b * a.pg.stride + min(key >> shift, a.pg.stride - 1)], 0), a.pg.n_pages - 1);
                const unsigned char* const vr = a.V + (((int64_t)page << shift) + (key & ((1 << shift) - 1))) * a.kv_stride + (int64_t)kvh * (D * ES);
                if constexpr (TR == 16) {
#pragma unroll
                    for (int db = 0; db < Tile::DB16; ++db)
#pragma unroll
                        for (int k = 0; k < 4; ++k) t.Oacc16[db][k] += value_if_not_finite<CODES>(vr + (16 * db + 4 * t.lg + k) * ES);
                } else {
#pragma unroll
                    for (int db = 0; db < Tile::DB; ++db)
#pragma unroll
                        for (int k = 0; k < 16; ++k) t.Oacc[db][k] += value_if_not_finite<CODES>(vr + (32 * db + 8 * (k / 4) + 4 * t.hl + k % 4) * ES);
                }
            }
    }

    // ---- the wavefronts' (m, l, O) meet: O as [row][16-byte piece ^ row], statistics behind the slots ----
    float lsum = t.lsum;
    if constexpr (TR == 16) lsum += __shfl_xor(lsum, 16);
    lsum = half_sum(lsum);
    const float m_row = lsum != lsum ? INFINITY : t.m_used;      // (as part_lse)
    float* const stat = reinterpret_cast<float*>(rr_smem + NW * R_::SLOT);      // [NW][2][TR]
    constexpr int PCS = D / 4;
    const auto piece = [&](unsigned char* base, int row, int c) { return reinterpret_cast<float4*>(base + row * (D * 4) + ((c ^ (row & (PCS - 1))) * 16)); };
    if constexpr (TR == 16) {
#pragma unroll
        for (int db = 0; db < Tile::DB16; ++db)
            *piece(slot, t.ln, 4 * db + t.lg) = make_float4(t.Oacc16[db][0], t.Oacc16[db][1], t.Oacc16[db][2], t.Oacc16[db][3]);
        if (t.lg == 0) { stat[(2 * w) * TR + t.ln] = m_row; stat[(2 * w + 1) * TR + t.ln] = lsum; }
    } else {
#pragma unroll
        for (int db = 0; db < Tile::DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *piece(slot, t.lq, 8 * db + 2 * q4 + t.hl) = make_float4(t.Oacc[db][4 * q4], t.Oacc[db][4 * q4 + 1], t.Oacc[db][4 * q4 + 2], t.Oacc[db][4 * q4 + 3]);
        if (t.hl == 0) { stat[(2 * w) * TR + t.lq] = m_row; stat[(2 * w + 1) * TR + t.lq] = lsum; }
    }
    __syncthreads();
    constexpr int LPR = D / 8;      // lanes per row, eight columns each
    for (int row = (int)threadIdx.x / LPR; row < TR; row += 64 * NW / LPR) {
        const int rr = r0 + row;
        if (rr >= nrows) break;
        const int c8 = (int)threadIdx.x % LPR;
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < NW; ++i) m = fmaxf(m, stat[(2 * i) * TR + row]);
        float o[8] = {}, den = 0.f;
        if (m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const float e = __builtin_amdgcn_exp2f((stat[(2 * i) * TR + row] - m) * t.c2);      // (a wavefront without a key: 0)
                den = fmaf(e, stat[(2 * i + 1) * TR + row], den);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float4 x = *piece(rr_smem + i * R_::SLOT, row, 2 * c8 + h);
                    o[4 * h] = fmaf(e, x.x, o[4 * h]);
                    o[4 * h + 1] = fmaf(e, x.y, o[4 * h + 1]);
                    o[4 * h + 2] = fmaf(e, x.z, o[4 * h + 2]);
                    o[4 * h + 3] = fmaf(e, x.w, o[4 * h + 3]);
                }
            }
        }
        const float inv = den == 0.f ? 0.f : a.v_scale / den;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] *= inv;
        const int tk = (int)a.by_group.of((unsigned)rr), gg = rr - tk * a.G;
        // one range: the result itself; several: part `sp`
        const int64_t at = !in_parts ? (int64_t)(q0 + tk) * a.Hq + kvh * a.G + gg : ((int64_t)b * a.Hkv + kvh) * a.few_most + (rr - row0);
        const float lse = den == 0.f ? -INFINITY : m * a.scale + __logf(den);
        if (in_parts) {
            float* const O = a.part_O + ((int64_t)sp * a.part_rows + at) * D + 8 * c8;
            *reinterpret_cast<float4*>(O) = make_float4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<float4*>(O + 4) = make_float4(o[4], o[5], o[6], o[7]);
            if (c8 == 0) a.part_L[(int64_t)sp * a.part_rows + at] = part_lse(lse);
            continue;
        }
        store_row8<D>(a.out, at, c8, o, lse);
    }
}

// Workgroup `id` of the launch: (range, tile, sequence, KV head), heads fastest, ranges slowest.  Later ranges and tiles are empty for most sequences; were they
// to alternate with the first ones, workgroups, which go to the shader engines of an XCD in turn, would leave some of those with little to do (64 x 32/8 heads, up
// to 4096 rows, two and four ranges 122 and 123 us so, 114 with one).  At most 16 rows make a tile of 16, more of them tiles of 32 (`BOTH`: there may be more).
// Codes of a row at D = 64 are half a line, and heads that follow each other on different XCDs fetched every line twice: 32 x 64/8 heads, 8192 keys 94 us, 40/40 heads, 2048 keys
// 114; in pairs (Hkv even) 69 and 84.
template <int D, bool CODES, bool BOTH, int NW, bool TREE = false>
__device__ __forceinline__ void rows_workgroup(const RaggedArgs& a, unsigned id) {
    typedef const __attribute__((address_space(4))) int32_t* const_i32;
    int rest, kvh;
    if (CODES && D == 64 && a.paired) {      // the two heads of a line on one XCD: its L2 fetches the line once
        const unsigned pair = 8u * (id >> 4) + (id & 7u);
        rest = (int)a.by_pairs.of(pair);
        kvh = 2 * ((int)pair - rest * (a.Hkv / 2)) + (int)((id >> 3) & 1u);
        if (rest >= a.B * a.tiles * a.nsplit) return;
    } else {
        rest = (int)a.by_heads.of(id);
        kvh = (int)id - rest * a.Hkv;
    }
    const int part = (int)a.by_seqs.of((unsigned)rest);
    const int sp = part / a.tiles, rt = part - sp * a.tiles;
    int b = rest - part * a.B + sp;
    b -= (int)a.by_seqs.of((unsigned)b) * a.B;
    const int q0 = min(max(((const_i32)(uintptr_t)a.q_off)[b], 0), a.rows);
    const int n = min(max(((const_i32)(uintptr_t)a.q_off)[b + 1], q0), a.rows) - q0;
    const int len = max(min(((const_i32)(uintptr_t)a.lengths)[b], a.max_len), 0);
    const int nrows = min(n, a.max_new) * a.G;
    const int row0 = rows_in_tiles<TREE>(nrows, a.few_rows);
    if (!BOTH || nrows - row0 <= 16) rows_tile<D, CODES, 16, NW, TREE>(a, b, rt, sp, kvh, q0, n, len, row0, nrows);
    else rows_tile<D, CODES, 32, NW, TREE>(a, b, rt, sp, kvh, q0, n, len, row0, nrows);
}

}  // namespace rr
}  // namespace hg
