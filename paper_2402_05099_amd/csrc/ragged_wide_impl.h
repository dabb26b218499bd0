// Causal attention of packed tokens on the matrix cores, 128 query rows to a workgroup: the body shared by ragged_wide.hip (D = 128) and
// ragged_wide_d64.hip (D = 64), which define HG_RW_D.  Prompts, and long chunks but for what remains behind their tiles.
//
// Mathematics and pipeline are those of prefix_wide_impl.h (transposed products with v_mfma_f32_32x32x16_bf16, a lane owns one query row, weights
// against a maximum that is only raised when their sum says so, one step = scores of stage j + 2, weights of stage j + 1 and P V of stage j, written out by
// gen_prefix_wide_step.py).  What differs, and why:
//   * A workgroup is four wavefronts x 32 rows with 80 KiB of LDS, two to a CU, so that one's start (its tile is looked up, Q and
//     the first stages arrive) and end lie under the other's products: a causal tile is short, 16 stages for a prompt of 1000 tokens.  A
//     tile of 128 rows also has half the triangle of one of 256 that is multiplied for nothing, and a wavefront stops at its own last key.
//   * K and V have rings of their own: in step j the K of stages j + 3 .. j + 5 and the V of j + 2 and j + 3 are in flight.  One barrier per step.
//   * A row's own tokens bound its keys: steps that reach that bound, or the end of the keys, mask the scores and copy with care (`kCareful`).
//   * Paged rows: a wavefront copies rows of one page per stage; the pages of its next 64 stages lie in the lanes of a register.
//   * Codes of K are copied to a staging ring of the wavefront's own, and become bf16 on the way from there into the K ring, once per workgroup; those of V stay
//     codes in LDS and become bf16 behind the transposing read, in every wavefront.  The LDS is what codes press on (K and V both expanded into rings: 1767 cycles a
//     stage where bf16 rows take 1417, of which the LDS needs some 770 for each of a CU's two workgroups), and this way the vector ALU carries half of it.
//   * The output is divided by the sum of the rounded weights (LSE has the sum of the unrounded ones): where one key has nearly all the weight its rounding
//     would otherwise show in O as a whole, since the largest weight is anywhere up to kMostWeight and not a power of two.
//
// What bounds it: the matrix pipes, and in calls of a millisecond the board's power.  One prompt of 8192 tokens, 64/8 heads: 0.95-1.01 ms, 1.10-1.16 PFLOP/s of what the mask leaves, at
// 1.67 GHz with the matrix pipes 67 % busy (1417 cycles a stage and workgroup, 1024 of them products; without exponentials, or with half the LDS reads, 5 % less).  16 prompts of up to 2048
// tokens, 40 heads 315-335 us (237 GFLOP; 43 % busy): a tile takes 7.6 us beside its 24 stages of 0.8, half of it until Q and the first rows are there.  45 prompts of up to 515 tokens,
// 16/2 heads 44-47 us: the same 7 us beside seven stages.  2K tokens of two prompts over 8K to 16K keys, 64/8 heads 1.26-1.32 ms, 1.11-1.16 PFLOP/s.
#include <algorithm>
#include <type_traits>

#include "ragged_rows_impl.h"

#pragma clang diagnostic ignored "-Winline-asm"

namespace hg {
namespace rw {
namespace {

constexpr int D = HG_RW_D;
constexpr int KT = D == 128 ? 32 : 64;  // keys per stage: 8 KiB of K and 8 KiB of V as bf16
constexpr int KB = KT / 32;             // 32-key score tiles per stage
constexpr int NW = 4;                   // wavefronts per workgroup
constexpr int NS = 4;                   // steps of a group; V slots
constexpr int KS = D / 16;              // MFMA k-steps of the score product
constexpr int DB = D / 32;              // 32-row blocks of O^T
constexpr int NKF = 4, NVF = 4;         // K and V fragment registers
constexpr int CPR = D / 8;              // 16-byte chunks per bf16 row
constexpr int RPI = 64 / CPR;           // rows one copy instruction covers
constexpr int RPW = KT / NW;            // rows of a stage that one wavefront copies
constexpr int CPW = RPW / RPI;          // ... in this many instructions per tensor
constexpr int ROWB = D * 2;             // bytes per row
constexpr int STB = KT * ROWB;          // bytes per stage and tensor
constexpr int kTileRows = 32 * NW;
static_assert(kTileRows == kTile, "");
constexpr float kMostWeight = 256.f;    // as in prefix_wide_impl.h
constexpr float kRoom = 16.f;
static_assert(CPW == 2 && RPW <= 16, "a wavefront's rows of a stage lie in one page");

enum { kDense = 0, kPaged = 1, kCodes = 2 };
// LDS: K ring (bf16), V ring (bf16 or codes), and for codes the wavefronts' staging rings of K
constexpr int k_slots(int mode) { return mode == kCodes ? 2 : 4; }
constexpr int v_stage(int mode) { return mode == kCodes ? STB / 2 : STB; }
constexpr int kCodeSlots = 4, kCodeBytes = RPW * D;      // staging: stages, and bytes of a wavefront's rows of one
constexpr int lds_bytes(int mode) {
    const int ring = k_slots(mode) * STB + NS * v_stage(mode) + (mode == kCodes ? NW * kCodeSlots * kCodeBytes : 0), results = NW * 32 * 2 * ROWB;
    return ring > results ? ring : results;
}
static_assert(kCodeBytes == 1024, "one copy instruction per wavefront, stage and tensor of codes");
static_assert(lds_bytes(kCodes) + 16 <= 81920 && lds_bytes(kDense) + 16 <= 81920, "two workgroups to a CU");      // (16: a flag)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef int intx2 __attribute__((ext_vector_type(2)));

// XOR swizzles of the 16-byte chunks of LDS row `row`, as in prefix_wide_impl.h
__device__ __forceinline__ int kswz(int row) { return D == 128 ? row % 16 : (row >> 1) & 7; }
__device__ __forceinline__ int vswz(int row) { return D == 128 ? 4 * (row % 4) : 4 * ((row >> 1) & 1); }
// ... and of those of a row of V codes: 32 lanes of a transposing read take 32 bytes of each of the rows 0 .. 3 and 8 .. 11 (or of those four further), 128 or 64 bytes apart
__device__ __forceinline__ int cswz(int row) { return 2 * (D == 128 ? ((row >> 1) & 1) | (((row >> 3) & 1) << 1) : (row >> 3) & 1); }

#if HG_RW_D == 128
typedef floatx16 STile;
#else
struct STile { floatx16 a, b; };
#endif

__device__ __forceinline__ void mfma_first(floatx16& S, const uintx4& a, const bf16x8& b) {
    floatx16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.f;
    S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, z, 0, 0, 0);
}
__device__ __forceinline__ void mfma_acc(floatx16& S, const uintx4& a, const bf16x8& b) {
    S = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, S, 0, 0, 0);
}
__device__ __forceinline__ void mfma_acc(floatx16& O, const shortx8& a, const uintx4& b) {
    O = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), O, 0, 0, 0);
}
__device__ __forceinline__ unsigned pack_bf16_pair(float lo, float hi) {
    floatx2 f = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf16x2));
}
__device__ __forceinline__ float sum_of_pair(unsigned pair, float acc) {      // acc + the pair's two values
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), acc, false);
}
template <int N>
__device__ __forceinline__ void wait_vm() {      // at most N vector memory operations outstanding
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}

extern __shared__ __attribute__((aligned(1024))) unsigned char rw_smem[];

}  // namespace

// Workgroup `id` of those that take tiles.
template <int MODE>
__device__ __forceinline__ void tile_workgroup(const RaggedArgs& a, unsigned id) {
    constexpr bool PAGED = MODE != kDense, CODES = MODE == kCodes;
    constexpr int ES = CODES ? 1 : 2, NKS = k_slots(MODE), VRING = NKS * STB, VSTB = v_stage(MODE), CRING = VRING + NS * VSTB;
    constexpr int KOPS = CODES ? 1 : CPW;                            // copy instructions per stage, tensor and wavefront
    // How far ahead of step j the copies run; the step needs K of stage j + 2 and V of stage j + 1.  Codes: the K that step j expands (of stage j + 3) was requested
    // kCodeSlots - 1 steps before.
    constexpr int KA = CODES ? 3 + kCodeSlots - 1 : 5, VA = 3;
    unsigned char* const smem = rw_smem;

    // ---- which tile, which keys ----
    int tile, kvh, sp;
    RaggedSeq sq;
    {
        // Workgroups whose ids are equal modulo 8 run on one XCD: the tiles of a KV head go to one of them, or to as few as there are heads for, so
        // that its rows are in that XCD's L2.  They go to the shader engines of an XCD in turn, whatever those have to do, so the numbers that are nobody's come
        // last (key ranges slowest, with each range's own of these: drafted tokens behind up to 64K rows of codes, 48 and 30 workgroups to an engine).
        unsigned v;
        if (a.Hkv % 8 == 0) {
            v = a.by_heads8.of(id >> 3);
            kvh = (int)(((id >> 3) - v * (unsigned)(a.Hkv / 8)) * 8u + (id & 7u));
        } else {
            v = a.by_heads.of(id);
            kvh = (int)(id - v * (unsigned)a.Hkv);
        }
        const int rank = (int)(v / (unsigned)a.tile_nsplit);
        sp = (int)(v - (unsigned)rank * (unsigned)a.tile_nsplit);
        if (!tile_of_rank(a, rank, sq, tile)) return;
    }
    const int b = __builtin_amdgcn_readfirstlane(sq.b);
    const int nrows = __builtin_amdgcn_readfirstlane(rows_in_tiles(sq.take * a.G, a.few_rows)), row0 = tile * kTileRows;      // rows that tiles take
    const int q0 = __builtin_amdgcn_readfirstlane(sq.q0);
    const int before = __builtin_amdgcn_readfirstlane(sq.len - (sq.n - 1));      // keys that the sequence's first token sees
    const int tid = threadIdx.x, l = tid & 63, lq = l & 31, hl = l >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const auto token_of = [&](int r) { return (int)a.by_group.of((unsigned)r); };
    const int k0 = sp * a.tile_chunk;
    const int k_all = __builtin_amdgcn_readfirstlane(before + token_of(min(row0 + kTileRows, nrows) - 1)), ke = min(k_all, k0 + a.tile_chunk);      // keys [k0, ke) of k_all
    const int nst = ke > k0 ? (ke - k0 + KT - 1) / KT : 0, nfull = ke > k0 ? (ke - k0) / KT : 0;
    if (sp > 0 && nst == 0) return;      // (the join looks at no part that starts behind a row's keys)
    // stages from here on have keys that some row of the tile does not see
    const int all_see = __builtin_amdgcn_readfirstlane(max(min(before + token_of(row0), ke), k0));
    const int masked = all_see < ke ? (all_see - k0) / KT : nst;
    // this wavefront's rows, and this lane's
    const int wrow0 = row0 + 32 * w;
    const bool any = wrow0 < nrows;
    const int w_least = __builtin_amdgcn_readfirstlane(any ? min(before + token_of(wrow0), ke) : 0);                              // every row of the wavefront sees the keys below
    const int w_most = __builtin_amdgcn_readfirstlane(any ? min(before + token_of(min(wrow0 + 32, nrows) - 1), ke) : 0);          // ... and none those from here on
    const int mine = w_most > k0 ? (w_most - k0 + KT - 1) / KT : 0;      // stages that this wavefront multiplies
    const int r = wrow0 + lq;
    const bool rv = r < nrows;
    const int tok = token_of(rv ? r : row0), head = (rv ? r : row0) - tok * a.G + kvh * a.G;
    const int seen = rv ? min(before + tok, ke) : 0;

    // ---- HBM -> LDS copies: wavefront w copies rows w RPW .. of a stage; the swizzle is applied on the global side ----
    const int64_t kv_stride = a.kv_stride;
    const int lrow = CODES ? l / (D / 16) : l / CPR, lch = CODES ? l % (D / 16) : l % CPR;
    unsigned voffK[KOPS], voffV;
#pragma unroll
    for (int i = 0; i < KOPS; ++i)
        voffK[i] = (unsigned)lrow * (unsigned)kv_stride + (CODES ? (unsigned)lch : (unsigned)(lch ^ kswz(w * RPW + i * RPI + lrow))) * 16u;
    voffV = (unsigned)lrow * (unsigned)kv_stride + (unsigned)(lch ^ (CODES ? cswz(w * RPW + lrow) : vswz(lrow))) * 16u;      // (bf16 rows RPI and RPW apart share their V swizzle)
    const unsigned lds0 = (unsigned)__builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)HG_LDS(smem));
    const unsigned lds_rows = lds0 + (unsigned)(w * RPW * ROWB);
    const unsigned char* const Kh = a.K + (int64_t)kvh * (D * ES);
    const unsigned char* const Vh = a.V + (int64_t)kvh * (D * ES);
    const auto scalar = [](const unsigned char* p) {
        const uint64_t v = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
        return reinterpret_cast<const unsigned char*>(((uint64_t)hi << 32) | lo);
    };
    const auto copy16 = [&](const unsigned char* base, unsigned voff, unsigned dst) {
        asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "s"(dst) : "memory", "m0");
    };
    int pages = 0, page_base = 0;      // lane i: page of this wavefront's rows of stage page_base + i
    const auto look_up = [&](int s0) {
        page_base = s0;
        const int e = min((int)((unsigned)(k0 + (s0 + l) * KT + w * RPW) >> a.pg.shift), a.pg.stride - 1);
        pages = min(max(a.pg.table[(int64_t)b * a.pg.stride + e], 0), a.pg.n_pages - 1);
    };
    const auto row_offset = [&](int s) -> int64_t {      // byte offset of the first of this wavefront's rows of stage s
        const int j = k0 + s * KT + w * RPW;
        if constexpr (PAGED) {
            const int page = __builtin_amdgcn_readlane(pages, (s - page_base) & 63);
            return (((int64_t)page << a.pg.shift) + (j & ((1 << a.pg.shift) - 1))) * kv_stride;
        } else {
            return (int64_t)(q0 + j) * kv_stride;
        }
    };
    // One tensor's rows of stage s to place `at` of its ring (s modulo its slots).  tail: rows may lie behind the last one of the tensor
    // (packed rows); those are read as the last: they are nobody's keys here.
    const auto copy_stage = [&](int s, int at, bool is_k, auto tail) {
        const unsigned char* const tensor = is_k ? Kh : Vh;
        unsigned dst;
        if constexpr (CODES) dst = lds0 + (unsigned)(is_k ? CRING + w * (kCodeSlots * kCodeBytes) + (at % kCodeSlots) * kCodeBytes : VRING + (at % NS) * VSTB + w * kCodeBytes);
        else dst = lds_rows + (unsigned)((is_k ? 0 : VRING) + (at % (is_k ? NKS : NS)) * STB);
        if constexpr (decltype(tail)::value && !PAGED) {
#pragma unroll
            for (int i = 0; i < KOPS; ++i) {
                const int j = q0 + k0 + s * KT + w * RPW + i * RPI, base = min(j, a.rows - 1);
                const int back = lrow - (min(j + lrow, a.rows - 1) - base);      // by how many rows this lane's comes before the one it would copy, at most lrow
                copy16(scalar(tensor + (int64_t)base * kv_stride), (is_k ? voffK[i] : voffV) - (unsigned)back * (unsigned)kv_stride, dst + (unsigned)i * 1024u);
            }
        } else {
            const unsigned char* const first = scalar(tensor + row_offset(s));
#pragma unroll
            for (int i = 0; i < KOPS; ++i) copy16(scalar(first + (int64_t)(i * RPI) * kv_stride), is_k ? voffK[i] : voffV, dst + (unsigned)i * 1024u);
        }
    };
    // codes: this wavefront's rows of K out of the staging ring, and as bf16 into the K ring (`at`: the stage, or a number equal to it modulo 4)
    const auto read_codes = [&](int at) -> uintx4 {
        return *reinterpret_cast<const uintx4*>(smem + CRING + w * (kCodeSlots * kCodeBytes) + (at % kCodeSlots) * kCodeBytes + l * 16);
    };
    const auto bf16_of = [](unsigned c0, unsigned c1) -> uintx4 {      // eight codes
        return uintx4{__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, 1.0f, false)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, 1.0f, true)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, 1.0f, false)),
                      __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, 1.0f, true))};
    };
    const auto write_k = [&](int at, const uintx4& c) {
        const int row = w * RPW + lrow;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<uintx4*>(smem + (at % NKS) * STB + row * ROWB + (((2 * lch + h) ^ kswz(row)) * 16)) = bf16_of(c[2 * h], c[2 * h + 1]);
    };
    const auto expand = [&](int s) { write_k(s, read_codes(s)); };

    // ---- LDS fragment reads, as in prefix_wide_impl.h ----
    unsigned kaddr[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) kaddr[s] = (unsigned)(lq * ROWB + (((2 * s + hl) ^ kswz(lq)) * 16));
    unsigned vaddr[DB];
    {
        const int i16 = l & 15, g1 = (l >> 4) & 1;
        const int keyq = 4 * hl + (i16 >> 2);
        const int fv = vswz(keyq);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            if constexpr (CODES) {      // ds_read_b64_tr_b8, see decode_mfma_core.h: lane s of 16 points at key 8 (j / 4) + 4 hl + j % 4, j = s / 2, columns 16 g1 + 8 (s % 2) .. + 7
                const int j = i16 >> 1, row = 8 * (j >> 2) + 4 * hl + (j & 3);
                vaddr[db] = (unsigned)(VRING + row * D + (((2 * db + g1) ^ cswz(row)) * 16) + (i16 & 1) * 8);
            } else {
                const int chunk = 4 * db + 2 * g1 + ((i16 & 3) >> 1);
                vaddr[db] = (unsigned)(VRING + keyq * ROWB + ((chunk ^ fv) * 16) + (i16 & 1) * 8);
            }
        }
    }
    const auto lds_k = [&](int slot, int f) -> uintx4 {
        return *reinterpret_cast<const uintx4*>(smem + (slot % NKS) * STB + (f / KS) * 32 * ROWB + kaddr[f % KS]);
    };
    typedef std::conditional_t<CODES, intx2, shortx8> VFragment;
    const auto lds_v = [&](int slot, int tt, int db) -> VFragment {
        const unsigned char* vp = smem + slot * VSTB + vaddr[db] + tt * 16 * (D * ES);
        if constexpr (CODES) {
            return __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) intx2*)HG_LDS(vp));
        } else {
            const shortx4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)HG_LDS(vp));
            const shortx4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) shortx4*)HG_LDS(vp + 8 * ROWB));
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };
    const auto v_operand = [&](const VFragment& v) -> shortx8 {
        if constexpr (CODES) return __builtin_bit_cast(shortx8, bf16_of((unsigned)v[0], (unsigned)v[1]));
        else return v;
    };

    // ---- online softmax state ----
    floatx16 Oacc[DB];
    float lsum, lround;         // this lane's share of the row's sum: of the unrounded weights, of the rounded ones
    float mc;                   // what the exponents are taken against, log2 units
    const float c2 = a.scale * kLog2e;
    const auto weights = [&](const STile& S, uintx4 (&p)[KT / 16], float& rsum) -> float {
        float sa = 0.f, sb = 0.f;
        rsum = 0.f;
#pragma unroll
        for (int h = 0; h < KT / 16; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = 8 * (h & 1) + 2 * i;
#if HG_RW_D == 128
                const float x0 = S[e], x1 = S[e + 1];
#else
                const float x0 = h < 2 ? S.a[e] : S.b[e], x1 = h < 2 ? S.a[e + 1] : S.b[e + 1];
#endif
                const float ea = __builtin_amdgcn_exp2f(fmaf(x0, c2, -mc)), eb = __builtin_amdgcn_exp2f(fmaf(x1, c2, -mc));
                const unsigned pair = pack_bf16_pair(ea, eb);
                p[h][i] = pair;
                rsum = sum_of_pair(pair, rsum);
                sa += ea;
                sb += eb;
            }
        return sa + sb;
    };
    const auto tile_max = [&](const STile& S) -> float {
#if HG_RW_D == 128
        float t = fmaxf(S[0], S[1]);
#pragma unroll
        for (int i = 2; i < 16; i += 2) t = fmaxf(fmaxf(t, S[i]), S[i + 1]);
#else
        float t = fmaxf(S.a[0], S.b[0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) t = fmaxf(fmaxf(t, S.a[i]), S.b[i]);
#endif
        return half_max(t);
    };
    const auto mask_stage = [&](STile& S, int s) {      // keys of stage s that this lane's row does not see
        const int hi = seen - (k0 + s * KT) - 4 * hl;   // row i of this lane is 8 (i / 4) + i % 4 + 4 hl (+ 32 in the second tile)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int ri = 8 * (i >> 2) + (i & 3);
#if HG_RW_D == 128
            if (ri >= hi) S[i] = -INFINITY;
#else
            if (ri >= hi) S.a[i] = -INFINITY;
            if (ri + 32 >= hi) S.b[i] = -INFINITY;
#endif
        }
    };

    // Copies of the start and of careful steps: with a look at the tensor's end only where the tile's keys come near it.
    const bool edge = !PAGED && q0 + k0 + nst * KT > a.rows;
    const auto copy_some = [&](auto what) {
        if constexpr (PAGED) {
            what(std::false_type{});
        } else {
            if (__builtin_expect(edge, 0)) what(std::true_type{});
            else what(std::false_type{});
        }
    };

    // ---- start: the first stages, Q, the stages behind them ----
    if constexpr (PAGED) look_up(0);
    copy_some([&](auto tail) {
        if constexpr (CODES) {
            static_assert(kCodeSlots == 4, "");
#pragma unroll
            for (int s = 0; s < kCodeSlots; ++s) {
                if (s < nst) copy_stage(s, s, true, tail);
                if (s < VA && s < nst) copy_stage(s, s, false, tail);
            }
        } else {
            if (0 < nst) { copy_stage(0, 0, true, tail); copy_stage(0, 0, false, tail); }
            if (1 < nst) copy_stage(1, 1, true, tail);
        }
    });
    bf16x8 qf[KS];
    {
        const unsigned char* const qp = reinterpret_cast<const unsigned char*>(a.Q) + (int64_t)(q0 + tok) * a.q_stride + head * ROWB + 16 * hl;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uintx4*>(qp + 32 * s));
#pragma unroll
        for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));
    }
    wait_vm<0>();
    // Rows of the last stage from ke on may hold anything, and 0 * NaN would be NaN: whoever has copied them clears them once they have landed
    const int partial = nst > nfull ? nst - 1 : -1;
    const auto clear_rows = [&](int s) {
        constexpr int RPC = CODES ? RPW : RPI;      // rows of one copy instruction
#pragma unroll
        for (int i = 0; i < KOPS; ++i)
            if (k0 + s * KT + w * RPW + i * RPC + lrow >= ke) *reinterpret_cast<uintx4*>(smem + VRING + (s % NS) * VSTB + (w * RPW + i * RPC) * (D * ES) + l * 16) = uintx4{0u, 0u, 0u, 0u};
    };
    // Whoever has copied the values of a stage that some row does not see as a whole takes those out that are not finite (take_out, ragged.h)
    unsigned char* const flag = smem + lds_bytes(MODE);
    bool spoiled = false;
    const auto finite_only = [&](int s) {
        constexpr int RPC = CODES ? RPW : RPI;
        if (take_out<CODES, KOPS>(smem + VRING + (s % NS) * VSTB + w * RPW * (D * ES) + l * 16, RPC * (D * ES))) spoiled = true;
    };
    const auto meet = [&]() {      // barrier of the workgroup, which no memory operation is moved over
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    const auto lds_done = [&]() { __builtin_amdgcn_s_waitcnt(0xC07F); };      // lgkmcnt(0)
    if constexpr (CODES) {
        // there are only two K slots: stage 2 waits for the scores of stage 0 (below)
        if (0 < nst) expand(0);
        if (1 < nst) expand(1);
        if (partial == 0) clear_rows(0);
        if (masked == 0 && nst > 0) finite_only(0);
        copy_some([&](auto tail) {
            if (4 < nst) copy_stage(4, 4, true, tail);
            if (5 < nst) copy_stage(5, 5, true, tail);
        });
    } else {
        if (partial == 0) clear_rows(0);
        if (masked == 0 && nst > 0) finite_only(0);
        // (in this order: step 0 waits for all but the last K and the last V)
        copy_some([&](auto tail) {
            if (2 < nst) copy_stage(2, 2, true, tail);
            if (1 < nst) copy_stage(1, 1, false, tail);
            if (3 < nst) copy_stage(3, 3, true, tail);
            if (2 < nst) copy_stage(2, 2, false, tail);
        });
        // K of stage 4 has the slot of stage 0, whose scores are taken first
    }
    if (tid == 0) *reinterpret_cast<int*>(flag) = 0;
    lds_done();
    meet();

    uintx4 kf[NKF];
    VFragment vf[NVF];
    STile SA, SB;
    uintx4 PA[KT / 16], PB[KT / 16];
    if (mine > 0) {      // scores of the first two stages, product by product in turn (each waits for its own one before)
        uintx4 k0[KB * KS], k1[KB * KS];
#pragma unroll
        for (int q = 0; q < KB * KS; ++q) { k0[q] = lds_k(0, q); k1[q] = lds_k(1, q); }
#if HG_RW_D == 128
        mfma_first(SB, k0[0], qf[0]);
        mfma_first(SA, k1[0], qf[0]);
#pragma unroll
        for (int q = 1; q < KS; ++q) { mfma_acc(SB, k0[q], qf[q]); mfma_acc(SA, k1[q], qf[q]); }
        asm volatile("s_nop 11" : "+v"(SB), "+v"(SA));
#else
        mfma_first(SB.a, k0[0], qf[0]);
        mfma_first(SB.b, k0[KS], qf[0]);
        mfma_first(SA.a, k1[0], qf[0]);
        mfma_first(SA.b, k1[KS], qf[0]);
#pragma unroll
        for (int q = 1; q < KS; ++q) {
            mfma_acc(SB.a, k0[q], qf[q]);
            mfma_acc(SB.b, k0[KS + q], qf[q]);
            mfma_acc(SA.a, k1[q], qf[q]);
            mfma_acc(SA.b, k1[KS + q], qf[q]);
        }
        asm volatile("s_nop 11" : "+v"(SB.a), "+v"(SB.b), "+v"(SA.a), "+v"(SA.b));
#endif
        __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (CODES) {
        // K of stage 2 takes the slot of stage 0 when everyone has its scores
        meet();
        if (2 < nst) expand(2);
    } else {
        meet();
        copy_some([&](auto tail) { if (4 < nst) copy_stage(4, 4, true, tail); });
    }
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) Oacc[i][k] = 0.f;
    lsum = lround = 0.f;
    mc = 0.f;
    if (mine > 0) {
        if (k0 + KT > w_least) mask_stage(SB, 0);
        // (a finite number for a row with nothing but -inf, see prefix_wide_impl.h)
        mc = fmaxf(tile_max(SB) * c2, -3.4028234e38f);
        lsum = weights(SB, PA, lround);
#pragma unroll
        for (int i = 0; i < NVF; ++i) vf[i] = lds_v(0, i / DB, i % DB);
    }

    // ---- steps ----
    // what step j starts with: everyone's copies for it have landed, everyone has finished step j - 1
    const auto add_sum = [&](const STile& S, float ssum, float rsum, uintx4 (&pn)[KT / 16]) {
        if (__builtin_expect(__any(!(ssum <= kMostWeight)), 0)) {
            float top = tile_max(S) * c2;
            if (__builtin_popcountll(__ballot(top > mc + 2.0f)) >= 48) top += kRoom;
            const float mc_new = fmaxf(mc, top);
            const float alpha = __builtin_amdgcn_exp2f(mc - mc_new);
            mc = mc_new;
            lsum *= alpha;
            lround *= alpha;
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                Oacc[i] *= alpha;
                __builtin_amdgcn_sched_barrier(0);
            }
            ssum = weights(S, pn, rsum);
        }
        lsum += ssum;
        lround += rsum;
    };
    // The wait before step j: its K and V have landed while the younger copies may be in flight (those of the step before, careful ones only where there were any)
    const auto wait_plain = [&]() {
        wait_vm<2 * KOPS>();
    };
    const auto wait_careful = [&](int j) {
        if (j + KA - 1 < nst) wait_vm<2 * KOPS>();
        else if (j + VA - 1 < nst) wait_vm<KOPS>();
        else wait_vm<0>();
    };
    const auto before_step = [&](int j) {      // the careful form; the partial stage's V rows are first read in the step before its own
        wait_careful(j);
        if (j + 1 == partial) clear_rows(partial);
        if (j + 1 >= masked && j + 1 < nst) finite_only(j + 1);
        lds_done();
        meet();
    };
    const auto careful_copies = [&](int j) {
        copy_some([&](auto tail) {
            if (j + KA < nst) copy_stage(j + KA, j + KA, true, tail);
            if (j + VA < nst) copy_stage(j + VA, j + VA, false, tail);
        });
    };
    const auto careful_expand = [&](int j) {
        if constexpr (CODES) {
            if (j + 3 < nst) expand(j + 3);
        }
    };
    const auto step = [&](int j, auto slotc, auto careful) {
        constexpr int slot = decltype(slotc)::value;
        constexpr bool kCareful = decltype(careful)::value;
        STile &Scur = slot % 2 == 0 ? SA : SB, &Snext = slot % 2 == 0 ? SB : SA;
        uintx4 (&pb)[KT / 16] = slot % 2 == 0 ? PA : PB, (&pn)[KT / 16] = slot % 2 == 0 ? PB : PA;
        constexpr int slot1 = (slot + 1) % NS, slot2 = (slot + 2) % NS;
        if constexpr (kCareful) {
            before_step(j);
            if (k0 + (j + 2) * KT > w_least) mask_stage(Scur, j + 1);
            careful_copies(j);
            careful_expand(j);
        } else {
            wait_plain();
            if constexpr (CODES) lds_done();
            meet();
        }
        float ssum, rsum;
        {
            const auto issue_k = [&](int j, int slot) { if constexpr (!kCareful) copy_stage(j + KA, slot + KA, true, std::false_type{}); };
            const auto issue_v = [&](int j, int slot) { if constexpr (!kCareful) copy_stage(j + VA, slot + VA, false, std::false_type{}); };
            uintx4 ck{};
            const auto read_k = [&](int slot) { if constexpr (!kCareful && CODES) ck = read_codes(slot + 3); };
            const auto work_k = [&](int slot) { if constexpr (!kCareful && CODES) write_k(slot + 3, ck); };
#if HG_RW_D == 128
#include "ragged_wide_step.inc"
#else
#include "ragged_wide_step_d64.inc"
#endif
        }
        add_sum(Scur, ssum, rsum, pn);
    };
    int j = 0;
    // groups of plain steps: every copy they make is of a full stage, every weight they take, and the values they are the first to read, of a stage that all rows see
    const int plain = min(min(nfull - KA, (w_least - k0) / KT - 1), masked - 1);
    for (; j + NS <= plain; j += NS) {
        if constexpr (PAGED) {
            if (j + NS + KA > page_base + 64) look_up(j);
        }
        step(j, std::integral_constant<int, 0>{}, std::false_type{});
        step(j + 1, std::integral_constant<int, 1>{}, std::false_type{});
        step(j + 2, std::integral_constant<int, 2>{}, std::false_type{});
        step(j + 3, std::integral_constant<int, 3>{}, std::false_type{});
    }
    for (; j < mine; j += NS) {
        if constexpr (PAGED) {
            if (j + NS + KA > page_base + 64) look_up(j);
        }
        step(j, std::integral_constant<int, 0>{}, std::true_type{});
        if (j + 1 < mine) {
            step(j + 1, std::integral_constant<int, 1>{}, std::true_type{});
            if (j + 2 < mine) {
                step(j + 2, std::integral_constant<int, 2>{}, std::true_type{});
                if (j + 3 < mine) step(j + 3, std::integral_constant<int, 3>{}, std::true_type{});
            }
        }
    }
    // stages that only the others multiply: this wavefront keeps its share of the copies going
    for (j = mine; j < nst; ++j) {
        if constexpr (PAGED) {
            if (j + 1 + KA > page_base + 64) look_up(j);
        }
        before_step(j);
        careful_copies(j);
        careful_expand(j);
    }

    // ---- results: a wavefront's 32 rows through LDS, to leave as whole lines (the ring is free once everyone is here) ----
    wait_vm<0>();
    if (spoiled && l == 0) *reinterpret_cast<int*>(flag) = 1;
    lds_done();
    meet();
    if (!any) return;
    if (__builtin_expect(*reinterpret_cast<const volatile int*>(flag) != 0, 0)) {      // the rows that see what was taken out
#pragma unroll 1
        for (int key = k0 + masked * KT; key < ke; ++key) {
            int64_t row;
            if constexpr (PAGED) {
                const int page = min(max(a.pg.table[(int64_t)b * a.pg.stride + min(key >> a.pg.shift, a.pg.stride - 1)], 0), a.pg.n_pages - 1);
                row = ((int64_t)page << a.pg.shift) + (key & ((1 << a.pg.shift) - 1));
            } else {
                row = q0 + key;
            }
            if (key >= seen) continue;
            const unsigned char* const vr = Vh + row * kv_stride + 4 * hl * ES;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
                    for (int i = 0; i < 4; ++i) Oacc[db][4 * q4 + i] += value_if_not_finite<CODES>(vr + (32 * db + 8 * q4 + i) * ES);
        }
    }
    const float ltot = half_sum(lsum), lr = half_sum(lround);
    const float inv = lr == 0.f ? 0.f : a.v_scale / lr;      // (a row whose scores are NaN stays NaN)
    const bool in_parts = k_all > a.tile_chunk;      // (a tile of one range has the result itself)
    const int64_t row_at = (int64_t)(q0 + tok) * a.Hq + head;
    if (rv && hl == 0) {
        const float lse = ltot == 0.f ? -INFINITY : (mc + __log2f(ltot)) * kLn2;
        if (in_parts) a.tile_part_L[(int64_t)sp * a.rows * a.Hq + row_at] = part_lse(lse);
        else if (a.out.LSE) a.out.LSE[row_at] = lse;
    }
    float* const Of = in_parts ? a.tile_part_O + (int64_t)sp * a.rows * a.Hq * D : static_cast<float*>(a.out.O);
    uint16_t* const Ob = static_cast<uint16_t*>(a.out.O);
    const int my_row = rv ? (int)row_at : -1;
    const auto element = [&](int db, int q4, int i) { return Oacc[db][4 * q4 + i] * inv; };      // column 32 db + 8 q4 + 4 hl + i of row lq
    if (a.out.bf16 && !in_parts) {
        unsigned char* const stg = smem + w * (32 * ROWB);
        // pieces of four columns, 8 bytes, at piece ^ 2 (row % 8): rows are 256 (128) bytes, a whole number of bank periods (half a one)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<uint2*>(stg + lq * ROWB + (((8 * db + 2 * q4 + hl) ^ (2 * (lq & 7))) * 8)) =
                    make_uint2(pack_bf16_pair(element(db, q4, 0), element(db, q4, 1)), pack_bf16_pair(element(db, q4, 2), element(db, q4, 3)));
#pragma unroll
        for (int kk = 0; kk < 32 / RPI; ++kk) {
            const int rr = RPI * kk + l / CPR, c = l % CPR;
            const uint4 v = *reinterpret_cast<const uint4*>(stg + rr * ROWB + ((c ^ (rr & 7)) * 16));
            const int row = __shfl(my_row, rr);
            if (row >= 0) *reinterpret_cast<uint4*>(Ob + (int64_t)row * D + 8 * c) = v;
        }
    } else {
        unsigned char* const stg = smem + w * (32 * 2 * ROWB);
        constexpr int PCS = D / 4;      // 16-byte pieces of an fp32 row
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<float4*>(stg + lq * (2 * ROWB) + (((8 * db + 2 * q4 + hl) ^ (lq & 15)) * 16)) =
                    make_float4(element(db, q4, 0), element(db, q4, 1), element(db, q4, 2), element(db, q4, 3));
#pragma unroll
        for (int kk = 0; kk < 32 * PCS / 64; ++kk) {
            const int rr = (64 / PCS) * kk + l / PCS, c = l % PCS;
            const float4 v = *reinterpret_cast<const float4*>(stg + rr * (2 * ROWB) + ((c ^ (rr & 15)) * 16));
            const int row = __shfl(my_row, rr);
            if (row >= 0) *reinterpret_cast<float4*>(Of + (int64_t)row * D + 4 * c) = v;
        }
    }
}

}  // namespace rw

using namespace rw;

// Packed rows: tiles are all there is.  Paged rows: what remains behind the tiles is in the same launch: they are bound by the matrix pipes, the
// others by the reads of their cache, and two workgroups of either kind share a CU.  While there are both, 256 workgroups of one kind, one for every CU, come
// after 256 of the other.
template <int MODE>
__global__ __launch_bounds__(64 * NW, 2) void HG_RW_KERNEL(RaggedArgs a) {
    if constexpr (MODE == kDense) {
        tile_workgroup<MODE>(a, blockIdx.x);
    } else {
        const unsigned tiles = (unsigned)a.tiles_all * (unsigned)a.Hkv * (unsigned)a.tile_nsplit, rows = a.row_wgs;
        const unsigned both = min((tiles + 255u) / 256u, (rows + 255u) / 256u), block = blockIdx.x >> 8, in = blockIdx.x & 255u;
        const bool is_tile = block < 2u * both ? (block & 1u) == 0u : tiles > rows;
        const unsigned id = (block < 2u * both ? block >> 1 : block - both) * 256u + in;
        if (id >= (is_tile ? tiles : rows)) return;
        if (is_tile) tile_workgroup<MODE>(a, id);
        else rr::rows_workgroup<D, MODE == kCodes, true, NW>(a, id);
    }
}

template <int MODE>
static hipError_t launch_mode(const RaggedArgs& a, hipStream_t s) {
    constexpr int bytes = MODE == kDense ? lds_bytes(MODE) + 16 : std::max(lds_bytes(MODE) + 16, rr::rows_lds<D, MODE == kCodes, true>(NW));
    static_assert(bytes <= 81920, "two workgroups to a CU");
    const int64_t grid = ragged_grid(a);
    if (grid >= (1LL << 31)) return hipErrorInvalidValue;
    static bool attr_set[64] = {};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&HG_RW_KERNEL<MODE>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    HG_RW_KERNEL<MODE><<<(unsigned)grid, 64 * NW, bytes, s>>>(a);
    return hipGetLastError();
}

hipError_t HG_RW_LAUNCH(const RaggedArgs& a, bool codes, hipStream_t s) {
    if (!a.pg.table) return launch_mode<kDense>(a, s);
    return codes ? launch_mode<kCodes>(a, s) : launch_mode<kPaged>(a, s);
}

}  // namespace hg
