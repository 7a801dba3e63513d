// Ragged causal verify attention over a paged cache of e4m3 codes with a scale for
// each block of tokens and head, on gfx950 matrix cores: head sizes up to 256, any
// page of 16-key blocks, bf16 and fp32 queries.
//
//   score(row, key) = s_k(block of key) * (q . code_k),  out = sum p * s_v(block) * code_v
//
// The codes widen to bf16 exactly (one instruction for two), so they enter bf16
// products as they are, and the scales stay outside: s_k multiplies the fp32 scores
// (a lane's eight keys lie in one block, so by one value), s_v the fp32
// probabilities.  fp32 queries enter as three bf16 terms (24 bits: exact), and so do
// their probabilities (2^-24), with the values' codes as bf16.  bf16 queries enter as
// they are, and their p * s_v rounded once to fp16 (2^-11, a quarter of the bf16
// output's 2^-9, and the values' codes as fp16): one product where two bf16 terms (2^-17)
// take two and four more instructions a value; 128 requests 283 us against 373.
// (The fp8 products of this part add with few bits: 2^-10 of a score's largest product.)
//
// Half the cache's bytes of bf16, the same products: bound by HBM, with the widening
// and the softmax on the vector ALUs next.  The work is cut as in attn_stream.hip into
// equal ranges of the batch's steps (attn_ranges.h), the heads of a range on one XCD
// (token-major pages have them side by side).  Whole calls: 128 requests of 2K-16K keys,
// 64/8 heads of 128, 565 tokens: 284 us, 4.4 TB/s; 16 of 32K-131K keys: 534 us, 5.0 TB/s; 256
// decoding on 16-token token-major pages of heads of 64: 144 us, 4.2 TB/s; 4 requests of
// 2K-16K keys: 37-42 us.  A range's worker is
//
//   * for few rows a single wave with one K and one V buffer in LDS, refilled as soon as
//     its operands are in registers: nothing in its loop waits for another wave, and
//     eight or twelve workers a CU hide its chain of dependences.  Its two row tiles share
//     one widening of the keys and values.  Four workers are a workgroup: consecutive
//     ones, so heads of one range, which on one CU stay abreast (a SIMD's oldest wave
//     goes first) and find each other's lines (256 decoding requests 154 against 143 us);
//   * for many rows four waves of one tile that share a ring of three buffers: every
//     wave copies a part of each step, two steps ahead, and all meet once a step.
//
//   * K and V rows are copied from their page straight into LDS, 32 or 64 keys a
//     step, 16 of them inside one page.  Rows are 16 * CH bytes (padded head sizes are
//     filled from a zero block), chunks XOR-swizzled by the copy so that the operand
//     reads are free of bank conflicts.  A step's scales are one more copy, of a value
//     per 16 keys.
//   * S^T = K Q^T on v_mfma_f32_16x16x32_bf16: a 16-byte read has 16 dims of a key, two
//     operand slices (the queries are laid out alike).  The keys of an operand row
//     are permuted so that the scores already have the B layout of the next product.
//   * O^T += V^T P^T, V^T by transposing 8-byte reads (eight keys of a dim).
//   * softmax online in exp2 units relative to a reference that seldom moves (exact
//     after the final normalisation), below;
//   * a worker that finds a sum non-finite, or too low for the rounding of what it adds up,
//     computes its rows again key by key (scaled_rows), so that a non-finite value reaches
//     only the rows that see it.  Slow: 16 ms where one of 128 requests has such rows.
#include <algorithm>
#include <type_traits>

#include "attn_ranges.h"

namespace dspark {
namespace scaled {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) float lds_f32;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// A row's reference m: its exponents are relative to it.  It moves when one exceeds it by
// kHead, to kBias below that.  fp32: of the scores, p is at most 2^8.  bf16 queries: of
// the scores + log2 |s_v|, so that p * s_v, which fp16 holds, is at most 2^15 and of full
// precision down to 2^-25 of the row's largest (fp16 is normal from 2^-14); p alone is
// fp32 (scales outside 2^-100 .. 2^100 count as those; larger ones overflow, and their rows
// are computed again).  2^4 is what a row's largest product may grow until its reference
// moves; with 2^8 (kBias 7) no call was more than 1 % faster.
template <bool F32> struct Ref {
    static constexpr float kBias = F32 ? 0.0f : 11.0f, kHead = F32 ? 8.0f : 15.0f;
};
constexpr float kMaxLog = 100.0f;
// Where the largest p * s_v goes with values near zero, what counts may be what fp16 rounds
// to multiples of 2^-24: an error of at most 2^-25 a key, times the largest code.  So a row
// is computed again where a code of its range is above kFine of the row's largest sum by the
// range's keys: there the error could exceed 2^-9 of that sum.  (A key with p * s_v of 2^11
// and a value of 1 is enough for 299000 keys, whatever the others' codes.)
constexpr float kFine = 65536.0f;
constexpr float kMaxCode = 448.0f;
constexpr int kMinUnits = 4;         // steps per wave, at least
constexpr int kPageRegs = 2;         // page ids per lane: 128 pages of a range at a time
constexpr int kMaxD = 256;
constexpr int kGroup = 4;            // single-wave workers of a workgroup

// CH: 16-byte chunks of an LDS row: head sizes up to 16 * CH.  W: waves of a worker;
// T: 16-row tiles of a wave.
template <bool F32, int CH, int W, int T>
struct Cfg {
    static constexpr int H = CH <= (W == 1 ? 4 : 8) ? 2 : 1;  // 32-key halves of a step
    static constexpr int Step = 32 * H;
    static constexpr int P = 2 * H;             // 16-key pieces
    static constexpr int S = CH / 4;            // 16-byte operand reads of a key; copies of a piece
    static constexpr int RowB = 16 * CH;
    static constexpr int TileB = Step * RowB;
    static constexpr int Dp = 16 * CH;          // padded head size
    static constexpr int DB = CH;               // 16-dim output blocks
    static constexpr int TQ = F32 ? 3 : 1;      // terms of a query (bf16)
    static constexpr int TP = F32 ? 3 : 1;      // of a probability (bf16; fp16)
    static constexpr int Rows = 16 * W * T;     // of a chunk
    // scales in LDS: of piece h at h * ScaleStep, the values' ScaleV behind the keys'
    static constexpr int ScaleStep = W == 1 ? 4 : 256 * W / P, ScaleV = W == 1 ? 4 * P : 4;
    static constexpr int BufB = 2 * TileB + 256 * W;          // K, V, scales
    static constexpr int Ring = W == 1 ? 1 : 3;  // buffers
    static constexpr int LdsB = Ring * BufB;                  // of a worker
    static constexpr int Group = W == 1 ? kGroup : 1;         // workers of a workgroup
    static constexpr int LdsFit = 160 * 1024 / LdsB;          // workers of a CU, by LDS
    // registers: accumulators, queries, scores and probabilities of the row tiles; operands
    static constexpr int Hr = W == 1 ? H : 1;  // (halves at a time)
    static constexpr int Regs = T * (4 * DB + 8 * S * TQ + Hr * (8 + 4 * TP)) + 8 * Hr * S + 80;
    static constexpr int RegFit = (Regs <= 128 ? 16 : Regs <= 168 ? 12 : Regs <= 256 ? 8 : 4) / W;
    static constexpr int Cu = LdsFit < RegFit ? LdsFit : RegFit;  // workers of a CU
    static constexpr int Eu = Cu * W >= 16 ? 4 : Cu * W >= 12 ? 3 : Cu * W >= 8 ? 2 : 1;  // waves of a SIMD
};

struct Params : Ranges {
    CacheScales cs;
    int64_t ks1, vs1;                // cache strides in bytes
    uint32_t ks0, vs0, ks2, vs2;
    int pad;                         // some row is shorter than the LDS row
    int nb;                          // blocks of a page
    uint32_t per_block;              // ceil(2^32 / (16-key pieces of a block))
    float scale2;
};

// Physical chunk of chunk c in LDS row t: XORs that keep c inside the row.  gfx950
// serves a 16-byte LDS read in four 16-lane phases (lanes split by bit 5 and the
// parity of bits 2 ^ 3 ^ 4) and a transposing 8-byte read in two 32-lane halves, over
// 64 four-byte banks.  A phase of the K read has the 16 rows 8 g + 0 .. 3 (or + 4 .. 7),
// g = 0 .. 3, with one chunk or its neighbour (the two middle g); a half of the V read
// 16 consecutive rows of one chunk.  With these, all of them are on distinct banks:
// a row of 4 chunks leaves four rows, of 8 two, in a line of banks.
template <int CH>
__device__ __forceinline__ int k_slot(int t, int c) {
    const int g = (t >> 3) & 3;
    if (CH == 4) return c ^ ((4 - g) & 3);
    if (CH == 8) return c ^ (((t >> 1) & 1) | (g << 1));
    return c ^ ((t & 3) | (g << 2));
}
template <int CH>
__device__ __forceinline__ int v_slot(int t, int c) {
    if (CH == 4) return c ^ ((t >> 2) & 3);
    if (CH == 8) return c ^ ((t >> 1) & 7);
    return c ^ (t & 15);
}

// zeros (zero-initialised at load, never written): keys at or past the context's end
// and the pad of short rows are copied from here
__device__ __align__(16) uint32_t g_zero[4];

// The wait is the builtin, which the compiler counts: with every ordinary load
// waited for before the step loop, it adds no wait of its own inside it.
template <int N>
__device__ __forceinline__ void wait_copies() {
    wait_vmcnt<N>();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// eight codes as fp16 (exact)
__device__ __forceinline__ f16x8 widen_half(uint32_t lo, uint32_t hi) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
    return __builtin_bit_cast(f16x8, r);
}

// eight codes as bf16 (exact)
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return __builtin_bit_cast(bf16x8, r);
}

// two values as T bf16 terms each: x = sum of the terms to within 2^-(8 T + 1)
template <int T>
__device__ __forceinline__ void terms(float a, float b, uint32_t (&w)[T]) {
#pragma unroll
    for (int t = 0; t < T; ++t) {
        w[t] = cvt_pk_bf16(a, b);
        if (t + 1 < T) {
            a -= __uint_as_float(w[t] << 16);
            b -= __uint_as_float(w[t] & 0xffff0000u);
        }
    }
}

// A value that the compiler cannot compute ahead: what the rare branches of a loop need
// would otherwise sit in registers throughout it.
__device__ __forceinline__ int here(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// block of a page that slot `slot` lies in: exact for pages below 2^20 keys
__device__ __forceinline__ uint32_t block_of(const Params& p, int slot) {
    return p.cs.block == 16 ? slot >> 4 : (uint32_t)(((uint64_t)(uint32_t)(slot >> 4) * p.per_block) >> 32);
}

__device__ __forceinline__ int clamp_page(const Params& p, int page) { return min(max(page, 0), p.cs.num_pages - 1); }

// Which tiles a wave of a worker takes (those of this place, every W).  The workers of a CU
// differ, so that few tiles leave no SIMD of it idle.
template <int W>
__device__ __forceinline__ int place(int wave) {
    return W == 1 ? 0 : (wave + 2 * (int)(blockIdx.x / kRangeCUs)) % W;
}

// The rows of a chunk over the same steps key by key on the vector ALUs, in fp32, where the
// products came out non-finite or too low for their roundings: a product over 16 rows and
// 32 keys also multiplies the keys that a row does not see, by a probability of 0, and 0
// times a non-finite value is NaN.  Every row takes only its own keys here, as the
// vector-ALU kernels do.  Codes up to `fine` need nothing (below 0: rows are not finite):
// a look at the values goes first, which a cache of zeros or of small values under a
// scale of 1 pays alone.
template <bool F32, int CH, int W, int T>
__device__ __forceinline__ void scaled_rows(const Params& p, const int r, const int g, const int rc, const int q0,
                                            const int ql, const int kv, const int s0, const int s1, const int ns,
                                            const int64_t slot, const float fine) {
    typedef Cfg<F32, CH, W, T> C;
    typedef typename std::conditional<F32, float, uint16_t>::type E;
    constexpr int kPer = (C::Dp + DSPARK_WAVE - 1) / DSPARK_WAVE;  // value dims per lane
    const AttnArgs& a = p.a;
    // (values in vector registers: the scalar ones that this would add to the kernel's
    // are spilled into vector registers that the step loop then lacks)
    int z = 0;
    asm volatile("" : "+v"(z));
    const int lane = threadIdx.x & (DSPARK_WAVE - 1), wave = threadIdx.x / DSPARK_WAVE;
    const int page = a.page + z, group = p.group + z, gv = g + z;
    const int row0 = (rc + z) * C::Rows, nrows = min(C::Rows, ql * group - row0);
    const int32_t* bt = a.block_table + (int64_t)(r + z) * a.max_pages;
    const uint8_t* kc = (const uint8_t*)a.k + gv * p.ks1;
    const uint8_t* vc = (const uint8_t*)a.v + gv * p.vs1;
    const bool whole = s0 + z == 0 && s1 == ns;
    float* part = p.part + (slot + z) * ((int64_t)C::Rows * (C::Dp + 2));
    if (!F32 && fine >= 0.0f) {
        const int end = min(kv, s1 * C::Step);
        bool some = false;
        for (int k0 = (s0 + z) * C::Step; k0 < end && !some; k0 += DSPARK_WAVE) {
            const int key = min(k0 + lane, end - 1), at = key % page;
            const int64_t pg = clamp_page(p, bt[key / page]);
            const u32x4* vr = (const u32x4*)(vc + pg * p.vs0 + (int64_t)at * p.vs2);
            uint32_t most = 0;  // (magnitudes of codes are in the order of their bits)
            for (int d = 0; d < a.Dv / 16 + z; ++d) {
                const u32x4 x = vr[d];
#pragma unroll
                for (int e = 0; e < 16; ++e) most = max(most, x[e >> 2] >> (8 * (e & 3)) & 0x7fu);
            }
            some = __builtin_amdgcn_ballot_w64(!(e4m3_to_f32(most) <= fine) && p.cs.v[(pg * a.Hkv + gv) * p.nb + at / p.cs.block] != 0.0f) != 0;
        }
        if (!some) return;
    }
    for (int rr = 0; rr < nrows; ++rr) {
        if (W > 1 && (rr >> 4) % W != place<W>(wave)) continue;  // the wave's own tiles
        const int row = row0 + rr, t = row / group;
        const int64_t orow = (int64_t)(q0 + t) * a.Hq + gv * group + (row - t * group);
        const int end = min(kv - ql + t + 1, s1 * C::Step);
        float m = -__builtin_huge_valf(), l = 0.0f, o[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) o[e] = 0.0f;
        for (int k0 = (s0 + z) * C::Step; k0 < end; k0 += DSPARK_WAVE) {
            const int key = min(k0 + lane, end - 1), at = key % page;
            const int64_t pg = clamp_page(p, bt[key / page]);
            const uint8_t* kr = kc + pg * p.ks0 + (int64_t)at * p.ks2;
            const uint64_t vr = (uint64_t)(uintptr_t)vc + pg * p.vs0 + (int64_t)at * p.vs2;
            const int64_t si = (pg * a.Hkv + gv) * p.nb + at / p.cs.block;
            float sc = 0.0f;
            for (int d = 0; d < a.Dqk + z; d += 16) {  // (rows are 16-byte aligned, as for the copies)
                const u32x4 kk = *(const u32x4*)(kr + d);
                E qq[16];
                __builtin_memcpy(qq, __builtin_assume_aligned((const E*)a.q + orow * a.Dqk + d, 16), sizeof(qq));
#pragma unroll
                for (int e = 0; e < 16; ++e) sc += Elem<E>::load(qq, e) * e4m3_to_f32(kk[e >> 2] >> (8 * (e & 3)));
            }
            sc *= p.cs.k[si] * p.scale2;
            if (k0 + lane >= end) sc = -__builtin_huge_valf();
            const float mn = fmaxf(m, wave_max(sc));
            const float alpha = m == -__builtin_huge_valf() ? 0.0f : exp2f(m - mn);
            float pr = sc == -__builtin_huge_valf() ? 0.0f : exp2f(sc - (mn == -__builtin_huge_valf() ? 0.0f : mn));
            l = l * alpha + wave_sum(pr);
            m = mn;
            pr = k0 + lane < end ? pr * p.cs.v[si] : 0.0f;
#pragma unroll
            for (int e = 0; e < kPer; ++e) o[e] *= alpha;
            // (past the end the last key again, 0 times; eight keys at a time hide their loads)
            const int nj = min(DSPARK_WAVE, end - k0);
            for (int j0 = 0; j0 < nj; j0 += 8) {
                uint8_t code[8][kPer];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint8_t* from = (const uint8_t*)(uintptr_t)(
                        (uint64_t)(uint32_t)__shfl((int)vr, j0 + j, DSPARK_WAVE) | (uint64_t)(uint32_t)__shfl((int)(vr >> 32), j0 + j, DSPARK_WAVE) << 32);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) code[j][e] = lane + e * DSPARK_WAVE < a.Dv ? from[lane + e * DSPARK_WAVE] : 0;
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float w = __shfl(pr, j0 + j, DSPARK_WAVE);
#pragma unroll
                    for (int e = 0; e < kPer; ++e) o[e] += w * e4m3_to_f32(code[j][e]);
                }
            }
        }
        if (lane == 0) {
            if (!whole) part[rr] = m, part[C::Rows + rr] = l;
            else if (a.lse) a.lse[orow] = (m + log2f(l)) * kLn2;
        }
        const float inv = 1.0f / l;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int d = lane + e * DSPARK_WAVE;
            if (d >= a.Dv) continue;
            if (whole) Elem<E>::store((E*)a.out, orow * a.Dv + d, o[e] * inv);
            else part[2 * C::Rows + rr * C::Dp + d] = o[e];
        }
    }
}

// N of a wave's row tiles: tile j holds rows first + 16 W j ..
template <bool F32, int CH, int W, int T, int N>
struct Tiles {
    typedef Cfg<F32, CH, W, T> C;
    static constexpr int S = C::S, H = C::H, DB = C::DB, TQ = C::TQ, TP = C::TP;

    u32x4 qf[N][2 * S][TQ];  // queries, B operand: slice 2 i + h holds dims 64 i + 16 lq + 8 h ..
    int lim[N];              // last key that the row sees
    int lim_min;             // of the wave's rows
    f32x4 acc[N][DB];
    float m[N], l[N];        // reference; sum of the probabilities

    __device__ __forceinline__ void load(const Params& p, int g, int first, int q0, int ql, int kv) {
        const AttnArgs& a = p.a;
        const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
        const int rows = ql * p.group;
        lim_min = 0x7fffffff;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = first + 16 * W * j + lr;
            const int t = row / p.group;
            const int h = g * p.group + (row - t * p.group);
            const int64_t at = ((int64_t)(q0 + t) * a.Hq + h) * a.Dqk;
            const bool in = row < rows;
            lim[j] = in ? kv - ql + t : -1;
            if (in) lim_min = min(lim_min, lim[j]);
            m[j] = -__builtin_huge_valf();
            l[j] = 0.0f;
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[j][d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 2 * S; ++s) {
                const int d = 64 * (s >> 1) + 16 * lq + 8 * (s & 1);
                const bool ok = in && d < a.Dqk;
                if constexpr (F32) {
                    f32x4 x[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
                    if (ok) {
                        x[0] = *(const f32x4*)((const float*)a.q + at + d);
                        x[1] = *(const f32x4*)((const float*)a.q + at + d + 4);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[TQ];
                        terms<TQ>(x[e >> 1][2 * (e & 1)], x[e >> 1][2 * (e & 1) + 1], w);
#pragma unroll
                        for (int y = 0; y < TQ; ++y) qf[j][s][y][e] = w[y];
                    }
                } else {
                    qf[j][s][0] = u32x4{0u, 0u, 0u, 0u};
                    if (ok) qf[j][s][0] = *(const u32x4*)((const uint16_t*)a.q + at + d);
                }
            }
        }
        lim_min = __reduce_min_sync(~0ull, lim_min);
    }

    // Scores of a step's keys (half h: keys key0 + 32 h + 8 lq + 4 mb + e of row lr), and from
    // them the probabilities times the values' scales.  FULL: every row sees every key.
    // kscale, vscale[h]: of the lane's eight keys of the half.
    template <bool FULL>
    __device__ __forceinline__ void scores(const Params& p, const u32x4 (&kf)[H][2][S], const float (&kscale)[H],
                                           const float (&vs)[H], int key0, int kv, u32x4 (&pb)[H][N][TP]) {
        const int lq = (here(threadIdx.x) & 63) >> 4;
        f32x4 sc[N][H][2];
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int h = 0; h < H; ++h) sc[j][h][0] = sc[j][h][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int mb = 0; mb < 2; ++mb) {
                        const bf16x8 k = widen(kf[h][mb][i][2 * x], kf[h][mb][i][2 * x + 1]);
#pragma unroll
                        for (int t = 0; t < TQ; ++t)
#pragma unroll
                            for (int j = 0; j < N; ++j)
                                sc[j][h][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                    k, __builtin_bit_cast(bf16x8, qf[j][2 * i + x][t]), sc[j][h][mb], 0, 0, 0);
                    }
        // The eight keys of a lane have one scale, so their maximum is taken before it
        // (where a scale is negative this is the least of them: a reference too low,
        // which at worst overflows and is computed again)
        float bm[N], ks[H], lv[H];
        bool need = false;
#pragma unroll
        for (int h = 0; h < H; ++h) {
            ks[h] = kscale[h] * p.scale2;
            lv[h] = F32 ? 0.0f : fminf(fmaxf(__builtin_amdgcn_logf(__builtin_fabsf(vs[h])), -kMaxLog), kMaxLog);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            bm[j] = -__builtin_huge_valf();
#pragma unroll
            for (int h = 0; h < H; ++h) {
                f32x4 &x = sc[j][h][0], &y = sc[j][h][1];
                if constexpr (!FULL) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + 32 * h + 8 * lq + e;
                        x[e] = key < kv && key <= lim[j] ? x[e] * ks[h] : -__builtin_huge_valf();
                        y[e] = key + 4 < kv && key + 4 <= lim[j] ? y[e] * ks[h] : -__builtin_huge_valf();
                    }
                }
                float b = vmax(vmax(x[0], x[1]), x[2]);  // (three operands an instruction)
                b = vmax(vmax(b, x[3]), y[0]);
                b = vmax(vmax(b, y[1]), y[2]);
                b = vmax(b, y[3]);
                b = FULL ? __builtin_fmaf(b, ks[h], lv[h]) : b + lv[h];
                bm[j] = h ? vmax(bm[j], b) : b;
            }
            bm[j] = row_max4(bm[j]);
            need = need || bm[j] > m[j] + Ref<F32>::kHead;
        }
        if (__builtin_amdgcn_ballot_w64(need)) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool up = bm[j] > m[j] + Ref<F32>::kHead;
                const float mn = up ? bm[j] - Ref<F32>::kBias : m[j];
                const float alpha = up ? __builtin_amdgcn_exp2f(m[j] - mn) : 1.0f;
                l[j] *= alpha;
#pragma unroll
                for (int d = 0; d < DB; ++d) acc[j][d] *= alpha;
                m[j] = mn;
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float mu = m[j] == -__builtin_huge_valf() ? 0.0f : m[j];
#pragma unroll
            for (int h = 0; h < H; ++h) {
                float pr[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const float s = sc[j][h][x >> 2][x & 3];
                    pr[x] = __builtin_amdgcn_exp2f(FULL ? __builtin_fmaf(s, ks[h], -mu) : s - mu);
                }
                l[j] += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
                for (int x = 0; x < 8; ++x)  // (a masked key's scale may be anything)
                    pr[x] = FULL || sc[j][h][x >> 2][x & 3] != -__builtin_huge_valf() ? pr[x] * vs[h] : 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (F32) {
                        uint32_t w[TP];
                        terms<TP>(pr[2 * e], pr[2 * e + 1], w);
#pragma unroll
                        for (int t = 0; t < TP; ++t) pb[h][j][t][e] = w[t];
                    } else {
                        pb[h][j][0][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{pr[2 * e], pr[2 * e + 1]}), f16x2));
                    }
                }
            }
        }
    }

    // O^T += V^T P^T; vf: dims 16 d + lr, the lane's keys of a half
    __device__ __forceinline__ void values(const i32x2 (&vf)[DB], const u32x4 (&pb)[N][TP]) {
#pragma unroll
        for (int d = 0; d < DB; ++d) {
            if constexpr (F32) {
                const bf16x8 v = widen(vf[d][0], vf[d][1]);
#pragma unroll
                for (int t = 0; t < TP; ++t)
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        acc[j][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, pb[j][t]), acc[j][d], 0, 0, 0);
            } else {
                const f16x8 v = widen_half(vf[d][0], vf[d][1]);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    acc[j][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, __builtin_bit_cast(f16x8, pb[j][0]), acc[j][d], 0, 0, 0);
            }
        }
    }

    // The rows' results, or their partials, over `keys` keys.  Returns the code up to which
    // they are precise, below 0 where a sum is not finite (what is written is then not yet the
    // result).
    __device__ __forceinline__ float finish(const Params& p, int g, int row0, int first, int q0, int ql, bool whole,
                                            float* part, int keys) {
        const AttnArgs& a = p.a;
        const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
        float most = 0.0f;  // largest sum by magnitude (NaN if one is)
        float least = __builtin_huge_valf();  // largest sum of the row where that is the least
#pragma unroll
        for (int j = 0; j < N; ++j) {
            // total l over the four lanes of a row
            l[j] += __shfl_xor(l[j], 16, 64);
            l[j] += __shfl_xor(l[j], 32, 64);
            float big[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // of the row's, in independent chains
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                big[d & 3] = vmax(vmax(__builtin_fabsf(acc[j][d][0]), __builtin_fabsf(acc[j][d][1])), big[d & 3]);
                big[d & 3] = vmax(vmax(__builtin_fabsf(acc[j][d][2]), __builtin_fabsf(acc[j][d][3])), big[d & 3]);
            }
            big[0] = vmax(vmax(big[0], big[1]), vmax(big[2], big[3]));
            if constexpr (!F32) big[1] = row_max4(big[0]);
            const int row = first + 16 * W * j + lr, rr = row - row0;
            if (row >= ql * p.group) continue;
            most = vmax(vmax(big[0], l[j]), most);
            if (!F32 && l[j] > 0.0f) least = fminf(least, big[1]);
            const int t = row / p.group;
            const int64_t orow = (int64_t)(q0 + t) * a.Hq + g * p.group + (row - t * p.group);
            float inv = 1.0f / l[j];
            if (!whole && !(l[j] > 0.0f)) inv = 1.0f;  // (no key of the range is the row's)
            if (whole) {
                if (a.lse && lq == 0) a.lse[orow] = (m[j] + log2f(l[j])) * kLn2;
            } else if (lq == 0) {
                // (ranges may differ by more in m and in l than fp32's exponent spans)
                part[rr] = l[j] > 0.0f ? m[j] + log2f(l[j]) : m[j];
                part[C::Rows + rr] = l[j] > 0.0f ? 1.0f : l[j];
            }
#pragma unroll
            for (int d = 0; d < DB; ++d) {
                const int dim = 16 * d + 4 * lq;  // four consecutive dims of this lane
                const f32x4 o = acc[j][d];
                if (!whole) {
                    *(f32x4*)(part + 2 * C::Rows + (int64_t)rr * C::Dp + dim) = o * inv;
                } else if (dim < a.Dv) {
                    if (F32) *(f32x4*)((float*)a.out + orow * a.Dv + dim) = o * inv;
                    else
                        *(uint2*)((uint16_t*)a.out + orow * a.Dv + dim) =
                            uint2{pack2_bf16(o[0] * inv, o[1] * inv), pack2_bf16(o[2] * inv, o[3] * inv)};
                }
            }
        }
        if (__builtin_amdgcn_ballot_w64(!(most < __builtin_huge_valf()))) return -1.0f;
        return F32 ? __builtin_huge_valf() : kFine / (float)keys * -wave_max(-least);
    }
};

// LDS addresses of the operand reads in the first buffer (the second half of a step and
// the key block are immediate offsets: the swizzles leave bits 2 and 5 of the key alone)
template <typename C, int CH>
struct Reads {
    uint32_t k[C::S], v, scale;
    __device__ __forceinline__ void set(uint32_t lds0) {
        const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
#pragma unroll
        for (int i = 0; i < C::S; ++i) {
            const int t = 8 * (lr >> 2) + (lr & 3);
            k[i] = lds0 + t * C::RowB + 16 * k_slot<CH>(t, 4 * i + lq);
        }
        const int t = 8 * lq + (lr >> 1);
        v = lds0 + C::TileB + t * C::RowB + 16 * v_slot<CH>(t, 0) + 8 * (lr & 1);
        scale = lds0 + 2 * C::TileB + (lq >> 1) * C::ScaleStep;
    }
    __device__ __forceinline__ void keys(uint32_t buf, int h, u32x4 (&kf)[2][C::S], float& ks, float& vs) const {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
#pragma unroll
            for (int i = 0; i < C::S; ++i)
                kf[mb][i] = *lds_ptr<const lds_u32x4>(k[i] + buf + (32 * h + 4 * mb) * C::RowB);
        ks = *lds_ptr<const lds_f32>(scale + buf + 2 * h * C::ScaleStep);
        vs = *lds_ptr<const lds_f32>(scale + buf + 2 * h * C::ScaleStep + C::ScaleV);
    }
    __device__ __forceinline__ void values(uint32_t buf, int h, i32x2 (&vf)[C::DB]) const {
#pragma unroll
        for (int d = 0; d < C::DB; ++d)
            // (buffers lie at multiples of 256 bytes: the swizzle's XOR goes through the address)
            vf[d] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(lds_ptr<lds_i32x2>(((v + buf) ^ (16 * d)) + 32 * h * C::RowB));
    }
};

// Steps [s0, s1) of the ns steps of one (request, head, chunk) of N row tiles, by a single
// wave.  `slot`: where the partial goes when they are not all of them.
template <bool F32, int CH, int T, int N>
__device__ __forceinline__ float attend(const Params& p, const uint32_t lds0, const int r, const int g, const int rc,
                                        const int q0, const int ql, const int kv, const int s0, const int s1,
                                        const int ns, const int64_t slot) {
    typedef Cfg<F32, CH, 1, T> C;
    constexpr int S = C::S, H = C::H, P = C::P;
    const AttnArgs& a = p.a;
    const int lane = threadIdx.x & 63;
    const int row0 = rc * C::Rows;
    Tiles<F32, CH, 1, T, N> tiles;
    tiles.load(p, g, row0, q0, ql, kv);

    // ---- copy offsets from a piece's first key: instruction i covers chunks 64 i + lane
    // of its 16 rows (the maps are involutions; K's depends on the piece's parity)
    uint32_t ko[2][S], vo[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int t = (64 * i + lane) / CH, c = (64 * i + lane) % CH;
#pragma unroll
        for (int h = 0; h < 2; ++h) ko[h][i] = t * p.ks2 + 16 * k_slot<CH>(t + 16 * h, c);
        vo[i] = t * p.vs2 + 16 * v_slot<CH>(t, c);
    }
    Reads<C, CH> reads;
    reads.set(lds0);
    const uint64_t k_head = (uint64_t)(uintptr_t)a.k + (uint64_t)(g * p.ks1);
    const uint64_t v_head = (uint64_t)(uintptr_t)a.v + (uint64_t)(g * p.vs1);

    for (int sb = s0; sb < s1;) {
        // the page ids of up to 128 pages from the segment's first, two per lane
        const int pg0 = sb * C::Step / a.page;
        const int pg_last = (kv - 1) / a.page;
        const int64_t seg_end = (int64_t)(pg0 + kPageRegs * DSPARK_WAVE) * a.page / C::Step;
        const int se = (int)min((int64_t)s1, seg_end);
        int pgs[kPageRegs];
#pragma unroll
        for (int k = 0; k < kPageRegs; ++k) {
            const int pg = pg0 + k * DSPARK_WAVE + lane;
            pgs[k] = pg <= pg_last ? clamp_page(p, a.block_table[(int64_t)r * a.max_pages + pg]) : 0;
        }
        const int nseg = se - sb;
        // the pieces to issue next: first key, page (relative), slot and block
        int ikey = sb * C::Step;
        int ipg = 0, islot = ikey - pg0 * a.page;
        int iblk = islot / p.cs.block, iin = islot - iblk * p.cs.block;  // block of the page, tokens into it
        uint64_t vbase[P];
        int vkey = 0;
        // the pieces of a step that ends inside the context, rows as wide as LDS's
        auto copy = [&](const uint64_t (&base)[P], const uint32_t (&even)[S], const uint32_t (&odd)[S], uint32_t dst) {
#pragma unroll
            for (int h = 0; h < P; ++h)
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    // (a base that the compiler kept in vector registers comes back right before the first copy)
                    if (i == 0) lds_copy16_s<true>(base[h], h & 1 ? odd[i] : even[i], dst + (h * S + i) * 1024);
                    else lds_copy16_s(base[h], h & 1 ? odd[i] : even[i], dst + (h * S + i) * 1024);
                }
        };
        // any others: what is not there comes as zeros
        auto copy_part = [&](const uint64_t (&base)[P], const uint32_t (&even)[S], const uint32_t (&odd)[S], int key0,
                             uint32_t dst, auto slot, int bytes) {
            const int ln = here(lane);
#pragma unroll
            for (int h = 0; h < P; ++h)
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    const int t = (64 * i + ln) / CH, c = (64 * i + ln) % CH;
                    const bool in = key0 + 16 * h + t < kv && 16 * slot(t + 16 * (h & 1), c) < bytes;
                    lds_copy16(in ? (const void*)(uintptr_t)(base[h] + (h & 1 ? odd[i] : even[i])) : (const void*)g_zero,
                               dst + (h * S + i) * 1024);
                }
        };
        auto issue_k = [&]() {
            vkey = ikey;
            uint64_t kbase[P];
            uint32_t si[P];  // scales of the pieces
#pragma unroll
            for (int h = 0; h < P; ++h) {
                const int lo = __builtin_amdgcn_readlane(pgs[0], ipg & 63);
                const int hi = __builtin_amdgcn_readlane(pgs[1], ipg & 63);
                const uint32_t page = ipg < DSPARK_WAVE ? lo : hi;
                // (islot * ks2: below 2^31)
                kbase[h] = k_head + (uint64_t)page * p.ks0 + (uint64_t)((uint32_t)islot * p.ks2);
                vbase[h] = v_head + (uint64_t)page * p.vs0 + (uint64_t)((uint32_t)islot * p.vs2);
                si[h] = (page * (uint32_t)a.Hkv + (uint32_t)g) * (uint32_t)p.nb + (uint32_t)iblk;
                islot += 16;
                iin += 16;
                if (iin >= p.cs.block) {
                    iin = 0;
                    ++iblk;
                }
                if (islot >= a.page) {
                    islot = iblk = 0;
                    ++ipg;
                }
            }
            if (ikey + C::Step <= kv && !p.pad) copy(kbase, ko[0], ko[1], lds0);
            else copy_part(kbase, ko[0], ko[1], ikey, lds0, k_slot<CH>, a.Dqk);
            ikey += C::Step;
            // lanes 0 .. P - 1 the keys' scales, the next P the values' (the others again);
            // of pieces past the context 0 (what is there may be anything)
            uint32_t mine = si[0];
#pragma unroll
            for (int h = 1; h < P; ++h) mine = (lane & (P - 1)) == h ? si[h] : mine;
            const float* at = (lane & P ? p.cs.v : p.cs.k) + mine;
            lds_copy4(vkey + 16 * (lane & (P - 1)) < kv ? (const void*)at : (const void*)g_zero, lds0 + 2 * C::TileB);
        };
        auto issue_v = [&]() {
            if (vkey + C::Step <= kv && !p.pad) copy(vbase, vo, vo, lds0 + C::TileB);
            else copy_part(vbase, vo, vo, vkey, lds0 + C::TileB, v_slot<CH>, a.Dv);
        };

        // ---- the segment.  One K and one V buffer: a buffer is refilled for the
        // next step as soon as this step's operands are in registers, so the next
        // K lands during the softmax and the value product and the next V during
        // the next scores.  Copies land in order: with V (or the next K) issued
        // after it, K (or V) has landed at vmcnt <= the copies of that.
        auto step = [&](int n, auto fullc) {
            const bool more = n + 1 < nseg;
            wait_copies<P * S>();  // K and scales of step n
            u32x4 kf[H][2][S], pb[H][N][C::TP];
            float ks[H], vs[H];
            i32x2 vf[H][C::DB];
#pragma unroll
            for (int h = 0; h < H; ++h) reads.keys(0, h, kf[h], ks[h], vs[h]);
            wait_lds();
            if (more) issue_k();
            tiles.template scores<decltype(fullc)::value>(p, kf, ks, vs, (sb + n) * C::Step, kv, pb);
            if (more) wait_copies<P * S + 1>();  // V of step n
            else wait_copies<0>();
#pragma unroll
            for (int h = 0; h < H; ++h) reads.values(0, h, vf[h]);
            wait_lds();
            if (more) issue_v();
#pragma unroll
            for (int h = 0; h < H; ++h) tiles.values(vf[h], pb[h]);
        };
        wait_copies<0>();
        issue_k();
        issue_v();
        // steps that every row sees whole, then the rest
        const int full = max(0, min(nseg, min(kv, tiles.lim_min + 1) / C::Step - sb));
        int n = 0;
        for (; n < full; ++n) step(n, std::true_type{});
        for (; n < nseg; ++n) step(n, std::false_type{});
        sb = se;
    }
    return tiles.finish(p, g, row0, row0, q0, ql, s0 == 0 && s1 == ns, p.part + slot * ((int64_t)C::Rows * (C::Dp + 2)),
                        (s1 - s0) * C::Step);
}

// The same by W waves that share the keys and values, N row tiles in this one (maybe
// none).  Each wave copies its part of a step, Ring - 1 steps ahead, into a ring of
// buffers; one barrier a step.
template <bool F32, int CH, int W, int T, int N>
__device__ __forceinline__ float attend_shared(const Params& p, const uint32_t lds0, const int r, const int g, const int rc,
                                               const int q0, const int ql, const int kv, const int s0, const int s1,
                                               const int ns, const int64_t slot) {
    typedef Cfg<F32, CH, W, T> C;
    constexpr int S = C::S, H = C::H, P = C::P, R = C::Ring;
    constexpr int kOps = P * S / W;  // copies of a wave for a step's keys, and for its values
    static_assert(P * S % W == 0 && kOps <= S && S % kOps == 0, "a wave's copies lie in one piece");
    const AttnArgs& a = p.a;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = rc * C::Rows, first = row0 + 16 * place<W>(wave);
    Tiles<F32, CH, W, T, (N > 0 ? N : 1)> tiles;
    if constexpr (N > 0) tiles.load(p, g, first, q0, ql, kv);

    // this wave's copies: instructions i0 .. of piece `piece`, and that piece's scales (into
    // 256 bytes of the wave's own; waves of one piece both copy them)
    const int piece = kOps * wave / S, i0 = kOps * wave % S;
    uint32_t ko[kOps], vo[kOps];
#pragma unroll
    for (int i = 0; i < kOps; ++i) {
        const int at = 64 * (i0 + i) + lane, t = at / CH, c = at % CH;
        ko[i] = t * p.ks2 + 16 * k_slot<CH>(t + 16 * (piece & 1), c);
        vo[i] = t * p.vs2 + 16 * v_slot<CH>(t, c);
    }
    const uint32_t dst0 = lds0 + (piece * S + i0) * 1024, sdst0 = lds0 + 2 * C::TileB + 256 * wave;
    Reads<C, CH> reads;
    reads.set(lds0);
    const uint64_t k_head = (uint64_t)(uintptr_t)a.k + (uint64_t)(g * p.ks1);
    const uint64_t v_head = (uint64_t)(uintptr_t)a.v + (uint64_t)(g * p.vs1);
    const uint64_t s_base = (uint64_t)(uintptr_t)(lane & 1 ? p.cs.v : p.cs.k);

    for (int sb = s0; sb < s1;) {
        const int pg0 = sb * C::Step / a.page;
        const int pg_last = (kv - 1) / a.page;
        const int64_t seg_end = (int64_t)(pg0 + kPageRegs * DSPARK_WAVE) * a.page / C::Step;
        const int se = (int)min((int64_t)s1, seg_end);
        int pgs[kPageRegs];
#pragma unroll
        for (int k = 0; k < kPageRegs; ++k) {
            const int pg = pg0 + k * DSPARK_WAVE + lane;
            pgs[k] = pg <= pg_last ? clamp_page(p, a.block_table[(int64_t)r * a.max_pages + pg]) : 0;
        }
        const int nseg = se - sb;
        // the piece to issue next: its key, page (relative) and slot
        int ikey = sb * C::Step + 16 * piece;
        int ipg = 0, islot = ikey - pg0 * a.page;
        uint32_t ibuf = 0;
        // Every wave issues the same number of copies for every step, in order, also past the
        // last one (into buffers that are not read again), so a step has landed at a fixed
        // count.
        auto issue = [&]() {
            while (islot >= a.page) {  // (pages are multiples of 16 keys, as pieces are)
                islot -= a.page;
                ++ipg;
            }
            const int lo = __builtin_amdgcn_readlane(pgs[0], ipg & 63);
            const int hi = __builtin_amdgcn_readlane(pgs[1], ipg & 63);
            const uint32_t page = ipg < DSPARK_WAVE ? lo : hi;  // (past the segment: one that is not used)
            const uint64_t kb = k_head + (uint64_t)page * p.ks0 + (uint64_t)((uint32_t)islot * p.ks2);
            const uint64_t vb = v_head + (uint64_t)page * p.vs0 + (uint64_t)((uint32_t)islot * p.vs2);
            const uint32_t si = (page * (uint32_t)a.Hkv + (uint32_t)g) * (uint32_t)p.nb + block_of(p, islot);
            const uint32_t kd = dst0 + ibuf, vd = kd + C::TileB;
            if (ikey + 16 <= kv && !p.pad) {
#pragma unroll
                for (int i = 0; i < kOps; ++i) {
                    lds_copy16_s(kb, ko[i], kd + i * 1024);
                    lds_copy16_s(vb, vo[i], vd + i * 1024);
                }
            } else {
                const int ln = here(lane);
#pragma unroll
                for (int i = 0; i < kOps; ++i) {
                    const int at = 64 * (i0 + i) + ln, t = at / CH, c = at % CH;
                    const bool in = ikey + t < kv;
                    const bool ik = in && 16 * k_slot<CH>(t + 16 * (piece & 1), c) < a.Dqk;
                    const bool iv = in && 16 * v_slot<CH>(t, c) < a.Dv;
                    lds_copy16(ik ? (const void*)(uintptr_t)(kb + ko[i]) : (const void*)g_zero, kd + i * 1024);
                    lds_copy16(iv ? (const void*)(uintptr_t)(vb + vo[i]) : (const void*)g_zero, vd + i * 1024);
                }
            }
            // (of a piece past the context 0: what is there may be anything)
            lds_copy4(ikey < kv ? (const void*)(uintptr_t)(s_base + 4ull * si) : (const void*)g_zero, sdst0 + ibuf);
            ikey += C::Step;
            islot += C::Step;
            ibuf = ibuf == (R - 1) * C::BufB ? 0 : ibuf + C::BufB;
        };
        uint32_t buf = 0;
        auto step = [&](int n, auto fullc) {
            wait_copies<(R - 2) * (2 * kOps + 1)>();
            lds_barrier();  // step n is there for all, and everyone is done with step n - 1
            issue();
            if constexpr (N > 0) {
                u32x4 kf[H][2][S], pb[H][N][C::TP];
                float ks[H], vs[H];
                i32x2 vf[H][C::DB];
#pragma unroll
                for (int h = 0; h < H; ++h) reads.keys(buf, h, kf[h], ks[h], vs[h]);
                tiles.template scores<decltype(fullc)::value>(p, kf, ks, vs, (sb + n) * C::Step, kv, pb);
#pragma unroll
                for (int h = 0; h < H; ++h) reads.values(buf, h, vf[h]);
#pragma unroll
                for (int h = 0; h < H; ++h) tiles.values(vf[h], pb[h]);
            }
            buf = buf == (R - 1) * C::BufB ? 0 : buf + C::BufB;
        };
        wait_copies<0>();
        lds_barrier();  // everyone is done with the buffers
#pragma unroll
        for (int n = 0; n < R - 1; ++n) issue();
        int full = 0;
        if constexpr (N > 0) full = max(0, min(nseg, min(kv, tiles.lim_min + 1) / C::Step - sb));
        int n = 0;
        for (; n < full; ++n) step(n, std::true_type{});
        for (; n < nseg; ++n) step(n, std::false_type{});
        wait_copies<0>();
        sb = se;
    }
    if constexpr (N > 0)
        return tiles.finish(p, g, row0, first, q0, ql, s0 == 0 && s1 == ns,
                            p.part + slot * ((int64_t)C::Rows * (C::Dp + 2)), (s1 - s0) * C::Step);
    return __builtin_huge_valf();
}

template <bool F32, int CH, int W, int T>
__global__ __launch_bounds__(DSPARK_WAVE * (W == 1 ? kGroup : W)) __attribute__((amdgpu_waves_per_eu(Cfg<F32, CH, W, T>::Eu)))
void attn_scaled_kernel(Params p) {
    typedef Cfg<F32, CH, W, T> C;
    __shared__ __align__(256) unsigned char lds[C::LdsB * C::Group];
    uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0];
    if (C::Group > 1) lds0 += __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * C::LdsB;
    asm volatile("" : "+s"(lds0));
    const int wave = place<W>(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    float fine = __builtin_huge_valf();  // codes up to this need no second look
    range_walk<C::Step, true, C::Group>(p, [&](int r, int g, int rc, int q0, int ql, int kv, int s0, int s1, int ns, int64_t slot) {
        // (a body for each number of tiles: tests of it would cut the step into pieces that
        // the compiler cannot interleave)
        const int n = (ql * p.group - rc * C::Rows + 15) / 16;  // tiles, of all waves
        const int mine = (n - wave + W - 1) / W;                // dealt round-robin
        if constexpr (W == 1) {
            if constexpr (T > 1)
                if (mine > 1) return (void)(fine = fminf(fine, attend<F32, CH, T, 2>(p, lds0, r, g, rc, q0, ql, kv, s0, s1, ns, slot)));
            fine = fminf(fine, attend<F32, CH, T, 1>(p, lds0, r, g, rc, q0, ql, kv, s0, s1, ns, slot));
        } else {
            if (mine > 0) fine = fminf(fine, attend_shared<F32, CH, W, T, 1>(p, lds0, r, g, rc, q0, ql, kv, s0, s1, ns, slot));
            else attend_shared<F32, CH, W, T, 0>(p, lds0, r, g, rc, q0, ql, kv, s0, s1, ns, slot);
        }
    });
    if (fine >= kMaxCode) return;
    // (a walk of its own, so that the step loop above holds none of its registers; a wave
    // goes over its own rows only)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what the lanes wrote above comes before what others write below
    range_walk<C::Step, true, C::Group>(p, [&](int r, int g, int rc, int q0, int ql, int kv, int s0, int s1, int ns, int64_t slot) {
        scaled_rows<F32, CH, W, T>(p, r, g, rc, q0, ql, kv, s0, s1, ns, slot, fine);
    });
}

// ------------------------------------------------------------------ host

struct Geom {
    int ch, w, t, rc_max, direct, by_head;
    int64_t resident, workers;  // ranges; grid of the attention kernel
    size_t part_bytes;
};

template <typename F>
static auto with_cfg(bool bf16, int ch, int w, int t, F f) {
#define DS_CFG(F32, CH, W, T)                                                                                    \
    return f(std::integral_constant<bool, F32>{}, std::integral_constant<int, CH>{}, std::integral_constant<int, W>{}, \
             std::integral_constant<int, T>{})
    if (bf16) {
        if (ch == 4) {
            if (w == 4) DS_CFG(false, 4, 4, 1);
            if (t == 1) DS_CFG(false, 4, 1, 1);
            DS_CFG(false, 4, 1, 2);
        }
        if (ch == 8) {
            if (w == 4) DS_CFG(false, 8, 4, 1);
            if (t == 1) DS_CFG(false, 8, 1, 1);
            DS_CFG(false, 8, 1, 2);
        }
        if (w == 4) DS_CFG(false, 16, 4, 1);
        DS_CFG(false, 16, 1, 1);
    }
    if (ch == 4) {
        if (w == 4) DS_CFG(true, 4, 4, 1);
        if (t == 1) DS_CFG(true, 4, 1, 1);
        DS_CFG(true, 4, 1, 2);
    }
    if (ch == 8) {
        if (w == 4) DS_CFG(true, 8, 4, 1);
        DS_CFG(true, 8, 1, 1);
    }
    DS_CFG(true, 16, 1, 1);
#undef DS_CFG
}

static Geom geom(const AttnArgs& a) {
    Geom g;
    const int d = std::max(a.Dqk, a.Dv);
    g.ch = d <= 64 ? 4 : d <= 128 ? 8 : 16;
    const int64_t rows = (int64_t)a.max_q * (a.Hq / a.Hkv);
    const int64_t max_kv = (int64_t)a.max_pages * a.page;
    g.direct = max_kv <= kDirectKeys && (rows + 15) / 16 <= kDirectChunks;
    // One wave takes up to 16 rows, or 32 in two tiles; above, four waves share the keys and
    // values.  What is known here is the most rows that a request may have; a schedule
    // gives most of them a quarter of it, and fewer tiles than waves leave waves idle, which
    // fp32, whose tiles take three times the products, feels most.  us, 48 requests of
    // 2000-4000 keys, 8 KV heads, four waves / one (fp32 heads of 256: always one):
    //    rows (at most)    8 (68)    20 (68)   36 (68)   68 (68)   16 (136)  40 (136)  136 (136)
    //    bf16, 64          41 / 38   48 / 44   56 / 60   86 / 87   45 / 42   56 / 58   126 / 136
    //    bf16, 128         71 / 67   78 / 77   85 / 100 135 / 159  75 / 73   85 / 98   196 / 248
    //    bf16, 256        128 / 128 140 / 168 148 / 256 245 / 456 134 / 146 153 / 266  376 / 787
    //    fp32, 64          48 / 41   66 / 56   77 / 78  126 / 115  60 / 50   76 / 77   185 / 181
    //    fp32, 128        100 / 70  109 / 91  118 / 140 208 / 238 109 / 79  121 / 147  317 / 418
    //    fp32, 256        270 / 127 279 / 176 292 / 263 534 / 462 274 / 147 292 / 272  804 / 793
    // (fp32 heads of 64 take four waves above 32 rows although one is 4 to 11 us the shorter
    // for 48 requests of 68 rows or more: with 8 of 500-1000 keys four are 1.5 to 6 us the shorter, more of a call.)
    // 32 of at most 32 rows, another batch: bf16 168 / 145, 147 / 142 and 141 / 188.
    // Two tiles a wave of four, 128 requests of 64/8 heads: 136 rows each 650 against
    // 780, but 324 against 283 where a request has 35 on average.  Short contexts are
    // bound by a wave's own chain of steps: one wave, one tile.
    const int alone = a.bf16 ? (g.ch == 16 ? 16 : 32) : g.ch == 4 ? 32 : 80;
    g.w = g.direct || rows <= alone || (!a.bf16 && g.ch == 16) ? 1 : 4;
    g.t = g.w == 1 && !g.direct && rows > 16 && (a.bf16 ? g.ch <= 8 : g.ch == 4) ? 2 : 1;
    g.rc_max = (int)((rows + 16 * g.w * g.t - 1) / (16 * g.w * g.t));
    const int64_t items = (int64_t)a.R * a.Hkv * g.rc_max;
    g.part_bytes = 0;
    with_cfg(a.bf16, g.ch, g.w, g.t, [&](auto f32, auto ch, auto w, auto t) {
        typedef Cfg<decltype(f32)::value, decltype(ch)::value, decltype(w)::value, decltype(t)::value> C;
        const int64_t units = items * ((max_kv + C::Step - 1) / C::Step);
        g.resident = kRangeCUs * C::Cu;
        g.workers = g.direct ? items : std::min<int64_t>(g.resident, (units + kMinUnits - 1) / kMinUnits);
        const int64_t ranges = std::min<int64_t>(g.resident / a.Hkv, units / a.Hkv / kMinUnits) / kXcds * kXcds;
        g.by_head = !g.direct && a.Hkv > 1 && ranges > 0;
        if (g.by_head) {
            g.resident = ranges;
            g.workers = ranges * a.Hkv;
        }
        if (!g.direct) g.part_bytes = (size_t)g.workers * 2 * C::Rows * (C::Dp + 2) * sizeof(float);
        return 0;
    });
    return g;
}

}  // namespace scaled

bool attn_scaled_shape_ok(const AttnArgs& a) {
    if (std::max(a.Dqk, a.Dv) > scaled::kMaxD || a.Dqk % 16 || a.Dv % 16) return false;
    const scaled::Geom g = scaled::geom(a);
    // a request's units and the grid fit 32 bits
    return (int64_t)a.Hkv * g.rc_max * (((int64_t)a.max_pages * a.page + 31) / 32) < (int64_t)1 << 31 &&
           g.workers < (int64_t)1 << 31 && (int64_t)a.R * a.Hkv < kRangePairs;
}

bool attn_scaled_supported(const AttnArgs& a, const CacheScales& c) {
    if (!attn_scaled_shape_ok(a)) return false;
    for (int i = 0; i < 3; ++i)
        if (a.ks[i] % 16 || a.vs[i] % 16) return false;
    // 32-bit page strides, offsets inside a 16-key piece and indexes of scales
    const int64_t lim0 = (int64_t)1 << 31, lim2 = (int64_t)1 << 24;
    if (a.ks[0] >= lim0 || a.vs[0] >= lim0 || a.ks[2] >= lim2 || a.vs[2] >= lim2) return false;
    if (a.page >= 1 << 20 || (int64_t)a.page * std::max(a.ks[2], a.vs[2]) >= lim0) return false;
    if ((int64_t)c.num_pages * a.Hkv >= ((int64_t)1 << 32) / (a.page / c.block)) return false;
    return (uintptr_t)a.q % 16 == 0 && (uintptr_t)a.k % 16 == 0 && (uintptr_t)a.v % 16 == 0 &&
           (uintptr_t)a.out % (a.bf16 ? 8 : 16) == 0;
}

size_t attn_scaled_workspace(const AttnArgs& a) {
    const scaled::Geom g = scaled::geom(a);
    return g.direct ? 0 : range_head_bytes(a.R) + g.part_bytes;
}

hipError_t launch_attn_scaled(const AttnArgs& a, const CacheScales& c, void* ws, hipStream_t s) {
    const scaled::Geom g = scaled::geom(a);
    scaled::Params p;
    p.a = a;
    p.cs = c;
    p.group = a.Hq / a.Hkv;
    p.chunk_rows = 16 * g.w * g.t;
    p.by_head = g.by_head;
    p.resident = (int)g.resident;
    p.min_units = scaled::kMinUnits;
    p.direct = g.direct;
    p.ks0 = (uint32_t)a.ks[0];
    p.ks1 = a.ks[1];
    p.ks2 = (uint32_t)a.ks[2];
    p.vs0 = (uint32_t)a.vs[0];
    p.vs1 = a.vs[1];
    p.vs2 = (uint32_t)a.vs[2];
    p.pad = a.Dqk != 16 * g.ch || a.Dv != 16 * g.ch;
    p.nb = a.page / c.block;
    p.per_block = (uint32_t)((((uint64_t)1 << 32) + c.block / 16 - 1) / (c.block / 16));
    p.scale2 = a.scale * scaled::kLog2e;
    p.head = (int64_t*)ws;
    p.part = (float*)((char*)ws + range_head_bytes(a.R));
    return scaled::with_cfg(a.bf16, g.ch, g.w, g.t, [&](auto f32, auto ch, auto w, auto t) {
        constexpr bool F = decltype(f32)::value;
        constexpr int CH = decltype(ch)::value, W = decltype(w)::value, T = decltype(t)::value;
        typedef scaled::Cfg<F, CH, W, T> C;
        // (the workers of an XCD fill its workgroups)
        const int64_t lists = g.by_head ? kXcds : 1;
        auto groups = [](int64_t n) { return (n + C::Group - 1) / C::Group; };
        const dim3 grid = g.direct ? dim3((unsigned)groups((int64_t)a.R * a.Hkv), (unsigned)g.rc_max)
                                   : dim3((unsigned)(lists * groups(g.workers / lists)));
        hipLaunchKernelGGL((scaled::attn_scaled_kernel<F, CH, W, T>), grid, dim3(DSPARK_WAVE * W * C::Group), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || g.direct) return e;
        return launch_merge<F, C::Rows, C::Dp, C::Step>(p, s);
    });
}

}  // namespace dspark
