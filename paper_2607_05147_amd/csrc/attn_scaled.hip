// Ragged causal verify attention over a paged cache of e4m3 codes with a scale for
// each block of tokens and head, on gfx950 matrix cores: head sizes up to 256, any
// page of 16-key blocks, bf16 and fp32 queries.
//
//   score(row, key) = s_k(block of key) * (q . code_k),  out = sum p * s_v(block) * code_v
//
// The codes widen to bf16 exactly (one instruction for two), so they enter bf16
// products as they are, and the scales stay outside: s_k multiplies the fp32 scores
// (a lane's eight keys lie in one block, so by one value), s_v the fp32
// probabilities.  bf16 queries enter as they are, fp32 ones as three bf16 terms
// (24 bits: exact); the probabilities as two terms (to within 2^-17, below the bf16
// output's 2^-9) or three (2^-24).
//
// Half the cache's bytes of bf16, the same products: bound by HBM, with the widening
// and the softmax on the vector ALUs next.  The work is cut as in attn_stream.hip: a
// worker is a single wave with its own K and V buffers in LDS and an equal range of
// the batch's steps (attn_ranges.h), so nothing in its loop waits for another wave;
// a wave's row tiles share one widening of the keys and values (waves that shared a
// buffer would each widen it).
//
//   * K and V rows are copied from their page straight into LDS, one step ahead:
//     64 keys a step (32 at head sizes above 128), 16 of them inside one page.  Rows
//     are 16 * CH bytes (padded head sizes are filled from a zero block), chunks
//     XOR-swizzled by the copy so that the operand reads are free of bank conflicts.
//     A step's scales are one more copy, of a value per 16 keys.
//   * S^T = K Q^T on v_mfma_f32_16x16x32_bf16: a 16-byte read has 16 dims of a key, two
//     operand slices (the queries are laid out alike).  The keys of an operand row
//     are permuted so that the scores already have the B layout of the next product.
//   * O^T += V^T P^T, V^T by transposing 8-byte reads (eight keys of a dim).
//   * softmax online in exp2 units, the running maximum moved only when it grows by
//     more than 2^8 (exact after the final normalisation);
//   * a worker that finds a sum non-finite computes its rows again key by key
//     (scaled_rows), so that a non-finite value reaches only the rows that see it.
#include <algorithm>
#include <type_traits>

#include "attn_ranges.h"

namespace dspark {
namespace scaled {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) float lds_f32;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescale = 8.0f;     // log2 headroom before the running max is moved
constexpr int kMinUnits = 4;         // steps per wave, at least
constexpr int kPageRegs = 2;         // page ids per lane: 128 pages of a range at a time
constexpr int kMaxD = 256;

// CH: 16-byte chunks of an LDS row: head sizes up to 16 * CH.  NT: 16-row tiles.
template <bool F32, int CH, int NT>
struct Cfg {
    static constexpr int H = CH <= 8 ? 2 : 1;   // 32-key halves of a step
    static constexpr int Step = 32 * H;
    static constexpr int P = 2 * H;             // 16-key pieces
    static constexpr int S = CH / 4;            // 16-byte operand reads of a key; copies of a piece
    static constexpr int RowB = 16 * CH;
    static constexpr int TileB = Step * RowB;
    static constexpr int Dp = 16 * CH;          // padded head size
    static constexpr int DB = CH;               // 16-dim output blocks
    static constexpr int TQ = F32 ? 3 : 1, TP = F32 ? 3 : 2;  // bf16 terms of a query, a probability
    static constexpr int LdsB = 2 * TileB + 256;              // K, V, scales
    static constexpr int LdsWaves = 160 * 1024 / LdsB;
    // registers: accumulators, queries, scores and probabilities of the row tiles; operands
    static constexpr int Regs = NT * (4 * DB + 8 * S * TQ + 8 * H * (TP > 2 ? TP + 1 : 2)) + 8 * H * S + 56;
    static constexpr int Eu = Regs <= 128 && LdsWaves >= 16 ? 4 : Regs <= 168 && LdsWaves >= 12 ? 3 : Regs <= 256 && LdsWaves >= 8 ? 2 : 1;
    static constexpr int Cu = LdsWaves < 4 * Eu ? LdsWaves : 4 * Eu;  // waves per CU
};

struct Params : Ranges {
    CacheScales cs;
    int64_t ks1, vs1;                // cache strides in bytes
    uint32_t ks0, vs0, ks2, vs2;
    int pad;                         // some row is shorter than the LDS row
    int nb;                          // blocks of a page
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

// eight codes as bf16
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

__device__ __forceinline__ int clamp_page(const Params& p, int page) { return min(max(page, 0), p.cs.num_pages - 1); }

// The rows of a chunk over the same steps key by key on the vector ALUs, where the
// products came out non-finite: a product over 16 rows and 32 keys also multiplies the
// keys that a row does not see, by a probability of 0, and 0 times a non-finite value
// is NaN.  Every row takes only its own keys here, as the vector-ALU kernels do.
template <bool F32, int CH, int NT>
__device__ __forceinline__ void scaled_rows(const Params& p, const int r, const int g, const int rc, const int q0,
                                            const int ql, const int kv, const int s0, const int s1, const int ns,
                                            const int64_t slot) {
    typedef Cfg<F32, CH, NT> C;
    typedef typename std::conditional<F32, float, uint16_t>::type T;
    constexpr int kPer = (C::Dp + DSPARK_WAVE - 1) / DSPARK_WAVE;  // value dims per lane
    const AttnArgs& a = p.a;
    // (values in vector registers: the scalar ones that this would add to the kernel's
    // are spilled into vector registers that the step loop then lacks)
    int z = 0;
    asm volatile("" : "+v"(z));
    const int lane = threadIdx.x, page = a.page + z, group = p.group + z, gv = g + z;
    const int row0 = (rc + z) * (16 * NT), nrows = min(16 * NT, ql * group - row0);
    const int32_t* bt = a.block_table + (int64_t)(r + z) * a.max_pages;
    const uint8_t* kc = (const uint8_t*)a.k + gv * p.ks1;
    const uint8_t* vc = (const uint8_t*)a.v + gv * p.vs1;
    const bool whole = s0 + z == 0 && s1 == ns;
    float* part = p.part + (slot + z) * ((int64_t)(16 * NT) * (C::Dp + 2));
    for (int rr = 0; rr < nrows; ++rr) {
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
            const int64_t si = (pg * a.Hkv + gv) * p.nb + at / p.cs.block;
            float sc = 0.0f;
            for (int d = 0; d < a.Dqk + z; ++d)
                sc += Elem<T>::load((const T*)a.q, orow * a.Dqk + d) * e4m3_to_f32(kr[d]);
            sc *= p.cs.k[si] * p.scale2;
            if (k0 + lane >= end) sc = -__builtin_huge_valf();
            const float mn = fmaxf(m, wave_max(sc));
            const float alpha = m == -__builtin_huge_valf() ? 0.0f : exp2f(m - mn);
            float pr = sc == -__builtin_huge_valf() ? 0.0f : exp2f(sc - (mn == -__builtin_huge_valf() ? 0.0f : mn));
            l = l * alpha + wave_sum(pr);
            m = mn;
            pr *= p.cs.v[si];
#pragma unroll
            for (int e = 0; e < kPer; ++e) o[e] *= alpha;
            for (int j = 0; j < min(DSPARK_WAVE, end - k0); ++j) {
                const int64_t pj = clamp_page(p, bt[(k0 + j) / page]);
                const uint8_t* vr = vc + pj * p.vs0 + (int64_t)((k0 + j) % page) * p.vs2;
                const float w = __shfl(pr, j, DSPARK_WAVE);
#pragma unroll
                for (int e = 0; e < kPer; ++e) {
                    const int d = lane + e * DSPARK_WAVE;
                    if (d < a.Dv) o[e] += w * e4m3_to_f32(vr[d]);
                }
            }
        }
        if (lane == 0) {
            if (!whole) part[rr] = m, part[16 * NT + rr] = l;
            else if (a.lse) a.lse[orow] = (m + log2f(l)) * kLn2;
        }
        const float inv = 1.0f / l;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int d = lane + e * DSPARK_WAVE;
            if (d >= a.Dv) continue;
            if (whole) Elem<T>::store((T*)a.out, orow * a.Dv + d, o[e] * inv);
            else part[2 * 16 * NT + rr * C::Dp + d] = o[e];
        }
    }
}

// Steps [s0, s1) of the ns steps of one (request, head, chunk).  `slot`: where
// the partial goes when they are not all of them.  Returns whether a sum of its rows is
// not finite (what is written is then not yet the result).
template <bool F32, int CH, int NT>
__device__ __forceinline__ bool attend(const Params& p, const uint32_t lds0, const int r, const int g, const int rc,
                                       const int q0, const int ql, const int kv, const int s0, const int s1,
                                       const int ns, const int64_t slot) {
    typedef Cfg<F32, CH, NT> C;
    constexpr int S = C::S, H = C::H, P = C::P, TQ = C::TQ, TP = C::TP;
    constexpr uint32_t kScales = 2 * C::TileB;  // LDS offset of the step's scales
    const AttnArgs& a = p.a;
    const int lane = threadIdx.x;
    const int lr = lane & 15, lq = lane >> 4;
    const int rows = ql * p.group;
    const int row0 = rc * (16 * NT);
    const int nt = min(NT, (rows - row0 + 15) >> 4);

    // ---- query fragments (B operand of S^T = K Q^T) and causal limits: slice 2 i + h holds
    // dims 64 i + 16 lq + 8 h ..
    u32x4 qf[NT][2 * S][TQ];
    int lim[NT];
    int lim_min = 0x7fffffff;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int row = row0 + 16 * j + lr;
        lim[j] = -1;
#pragma unroll
        for (int s = 0; s < 2 * S; ++s)
#pragma unroll
            for (int t = 0; t < TQ; ++t) qf[j][s][t] = u32x4{0u, 0u, 0u, 0u};
        if (row < rows) {
            const int t = row / p.group;
            const int h = g * p.group + (row - t * p.group);
            const int64_t at = ((int64_t)(q0 + t) * a.Hq + h) * a.Dqk;
#pragma unroll
            for (int s = 0; s < 2 * S; ++s) {
                const int d = 64 * (s >> 1) + 16 * lq + 8 * (s & 1);
                if (d >= a.Dqk) continue;
                if constexpr (F32) {
                    const f32x4 lo = *(const f32x4*)((const float*)a.q + at + d), hi = *(const f32x4*)((const float*)a.q + at + d + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[TQ];
                        terms<TQ>(e < 2 ? lo[2 * e] : hi[2 * e - 4], e < 2 ? lo[2 * e + 1] : hi[2 * e - 3], w);
#pragma unroll
                        for (int x = 0; x < TQ; ++x) qf[j][s][x][e] = w[x];
                    }
                } else {
                    qf[j][s][0] = *(const u32x4*)((const uint16_t*)a.q + at + d);
                }
            }
            lim[j] = kv - ql + t;
            lim_min = min(lim_min, lim[j]);
        }
    }
    lim_min = __reduce_min_sync(~0ull, lim_min);

    f32x4 acc[NT][C::DB];
    float mrow[NT], lsum[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        mrow[j] = -__builtin_huge_valf();
        lsum[j] = 0.0f;
#pragma unroll
        for (int d = 0; d < C::DB; ++d) acc[j][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

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
    // LDS addresses of the operand reads (the second half of a step and the key block are
    // immediate offsets: the swizzles leave bits 2 and 5 of the key alone)
    uint32_t kaddr[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int t = 8 * (lr >> 2) + (lr & 3);
        kaddr[i] = lds0 + t * C::RowB + 16 * k_slot<CH>(t, 4 * i + lq);
    }
    uint32_t vaddr[C::DB];
#pragma unroll
    for (int d = 0; d < C::DB; ++d) {
        const int t = 8 * lq + (lr >> 1);
        vaddr[d] = lds0 + C::TileB + t * C::RowB + 16 * v_slot<CH>(t, d) + 8 * (lr & 1);
    }
    const uint32_t saddr = lds0 + kScales + 4 * (lq >> 1);
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
        uint64_t kslot = (uint64_t)islot * p.ks2, vslot = (uint64_t)islot * p.vs2;  // bytes
        uint64_t vbase[P];
        int vkey = 0;
        auto copy = [&](uint64_t base, const uint32_t (&off)[S], int piece, int key0, uint32_t dst, auto slot, int bytes) {
            if (key0 + 16 <= kv && !p.pad) {
#pragma unroll
                for (int i = 0; i < S; ++i) lds_copy16_s(base, off[i], dst + (piece * S + i) * 1024);
            } else {
#pragma unroll
                for (int i = 0; i < S; ++i) {
                    const int t = (64 * i + lane) / CH, c = (64 * i + lane) % CH;
                    const bool in = key0 + t < kv && 16 * slot(t + 16 * (piece & 1), c) < bytes;
                    lds_copy16(in ? (const void*)(uintptr_t)(base + off[i]) : (const void*)g_zero,
                               dst + (piece * S + i) * 1024);
                }
            }
        };
        auto issue_k = [&]() {
            vkey = ikey;
            uint32_t si[P];  // scales of the pieces
#pragma unroll
            for (int h = 0; h < P; ++h) {
                const int lo = __builtin_amdgcn_readlane(pgs[0], ipg & 63);
                const int hi = __builtin_amdgcn_readlane(pgs[1], ipg & 63);
                const uint32_t page = ipg < DSPARK_WAVE ? lo : hi;
                vbase[h] = v_head + (uint64_t)page * p.vs0 + vslot;
                copy(k_head + (uint64_t)page * p.ks0 + kslot, ko[h & 1], h, ikey, lds0, k_slot<CH>, a.Dqk);
                si[h] = (page * (uint32_t)a.Hkv + (uint32_t)g) * (uint32_t)p.nb + (uint32_t)iblk;
                ikey += 16;
                islot += 16;
                iin += 16;
                kslot += 16 * p.ks2;  // 16 keys: below 2^32 bytes
                vslot += 16 * p.vs2;
                if (iin >= p.cs.block) {
                    iin = 0;
                    ++iblk;
                }
                if (islot >= a.page) {
                    islot = iblk = 0;
                    kslot = vslot = 0;
                    ++ipg;
                }
            }
            // lanes 0 .. P - 1 the keys' scales, the next P the values' (the others again)
            uint32_t mine = si[0];
#pragma unroll
            for (int h = 1; h < P; ++h) mine = (lane & (P - 1)) == h ? si[h] : mine;
            lds_copy4((lane & P ? p.cs.v : p.cs.k) + mine, lds0 + kScales);
        };
        auto issue_v = [&]() {
#pragma unroll
            for (int h = 0; h < P; ++h) copy(vbase[h], vo, h, vkey + 16 * h, lds0 + C::TileB, v_slot<CH>, a.Dv);
        };

        // ---- the segment.  One K and one V buffer: a buffer is refilled for the
        // next step as soon as this step's operands are in registers, so the next
        // K lands during the softmax and the value product and the next V during
        // the next scores.  Copies land in order: with V (or the next K) issued
        // after it, K (or V) has landed at vmcnt <= the copies of that.
        wait_copies<0>();
        issue_k();
        issue_v();
        for (int n = 0; n < nseg; ++n) {
            const int tok0 = (sb + n) * C::Step;
            const bool more = n + 1 < nseg;
            const bool full = tok0 + C::Step <= kv && tok0 + C::Step - 1 <= lim_min;
            wait_copies<P * S>();  // K and scales of step n
            u32x4 kf[H][2][S];
            float ksc[H], vsc[H];  // of the lane's eight keys of a half
#pragma unroll
            for (int h = 0; h < H; ++h) {
#pragma unroll
                for (int mb = 0; mb < 2; ++mb)
#pragma unroll
                    for (int i = 0; i < S; ++i)
                        kf[h][mb][i] = *lds_ptr<const lds_u32x4>(kaddr[i] + (32 * h + 4 * mb) * C::RowB);
                ksc[h] = *lds_ptr<const lds_f32>(saddr + 8 * h);
                vsc[h] = *lds_ptr<const lds_f32>(saddr + 8 * h + 4 * P);
            }
            wait_lds();
            if (more) issue_k();
            // scores: half h, keys tok0 + 32 h + 8 lq + 4 mb + e of query row lr
            f32x4 sc[NT][H][2];
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int mb = 0; mb < 2; ++mb) {
#pragma unroll
                    for (int j = 0; j < NT; ++j) sc[j][h][mb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < S; ++i)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const bf16x8 k = widen(kf[h][mb][i][2 * x], kf[h][mb][i][2 * x + 1]);
#pragma unroll
                            for (int j = 0; j < NT; ++j) {
                                if (j > 0 && j >= nt) continue;
#pragma unroll
                                for (int t = 0; t < TQ; ++t)
                                    sc[j][h][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                        k, __builtin_bit_cast(bf16x8, qf[j][2 * i + x][t]), sc[j][h][mb], 0, 0, 0);
                            }
                        }
                }
            u32x4 pb[NT][H][TP];  // probabilities times the values' scales
#pragma unroll
            for (int h = 0; h < H; ++h) ksc[h] *= p.scale2;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                if (j > 0 && j >= nt) continue;
                float sv[H][8];
#pragma unroll
                for (int h = 0; h < H; ++h)
#pragma unroll
                    for (int x = 0; x < 8; ++x) sv[h][x] = sc[j][h][x >> 2][x & 3] * ksc[h];
                if (!full) {
#pragma unroll
                    for (int h = 0; h < H; ++h)
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            const int key = tok0 + 32 * h + 8 * lq + x;
                            if (!(key < kv && key <= lim[j])) sv[h][x] = -__builtin_huge_valf();
                        }
                }
                float bm = -__builtin_huge_valf();
#pragma unroll
                for (int h = 0; h < H; ++h)
                    bm = vmax(bm, vmax(vmax(vmax(sv[h][0], sv[h][1]), vmax(sv[h][2], sv[h][3])),
                                       vmax(vmax(sv[h][4], sv[h][5]), vmax(sv[h][6], sv[h][7]))));
                bm = row_max4(bm);
                const bool need = bm > mrow[j] + kRescale;
                if (__builtin_amdgcn_ballot_w64(need)) {
                    const float mn = need ? bm : mrow[j];
                    const float alpha = need ? __builtin_amdgcn_exp2f(mrow[j] - mn) : 1.0f;
                    lsum[j] *= alpha;
#pragma unroll
                    for (int d = 0; d < C::DB; ++d) acc[j][d] *= alpha;
                    mrow[j] = mn;
                }
                const float mu = mrow[j] == -__builtin_huge_valf() ? 0.0f : mrow[j];
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    float pr[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) pr[x] = __builtin_amdgcn_exp2f(sv[h][x] - mu);
                    lsum[j] += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
                    if (full) {
#pragma unroll
                        for (int x = 0; x < 8; ++x) pr[x] *= vsc[h];
                    } else {  // (a masked key's scale may be anything)
#pragma unroll
                        for (int x = 0; x < 8; ++x) pr[x] = sv[h][x] == -__builtin_huge_valf() ? 0.0f : pr[x] * vsc[h];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t w[TP];
                        terms<TP>(pr[2 * e], pr[2 * e + 1], w);
#pragma unroll
                        for (int t = 0; t < TP; ++t) pb[j][h][t][e] = w[t];
                    }
                }
            }
            if (more) wait_copies<P * S + 1>();  // V of step n
            else wait_copies<0>();
            i32x2 vf[H][C::DB];  // dims 16 d + lr, keys 32 h + 8 lq ..
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int d = 0; d < C::DB; ++d)
                    vf[h][d] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(lds_ptr<lds_i32x2>(vaddr[d] + 32 * h * C::RowB));
            wait_lds();
            if (more) issue_v();
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int d = 0; d < C::DB; ++d) {
                    const bf16x8 v = widen(vf[h][d][0], vf[h][d][1]);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        if (j > 0 && j >= nt) continue;
#pragma unroll
                        for (int t = 0; t < TP; ++t)
                            acc[j][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                v, __builtin_bit_cast(bf16x8, pb[j][h][t]), acc[j][d], 0, 0, 0);
                    }
                }
        }
        sb = se;
    }

    // ---- rows: total l over the four lanes of a row
    const bool whole = s0 == 0 && s1 == ns;
    float* part = p.part + slot * ((int64_t)(16 * NT) * (C::Dp + 2));
    float big[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // largest sum by magnitude (NaN if one is), in independent chains
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        lsum[j] += __shfl_xor(lsum[j], 16, 64);
        lsum[j] += __shfl_xor(lsum[j], 32, 64);
        const int rr = 16 * j + lr, row = row0 + rr;
        if (row >= rows) continue;
        big[0] = vmax(big[0], lsum[j]);
#pragma unroll
        for (int d = 0; d < C::DB; ++d) {
            big[d & 3] = vmax(vmax(__builtin_fabsf(acc[j][d][0]), __builtin_fabsf(acc[j][d][1])), big[d & 3]);
            big[d & 3] = vmax(vmax(__builtin_fabsf(acc[j][d][2]), __builtin_fabsf(acc[j][d][3])), big[d & 3]);
        }
        const int t = row / p.group;
        const int64_t orow = (int64_t)(q0 + t) * a.Hq + g * p.group + (row - t * p.group);
        const float inv = 1.0f / lsum[j];
        if (whole) {
            if (a.lse && lq == 0) a.lse[orow] = (mrow[j] + log2f(lsum[j])) * kLn2;
        } else if (lq == 0) {
            part[rr] = mrow[j];
            part[16 * NT + rr] = lsum[j];
        }
#pragma unroll
        for (int d = 0; d < C::DB; ++d) {
            const int dim = 16 * d + 4 * lq;  // four consecutive dims of this lane
            const f32x4 o = acc[j][d];
            if (!whole) {
                *(f32x4*)(part + 2 * 16 * NT + (int64_t)rr * C::Dp + dim) = o;
            } else if (dim < a.Dv) {
                if (F32) *(f32x4*)((float*)a.out + orow * a.Dv + dim) = o * inv;
                else
                    *(uint2*)((uint16_t*)a.out + orow * a.Dv + dim) =
                        uint2{pack2_bf16(o[0] * inv, o[1] * inv), pack2_bf16(o[2] * inv, o[3] * inv)};
            }
        }
    }
    return __builtin_amdgcn_ballot_w64(!(vmax(vmax(big[0], big[1]), vmax(big[2], big[3])) < __builtin_huge_valf())) != 0;
}

template <bool F32, int CH, int NT>
__global__ __launch_bounds__(DSPARK_WAVE) __attribute__((amdgpu_waves_per_eu(Cfg<F32, CH, NT>::Eu)))
void attn_scaled_kernel(Params p) {
    typedef Cfg<F32, CH, NT> C;
    __shared__ __align__(16) unsigned char lds[C::LdsB];
    uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0];
    asm volatile("" : "+s"(lds0));
    bool again = false;
    range_walk<C::Step>(p, [&](int r, int g, int rc, int q0, int ql, int kv, int s0, int s1, int ns, int64_t slot) {
        again |= attend<F32, CH, NT>(p, lds0, r, g, rc, q0, ql, kv, s0, s1, ns, slot);
    });
    if (!again) return;
    // (a walk of its own, so that the step loop above holds none of its registers)
    __syncthreads();  // what the lanes of the wave wrote above comes before what others write below
    range_walk<C::Step>(p, [&](int r, int g, int rc, int q0, int ql, int kv, int s0, int s1, int ns, int64_t slot) {
        scaled_rows<F32, CH, NT>(p, r, g, rc, q0, ql, kv, s0, s1, ns, slot);
    });
}

// ------------------------------------------------------------------ host

struct Geom {
    int ch, nt, rc_max, direct;
    int64_t resident, waves;  // ranges; grid of the attention kernel
    size_t part_bytes;
};

template <typename F>
static auto with_cfg(bool bf16, int ch, int nt, F f) {
#define DS_CFG(F32, CH, NT) \
    return f(std::integral_constant<bool, F32>{}, std::integral_constant<int, CH>{}, std::integral_constant<int, NT>{})
    if (bf16) {
        if (ch == 4) {
            if (nt == 1) DS_CFG(false, 4, 1);
            if (nt == 2) DS_CFG(false, 4, 2);
            DS_CFG(false, 4, 4);
        }
        if (ch == 8) {
            if (nt == 1) DS_CFG(false, 8, 1);
            DS_CFG(false, 8, 2);
        }
        DS_CFG(false, 16, 1);
    }
    if (ch == 4) {
        if (nt == 1) DS_CFG(true, 4, 1);
        DS_CFG(true, 4, 2);
    }
    if (ch == 8) DS_CFG(true, 8, 1);
    DS_CFG(true, 16, 1);
#undef DS_CFG
}

static Geom geom(const AttnArgs& a) {
    Geom g;
    const int d = std::max(a.Dqk, a.Dv);
    g.ch = d <= 64 ? 4 : d <= 128 ? 8 : 16;
    const int64_t rows = (int64_t)a.max_q * (a.Hq / a.Hkv);
    const int64_t max_kv = (int64_t)a.max_pages * a.page;
    g.direct = max_kv <= kDirectKeys && (rows + 15) / 16 <= kDirectChunks;
    // row tiles per wave: as many as a request can fill, up to what the registers hold
    // (more tiles than these read the keys again, from the last-level cache).  Short
    // contexts have few waves and are bound by a wave's own chain of steps: one tile.
    const int most = a.bf16 ? (g.ch == 4 ? 4 : g.ch == 8 ? 2 : 1) : (g.ch == 4 ? 2 : 1);
    g.nt = g.direct ? 1 : (int)std::min<int64_t>(rows <= 16 ? 1 : rows <= 32 ? 2 : 4, most);
    g.rc_max = (int)((rows + 16 * g.nt - 1) / (16 * g.nt));
    const int64_t items = (int64_t)a.R * a.Hkv * g.rc_max;
    g.part_bytes = 0;
    with_cfg(a.bf16, g.ch, g.nt, [&](auto f32, auto ch, auto nt) {
        typedef Cfg<decltype(f32)::value, decltype(ch)::value, decltype(nt)::value> C;
        const int64_t units = items * ((max_kv + C::Step - 1) / C::Step);
        g.resident = kRangeCUs * C::Cu;
        g.waves = g.direct ? items : std::min<int64_t>(g.resident, (units + kMinUnits - 1) / kMinUnits);
        if (!g.direct) g.part_bytes = (size_t)g.waves * 2 * (16 * decltype(nt)::value) * (C::Dp + 2) * sizeof(float);
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
           g.waves < (int64_t)1 << 31 && (int64_t)a.R * a.Hkv < kRangePairs;
}

bool attn_scaled_supported(const AttnArgs& a, const CacheScales& c) {
    if (!attn_scaled_shape_ok(a)) return false;
    for (int i = 0; i < 3; ++i)
        if (a.ks[i] % 16 || a.vs[i] % 16) return false;
    // 32-bit page strides, offsets inside a 16-key piece and indexes of scales
    const int64_t lim0 = (int64_t)1 << 31, lim2 = (int64_t)1 << 24;
    if (a.ks[0] >= lim0 || a.vs[0] >= lim0 || a.ks[2] >= lim2 || a.vs[2] >= lim2) return false;
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
    p.chunk_rows = 16 * g.nt;
    p.by_head = 0;
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
    p.scale2 = a.scale * scaled::kLog2e;
    p.head = (int64_t*)ws;
    p.part = (float*)((char*)ws + range_head_bytes(a.R));
    return scaled::with_cfg(a.bf16, g.ch, g.nt, [&](auto f32, auto ch, auto nt) {
        constexpr bool F = decltype(f32)::value;
        constexpr int CH = decltype(ch)::value, NT = decltype(nt)::value;
        typedef scaled::Cfg<F, CH, NT> C;
        const dim3 grid = g.direct ? dim3((unsigned)(a.R * a.Hkv), (unsigned)g.rc_max) : dim3((unsigned)g.waves);
        hipLaunchKernelGGL((scaled::attn_scaled_kernel<F, CH, NT>), grid, dim3(DSPARK_WAVE), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess || g.direct) return e;
        return launch_merge<F, 16 * NT, C::Dp, C::Step>(p, s);
    });
}

}  // namespace dspark
