// Quantises a step's new key and value rows into a paged cache of e4m3 codes
// with a scale for each block of tokens and head.
//
// For every (request, head, block of tokens that gets new rows, keys | values):
//   s = the smallest power of two with max |x| <= 448 s over the block's new
//       finite values, and no smaller than the scale its earlier tokens have;
//   code = e4m3(x / s), to nearest even; where s grew, the earlier tokens'
//       codes become e4m3(code * s_old / s).
// With powers of two x / s is exact, so a code is one rounding of its value, and
// rescaling changes only what falls below 2^-6 of the range: a block can be filled
// a few tokens at a time, and rolled back, without its values drifting (with
// s = max / 448 every growth would round the whole block again).
//
// A wave takes a block of one head: a step brings a request a few rows, 64 lanes x 8
// values hold four rows of 128, and nothing waits for another wave.  The new values
// stay in registers between the maximum and the rounding (eight passes of 64 x 16
// bytes, 32 rows of 128 in bf16; more than that is read twice, from L2).  Heads
// are the fastest index of the grid, so neighbours read one row of the step.  Passes
// are uniform: with lanes that walked rows and columns on their own the compiler kept
// an address and a mask a pass (151 registers, three waves a SIMD instead of five).
//
// Bound by launch and three dependent loads at a step's sizes (565 rows of 8 heads:
// 7.0 us).  Prompts: 40000 rows of 8 heads of 128, 246 MB, 70 us, 3.5 TB/s; a wave's loads,
// maximum and stores follow each other, and workgroups of a grid for max_q find no rows.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace dspark {

namespace {

constexpr int kApThreads = 256;
constexpr int kApWaves = kApThreads / DSPARK_WAVE;
constexpr int kApBlocks = 65535;          // of a grid's third dimension, at most (workgroups stride over the rest)

struct ApParams {
    AppendArgs a;
    int nblk;         // blocks that a request's rows can reach
    int head_groups;  // of kApWaves heads
};

// N consecutive values of a row, as they are there (keep: the compiler does not hold
// their fp32 forms instead, which are twice as wide)
template <typename T, int N>
struct Group;
template <typename T>
struct Group<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = Elem<T>::load(&v, 0); }
    __device__ __forceinline__ void keep() { asm("" : "+v"(v)); }
};
template <>
struct Group<uint16_t, 8> {
    uint4 v;
    __device__ __forceinline__ void load(const uint16_t* p) { v = *(const uint4*)p; }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void keep() { asm("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }
};
template <>
struct Group<float, 8> {
    float4 lo, hi;
    __device__ __forceinline__ void load(const float* p) { lo = *(const float4*)p, hi = *(const float4*)(p + 4); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
        x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w;
        x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
    }
    __device__ __forceinline__ void keep() {}
};

typedef uint32_t Codes8 __attribute__((ext_vector_type(2)));

// (past the caches: what a prompt writes is not read soon; 74 against 70 us)
template <int N>
__device__ __forceinline__ void store_codes(uint8_t* p, const float (&x)[N], float inv) {
    if constexpr (N == 1) {
        *p = (uint8_t)to_e4m3(x[0], 0.0f, inv, 0, false);
    } else {
        Codes8 w;
        w.x = to_e4m3(x[2], x[3], inv, to_e4m3(x[0], x[1], inv, 0, false), true);
        w.y = to_e4m3(x[6], x[7], inv, to_e4m3(x[4], x[5], inv, 0, false), true);
        __builtin_nontemporal_store(w, (Codes8*)p);
    }
}

// exponent of the smallest power of two that is not below s
__device__ __forceinline__ int ceil_exp(float s) {
    const uint32_t u = __float_as_uint(s);
    const int k = (int)(u >> 23) - 127 + ((u & 0x7fffffu) != 0);
    return min(max(k, kMinScaleExp), kMaxScaleExp);
}

// Workgroups: side and four heads, request, block of its new rows.
template <typename T, int N>
__global__ __launch_bounds__(kApThreads) void cache_append(ApParams p) {
    const AppendArgs& a = p.a;
    const int lane = threadIdx.x & (DSPARK_WAVE - 1);
    const int r = blockIdx.y, side = blockIdx.x / p.head_groups;
    const int h = (blockIdx.x - side * p.head_groups) * kApWaves + (int)__builtin_amdgcn_readfirstlane(threadIdx.x / DSPARK_WAVE);
    const int q0 = a.cu_q[r], ql = a.cu_q[r + 1] - q0, kv = a.kv_len[r];
    const int64_t total_rows = min((int64_t)max(a.cu_q[a.R], 0), (int64_t)a.R * a.max_q);
    if (h >= a.Hkv || ql < 1 || ql > a.max_q || kv < ql || kv > a.max_pages * a.page || q0 < 0 || (int64_t)q0 + ql > total_rows) return;
    const int kv0 = kv - ql;
    const int D = side ? a.Dv : a.Dqk;
    const int64_t ld = side ? a.v_ld : a.k_ld, s0 = side ? a.vs[0] : a.ks[0], s1 = side ? a.vs[1] : a.ks[1], s2 = side ? a.vs[2] : a.ks[2];
    const T* rows = (const T*)(side ? a.v : a.k) + (int64_t)h * D;
    uint8_t* cache = (uint8_t*)(side ? a.v_cache : a.k_cache) + h * s1;
    float* scales = side ? a.v_scale : a.k_scale;
    // a pass: 64 / width rows of `width` groups of N values (a power of two; of wider rows
    // 64 groups at a time), so that what changes from pass to pass is the same in every lane
    const int per = D / N;
    int width = 64;
    while (width / 2 >= per) width /= 2;
    const int lrow = lane / width, lcol = lane % width, rows_of = DSPARK_WAVE / width;
    const int64_t from0 = lrow * ld + lcol * N, to0 = lrow * s2 + lcol * N;  // this lane's group of the first pass
    for (int i = blockIdx.z; i < p.nblk; i += gridDim.z) {
        const int lo = (kv0 / a.block + i) * a.block;  // first token of the block
        if (lo >= kv) return;
        const int pid = a.block_table[(int64_t)r * a.max_pages + lo / a.page];
        const int first = max(lo, kv0), n = min(kv, lo + a.block) - first;  // new tokens of the block
        const T* src = rows + (int64_t)(q0 + first - kv0) * ld + from0;
        constexpr int kKeep = sizeof(Group<T, N>) == 32 ? 4 : 8;  // groups a lane keeps
        Group<T, N> x[kKeep];
        float most = 0.0f;
        auto look = [&](const Group<T, N>& from) {
            float y[N];
            from.get(y);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float b = __builtin_fabsf(y[e]);
                if (b < __builtin_huge_valf()) most = fmaxf(most, b);
            }
        };
        // f(k, row, column) for the passes over `tokens` rows: the first kKeep, then the rest
        auto next = [&](int& row, int& col) {
            col += DSPARK_WAVE;
            if (col >= per) col = 0, row += rows_of;
        };
        auto walk = [&](int tokens, auto kept, auto rest) {
            int row = 0, col = 0;
            asm("" : "+s"(tokens));  // (the passes' masks are made anew, not held)
#pragma unroll
            for (int k = 0; k < kKeep; ++k) {
                if (row >= tokens) return;
                if (row + lrow < tokens && col + lcol < per) kept(k, row, col * N);
                next(row, col);
            }
            for (; row < tokens; next(row, col))
                if (row + lrow < tokens && col + lcol < per) rest(row, col * N);
        };
        // (the rows, the page and its scale are loaded together)
        walk(n, [&](int k, int row, int c) { x[k].load(src + row * ld + c); }, [](int, int) {});
        if ((unsigned)pid >= (unsigned)a.num_pages) continue;
        const int slot = lo % a.page;
        uint8_t* dst = cache + pid * s0 + slot * s2 + to0;
        float* scale = scales + ((int64_t)pid * a.Hkv + h) * (a.page / a.block) + slot / a.block;
        const float s_old = first > lo ? *scale : 0.0f;
        walk(n, [&](int k, int, int) { look(x[k]); },
             [&](int row, int c) {
                 Group<T, N> y;
                 y.load(src + row * ld + c);
                 look(y);
             });
        most = wave_max(most);

        int e = 0x7fffffff;  // of the scale
        const float so = __builtin_fabsf(s_old);
        if (most > 0.0f) e = e4m3_scale_exp(most);
        if (so > 0.0f && so < __builtin_huge_valf()) e = e == 0x7fffffff ? ceil_exp(so) : max(e, ceil_exp(so));
        if (e == 0x7fffffff) e = 0;  // nothing but zeros (or nothing finite)
        const float s = __uint_as_float((uint32_t)(e + 127) << 23), inv = __uint_as_float((uint32_t)(127 - e) << 23);

        uint8_t* to = dst + (first - lo) * s2;
        auto round = [&](const Group<T, N>& from, int row, int c) {
            float y[N];
            from.get(y);
            store_codes<N>(to + row * s2 + c, y, inv);
        };
        walk(n, [&](int k, int row, int c) { x[k].keep(), round(x[k], row, c); },
             [&](int row, int c) {
                 Group<T, N> y;
                 y.load(src + row * ld + c);
                 round(y, row, c);
             });
        if (first > lo && s_old != s) {
            const float ratio = s_old * inv;
            auto again = [&](int row, int c) {
                uint8_t* at = dst + row * s2 + c;
                float y[N];
                if constexpr (N == 1) {
                    y[0] = e4m3_to_f32(*at);
                } else {
                    const uint2 w = *(const uint2*)at;
#pragma unroll
                    for (int b = 0; b < 4; ++b) y[b] = e4m3_to_f32(w.x >> (8 * b)), y[4 + b] = e4m3_to_f32(w.y >> (8 * b));
                }
                store_codes<N>(at, y, ratio);
            };
            for (int row = 0, col = 0; row < first - lo; next(row, col))
                if (row + lrow < first - lo && col + lcol < per) again(row, col * N);
        }
        if (lane == 0) *scale = s;
    }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
    ApParams p;
    p.a = a;
    p.nblk = (int)(((int64_t)a.max_q - 1) / a.block + 2);
    p.head_groups = (a.Hkv + kApWaves - 1) / kApWaves;
    // 8 values at a time where rows and slots allow 16-byte loads and 8-byte stores
    const int64_t per = a.bf16 ? 8 : 4;
    bool wide = (uintptr_t)a.k % 16 == 0 && (uintptr_t)a.v % 16 == 0 && (uintptr_t)a.k_cache % 8 == 0 &&
                (uintptr_t)a.v_cache % 8 == 0 && a.k_ld % per == 0 && (!a.v || a.v_ld % per == 0);
    for (int i = 0; i < 3; ++i) wide = wide && a.ks[i] % 8 == 0 && (!a.v || a.vs[i] % 8 == 0);
    const dim3 grid((unsigned)(p.head_groups * (a.v ? 2 : 1)), (unsigned)a.R, (unsigned)std::min(p.nblk, kApBlocks));
    if (a.bf16 && wide) hipLaunchKernelGGL((cache_append<uint16_t, 8>), grid, dim3(kApThreads), 0, s, p);
    else if (a.bf16) hipLaunchKernelGGL((cache_append<uint16_t, 1>), grid, dim3(kApThreads), 0, s, p);
    else if (wide) hipLaunchKernelGGL((cache_append<float, 8>), grid, dim3(kApThreads), 0, s, p);
    else hipLaunchKernelGGL((cache_append<float, 1>), grid, dim3(kApThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace dspark
