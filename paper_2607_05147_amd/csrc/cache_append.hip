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
// An item is one wave: a step brings a request a few rows, 64 lanes x 8 values
// hold a row of four heads of 128, and nothing waits for another wave.  The new
// values stay in registers between the maximum and the rounding.  Bound by launch
// and three dependent loads at a step's sizes, by HBM for prompts.
#include <algorithm>
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace dspark {

namespace {

constexpr int kApThreads = 256;
constexpr int kApWaves = kApThreads / DSPARK_WAVE;
constexpr int kApKeep = 8;                // groups of values a lane keeps
constexpr int64_t kApGrid = 1 << 20;      // workgroups, at most (they stride over the items)

struct ApParams {
    AppendArgs a;
    int nblk;       // blocks that a request's rows can reach
    int sides;      // 2: keys and values, 1: keys alone
    int64_t items;
};

// N consecutive values of a row, as fp32
template <typename T, int N>
__device__ __forceinline__ void load_values(const T* p, float (&x)[N]) {
    if constexpr (N == 1) {
        x[0] = Elem<T>::load(p, 0);
    } else if constexpr (std::is_same<T, float>::value) {
        const float4 lo = *(const float4*)p, hi = *(const float4*)(p + 4);
        x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w;
        x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
    } else {
        const uint4 v = *(const uint4*)p;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

template <int N>
__device__ __forceinline__ void store_codes(uint8_t* p, const float (&x)[N], float inv) {
    if constexpr (N == 1) {
        *p = (uint8_t)to_e4m3(x[0], 0.0f, inv, 0, false);
    } else {
        uint2 w;
        w.x = to_e4m3(x[2], x[3], inv, to_e4m3(x[0], x[1], inv, 0, false), true);
        w.y = to_e4m3(x[6], x[7], inv, to_e4m3(x[4], x[5], inv, 0, false), true);
        *(uint2*)p = w;
    }
}

// exponent of the smallest power of two that is not below s
__device__ __forceinline__ int ceil_exp(float s) {
    const uint32_t u = __float_as_uint(s);
    const int k = (int)(u >> 23) - 127 + ((u & 0x7fffffu) != 0);
    return min(max(k, kMinScaleExp), kMaxScaleExp);
}

template <typename T, int N>
__global__ __launch_bounds__(kApThreads) void cache_append(ApParams p) {
    const AppendArgs& a = p.a;
    const int lane = threadIdx.x & (DSPARK_WAVE - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / DSPARK_WAVE);
    const int64_t total_rows = min((int64_t)max(a.cu_q[a.R], 0), (int64_t)a.R * a.max_q);
    for (int64_t it = (int64_t)blockIdx.x * kApWaves + wave; it < p.items; it += (int64_t)gridDim.x * kApWaves) {
        int64_t id = it;
        const int h = (int)(id % a.Hkv);
        id /= a.Hkv;
        const int side = (int)(id % p.sides);
        id /= p.sides;
        const int i = (int)(id % p.nblk), r = (int)(id / p.nblk);
        const int q0 = a.cu_q[r], ql = a.cu_q[r + 1] - q0, kv = a.kv_len[r];
        if (ql < 1 || ql > a.max_q || kv < ql || kv > a.max_pages * a.page || q0 < 0 || (int64_t)q0 + ql > total_rows) continue;
        const int kv0 = kv - ql;
        const int lo = (kv0 / a.block + i) * a.block;  // first token of the block
        if (lo >= kv) continue;
        const int pid = a.block_table[(int64_t)r * a.max_pages + lo / a.page];
        if ((unsigned)pid >= (unsigned)a.num_pages) continue;
        const int slot = lo % a.page;
        const int first = max(lo, kv0), n = min(kv, lo + a.block) - first;  // new tokens of the block
        const int D = side ? a.Dv : a.Dqk;
        const int64_t* st = side ? a.vs : a.ks;
        const T* src = (const T*)(side ? a.v : a.k) + (int64_t)(q0 + first - kv0) * (side ? a.v_ld : a.k_ld) + (int64_t)h * D;
        const int64_t ld = side ? a.v_ld : a.k_ld;
        uint8_t* dst = (uint8_t*)(side ? a.v_cache : a.k_cache) + pid * st[0] + h * st[1] + (int64_t)slot * st[2];
        float* scale = (side ? a.v_scale : a.k_scale) + ((int64_t)pid * a.Hkv + h) * (a.page / a.block) + slot / a.block;
        const float s_old = first > lo ? *scale : 0.0f;

        const int per = D / N, groups = n * per;  // groups of N values
        float x[kApKeep][N], most = 0.0f;
        auto look = [&](const float (&y)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float b = __builtin_fabsf(y[e]);
                if (b < __builtin_huge_valf()) most = fmaxf(most, b);
            }
        };
#pragma unroll
        for (int k = 0; k < kApKeep; ++k) {
            const int g = k * DSPARK_WAVE + lane;
            if (g < groups) load_values<T, N>(src + (int64_t)(g / per) * ld + (g % per) * N, x[k]);
        }
#pragma unroll
        for (int k = 0; k < kApKeep; ++k)
            if (k * DSPARK_WAVE + lane < groups) look(x[k]);
        for (int g = kApKeep * DSPARK_WAVE + lane; g < groups; g += DSPARK_WAVE) {
            float y[N];
            load_values<T, N>(src + (int64_t)(g / per) * ld + (g % per) * N, y);
            look(y);
        }
        most = wave_max(most);

        int e = 0x7fffffff;  // of the scale
        const float so = __builtin_fabsf(s_old);
        if (most > 0.0f) e = e4m3_scale_exp(most);
        if (so > 0.0f && so < __builtin_huge_valf()) e = e == 0x7fffffff ? ceil_exp(so) : max(e, ceil_exp(so));
        if (e == 0x7fffffff) e = 0;  // nothing but zeros (or nothing finite)
        const float s = __uint_as_float((uint32_t)(e + 127) << 23), inv = __uint_as_float((uint32_t)(127 - e) << 23);

#pragma unroll
        for (int k = 0; k < kApKeep; ++k) {
            const int g = k * DSPARK_WAVE + lane;
            if (g < groups) store_codes<N>(dst + (int64_t)(first - lo + g / per) * st[2] + (g % per) * N, x[k], inv);
        }
        for (int g = kApKeep * DSPARK_WAVE + lane; g < groups; g += DSPARK_WAVE) {
            float y[N];
            load_values<T, N>(src + (int64_t)(g / per) * ld + (g % per) * N, y);
            store_codes<N>(dst + (int64_t)(first - lo + g / per) * st[2] + (g % per) * N, y, inv);
        }
        if (first > lo && s_old != s) {
            const float ratio = s_old * inv;
            for (int g = lane; g < (first - lo) * per; g += DSPARK_WAVE) {
                uint8_t* c = dst + (int64_t)(g / per) * st[2] + (g % per) * N;
                float y[N];
                if constexpr (N == 1) {
                    y[0] = e4m3_to_f32(*c);
                } else {
                    const uint2 w = *(const uint2*)c;
#pragma unroll
                    for (int b = 0; b < 4; ++b) y[b] = e4m3_to_f32(w.x >> (8 * b)), y[4 + b] = e4m3_to_f32(w.y >> (8 * b));
                }
                store_codes<N>(c, y, ratio);
            }
        }
        if (lane == 0) *scale = s;
    }
}

}  // namespace

hipError_t launch_cache_append(const AppendArgs& a, hipStream_t s) {
    ApParams p;
    p.a = a;
    p.nblk = (int)(((int64_t)a.max_q - 1) / a.block + 2);
    p.sides = a.v ? 2 : 1;
    p.items = (int64_t)a.R * p.nblk * p.sides * a.Hkv;
    // 8 values at a time where rows and slots allow 16-byte loads and 8-byte stores
    const int64_t per = a.bf16 ? 8 : 4;
    bool wide = (uintptr_t)a.k % 16 == 0 && (uintptr_t)a.v % 16 == 0 && (uintptr_t)a.k_cache % 8 == 0 &&
                (uintptr_t)a.v_cache % 8 == 0 && a.k_ld % per == 0 && (!a.v || a.v_ld % per == 0);
    for (int i = 0; i < 3; ++i) wide = wide && a.ks[i] % 8 == 0 && (!a.v || a.vs[i] % 8 == 0);
    const dim3 grid((unsigned)std::min<int64_t>((p.items + kApWaves - 1) / kApWaves, kApGrid));
    if (a.bf16 && wide) hipLaunchKernelGGL((cache_append<uint16_t, 8>), grid, dim3(kApThreads), 0, s, p);
    else if (a.bf16) hipLaunchKernelGGL((cache_append<uint16_t, 1>), grid, dim3(kApThreads), 0, s, p);
    else if (wide) hipLaunchKernelGGL((cache_append<float, 8>), grid, dim3(kApThreads), 0, s, p);
    else hipLaunchKernelGGL((cache_append<float, 1>), grid, dim3(kApThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace dspark
