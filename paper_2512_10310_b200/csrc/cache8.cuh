// A paged cache held in 8 bits (e4m3: 4 exponent and 3 fraction bits), with a scale for each page (64 tokens) and kv head.
//
//     value = code * scale,   scale = the smallest power of two with |x| <= 448 scale for every x of the page and head
//
// A power of two costs a floating code nothing (the spacing of e4m3 is relative down to 2^-6) and makes everything that
// follows exact: code * scale is a bf16 number, and a page that fills up token by token can be rounded anew when a larger
// token arrives: codes that stay normal numbers only change their exponents, so no error piles up.
//
// append8_kernel: a block for every (touched page, kv head, keys or values), and blocks for the tokens' queries.  A page
// block holds its tokens (8 lanes a token, 16 channels a lane) in registers from the load over norm, rotation and the block's
// maximum to the codes: one pass.  Codes of earlier tokens are loaded instead of new ones and stored again only if the scale grew.
// Bound: latency for a token an episode (a chain of loads, the block's maximum, stores), else the queries' traffic.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "head_norm.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

constexpr int kPage8 = 64, kAppend8Threads = 8 * kPage8;
constexpr int kAppend8Tokens = 16;                     // most tokens of a query block
constexpr int kScaleMin8 = -120, kScaleMax8 = 120;     // exponents; a page of zeros has the least scale

struct Append8Args {
    RopeArgs r;              // k_cache, v_cache: the code pools [pages, Hkv, 64, 128]
    NormArgs norm;
    float* k_scale;          // [pages, Hkv]
    float* v_scale;
    int page_blocks;         // touched pages * Hkv
    int q_threads;           // threads per token for its queries (whole warps); a block takes kAppend8Threads / q_threads tokens
    int q_tokens;            // ... of them
    FastDiv div_hkv;
};

__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// The exponent of the scale that `most` (finite, >= 0) asks for: the least e with most <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ __forceinline__ int scale_exponent8(float most)
{
    const uint32_t bits = __float_as_uint(most);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < kScaleMin8 ? kScaleMin8 : e > kScaleMax8 ? kScaleMax8 : e;
}

// |x| for the page's maximum: infinities and NaN do not count (an infinity becomes the largest code, NaN a NaN code)
__device__ __forceinline__ float finite_abs(float x)
{
    const float m = fabsf(x);
    return m < INFINITY ? m : 0.f;
}

// floats to codes (nearest, ties to even; beyond 448 the largest code)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
__device__ __forceinline__ uint2 codes8(const float (&x)[8], float inv)
{
    return make_uint2(codes4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), codes4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
}
// four codes to four halves, exactly (NaN stays NaN)
__device__ __forceinline__ void halves4(uint32_t codes, uint32_t& lo, uint32_t& hi)
{
    asm("{\n\t.reg .b16 t, u;\n\tmov.b32 {t, u}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\tcvt.rn.f16x2.e4m3x2 %1, u;\n\t}" : "=r"(lo), "=r"(hi) : "r"(codes));
}
__device__ __forceinline__ void floats4(uint32_t codes, float* x)
{
    uint32_t lo, hi;
    halves4(codes, lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}

template <bool NORM>
__global__ void __launch_bounds__(kAppend8Threads, 2)
append8_kernel(const Append8Args p, const __grid_constant__ BatchLens lens)
{
    typedef __nv_bfloat16 T;
    constexpr int D = 128, half = 64, kVectors = 8;        // vector pairs of a head
    __shared__ __align__(16) TokenAngles<T, NORM> s_angles[kAppend8Tokens];
    __shared__ float s_most[kAppend8Threads / 32];
    const RopeArgs& a = p.r;
    const int blk = blockIdx.x, k = threadIdx.x & (kVectors - 1), c0 = k * 8;      // a lane's channels: c0 .. and c0 + 64 ..
    if (blk >= 2 * p.page_blocks) {
        // ---- queries of a few tokens ----
        const int tok0 = (blk - 2 * p.page_blocks) * p.q_tokens, tokens = min(p.q_tokens, a.num_new - tok0);
        auto position = [&](int tok) -> int {
            int b = 0, hi = a.batch;                          // largest b with new_off[b] <= tok
            while (hi - b > 1) {
                const int mid = (b + hi) >> 1;
                if (lens.new_off[mid] <= tok) b = mid; else hi = mid;
            }
            return lens.cache_len[b] + tok - lens.new_off[b];
        };
        const double omega = a.table ? 0.0 : rope_omega(threadIdx.x & (half - 1), D, a.log2_theta);
        const int group = threadIdx.x / p.q_threads, tok = tok0 + group, items = a.Hq * kVectors;
        ptx::grid_dependency_wait();
        ptx::grid_launch_dependents();
        int it = threadIdx.x - group * p.q_threads;
        const bool there = group < tokens;
        const T* src = (const T*)a.q_new + tok * a.q_stride + c0;
        uint4 r0 = make_uint4(0u, 0u, 0u, 0u), r1 = r0;
        auto load = [&]() {
            if (there && it < items) {
                r0 = *reinterpret_cast<const uint4*>(src + (it / kVectors) * D);
                r1 = *reinterpret_cast<const uint4*>(src + (it / kVectors) * D + half);
            }
        };
        load();                                               // in flight while the angles arrive
        for (int e = threadIdx.x; e < tokens * half; e += kAppend8Threads) {
            const int j = e & (half - 1), pos = position(tok0 + e / half);
            s_angles[e / half].put(j, a.table ? a.table[(long)(pos - a.table_first) * half + j] : rope_cos_sin_at(pos, omega));
        }
        __syncthreads();
        if (!there) return;                                   // (whole warps)
        for (; it - (int)(threadIdx.x & 31) < items; it += p.q_threads, load()) {
            uint4 y0, y1;
            if constexpr (NORM) norm_turn<T>(s_angles[group], k, 3, D, p.norm.eps, (const T*)p.norm.q_weight, r0, r1, y0, y1);
            else Rotation<T>::turn(s_angles[group].at, k, r0, r1, y0, y1);
            if (it >= items) continue;
            const int h = it / kVectors, g = (int)fast_div((uint32_t)h, a.div_g);
            T* dst = (T*)a.q_rot + ((long)g * a.num_new * a.G + (long)tok * a.G + (h - g * a.G)) * D + c0;
            *reinterpret_cast<uint4*>(dst) = y0;
            *reinterpret_cast<uint4*>(dst + half) = y1;
        }
        return;
    }
    // ---- a page of one kv head: keys (first, they have the longer chain) or values ----
    const bool is_v = blk >= p.page_blocks;
    const int item = is_v ? blk - p.page_blocks : blk;
    const int pg = (int)fast_div((uint32_t)item, p.div_hkv), g = item - pg * a.Hkv;
    int b = 0, hi = a.batch;
    while (hi - b > 1) {                                  // largest b with item_off[b] <= pg: touched pages before an episode's
        const int mid = (b + hi) >> 1;
        if (lens.item_off[mid] <= pg) b = mid; else hi = mid;
    }
    const int L = lens.cache_len[b], off = lens.new_off[b], n = lens.new_off[b + 1] - off;
    const int p0 = (L / kPage8 + pg - lens.item_off[b]) * kPage8;          // position of the page's first slot
    const int slot = threadIdx.x / kVectors, pos = p0 + slot;
    const bool is_old = pos < L, is_new = pos >= L && pos < L + n, held = p0 < L;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int page = a.page_table[(long)b * a.max_pages + p0 / kPage8];
    uint8_t* at = (uint8_t*)(is_v ? a.v_cache : a.k_cache) + (((long)page * a.Hkv + g) * kPage8 + slot) * D + c0;
    float* scale_at = (is_v ? p.v_scale : p.k_scale) + (long)page * a.Hkv + g;

    uint4 r0 = make_uint4(0u, 0u, 0u, 0u), r1 = r0;       // a new token's 16 numbers, or an earlier one's 16 codes
    if (is_new) {
        const long tok = off + pos - L;
        const T* src = (is_v ? (const T*)a.v_new + tok * a.v_stride : (const T*)a.k_new + tok * a.k_stride) + (long)g * D + c0;
        r0 = *reinterpret_cast<const uint4*>(src);
        r1 = *reinterpret_cast<const uint4*>(src + half);
    } else if (is_old) {
        const uint2 lo = *reinterpret_cast<const uint2*>(at), hi8 = *reinterpret_cast<const uint2*>(at + half);
        r0 = make_uint4(lo.x, lo.y, hi8.x, hi8.y);
    }
    const float old_scale = held ? *scale_at : 0.f;
    float x[2][8], most = 0.f;
    float inv = 1.f;
    if (NORM && !is_v) inv = norm_factor<T>(r0, r1, 3, D, p.norm.eps);
    if (is_new) {
        to_floats<T, 8>(r0, x[0]);
        to_floats<T, 8>(r1, x[1]);
        if (!is_v) {
            if (NORM) {
                const T* w = (const T*)p.norm.k_weight;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[0][i] *= inv * (w ? to_float(w[c0 + i]) : 1.f);
                    x[1][i] *= inv * (w ? to_float(w[c0 + half + i]) : 1.f);
                }
            }
            // every angle of a token serves one pair of this head, so the lanes take them straight from the table
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double2 cs = a.table ? a.table[(long)(pos - a.table_first) * half + c0 + i] : rope_cos_sin(pos, c0 + i, D, a.log2_theta);
                const float c = (float)cs.x, s = (float)cs.y, u = x[0][i], v = x[1][i];
                x[0][i] = fmaf(u, c, -(v * s));
                x[1][i] = fmaf(v, c, u * s);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, fmaxf(finite_abs(x[0][i]), finite_abs(x[1][i])));
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
    if ((threadIdx.x & 31) == 0) s_most[threadIdx.x >> 5] = most;
    __syncthreads();
    most = s_most[threadIdx.x & (kAppend8Threads / 32 - 1)];
#pragma unroll
    for (int s = kAppend8Threads / 64; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
    const float need = exp2_int(scale_exponent8(most)), scale = held && old_scale > need ? old_scale : need;
    const bool grew = held && scale > old_scale;
    const float down = 1.f / scale;                        // powers of two: exact
    if (is_old && grew) {
        const float again = old_scale * down;
        floats4(r0.x, x[0]); floats4(r0.y, x[0] + 4);
        floats4(r0.z, x[1]); floats4(r0.w, x[1] + 4);
        *reinterpret_cast<uint2*>(at) = codes8(x[0], again);
        *reinterpret_cast<uint2*>(at + half) = codes8(x[1], again);
    } else if (is_new) {
        *reinterpret_cast<uint2*>(at) = codes8(x[0], down);
        *reinterpret_cast<uint2*>(at + half) = codes8(x[1], down);
    } else if (is_v && !is_old) {
        *reinterpret_cast<uint2*>(at) = *reinterpret_cast<uint2*>(at + half) = make_uint2(0u, 0u);      // behind the last token: nothing that could be NaN
    }
    if (threadIdx.x == 0 && (!held || grew)) *scale_at = scale;
}

// The batch's pages as bf16, exactly: page i of an episode goes to page first + i of the copy, whose table says so.  Each code
// is read once, and the copy is what the tensor-core kernel of the bf16 cache reads.
struct Expand8Args {
    const uint8_t* k_pool;
    const uint8_t* v_pool;
    const float* k_scale;
    const float* v_scale;
    __nv_bfloat16* k_out;    // [pages of the batch, Hkv, 64, 128]
    __nv_bfloat16* v_out;
    const int* page_table;
    int* out_table;          // [batch, max_pages]
    int Hkv, batch, max_pages;
};

__global__ void __launch_bounds__(256)
expand8_kernel(const Expand8Args a, const __grid_constant__ BatchLens lens)
{
    const int pg = blockIdx.x, g = blockIdx.y;
    const bool is_v = blockIdx.z != 0;
    int b = 0, hi = a.batch;
    while (hi - b > 1) {                                  // largest b with item_off[b] <= pg: pages before an episode's
        const int mid = (b + hi) >> 1;
        if (lens.item_off[mid] <= pg) b = mid; else hi = mid;
    }
    const int i = pg - lens.item_off[b];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int page = a.page_table[(long)b * a.max_pages + i];
    const long from = (long)page * a.Hkv + g, to = (long)pg * a.Hkv + g;
    if (g == 0 && !is_v && threadIdx.x == 0) a.out_table[(long)b * a.max_pages + i] = pg;
    const uint4* src = reinterpret_cast<const uint4*>((is_v ? a.v_pool : a.k_pool) + from * (kPage8 * 128));
    uint4* dst = reinterpret_cast<uint4*>((is_v ? a.v_out : a.k_out) + to * (kPage8 * 128));
    const float scale = (is_v ? a.v_scale : a.k_scale)[from];
    uint4 c[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) c[r] = src[threadIdx.x + 256 * r];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float x[16];
        floats4(c[r].x, x); floats4(c[r].y, x + 4); floats4(c[r].z, x + 8); floats4(c[r].w, x + 12);
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = ptx::pack_bf16x2(x[2 * k] * scale, x[2 * k + 1] * scale);
        dst[2 * (threadIdx.x + 256 * r)] = make_uint4(w[0], w[1], w[2], w[3]);
        dst[2 * (threadIdx.x + 256 * r) + 1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

}  // namespace evln
