// A paged cache held in 8 bits (e4m3: 4 exponent and 3 fraction bits), with a scale for each page (64 tokens) and kv head.
//
//     value = code * scale,   scale = the smallest power of two with |x| <= 448 scale for every x of the page and head
//
// A power of two costs a floating code nothing (the spacing of e4m3 is relative down to 2^-6) and makes everything that
// follows exact: code * scale is a bf16 number, and a page that fills up token by token can be rounded anew when a larger
// token arrives: codes that stay normal numbers only change their exponents, so no error piles up.
//
// append8_kernel: a block for every (touched page, kv head, keys or values), and blocks for the tokens' queries.  A page
// block holds its new tokens (8 lanes a token, 16 channels a lane, two tokens a thread) in registers from the load over
// norm, rotation and the block's maximum to the codes: one pass.  Codes of earlier tokens are loaded beside them and stored
// again only if the scale grew.
// Bound: latency for a token an episode (a chain of loads, the block's maximum, stores), else the queries' traffic.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "head_norm.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

constexpr int kPage8 = 64, kAppend8Threads = 256;
constexpr int kScaleMin8 = -120, kScaleMax8 = 120;     // exponents; a page of zeros has the least scale

struct Append8Args {
    RopeArgs r;              // k_cache, v_cache: the code pools [pages, Hkv, 64, 128]
    NormArgs norm;
    float* k_scale;          // [pages, Hkv]
    float* v_scale;
    int page_blocks;         // touched pages * Hkv
    int q_parts;             // blocks per token for its queries
    FastDiv div_hkv, div_parts;
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
__global__ void __launch_bounds__(kAppend8Threads)
append8_kernel(const Append8Args p, const __grid_constant__ BatchLens lens)
{
    typedef __nv_bfloat16 T;
    constexpr int D = 128, half = 64;
    const RopeArgs& a = p.r;
    const int blk = blockIdx.x;
    int b = 0, hi = a.batch;
    if (blk >= 2 * p.page_blocks) {
        // ---- a token's queries ----
        const int at = blk - 2 * p.page_blocks, tok = (int)fast_div((uint32_t)at, p.div_parts), part = at - tok * p.q_parts;
        while (hi - b > 1) {                              // largest b with new_off[b] <= tok
            const int mid = (b + hi) >> 1;
            if (lens.new_off[mid] <= tok) b = mid; else hi = mid;
        }
        const int pos = lens.cache_len[b] + tok - lens.new_off[b];
        const double omega = !a.table && (int)threadIdx.x < half ? rope_omega(threadIdx.x, D, a.log2_theta) : 0.0;
        ptx::grid_dependency_wait();
        ptx::grid_launch_dependents();
        norm_token<T, NORM, false>(
            a, p.norm, tok, part, p.q_parts,
            [&](int h) -> T* {
                const int g = (int)fast_div((uint32_t)h, a.div_g);
                return (T*)a.q_rot + ((long)g * a.num_new * a.G + (long)tok * a.G + (h - g * a.G)) * D;
            },
            [](int) -> T* { return nullptr; }, [](int) -> T* { return nullptr; },
            [&](int j) -> double2 { return a.table ? a.table[(long)(pos - a.table_first) * half + j] : rope_cos_sin_at(pos, omega); });
        return;
    }
    // ---- a page of one kv head: keys (first, they have the longer chain) or values ----
    const bool is_v = blk >= p.page_blocks;
    const int item = is_v ? blk - p.page_blocks : blk;
    const int pg = (int)fast_div((uint32_t)item, p.div_hkv), g = item - pg * a.Hkv;
    while (hi - b > 1) {                                  // largest b with item_off[b] <= pg: touched pages before an episode's
        const int mid = (b + hi) >> 1;
        if (lens.item_off[mid] <= pg) b = mid; else hi = mid;
    }
    const int L = lens.cache_len[b], off = lens.new_off[b], n = lens.new_off[b + 1] - off;
    const int p0 = (L / kPage8 + pg - lens.item_off[b]) * kPage8;          // position of the page's first slot
    const int lane8 = threadIdx.x & 7, slot0 = threadIdx.x >> 3;           // slots slot0, slot0 + 32
    const int c0 = lane8 * 8;                                              // channels c0.., c0 + 64..
    __shared__ float s_most[kAppend8Threads / 32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int page = a.page_table[(long)b * a.max_pages + p0 / kPage8];
    uint8_t* pool = (uint8_t*)(is_v ? a.v_cache : a.k_cache) + ((long)page * a.Hkv + g) * (kPage8 * D);
    float* scale_at = (is_v ? p.v_scale : p.k_scale) + (long)page * a.Hkv + g;
    const bool held = p0 < L;

    uint4 raw[2][2];
    uint2 old[2][2];
    bool is_new[2], is_old[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int pos = p0 + slot0 + 32 * r;
        is_old[r] = pos < L;
        is_new[r] = pos >= L && pos < L + n;
        raw[r][0] = raw[r][1] = make_uint4(0u, 0u, 0u, 0u);
        if (is_new[r]) {
            const long tok = off + pos - L;
            const T* src = (is_v ? (const T*)a.v_new + tok * a.v_stride : (const T*)a.k_new + tok * a.k_stride) + (long)g * D + c0;
            raw[r][0] = *reinterpret_cast<const uint4*>(src);
            raw[r][1] = *reinterpret_cast<const uint4*>(src + half);
        }
        if (is_old[r]) {
            const uint8_t* at = pool + (slot0 + 32 * r) * D + c0;
            old[r][0] = *reinterpret_cast<const uint2*>(at);
            old[r][1] = *reinterpret_cast<const uint2*>(at + half);
        }
    }
    const float old_scale = held ? *scale_at : 0.f;
    uint4 w0 = make_uint4(0u, 0u, 0u, 0u), w1 = w0;
    if (NORM && !is_v && p.norm.k_weight) {
        w0 = *reinterpret_cast<const uint4*>((const T*)p.norm.k_weight + c0);
        w1 = *reinterpret_cast<const uint4*>((const T*)p.norm.k_weight + c0 + half);
    }
    float x[2][2][8];
    float most = 0.f;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        to_floats<T, 8>(raw[r][0], x[r][0]);
        to_floats<T, 8>(raw[r][1], x[r][1]);
        if (NORM && !is_v) norm_head<T, 8>(x[r][0], x[r][1], 3, D, p.norm.eps, p.norm.k_weight ? &w0 : nullptr, p.norm.k_weight ? &w1 : nullptr);
    }
    if (!is_v) {
        // every angle of a token serves one pair of this head, so the lanes take them straight from the table
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double omega = a.table ? 0.0 : rope_omega(c0 + i, D, a.log2_theta);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (!is_new[r]) continue;
                const int pos = p0 + slot0 + 32 * r;
                const double2 cs = a.table ? a.table[(long)(pos - a.table_first) * half + c0 + i] : rope_cos_sin_at(pos, omega);
                const float c = (float)cs.x, s = (float)cs.y, u = x[r][0][i], v = x[r][1][i];
                x[r][0][i] = fmaf(u, c, -(v * s));
                x[r][1][i] = fmaf(v, c, u * s);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if (is_new[r]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, fmaxf(finite_abs(x[r][0][i]), finite_abs(x[r][1][i])));
        }
    }
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
    if ((threadIdx.x & 31) == 0) s_most[threadIdx.x >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kAppend8Threads / 32; ++w) most = fmaxf(most, s_most[w]);
    const int e = scale_exponent8(most);
    const float need = exp2_int(e), scale = held && old_scale > need ? old_scale : need;
    const bool grew = held && scale > old_scale;
    const float inv = 1.f / scale, again = grew ? old_scale * inv : 1.f;   // powers of two: exact
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        uint2* to_lo = reinterpret_cast<uint2*>(pool + (slot0 + 32 * r) * D + c0);
        uint2* to_hi = reinterpret_cast<uint2*>(pool + (slot0 + 32 * r) * D + c0 + half);
        if (is_new[r]) {
            *to_lo = codes8(x[r][0], inv);
            *to_hi = codes8(x[r][1], inv);
        } else if (is_old[r]) {
            if (grew) {
                float y[8];
                floats4(old[r][0].x, y); floats4(old[r][0].y, y + 4);
                *to_lo = codes8(y, again);
                floats4(old[r][1].x, y); floats4(old[r][1].y, y + 4);
                *to_hi = codes8(y, again);
            }
        } else if (is_v) {
            *to_lo = *to_hi = make_uint2(0u, 0u);          // behind the last token: nothing that could be NaN
        }
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
