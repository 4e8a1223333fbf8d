// A paged cache held in 8 bits (e4m3: 4 exponent and 3 fraction bits), with a scale for each page (64 tokens) and kv head.
//
//     value = code * scale,   scale = the smallest power of two with |x| <= 448 scale for every x of the page and head
//
// A power of two costs a floating code nothing (the spacing of e4m3 is relative down to 2^-6) and makes everything that
// follows exact: code * scale is a bf16 number, and a page that fills up token by token can be rounded anew when a larger
// token arrives: codes that stay normal numbers only change their exponents, so no error piles up.
//
// append8_kernel: a block for every (touched page, kv head, keys or values), and blocks for the tokens' queries (warps as in
// head_norm.cuh).  A page block holds its tokens (8 lanes and 16 channels a lane for each, two tokens a lane) in registers from the load over
// norm, rotation and the block's maximum to the codes: one pass.  Codes of earlier tokens are loaded instead of new ones and stored again only
// if the scale grew.
// Bound: latency for a token an episode (a chain of loads, the block's maximum, stores: 16 episodes 2.4 us), else the queries' traffic (16 frames of
// 196 tokens with norms, 56 MB, 16.4 us).  (One token a lane, blocks of 512 threads: 2.7 and 21.4 us.)
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "head_norm.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

constexpr int kPage8 = 64, kAppend8Threads = 4 * kPage8, kAppend8Blocks = 3;
constexpr int kScaleMin8 = -120, kScaleMax8 = 120;     // exponents; a page of zeros has the least scale

struct Append8Args {
    RopeArgs r;              // k_cache, v_cache: the code pools [pages, Hkv, 64, 128]
    NormArgs norm;
    float* k_scale;          // [pages, Hkv]
    float* v_scale;
    int page_blocks;         // touched pages * Hkv
    int q_warps;             // warps per token for its queries
    FastDiv div_hkv, div_warps;
};

__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

// The exponent of the scale that `most` (finite, >= 0) asks for: the least e with most <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ __forceinline__ int scale_exponent8(float most)
{
    const uint32_t bits = __float_as_uint(most);
    const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < kScaleMin8 ? kScaleMin8 : e > kScaleMax8 ? kScaleMax8 : e;
}

// floats to codes (nearest, ties to even; beyond 448 the largest code)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
// eight floats (four pairs) times down to codes
__device__ __forceinline__ uint2 codes8(const uint64_t (&x)[4], float down)
{
    const uint64_t d = ptx::pack2(down, down);
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) ptx::unpack2(ptx::mul2(x[i], d), f[2 * i], f[2 * i + 1]);
    return make_uint2(codes4(f[0], f[1], f[2], f[3]), codes4(f[4], f[5], f[6], f[7]));
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

template <bool NORM, bool TABLE>
__global__ void __launch_bounds__(kAppend8Threads, kAppend8Blocks)
append8_kernel(const Append8Args p, const __grid_constant__ BatchLens lens)
{
    typedef __nv_bfloat16 T;
    constexpr int D = 128, half = 64, kVectors = 8;        // vector pairs of a head
    constexpr int kWarps = kAppend8Threads / 32;
    __shared__ union {
        TokenAngles<T, NORM> of_token[kWarps];             // queries: a warp's token
        TokenAngles<T, true> of_slots[kWarps][4];          // keys: a warp's four tokens
    } s_angles;
    __shared__ float s_most[kWarps];
    const RopeArgs& a = p.r;
    const int blk = blockIdx.x, k = threadIdx.x & (kVectors - 1), c0 = k * 8;      // a lane's channels: c0 .. and c0 + 64 ..
    if (blk >= 2 * p.page_blocks) {
        // ---- queries: q_warps warps per token ----
        const int wid = threadIdx.x >> 5, w = (blk - 2 * p.page_blocks) * kWarps + wid, tok = (int)fast_div((uint32_t)w, p.div_warps);
        double omega[2];
        own_omegas<TABLE>(a, omega);
        ptx::grid_dependency_wait();
        ptx::grid_launch_dependents();
        if (tok >= a.num_new) return;
        const int items = a.Hq * kVectors;
        token_heads<T, NORM>(a, p.norm, &s_angles.of_token[wid], tok, 32 * (w - tok * p.q_warps) + (threadIdx.x & 31), 32 * p.q_warps, items, items, items, 0, [&]() -> long {
            int b = 0, hi = a.batch;                          // largest b with new_off[b] <= tok
            while (hi - b > 1) {
                const int mid = (b + hi) >> 1;
                if (lens.new_off[mid] <= tok) b = mid; else hi = mid;
            }
            fill_angles<T, NORM, TABLE>(&s_angles.of_token[wid], a, p.norm, lens.cache_len[b] + tok - lens.new_off[b], omega, true, false);
            return 0;
        });
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
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, slot0 = threadIdx.x / kVectors;      // a lane's slots: slot0 and slot0 + 32
    const bool held = p0 < L;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int page = a.page_table[(long)b * a.max_pages + p0 / kPage8];
    uint8_t* const at = (uint8_t*)(is_v ? a.v_cache : a.k_cache) + (((long)page * a.Hkv + g) * kPage8 + slot0) * D + c0;
    float* scale_at = (is_v ? p.v_scale : p.k_scale) + (long)page * a.Hkv + g;
    auto is_old = [&](int u) { return p0 + slot0 + 32 * u < L; };
    auto is_new = [&](int u) { const int pos = p0 + slot0 + 32 * u; return pos >= L && pos < L + n; };

    uint4 r0[2], r1[2];                                   // a new token's 16 numbers, or an earlier one's 16 codes
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        r0[u] = r1[u] = make_uint4(0u, 0u, 0u, 0u);
        if (is_new(u)) {
            const long tok = off + p0 + slot0 + 32 * u - L;
            const T* src = (is_v ? (const T*)a.v_new + tok * a.v_stride : (const T*)a.k_new + tok * a.k_stride) + (long)g * D + c0;
            r0[u] = *reinterpret_cast<const uint4*>(src);
            r1[u] = *reinterpret_cast<const uint4*>(src + half);
        } else if (is_old(u)) {
            const uint2 lo = *reinterpret_cast<const uint2*>(at + 32 * u * D), hi8 = *reinterpret_cast<const uint2*>(at + 32 * u * D + half);
            r0[u] = make_uint4(lo.x, lo.y, hi8.x, hi8.y);
        }
    }
    const float old_scale = held ? *scale_at : 0.f;
    uint64_t x[2][2][4];                                  // the numbers to store, in pairs
    float w[2][2] = {{1.f, 1.f}, {1.f, 1.f}};             // keys: the weights of channels lane, lane + 64, then lane + 32, lane + 96
    if (NORM && !is_v)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i & 1][i >> 1] = weight_of<T>(p.norm.k_weight, lane + 32 * i);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (is_v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[u][0][i] = pair_of<T>(r0[u], i);
                x[u][1][i] = pair_of<T>(r1[u], i);
            }
            continue;
        }
        // the angles of the warp's four tokens (an angle serves one pair of this head)
        const int first = p0 + 32 * u + 4 * wid;          // position of the first
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = (lane + 32 * i) & (half - 1), pos = first + i / 2;
            if (pos >= L && pos < L + n)
                s_angles.of_slots[wid][i / 2].put(j, TABLE ? a.table[(long)(pos - a.table_first) * half + j] : rope_cos_sin(pos, j, D, a.log2_theta), w[i & 1][0], w[i & 1][1]);
        }
        __syncwarp();
        const float inv = NORM ? NormFactor<T>::of(r0[u], r1[u], 3, D, p.norm.eps) : 1.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) norm_turn_pair(s_angles.of_slots[wid][slot0 & 3], k, i, inv, r0[u], r1[u], x[u][0][i], x[u][1][i]);
    }
    // the page's maximum; infinities and NaN do not count (an infinity becomes the largest code, NaN a NaN code)
    float most = 0.f;
    auto meet = [&](auto size) {
        most = 0.f;
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (is_new(u)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float lo, hi;
                    ptx::unpack2(x[u][i >> 2][i & 3], lo, hi);
                    most = ptx::max3(most, size(lo), size(hi));
                }
            }
    };
    meet([](float v) { return fabsf(v); });               // (the maximum of a number and NaN is the number)
    if (most == INFINITY) meet([](float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.f; });
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
    if (lane == 0) s_most[wid] = most;
    __syncthreads();
    most = s_most[lane & (kWarps - 1)];
#pragma unroll
    for (int s = kWarps / 2; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
    const float need = exp2_int(scale_exponent8(most)), scale = held && old_scale > need ? old_scale : need;
    const bool grew = held && scale > old_scale;
    const float down = 1.f / scale;                       // powers of two: exact
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        uint2* const to = reinterpret_cast<uint2*>(at + 32 * u * D);
        if (is_old(u)) {
            if (!grew) continue;
            float f[16];
            floats4(r0[u].x, f); floats4(r0[u].y, f + 4); floats4(r0[u].z, f + 8); floats4(r0[u].w, f + 12);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[u][i >> 2][i & 3] = ptx::pack2(f[2 * i], f[2 * i + 1]);
            to[0] = codes8(x[u][0], old_scale * down);
            to[half / 8] = codes8(x[u][1], old_scale * down);
        } else if (is_new(u)) {
            to[0] = codes8(x[u][0], down);
            to[half / 8] = codes8(x[u][1], down);
        } else if (is_v) {
            to[0] = to[half / 8] = make_uint2(0u, 0u);    // behind the last token: nothing that could be NaN
        }
    }
    if (threadIdx.x == 0 && (!held || grew)) *scale_at = scale;
}

// The batch's pages as bf16, exactly: page i of an episode goes to page first + i of the copy, whose table says so.  Each code
// is read once, and the copy is what the tensor-core kernel of the bf16 cache reads.  Bound: HBM, at the copy rate (100 K keys of 4 heads, 464 MB,
// 72.5 us = 6.4 TB/s; with 16 codes a lane, whose stores left every second 16 bytes to the next one, 88).
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
    const uint2* src = reinterpret_cast<const uint2*>((is_v ? a.v_pool : a.k_pool) + from * (kPage8 * 128));
    uint4* dst = reinterpret_cast<uint4*>((is_v ? a.v_out : a.k_out) + to * (kPage8 * 128));
    const float scale = (is_v ? a.v_scale : a.k_scale)[from];
    uint2 c[4];                                           // eight codes a lane, so that a warp's 16-byte stores are neighbours
#pragma unroll
    for (int r = 0; r < 4; ++r) c[r] = src[threadIdx.x + 256 * r];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        float x[8];
        floats4(c[r].x, x); floats4(c[r].y, x + 4);
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = ptx::pack_bf16x2(x[2 * k] * scale, x[2 * k + 1] * scale);
        dst[threadIdx.x + 256 * r] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

}  // namespace evln
