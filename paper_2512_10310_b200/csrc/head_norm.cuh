// Norms of queries and keys for each head, with the rotation and the append in the same pass.
//
//     y = w * x / sqrt(mean(x^2) + eps)       over the D channels of a head, queries and keys
//
// then the rotation of Sec. 3.2 at the token's position and the stores of rope_append.cuh.  A head vector is 2^s lanes of
// one warp, a pair of 16-byte vectors (channels j.. and j + D/2..) each: the sum of squares is V FMAs a half and s
// shuffles, and the pair is what the rotation wants.  Everything after the load is in floats and rounded once, to the
// storage type: there is no rounding between norm and rotation, as there is where they are two passes.
// Bound: as rope_append.cuh (latency for few tokens, then instructions and HBM); a norm adds one dependent chain of
// shuffles and a square root to a token.
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

struct NormArgs {
    const void* q_weight;    // [D] of the tokens' type, or null: ones
    const void* k_weight;
    float eps;
};

// 16 bytes of T as floats and back (one rounding)
template <typename T, int V>
__device__ __forceinline__ void to_floats(const uint4& raw, float (&x)[V])
{
    const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = to_float(e[i]);
}
template <typename T, int V>
__device__ __forceinline__ uint4 from_floats(const float (&x)[V])
{
    uint4 raw;
    T* e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int i = 0; i < V; ++i) from_float(x[i], e[i]);
    return raw;
}
// elements 2 i, 2 i + 1 of 16 bytes
template <typename T>
__device__ __forceinline__ float2 pair_of(const uint4& raw, int i)
{
    const T* e = reinterpret_cast<const T*>(&raw);
    return make_float2(to_float(e[2 * i]), to_float(e[2 * i + 1]));
}
template <typename T>
__device__ __forceinline__ void set_pair(uint4& raw, int i, float x, float y)
{
    T* e = reinterpret_cast<T*>(&raw);
    from_float(x, e[2 * i]);
    from_float(y, e[2 * i + 1]);
}

// 1 / sqrt(mean square + eps) of a head vector that 2^shift neighbouring lanes hold, lo and hi each (all lanes of the warp call this)
template <typename T>
__device__ __forceinline__ float norm_factor(const uint4& lo, const uint4& hi, int shift, int D, float eps)
{
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < VecTraits<T>::kVec / 2; ++i) {
        const float2 x = pair_of<T>(lo, i), y = pair_of<T>(hi, i);
        ss = fmaf(x.x, x.x, fmaf(x.y, x.y, fmaf(y.x, y.x, fmaf(y.y, y.y, ss))));
    }
    for (int s = 0; s < shift; ++s) ss += __shfl_xor_sync(0xffffffffu, ss, 1 << s);
    return 1.f / sqrtf(ss / (float)D + eps);
}

// (cos, sin) of a token's D/2 angles in shared memory.  NORM: as floats, eight to 80 bytes, so that the lanes of a head start in
// different banks; else as the rotation of a stored number wants them.
template <typename T, bool NORM> struct TokenAngles;
template <typename T> struct TokenAngles<T, true> {
    float2 at[80];
    static __device__ __forceinline__ int place(int j) { return (j >> 3) * 10 + (j & 7); }
    __device__ __forceinline__ void put(int j, const double2& cs) { at[place(j)] = make_float2((float)cs.x, (float)cs.y); }
};
template <typename T> struct TokenAngles<T, false> {
    typename Rotation<T>::Angle at[Rotation<T>::kAngles];
    __device__ __forceinline__ void put(int j, const double2& cs) { Rotation<T>::put(at, j, cs); }
};

// A pair of vectors of a head, normed (all lanes of the warp call this) and turned; vector k of the half.  (Elements are taken out of the
// vectors two at a time, and weights come late: with both as floats in registers the kernel needed 80 of them, and 3136 tokens took 27 us.)
template <typename T>
__device__ __forceinline__ void norm_turn(const TokenAngles<T, true>& angles, int k, int shift, int D, float eps, const T* weight, const uint4& lo, const uint4& hi,
                                          uint4& out_lo, uint4& out_hi)
{
    constexpr int V = VecTraits<T>::kVec;
    uint4 w0 = make_uint4(0u, 0u, 0u, 0u), w1 = w0;
    if (weight) {
        w0 = *reinterpret_cast<const uint4*>(weight + k * V);
        w1 = *reinterpret_cast<const uint4*>(weight + k * V + D / 2);
    }
    const float inv = norm_factor<T>(lo, hi, shift, D, eps);
    const float4* a = reinterpret_cast<const float4*>(angles.at + TokenAngles<T, true>::place(k * V));
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        float2 x = pair_of<T>(lo, i), y = pair_of<T>(hi, i);
        x.x *= inv; x.y *= inv; y.x *= inv; y.y *= inv;
        if (weight) {
            const float2 u = pair_of<T>(w0, i), v = pair_of<T>(w1, i);
            x.x *= u.x; x.y *= u.y; y.x *= v.x; y.y *= v.y;
        }
        const float4 cs = a[i];
        set_pair<T>(out_lo, i, fmaf(x.x, cs.x, -(y.x * cs.y)), fmaf(x.y, cs.z, -(y.y * cs.w)));
        set_pair<T>(out_hi, i, fmaf(y.x, cs.x, x.x * cs.y), fmaf(y.y, cs.z, x.y * cs.w));
    }
}

// One block per new token (gridDim.y: and part of its work items); PAGED: then one per episode that clears the value slots behind
// its last token.
template <typename T, bool PAGED, typename LensT>
__global__ void __launch_bounds__(kRopeThreadsMax, 3)
norm_append_kernel(const RopeArgs a, const NormArgs nrm, const __grid_constant__ LensT lens)
{
    constexpr int V = VecTraits<T>::kVec;
    __shared__ __align__(16) TokenAngles<T, true> s_angles;
    const int D = a.D, half = D / 2, vph = a.vph_shift;
    int b = 0;
    if (PAGED && (int)blockIdx.x >= a.num_new) {
        b = blockIdx.x - a.num_new;
        const int len = lens.cache_len[b] + lens.new_off[b + 1] - lens.new_off[b], used = len & (a.page_size - 1);
        ptx::grid_dependency_wait();
        ptx::grid_launch_dependents();
        if (lens.new_off[b + 1] == lens.new_off[b] || used == 0) return;
        const long row = (long)a.page_table[(long)b * a.max_pages + (len >> a.page_shift)] * a.Hkv * a.page_size + used;
        for (int g = blockIdx.y; g < a.Hkv; g += gridDim.y) {
            uint4* dst = reinterpret_cast<uint4*>((T*)a.v_cache + (row + (long)g * a.page_size) * D);
            for (int it = threadIdx.x; it < (a.page_size - used) * (D / V); it += blockDim.x) dst[it] = make_uint4(0u, 0u, 0u, 0u);
        }
        return;
    }
    const int tok = blockIdx.x;
    if (PAGED) {
        int hi = a.batch;                         // largest b with new_off[b] <= tok
        while (hi - b > 1) {
            const int mid = (b + hi) >> 1;
            if (lens.new_off[mid] <= tok) b = mid; else hi = mid;
        }
    }
    const int pos = PAGED ? lens.cache_len[b] + tok - lens.new_off[b] : a.cache_len + tok;
    // without a table: the thread's frequency, ahead of the wait (launch parameters only)
    const double omega = !a.table && (int)threadIdx.x < half ? rope_omega(threadIdx.x, D, a.log2_theta) : 0.0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    const int q_items = a.Hq << vph, qk_items = q_items + (a.Hkv << vph), items = qk_items + (a.Hkv << (vph + 1)), step = gridDim.y * blockDim.x;
    const int k = (int)threadIdx.x & ((1 << vph) - 1);            // (blocks are whole warps, so a thread's place in a head stays)
    auto load = [&](int it, uint4& r0, uint4& r1) {               // a pair of vectors of a query or key head, or a vector of a value head
        r0 = r1 = make_uint4(0u, 0u, 0u, 0u);
        if (it < qk_items) {
            const bool is_q = it < q_items;
            const T* src = (is_q ? (const T*)a.q_new + tok * a.q_stride : (const T*)a.k_new + tok * a.k_stride) + (long)((is_q ? it : it - q_items) >> vph) * D + k * V;
            r0 = *reinterpret_cast<const uint4*>(src);
            r1 = *reinterpret_cast<const uint4*>(src + half);
        } else if (it < items) {
            r0 = *reinterpret_cast<const uint4*>((const T*)a.v_new + tok * a.v_stride + (long)(it - qk_items) * V);
        }
    };
    uint4 r0, r1;
    int it = blockIdx.y * blockDim.x + threadIdx.x;
    load(it, r0, r1);                              // in flight while the angles arrive
    if ((int)threadIdx.x < half) s_angles.put(threadIdx.x, a.table ? a.table[(long)(pos - a.table_first) * half + threadIdx.x] : rope_cos_sin_at(pos, omega));
    const long row = PAGED ? (long)a.page_table[(long)b * a.max_pages + (pos >> a.page_shift)] * a.Hkv * a.page_size + (pos & (a.page_size - 1)) : pos;
    const long kv_rows = PAGED ? a.page_size : a.cache_cap;
    __syncthreads();
    for (;;) {
        uint4 y0 = r0, y1 = r1;
        const bool is_q = it < q_items;
        if (it - (int)(threadIdx.x & 31) < qk_items)              // (some lane of the warp)
            norm_turn<T>(s_angles, k, vph, D, nrm.eps, (const T*)(is_q ? nrm.q_weight : nrm.k_weight), r0, r1, y0, y1);
        if (it < qk_items) {
            const int h = (is_q ? it : it - q_items) >> vph;
            T* dst;
            if (is_q) {
                const int g = (int)fast_div((uint32_t)h, a.div_g);
                dst = (T*)a.q_rot + ((long)g * a.num_new * a.G + (long)tok * a.G + (h - g * a.G)) * D;
            } else {
                dst = (T*)a.k_cache + (h * kv_rows + row) * D;
            }
            *reinterpret_cast<uint4*>(dst + k * V) = y0;
            *reinterpret_cast<uint4*>(dst + k * V + half) = y1;
        } else if (it < items) {
            const int e = it - qk_items;
            *reinterpret_cast<uint4*>((T*)a.v_cache + ((e >> (vph + 1)) * kv_rows + row) * D + (e & ((2 << vph) - 1)) * V) = r0;
        }
        it += step;
        if (it - (int)(threadIdx.x & 31) >= items) break;
        load(it, r0, r1);
    }
}

}  // namespace evln
