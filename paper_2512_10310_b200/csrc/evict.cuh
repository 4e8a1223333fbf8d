// Eviction: which keys of a kv head to keep, by weight, and the chosen ones laid out anew.
//
// select_keys_kernel: a block per kv head.  The threshold is the m-th largest of the weights in the open range, found digit by
// digit (11, 11 and 10 bits of the float as an ordered integer, a histogram in shared memory each); then one ordered pass
// writes the slots above it, of those equal to it the lowest, and the protected ends.  A thread holds a run of neighbouring slots, so one
// scan over the block's counts gives every slot its place, ascending.
// gather_keys_kernel: a block takes a few working slots for all kv heads: their angles once into shared memory, then every
// head's chosen key (turned as in rope_append.cuh, or copied) and value.
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

struct SelectArgs {
    const float* weights;    // [Hkv, stride]
    int* kept;               // [Hkv, num_kept]
    int stride, num_keys, num_kept;
    int sinks, recent, open; // open: how many of the slots between the ends are kept
    int cached;              // the weights fit the block's shared memory
};

constexpr int kSelectThreads = 1024, kSelectBins = 2048, kSelectCache = 48 * 1024;   // floats held on chip

// floats in order as unsigned integers; -0 as 0, NaN as -infinity
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = x != x ? 0xff800000u : __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Inclusive sums of a pair of counts over the block (all threads), by thread number.
__device__ __forceinline__ int2 block_scan(int2 v, int2* s_warp)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) { v.x += x; v.y += y; }
    }
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int2 w = s_warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, w.x, o), y = __shfl_up_sync(0xffffffffu, w.y, o);
            if (lane >= o) { w.x += x; w.y += y; }
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    if (warp > 0) { v.x += s_warp[warp - 1].x; v.y += s_warp[warp - 1].y; }
    return v;
}

__global__ void __launch_bounds__(kSelectThreads, 1)
select_keys_kernel(const SelectArgs a)
{
    extern __shared__ uint32_t s_key[];                   // [num_keys] where they fit
    __shared__ int s_bin[kSelectBins];
    __shared__ int2 s_warp[32];
    __shared__ int s_digit, s_left;
    const int g = blockIdx.x, tid = threadIdx.x;
    const float* w = a.weights + (long)g * a.stride;
    const int lo = a.sinks, hi = a.num_keys - a.recent;   // the open range
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    auto key = [&](int j) -> uint32_t { return a.cached ? s_key[j] : ordered(w[j]); };
    if (a.cached)
        for (int j = tid; j < a.num_keys; j += kSelectThreads) s_key[j] = ordered(w[j]);
    uint32_t prefix = 0, mask = 0;
    int left = a.open;                                    // still to be found among the keys with this prefix
    if (a.num_kept < a.num_keys && a.open > 0) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < kSelectBins; i += kSelectThreads) s_bin[i] = 0;
            __syncthreads();
            for (int j = lo + tid; j < hi; j += kSelectThreads) {
                const uint32_t k = key(j);
                if ((k & mask) == prefix) atomicAdd(&s_bin[(k >> shift) & ((1 << bits) - 1)], 1);
            }
            __syncthreads();
            // bins from the largest digit down, two a thread: where does the count reach `left`?
            const int d0 = kSelectBins - 1 - 2 * tid, n0 = s_bin[d0], n1 = s_bin[d0 - 1];
            const int upto = block_scan(make_int2(n0 + n1, 0), s_warp).x, before = upto - n0 - n1;
            if (before < left && upto >= left) {
                const bool second = before + n0 < left;
                s_digit = second ? d0 - 1 : d0;
                s_left = left - before - (second ? n0 : 0);
            }
            __syncthreads();
            prefix |= (uint32_t)s_digit << shift;
            mask |= ((1u << bits) - 1u) << shift;
            left = s_left;
            __syncthreads();
        }
    }
    __syncthreads();
    // ---- every thread a run of neighbouring slots (of odd length: the runs start in different banks) ----
    const bool all = a.num_kept == a.num_keys;
    const int run = ((a.num_keys + kSelectThreads - 1) / kSelectThreads) | 1, j0 = min(a.num_keys, tid * run), j1 = min(a.num_keys, j0 + run);
    int2 n = make_int2(0, 0);                             // kept for certain, equal to the threshold
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = key(j);
        const bool end = j < lo || j >= hi || all;
        n.x += end || (a.open > 0 && k > prefix);
        n.y += !end && a.open > 0 && k == prefix;
    }
    int2 at = block_scan(n, s_warp);
    at.x -= n.x;
    at.y -= n.y;
    int* out = a.kept + (long)g * a.num_kept;
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = key(j);
        const bool end = j < lo || j >= hi || all;
        const bool sure = end || (a.open > 0 && k > prefix), equal = !end && a.open > 0 && k == prefix;
        if (sure || (equal && at.y < left)) out[at.x + min(at.y, left)] = j;
        at.x += sure;
        at.y += equal;
    }
}

struct GatherKeysArgs {
    const void* k_src;       // [Hkv, src_cap, D]
    const void* v_src;
    const float* w_src;      // [Hkv, src_cap] or null
    void* k_dst;             // [Hkv, dst_cap, D]
    void* v_dst;
    float* w_dst;            // [Hkv, dst_cap]
    const int* kept;         // [Hkv, num_kept]
    int Hkv, D, src_cap, dst_cap, num_kept, rotate;
    double log2_theta;
    const double2* table;    // optional
    int table_first;
    int vph_shift;           // log2 of the 16-byte vectors per half head vector
};

constexpr int kGatherKeysThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kGatherKeysThreads)
gather_keys_kernel(const GatherKeysArgs a)
{
    constexpr int V = VecTraits<T>::kVec;
    __shared__ __align__(16) typename Rotation<T>::Angle s_angle[8][Rotation<T>::kAngles];
    const int D = a.D, half = D / 2, tid = threadIdx.x;
    const int slots = kGatherKeysThreads / half;          // 4 or 8 working slots a block
    const int p0 = blockIdx.x * slots, here = min(slots, a.num_kept - p0);
    const int vph = a.vph_shift, k_items = 1 << vph, per_head = 3 << vph;      // pairs of a key, vectors of a value
    const double omega = a.rotate && !a.table ? rope_omega(tid % half, D, a.log2_theta) : 0.0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    if (a.rotate) {
        const int p = p0 + tid / half, j = tid % half;
        if (tid / half < here) Rotation<T>::put(s_angle[tid / half], j, a.table ? a.table[(long)(p - a.table_first) * half + j] : rope_cos_sin_at(p, omega));
        __syncthreads();
    }
    const int items = here * a.Hkv * per_head;
    for (int it = tid; it < items; it += kGatherKeysThreads) {
        const int row = it / per_head, e = it - row * per_head;                // row: slot and head, slots side by side
        const int g = row / here, s = row - g * here, p = p0 + s;
        const int from = a.kept[(long)g * a.num_kept + p];
        const bool good = (unsigned)from < (unsigned)a.src_cap;
        const long src = ((long)g * a.src_cap + (good ? from : 0)) * D, dst = ((long)g * a.dst_cap + p) * D;
        const uint4 none = make_uint4(0u, 0u, 0u, 0u);
        if (e < k_items) {
            const T* k = (const T*)a.k_src + src + e * V;
            uint4 lo = good ? *reinterpret_cast<const uint4*>(k) : none, hi = good ? *reinterpret_cast<const uint4*>(k + half) : none;
            if (a.rotate) {
                uint4 x = lo, y = hi;
                Rotation<T>::turn(s_angle[s], e, x, y, lo, hi);
            }
            T* to = (T*)a.k_dst + dst + e * V;
            *reinterpret_cast<uint4*>(to) = lo;
            *reinterpret_cast<uint4*>(to + half) = hi;
            if (e == 0 && a.w_src) a.w_dst[(long)g * a.dst_cap + p] = good ? a.w_src[(long)g * a.src_cap + from] : 0.f;
        } else {
            const int d = (e - k_items) * V;
            *reinterpret_cast<uint4*>((T*)a.v_dst + dst + d) = good ? *reinterpret_cast<const uint4*>((const T*)a.v_src + src + d) : none;
        }
    }
}

}  // namespace evln
