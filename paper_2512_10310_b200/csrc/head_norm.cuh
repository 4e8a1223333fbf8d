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

// Norm of a head vector that 2^shift neighbouring lanes hold (all lanes of the warp call this; `w_lo`, `w_hi`: the lane's
// weights, null pointers for ones).
template <typename T, int V>
__device__ __forceinline__ void norm_head(float (&lo)[V], float (&hi)[V], int shift, int D, float eps, const uint4* w_lo, const uint4* w_hi)
{
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) ss = fmaf(lo[i], lo[i], fmaf(hi[i], hi[i], ss));
    for (int s = 0; s < shift; ++s) ss += __shfl_xor_sync(0xffffffffu, ss, 1 << s);
    const float inv = 1.f / sqrtf(ss / (float)D + eps);
    float w[V];
    if (w_lo) to_floats<T, V>(*w_lo, w);
#pragma unroll
    for (int i = 0; i < V; ++i) lo[i] = w_lo ? lo[i] * inv * w[i] : lo[i] * inv;
    if (w_hi) to_floats<T, V>(*w_hi, w);
#pragma unroll
    for (int i = 0; i < V; ++i) hi[i] = w_hi ? hi[i] * inv * w[i] : hi[i] * inv;
}

// (cos, sin) of a token's D/2 angles in shared memory, as floats: eight to 80 bytes, so that the lanes of a head start in
// different banks.
constexpr int kFloatAngles = 80;
__device__ __forceinline__ int angle_place(int j) { return (j >> 3) * 10 + (j & 7); }
template <int V>
__device__ __forceinline__ void turn_floats(const float2* s, int j0, float (&lo)[V], float (&hi)[V])
{
    float2 a[V];
    const float4* from = reinterpret_cast<const float4*>(s + angle_place(j0));
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float4 v = from[i >> 1];
        a[i] = make_float2(v.x, v.y);
        a[i + 1] = make_float2(v.z, v.w);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float x = lo[i], y = hi[i];
        lo[i] = fmaf(x, a[i].x, -(y * a[i].y));
        hi[i] = fmaf(y, a[i].x, x * a[i].y);
    }
}

// Queries (and, KV, keys and values) of one token: the whole block, gridDim-free (part of parts).  NORM: with the norms.
// dst_q(h): where query head h goes; dst_kv(k, h): key (or value) head h.  All lanes of a warp run the same number of rounds.
template <typename T, bool NORM, bool KV, typename DstQ, typename DstK, typename DstV, typename Angle>
__device__ __forceinline__ void norm_token(const RopeArgs& a, const NormArgs& nrm, int src_tok, int part, int parts, DstQ&& dst_q, DstK&& dst_k, DstV&& dst_v,
                                           Angle&& angle)
{
    constexpr int V = VecTraits<T>::kVec;
    __shared__ __align__(16) float2 s_angle[kFloatAngles];
    __shared__ typename Rotation<T>::Angle s_exact[NORM ? 1 : Rotation<T>::kAngles];
    const int D = a.D, half = D / 2, vph = a.vph_shift;
    const int q_items = a.Hq << vph, k_items = KV ? a.Hkv << vph : 0, v_items = KV ? a.Hkv << (vph + 1) : 0;
    const int items = q_items + k_items + v_items, step = parts * (int)blockDim.x;
    const int j0 = ((int)threadIdx.x & ((1 << vph) - 1)) * V;        // (blocks are whole warps, so a thread's place in a head stays)

    auto load = [&](int it, uint4& r0, uint4& r1, uint4& w0, uint4& w1) {
        r0 = r1 = w0 = w1 = make_uint4(0u, 0u, 0u, 0u);
        if (it < q_items + k_items) {
            const bool is_q = it < q_items;
            const int h = (is_q ? it : it - q_items) >> vph;
            const T* src = (is_q ? (const T*)a.q_new + src_tok * a.q_stride : (const T*)a.k_new + src_tok * a.k_stride) + (long)h * D;
            r0 = *reinterpret_cast<const uint4*>(src + j0);
            r1 = *reinterpret_cast<const uint4*>(src + j0 + half);
            const T* w = (const T*)(is_q ? nrm.q_weight : nrm.k_weight);
            if (NORM && w) {
                w0 = *reinterpret_cast<const uint4*>(w + j0);
                w1 = *reinterpret_cast<const uint4*>(w + j0 + half);
            }
        } else if (it < items) {
            const int e = it - q_items - k_items, h = e >> (vph + 1), d0 = (e & ((2 << vph) - 1)) * V;
            r0 = *reinterpret_cast<const uint4*>((const T*)a.v_new + src_tok * a.v_stride + (long)h * D + d0);
        }
    };
    auto finish = [&](int it, const uint4& r0, const uint4& r1, const uint4& w0, const uint4& w1) {
        const bool is_q = it < q_items, turns = it < q_items + k_items;
        uint4 y0 = r0, y1 = r1;
        if (NORM) {
            float lo[V], hi[V];
            to_floats<T, V>(r0, lo);
            to_floats<T, V>(r1, hi);
            const bool weighed = (is_q ? nrm.q_weight : nrm.k_weight) != nullptr;
            norm_head<T, V>(lo, hi, vph, D, nrm.eps, weighed ? &w0 : nullptr, weighed ? &w1 : nullptr);
            turn_floats<V>(s_angle, j0, lo, hi);
            if (turns) {
                y0 = from_floats<T, V>(lo);
                y1 = from_floats<T, V>(hi);
            }
        } else if (turns) {
            Rotation<T>::turn(s_exact, j0 / V, r0, r1, y0, y1);
        }
        if (turns) {
            T* dst = is_q ? dst_q(it >> vph) : dst_k((it - q_items) >> vph);
            *reinterpret_cast<uint4*>(dst + j0) = y0;
            *reinterpret_cast<uint4*>(dst + j0 + half) = y1;
        } else if (it < items) {
            const int e = it - q_items - k_items;
            *reinterpret_cast<uint4*>(dst_v(e >> (vph + 1)) + (e & ((2 << vph) - 1)) * V) = y0;
        }
    };
    uint4 r0, r1, w0, w1;
    int it = part * (int)blockDim.x + (int)threadIdx.x;
    load(it, r0, r1, w0, w1);                      // in flight while the angles arrive
    if ((int)threadIdx.x < half) {
        const double2 cs = angle((int)threadIdx.x);
        if (NORM) s_angle[angle_place((int)threadIdx.x)] = make_float2((float)cs.x, (float)cs.y);
        else Rotation<T>::put(s_exact, (int)threadIdx.x, cs);
    }
    __syncthreads();
    for (;;) {
        finish(it, r0, r1, w0, w1);
        it += step;
        if (it - (int)(threadIdx.x & 31) >= items) break;
        load(it, r0, r1, w0, w1);
    }
}

// One block per new token (FEW: and part of its work items); PAGED: then one per episode that clears the value slots behind
// its last token.
template <typename T, bool PAGED, typename LensT>
__global__ void __launch_bounds__(kRopeThreadsMax, PAGED ? 2 : 1)
norm_append_kernel(const RopeArgs a, const NormArgs nrm, const __grid_constant__ LensT lens)
{
    constexpr int V = VecTraits<T>::kVec;
    const int D = a.D;
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
    const double omega = !a.table && (int)threadIdx.x < D / 2 ? rope_omega(threadIdx.x, D, a.log2_theta) : 0.0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const long row = PAGED ? (long)a.page_table[(long)b * a.max_pages + (pos >> a.page_shift)] * a.Hkv * a.page_size + (pos & (a.page_size - 1)) : pos;
    const long kv_rows = PAGED ? a.page_size : a.cache_cap;
    norm_token<T, true, true>(
        a, nrm, tok, blockIdx.y, gridDim.y,
        [&](int h) -> T* {
            const int g = (int)fast_div((uint32_t)h, a.div_g);
            return (T*)a.q_rot + ((long)g * a.num_new * a.G + (long)tok * a.G + (h - g * a.G)) * D;
        },
        [&](int g) -> T* { return (T*)a.k_cache + (g * kv_rows + row) * D; }, [&](int g) -> T* { return (T*)a.v_cache + (g * kv_rows + row) * D; },
        [&](int j) -> double2 { return a.table ? a.table[(long)(pos - a.table_first) * (D / 2) + j] : rope_cos_sin_at(pos, omega); });
}

}  // namespace evln
