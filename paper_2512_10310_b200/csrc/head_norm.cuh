// Norms of queries and keys for each head, with the rotation and the append in the same pass.
//
//     y = w * x / sqrt(mean(x^2) + eps)       over the D channels of a head, queries and keys
//
// then the rotation of Sec. 3.2 at the token's position and the stores of rope_append.cuh.  A head vector is 2^s lanes of
// one warp, a pair of 16-byte vectors (channels j.. and j + D/2..) each: the sum of squares is V packed FMAs and s
// shuffles, and the pair is what the rotation wants.  Everything after the load is in floats (two channels an instruction; fp32: in double, as the
// rotation without norms) and rounded once, to the storage type: there is no rounding between norm and rotation, as there is where they are two passes.
// A warp serves one token: it fills the token's angles, the weights multiplied into them, into its own corner of shared memory, then takes 32 work items
// after the other, so that no warp waits for another one and the angles' cost is shared.  As many warps per token as are resident together: a second
// wave costs more than a longer loop (392 tokens of 28 + 8 heads: 9 warps each 4.1 us, 10 warps and two waves 6.2).
// Bound: for few tokens latency (1.7 us for one), for many HBM: 3136 tokens, 58 MB, 13.9 us = 4.2 TB/s, where the same bytes take 10.4 us in an
// elementwise pass.  (A block per token with a thread per item issued 2.5 times the instructions and took 19.8 us, blocks of two tokens 17.5; weights
// multiplied to the numbers instead of to the angles 15.2, and 1.5 for a token.)
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

// A block: four warps (of eight, the first of few tokens started later: 1.9 us for a token, 1.5).  Seven blocks an SM leave a thread 72 registers, which the
// loop fits (392 tokens 4.2 us, 4.3 with six blocks, 3136 13.9 with both; eight blocks and 64 registers 15.8: the compiler puts some of it aside).
// In fp32 a thread holds doubles: four blocks an SM.  (28/4 heads: a token 1.7 us, 392 tokens 5.6, 3136 33.7, in floats 1.6, 4.8 and 23.9 with errors of
// 700 roundings where the products cancel: conversions to double and back bind.)
constexpr int kNormWarps = 4;
template <typename T> constexpr int kNormBlocks = sizeof(T) == 4 ? 4 : 7;

struct NormArgs {
    const void* q_weight;    // [D] of the tokens' type, or null: ones
    const void* k_weight;
    float eps;
};

// elements 2 i, 2 i + 1 of 16 bytes of T, as a pair of floats for the packed instructions, and back
template <typename T>
__device__ __forceinline__ uint64_t pair_of(const uint4& raw, int i)
{
    const T* e = reinterpret_cast<const T*>(&raw);
    return ptx::pack2(to_float(e[2 * i]), to_float(e[2 * i + 1]));
}
template <typename T>
__device__ __forceinline__ void set_pair(uint4& raw, int i, uint64_t v)
{
    float x, y;
    ptx::unpack2(v, x, y);
    T* e = reinterpret_cast<T*>(&raw);
    from_float(x, e[2 * i]);
    from_float(y, e[2 * i + 1]);
}
template <>
__device__ __forceinline__ void set_pair<__nv_bfloat16>(uint4& raw, int i, uint64_t v)
{
    float x, y;
    ptx::unpack2(v, x, y);
    reinterpret_cast<uint32_t*>(&raw)[i] = ptx::pack_bf16x2(x, y);
}

// 1 / sqrt(mean square + eps) of a head vector that 2^shift neighbouring lanes hold, lo and hi each (all lanes of the warp call this).  D: 2^n.
template <typename T> struct NormFactor;
template <> struct NormFactor<__nv_bfloat16> {
    typedef float F;
    static __device__ __forceinline__ F of(const uint4& lo, const uint4& hi, int shift, int D, float eps)
    {
        uint64_t ss2 = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint64_t x = pair_of<__nv_bfloat16>(lo, i), y = pair_of<__nv_bfloat16>(hi, i);
            ss2 = ptx::fma2(x, x, ptx::fma2(y, y, ss2));
        }
        float ss, other;
        ptx::unpack2(ss2, ss, other);
        ss += other;
        for (int s = 0; s < shift; ++s) ss += __shfl_xor_sync(0xffffffffu, ss, 1 << s);
        return rsqrtf(fmaf(ss, 1.f / (float)D, eps));
    }
};
template <> struct NormFactor<float> {
    typedef double F;
    static __device__ __forceinline__ F of(const uint4& lo, const uint4& hi, int shift, int D, float eps)
    {
        const float* x = reinterpret_cast<const float*>(&lo);
        const float* y = reinterpret_cast<const float*>(&hi);
        double ss = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) ss = fma((double)x[i], (double)x[i], fma((double)y[i], (double)y[i], ss));
        for (int s = 0; s < shift; ++s) ss += __shfl_xor_sync(0xffffffffu, ss, 1 << s);
        return rsqrt(fma(ss, 1.0 / (double)D, (double)eps));
    }
};

// A token's D/2 angles in shared memory.  NORM: with the weights w of a head's channels j and j + D/2 in them, (c w_j, -s w_j'; c w_j', s w_j), bf16 for
// two channels side by side; the vectors of a head (eight channels, fp32 four) 144 bytes apart, so that its lanes start in different banks.  Else as the
// rotation of a stored number wants them.
template <typename T, bool NORM> struct TokenAngles;
template <> struct TokenAngles<float, true> {
    double2 at[144];
    static __device__ __forceinline__ int place(int j) { return 9 * (j >> 2) + 2 * (j & 3); }
    __device__ __forceinline__ void put(int j, const double2& cs, float lo, float hi)
    {
        double2* to = at + place(j);
        to[0] = make_double2(cs.x * lo, -(cs.y * hi));
        to[1] = make_double2(cs.x * hi, cs.y * lo);
    }
};
template <> struct TokenAngles<__nv_bfloat16, true> {
    float4 at[72];
    static __device__ __forceinline__ int place(int pair) { return 9 * (pair >> 2) + 2 * (pair & 3); }
    __device__ __forceinline__ void put(int j, const double2& cs, float lo, float hi)
    {
        float* to = reinterpret_cast<float*>(at + place(j >> 1)) + (j & 1);
        const float c = (float)cs.x, s = (float)cs.y;
        to[0] = c * lo;
        to[2] = -(s * hi);
        to[4] = c * hi;
        to[6] = s * lo;
    }
};
template <typename T> struct TokenAngles<T, false> {
    typename Rotation<T>::Angle at[Rotation<T>::kAngles];
    __device__ __forceinline__ void put(int j, const double2& cs) { Rotation<T>::put(at, j, cs); }
};
template <typename T>
__device__ __forceinline__ float weight_of(const void* weight, int channel)
{
    return weight ? to_float(reinterpret_cast<const T*>(weight)[channel]) : 1.f;
}

// Channels 2 i, 2 i + 1 of a head's vectors lo, hi (vector k of the half), times inv and the weights, turned.
__device__ __forceinline__ void norm_turn_pair(const TokenAngles<__nv_bfloat16, true>& angles, int k, int i, float inv, const uint4& lo, const uint4& hi,
                                               uint64_t& out_lo, uint64_t& out_hi)
{
    typedef __nv_bfloat16 T;
    const uint64_t inv2 = ptx::pack2(inv, inv), x = ptx::mul2(pair_of<T>(lo, i), inv2), y = ptx::mul2(pair_of<T>(hi, i), inv2);
    const float4* a = angles.at + TokenAngles<T, true>::place(4 * k + i);
    const float4 f = a[0], g = a[1];
    out_lo = ptx::fma2(x, ptx::pack2(f.x, f.y), ptx::mul2(y, ptx::pack2(f.z, f.w)));
    out_hi = ptx::fma2(y, ptx::pack2(g.x, g.y), ptx::mul2(x, ptx::pack2(g.z, g.w)));
}
__device__ __forceinline__ void norm_turn_pair(const TokenAngles<float, true>& angles, int k, int i, double inv, const uint4& lo, const uint4& hi,
                                               uint64_t& out_lo, uint64_t& out_hi)
{
    float to_lo[2], to_hi[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const double x = (double)reinterpret_cast<const float*>(&lo)[2 * i + e] * inv, y = (double)reinterpret_cast<const float*>(&hi)[2 * i + e] * inv;
        const double2* a = angles.at + TokenAngles<float, true>::place(4 * k + 2 * i + e);
        const double2 f = a[0], g = a[1];
        to_lo[e] = (float)fma(x, f.x, y * f.y);
        to_hi[e] = (float)fma(y, g.x, x * g.y);
    }
    out_lo = ptx::pack2(to_lo[0], to_lo[1]);
    out_hi = ptx::pack2(to_hi[0], to_hi[1]);
}

// The heads of a token, by the lanes of one or several warps: work items it, it + step, ... of its items (pairs of vectors of query heads, of key
// heads from q_items on, vectors of value heads from qk_items on; step is a multiple of 32, so a lane's place k in a head stays).  prepare() fills
// the angles (NORM: two sets, with the queries' weights and with the keys'), while the first item's vectors are on their way, and returns the token's row in the cache; the next item's are requested
// before an item is worked on.  All lanes of the warp call this.
template <typename T, bool NORM, typename F>
__device__ __forceinline__ void token_heads(const RopeArgs& a, const NormArgs& nrm, const TokenAngles<T, NORM>* angles, int tok, int it, int step, int q_items,
                                            int qk_items, int items, long kv_rows, F&& prepare)
{
    constexpr int V = VecTraits<T>::kVec;
    const int D = a.D, half = D / 2, vph = a.vph_shift, k = it & ((1 << vph) - 1), lane = threadIdx.x & 31;
    const T* q = (const T*)a.q_new + tok * a.q_stride + k * V;
    const T* kk = (const T*)a.k_new + tok * a.k_stride + k * V;
    const T* v = (const T*)a.v_new + tok * a.v_stride;
    auto load = [&](int i, uint4& r0, uint4& r1) {
        r0 = r1 = make_uint4(0u, 0u, 0u, 0u);
        if (i < qk_items) {
            const T* src = (i < q_items ? q : kk) + ((i < q_items ? i : i - q_items) >> vph) * D;
            r0 = *reinterpret_cast<const uint4*>(src);
            r1 = *reinterpret_cast<const uint4*>(src + half);
        } else if (i < items) {
            r0 = *reinterpret_cast<const uint4*>(v + (i - qk_items) * V);
        }
    };
    uint4 n0, n1;
    load(it, n0, n1);
    const long row = prepare();
    T* q_rot = (T*)a.q_rot + (long)tok * a.G * D + k * V;
    T* k_to = (T*)a.k_cache + row * D + k * V;
    T* v_to = (T*)a.v_cache + row * D;
#pragma unroll 1
    for (; it - lane < items; it += step) {
        const uint4 r0 = n0, r1 = n1;
        load(it + step, n0, n1);                   // (two ahead: 16.0 us for 3136 tokens, one 15.0)
        if (it - lane < qk_items) {                // (some lane of the warp)
            const bool is_q = it < q_items;
            uint4 y0, y1;
            if constexpr (NORM) {
                const typename NormFactor<T>::F inv = NormFactor<T>::of(r0, r1, vph, D, nrm.eps);
#pragma unroll
                for (int i = 0; i < V / 2; ++i) {
                    uint64_t lo, hi;
                    norm_turn_pair(angles[is_q ? 0 : 1], k, i, inv, r0, r1, lo, hi);
                    set_pair<T>(y0, i, lo);
                    set_pair<T>(y1, i, hi);
                }
            } else {
                Rotation<T>::turn(angles->at, k, r0, r1, y0, y1);
            }
            if (it < qk_items) {
                const int h = (is_q ? it : it - q_items) >> vph, g = (int)fast_div((uint32_t)h, a.div_g);
                T* dst = is_q ? q_rot + ((long)g * (a.num_new - 1) * a.G + h) * D : k_to + h * kv_rows * D;
                *reinterpret_cast<uint4*>(dst) = y0;
                *reinterpret_cast<uint4*>(dst + half) = y1;
            }
        }
        if (it >= qk_items && it < items) {
            const int e = it - qk_items;
            *reinterpret_cast<uint4*>(v_to + (e >> (vph + 1)) * kv_rows * D + (e & ((2 << vph) - 1)) * V) = r0;
        }
    }
}

// Fills a token's angles by the lanes of a warp (the sets that it needs); omega: of angle lane and, D = 128, lane + 32 (without a table).
template <typename T, bool NORM, bool TABLE>
__device__ __forceinline__ void fill_angles(TokenAngles<T, NORM>* s, const RopeArgs& a, const NormArgs& nrm, int pos, const double (&omega)[2], bool for_q, bool for_k)
{
    const int half = a.D / 2, lane = threadIdx.x & 31, last = half - 1;         // (a lane without a second angle reads another one's)
    double2 cs[2];
    float wq[2][2], wk[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (TABLE) cs[i] = a.table[(long)(pos - a.table_first) * half + min(lane + 32 * i, last)];
    if (NORM) {                                    // in flight together with the table's
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int channel = min(lane + 32 * (i & 1), last) + half * (i >> 1);
            if (for_q) wq[i & 1][i >> 1] = weight_of<T>(nrm.q_weight, channel);
            if (for_k) wk[i & 1][i >> 1] = weight_of<T>(nrm.k_weight, channel);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int j = lane + 32 * i;
        if (j >= half) break;
        if (!TABLE) cs[i] = rope_cos_sin_at(pos, omega[i]);
        if constexpr (NORM) {
            if (for_q) s[0].put(j, cs[i], wq[i][0], wq[i][1]);
            if (for_k) s[1].put(j, cs[i], wk[i][0], wk[i][1]);
        } else {
            s->put(j, cs[i]);
        }
    }
    __syncwarp();
}
template <bool TABLE>
__device__ __forceinline__ void own_omegas(const RopeArgs& a, double (&omega)[2])
{
    const int lane = threadIdx.x & 31;
    omega[0] = omega[1] = 0.0;
    if (!TABLE) {
        omega[0] = rope_omega(lane, a.D, a.log2_theta);
        if (a.D > 64) omega[1] = rope_omega(lane + 32, a.D, a.log2_theta);
    }
}

// token_warps warps per new token, each with every token_warps-th 32 of its items; PAGED: then one per episode and head that clears the value
// slots behind the episode's last token.
template <typename T, bool PAGED, bool TABLE, typename LensT>
__global__ void __launch_bounds__(32 * kNormWarps, kNormBlocks<T>)
norm_append_kernel(const RopeArgs a, const NormArgs nrm, int token_warps, FastDiv div_warps, const __grid_constant__ LensT lens)
{
    constexpr int V = VecTraits<T>::kVec;
    __shared__ __align__(16) TokenAngles<T, true> s_angles[kNormWarps][2];
    const int D = a.D, vph = a.vph_shift, wid = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int w = blockIdx.x * kNormWarps + wid, tok = (int)fast_div((uint32_t)w, div_warps), part = w - tok * token_warps;
    if (tok >= a.num_new) {
        const int at = w - a.num_new * token_warps, b = at / a.Hkv, g = at - b * a.Hkv;
        ptx::grid_dependency_wait();
        ptx::grid_launch_dependents();
        if (!PAGED || b >= a.batch) return;
        const int len = lens.cache_len[b] + lens.new_off[b + 1] - lens.new_off[b], used = len & (a.page_size - 1);
        if (lens.new_off[b + 1] == lens.new_off[b] || used == 0) return;
        const long row = ((long)a.page_table[(long)b * a.max_pages + (len >> a.page_shift)] * a.Hkv + g) * a.page_size + used;
        uint4* dst = reinterpret_cast<uint4*>((T*)a.v_cache + row * D);
        for (int it = lane; it < (a.page_size - used) * (D / V); it += 32) dst[it] = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    double omega[2];
    own_omegas<TABLE>(a, omega);
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int q_items = a.Hq << vph, qk_items = q_items + (a.Hkv << vph), items = qk_items + (a.Hkv << (vph + 1));
    token_heads<T, true>(a, nrm, s_angles[wid], tok, 32 * part + lane, 32 * token_warps, q_items, qk_items, items, PAGED ? a.page_size : a.cache_cap, [&]() -> long {
        int b = 0;
        if (PAGED) {
            int hi = a.batch;                     // largest b with new_off[b] <= tok
            while (hi - b > 1) {
                const int mid = (b + hi) >> 1;
                if (lens.new_off[mid] <= tok) b = mid; else hi = mid;
            }
        }
        const int pos = PAGED ? lens.cache_len[b] + tok - lens.new_off[b] : a.cache_len + tok;
        const long row = PAGED ? (long)a.page_table[(long)b * a.max_pages + (pos >> a.page_shift)] * a.Hkv * a.page_size + (pos & (a.page_size - 1)) : pos;
        const int first = 32 * part, step = 32 * token_warps;     // (several rounds: the keys' come in one of them)
        if (first < qk_items) fill_angles<T, true, TABLE>(s_angles[wid], a, nrm, pos, omega, first < q_items, first + 32 > q_items || first + step < qk_items);
        return row;
    });
}

}  // namespace evln
