// The rotation of queries and keys (Sec. 3.2), shared by every kernel that turns them: angles of a position and
// the products with a pair of 16-byte vectors.
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"

namespace evln {

// New tokens and where they go: what the append kernels take.
struct RopeArgs {
    const void* q_new;
    const void* k_new;
    const void* v_new;
    void* q_rot;
    void* k_cache;      // contiguous: [Hkv, cap, D]; paged: pool [pages, Hkv, page, D]
    void* v_cache;
    const int* page_table;   // paged only: [batch, max_pages]
    long q_stride, k_stride, v_stride;   // token strides in elements
    int Hq, Hkv, D;
    int cache_len;      // contiguous only
    int num_new;        // contiguous: n; paged: total new tokens
    int cache_cap;      // contiguous only
    int batch, page_size, max_pages;     // paged only
    double log2_theta;
    const double2* table;   // optional: (cos, sin) per (position - table_first, j), [count][D/2]
    int table_first;
    // derived by the host (finish_rope_args): the threads decode their work with shifts and one
    // multiplication instead of integer divisions
    int G;                  // Hq / Hkv
    FastDiv div_g;
    int vph_shift;          // log2 of the 16-byte vectors per half head vector (D/2 / V)
    int page_shift;         // log2(page_size)
};

// A block per token with one thread per work item (in whole warps, at most kRopeThreadsMax): every load of
// the token is in flight at once, and the other blocks of the SM hide its chain.  (Blocks that run through
// several tokens and prefetch the next one's vectors were measured slower, 10.3 against 9.8 us for 2048
// tokens and 19 against 17.6 for 3136 paged ones: what counts is warps, i.e. registers.)
constexpr int kRopeThreadsMax = 448;
constexpr int kRopeFewTokens = 256;      // (64 query heads: 8 tokens 27.2 us a step, 25.7 with two blocks each; 256 tokens 38.7 and 37.3)

// cos/sin of pos * theta^(-2j/D): the one definition the append, gather and table kernels share
__device__ __forceinline__ double rope_omega(int j, int D, double log2_theta)
{
    return exp2(-(2.0 * (double)j / (double)D) * log2_theta);
}
__device__ __forceinline__ double2 rope_cos_sin_at(long pos, double omega)
{
    double s, c;
    // sin/cos(pos * omega) through sincospi: its range reduction is exact and cheap, where a
    // plain sincos of an argument of thousands of radians takes the slow reduction path
    sincospi((double)pos * omega * 0.31830988618379067154, &s, &c);
    return make_double2(c, s);
}
__device__ __forceinline__ double2 rope_cos_sin(long pos, int j, int D, double log2_theta)
{
    return rope_cos_sin_at(pos, rope_omega(j, D, log2_theta));
}

// The rotation itself.  Products and sums are formed with at least 40 bits, then rounded once to float and
// once to the storage dtype (a float product would lose bits exactly where x0*c and x1*s cancel).
//  - float: in double.
//  - bf16: in pairs of floats, two channels per packed instruction.  A double operation and the
//    conversions around it issue at a small fraction of the float rate (32 double operations and 32
//    conversions per vector pair kept an SM at ~7 per cycle), and what bounds the append and gather
//    kernels for thousands of tokens is the instructions they issue.  The angle is split into 16 bits and
//    a float rest (40 bits), so a bf16 value times the first part is an exact float; the two exact products
//    are added with the rounding error recovered (Knuth's two-sum), which the products with the rest join.
// put(): angle j into a shared-memory array of kAngles; turn(): vector k (of a half head) of both halves.
template <typename T> struct Rotation;
template <> struct Rotation<float> {
    typedef double2 Angle;                       // (cos, sin); angle j at j + j / 8 (bank spread)
    static constexpr int kAngles = 72;
    static __device__ __forceinline__ void put(Angle* s, int j, const double2& cs) { s[j + (j >> 3)] = cs; }
    static __device__ __forceinline__ void turn(const Angle* s, int k, const uint4& lo, const uint4& hi, uint4& out_lo, uint4& out_hi)
    {
        const float* x0 = reinterpret_cast<const float*>(&lo);
        const float* x1 = reinterpret_cast<const float*>(&hi);
        float* y0 = reinterpret_cast<float*>(&out_lo);
        float* y1 = reinterpret_cast<float*>(&out_hi);
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int j = 4 * k + v;
            const Angle a = s[j + (j >> 3)];
            y0[v] = (float)((double)x0[v] * a.x - (double)x1[v] * a.y);
            y1[v] = (float)((double)x1[v] * a.x + (double)x0[v] * a.y);
        }
    }
};
template <> struct Rotation<__nv_bfloat16> {
    // a channel pair is two of these: (cos 16 bits of both, rest of both), (sin ..., ...); the pairs of a
    // 16-byte vector take 9 places, so that the vectors of a half head start in different banks
    typedef float4 Angle;
    static constexpr int kAngles = 72;
    static __device__ __forceinline__ int place(int pair) { return 2 * pair + (pair >> 2); }
    static __device__ __forceinline__ void put(Angle* s, int j, const double2& cs)
    {
        const float ch = __uint_as_float(__float_as_uint((float)cs.x) & 0xffffff00u);
        const float sh = __uint_as_float(__float_as_uint((float)cs.y) & 0xffffff00u);
        float* at = reinterpret_cast<float*>(s + place(j >> 1)) + (j & 1);
        at[0] = ch;
        at[2] = (float)(cs.x - (double)ch);
        at[4] = sh;
        at[6] = (float)(cs.y - (double)sh);
    }
    // x * (ch + cl) + z * (sh + sl)
    static __device__ __forceinline__ uint64_t combine(uint64_t x, uint64_t z, uint64_t ch, uint64_t cl, uint64_t sh, uint64_t sl)
    {
        const uint64_t minus = ptx::pack2(-1.f, -1.f);
        const uint64_t p = ptx::mul2(x, ch), q = ptx::mul2(z, sh);
        const uint64_t d = ptx::add2(p, q);
        const uint64_t nb = ptx::fma2(d, minus, p);                     // p - d: minus the part of q that d holds
        const uint64_t err = ptx::add2(ptx::fma2(ptx::add2(d, nb), minus, p), ptx::add2(q, nb));
        float r0, r1;
        ptx::unpack2(ptx::fma2(z, sl, ptx::fma2(x, cl, err)), r0, r1);
        // (an infinite or undefined d stays what it is: its rest is undefined, and min() drops that)
        return ptx::add2(d, ptx::pack2(fminf(r0, 3.0e38f), fminf(r1, 3.0e38f)));
    }
    // a channel pair: words of the lower and the upper half
    static __device__ __forceinline__ void turn_pair(const Angle& c, const Angle& s, uint32_t lo, uint32_t hi, uint32_t& out_lo,
                                                     uint32_t& out_hi)
    {
        const uint32_t nhi = hi ^ 0x80008000u;
        const uint64_t x0 = ptx::pack2(__uint_as_float(lo << 16), __uint_as_float(lo & 0xffff0000u));
        const uint64_t x1 = ptx::pack2(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u));
        const uint64_t n1 = ptx::pack2(__uint_as_float(nhi << 16), __uint_as_float(nhi & 0xffff0000u));
        const uint64_t ch = ptx::pack2(c.x, c.y), cl = ptx::pack2(c.z, c.w), sh = ptx::pack2(s.x, s.y), sl = ptx::pack2(s.z, s.w);
        float a, b;
        ptx::unpack2(combine(x0, n1, ch, cl, sh, sl), a, b);
        out_lo = ptx::pack_bf16x2(a, b);
        ptx::unpack2(combine(x1, x0, ch, cl, sh, sl), a, b);
        out_hi = ptx::pack_bf16x2(a, b);
    }
    static __device__ __forceinline__ void turn(const Angle* s, int k, const uint4& lo, const uint4& hi, uint4& out_lo, uint4& out_hi)
    {
        const Angle* a = s + place(4 * k);
        const uint32_t x0[4] = {lo.x, lo.y, lo.z, lo.w}, x1[4] = {hi.x, hi.y, hi.z, hi.w};
        uint32_t y0[4], y1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) turn_pair(a[2 * i], a[2 * i + 1], x0[i], x1[i], y0[i], y1[i]);
        out_lo = make_uint4(y0[0], y0[1], y0[2], y0[3]);
        out_hi = make_uint4(y1[0], y1[1], y1[2], y1[3]);
    }
};

}  // namespace evln
