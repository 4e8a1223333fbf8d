// Step attention over a paged cache in 8 bits (cache8.cuh), for up to a few hundred query rows per kv head.
//
//     out = softmax(scale * q K^T) V,    K, V = code * scale of its page,    a query sees the keys up to its own position
//
// Bound: reading every code once; a code is one byte, so an SM takes 23 elements a cycle at the copy rate and turning
// them into operands has to keep up with that.  Hence mma.sync on halves: two codes become two halves in ONE instruction
// (cvt f16x2 <- e4m3x2, exact), and everything else that the format asks for is free or done once per row:
//  - the query row is scaled by a power of two into the range of halves (exact above 2^-29 of the row's maximum), and that
//    factor, the page's key scale and the softmax scale are one factor on the scores;
//  - the page's value scale, a power of two, goes into the exponent of the probabilities: p' = 2^(s - m + log2(scale / r)),
//    r the largest value scale that the warp has met; the row sums take it out again.  (Probabilities are rounded to halves:
//    2^-11, finer than bf16.)
// The operands come out of ldmatrix as bytes: a key's 16 bytes are a k-step of the score product (four channels a lane, the
// queries are laid out the same way), and a transposed load of byte PAIRS gives two keys of two neighbouring channels,
// which one byte permutation parts into the operands of two column tiles.
//
// A block: 8 warps, RG row groups x KG key groups, each warp 16 MT rows.  A key group has a ring of its own of 32-key stages
// (4 KB keys + 4 KB values, TMA, 128-byte swizzle), which one warp of it refills itself as it goes: warps of different key
// groups never wait for each other before the block's merge.  The lanes of a warp look 32 stages ahead for page numbers and
// scales (a lane each).  A block per SM, each with an equal share of the batch's stages, walked unit by unit (unit: episode, kv
// head, tile of rows); a unit that the shares cut leaves normalised parts, which merge8_kernel joins.
// A row's reference m follows its maximum only when that is 2^8 above it, so outputs are rarely scaled anew.
#pragma once

#include <cuda.h>

#include "cache8.cuh"
#include "common.cuh"
#include "ptx_sm100.cuh"
#include "tc_common.cuh"

namespace evln {

constexpr int kA8Keys = 32, kA8StageBytes = 2 * kA8Keys * 128, kA8Warps = 8, kA8Threads = 32 * kA8Warps;
constexpr int kA8QStride = 288;                       // bytes between query rows in shared memory (256 + a bank spread)
constexpr int kA8OStride = 132;                       // floats between rows of the merge buffers
constexpr float kA8Headroom = 8.f, kA8Lift = 6.f;     // p' <= 2^(headroom + lift), below the largest half
constexpr float kA8LeastRatio = -40.f;                // log2 of the smallest value-scale ratio that is told apart (halves end at -24 - lift)

template <int MT, int RG>
struct Attn8Plan {
    static constexpr int kRows = 16 * MT * RG;
    static constexpr int kKeyGroups = kA8Warps / RG;
    static constexpr int kBufs = 2;
    static constexpr int kQBytes = kRows * kA8QStride, kMergeBytes = kBufs * kRows * kA8OStride * 4;
    static constexpr int kStatBytes = kKeyGroups * kRows * 8 + kRows * 4;
    static constexpr int kBarBytes = 512;
    static constexpr int kRest = kQBytes + kMergeBytes + kStatBytes + kBarBytes + 1024;
    static constexpr int kSlots = (227 * 1024 - kRest) / kA8StageBytes / kKeyGroups < 32 ? (227 * 1024 - kRest) / kA8StageBytes / kKeyGroups : 32;
    static constexpr int kRing = kKeyGroups * kSlots * kA8StageBytes;
    static constexpr int kQOff = kRing, kMergeOff = kQOff + kQBytes, kStatOff = kMergeOff + kMergeBytes, kBarOff = kStatOff + kStatBytes;
    static constexpr int kBytes = kRing + kRest;
    static_assert(kSlots >= 2, "a stage in flight beside the one that is read");
    static_assert(16 * kKeyGroups * kSlots + 8 <= kBarBytes, "barriers");
    static_assert(kBarOff % 8 == 0 && kBytes <= 227 * 1024, "shared memory of a block");
};

struct Attn8Args {
    const __nv_bfloat16* q_rot;      // [Hkv, rows, 128]
    const float* k_scale;            // [pages, Hkv]
    const float* v_scale;
    const int* page_table;
    __nv_bfloat16* out;              // [tokens, Hq, 128]
    float* lse_out;                  // [tokens, Hq] or null
    float* o_part;                   // [2 * blocks, rows of a tile, 128]
    float* lse_part;                 // [2 * blocks, rows of a tile], log2
    int* status;
    int Hkv, G, rows, batch, max_pages;
    int share, total;                // stages of a block, of the batch
    float scale_log2;
    FastDiv div_g;
};

// Unit u of episode b: kv head u / tiles, row tile u % tiles.  lens.item_off[b]: stages before the episode.
struct Unit8 {
    int b, g, tile, L, n, stages;
    int first;                       // the batch's stages before the unit
};
template <int ROWS>
__device__ __forceinline__ Unit8 unit8_at(const BatchLens& lens, int batch, int Hkv, int G, int stage)
{
    Unit8 u;
    int lo = 0, hi = batch;          // largest b with item_off[b] <= stage (episodes without new tokens have none)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (lens.item_off[mid] <= stage) lo = mid; else hi = mid;
    }
    u.b = lo;
    u.L = lens.cache_len[lo];
    u.n = lens.new_off[lo + 1] - lens.new_off[lo];
    u.stages = (u.L + u.n + kA8Keys - 1) / kA8Keys;
    const int at = (int)((unsigned)(stage - lens.item_off[lo]) / (unsigned)u.stages);
    const int tiles = (u.n * G + ROWS - 1) / ROWS;
    u.g = (int)((unsigned)at / (unsigned)tiles);
    u.tile = at - u.g * tiles;
    u.first = lens.item_off[lo] + at * u.stages;
    return u;
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int MT, int RG>
__global__ void __launch_bounds__(kA8Threads, 1)
attn8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Attn8Args a, const __grid_constant__ BatchLens lens)
{
    using Plan = Attn8Plan<MT, RG>;
    constexpr int ROWS = Plan::kRows, KG = Plan::kKeyGroups, SLOTS = Plan::kSlots;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    float* s_o = reinterpret_cast<float*>(smem_gen + Plan::kMergeOff);             // [kBufs][ROWS][kA8OStride]
    float* s_m = reinterpret_cast<float*>(smem_gen + Plan::kStatOff);              // [KG][ROWS]
    float* s_l = s_m + KG * ROWS;                                                  // [KG][ROWS]
    float* s_c = s_l + KG * ROWS;                                                  // [ROWS] score factor of a row
    volatile int* s_abort = reinterpret_cast<volatile int*>(smem_gen + Plan::kBarOff + 16 * KG * SLOTS);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = lane & 3, lrow = lane >> 2;
    const int rg = warp % RG, kg = warp / RG;
    const uint32_t ring = smem_base + kg * SLOTS * kA8StageBytes;
    const uint32_t bar_full = smem_base + Plan::kBarOff + 16 * kg * SLOTS, bar_empty = bar_full + 8 * SLOTS;

    const int s0 = blockIdx.x * a.share, s1 = min(a.total, s0 + a.share);          // the block's stages
    const int mine = s1 - s0 > kg ? (s1 - s0 - kg + KG - 1) / KG : 0;              // of them this key group's: s0 + kg + i KG

    if (tid == 0) {
        *s_abort = 0;
        for (int k = 0; k < KG; ++k)
            for (int i = 0; i < SLOTS; ++i) {
                ptx::mbar_init(smem_base + Plan::kBarOff + 16 * k * SLOTS + 8 * i, 1);
                ptx::mbar_init(smem_base + Plan::kBarOff + 16 * k * SLOTS + 8 * (SLOTS + i), RG);
            }
        ptx::fence_barrier_init();
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_v);
    }
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    // ---- looking ahead: lane j knows stage 32 w + j of the key group for window w ----
    struct Ahead { int row; float ks, vs; };           // first row of the code pools, scales
    auto look = [&](int window) -> Ahead {
        const int i = 32 * window + lane;
        Ahead h = {0, 0.f, 0.f};
        if (i < mine) {
            const int s = s0 + kg + i * KG;
            const Unit8 u = unit8_at<ROWS>(lens, a.batch, a.Hkv, a.G, s);
            const int key = (s - u.first) * kA8Keys;
            const int page = a.page_table[(long)u.b * a.max_pages + key / kPage8], at = page * a.Hkv + u.g;
            h.row = at * kPage8 + (key & (kPage8 - 1));
            h.ks = a.k_scale[at];
            h.vs = a.v_scale[at];
        }
        return h;
    };
    auto load = [&](int i, int row) {                  // one lane
        const uint32_t dst = ring + (i % SLOTS) * kA8StageBytes, bar = bar_full + 8 * (i % SLOTS);
        ptx::mbar_expect_tx(bar, kA8StageBytes);
        ptx::tma_load_2d(dst, &tm_k, bar, 0, row);
        ptx::tma_load_2d(dst + kA8StageBytes / 2, &tm_v, bar, 0, row);
    };
    Ahead now = look(0), next = look(1);
    if (rg == 0 && lane < SLOTS && lane < mine) load(lane, now.row);
    __syncwarp();

    bool ok = true;
    int i = 0;                                         // the key group's next stage
    for (int s = s0; s < s1;) {
        const Unit8 u = unit8_at<ROWS>(lens, a.batch, a.Hkv, a.G, s);
        const int end = min(s1, u.first + u.stages);
        const int rows_here = min(ROWS, u.n * a.G - u.tile * ROWS), row0 = u.tile * ROWS;

        // ---- queries: halves of each row's own size ----
#pragma unroll
        for (int r = tid >> 4; r < ROWS; r += kA8Threads / 16) {
            uint4 raw = make_uint4(0u, 0u, 0u, 0u);
            if (r < rows_here)
                raw = reinterpret_cast<const uint4*>(a.q_rot + ((long)u.g * a.rows + (long)lens.new_off[u.b] * a.G + row0 + r) * 128)[tid & 15];
            float x[8], most = 0.f;
            to_floats<__nv_bfloat16, 8>(raw, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(x[e]));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            int e = 14 - ((int)(__float_as_uint(most) >> 23) - 127);       // the row's maximum into [2^14, 2^15)
            e = e > 100 ? 100 : e;
            const float up = exp2_int(e);
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = pack_f16x2(x[2 * k] * up, x[2 * k + 1] * up);
            *reinterpret_cast<uint4*>(smem_gen + Plan::kQOff + r * kA8QStride + (tid & 15) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
            if ((tid & 15) == 0) s_c[r] = a.scale_log2 * exp2_int(-e);
        }
        __syncthreads();

        const uint8_t* q_at = smem_gen + Plan::kQOff + (rg * 16 * MT + lrow) * kA8QStride + quad * 8;
        uint32_t qf[MT == 1 ? 8 : 1][4];               // one row tile: its queries stay in registers
        auto q_frag = [&](int mt, int c, uint32_t (&f)[4]) {
            const uint2 top = *reinterpret_cast<const uint2*>(q_at + mt * 16 * kA8QStride + c * 32);
            const uint2 low = *reinterpret_cast<const uint2*>(q_at + (mt * 16 + 8) * kA8QStride + c * 32);
            f[0] = top.x; f[1] = low.x; f[2] = top.y; f[3] = low.y;
        };
        if (MT == 1) {
#pragma unroll
            for (int c = 0; c < 8; ++c) q_frag(0, c, qf[MT == 1 ? c : 0]);
        }
        float factor[MT][2];
        int last[MT][2];                               // the row's last key
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = rg * 16 * MT + mt * 16 + h * 8 + lrow;
                factor[mt][h] = s_c[r];
                last[mt][h] = r < rows_here ? u.L + (int)fast_div((uint32_t)(row0 + r), a.div_g) : u.L + u.n - 1;
            }
        float o[MT][16][4], m[MT][2], l[MT][2], ref_scale = 0.f;      // ref_scale: the largest value scale so far
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
            for (int t = 0; t < 16; ++t) o[mt][t][0] = o[mt][t][1] = o[mt][t][2] = o[mt][t][3] = 0.f;
            m[mt][0] = m[mt][1] = -INFINITY;
            l[mt][0] = l[mt][1] = 0.f;
        }

        for (; i < mine && s0 + kg + i * KG < end; ++i) {
            if ((i & 31) == 0 && i > 0) {
                now = next;
                next = look((i >> 5) + 1);
            }
            const int slot = i % SLOTS;
            const uint32_t parity = (uint32_t)(i / SLOTS) & 1u;
            const uint32_t kbase = ring + slot * kA8StageBytes, vbase = kbase + kA8StageBytes / 2;
            const float ks = __shfl_sync(0xffffffffu, now.ks, i & 31), vs = __shfl_sync(0xffffffffu, now.vs, i & 31);
            const int key0 = (s0 + kg + i * KG - u.first) * kA8Keys;
            ok = ok && warp_wait(bar_full + 8 * slot, parity, kDevTimeoutMmaKV, a.status, s_abort, lane);
            if (ok) {
                // ---- scores: 16 MT rows x 32 keys ----
                float sc[MT][4][4];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int t = 0; t < 4; ++t) sc[mt][t][0] = sc[mt][t][1] = sc[mt][t][2] = sc[mt][t][3] = 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t kk[4], f[MT][4];
                    ptx::ldmatrix_x4(kk, kbase + lane * 128 + (uint32_t)((c ^ (lane & 7)) << 4));
                    if (MT == 1) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) f[0][e] = qf[MT == 1 ? c : 0][e];
                    } else {
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) q_frag(mt, c, f[mt]);
                    }
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint32_t b0 = halves2(kk[t]), b1 = halves2(kk[t] >> 16);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) mma_f16(sc[mt][t], f[mt], b0, b1);
                    }
                }
                // ---- softmax: references, probabilities, sums ----
                const bool grew = vs > ref_scale;                     // uniform over the warp
                const float shrink = grew ? ref_scale / vs : 1.f;
                if (grew) ref_scale = vs;
                const float ratio = fmaxf(log2f(vs / ref_scale), kA8LeastRatio) + kA8Lift, unlift = ptx::ex2(-ratio);
                const bool masked = key0 + kA8Keys - 1 > u.L;
                uint32_t p[MT][2][4];
                bool moved = grew && shrink > 0.f;
                float keep[MT][2];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float f = factor[mt][h] * ks;
                        float top = -INFINITY;
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float& x = sc[mt][t][2 * h + e];
                                x *= f;
                                if (masked && key0 + 8 * t + 2 * quad + e > last[mt][h]) x = -INFINITY;
                                top = fmaxf(top, x);
                            }
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                        const bool move = top > m[mt][h] + kA8Headroom;      // (from -inf: whenever there is a score)
                        const float was = m[mt][h];
                        if (move) m[mt][h] = top;
                        const float alpha = move ? ptx::ex2(was - top) : 1.f;
                        keep[mt][h] = alpha * shrink;
                        moved = moved || move;
                        const float off = ratio - (m[mt][h] == -INFINITY ? 0.f : m[mt][h]);
                        float sum = 0.f;
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float& x = sc[mt][t][2 * h + e];
                                x = ptx::ex2(x + off);
                                sum += x;
                            }
                        l[mt][h] = fmaf(l[mt][h], alpha, sum * unlift);
                    }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        p[mt][j][0] = pack_f16x2(sc[mt][2 * j][0], sc[mt][2 * j][1]);
                        p[mt][j][1] = pack_f16x2(sc[mt][2 * j][2], sc[mt][2 * j][3]);
                        p[mt][j][2] = pack_f16x2(sc[mt][2 * j + 1][0], sc[mt][2 * j + 1][1]);
                        p[mt][j][3] = pack_f16x2(sc[mt][2 * j + 1][2], sc[mt][2 * j + 1][3]);
                    }
                if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (int t = 0; t < 16; ++t) {
                            o[mt][t][0] *= keep[mt][0]; o[mt][t][1] *= keep[mt][0];
                            o[mt][t][2] *= keep[mt][1]; o[mt][t][3] *= keep[mt][1];
                        }
                }
                // ---- products with the values ----
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t vv[4], even[4], odd[4];
                    ptx::ldmatrix_x4_trans(vv, vbase + lane * 128 + (uint32_t)((c ^ (lane & 7)) << 4));
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const uint32_t parted = __byte_perm(vv[t], 0, 0x3120);    // two keys of a channel, two of the next
                        even[t] = halves2(parted);
                        odd[t] = halves2(parted >> 16);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) {
                            mma_f16(o[mt][2 * c], p[mt][j], even[2 * j], even[2 * j + 1]);
                            mma_f16(o[mt][2 * c + 1], p[mt][j], odd[2 * j], odd[2 * j + 1]);
                        }
                }
            }
            // ---- the slot is read: the group's first warp refills it ----
            __syncwarp();
            if (RG > 1 && lane == 0) ptx::mbar_arrive(bar_empty + 8 * slot);
            if (rg == 0 && i + SLOTS < mine) {
                const int ahead = i + SLOTS;
                const int row = __shfl_sync(0xffffffffu, (ahead >> 5) == (i >> 5) ? now.row : next.row, ahead & 31);
                if (RG > 1) ok = ok && warp_wait(bar_empty + 8 * slot, parity, kDevTimeoutProducer, a.status, s_abort, lane);
                if (ok && lane == 0) load(ahead, row);
            }
        }

        // ---- the key groups' results are joined: references and sums, then the outputs in turn ----
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float sum = l[mt][h];
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                const int r = rg * 16 * MT + mt * 16 + h * 8 + lrow;
                if (quad == 0) {
                    s_m[kg * ROWS + r] = m[mt][h];
                    s_l[kg * ROWS + r] = sum;
                }
            }
        __syncthreads();
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = rg * 16 * MT + mt * 16 + h * 8 + lrow;
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < KG; ++k) top = fmaxf(top, s_m[k * ROWS + r]);
                const float w = m[mt][h] == -INFINITY ? 0.f : ptx::ex2(m[mt][h] - top) * ref_scale * exp2_int(-(int)kA8Lift);
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    o[mt][t][2 * h] *= w;
                    o[mt][t][2 * h + 1] *= w;
                }
            }
        for (int turn = 0; turn < KG / Plan::kBufs; ++turn) {
            if (kg / Plan::kBufs == turn) {
                float* buf = s_o + (kg % Plan::kBufs) * ROWS * kA8OStride;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float4* to = reinterpret_cast<float4*>(buf + (rg * 16 * MT + mt * 16 + h * 8 + lrow) * kA8OStride + quad * 4);
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            float4 x = make_float4(o[mt][2 * c][2 * h], o[mt][2 * c + 1][2 * h], o[mt][2 * c][2 * h + 1], o[mt][2 * c + 1][2 * h + 1]);
                            if (turn > 0) {
                                const float4 y = to[4 * c];
                                x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
                            }
                            to[4 * c] = x;
                        }
                    }
            }
            __syncthreads();
        }
        const bool whole = s == u.first && end == u.first + u.stages;
        const long part = 2L * blockIdx.x + (u.first <= s0 ? 0 : 1);
        for (int r = tid >> 4; r < rows_here; r += kA8Threads / 16) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int k = 0; k < KG; ++k) top = fmaxf(top, s_m[k * ROWS + r]);
#pragma unroll
            for (int k = 0; k < KG; ++k) sum += s_m[k * ROWS + r] == -INFINITY ? 0.f : s_l[k * ROWS + r] * ptx::ex2(s_m[k * ROWS + r] - top);
            const float inv = sum > 0.f ? 1.f / sum : 0.f, lse2 = sum > 0.f ? top + log2f(sum) : -INFINITY;
            const bool nan = !(sum >= 0.f);            // undefined scores: an undefined row
            const int c0 = (tid & 15) * 8;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float4 y = *reinterpret_cast<const float4*>(s_o + r * kA8OStride + c0 + e);
                const float4 z = *reinterpret_cast<const float4*>(s_o + (ROWS + r) * kA8OStride + c0 + e);
                x[e] = (y.x + z.x) * inv; x[e + 1] = (y.y + z.y) * inv; x[e + 2] = (y.z + z.z) * inv; x[e + 3] = (y.w + z.w) * inv;
            }
            if (nan) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = sum;
            }
            if (whole) {
                const int rl = row0 + r, tok = (int)fast_div((uint32_t)rl, a.div_g);
                const long at = ((long)lens.new_off[u.b] + tok) * (a.Hkv * a.G) + u.g * a.G + (rl - tok * a.G);
                *reinterpret_cast<uint4*>(a.out + at * 128 + c0) = from_floats<__nv_bfloat16, 8>(x);
                if (a.lse_out && c0 == 0) a.lse_out[at] = nan ? sum : lse2 * 0.69314718055994531f;
            } else {
                float4* to = reinterpret_cast<float4*>(a.o_part + (part * ROWS + r) * 128 + c0);
                to[0] = make_float4(x[0], x[1], x[2], x[3]);
                to[1] = make_float4(x[4], x[5], x[6], x[7]);
                if (c0 == 0) a.lse_part[part * ROWS + r] = nan ? sum : lse2;
            }
        }
        __syncthreads();
        s = end;
    }
    if (*s_abort && lane == 0) {
        const long long t0 = clock64();                // loads in flight land before the block may leave
        while (clock64() - t0 < 400000) { }
    }
}

// Joins the parts of the units that the blocks' shares cut: a warp per row.  grid (blocks - 1, warps of rows): block x serves the
// unit that the start of share x + 1 lies in, if no earlier start does.
template <int ROWS>
__global__ void __launch_bounds__(128)
merge8_kernel(const Attn8Args a, const __grid_constant__ BatchLens lens)
{
    const int lane = threadIdx.x & 31, i0 = blockIdx.x, cut = (i0 + 1) * a.share;
    const Unit8 u = unit8_at<ROWS>(lens, a.batch, a.Hkv, a.G, cut);
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const int r = blockIdx.y * 4 + (threadIdx.x >> 5), rl = u.tile * ROWS + r;
    if (u.first == cut || u.first < i0 * a.share || rl >= u.n * a.G) return;
    const int i1 = (u.first + u.stages - 1) / a.share;
    float top = -INFINITY, sum = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = i0; i <= i1; ++i) {
        const long part = 2L * i + (u.first <= i * a.share ? 0 : 1);
        const float lse = a.lse_part[part * ROWS + r];
        if (lse == -INFINITY) continue;                // no key of the row in this part
        const float4 y = reinterpret_cast<const float4*>(a.o_part + (part * ROWS + r) * 128)[lane];
        const float up = fmaxf(top, lse), was = ptx::ex2(top - up), is = ptx::ex2(lse - up);
        top = up;
        sum = fmaf(sum, was, is);
        x.x = fmaf(x.x, was, y.x * is); x.y = fmaf(x.y, was, y.y * is); x.z = fmaf(x.z, was, y.z * is); x.w = fmaf(x.w, was, y.w * is);
    }
    const float inv = 1.f / sum;
    const int tok = (int)fast_div((uint32_t)rl, a.div_g);
    const long at = ((long)lens.new_off[u.b] + tok) * (a.Hkv * a.G) + u.g * a.G + (rl - tok * a.G);
    reinterpret_cast<uint2*>(a.out + at * 128)[lane] = make_uint2(ptx::pack_bf16x2(x.x * inv, x.y * inv), ptx::pack_bf16x2(x.z * inv, x.w * inv));
    if (a.lse_out && lane == 0) a.lse_out[at] = (top + log2f(sum)) * 0.69314718055994531f;
}

}  // namespace evln
