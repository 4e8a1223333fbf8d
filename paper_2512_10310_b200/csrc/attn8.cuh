// Step attention over a paged cache in 8 bits (cache8.cuh), for up to 64 query rows per kv head and episode.
//
//     out = softmax(scale * q K^T) V,    K, V = code * scale of its page,    a query sees the keys up to its own position
//
// Bound: reading every code once; a code is one byte, so an SM takes 23 elements a cycle at the copy rate and turning
// them into operands has to keep up with that.  Hence mma.sync on halves: two codes become two halves in ONE instruction
// (cvt f16x2 <- e4m3x2, exact), and everything else that the format asks for is free or done once per row:
//  - the query row is scaled by a power of two into the range of halves (exact above 2^-29 of the row's maximum), and that
//    factor, the page's key scale and the softmax scale are one factor on the scores;
//  - the page's value scale 2^v goes into the exponent of the probabilities: p' = 2^(s + v - (m + r)), r a number of the row that keeps
//    p' between the ends of the halves; the row sums, of 2^(s - m), take it out again.  A row's r follows the largest product of probability and
//    value scale that it has met, not the largest scale: pages that the row gives no weight do not move it, however large their values.
//    (p' is rounded to halves: 2^-11 of itself, finer than bf16, or 2^-31 of the row's largest p * scale.)
// The operands come out of ldmatrix as bytes: a key's 16 bytes are a k-step of the score product (four channels a lane, the
// queries are laid out the same way), and a transposed load of byte PAIRS gives two keys of two neighbouring channels,
// which one byte permutation parts.  The second product is transposed, O^T = V^T P^T: what the scores leave in a lane's registers is
// its right operand as it stands, and 8 rows (a token of 8 query heads a kv head) are one column tile, not half of a row tile.
//
// A block: RG row groups x KG key groups of warps, each warp 8 NQ rows.  A key group takes a RUN of neighbouring stages (32 keys:
// 4 KB keys + 4 KB values, TMA, 128-byte swizzle) through a ring of its own, which one warp of it refills as it goes, and walks it
// unit by unit (unit: episode, kv head).  Nothing is shared between key groups until all are done: then the
// results of neighbouring runs that ended in the same unit are joined in the shared memory that the rings leave.  (Stages dealt
// to the warps in turn, which joins all of them at the end of every unit, took 45 us for 16 ragged episodes of a token, runs 38.)
// Runs are equally long, KG of them per SM; a unit that the runs cut across blocks leaves parts, which merge8_kernel
// joins.  The lanes of a warp look 32 stages ahead for page numbers and scales (a lane each).
// A row's references m and m + r follow the maxima of s and s + v only when those are 2^8 above them, so outputs are rarely scaled anew.
#pragma once

#include <cuda.h>

#include "cache8.cuh"
#include "common.cuh"
#include "ptx_sm100.cuh"
#include "tc_common.cuh"

namespace evln {

constexpr int kA8Keys = 32, kA8StageBytes = 2 * kA8Keys * 128;
constexpr int kA8OStride = 132;                       // floats between rows of the joint's buffers (every second one starts 8 banks on)
constexpr float kA8Headroom = 8.f;                    // p' <= 2^(headroom + lift), below the largest half
constexpr int kA8Lift = 6;
constexpr float kA8LeastGap = -90.f;                  // least v - r that is told apart: below it p' is 0 as a half, and its float is still what the sum needs

template <int NQ, int RG>
struct Attn8Plan {
    // Twelve warps, three a scheduler that hide each other's chains.  (Eight of 255 registers with 32 rows each take 5 to 10 % less for large batches of
    // 17 to 64 rows, 16 episodes of 8000 keys 86 us and 95, but more where latency counts, one of 4096 keys 14.5 and 12.5; figures at the time.)
    static constexpr int kWarps = 12, kThreads = 32 * kWarps;
    static constexpr int kRegs = 168;
    static constexpr int kWarpRows = 8 * NQ, kRows = kWarpRows * RG;
    static constexpr int kKeyGroups = kWarps / RG;
    static constexpr int kStatBytes = kWarps * kWarpRows * 16 + 128;           // references and sums; the units that the runs ended in
    static constexpr int kBarBytes = 512;
    static constexpr int kRest = kStatBytes + kBarBytes + 1024;
    static constexpr int kFit = (227 * 1024 - kRest) / kA8StageBytes / kKeyGroups;
    static constexpr int kSlots = kFit < 32 ? kFit : 32;
    static constexpr int kRing = kKeyGroups * kSlots * kA8StageBytes;
    static constexpr int kStatOff = kRing, kBarOff = kStatOff + kStatBytes;
    static constexpr int kBytes = kRing + kRest;
    static_assert(kSlots >= 2, "a stage in flight beside the one that is read");
    static_assert(16 * kKeyGroups * kSlots + 8 <= kBarBytes, "barriers");
    static_assert(kRows * kA8OStride * 4 <= kSlots * kA8StageBytes, "the joint's buffers, each in its own ring");
    static_assert(NQ <= 2, "a 16-row tile of queries in a warp's registers");
    static_assert(kBarOff % 8 == 0 && kBytes <= 227 * 1024, "shared memory of a block");
};

struct Attn8Args {
    const __nv_bfloat16* q_rot;      // [Hkv, rows, 128]
    const float* k_scale;            // [pages, Hkv]
    const float* v_scale;
    const int* page_table;
    __nv_bfloat16* out;              // [tokens, Hq, 128]
    float* lse_out;                  // [tokens, Hq] or null
    float* o_part;                   // [2 * runs, rows of a block, 128]
    float4* ml_part;                 // [2 * runs, rows of a block]: m (log2), sum in units of 2^m, r: o_part is in units of 2^(m + r - lift)
    int* status;
    int Hkv, G, rows, batch, max_pages;
    int run, total;                  // stages of a run, of the batch
    float scale_log2;
    FastDiv div_g;
};

// A unit: a kv head of an episode.  lens.item_off[b]: stages before the episode.
struct Unit8 {
    int b, g, L, n, stages;
    int first;                       // the batch's stages before the unit
};
__device__ __forceinline__ Unit8 unit8_at(const BatchLens& lens, int batch, int stage)
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
    u.g = (int)((unsigned)(stage - lens.item_off[lo]) / (unsigned)u.stages);
    u.first = lens.item_off[lo] + u.g * u.stages;
    return u;
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 2^e of a whole number e between -126 and 127 that is held as a float
__device__ __forceinline__ float exp2_whole(float e) { return __uint_as_float(__float_as_uint(8388608.f + 127.f + e) << 23); }
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// warp_wait for a barrier that has most often completed: every lane looks once, which takes 0.1 us less than one lane's polling and sharing.
__device__ __forceinline__ bool warp_wait_ready(uint32_t bar, uint32_t parity, int code, int* status, volatile int* s_abort, int lane)
{
    if (__all_sync(0xffffffffu, ptx::mbar_try_wait(bar, parity))) return true;
    const bool ok = warp_wait(bar, parity, code, status, s_abort, lane);
    __syncwarp();
    return ok;
}

// Where query row rl of a unit goes: row of [tokens, Hq].
__device__ __forceinline__ long out_row8(const Attn8Args& a, const BatchLens& lens, const Unit8& u, int rl)
{
    const int tok = (int)fast_div((uint32_t)rl, a.div_g);
    return ((long)lens.new_off[u.b] + tok) * (a.Hkv * a.G) + u.g * a.G + (rl - tok * a.G);
}
constexpr float kLn2 = 0.69314718055994531f;

// Parts of a row with references m and m + r, joined at top and top + joint_r: the largest m, and about the largest m + r (`high`), so that no part's
// outputs leave the range of floats.  (-inf: no part has a key of the row.)
__device__ __forceinline__ float joint_base(float top) { return top == -INFINITY ? 0.f : top; }
__device__ __forceinline__ float joint_r(float top, float high) { return top == -INFINITY ? 0.f : fminf(fmaxf(high - top, -120.f), 120.f); }

template <int NQ, int RG>
__global__ void __launch_bounds__(Attn8Plan<NQ, RG>::kThreads) __maxnreg__((Attn8Plan<NQ, RG>::kRegs))
attn8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Attn8Args a, const __grid_constant__ BatchLens lens)
{
    using Plan = Attn8Plan<NQ, RG>;
    constexpr int ROWS = Plan::kRows, KG = Plan::kKeyGroups, SLOTS = Plan::kSlots, WROWS = Plan::kWarpRows;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    float4* s_ml = reinterpret_cast<float4*>(smem_gen + Plan::kStatOff);           // [KG][ROWS] as ml_part
    int* s_unit = reinterpret_cast<int*>(s_ml + KG * ROWS);                        // [KG] first stage of the unit that the run ended in, -1: nothing left
    volatile int* s_abort = reinterpret_cast<volatile int*>(smem_gen + Plan::kBarOff + 16 * KG * SLOTS);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, quad = lane & 3, lrow = lane >> 2;
    const int rg = warp % RG, kg = warp / RG;
    const uint32_t ring = smem_base + kg * SLOTS * kA8StageBytes;
    const uint32_t bar_full = smem_base + Plan::kBarOff + 16 * kg * SLOTS, bar_empty = bar_full + 8 * SLOTS;

    const int run = blockIdx.x * KG + kg;
    const int r0 = min(a.total, run * a.run), r1 = min(a.total, r0 + a.run), mine = r1 - r0;      // the run: stages r0 .. r1-1

    if (lane == 0 && rg == 0) {
        for (int i = 0; i < SLOTS; ++i) {
            ptx::mbar_init(bar_full + 8 * i, 1);
            ptx::mbar_init(bar_empty + 8 * i, RG);
        }
        ptx::fence_barrier_init();
        if (warp == 0) {
            *s_abort = 0;
            ptx::prefetch_tensormap(&tm_k);
            ptx::prefetch_tensormap(&tm_v);
        }
    }
    Unit8 u = {};
    if (mine > 0) u = unit8_at(lens, a.batch, r0);
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();

    // ---- looking ahead: lane j knows stage 32 w + j of the run for window w ----
    struct Ahead { int row; float ks, vs; };           // first row of the code pools, scales
    auto look = [&](int window) -> Ahead {
        const int i = 32 * window + lane;
        Ahead h = {0, 0.f, 0.f};
        if (i < mine) {
            Unit8 w = u;
            if (r0 + i >= u.first + u.stages) w = unit8_at(lens, a.batch, r0 + i);
            const int key = (r0 + i - w.first) * kA8Keys;
            const int page = a.page_table[(long)w.b * a.max_pages + key / kPage8], at = page * a.Hkv + w.g;
            h.row = at * kPage8 + (key & (kPage8 - 1));
            h.ks = a.k_scale[at];
            h.vs = a.v_scale[at];
        }
        return h;
    };
    auto load = [&](int slot, int row) {               // one lane
        const uint32_t dst = ring + slot * kA8StageBytes, bar = bar_full + 8 * slot;
        ptx::mbar_expect_tx(bar, kA8StageBytes);
        ptx::tma_load_2d(dst, &tm_k, bar, 0, row);
        ptx::tma_load_2d(dst + kA8StageBytes / 2, &tm_v, bar, 0, row);
    };
    // ---- a unit's queries: halves of each row's own size, in operand order (k-step c: channels 16 c + 4 quad .. + 3 of rows lrow, lrow + 8) ----
    uint32_t qf[8][2 * NQ];
    float factor[NQ];
    auto load_q = [&](uint2 (&raw)[NQ][8]) {
#pragma unroll
        for (int h = 0; h < NQ; ++h) {
            const int rl = rg * WROWS + h * 8 + lrow;
            const uint2* src = reinterpret_cast<const uint2*>(a.q_rot + ((long)u.g * a.rows + (long)lens.new_off[u.b] * a.G + rl) * 128) + quad;
#pragma unroll
            for (int c = 0; c < 8; ++c) raw[h][c] = rl < u.n * a.G ? src[4 * c] : make_uint2(0u, 0u);
        }
    };
    auto put_q = [&](const uint2 (&raw)[NQ][8]) {
        float up[NQ];
#pragma unroll
        for (int h = 0; h < NQ; ++h) {
            float most = 0.f;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                most = ptx::max3(most, fabsf(__uint_as_float(raw[h][c].x << 16)), fabsf(__uint_as_float(raw[h][c].x & 0xffff0000u)));
                most = ptx::max3(most, fabsf(__uint_as_float(raw[h][c].y << 16)), fabsf(__uint_as_float(raw[h][c].y & 0xffff0000u)));
            }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            int e = 14 - ((int)(__float_as_uint(most) >> 23) - 127);                 // the row's maximum into [2^14, 2^15)
            e = e > 100 ? 100 : e;
            up[h] = exp2_int(e);
            factor[h] = a.scale_log2 * exp2_int(-e);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) {
#pragma unroll
            for (int h = 0; h < NQ; ++h) {                                            // channels 4 quad, + 1 of each half, then + 2, + 3
                qf[c][h] = pack_f16x2(__uint_as_float(raw[h][c].x << 16) * up[h], __uint_as_float(raw[h][c].x & 0xffff0000u) * up[h]);
                qf[c][h + NQ] = pack_f16x2(__uint_as_float(raw[h][c].y << 16) * up[h], __uint_as_float(raw[h][c].y & 0xffff0000u) * up[h]);
            }
        }
    };

    Ahead now, next;
    {
        // the first unit's queries are on their way while the first stages' pages are looked up
        uint2 raw[NQ][8];
        if (mine > 0) load_q(raw);
        now = look(0);
        if (rg == 0 && lane < SLOTS && lane < mine) load(lane, now.row);
        __syncwarp();
        if (mine > 0) put_q(raw);
    }
    next = look(1);

    bool ok = true;
    int i = 0, slot = 0;                               // the run's next stage
    uint32_t parity = 0;
    // o: transposed, [8-row tile][16 channels 16 c ..]: channels 16 c + 2 lrow (first two) and + 1, rows 2 quad and 2 quad + 1 of the tile; m, l, r: rows
    // lrow (r: a whole number)
    float o[NQ][8][4], m[NQ], l[NQ], r[NQ];
    bool left = false;                                 // the unit at hand goes to the joint
    while (i < mine) {
        if (i > 0) {
            u = unit8_at(lens, a.batch, r0 + i);
            uint2 raw[NQ][8];
            load_q(raw);
            put_q(raw);
        }
        const int begin = r0 + i, end = min(r1, u.first + u.stages);
        const int rows_here = u.n * a.G, row0 = rg * WROWS;      // this warp's rows: row0 ..
        int last[NQ];                                  // the row's last key
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            const int row = row0 + q * 8 + lrow;
            last[q] = row < rows_here ? u.L + (int)fast_div((uint32_t)row, a.div_g) : u.L + u.n - 1;
#pragma unroll
            for (int c = 0; c < 8; ++c) o[q][c][0] = o[q][c][1] = o[q][c][2] = o[q][c][3] = 0.f;
            m[q] = -INFINITY;
            l[q] = r[q] = 0.f;
        }

        for (; r0 + i < end; ++i) {
            if ((i & 31) == 0 && i > 0) {
                now = next;
                next = look((i >> 5) + 1);
            }
            const uint32_t kbase = (ring + slot * kA8StageBytes + lane * 128) ^ ((lane & 7) << 4), vbase = kbase + kA8StageBytes / 2;
            const float ks = __shfl_sync(0xffffffffu, now.ks, i & 31), vs = __shfl_sync(0xffffffffu, now.vs, i & 31);
            const int key0 = (r0 + i - u.first) * kA8Keys;
            ok = ok && warp_wait_ready(bar_full + 8 * slot, parity, kDevTimeoutMmaKV, a.status, s_abort, lane);
            if (ok) {
                // ---- scores: 16 rows (8 of them used, NQ = 1) x 32 keys ----
                float sc[4][4];
#pragma unroll
                for (int t = 0; t < 4; ++t) sc[t][0] = sc[t][1] = sc[t][2] = sc[t][3] = 0.f;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t kk[4], f[4];
                    ptx::ldmatrix_x4(kk, kbase ^ (c << 4));
                    f[0] = qf[c][0];
                    f[2] = qf[c][NQ];
                    f[1] = NQ == 2 ? qf[c][1] : 0u;
                    f[3] = NQ == 2 ? qf[c][2 * NQ - 1] : 0u;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        uint32_t b0, b1;
                        halves4(kk[t], b0, b1);
                        mma_f16(sc[t], f, b0, b1);
                    }
                }
                // ---- softmax: references, probabilities, sums ----
                const float v = (float)((int)(__float_as_uint(vs) >> 23) - 127);      // (a power of two; uniform over the warp)
                if (key0 + kA8Keys - 1 > u.L) {                       // keys that not every row sees
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (key0 + 8 * t + 2 * quad + e > last[q]) sc[t][2 * q + e] = -INFINITY;
                }
                float f[NQ], top[NQ];
                bool move[NQ], moved = false;
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    // > 0 and finite: zeros times it stay zeros and masked scores -inf (a page of zero keys has the scale 2^-120, which
                    // small queries' factor would take below the least float)
                    f[q] = fminf(fmaxf(factor[q] * ks, 0x1p-126f), 0x1p127f);
                    top[q] = -INFINITY;
#pragma unroll
                    for (int t = 0; t < 4; ++t) top[q] = ptx::max3(top[q], sc[t][2 * q], sc[t][2 * q + 1]);
                    top[q] = fmaxf(top[q], __shfl_xor_sync(0xffffffffu, top[q], 1));
                    top[q] = fmaxf(top[q], __shfl_xor_sync(0xffffffffu, top[q], 2)) * f[q];
                    move[q] = top[q] + fmaxf(v - r[q], 0.f) > m[q] + kA8Headroom;     // (from -inf: whenever there is a score)
                    moved = moved || move[q];
                }
                if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                    for (int q = 0; q < NQ; ++q) {
                        float keep = 1.f;
                        if (move[q]) {
                            // m + r as it was or as this page wants it, whichever is larger; rounded down, so that it does not creep up
                            const float to = fmaxf(m[q], top[q]), back = m[q] - to, r_to = floorf(fmaxf(r[q] + back, v + (top[q] - to)));
                            l[q] *= ptx::ex2(back);
                            keep = ptx::ex2(back + (r[q] - r_to));
                            m[q] = to;
                            r[q] = r_to;
                        }
                        const float k0 = __shfl_sync(0xffffffffu, keep, 8 * quad), k1 = __shfl_sync(0xffffffffu, keep, 8 * quad + 4);   // rows 2 quad, 2 quad + 1
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            o[q][c][0] *= k0; o[q][c][1] *= k1;
                            o[q][c][2] *= k0; o[q][c][3] *= k1;
                        }
                    }
                }
                uint32_t p[NQ][2][2];                                 // the transposed product's operand: two k-steps of 16 keys
#pragma unroll
                for (int q = 0; q < NQ; ++q) {
                    const float steps = fmaxf(v - r[q], kA8LeastGap) + (float)kA8Lift, off = steps - (m[q] == -INFINITY ? 0.f : m[q]);
                    const uint64_t f2 = ptx::pack2(f[q], f[q]), off2 = ptx::pack2(off, off);
                    uint64_t sum2 = 0;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        float x, y;
                        ptx::unpack2(ptx::fma2(ptx::pack2(sc[t][2 * q], sc[t][2 * q + 1]), f2, off2), x, y);
                        x = ptx::ex2(x);
                        y = ptx::ex2(y);
                        sum2 = ptx::add2(sum2, ptx::pack2(x, y));
                        p[q][t >> 1][t & 1] = pack_f16x2(x, y);
                    }
                    float x, y;
                    ptx::unpack2(sum2, x, y);
                    l[q] = fmaf(x + y, exp2_whole(fmaxf(-steps, -126.f)), l[q]);
                }
                // ---- products with the values, transposed: 16 channels down, 8 rows across ----
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    uint32_t vv[4], even[4], odd[4];
                    ptx::ldmatrix_x4_trans(vv, vbase ^ (c << 4));
#pragma unroll
                    for (int t = 0; t < 4; ++t) halves4(__byte_perm(vv[t], 0, 0x3120), even[t], odd[t]);    // two keys of a channel, two of the next
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t v[4] = {even[2 * j], odd[2 * j], even[2 * j + 1], odd[2 * j + 1]};
#pragma unroll
                        for (int q = 0; q < NQ; ++q) mma_f16(o[q][c], v, p[q][j][0], p[q][j][1]);
                    }
                }
            }
            // ---- the slot is read: the group's first warp refills it ----
            __syncwarp();
            if (RG > 1 && lane == 0) ptx::mbar_arrive(bar_empty + 8 * slot);
            if (rg == 0 && i + SLOTS < mine) {
                const int ahead = i + SLOTS;
                const int row = __shfl_sync(0xffffffffu, (ahead >> 5) == (i >> 5) ? now.row : next.row, ahead & 31);
                if (RG > 1) ok = ok && warp_wait_ready(bar_empty + 8 * slot, parity, kDevTimeoutProducer, a.status, s_abort, lane);
                if (ok && lane == 0) load(slot, row);
            }
            if (++slot == SLOTS) {
                slot = 0;
                parity ^= 1u;
            }
        }

        // ---- sums over the row's four lanes; a unit that this run ends is done here, whole or a part ----
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            l[q] += __shfl_xor_sync(0xffffffffu, l[q], 1);
            l[q] += __shfl_xor_sync(0xffffffffu, l[q], 2);
        }
        const bool whole = begin == u.first && end == u.first + u.stages;
        left = !whole && end == r1;
        if (!left) {
#pragma unroll
            for (int q = 0; q < NQ; ++q) {
                const float by_row = l[q] == 0.f ? 0.f : 1.f / l[q], value = exp2_whole(r[q] - (float)kA8Lift);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int from = 8 * quad + 4 * e;
                    const float by = __shfl_sync(0xffffffffu, by_row, from), scale = __shfl_sync(0xffffffffu, value, from);
                    const float mr = __shfl_sync(0xffffffffu, m[q], from), lr = __shfl_sync(0xffffffffu, l[q], from), rr = __shfl_sync(0xffffffffu, r[q], from);
                    const int row = q * 8 + 2 * quad + e;
                    if (row0 + row >= rows_here) continue;
                    if (whole) {
                        const long at = out_row8(a, lens, u, row0 + row);
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            reinterpret_cast<uint32_t*>(a.out + at * 128)[8 * c + lrow] = ptx::pack_bf16x2(o[q][c][e] * by * scale, o[q][c][2 + e] * by * scale);
                        if (a.lse_out && lrow == 0) a.lse_out[at] = (mr + log2f(lr)) * kLn2;
                    } else {
                        const long at = 2L * run * ROWS + row0 + row;
#pragma unroll
                        for (int c = 0; c < 8; ++c) reinterpret_cast<float2*>(a.o_part + at * 128)[8 * c + lrow] = make_float2(o[q][c][e], o[q][c][2 + e]);
                        if (lrow == 0) a.ml_part[at] = make_float4(mr, lr, rr, 0.f);
                    }
                }
            }
        }
    }

    // ---- the joint: runs of the block that ended in the same unit; a group's rows go to its own ring, whose loads have all been waited for ----
    // (Code that runs once costs its fetch, some 0.1 us for each 100 instructions: hence one barrier and rolled loops.)
    if (RG > 1) asm volatile("bar.sync %0, %1;" :: "r"(1 + kg), "n"(32 * RG) : "memory");
    else __syncwarp();
    if (rg == 0 && lane == 0) {
        s_unit[kg] = left ? u.first : -1;
    }
    if (left) {
        float* to = reinterpret_cast<float*>(smem_gen + kg * SLOTS * kA8StageBytes) + (rg * WROWS + 2 * quad) * kA8OStride + 2 * lrow;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int c = 0; c < 8; ++c) *reinterpret_cast<float2*>(to + (q * 8 + e) * kA8OStride + 16 * c) = make_float2(o[q][c][e], o[q][c][2 + e]);
            if (quad == 0) s_ml[kg * ROWS + rg * WROWS + q * 8 + lrow] = make_float4(m[q], l[q], r[q], 0.f);
        }
    }
    __syncthreads();
    if (*s_abort) {
        const long long t0 = clock64();                // loads in flight land before the block may leave
        while (clock64() - t0 < 400000) { }
        return;
    }
    const int unit_of = s_unit[lane < KG ? lane : KG - 1];
    for (int k0 = 0; k0 < KG;) {
        const int at_unit = __shfl_sync(0xffffffffu, unit_of, k0);
        const unsigned others = __ballot_sync(0xffffffffu, lane > k0 && lane < KG && unit_of != at_unit);
        const int k1 = others ? __ffs(others) - 1 : KG;
        if (at_unit >= 0) {
            const Unit8 w = left && u.first == at_unit ? u : unit8_at(lens, a.batch, at_unit);
            const int first_run = blockIdx.x * KG + k0, ends = min(a.total, (blockIdx.x * KG + k1) * a.run);
            const bool whole = first_run * a.run <= w.first && ends == w.first + w.stages;
            const int rows_here = w.n * a.G;
#pragma unroll 1
            for (int row = warp; row < rows_here; row += Plan::kWarps) {             // a warp per row, four channels a lane
                float4 ml[KG], y[KG];
                float top = -INFINITY, high = -INFINITY, sum = 0.f;                 // of m, of m + r
#pragma unroll
                for (int k = 0; k < KG; ++k) {
                    const bool in = k >= k0 && k < k1;
                    ml[k] = in ? s_ml[k * ROWS + row] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
                    y[k] = in ? *reinterpret_cast<const float4*>(smem_gen + k * SLOTS * kA8StageBytes + (row * kA8OStride + 4 * lane) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
                    top = fmaxf(top, ml[k].x);
                    high = fmaxf(high, ml[k].x + ml[k].z);
                }
                const float base = joint_base(top), r_to = joint_r(top, high);
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int k = 0; k < KG; ++k) {
                    const float back = ml[k].x - base, f = ptx::ex2(back + (ml[k].z - r_to));
                    sum = fmaf(ml[k].y, ptx::ex2(back), sum);
                    x.x = fmaf(y[k].x, f, x.x); x.y = fmaf(y[k].y, f, x.y); x.z = fmaf(y[k].z, f, x.z); x.w = fmaf(y[k].w, f, x.w);
                }
                if (whole) {
                    const long at = out_row8(a, lens, w, row);
                    const float by = sum == 0.f ? 0.f : 1.f / sum, scale = ptx::ex2(r_to - (float)kA8Lift);
                    reinterpret_cast<uint2*>(a.out + at * 128)[lane] =
                        make_uint2(ptx::pack_bf16x2(x.x * by * scale, x.y * by * scale), ptx::pack_bf16x2(x.z * by * scale, x.w * by * scale));
                    if (a.lse_out && lane == 0) a.lse_out[at] = (top + log2f(sum)) * kLn2;
                } else {
                    const long at = (2L * first_run + 1) * ROWS + row;
                    reinterpret_cast<float4*>(a.o_part + at * 128)[lane] = x;
                    if (lane == 0) a.ml_part[at] = make_float4(top, sum, r_to, 0.f);
                }
            }
        }
        k0 = k1;
    }
}

// The units that merge8_kernel looks at: all of the batch's where they are few, by the stages before them; else (count 0) block x takes
// those that begin in block x's share of the attention kernel.
constexpr int kMergeUnits = 192;
struct MergeList {
    int count;
    int first[kMergeUnits];
};

// Joins the parts of the units that the runs cut: what each block's runs that end in the unit left jointly, and what a run left that goes on
// behind its end.  Blocks (x, y): units as in MergeList, rows y, y + gridDim.y, ...; the warps share a row's parts, each with up to kMergeAhead
// of them in flight beside the references, before it is known what they weigh.
// Blocks without such a unit leave at once (the first one does not: the next kernel in the stream waits for this grid, which
// therefore must not end before the attention kernel has), so the others are on the SMs, and know what to read, when the parts are there.
constexpr int kMergeAhead = 5;                         // (with 3 64 rows of one episode of 20656 keys took 0.9 us longer)
template <int ROWS> constexpr int kMergeWarps = ROWS >= 32 ? 8 : 4;            // (8 and 16 rows: few parts, many units)
template <int ROWS, int KG>
__global__ void __launch_bounds__(32 * kMergeWarps<ROWS>)
merge8_kernel(const Attn8Args a, const __grid_constant__ BatchLens lens, const __grid_constant__ MergeList list)
{
    constexpr int WARPS = kMergeWarps<ROWS>;
    __shared__ float4 s_x[WARPS][32];
    __shared__ float s_sum[WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Unit8 u;
    int u1, ra, rb;
    bool on;                                           // the unit's last run goes on behind it
    auto cut = [&](int first) -> bool {
        u = unit8_at(lens, a.batch, first);
        u1 = u.first + u.stages;
        ra = u.first / a.run;
        rb = (u1 - 1) / a.run;
        on = min(a.total, (rb + 1) * a.run) > u1;
        return ra != rb && (on || ra / KG != rb / KG); // else whole: in one run, or in the joint of one block
    };
    int next, to;
    if (list.count > 0) {
        next = list.first[blockIdx.x];
        to = next + 1;
    } else {
        next = blockIdx.x * KG * a.run;
        to = min(a.total, next + KG * a.run);
        u = unit8_at(lens, a.batch, next);
        if (u.first < next) next = u.first + u.stages;
    }
    bool found = false;
    while (next < to && !(found = cut(next))) next = u1;
    if (!found && (blockIdx.x > 0 || blockIdx.y > 0)) return;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    while (found) {
        const int b0 = ra / KG, joints = (on ? rb - 1 : rb) / KG - b0 + 1, parts = joints + (on ? 1 : 0);
        auto row_of = [&](int p, int r) -> long { return (p < joints ? 2L * max(ra, (b0 + p) * KG) + 1 : 2L * rb) * ROWS + r; };
        for (int r = blockIdx.y; r < u.n * a.G; r += gridDim.y) {
            float4 y[kMergeAhead], ml[kMergeAhead];
            auto fetch = [&](int p0) {
#pragma unroll
                for (int i = 0; i < kMergeAhead; ++i) {
                    const int p = p0 + WARPS * i;
                    if (p < parts) {
                        const long at = row_of(p, r);
                        y[i] = reinterpret_cast<const float4*>(a.o_part + at * 128)[lane];
                        ml[i] = a.ml_part[at];
                    }
                }
            };
            fetch(warp);
            float top = -INFINITY, high = -INFINITY, sum = 0.f;      // of m, of m + r
            for (int p = lane; p < parts; p += 32) {
                const float4 of = a.ml_part[row_of(p, r)];
                top = fmaxf(top, of.x);
                high = fmaxf(high, of.x + of.z);
            }
#pragma unroll
            for (int s = 16; s > 0; s >>= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
                high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, s));
            }
            const float base = joint_base(top), r_to = joint_r(top, high);
            float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
            for (int p0 = warp;;) {
#pragma unroll
                for (int i = 0; i < kMergeAhead; ++i) {
                    if (p0 + WARPS * i >= parts) break;
                    const float back = ml[i].x - base, w = ptx::ex2(back + (ml[i].z - r_to));      // -inf: no key of the row in this part
                    sum = fmaf(ml[i].y, ptx::ex2(back), sum);
                    x.x = fmaf(y[i].x, w, x.x); x.y = fmaf(y[i].y, w, x.y); x.z = fmaf(y[i].z, w, x.z); x.w = fmaf(y[i].w, w, x.w);
                }
                p0 += WARPS * kMergeAhead;
                if (p0 >= parts) break;
                fetch(p0);
            }
            s_x[warp][lane] = x;
            if (lane == 0) s_sum[warp] = sum;
            __syncthreads();
            if (threadIdx.x < 64) {                                  // a pair of channels a thread
                float2 z = make_float2(0.f, 0.f);
                sum = 0.f;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) {
                    const float2 part = reinterpret_cast<const float2*>(s_x[w])[threadIdx.x];
                    z.x += part.x; z.y += part.y;
                    sum += s_sum[w];
                }
                const float by = 1.f / sum, scale = ptx::ex2(r_to - (float)kA8Lift);
                const long at = out_row8(a, lens, u, r);
                reinterpret_cast<uint32_t*>(a.out + at * 128)[threadIdx.x] = ptx::pack_bf16x2(z.x * by * scale, z.y * by * scale);
                if (a.lse_out && threadIdx.x == 0) a.lse_out[at] = (top + log2f(sum)) * kLn2;
            }
            __syncthreads();
        }
        next = u1;
        found = false;
        while (next < to && !(found = cut(next))) next = u1;
    }
}

}  // namespace evln
