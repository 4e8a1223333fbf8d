// The attention weight that a step's queries give each key:  w_j = sum_r 2^(s_rj - lse_r),  s = scale log2(e) q_r . k_j,
// over the packed query rows r of a kv head that see key j, added to decay * (what the key had).
//
// Knowing each row's log-sum-exp, there is no running maximum and no order: the sum over rows wants the scores TRANSPOSED,
// keys down and query rows across.  So a key is a lane of tensor memory (M = 128 keys a tile, N query rows), a thread owns a
// key, and its sum is a loop over columns in its own registers: no shuffles and no atomics, and few rows cost few
// columns instead of a padded 128-row tile.
//
// bf16: S^T = K Q^T on tcgen05 (kind::f16, fp32 sums).  Per CTA, 640 threads: warp 0 loads (TMA, a ring of K tiles and one of
// query chunks), warp 1 issues, warps 2 and 3 fetch the rows' log-sum-exps, warps 4-19 exponentiate: four groups of four (one warp per TMEM lane
// quarter), two of which share a chunk of 128 rows, or which take whole tiles in turn where a tile is one chunk.  Score buffers: 4 x 128 columns.
// Bound: many rows, the special-function unit (16 exponentials a cycle and SM; the products take a quarter of that); few
// rows, reading the keys once.  (1372 rows of 4 kv heads over 4292 keys: 13.5 us with inputs out of DRAM, 11.3 with three sets of them in L2, 5.9 of them
// exponentials; over 20196 46.4.  Two groups that fetched their
// log-sum-exps themselves, and masked every block of a tile that some row does not see, took 15.3 and 58.8: a wait that has to poll costs 0.1 us,
// a fetch 0.3 us.  Chunks of 64 rows are bound by the issuing warp, 17.9, of 256 have too few buffers, 14.5; a quarter to a half of the exponentials on the
// FMA pipe, by a polynomial of degree 5: 13.9 to 14.4.  Per SM sub-partition, 32 scores of 32 keys take 360 cycles: 256 of exponentials, beside
// loads from tensor memory and products that alone take 340.)
// Few tiles: the chunks of a tile are dealt to the CTAs of a cluster, whose sums meet in the first one's shared memory, in order.
// fp32: a thread per key with its row in registers, query rows broadcast from shared memory, float FMAs; or 8 keys x 8 rows a thread.
#pragma once

#include <cuda.h>

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "tc_common.cuh"

namespace evln {

struct KeyWeightArgs {
    const float* lse;        // [n, Hq]
    const float* in;         // [Hkv, cap]
    float* out;              // [Hkv, cap]
    const void* q_rot;       // fp32 kernel: [Hkv, rows, D]
    const void* k_cache;     // fp32 kernel: [Hkv, cap, D]
    int* status;
    int Hkv, G, rows, L, n, cap;
    int chunk_rows, chunks;  // query rows of a chunk (the tensor kernel's N), chunks of a kv head
    int items;               // kv heads * key tiles
    float scale_log2, decay;
    FastDiv div_g, div_hkv;
};

constexpr int kKwGroups = 4, kKwThreads = 128 + 128 * kKwGroups, kKwStages = 3, kKwQStages = 3, kKwBufs = 4, kKwMaxCluster = 8;
constexpr int kKwRows = 128;                              // most query rows of a chunk (fewer: a multiple of 32)
template <int D>
struct KeyWeightPlan {
    static constexpr int kTile = 128 * D * 2, kChunk = kKwRows * D * 2;
    static constexpr int kQOff = kKwStages * kTile, kBarOff = kQOff + kKwQStages * kChunk;
    static constexpr int kLseOff = kBarOff + 512;        // float [kKwBufs][kKwRows]
    static constexpr int kPartOff = kLseOff + kKwBufs * kKwRows * 4;             // float [2][kKwGroups - 1][128]: the other groups' sums, tiles in turn
    static constexpr int kRemoteOff = kPartOff + 2 * (kKwGroups - 1) * 128 * 4;  // float [kKwMaxCluster][128]
    // (never two CTAs on an SM: each takes all of tensor memory, and CTAs of a cluster wait for each other)
    static constexpr int kNeeded = kRemoteOff + kKwMaxCluster * 128 * 4 + 1024, kBytes = kNeeded < 120 * 1024 ? 120 * 1024 : kNeeded;
    static_assert(kBytes <= 227 * 1024, "shared memory of a block");
};

// the first chunk of the tile at `key0` with a row that sees one of its keys
__device__ __forceinline__ int first_chunk(const KeyWeightArgs& a, int key0)
{
    const int behind = key0 - a.L;                       // tokens before this one see none of the tile's keys
    return behind <= 0 ? 0 : behind * a.G / a.chunk_rows;
}

template <int D>
__global__ void __launch_bounds__(kKwThreads, 1)
key_weights_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_q, const KeyWeightArgs a)
{
    using Plan = KeyWeightPlan<D>;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
    const uint32_t bar_k_full = smem_base + Plan::kBarOff, bar_k_empty = bar_k_full + 8 * kKwStages;
    const uint32_t bar_q_full = bar_k_empty + 8 * kKwStages, bar_q_empty = bar_q_full + 8 * kKwQStages;
    const uint32_t bar_s_full = bar_q_empty + 8 * kKwQStages, bar_s_free = bar_s_full + 8 * kKwBufs;
    const uint32_t bar_l_full = bar_s_free + 8 * kKwBufs, bar_l_free = bar_l_full + 8 * kKwBufs;
    const uint32_t tmem_slot = bar_l_free + 8 * kKwBufs;
    volatile uint32_t* s_tmem = reinterpret_cast<volatile uint32_t*>(smem_gen + (tmem_slot - smem_base));
    volatile int* s_abort = reinterpret_cast<volatile int*>(smem_gen + (tmem_slot - smem_base) + 4);
    float* s_lse = reinterpret_cast<float*>(smem_gen + Plan::kLseOff);
    float* s_part = reinterpret_cast<float*>(smem_gen + Plan::kPartOff);
    float* s_remote = reinterpret_cast<float*>(smem_gen + Plan::kRemoteOff);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // A CTA (cluster size 1) takes tiles blockIdx.x, + gridDim.x, ...; a cluster of several takes one, its chunks dealt out.
    const int csize = (int)gridDim.y, rank = (int)blockIdx.y, stride = (int)gridDim.x, cshift = __ffs(csize) - 1;
    auto tile_of = [&](int item, int& g) -> int {         // kv heads side by side
        const int t = (int)fast_div((uint32_t)item, a.div_hkv);
        g = item - t * a.Hkv;
        return t * kTileN;
    };

    if (threadIdx.x == 0) {
        ptx::prefetch_tensormap(&tm_k);
        ptx::prefetch_tensormap(&tm_q);
        for (int i = 0; i < kKwStages; ++i) {
            ptx::mbar_init(bar_k_full + 8 * i, 1);
            ptx::mbar_init(bar_k_empty + 8 * i, 1);
        }
        for (int i = 0; i < kKwQStages; ++i) {
            ptx::mbar_init(bar_q_full + 8 * i, 1);
            ptx::mbar_init(bar_q_empty + 8 * i, 1);
        }
        for (int i = 0; i < kKwBufs; ++i) {
            ptx::mbar_init(bar_s_full + 8 * i, 1);
            ptx::mbar_init(bar_s_free + 8 * i, a.chunks == 1 ? 4 : 8);
            ptx::mbar_init(bar_l_full + 8 * i, 1);
            ptx::mbar_init(bar_l_free + 8 * i, a.chunks == 1 ? 4 : 8);
        }
        ptx::fence_barrier_init();
        *s_abort = 0;
    }
    if (warp == 1) {
        ptx::tmem_alloc(tmem_slot, 512);
        ptx::tmem_relinquish();
    }
    ptx::fence_before_sync();
    __syncthreads();
    ptx::fence_after_sync();
    const uint32_t tmem = *s_tmem;
    if (csize > 1) ptx::cluster_arrive_relaxed();         // (waited for before the first remote store: all CTAs have started)
    ptx::grid_launch_dependents();
    ptx::grid_dependency_wait();

    bool ok = true;
    float own_sum = 0.f;                                  // cluster: this CTA's sums (group 0's threads)
    if (warp == 0) {
        if (lane == 0) {
            int kt = 0, qt = 0;                           // tiles and chunks so far
            for (int item = blockIdx.x; item < a.items && ok; item += stride, ++kt) {
                int g;
                const int key0 = tile_of(item, g), ks = kt % kKwStages;
                bool fresh = true;
                for (int c = first_chunk(a, key0) + rank; c < a.chunks && ok; c += csize, ++qt) {
                    if (fresh) {
                        if (kt >= kKwStages) ok = wait_bounded(bar_k_empty + 8 * ks, ((kt / kKwStages) & 1) ^ 1, kDevTimeoutProducer, a.status, s_abort);
                        if (!ok) break;
                        ptx::mbar_expect_tx(bar_k_full + 8 * ks, Plan::kTile);
                        for (int d = 0; d < D; d += 64) ptx::tma_load_3d(smem_base + ks * Plan::kTile + d * 256, &tm_k, bar_k_full + 8 * ks, d, key0, g);
                        fresh = false;
                    }
                    const int qs = qt % kKwQStages;
                    if (qt >= kKwQStages) ok = wait_bounded(bar_q_empty + 8 * qs, ((qt / kKwQStages) & 1) ^ 1, kDevTimeoutProducer, a.status, s_abort);
                    if (!ok) break;
                    ptx::mbar_expect_tx(bar_q_full + 8 * qs, a.chunk_rows * D * 2);
                    for (int d = 0; d < D; d += 64)
                        ptx::tma_load_3d(smem_base + Plan::kQOff + qs * Plan::kChunk + d * (kKwRows * 2), &tm_q, bar_q_full + 8 * qs, d, c * a.chunk_rows, g);
                }
                if (fresh) --kt;                          // no chunk of this CTA's: the tile was not loaded
            }
            if (!ok || *s_abort) {
                const long long t0 = clock64();           // loads in flight land before the CTA may leave
                while (clock64() - t0 < 400000) { }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = make_idesc(false, 128, a.chunk_rows);
            const uint64_t kd0 = make_sdesc(smem_base, 16, 1024), qd0 = make_sdesc(smem_base + Plan::kQOff, 16, 1024);
            int kt = 0, qt = 0;
            for (int item = blockIdx.x; item < a.items && ok; item += stride) {
                int g;
                const int key0 = tile_of(item, g), ks = kt % kKwStages, c0 = first_chunk(a, key0) + rank;
                for (int c = c0; c < a.chunks; c += csize, ++qt) {
                    const int qs = qt % kKwQStages, buf = qt % kKwBufs;
                    if (c == c0) ok = wait_bounded(bar_k_full + 8 * ks, (kt / kKwStages) & 1, kDevTimeoutMmaKV, a.status, s_abort);
                    ok = ok && wait_bounded(bar_q_full + 8 * qs, (qt / kKwQStages) & 1, kDevTimeoutMmaQ, a.status, s_abort);
                    if (qt >= kKwBufs) ok = ok && wait_bounded(bar_s_free + 8 * buf, ((qt / kKwBufs) & 1) ^ 1, kDevTimeoutMmaP, a.status, s_abort);
                    if (!ok) break;
                    ptx::fence_after_sync();
                    const uint64_t kd = kd0 + (uint64_t)((ks * Plan::kTile) >> 4), qd = qd0 + (uint64_t)((qs * Plan::kChunk) >> 4);
#pragma unroll
                    for (int s = 0; s < D / 16; ++s) {
                        const uint64_t k_off = (uint64_t)(((s >> 2) * 64 * 256 + (s & 3) * 32) >> 4);
                        const uint64_t q_off = (uint64_t)(((s >> 2) * 64 * (kKwRows * 2) + (s & 3) * 32) >> 4);
                        ptx::mma_ss(tmem + buf * kKwRows, kd + k_off, qd + q_off, idesc, s > 0);
                    }
                    ptx::mma_commit(bar_s_full + 8 * buf);
                    ptx::mma_commit(bar_q_empty + 8 * qs);
                    if (c + csize >= a.chunks) ptx::mma_commit(bar_k_empty + 8 * ks);
                }
                if (c0 < a.chunks) ++kt;
            }
        }
        __syncwarp();
    } else if (warp < 4) {
        // the rows' log-sum-exps, negative and in base 2, of every second chunk: a row behind the last one counts as nothing
        int qt = 0;
        for (int item = blockIdx.x; item < a.items && ok; item += stride) {
            int g;
            const int key0 = tile_of(item, g);
            for (int c = first_chunk(a, key0) + rank; c < a.chunks && ok; c += csize, ++qt) {
                if ((qt & 1) != warp - 2) continue;
                const int buf = qt % kKwBufs, row0 = c * a.chunk_rows;
                float mine[kKwRows / 32];
#pragma unroll
                for (int i = 0; i < kKwRows / 32; ++i) {
                    const int r = row0 + 32 * i + lane, tok = (int)fast_div((uint32_t)r, a.div_g);
                    mine[i] = 32 * i < a.chunk_rows && r < a.rows ? a.lse[(long)tok * (a.Hkv * a.G) + g * a.G + (r - tok * a.G)] : INFINITY;
                }
                if (qt >= kKwBufs) ok = warp_wait(bar_l_free + 8 * buf, ((qt / kKwBufs) & 1) ^ 1, kDevTimeoutProducer, a.status, s_abort, lane);
                if (!ok) break;
#pragma unroll
                for (int i = 0; i < kKwRows / 32; ++i) s_lse[buf * kKwRows + 32 * i + lane] = mine[i] * -1.4426950408889634f;
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(bar_l_full + 8 * buf);
            }
        }
    } else {
        const int quarter = warp & 3, grp = (warp - 4) >> 2;
        const int key_lane = (quarter << 5) + lane;       // = TMEM lane = the thread's key within a tile
        const uint32_t t_lane = tmem + ((uint32_t)(quarter << 5) << 16);
        // one chunk a tile: the groups take the tiles in turn; else two take every second chunk, half of it each
        const bool turns = a.chunks == 1;
        const int col0 = turns ? 0 : (grp & 1) * (kKwRows / 2), col1 = turns ? a.chunk_rows : col0 + kKwRows / 2;
        const uint64_t scale2 = ptx::pack2(a.scale_log2, a.scale_log2);
        int qt = 0, kt = 0;                               // chunks, tiles
        for (int item = blockIdx.x; item < a.items; item += stride) {
            int g;
            const int key0 = tile_of(item, g), key = key0 + key_lane, c0 = first_chunk(a, key0) + rank;
            const bool writes = key < a.L + a.n && rank == 0 && grp == (turns ? kt % kKwGroups : 0);
            const float had = writes && key < a.L ? a.in[(long)g * a.cap + key] : 0.f;
            const int from = key > a.L ? (key - a.L) * a.G : 0;           // the first row that sees the key
            const bool edge = key0 + kTileN - 1 > a.L;                    // (uniform) some key of the tile is not seen by all
            uint64_t sum0 = 0, sum1 = 0;                                  // two floats each
            const int count = c0 < a.chunks ? (a.chunks - c0 + csize - 1) >> cshift : 0;
            const int first = turns ? (kt % kKwGroups == grp ? 0 : count) : ((grp >> 1) ^ qt) & 1;
            for (int i = first; i < count; i += 2) {
                const int at = qt + i, buf = at % kKwBufs, row0 = (c0 + i * csize) * a.chunk_rows, valid = min(a.chunk_rows, a.rows - row0);
                const uint32_t parity = (at / kKwBufs) & 1;
                const float* lse = s_lse + buf * kKwRows;
                const uint32_t have = ptx::mbar_try_wait(bar_l_full + 8 * buf, parity) & ptx::mbar_try_wait(bar_s_full + 8 * buf, parity);
                if (!__all_sync(0xffffffffu, have)) {                     // (seldom: and 0.2 us more)
                    ok = ok && warp_wait(bar_l_full + 8 * buf, parity, kDevTimeoutSoftmaxS, a.status, s_abort, lane);
                    ok = ok && warp_wait(bar_s_full + 8 * buf, parity, kDevTimeoutSoftmaxS, a.status, s_abort, lane);
                    __syncwarp();
                }
                if (!ok) break;
                ptx::fence_after_sync();
                const bool plain = !edge && valid == a.chunk_rows;
#pragma unroll 1
                for (int col = col0; col < col1; col += 32) {
                    uint32_t s[32];
                    ptx::tmem_ld32(t_lane + buf * kKwRows + col, s);
                    ptx::tmem_ld_wait();
                    if (col + 32 >= col1) {
                        ptx::fence_before_sync();
                        if (ptx::elect_one()) ptx::mbar_arrive(bar_s_free + 8 * buf);
                    }
                    const float4* l4 = reinterpret_cast<const float4*>(lse + col);
                    const int lo = from - row0 - col, hi = valid - col;   // columns lo .. hi-1 count
                    if (plain || __all_sync(0xffffffffu, lo <= 0 && hi >= 32)) {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 m = l4[e >> 2];
                            float x0, x1, x2, x3;
                            ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), scale2, ptx::pack2(m.x, m.y)), x0, x1);
                            ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(s[e + 2]), __uint_as_float(s[e + 3])), scale2, ptx::pack2(m.z, m.w)), x2, x3);
                            sum0 = ptx::add2(sum0, ptx::pack2(ptx::ex2(x0), ptx::ex2(x1)));
                            sum1 = ptx::add2(sum1, ptx::pack2(ptx::ex2(x2), ptx::ex2(x3)));
                        }
                    } else if (__any_sync(0xffffffffu, lo < 32 && hi > 0)) {
                        const uint32_t count_in = (hi >= 32 ? ~0u : hi <= 0 ? 0u : (1u << hi) - 1u) & (lo <= 0 ? ~0u : lo >= 32 ? 0u : ~0u << lo);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 m = l4[e >> 2];
                            const float in[4] = {m.x, m.y, m.z, m.w};
                            float x[4];
#pragma unroll
                            for (int o = 0; o < 4; ++o) {
                                const float x_all = ptx::ex2(fmaf(__uint_as_float(s[e + o]), a.scale_log2, in[o]));
                                x[o] = count_in & (1u << (e + o)) ? x_all : 0.f;
                            }
                            sum0 = ptx::add2(sum0, ptx::pack2(x[0], x[1]));
                            sum1 = ptx::add2(sum1, ptx::pack2(x[2], x[3]));
                        }
                    }
                }
                __syncwarp();
                if (ptx::elect_one()) ptx::mbar_arrive(bar_l_free + 8 * buf);
            }
            qt += count;
            float u0, u1, u2, u3;
            ptx::unpack2(sum0, u0, u1);
            ptx::unpack2(sum1, u2, u3);
            float sum = (u0 + u1) + (u2 + u3);
            if (!turns) {
                float* part = s_part + (kt & 1) * ((kKwGroups - 1) * 128) + key_lane;
                if (grp > 0) part[(grp - 1) * 128] = sum;
                asm volatile("bar.sync 1, %0;" :: "n"(128 * kKwGroups) : "memory");
                if (grp == 0)
#pragma unroll
                    for (int o = 0; o < kKwGroups - 1; ++o) sum += part[o * 128];
            }
            if (csize > 1) own_sum = sum;
            else if (writes && ok) a.out[(long)g * a.cap + key] = fmaf(had, a.decay, sum);
            ++kt;
        }
    }
    if (csize > 1) {
        // one tile per cluster: the sums of the other CTAs come to the first one's shared memory
        const int key_lane = ((warp & 3) << 5) + lane;
        __syncwarp();
        ptx::cluster_wait();
        if (warp >= 4 && warp < 8 && rank > 0) {
            const uint32_t to = ptx::map_to_cta(smem_base + Plan::kRemoteOff + (rank * 128 + key_lane) * 4, 0);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(own_sum) : "memory");
        }
        __syncwarp();
        ptx::cluster_arrive();
        ptx::cluster_wait();
        if (warp >= 4 && warp < 8 && rank == 0) {
            int g;
            const int key = tile_of(blockIdx.x, g) + key_lane;
            float sum = own_sum;
            for (int r = 1; r < csize; ++r) sum += s_remote[r * 128 + key_lane];
            if (key < a.L + a.n && ok) a.out[(long)g * a.cap + key] = (key < a.L ? a.in[(long)g * a.cap + key] * a.decay : 0.f) + sum;
        }
    }
    ptx::fence_before_sync();
    __syncthreads();
    if (warp == 1) ptx::tmem_dealloc(tmem, 512);
}

// ---- fp32: a thread per key -------------------------------------------------------------------
constexpr int kKwF32Keys = 128, kKwF32Rows = 16;          // keys of a block, query rows staged at a time
template <int D>
__global__ void __launch_bounds__(kKwF32Keys)
key_weights_f32_kernel(const KeyWeightArgs a)
{
    __shared__ __align__(16) float s_q[kKwF32Rows][D];
    __shared__ float s_lse[kKwF32Rows];
    __shared__ float s_remote[kKwMaxCluster][kKwF32Keys];
    const int csize = (int)gridDim.y, rank = (int)blockIdx.y;
    const int t = (int)fast_div(blockIdx.x, a.div_hkv), g = (int)blockIdx.x - t * a.Hkv;
    const int key0 = t * kKwF32Keys, key = key0 + (int)threadIdx.x, total = a.L + a.n;
    if (csize > 1) ptx::cluster_arrive_relaxed();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    float k[D];
    {
        const float4* row = reinterpret_cast<const float4*>((const float*)a.k_cache + ((long)g * a.cap + min(key, total - 1)) * D);
#pragma unroll
        for (int d = 0; d < D; d += 4) {
            const float4 v = row[d >> 2];
            k[d] = v.x; k[d + 1] = v.y; k[d + 2] = v.z; k[d + 3] = v.w;
        }
    }
    const int from = key > a.L ? (key - a.L) * a.G : 0;   // the first row that sees the key
    float sum = 0.f;
    for (int c = first_chunk(a, key0) + rank; c < a.chunks; c += csize) {
        const int row0 = c * kKwF32Rows, valid = min(kKwF32Rows, a.rows - row0);
        __syncthreads();
        const float4* src = reinterpret_cast<const float4*>((const float*)a.q_rot + ((long)g * a.rows + row0) * D);
        for (int e = threadIdx.x; e < valid * D / 4; e += kKwF32Keys) reinterpret_cast<float4*>(&s_q[0][0])[e] = src[e];
        if ((int)threadIdx.x < valid) {
            const int r = row0 + (int)threadIdx.x, i = (int)fast_div((uint32_t)r, a.div_g);
            s_lse[threadIdx.x] = a.lse[(long)i * (a.Hkv * a.G) + g * a.G + (r - i * a.G)] * 1.4426950408889634f;
        }
        __syncthreads();
        for (int r = 0; r < valid; ++r) {
            float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
#pragma unroll
            for (int d = 0; d < D; d += 4) {
                const float4 q = *reinterpret_cast<const float4*>(&s_q[r][d]);
                s0 = fmaf(q.x, k[d], s0); s1 = fmaf(q.y, k[d + 1], s1); s2 = fmaf(q.z, k[d + 2], s2); s3 = fmaf(q.w, k[d + 3], s3);
            }
            const float p = exp2f(fmaf((s0 + s1) + (s2 + s3), a.scale_log2, -s_lse[r]));
            sum += row0 + r >= from ? p : 0.f;
        }
    }
    if (csize > 1) {
        ptx::cluster_wait();
        if (rank > 0) {
            const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_remote[rank][threadIdx.x]), 0);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(sum) : "memory");
        }
        ptx::cluster_arrive();
        ptx::cluster_wait();
        if (rank > 0) return;
        for (int r = 1; r < csize; ++r) sum += s_remote[r][threadIdx.x];
    }
    if (key < total) a.out[(long)g * a.cap + key] = (key < a.L ? a.in[(long)g * a.cap + key] * a.decay : 0.f) + sum;
}

// ---- fp32, many rows and keys: a matrix product in registers ---------------------------------
// A thread of the kernel above loads four numbers of a query row for four FMAs, and the loads bind (448 rows of 4 heads over 4096 keys 121 us,
// 15.8 TFLOP/s).  Here a thread owns 8 keys and 8 rows, whose vectors come out of shared memory four channels at a time: 256 FMAs for 16 loads (78 us:
// now latency, two blocks of four warps an SM).  A warp: 128 keys x 16 rows; a block: a tile of keys, 64 rows at a time.
constexpr int kKwTileRows = 64, kKwTileLeastRows = 32;
template <int D>
struct KwTilePlan {
    static constexpr int kRow = D + 4;                    // floats between rows: eight lanes' 16 bytes start in different banks
    static constexpr int kQOff = kTileN * kRow, kLseOff = kQOff + kKwTileRows * kRow, kSumOff = kLseOff + kKwTileRows;      // floats
    static constexpr int kRemoteOff = kSumOff + 4 * kTileN, kBytes = (kRemoteOff + kKwMaxCluster * kTileN) * 4;
};

template <int D>
__global__ void __launch_bounds__(128, 2)
key_weights_tile_kernel(const KeyWeightArgs a)
{
    using Plan = KwTilePlan<D>;
    constexpr int ROW = Plan::kRow, V = D / 4;
    extern __shared__ __align__(16) float s_all[];
    float* s_q = s_all + Plan::kQOff;
    float* s_lse = s_all + Plan::kLseOff;
    float* s_sum = s_all + Plan::kSumOff;
    float* s_remote = s_all + Plan::kRemoteOff;
    const int csize = (int)gridDim.y, rank = (int)blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int t = (int)fast_div(blockIdx.x, a.div_hkv), g = (int)blockIdx.x - t * a.Hkv;
    const int key0 = t * kTileN, total = a.L + a.n;
    if (csize > 1) ptx::cluster_arrive_relaxed();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    for (int e = tid; e < kTileN * V; e += 128) {
        const int r = e / V, c = e % V;
        const float4* row = reinterpret_cast<const float4*>((const float*)a.k_cache + ((long)g * a.cap + min(key0 + r, total - 1)) * D);
        *reinterpret_cast<float4*>(s_all + r * ROW + 4 * c) = row[c];
    }
    const int kl = lane & 15, my_row = warp * 16 + (lane >> 4) * 8;        // the thread's keys: kl + 16 j, rows my_row + i
    float sums[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[j] = 0.f;
    for (int c = first_chunk(a, key0) + rank; c < a.chunks; c += csize) {
        const int row0 = c * kKwTileRows;
        __syncthreads();
        for (int e = tid; e < kKwTileRows * V; e += 128) {
            const int r = e / V, d = e % V;
            const float4* row = reinterpret_cast<const float4*>((const float*)a.q_rot + ((long)g * a.rows + row0 + r) * D);
            *reinterpret_cast<float4*>(s_q + r * ROW + 4 * d) = row0 + r < a.rows ? row[d] : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        if (tid < kKwTileRows && row0 + tid < a.rows) {
            const int r = row0 + tid, i = (int)fast_div((uint32_t)r, a.div_g);
            s_lse[tid] = a.lse[(long)i * (a.Hkv * a.G) + g * a.G + (r - i * a.G)] * 1.4426950408889634f;
        }
        __syncthreads();
        if (row0 + warp * 16 >= a.rows) continue;         // (whole warps; the barriers above are reached by all)
        float s[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[i][j] = 0.f;
#pragma unroll 1
        for (int d = 0; d < D; d += 4) {
            float4 k[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) k[j] = *reinterpret_cast<const float4*>(s_all + (kl + 16 * j) * ROW + d);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 q = *reinterpret_cast<const float4*>(s_q + (my_row + i) * ROW + d);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[i][j] = fmaf(q.x, k[j].x, fmaf(q.y, k[j].y, fmaf(q.z, k[j].z, fmaf(q.w, k[j].w, s[i][j]))));
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = row0 + my_row + i;
            const float l = s_lse[my_row + i];
            if (r >= a.rows) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int key = key0 + kl + 16 * j;       // row r sees keys up to L + r / G
                if (r >= max(key - a.L, 0) * a.G) sums[j] += exp2f(fmaf(s[i][j], a.scale_log2, -l));
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        sums[j] += __shfl_xor_sync(0xffffffffu, sums[j], 16);
        if (lane < 16) s_sum[warp * kTileN + kl + 16 * j] = sums[j];
    }
    __syncthreads();
    float sum = (s_sum[tid] + s_sum[kTileN + tid]) + (s_sum[2 * kTileN + tid] + s_sum[3 * kTileN + tid]);
    if (csize > 1) {
        ptx::cluster_wait();
        if (rank > 0) {
            const uint32_t to = ptx::map_to_cta(ptx::smem_u32(s_remote + rank * kTileN + tid), 0);
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(sum) : "memory");
        }
        ptx::cluster_arrive();
        ptx::cluster_wait();
        if (rank > 0) return;
        for (int r = 1; r < csize; ++r) sum += s_remote[r * kTileN + tid];
    }
    const int key = key0 + tid;
    if (key < total) a.out[(long)g * a.cap + key] = (key < a.L ? a.in[(long)g * a.cap + key] * a.decay : 0.f) + sum;
}

}  // namespace evln
