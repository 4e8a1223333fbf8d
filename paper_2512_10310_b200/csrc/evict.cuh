// Eviction: which keys of a kv head to keep, by weight, and the chosen ones laid out anew.
//
// select_keys_kernel: a cluster of blocks per kv head, each with a run of its slots (one block where they are few).  The threshold is the m-th
// largest of the weights in the open range, found digit by digit (11, 11 and 10 bits of the float as an ordered integer): each block
// counts its keys' digits in shared memory, and the blocks read one another's counts over distributed shared memory, first 64 sums of 32 digits, then the
// 32 digits in question.  Then one ordered pass writes the slots above the threshold, of those equal to it the lowest, and the protected ends,
// ascending: every thread counts its run of slots, and scans over the counts give them their places.
// Most often the keys with the first 22 bits of the threshold are all kept, and the last digit is not looked for.
// Bound: latency: loads, meetings of the cluster (0.6 us each, one per digit), reads of other
// blocks' counts (0.3 us each, so never one after the other); loops stay rolled.  (20656 keys of 4 heads: one block per head
// 15 us, 21 with its keys in registers and everything unrolled; eight blocks that read all 2048 counts of all, 13.)
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
    int slice;               // slots of a block
    int cached;              // a slice fits the block's shared memory
};

constexpr int kSelectThreads = 512, kSelectBins = 2048, kSelectCluster = 8, kSelectGroups = 64;      // groups of 32 digits
constexpr int kSelectSlice = 4096;                        // most slots that one block takes alone
constexpr int kSelectCache = 40 * 1024;                   // most slots of a slice held in shared memory

// floats in order as unsigned integers; -0 as 0, NaN as -infinity
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = x != x ? 0xff800000u : __float_as_uint(x + 0.f);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Inclusive sums over the lanes of a warp.
__device__ __forceinline__ int warp_scan(int x)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if ((int)(threadIdx.x & 31) >= o) x += y;
    }
    return x;
}

// The cluster's blocks meet; what any of their threads wrote to shared memory before is visible to all after it (one warp's cluster-wide release
// covers what the block's own meeting ordered before it).
__device__ __forceinline__ void cluster_meet()
{
    __syncthreads();
    if (threadIdx.x < 32) ptx::cluster_arrive();
    else ptx::cluster_arrive_relaxed();
    ptx::cluster_wait();
}
__device__ __forceinline__ int ld_cluster_int(const int* shared, int rank)
{
    return __float_as_int(ptx::ld_cluster_f32(ptx::map_to_cta(ptx::smem_u32(shared), rank)));
}

// grid (kv heads, cluster): blockIdx.y is the block's rank in its cluster.
__global__ void __launch_bounds__(kSelectThreads, 1)
select_keys_kernel(const SelectArgs a)
{
    extern __shared__ uint32_t s_key[];                   // [slice] where it fits
    __shared__ __align__(16) int s_bin[3][kSelectBins];
    __shared__ int s_group[3][kSelectGroups], s_sum[kSelectGroups], s_digit[32];
    __shared__ int s_sure[kSelectThreads / 32], s_same[kSelectThreads / 32], s_total[2];
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, csize = gridDim.y, rank = blockIdx.y;
    const float* w = a.weights + (long)g * a.stride;
    const int lo = a.sinks, hi = a.num_keys - a.recent;   // the open range
    const int first = min(a.num_keys, rank * a.slice), last = min(a.num_keys, first + a.slice);      // this block's slots
    for (int i = tid; i < 3 * kSelectBins / 4; i += kSelectThreads) reinterpret_cast<int4*>(s_bin)[i] = make_int4(0, 0, 0, 0);
    __syncthreads();
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const bool search = a.num_kept < a.num_keys && a.open > 0, all = a.num_kept == a.num_keys;
    const int from = max(lo, first), to = min(hi, last);  // of them open
    uint32_t prefix = 0;
    int left = a.open;                                    // still to be found among the keys with this prefix
    if (search) {
        // the keys, and their first digits: eight loads in flight
        constexpr int kBatch = 8;
        for (int base = from + tid; base < to; base += kBatch * kSelectThreads) {
            float x[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) x[i] = base + i * kSelectThreads < to ? w[base + i * kSelectThreads] : 0.f;
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int j = base + i * kSelectThreads;
                if (j >= to) break;
                const uint32_t k = ordered(x[i]);
                if (a.cached) s_key[j - first] = k;
                atomicAdd(&s_bin[0][k >> 21], 1);
            }
        }
    }
    auto key = [&](int j) -> uint32_t { return a.cached ? s_key[j - first] : ordered(w[j]); };
    for (int pass = 0; search && pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above = pass == 1 ? 21 : 10;
        if (pass > 0) {
#pragma unroll 4
            for (int j = from + tid; j < to; j += kSelectThreads) {
                const uint32_t k = key(j);
                if (k >> above == prefix >> above) atomicAdd(&s_bin[pass][(k >> shift) & (pass == 2 ? 1023 : 2047)], 1);
            }
        }
        __syncthreads();
        {   // sums of 32 digits, eight lanes of four each
            const int4 n = *reinterpret_cast<const int4*>(&s_bin[pass][4 * tid]);
            int sum = n.x + n.y + n.z + n.w;
            for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if ((lane & 7) == 0) s_group[pass][tid >> 3] = sum;
        }
        if (csize > 1) {
            cluster_meet();
            int sum = ld_cluster_int(&s_group[pass][tid >> 3], tid & 7);
            for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if ((lane & 7) == 0) s_sum[tid >> 3] = sum;
        }
        __syncthreads();
        // every warp for itself: the group in which the count from the largest digit down reaches `left` (lane: two groups), then the digit
        const int* sums = csize > 1 ? s_sum : s_group[pass];
        const int g0 = kSelectGroups - 1 - 2 * lane, n0 = sums[g0], n1 = sums[g0 - 1], upto = warp_scan(n0 + n1);
        const int who = __ffs(__ballot_sync(0xffffffffu, upto >= left)) - 1;
        int group = g0, before = upto - n0 - n1;
        if (before + n0 < left) { --group; before += n0; }
        group = __shfl_sync(0xffffffffu, group, who);
        before = __shfl_sync(0xffffffffu, before, who);
        int n;
        if (csize > 1) {                                  // (a lane that reads all eight blocks' counts, one after the other: 2.4 us a pass)
            if (tid < 32 * kSelectCluster) {
                int part = ld_cluster_int(&s_bin[pass][32 * group + (tid >> 3)], tid & 7);
                for (int o = 1; o < 8; o <<= 1) part += __shfl_xor_sync(0xffffffffu, part, o);
                if ((lane & 7) == 0) s_digit[tid >> 3] = part;
            }
            __syncthreads();
            n = s_digit[31 - lane];
        } else {
            n = s_bin[pass][32 * group + 31 - lane];
        }
        const int sum = warp_scan(n), at = __ffs(__ballot_sync(0xffffffffu, before + sum >= left)) - 1;
        prefix |= (uint32_t)(32 * group + 31 - at) << shift;
        left -= before + __shfl_sync(0xffffffffu, sum - n, at);
        if (__shfl_sync(0xffffffffu, n, at) == left) {    // all with this prefix are kept: what is left of the digits does not matter
            --prefix;                                     // (no key is below -infinity's, so no prefix is 0)
            left = 0;
            break;
        }
    }
    // ---- places: every thread a run of neighbouring slots ----
    const int per = (a.slice + kSelectThreads - 1) / kSelectThreads, j0 = min(last, first + tid * per), j1 = min(last, j0 + per);
    auto look = [&](int j, bool& certain, bool& equal) {  // kept for certain, equal to the threshold
        const bool open = j >= from && j < to;
        const uint32_t k = open && search ? key(j) : 0u;
        certain = !open || all || (search && k > prefix);
        equal = search && open && k == prefix;
    };
    int sure = 0, same = 0;
#pragma unroll 2
    for (int j = j0; j < j1; ++j) {
        bool certain, equal;
        look(j, certain, equal);
        sure += certain;
        same += equal;
    }
    const int sure_upto = warp_scan(sure), same_upto = warp_scan(same);
    if (lane == 31) {
        s_sure[warp] = sure_upto;
        s_same[warp] = same_upto;
    }
    __syncthreads();
    const int sure_warps = warp_scan(lane < kSelectThreads / 32 ? s_sure[lane] : 0), same_warps = warp_scan(lane < kSelectThreads / 32 ? s_same[lane] : 0);
    if (tid == 31) {
        s_total[0] = sure_warps;
        s_total[1] = same_warps;
    }
    sure = sure_upto - sure;                              // before this thread's slots
    same = same_upto - same;
    const int sure_before = __shfl_sync(0xffffffffu, sure_warps, max(warp - 1, 0)), same_before = __shfl_sync(0xffffffffu, same_warps, max(warp - 1, 0));
    if (warp > 0) {
        sure += sure_before;
        same += same_before;
    }
    if (csize > 1) {
        cluster_meet();
        int x = lane < 2 * kSelectCluster && (lane & 7) < rank ? ld_cluster_int(&s_total[lane >> 3], lane & 7) : 0;      // sure, then same
        for (int o = 1; o < 8; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        sure += __shfl_sync(0xffffffffu, x, 0);
        same += __shfl_sync(0xffffffffu, x, 8);
    }
    int* out = a.kept + (long)g * a.num_kept;
#pragma unroll 2
    for (int j = j0; j < j1; ++j) {
        bool certain, equal;
        look(j, certain, equal);
        if (certain || (equal && same < left)) out[sure + min(same, left)] = j;
        sure += certain;
        same += equal;
    }
    if (csize > 1) {
        ptx::cluster_arrive_relaxed();                    // nobody leaves while another block may read its counts
        ptx::cluster_wait();
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
    double omega[6];         // theta^(-2 2^b / D): a frequency is a product of them
    const double2* table;    // optional
    int table_first;
    int vph_shift;           // log2 of the 16-byte vectors per half head vector
    int log_slots;           // log2 of a block's working slots
};

constexpr int kGatherKeysThreads = 256, kGatherKeysBlocks = 4, kGatherKeysSlots = 16;      // most slots of a block
template <typename T>
__global__ void __launch_bounds__(kGatherKeysThreads, kGatherKeysBlocks)
gather_keys_kernel(const GatherKeysArgs a)
{
    constexpr int V = VecTraits<T>::kVec;
    __shared__ __align__(16) typename Rotation<T>::Angle s_angle[kGatherKeysSlots][Rotation<T>::kAngles];
    const int D = a.D, half = D / 2, tid = threadIdx.x, vph = a.vph_shift;
    const int log_slots = a.log_slots, p0 = blockIdx.x << log_slots, j = tid & (half - 1);
    const int slots = min(1 << log_slots, a.num_kept - p0), first_slot = tid >> (D == 128 ? 6 : 5), step = kGatherKeysThreads / half;
    // Without a table the angles hang on launch parameters only and are formed ahead of the wait: a sine and cosine in double precision, 80
    // instructions, of theta^(-2 j / D) as a product of at most six powers (an exponential, 70 more).
    if (a.rotate && !a.table) {
        double omega = 1.0;
#pragma unroll
        for (int b = 0; b < 6; ++b)
            if ((j >> b) & 1) omega *= a.omega[b];
#pragma unroll 1
        for (int s = first_slot; s < slots; s += step) Rotation<T>::put(s_angle[s], j, rope_cos_sin_at(p0 + s, omega));
    }
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    // A work item: a pair of 16-byte vectors (channels e V .., + D/2) of a slot's key or value of one head; a key's lanes, then a value's.
    const int items = a.Hkv << (log_slots + vph + 1);
    struct Item { uint4 x0, x1; long dst; bool there; };
    auto load = [&](int it) -> Item {
        const int row = it >> (vph + 1), e = it & ((1 << vph) - 1), p = p0 + (row & ((1 << log_slots) - 1)), g = row >> log_slots;
        Item i;
        i.x0 = i.x1 = make_uint4(0u, 0u, 0u, 0u);
        i.dst = 0;
        i.there = it < items && p < a.num_kept;
        if (!i.there) return i;
        const int from = a.kept[(long)g * a.num_kept + p];
        const bool good = (unsigned)from < (unsigned)a.src_cap, is_v = (it >> vph) & 1;
        i.dst = ((long)g * a.dst_cap + p) * D + e * V;
        if (good) {
            const T* src = (const T*)(is_v ? a.v_src : a.k_src) + ((long)g * a.src_cap + from) * D + e * V;
            i.x0 = *reinterpret_cast<const uint4*>(src);
            i.x1 = *reinterpret_cast<const uint4*>(src + half);
        }
        if (e == 0 && is_v && a.w_src) a.w_dst[(long)g * a.dst_cap + p] = good ? a.w_src[(long)g * a.src_cap + from] : 0.f;
        return i;
    };
    Item next = load(tid);                                // in flight while the table is read
    if (a.rotate) {
        if (a.table)
            for (int s = first_slot; s < slots; s += step) Rotation<T>::put(s_angle[s], j, a.table[(long)(p0 + s - a.table_first) * half + j]);
        __syncthreads();
    }
    for (int it = tid; it < items; it += kGatherKeysThreads) {
        const Item i = next;
        next = load(it + kGatherKeysThreads);
        if (!i.there) continue;
        const bool is_v = (it >> vph) & 1;
        uint4 y0 = i.x0, y1 = i.x1;
        if (a.rotate && !is_v) Rotation<T>::turn(s_angle[(it >> (vph + 1)) & ((1 << log_slots) - 1)], it & ((1 << vph) - 1), i.x0, i.x1, y0, y1);
        T* to = (T*)(is_v ? a.v_dst : a.k_dst) + i.dst;
        *reinterpret_cast<uint4*>(to) = y0;
        *reinterpret_cast<uint4*>(to + half) = y1;
    }
}

}  // namespace evln
