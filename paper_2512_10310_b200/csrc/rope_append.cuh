// Fused RoPE-rotate-and-append kernel (Sec. 3.2: contiguous position ids, rotation,
// concatenation of the new frame with the reused cache).
//
// One CTA per new token.  D/2 threads get the token's cos/sin of phi_j = pos * theta^(-2j/D) in double
// precision (pos reaches tens of thousands; a float angle would be off by ~1e-3 rad) into shared memory
// for all heads: from the caller's position table when there is one (the table depends on the positions
// only, so a model makes it once per navigation step for all its layers: rope_table_kernel below), else
// formed on the spot.  Every thread moves 16-byte vectors (a work item is a pair of vectors (j.., j + D/2..)
// of a query or key head, or one vector of a value head): rotated query halves to the kv-head-grouped
// q_rot scratch, rotated key halves and the unchanged values to the token's cache slot; the loads are
// issued before the cos/sin are waited for.
// Bound: a step's few hundred tokens are one chain of latencies (2.3 us for 196 tokens of the 7B shape,
// 1.8 for one; 3.4 and 2.6 before the rotation was packed), thousands are bound by the instructions of
// the rotation and then by HBM (each element read once and written once: 2048 tokens 9.8 us, 3136 paged
// ones 17.6, 16 and 25 before; 6 and 9 us at the copy rate).
// (Letting every thread read the table entries of its own vector instead of sharing them through shared
// memory was measured slower: 32 heads re-read the same 64 entries.)
#pragma once

#include "common.cuh"
#include "ptx_sm100.cuh"
#include "rotation.cuh"

namespace evln {

// Position table: entry (p, j) = (cos, sin) of (first_pos + p) * theta^(-2j/D).
__global__ void __launch_bounds__(128)
rope_table_kernel(double2* table, int first_pos, int count, int D, double log2_theta)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int half = D / 2;
    const long i = (long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (long)count * half) return;
    const int p = (int)(i / half), j = (int)(i % half);
    table[i] = rope_cos_sin((long)first_pos + p, j, D, log2_theta);
}

// LensT is BatchLens for the paged kernel and NoLens (a stub) for the contiguous one.

// Where one new token comes from and goes to.
struct TokenPlace {
    int src_tok;             // its row of q_new / k_new / v_new
    int m;                   // its number in its run: query rows m * G ..
    int episode;             // paged: its episode; packed: 1 for an action token
    long kv_row;             // its key / value row of kv head 0
};
// The buffers a token's run goes to.
template <typename T>
struct TokenRun {
    T* q;                    // [Hkv, q_rows, D]
    T* k;                    // rows of kv head g start kv_rows * g behind those of head 0
    T* v;
    long q_rows, kv_rows;
};

// Rotates and stores token blockIdx.x with the whole block (gridDim.y > 1: a share of its work items).  place(token, t) fills in the token's place and
// returns its position, run(t) says which buffers it goes to.
template <typename T, typename Place, typename Run>
__device__ __forceinline__ void rope_token(const RopeArgs& a, Place&& place, Run&& run)
{
    constexpr int V = VecTraits<T>::kVec;
    typedef typename Rotation<T>::Angle Angle;
    __shared__ Angle s_angle[Rotation<T>::kAngles];
    const int D = a.D, half = D / 2, G = a.G;
    const int vph = a.vph_shift, vpr = a.vph_shift + 1;       // vectors per half head vector / per head vector (log2)
    const int q_items = a.Hq << vph;
    const int k_items = a.Hkv << vph;
    const int v_items = a.Hkv << vpr;
    const int items = q_items + k_items + v_items;

    // a work item `it` of a token: a pair of 16-byte vectors (j0.., j0+half..) of a query or key head, or one
    // 16-byte vector of a value head
    auto load_item = [&](const TokenPlace& t, int it, uint4& r0, uint4& r1) {
        if (it < q_items + k_items) {
            const bool is_q = it < q_items;
            const int e = is_q ? it : it - q_items;
            const int h = e >> vph;
            const int j0 = (e & ((1 << vph) - 1)) * V;
            const T* src = (is_q ? (const T*)a.q_new + t.src_tok * a.q_stride : (const T*)a.k_new + t.src_tok * a.k_stride) + (long)h * D;
            r0 = *reinterpret_cast<const uint4*>(src + j0);
            r1 = *reinterpret_cast<const uint4*>(src + j0 + half);
        } else {
            const int e = it - q_items - k_items;
            const int g = e >> vpr;
            const int d0 = (e & ((1 << vpr) - 1)) * V;
            r0 = *reinterpret_cast<const uint4*>((const T*)a.v_new + t.src_tok * a.v_stride + (long)g * D + d0);
        }
    };
    auto finish_item = [&](const TokenPlace& t, const Angle* s_angle, int it, const uint4& lo_raw, const uint4& hi_raw) {
        const TokenRun<T> to = run(t);
        if (it < q_items + k_items) {
            const bool is_q = it < q_items;
            const int e = is_q ? it : it - q_items;
            const int h = e >> vph;
            const int j0 = (e & ((1 << vph) - 1)) * V;
            T* dst;
            if (is_q) {
                const int g = (int)fast_div((uint32_t)h, a.div_g);
                dst = to.q + ((long)g * to.q_rows + (long)t.m * G + (h - g * G)) * D;
            } else {
                dst = to.k + ((long)h * to.kv_rows + t.kv_row) * D;
            }
            uint4 out_lo_raw, out_hi_raw;
            Rotation<T>::turn(s_angle, e & ((1 << vph) - 1), lo_raw, hi_raw, out_lo_raw, out_hi_raw);
            *reinterpret_cast<uint4*>(dst + j0) = out_lo_raw;
            *reinterpret_cast<uint4*>(dst + j0 + half) = out_hi_raw;
        } else {
            const int e = it - q_items - k_items;
            const int g = e >> vpr;
            const int d0 = (e & ((1 << vpr) - 1)) * V;
            *reinterpret_cast<uint4*>(to.v + ((long)g * to.kv_rows + t.kv_row) * D + d0) = lo_raw;
        }
    };

    const int j = threadIdx.x;
    // without a table: the thread's frequency, once (j / D as in rope_cos_sin)
    const double omega = !a.table && j < half ? rope_omega(j, D, a.log2_theta) : 0.0;
    auto angle_of = [&](long pos) -> double2 {
        return a.table ? a.table[(pos - a.table_first) * half + j] : rope_cos_sin_at(pos, omega);
    };

    const int tok = blockIdx.x;
    TokenPlace t;
    const long pos = place(tok, t);
    uint4 r0 = make_uint4(0u, 0u, 0u, 0u), r1 = r0;
    const int first = j + (int)(blockIdx.y * blockDim.x);
    if (first < items) load_item(t, first, r0, r1);   // in flight while the angles arrive
    if (j < half) Rotation<T>::put(s_angle, j, angle_of(pos));
    __syncthreads();
    if (first < items) finish_item(t, s_angle, first, r0, r1);
    for (int it = first + (int)(gridDim.y * blockDim.x); it < items; it += (int)(gridDim.y * blockDim.x)) {
        load_item(t, it, r0, r1);
        finish_item(t, s_angle, it, r0, r1);
    }
}

// FEW: at most kRopeFewTokens tokens.  Their blocks are all there while the previous kernel ends, so each requests its token's
// vectors into L2 meanwhile.  (28 layers of 256 tokens on an empty cache 277 us a pass, 271 so; 8 tokens over 20656 505 and 497.
// Many tokens, whose blocks are in line, 22.4 us for 21.8 of a step of 1024.)
template <typename T, bool PAGED, typename LensT, bool FEW>
__global__ void __launch_bounds__(kRopeThreadsMax, PAGED ? 3 : 1)
rope_append_kernel(const RopeArgs a, const __grid_constant__ LensT lens)
{
    constexpr int V = VecTraits<T>::kVec;
    const int D = a.D;
    int b = 0;                                    // the token's episode
    if (PAGED && (int)blockIdx.x >= a.num_new) {
        // An episode's last page is only partly filled: clear the value slots behind its last token so that a
        // tile load of the whole page never brings in stale bits.  (A block per episode: behind the stores of
        // the last token's block it was the longest chain of the launch, 4.65 us for 16 episodes of one token.)
        b = blockIdx.x - a.num_new;
        const int len = lens.cache_len[b] + lens.new_off[b + 1] - lens.new_off[b], used = len & (a.page_size - 1);
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
        if (lens.new_off[b + 1] == lens.new_off[b] || used == 0) return;
        const long row = (long)a.page_table[(long)b * a.max_pages + (len >> a.page_shift)] * a.Hkv * a.page_size + used;
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int g = blockIdx.y; g < a.Hkv; g += gridDim.y) {
            uint4* dst = reinterpret_cast<uint4*>((T*)a.v_cache + (row + (long)g * a.page_size) * D);
            for (int it = threadIdx.x; it < (a.page_size - used) * (D / V); it += blockDim.x) dst[it] = zero;
        }
        return;
    }
    if (PAGED) {
        int hi = a.batch;                         // largest b with new_off[b] <= tok
        while (hi - b > 1) {
            const int mid = (b + hi) >> 1;
            if (lens.new_off[mid] <= (int)blockIdx.x) b = mid; else hi = mid;
        }
    }
    if constexpr (FEW) {
        const int tok = blockIdx.x, lines = D * (int)sizeof(T) / 128, q = a.Hq * lines, kv = a.Hkv * lines;
        for (int i = (int)(blockIdx.y * blockDim.x + threadIdx.x); i < q + 2 * kv; i += (int)(gridDim.y * blockDim.x)) {
            const T* row = i < q ? (const T*)a.q_new + tok * a.q_stride : i < q + kv ? (const T*)a.k_new + tok * a.k_stride : (const T*)a.v_new + tok * a.v_stride;
            ptx::prefetch_l2(reinterpret_cast<const char*>(row) + (i < q ? i : i < q + kv ? i - q : i - q - kv) * 128);
        }
    }
    // (so far launch parameters only; what follows reads memory that earlier kernels may have written)
    asm volatile("griddepcontrol.wait;" ::: "memory");          // programmatic dependent launch: inputs ready
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto place = [&](int tok, TokenPlace& t) -> long {          // tok: index into the packed new tokens
        t.src_tok = t.m = tok;
        if (!PAGED) return t.kv_row = (long)a.cache_len + tok;
        const int pos = lens.cache_len[b] + tok - lens.new_off[b];
        t.episode = b;
        t.kv_row = (long)a.page_table[(long)b * a.max_pages + (pos >> a.page_shift)] * a.Hkv * a.page_size + (pos & (a.page_size - 1));
        return pos;
    };
    auto run = [&](const TokenPlace&) -> TokenRun<T> {
        return {(T*)a.q_rot, (T*)a.k_cache, (T*)a.v_cache, (long)a.num_new * a.G, PAGED ? (long)a.page_size : (long)a.cache_cap};
    };
    rope_token<T>(a, place, run);
}

// The tokens of a packed sequence I, v_1, a_1, ..., v_N, a_N in one launch (Sec. 3.3): the instruction and
// visual tokens at contiguous positions into the cache, then the action tokens, chunk t at the positions
// that continue v_t, into buffers of their own.
struct RopePackedArgs {
    RopeArgs r;              // visual run: q_rot, k_cache, v_cache, cache_cap; num_new = all tokens
    int num_visual, num_action;
    int I, F, A;
    FastDiv div_f, div_a;
    void* q_rot_act;         // [Hkv, num_action * G, D]
    void* k_act;             // [Hkv, num_action, D]
    void* v_act;
};

__global__ void __launch_bounds__(kRopeThreadsMax, 3)
rope_packed_kernel(const RopePackedArgs p)
{
    typedef __nv_bfloat16 T;
    const RopeArgs& a = p.r;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    auto place = [&](int tok, TokenPlace& t) -> long {
        const bool action = tok >= p.num_visual;
        const int m = action ? tok - p.num_visual : tok;             // within its run
        long pos = m;
        t.src_tok = m;
        if (action) {
            const int c = (int)fast_div((uint32_t)m, p.div_a), i = m - c * p.A;
            pos = (long)p.I + (long)(c + 1) * p.F + i;
            t.src_tok = p.I + c * (p.F + p.A) + p.F + i;
        } else if (m >= p.I && p.F > 0) {
            t.src_tok += (int)fast_div((uint32_t)(m - p.I), p.div_f) * p.A;
        }
        t.m = m;
        t.kv_row = m;
        t.episode = action;
        return pos;
    };
    auto run = [&](const TokenPlace& t) -> TokenRun<T> {
        if (t.episode) return {(T*)p.q_rot_act, (T*)p.k_act, (T*)p.v_act, (long)p.num_action * a.G, p.num_action};
        return {(T*)a.q_rot, (T*)a.k_cache, (T*)a.v_cache, (long)p.num_visual * a.G, a.cache_cap};
    };
    rope_token<T>(a, place, run);
}

}  // namespace evln
