// C-ABI entry points of the operators around the cache (contract: include/evln.h): norms of queries and keys with the append,
// the cache in 8 bits, and eviction by attention weight.  Host-side checks, schedules and launches.
#include "../../include/evln.h"

#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <utility>

#include "attn8.cuh"
#include "cache8.cuh"
#include "common.cuh"
#include "context.cuh"
#include "evict.cuh"
#include "head_norm.cuh"
#include "key_weights.cuh"

using namespace evln;

namespace evln {

cudaError_t prepare_cache_kernels()
{
    const std::pair<const void*, int> kernels[] = {{(const void*)attn8_kernel<1, 1>, Attn8Plan<1, 1>::kBytes},
                                                   {(const void*)attn8_kernel<2, 1>, Attn8Plan<2, 1>::kBytes},
                                                   {(const void*)attn8_kernel<2, 2>, Attn8Plan<2, 2>::kBytes},
                                                   {(const void*)attn8_kernel<2, 4>, Attn8Plan<2, 4>::kBytes},
                                                   {(const void*)key_weights_tile_kernel<128>, KwTilePlan<128>::kBytes},
                                                   {(const void*)key_weights_kernel<64>, KeyWeightPlan<64>::kBytes},
                                                   {(const void*)key_weights_kernel<128>, KeyWeightPlan<128>::kBytes},
                                                   {(const void*)select_keys_kernel, kSelectCache * 4}};
    for (const auto& k : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(k.first, cudaFuncAttributeMaxDynamicSharedMemorySize, k.second);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace evln

namespace {

// As launch_pdl, in clusters of `cluster` blocks along y.
template <typename... KArgs, typename... Args>
cudaError_t launch_cluster_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster, cudaStream_t st, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1;
    attr[1].val.clusterDim.y = (unsigned)cluster;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

evlnStatus_t launched(evlnHandle_t h, cudaError_t e)
{
    return e == cudaSuccess ? EVLN_OK : cuda_fail(h, e);
}

// ---- norms with the append -------------------------------------------------------------------

evlnStatus_t check_norm(const evlnHeadNorm* norm)
{
    if (!norm || norm->struct_size != sizeof(evlnHeadNorm) || !(norm->eps >= 0.f)) return EVLN_INVALID_VALUE;
    if ((norm->q_weight && !aligned16(norm->q_weight)) || (norm->k_weight && !aligned16(norm->k_weight))) return EVLN_INVALID_VALUE;
    return EVLN_OK;
}

// New tokens and where they go: pointers, alignment, strides (elements; vec: of a 16-byte vector).
evlnStatus_t check_tokens(const void* const* pointers, int count, int hq, int hkv, int D, int vec, long qs, long ks, long vs)
{
    for (int i = 0; i < count; ++i)
        if (!pointers[i] || !aligned16(pointers[i])) return EVLN_INVALID_VALUE;
    if (qs < (long)hq * D || ks < (long)hkv * D || vs < (long)hkv * D) return EVLN_INVALID_VALUE;
    if (qs % vec || ks % vec || vs % vec) return EVLN_INVALID_VALUE;
    return EVLN_OK;
}

// Rotated queries must not lie over the new tokens, which other warps still read, unless every query goes where it lies (the layouts of one token,
// or of one kv head without gaps between tokens, are the same).
evlnStatus_t check_q_rot(const void* q_rot, long tokens, int hq, int hkv, int D, int bytes, const void* q, const void* k, const void* v, long qs, long ks, long vs)
{
    auto extent = [&](int heads, long stride) { return ((size_t)(tokens - 1) * stride + (size_t)heads * D) * bytes; };
    const size_t size = (size_t)tokens * hq * D * bytes;
    const bool in_place = q_rot == q && (tokens == 1 || (hkv == 1 && qs == (long)hq * D));
    if ((!in_place && overlap(q_rot, size, q, extent(hq, qs))) || overlap(q_rot, size, k, extent(hkv, ks)) || overlap(q_rot, size, v, extent(hkv, vs)))
        return EVLN_INVALID_VALUE;
    return EVLN_OK;
}

RopeArgs token_args(int hq, int hkv, int D, int vec, const void* q, const void* k, const void* v, long qs, long ks, long vs, double theta, const void* table,
                    int table_first)
{
    RopeArgs a = {};
    a.q_new = q; a.k_new = k; a.v_new = v;
    a.q_stride = qs; a.k_stride = ks; a.v_stride = vs;
    a.Hq = hq; a.Hkv = hkv; a.D = D;
    a.log2_theta = log2(theta);
    a.table = (const double2*)table;
    a.table_first = table_first;
    a.G = hq / hkv;
    a.div_g = make_fast_div((uint32_t)a.G);
    while ((1 << a.vph_shift) < D / 2 / vec) ++a.vph_shift;
    return a;
}

NormArgs norm_args(const evlnHeadNorm* norm)
{
    NormArgs n = {};
    if (norm) { n.q_weight = norm->q_weight; n.k_weight = norm->k_weight; n.eps = norm->eps; }
    return n;
}

// Warps per token for its items: one for each 32 of them while all are resident at once (so many that the GPU has room for), else fewer.
int token_warps(long tokens, int items, long room)
{
    const int most = ceil_div(items, 32);
    const long fill = room / tokens;
    return fill >= most ? most : fill < 1 ? 1 : (int)fill;
}

// Launches the append with the norms; extra: warps behind the tokens'.
template <typename T, bool PAGED, typename LensT>
evlnStatus_t launch_norm_append(evlnHandle_t h, const RopeArgs& a, const evlnHeadNorm* norm, int extra, const LensT& lens, void* stream)
{
    const int items = ((a.Hq + a.Hkv) << a.vph_shift) + (a.Hkv << (a.vph_shift + 1));
    const int warps = token_warps(a.num_new, items, (long)h->num_sms * kNormWarps * kNormBlocks<T> - extra);
    const long blocks = ((long)a.num_new * warps + extra + kNormWarps - 1) / kNormWarps;
    if (blocks > 0x7fffffL) return EVLN_NOT_SUPPORTED;
    auto launch = [&](auto kernel) {
        return launched(h, launch_pdl(kernel, dim3((unsigned)blocks), dim3(32 * kNormWarps), 0, (cudaStream_t)stream, a, norm_args(norm), warps,
                                      make_fast_div((uint32_t)warps), lens));
    };
    return a.table ? launch(norm_append_kernel<T, PAGED, true, LensT>) : launch(norm_append_kernel<T, PAGED, false, LensT>);
}

void batch_lens(BatchLens* bl, const evlnPagedParams* p, const int* lens, const int* offs)
{
    memset(bl, 0, sizeof(*bl));
    memcpy(bl->cache_len, lens, (size_t)p->batch * sizeof(int));
    memcpy(bl->new_off, offs, ((size_t)p->batch + 1) * sizeof(int));
}

// ---- attention over the cache in 8 bits ----------------------------------------------------------

// Most query rows of an episode (per kv head) that the kernel on the codes serves: a block's.  More go through a bf16 copy, which takes the same time for
// 70 rows as for 250, less than the codes twice.  (us, 63 rows on the codes, 70 and 252 through the copy: one episode of 4096 keys 14.4, 14.3 and
// 16.4; of 20656 22.8, 27.5, 31.0; 16 of 8000 98, 121, 125.)
constexpr int kA8MostRows = 64;

struct Plan8 {
    bool expand;
    int most, rows;          // query rows of the longest episode (per kv head), of a block: 8, 16, 32 or 64
    int run, total, runs, blocks;        // stages of a run, of the batch; runs, blocks
    int pages;               // expand: pages of the copy
    size_t copy_bytes;       // expand: table and pools
};

template <typename F>
void for_episodes(const evlnPagedParams* p, const int* lens, const int* offs, F&& f)
{
    for (int b = 0; b < p->batch; ++b) f(b, lens[b], offs[b + 1] - offs[b]);
}

evlnStatus_t plan8(evlnHandle_t h, const evlnPagedParams* p, const int* lens, const int* offs, Plan8* pl)
{
    const int G = p->num_q_heads / p->num_kv_heads;
    long most = 0, total = 0, pages = 0;
    for_episodes(p, lens, offs, [&](int, int, int n) { if ((long)n * G > most) most = (long)n * G; });
    *pl = Plan8();
    pl->most = (int)most;
    pl->expand = most > kA8MostRows;
    pl->rows = most <= 8 ? 8 : most <= 16 ? 16 : most <= 32 ? 32 : 64;
    for_episodes(p, lens, offs, [&](int, int L, int n) {
        if (n == 0) return;
        pages += ((long)L + n + kPage8 - 1) / kPage8;
        total += (long)p->num_kv_heads * (((long)L + n + kA8Keys - 1) / kA8Keys);
    });
    if (total > 0x3fffffffL || pages > 0x3fffffffL) return EVLN_NOT_SUPPORTED;
    if (pl->expand) {
        pl->pages = (int)pages;
        pl->copy_bytes = round_up((size_t)p->batch * p->max_pages_per_seq * sizeof(int), 1024) + (size_t)pages * p->num_kv_heads * kPage8 * 128 * 2 * 2;
        return EVLN_OK;
    }
    // the SMs' key groups each a run of the same length
    const int groups = pl->rows == 8 ? Attn8Plan<1, 1>::kKeyGroups : pl->rows == 16 ? Attn8Plan<2, 1>::kKeyGroups
                     : pl->rows == 32 ? Attn8Plan<2, 2>::kKeyGroups : Attn8Plan<2, 4>::kKeyGroups;
    pl->total = (int)total;
    pl->run = ceil_div(pl->total, h->num_sms * groups);
    if (pl->run < 1) pl->run = 1;
    pl->runs = ceil_div(pl->total, pl->run);
    pl->blocks = ceil_div(pl->runs, groups);
    return EVLN_OK;
}

size_t part_bytes8(const Plan8& pl) { return round_up((size_t)2 * pl.runs * pl.rows * (128 + 4) * sizeof(float), 256); }

// The paged call that serves the bf16 copy.
evlnPagedParams copy_params(const evlnPagedParams* p, const Plan8& pl)
{
    evlnPagedParams c = *p;
    c.num_pages = pl.pages;
    return c;
}

template <int NQ, int RG>
cudaError_t launch_attn8(const Plan8& pl, cudaStream_t st, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Attn8Args& a, const BatchLens& bl)
{
    using Plan = Attn8Plan<NQ, RG>;
    cudaError_t e = launch_pdl(attn8_kernel<NQ, RG>, dim3(pl.blocks), dim3(Plan::kThreads), Plan::kBytes, st, tm_k, tm_v, a, bl);
    if (e == cudaSuccess && pl.runs > 1) {
        MergeList list = {};
        for (int b = 0; b < a.batch && list.count <= kMergeUnits; ++b) {
            const int n = bl.new_off[b + 1] - bl.new_off[b];
            if (n == 0) continue;
            const int stages = ceil_div(bl.cache_len[b] + n, kA8Keys), units = (bl.item_off[b + 1] - bl.item_off[b]) / stages;
            for (int i = 0; i < units && list.count <= kMergeUnits; ++i, ++list.count)
                if (list.count < kMergeUnits) list.first[list.count] = bl.item_off[b] + i * stages;
        }
        const bool few = list.count <= kMergeUnits;
        if (!few) list.count = 0;
        e = launch_pdl(merge8_kernel<Plan::kRows, Plan::kKeyGroups>, dim3(few ? list.count : pl.blocks, few || pl.most < 16 ? pl.most : 16), dim3(32 * kMergeWarps<Plan::kRows>), 0, st, a, bl, list);
    }
    return e;
}

}  // namespace

extern "C" {

evlnStatus_t evlnNormRopeAppend(evlnHandle_t h, const evlnStepParams* p, const evlnHeadNorm* norm, const void* q_new, const void* k_new,
                                const void* v_new, long q_stride_tok, long k_stride_tok, long v_stride_tok, void* q_rot, void* k_cache,
                                void* v_cache, void* stream)
{
    evlnStatus_t s = check_step_params(h, p);
    if (s == EVLN_OK) s = check_norm(norm);
    if (s != EVLN_OK) return s;
    if (p->num_new == 0) return EVLN_OK;
    const int vec = 16 / elem_bytes(p->dtype);
    const void* pointers[6] = {q_new, k_new, v_new, q_rot, k_cache, v_cache};
    s = check_tokens(pointers, 6, p->num_q_heads, p->num_kv_heads, p->head_dim, vec, q_stride_tok, k_stride_tok, v_stride_tok);
    if (s == EVLN_OK)
        s = check_q_rot(q_rot, p->num_new, p->num_q_heads, p->num_kv_heads, p->head_dim, elem_bytes(p->dtype), q_new, k_new, v_new, q_stride_tok, k_stride_tok,
                        v_stride_tok);
    if (s != EVLN_OK) return s;
    if (!device_is_current(h)) return EVLN_INVALID_VALUE;
    RopeArgs a = token_args(p->num_q_heads, p->num_kv_heads, p->head_dim, vec, q_new, k_new, v_new, q_stride_tok, k_stride_tok, v_stride_tok, p->rope_theta,
                            p->rope_table, p->rope_table_first_pos);
    a.q_rot = q_rot; a.k_cache = k_cache; a.v_cache = v_cache;
    a.cache_len = p->cache_len; a.num_new = p->num_new; a.cache_cap = p->cache_capacity;
    return p->dtype == EVLN_BF16 ? launch_norm_append<__nv_bfloat16, false>(h, a, norm, 0, NoLens(), stream)
                                 : launch_norm_append<float, false>(h, a, norm, 0, NoLens(), stream);
}

evlnStatus_t evlnPagedNormRopeAppend(evlnHandle_t h, const evlnPagedParams* p, const evlnHeadNorm* norm, const void* q_new, const void* k_new,
                                     const void* v_new, long q_stride_tok, long k_stride_tok, long v_stride_tok, const int* h_cache_lens,
                                     const int* h_new_offsets, const int* d_page_table, void* q_rot, void* k_pool, void* v_pool, void* stream)
{
    evlnStatus_t s = check_paged_params(h, p, h_cache_lens, h_new_offsets);
    if (s == EVLN_OK) s = check_norm(norm);
    if (s != EVLN_OK) return s;
    const int total = h_new_offsets[p->batch];
    if (total == 0) return EVLN_OK;
    const void* pointers[6] = {q_new, k_new, v_new, q_rot, k_pool, v_pool};
    s = check_tokens(pointers, 6, p->num_q_heads, p->num_kv_heads, 128, 8, q_stride_tok, k_stride_tok, v_stride_tok);
    if (s == EVLN_OK)
        s = check_q_rot(q_rot, total, p->num_q_heads, p->num_kv_heads, 128, 2, q_new, k_new, v_new, q_stride_tok, k_stride_tok, v_stride_tok);
    if (s != EVLN_OK) return s;
    if (!d_page_table || !aligned4(d_page_table) || !device_is_current(h)) return EVLN_INVALID_VALUE;
    RopeArgs a = token_args(p->num_q_heads, p->num_kv_heads, 128, 8, q_new, k_new, v_new, q_stride_tok, k_stride_tok, v_stride_tok, p->rope_theta, p->rope_table,
                            p->rope_table_first_pos);
    a.q_rot = q_rot; a.k_cache = k_pool; a.v_cache = v_pool; a.page_table = d_page_table;
    a.num_new = total; a.batch = p->batch; a.page_size = p->page_size; a.max_pages = p->max_pages_per_seq;
    while ((1 << a.page_shift) < a.page_size) ++a.page_shift;
    BatchLens bl;
    batch_lens(&bl, p, h_cache_lens, h_new_offsets);
    return launch_norm_append<__nv_bfloat16, true>(h, a, norm, p->batch * a.Hkv, bl, stream);
}

evlnStatus_t evlnPaged8RopeAppend(evlnHandle_t h, const evlnPagedParams* p, const evlnHeadNorm* norm, const void* q_new, const void* k_new,
                                  const void* v_new, long q_stride_tok, long k_stride_tok, long v_stride_tok, const int* h_cache_lens,
                                  const int* h_new_offsets, const int* d_page_table, void* q_rot, void* k_pool, void* v_pool, float* k_scale,
                                  float* v_scale, void* stream)
{
    evlnStatus_t s = check_paged_params(h, p, h_cache_lens, h_new_offsets);
    if (s == EVLN_OK && norm) s = check_norm(norm);
    if (s != EVLN_OK) return s;
    const int total = h_new_offsets[p->batch];
    if (total == 0) return EVLN_OK;
    const void* pointers[6] = {q_new, k_new, v_new, q_rot, k_pool, v_pool};
    s = check_tokens(pointers, 6, p->num_q_heads, p->num_kv_heads, 128, 8, q_stride_tok, k_stride_tok, v_stride_tok);
    if (s == EVLN_OK)
        s = check_q_rot(q_rot, total, p->num_q_heads, p->num_kv_heads, 128, 2, q_new, k_new, v_new, q_stride_tok, k_stride_tok, v_stride_tok);
    if (s != EVLN_OK) return s;
    if (!d_page_table || !k_scale || !v_scale || !aligned4(d_page_table, k_scale, v_scale) || !device_is_current(h)) return EVLN_INVALID_VALUE;
    Append8Args a = {};
    a.r = token_args(p->num_q_heads, p->num_kv_heads, 128, 8, q_new, k_new, v_new, q_stride_tok, k_stride_tok, v_stride_tok, p->rope_theta, p->rope_table,
                     p->rope_table_first_pos);
    a.r.q_rot = q_rot; a.r.k_cache = k_pool; a.r.v_cache = v_pool; a.r.page_table = d_page_table;
    a.r.num_new = total; a.r.batch = p->batch; a.r.page_size = kPage8; a.r.max_pages = p->max_pages_per_seq;
    a.norm = norm_args(norm);
    a.k_scale = k_scale; a.v_scale = v_scale;
    BatchLens bl;
    batch_lens(&bl, p, h_cache_lens, h_new_offsets);
    long pages = 0;
    for (int b = 0; b <= p->batch; ++b) {
        bl.item_off[b] = (int)pages;
        if (b >= p->batch) continue;
        const int L = h_cache_lens[b], n = h_new_offsets[b + 1] - h_new_offsets[b];
        if (n > 0) pages += ((long)L + n + kPage8 - 1) / kPage8 - L / kPage8;
    }
    a.q_warps = token_warps(total, a.r.Hq * 8, (long)h->num_sms * (kAppend8Threads / 32) * kAppend8Blocks);
    a.div_warps = make_fast_div((uint32_t)a.q_warps);
    const long blocks = 2 * pages * p->num_kv_heads + ((long)total * a.q_warps * 32 + kAppend8Threads - 1) / kAppend8Threads;
    if (blocks > 0x3fffffffL) return EVLN_NOT_SUPPORTED;
    a.page_blocks = (int)(pages * p->num_kv_heads);
    a.div_hkv = make_fast_div((uint32_t)p->num_kv_heads);
    auto launch = [&](auto kernel) { return launched(h, launch_pdl(kernel, dim3((unsigned)blocks), dim3(kAppend8Threads), 0, (cudaStream_t)stream, a, bl)); };
    if (a.r.table) return norm ? launch(append8_kernel<true, true>) : launch(append8_kernel<false, true>);
    return norm ? launch(append8_kernel<true, false>) : launch(append8_kernel<false, false>);
}

evlnStatus_t evlnPaged8WorkspaceSize(evlnHandle_t h, const evlnPagedParams* p, const int* h_cache_lens, const int* h_new_offsets, size_t* bytes)
{
    evlnStatus_t s = check_paged_params(h, p, h_cache_lens, h_new_offsets);
    if (s != EVLN_OK) return s;
    if (!bytes) return EVLN_INVALID_VALUE;
    Plan8 pl;
    s = plan8(h, p, h_cache_lens, h_new_offsets, &pl);
    if (s != EVLN_OK) return s;
    if (!pl.expand) {
        *bytes = part_bytes8(pl);
        return EVLN_OK;
    }
    const evlnPagedParams c = copy_params(p, pl);
    size_t inner = 0;
    s = evlnPagedWorkspaceSize(h, &c, h_cache_lens, h_new_offsets, &inner);
    *bytes = pl.copy_bytes + inner;
    return s;
}

evlnStatus_t evlnPaged8StepAttention(evlnHandle_t h, const evlnPagedParams* p, const void* q_rot, const void* k_pool, const void* v_pool,
                                     const float* k_scale, const float* v_scale, const int* h_cache_lens, const int* h_new_offsets,
                                     const int* d_page_table, void* workspace, size_t workspace_bytes, void* out, float* lse_out, void* stream)
{
    size_t need = 0;
    evlnStatus_t s = evlnPaged8WorkspaceSize(h, p, h_cache_lens, h_new_offsets, &need);
    if (s != EVLN_OK) return s;
    const int total = h_new_offsets[p->batch];
    if (total == 0) return EVLN_OK;
    const void* pointers[5] = {q_rot, k_pool, v_pool, workspace, out};
    for (const void* x : pointers)
        if (!x || !aligned16(x)) return EVLN_INVALID_VALUE;
    if (!k_scale || !v_scale || !d_page_table || !aligned4(d_page_table, k_scale, v_scale, lse_out) || !device_is_current(h)) return EVLN_INVALID_VALUE;
    // Outputs are written while other blocks read queries: not over them, unless every row goes where its own query lies (the layouts of one
    // token or one kv head are the same).
    const size_t rows_all = (size_t)total * p->num_q_heads, q_bytes = rows_all * 128 * 2;
    const bool in_place = out == q_rot && (total == 1 || p->num_kv_heads == 1);
    if ((!in_place && overlap(out, q_bytes, q_rot, q_bytes)) || (lse_out && overlap(lse_out, rows_all * sizeof(float), q_rot, q_bytes))) return EVLN_INVALID_VALUE;
    if (workspace_bytes < need) return EVLN_WORKSPACE_TOO_SMALL;
    Plan8 pl;
    s = plan8(h, p, h_cache_lens, h_new_offsets, &pl);
    if (s != EVLN_OK) return s;
    cudaStream_t st = (cudaStream_t)stream;
    const int G = p->num_q_heads / p->num_kv_heads, hkv = p->num_kv_heads;
    BatchLens bl;
    batch_lens(&bl, p, h_cache_lens, h_new_offsets);

    if (pl.expand) {
        const evlnPagedParams c = copy_params(p, pl);
        int at = 0;
        for (int b = 0; b <= p->batch; ++b) {
            bl.item_off[b] = at;
            if (b < p->batch && h_new_offsets[b + 1] > h_new_offsets[b]) at += ceil_div(h_cache_lens[b] + h_new_offsets[b + 1] - h_new_offsets[b], kPage8);
        }
        Expand8Args a = {};
        a.k_pool = (const uint8_t*)k_pool; a.v_pool = (const uint8_t*)v_pool;
        a.k_scale = k_scale; a.v_scale = v_scale;
        a.page_table = d_page_table;
        a.out_table = (int*)workspace;
        a.k_out = (__nv_bfloat16*)((char*)workspace + round_up((size_t)p->batch * p->max_pages_per_seq * sizeof(int), 1024));
        a.v_out = a.k_out + (size_t)pl.pages * hkv * kPage8 * 128;
        a.Hkv = hkv; a.batch = p->batch; a.max_pages = p->max_pages_per_seq;
        void* inner = (char*)workspace + pl.copy_bytes;
        s = launched(h, launch_pdl(expand8_kernel, dim3((unsigned)pl.pages, (unsigned)hkv, 2), dim3(256), 0, st, a, bl));
        if (s == EVLN_OK)
            s = paged_attention_to(h, &c, q_rot, a.k_out, a.v_out, h_cache_lens, h_new_offsets, a.out_table, inner, workspace_bytes - pl.copy_bytes, out, lse_out, stream);
        return s;
    }

    int at = 0;
    for (int b = 0; b <= p->batch; ++b) {
        bl.item_off[b] = at;
        if (b >= p->batch) continue;
        const int L = h_cache_lens[b], n = h_new_offsets[b + 1] - h_new_offsets[b];
        if (n > 0) at += hkv * ceil_div(L + n, kA8Keys);
    }
    CUtensorMap tm_k, tm_v;
    const cuuint64_t dims[2] = {128, (cuuint64_t)p->num_pages * hkv * kPage8}, strides[1] = {128};
    const cuuint32_t box[2] = {128, kA8Keys};
    if (dims[1] > 0x7fffffffULL) return EVLN_NOT_SUPPORTED;
    if (!encode_map(h, &tm_k, k_pool, 2, dims, strides, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return EVLN_INVALID_VALUE;
    if (!encode_map(h, &tm_v, v_pool, 2, dims, strides, box, CU_TENSOR_MAP_DATA_TYPE_UINT8)) return EVLN_INVALID_VALUE;
    Attn8Args a = {};
    a.q_rot = (const __nv_bfloat16*)q_rot;
    a.k_scale = k_scale; a.v_scale = v_scale;
    a.page_table = d_page_table;
    a.out = (__nv_bfloat16*)out; a.lse_out = lse_out;
    a.o_part = (float*)workspace;
    a.ml_part = (float4*)(a.o_part + (size_t)2 * pl.runs * pl.rows * 128);
    a.status = h->d_status;
    a.Hkv = hkv; a.G = G; a.rows = total * G; a.batch = p->batch; a.max_pages = p->max_pages_per_seq;
    a.run = pl.run; a.total = pl.total;
    a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf(128.f)) * 1.4426950408889634f;
    a.div_g = make_fast_div((uint32_t)G);
    return launched(h, pl.rows == 8    ? launch_attn8<1, 1>(pl, st, tm_k, tm_v, a, bl)
                       : pl.rows == 16 ? launch_attn8<2, 1>(pl, st, tm_k, tm_v, a, bl)
                       : pl.rows == 32 ? launch_attn8<2, 2>(pl, st, tm_k, tm_v, a, bl)
                                       : launch_attn8<2, 4>(pl, st, tm_k, tm_v, a, bl));
}

// ---- eviction --------------------------------------------------------------------------------

evlnStatus_t evlnKeyWeights(evlnHandle_t h, const evlnStepParams* p, const void* q_rot, const void* k_cache, const float* lse, float decay,
                            const float* weights_in, float* weights_out, void* stream)
{
    evlnStatus_t s = check_step_params(h, p);
    if (s != EVLN_OK) return s;
    if (!(decay >= 0.f)) return EVLN_INVALID_VALUE;
    if (p->num_new == 0) return EVLN_INVALID_VALUE;
    if (!q_rot || !k_cache || !lse || !weights_in || !weights_out || !aligned16(q_rot) || !aligned16(k_cache) || !aligned4(lse, weights_in, weights_out))
        return EVLN_INVALID_VALUE;
    const size_t w_bytes = (size_t)p->num_kv_heads * p->cache_capacity * sizeof(float);
    if (weights_in != weights_out && overlap(weights_in, w_bytes, weights_out, w_bytes)) return EVLN_INVALID_VALUE;
    if (!device_is_current(h)) return EVLN_INVALID_VALUE;
    const int D = p->head_dim, total = p->cache_len + p->num_new;
    const long tiles = ((long)total + kTileN - 1) / kTileN;
    if (tiles * p->num_kv_heads > 0x3fffffffL) return EVLN_NOT_SUPPORTED;
    KeyWeightArgs a = {};
    a.lse = lse; a.in = weights_in; a.out = weights_out;
    a.q_rot = q_rot; a.k_cache = k_cache;
    a.status = h->d_status;
    a.Hkv = p->num_kv_heads; a.G = p->num_q_heads / p->num_kv_heads; a.rows = p->num_new * a.G;
    a.L = p->cache_len; a.n = p->num_new; a.cap = p->cache_capacity;
    a.items = (int)tiles * p->num_kv_heads;
    a.scale_log2 = (p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / sqrtf((float)D)) * 1.4426950408889634f;
    a.decay = decay;
    a.div_g = make_fast_div((uint32_t)a.G);
    a.div_hkv = make_fast_div((uint32_t)a.Hkv);
    const bool f32 = p->dtype == EVLN_F32;
    // fp32, both sides in us (28/4 heads of 128): 28 rows over 4096 keys 16.8 a thread per key, 17.3 as tiles; 56 rows 29.4 and 18.3, over 9000 46.3 and 24.6;
    // 448 rows over 4096 121 and 78, but over 3000, which leave a third of the SMs without a tile, 196 rows 34.6 and 48.2.  Heads of 64 gain nothing (9000
    // keys, 196 rows 48.3 and 56.3): their keys leave room for more warps.
    const bool tile = f32 && D == 128 && a.rows > kKwTileLeastRows && 4L * a.items >= 3L * h->num_sms;
    a.chunk_rows = tile ? kKwTileRows : f32 ? kKwF32Rows : a.rows >= kKwRows ? kKwRows : (a.rows + 31) / 32 * 32;
    a.chunks = ceil_div(a.rows, a.chunk_rows);
    // few tiles: a cluster of CTAs for each, as many as the SMs (fp32: four blocks an SM, two of tiles) and the chunks allow
    int cluster = 1;
    while (cluster < kKwMaxCluster && 2 * cluster <= a.chunks && 2L * cluster * a.items <= (tile ? 2L : f32 ? 4L : 1L) * h->num_sms) cluster *= 2;
    const dim3 grid((unsigned)(cluster > 1 || f32 || a.items < h->num_sms ? a.items : h->num_sms), (unsigned)cluster);
    cudaStream_t st = (cudaStream_t)stream;
    if (tile)
        return launched(h, launch_cluster_pdl(key_weights_tile_kernel<128>, grid, dim3(128), KwTilePlan<128>::kBytes, cluster, st, a));
    if (f32)
        return launched(h, D == 128 ? launch_cluster_pdl(key_weights_f32_kernel<128>, grid, dim3(kKwF32Keys), 0, cluster, st, a)
                                    : launch_cluster_pdl(key_weights_f32_kernel<64>, grid, dim3(kKwF32Keys), 0, cluster, st, a));
    CUtensorMap tm_k, tm_q;
    const cuuint64_t kdims[3] = {(cuuint64_t)D, (cuuint64_t)p->cache_capacity, (cuuint64_t)p->num_kv_heads};
    const cuuint64_t kstrides[2] = {(cuuint64_t)D * 2, (cuuint64_t)p->cache_capacity * D * 2};
    const cuuint64_t qdims[3] = {(cuuint64_t)D, (cuuint64_t)a.rows, (cuuint64_t)p->num_kv_heads};
    const cuuint64_t qstrides[2] = {(cuuint64_t)D * 2, (cuuint64_t)a.rows * D * 2};
    const cuuint32_t kbox[3] = {64, kTileN, 1}, qbox[3] = {64, (cuuint32_t)a.chunk_rows, 1};
    if (!encode_map(h, &tm_k, k_cache, 3, kdims, kstrides, kbox)) return EVLN_INVALID_VALUE;
    if (!encode_map(h, &tm_q, q_rot, 3, qdims, qstrides, qbox)) return EVLN_INVALID_VALUE;
    return launched(h, D == 128 ? launch_cluster_pdl(key_weights_kernel<128>, grid, dim3(kKwThreads), KeyWeightPlan<128>::kBytes, cluster, st, tm_k, tm_q, a)
                                : launch_cluster_pdl(key_weights_kernel<64>, grid, dim3(kKwThreads), KeyWeightPlan<64>::kBytes, cluster, st, tm_k, tm_q, a));
}

evlnStatus_t evlnSelectKeys(evlnHandle_t h, const evlnGatherParams* p, const float* weights, int num_keys, int budget, int sinks, int recent,
                            int* kept, void* stream)
{
    evlnStatus_t s = check_gather_params(h, p);
    if (s != EVLN_OK) return s;
    if (num_keys > (1 << 30)) return EVLN_NOT_SUPPORTED;
    if (num_keys < 0 || num_keys > p->store_capacity || budget < 0 || sinks < 0 || recent < 0 || (long)sinks + recent > budget) return EVLN_INVALID_VALUE;
    SelectArgs a = {};
    a.num_kept = budget < num_keys ? budget : num_keys;
    if (a.num_kept == 0) return EVLN_OK;
    if (!weights || !kept || !aligned4(weights, kept)) return EVLN_INVALID_VALUE;
    a.weights = weights; a.kept = kept;
    a.stride = p->store_capacity; a.num_keys = num_keys;
    a.sinks = sinks; a.recent = recent; a.open = budget - sinks - recent;
    if (a.num_kept == num_keys) a.sinks = a.recent = a.open = 0;
    const int cluster = num_keys > kSelectSlice ? kSelectCluster : 1;
    a.slice = ceil_div(num_keys, cluster);
    a.cached = a.slice <= kSelectCache;
    return launched(h, launch_cluster_pdl(select_keys_kernel, dim3((unsigned)p->num_kv_heads, (unsigned)cluster), dim3(kSelectThreads), a.cached ? (size_t)a.slice * 4 : 0,
                                          cluster, (cudaStream_t)stream, a));
}

evlnStatus_t evlnGatherKeys(evlnHandle_t h, const evlnGatherParams* p, int num_kept, const int* kept, const float* weights, const void* k_store,
                            const void* v_store, float* weights_work, void* k_work, void* v_work, int rotate, void* stream)
{
    evlnStatus_t s = check_gather_params(h, p);
    if (s != EVLN_OK) return s;
    if (num_kept < 0) return EVLN_INVALID_VALUE;
    if (num_kept > p->work_capacity) return EVLN_CACHE_FULL;
    if (num_kept == 0) return EVLN_OK;
    const void* pointers[4] = {k_store, v_store, k_work, v_work};
    for (const void* x : pointers)
        if (!x || !aligned16(x)) return EVLN_INVALID_VALUE;
    if (!kept || !aligned4(kept, weights, weights_work) || (weights == nullptr) != (weights_work == nullptr)) return EVLN_INVALID_VALUE;
    if (rotate && !rope_table_covers(p->rope_table, p->rope_table_first_pos, p->rope_table_count, 0, num_kept)) return EVLN_INVALID_VALUE;
    const size_t row = (size_t)p->num_kv_heads * p->head_dim * elem_bytes(p->dtype), src = row * p->store_capacity, dst = row * p->work_capacity;
    for (int i = 0; i < 2; ++i)
        for (int j = 2; j < 4; ++j)
            if (overlap(pointers[i], src, pointers[j], dst)) return EVLN_INVALID_VALUE;
    if (weights && overlap(weights, (size_t)p->num_kv_heads * p->store_capacity * 4, weights_work, (size_t)p->num_kv_heads * p->work_capacity * 4)) return EVLN_INVALID_VALUE;
    GatherKeysArgs a = {};
    a.k_src = k_store; a.v_src = v_store; a.w_src = weights;
    a.k_dst = k_work; a.v_dst = v_work; a.w_dst = weights_work;
    a.kept = kept;
    a.Hkv = p->num_kv_heads; a.D = p->head_dim; a.src_cap = p->store_capacity; a.dst_cap = p->work_capacity;
    a.num_kept = num_kept; a.rotate = rotate != 0;
    for (int b = 0; b < 6; ++b) a.omega[b] = b == 0 ? exp2(-2.0 / a.D * log2(p->rope_theta)) : a.omega[b - 1] * a.omega[b - 1];
    a.table = (const double2*)p->rope_table;
    a.table_first = p->rope_table_first_pos;
    const int vec = 16 / elem_bytes(p->dtype);
    while ((1 << a.vph_shift) < a.D / 2 / vec) ++a.vph_shift;
    // a slot's angles a thread, more where the blocks would not all be resident (and so could not form theirs while the kernel before them runs)
    while ((kGatherKeysThreads / (a.D / 2)) >> (a.log_slots + 1)) ++a.log_slots;
    while ((1 << a.log_slots) < kGatherKeysSlots && (num_kept + (1 << a.log_slots) - 1) >> a.log_slots > h->num_sms * kGatherKeysBlocks) ++a.log_slots;
    const dim3 grid((unsigned)ceil_div(num_kept, 1 << a.log_slots)), block(kGatherKeysThreads);
    return launched(h, p->dtype == EVLN_BF16 ? launch_pdl(gather_keys_kernel<__nv_bfloat16>, grid, block, 0, (cudaStream_t)stream, a)
                                             : launch_pdl(gather_keys_kernel<float>, grid, block, 0, (cudaStream_t)stream, a));
}

}  // extern "C"
