// What the host side of every entry point shares: the handle, launches, argument checks.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <utility>

#include "../../include/evln.h"
#include "common.cuh"

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

struct evlnContext {
    int device;
    int num_sms;
    int last_cuda_error;
    int* d_status;
    EncodeTiledFn encode;
    int max_clusters[5];     // clusters of 1, 2, 4, 8, 16 blocks of the few-row kernel that fit the device at once
    int small_clusters[evln::kSmallCluster];   // clusters of 1, 2, .. blocks of the small fp32 kernel
};

namespace evln {

// Every kernel is launched with programmatic stream serialisation: its prologue may overlap the
// tail of the previous kernel in the stream; each kernel waits (griddepcontrol.wait) before it
// touches global memory.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st,
                       Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
// Arrays of floats and ints (null: one that the call may go without).
template <typename... P>
bool aligned4(const P*... p)
{
    return (((reinterpret_cast<uintptr_t>(p) & 3u) == 0) && ...);
}
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a_bytes > 0 && b_bytes > 0 && x < y + b_bytes && y < x + a_bytes;
}
inline int elem_bytes(int dtype) { return dtype == EVLN_BF16 ? 2 : 4; }

inline evlnStatus_t cuda_fail(evlnHandle_t h, cudaError_t e)
{
    h->last_cuda_error = (int)e;
    return EVLN_CUDA_ERROR;
}

// The handle's device must be current when work is launched: the kernels' attributes and the
// tensor maps belong to that device's context.
inline bool device_is_current(evlnHandle_t h)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == h->device;
}

// An optional position table must cover the positions [first, first + count) of the call.
inline bool rope_table_covers(const void* table, int table_first, int table_count, long first, long count)
{
    if (!table) return true;
    if (!aligned16(table) || table_first < 0 || table_count < 0) return false;
    return (long)table_first <= first && first + count <= (long)table_first + table_count;
}

inline evlnStatus_t check_step_params(evlnHandle_t h, const evlnStepParams* p)
{
    if (!h || !p) return EVLN_INVALID_VALUE;
    if (p->struct_size != sizeof(evlnStepParams)) return EVLN_INVALID_VALUE;
    if (p->dtype != EVLN_BF16 && p->dtype != EVLN_F32) return EVLN_INVALID_VALUE;
    if (p->num_q_heads <= 0 || p->num_kv_heads <= 0 || p->num_q_heads % p->num_kv_heads != 0)
        return EVLN_INVALID_VALUE;
    if (p->cache_len < 0 || p->num_new < 0 || p->cache_capacity < 0) return EVLN_INVALID_VALUE;
    if (!(p->rope_theta > 0.0) || !(p->softmax_scale >= 0.f)) return EVLN_INVALID_VALUE;
    if (p->num_splits < 0 || p->num_splits > kMaxSplits) return EVLN_INVALID_VALUE;
    if (p->kernel != EVLN_KERNEL_AUTO && p->kernel != EVLN_KERNEL_SIMT) return EVLN_INVALID_VALUE;
    if (p->head_dim != 64 && p->head_dim != 128) return EVLN_NOT_SUPPORTED;
    if ((long)p->cache_len + p->num_new > (long)p->cache_capacity) return EVLN_CACHE_FULL;
    if ((long)p->num_new * p->num_q_heads / p->num_kv_heads > (1 << 24)) return EVLN_NOT_SUPPORTED;
    if (!rope_table_covers(p->rope_table, p->rope_table_first_pos, p->rope_table_count, p->cache_len, p->num_new))
        return EVLN_INVALID_VALUE;
    return EVLN_OK;
}

inline evlnStatus_t check_paged_params(evlnHandle_t h, const evlnPagedParams* p, const int* lens, const int* offs)
{
    if (!h || !p || !lens || !offs) return EVLN_INVALID_VALUE;
    if (p->struct_size != sizeof(evlnPagedParams)) return EVLN_INVALID_VALUE;
    if (p->num_q_heads <= 0 || p->num_kv_heads <= 0 || p->num_q_heads % p->num_kv_heads != 0)
        return EVLN_INVALID_VALUE;
    if (p->batch < 1 || p->num_pages < 1 || p->max_pages_per_seq < 1 || p->kv_chunk_tiles < 0)
        return EVLN_INVALID_VALUE;
    if (!(p->rope_theta > 0.0) || !(p->softmax_scale >= 0.f)) return EVLN_INVALID_VALUE;
    if (p->dtype != EVLN_BF16 || p->head_dim != 128 || p->page_size != 64 || p->batch > kMaxBatch)
        return EVLN_NOT_SUPPORTED;
    if (offs[0] != 0) return EVLN_INVALID_VALUE;
    for (int b = 0; b < p->batch; ++b) {
        if (lens[b] < 0 || offs[b + 1] < offs[b]) return EVLN_INVALID_VALUE;
        const long tokens = (long)lens[b] + (offs[b + 1] - offs[b]);
        if ((tokens + p->page_size - 1) / p->page_size > p->max_pages_per_seq) return EVLN_CACHE_FULL;
        if (!rope_table_covers(p->rope_table, p->rope_table_first_pos, p->rope_table_count, lens[b], offs[b + 1] - offs[b]))
            return EVLN_INVALID_VALUE;
    }
    if ((long)offs[p->batch] * p->num_q_heads / p->num_kv_heads > (1 << 24)) return EVLN_NOT_SUPPORTED;
    return EVLN_OK;
}

inline evlnStatus_t check_gather_params(evlnHandle_t h, const evlnGatherParams* p)
{
    if (!h || !p) return EVLN_INVALID_VALUE;
    if (p->struct_size != sizeof(evlnGatherParams)) return EVLN_INVALID_VALUE;
    if (p->dtype != EVLN_BF16 && p->dtype != EVLN_F32) return EVLN_INVALID_VALUE;
    if (p->num_kv_heads <= 0 || p->store_capacity < 0 || p->work_capacity < 0) return EVLN_INVALID_VALUE;
    if (!(p->rope_theta > 0.0)) return EVLN_INVALID_VALUE;
    if (p->head_dim != 64 && p->head_dim != 128) return EVLN_NOT_SUPPORTED;
    if (!device_is_current(h)) return EVLN_INVALID_VALUE;
    return EVLN_OK;
}

// A tensor map of 128-byte swizzled boxes; elements outside the tensor read as zeros.
inline bool encode_map(evlnHandle_t h, CUtensorMap* map, const void* base, int rank, const cuuint64_t* dims,
                const cuuint64_t* strides_bytes, const cuuint32_t* box,
                       CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16)
{
    cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    CUresult r = h->encode(map, type, (cuuint32_t)rank, const_cast<void*>(base),
                           dims, strides_bytes, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

// evlnPagedStepAttention + evlnPagedStepCombine in one (evln_api.cu).
evlnStatus_t paged_attention_to(evlnHandle_t h, const evlnPagedParams* p, const void* q_rot, const void* k_pool, const void* v_pool, const int* h_cache_lens,
                                const int* h_new_offsets, const int* d_page_table, void* workspace, size_t workspace_bytes, void* out, float* lse_out, void* stream);

// Shared-memory limits of the kernels in cache_ops.cu, on the current device.
cudaError_t prepare_cache_kernels();

}  // namespace evln
