// Launchers of the operators on heads (heads.cu, attend.cu), called by their C ABI (api_heads.cu) with checked arguments.
#pragma once

#include <atomic>

#include "attend.cuh"

namespace meteora {

// A launch that may be set up under the kernel ahead (every kernel here waits for it before it touches memory).
template <auto kernel, typename... A>
int launch_dependent(dim3 grid, int threads, size_t smem, cudaStream_t st, const A&... args) {
    if (smem > 20 * 1024) {                                         // (48 KB with the static arrays, 25 KB at most)
        static std::atomic<bool> allowed[64];                       // per device: all that static arrays leave, for launches of any size
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e == cudaSuccess && (dev >= 64 || !allowed[dev].load(std::memory_order_relaxed))) {
            cudaFuncAttributes fa;
            e = cudaFuncGetAttributes(&fa, kernel);
            if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)fa.sharedSizeBytes);
            if (e == cudaSuccess && dev < 64) allowed[dev].store(true, std::memory_order_relaxed);
        }
        if (e != cudaSuccess) return cuda_status(e);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = tuning().pdl ? 1 : 0;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, args...));
}

struct HeadRows {
    meteora_heads_t in;
    void* out;               // paged: the cache's keys or values
    int64_t out_t, out_h;
    const void* gain;        // nullptr: no norm
    int paged, turn;
};
struct HeadPassArgs {
    int T, head_dim;
    meteora_dtype_t dtype;
    const void* positions;   // [T]; nullptr with a batch
    int positions_64;
    const meteora_rotary_t* rot;
    int inverse;
    float eps;
    const BatchView* batch;
};
int launch_head_pass(const HeadRows* segs, int n_segs, const HeadPassArgs& args, cudaStream_t st);
size_t head_grad_workspace_bytes(int T, int head_dim);
int launch_head_grad(const meteora_heads_t* dy, const meteora_heads_t* x, const void* const* gain, const meteora_heads_t* dx,
                     float* dq_gain, float* dk_gain, const HeadPassArgs& args, float* part, cudaStream_t st);

struct AttendSizes {
    int T, B, q_heads, kv_heads, head_dim, page_size, table_width, prefix_len;
    long long n_pages;
    meteora_dtype_t dtype;
};
// wgemm_tcgen05.cu: units of `rows` rows on the tensor cores, the prefix's or the own tokens'
bool attend_tc_supported(const AttendSizes& z, long long rows);
int launch_attend_tc(const AttendParams& p, bool own, cudaStream_t st);
// and units of 16 or 64 rows through warp-level products (entries of a head padded to `padded`: 64, 128 or 256)
int launch_attend_warps(const AttendParams& p, int padded, cudaStream_t st);
size_t attend_workspace_bytes(const AttendSizes& z);
int launch_prefix_attention(const meteora_heads_t& q, const meteora_heads_t& out, float* lse, const meteora_cache_t& cache,
                            const BatchView& batch, const AttendSizes& z, float scale, void* workspace, cudaStream_t st);

}  // namespace meteora
