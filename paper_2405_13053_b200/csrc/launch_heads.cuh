// Launchers of the operators on heads (heads.cu, attend.cu), called by their C ABI (api_heads.cu) with checked arguments.
#pragma once

#include "heads.cuh"

namespace meteora {

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
size_t head_grad_workspace_bytes(int T, int q_heads, int k_heads, int head_dim);
int launch_head_grad(const meteora_heads_t* dy, const meteora_heads_t* x, const void* const* gain, const meteora_heads_t* dx,
                     float* dq_gain, float* dk_gain, const HeadPassArgs& args, float* part, cudaStream_t st);

struct AttendSizes {
    int T, B, q_heads, kv_heads, head_dim, page_size, table_width, prefix_len;
    meteora_dtype_t dtype;
};
size_t attend_workspace_bytes(const AttendSizes& z);
int launch_prefix_attention(const meteora_heads_t& q, const meteora_heads_t& out, float* lse, const meteora_cache_t& cache,
                            const BatchView& batch, const AttendSizes& z, float scale, void* workspace, cudaStream_t st);

}  // namespace meteora
