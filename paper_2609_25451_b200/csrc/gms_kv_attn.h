// Internal declarations of the attention and eviction kernels on the paged KV pool.
#pragma once
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "gms.h"

namespace gms {

// What every attention kernel gets (by value).  Strides of pool and of q / out are in bytes.
struct AttnArgs {
    const uint8_t *k_base, *v_base;  // planes of this layer
    uint64_t block_stride;
    uint32_t n_blocks, token_stride, head_stride, block_shift;  // block_tokens = 1 << block_shift
    const uint8_t *q;
    uint8_t *out;
    float *lse;
    const int32_t *cu_q, *kv_lens, *table;
    uint64_t table_stride;
    uint64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    uint32_t n_seq, n_heads, n_kv, group;  // group = n_heads / n_kv
    uint32_t total_q, max_q, max_kv, window, sinks;
    float scale;
    // shared prefixes (n_groups = 0: none)
    const int32_t *group_start, *prefix_lens, *prefix_table;
    uint64_t prefix_stride;
    uint32_t n_groups, max_prefix, max_group_q;
    // accumulated weights (w_out = null: none)
    const float *w_in;
    float *w_out;
    uint64_t w_seq_stride, w_head_stride;
    float decay;
    unsigned long long *status;  // may be null
};

struct EvictArgs {
    uint8_t *base;
    uint64_t plane_stride, block_stride;
    uint32_t k_plane, v_plane, n_blocks, token_stride, head_stride, block_shift, row_bytes;
    const float *weights;
    float *weights_out;
    const int32_t *lens;
    int32_t *lens_out;
    const int32_t *src_table, *dst_table;
    int32_t *kept;
    uint64_t w_layer_stride, w_seq_stride, w_head_stride, o_layer_stride, o_seq_stride, o_head_stride, src_stride, dst_stride;
    uint32_t n_layers, layer_planes, n_seq, n_kv, max_len, budget, sinks, recent;
};

cudaError_t launch_kv_attention_rows(const AttnArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s);
cudaError_t launch_kv_weights(const AttnArgs &a, const float *lse, uint32_t dtype, uint32_t head_dim, cudaStream_t s);
cudaError_t launch_kv_evict(const EvictArgs &a, cudaStream_t s);

#ifdef __CUDACC__
// ------------------------------------------------------------------ device helpers
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// Query rows and cached tokens of one sequence, clamped to what the host announced (so that no index leaves a buffer
// whatever the device arrays hold).
__device__ __forceinline__ int seq_q_begin(const AttnArgs &a, uint32_t s)
{
    return a.cu_q ? min(max(a.cu_q[s], 0), (int)a.total_q) : (int)s;
}
__device__ __forceinline__ int seq_q_len(const AttnArgs &a, uint32_t s)
{
    if (!a.cu_q) return 1;
    const int b = seq_q_begin(a, s);
    return min(max(min(a.cu_q[s + 1], (int)a.total_q) - b, 0), (int)a.max_q);
}
__device__ __forceinline__ int seq_kv_len(const AttnArgs &a, uint32_t s) { return min(max(a.kv_lens[s], 0), (int)a.max_kv); }
__device__ __forceinline__ int prefix_len(const AttnArgs &a, uint32_t g)
{
    return min(max(a.prefix_lens[g], 0), (int)a.max_prefix);
}
// Whether the query at position `pos` sees token t.
__device__ __forceinline__ bool sees(const AttnArgs &a, int pos, int t)
{
    return t <= pos && (a.window == 0 || (long long)t > (long long)pos - (long long)a.window || (uint32_t)t < a.sinks);
}
// Last index i in [0, n) with v[i] <= x (v ascending, v[0] <= x).
__device__ __forceinline__ uint32_t last_not_above(const int32_t *v, uint32_t n, int x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (v[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
// Sequence that owns query row `tok`, or n_seq.  Equal offsets (empty sequences) resolve to the last of them.
__device__ __forceinline__ uint32_t owner_of_row(const AttnArgs &a, int tok)
{
    if (!a.cu_q) return (uint32_t)tok < a.n_seq ? (uint32_t)tok : a.n_seq;
    if (tok < a.cu_q[0] || tok >= a.cu_q[a.n_seq]) return a.n_seq;
    const uint32_t s = last_not_above(a.cu_q, a.n_seq, tok);
    return tok - seq_q_begin(a, s) < seq_q_len(a, s) ? s : a.n_seq;
}
// Group of a sequence, or n_groups.
__device__ __forceinline__ uint32_t group_of_seq(const AttnArgs &a, uint32_t s)
{
    if (a.n_groups == 0 || (int)s < a.group_start[0] || (int)s >= a.group_start[a.n_groups]) return a.n_groups;
    return last_not_above(a.group_start, a.n_groups, (int)s);
}
__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
#endif

}  // namespace gms
