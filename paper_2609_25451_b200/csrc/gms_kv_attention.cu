// Attention over the paged KV pool: host entry points, and the row kernel.
#include <cmath>

#include "gms_internal.h"
#include "gms_kv_attn.h"

namespace gms {
namespace {

// One warp computes one (query row, head) in 32 bits, token by token: the definition, written down.  Lanes split the
// head dimension; the running maximum m, sum l and weighted values o are rescaled when the maximum moves.
template <class T, int D>
__device__ void attend_tokens(const AttnArgs &a, const float *q, uint32_t c, const int32_t *table, int n, int pos, bool whole,
                              float &m, float &l, float *o)
{
    constexpr int E = D / 32;
    const uint32_t lane = threadIdx.x & 31u;
    for (int t = 0; t < n; ++t) {
        if (!whole && !sees(a, pos, t)) continue;
        const int id = table[t >> a.block_shift];
        if ((uint32_t)id >= a.n_blocks) continue;
        const uint64_t off = (uint64_t)id * a.block_stride + (uint64_t)(t & ((1 << a.block_shift) - 1)) * a.token_stride +
                             (uint64_t)c * a.head_stride;
        const T *k = reinterpret_cast<const T *>(a.k_base + off), *v = reinterpret_cast<const T *>(a.v_base + off);
        float x = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) x += q[e] * to_f32(k[lane + 32 * e]);
        x = warp_sum(x) * a.scale * kLog2e;
        const float mn = fmaxf(m, x), f = mn == neg_inf() ? 1.f : exp2f(m - mn), p = exp2f(x - (mn == neg_inf() ? 0.f : mn));
        l = l * f + p;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * to_f32(v[lane + 32 * e]);
        m = mn;
    }
}

template <class T, int D>
__global__ void __launch_bounds__(128) kv_attention_rows_kernel(AttnArgs a)
{
    constexpr int E = D / 32;
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t row = (uint64_t)blockIdx.x * 4 + threadIdx.x / 32;
    if (row >= (uint64_t)a.total_q * a.n_heads) return;
    const int tok = (int)(row / a.n_heads);
    const uint32_t h = (uint32_t)(row % a.n_heads), c = h / a.group, s = owner_of_row(a, tok);
    if (s >= a.n_seq) return;
    const T *qp = reinterpret_cast<const T *>(a.q + (uint64_t)tok * a.q_token_stride + (uint64_t)h * a.q_head_stride);
    float q[E], o[E], m = neg_inf(), l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) q[e] = to_f32(qp[lane + 32 * e]), o[e] = 0.f;
    const uint32_t g = group_of_seq(a, s);
    if (g < a.n_groups) attend_tokens<T, D>(a, q, c, a.prefix_table + g * a.prefix_stride, prefix_len(a, g), 0, true, m, l, o);
    const int n = seq_kv_len(a, s);
    attend_tokens<T, D>(a, q, c, a.table + s * a.table_stride, n, n - seq_q_len(a, s) + tok - seq_q_begin(a, s), false, m, l, o);
    T *op = reinterpret_cast<T *>(a.out + (uint64_t)tok * a.out_token_stride + (uint64_t)h * a.out_head_stride);
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) op[lane + 32 * e] = from_f32<T>(l == 0.f ? 0.f : o[e] * inv);
    if (a.lse && lane == 0) a.lse[row] = l == 0.f ? neg_inf() : (m + log2f(l)) * kLn2;
}

// One warp accumulates the weight of one (sequence, KV head, token), rows in order.
template <class T, int D>
__global__ void __launch_bounds__(128) kv_weights_kernel(AttnArgs a, const float *lse)
{
    constexpr int E = D / 32;
    const uint32_t lane = threadIdx.x & 31u;
    const uint64_t w = (uint64_t)blockIdx.x * 4 + threadIdx.x / 32;
    const int t = (int)(w % a.max_kv);
    const uint32_t c = (uint32_t)(w / a.max_kv % a.n_kv), s = (uint32_t)(w / a.max_kv / a.n_kv);
    if (s >= a.n_seq || t >= seq_kv_len(a, s)) return;
    const int id = a.table[s * a.table_stride + (t >> a.block_shift)];
    const int q0 = seq_q_begin(a, s), ql = seq_q_len(a, s), first = seq_kv_len(a, s) - ql;
    const uint64_t at = s * a.w_seq_stride + c * a.w_head_stride + t;
    float sum = 0.f;
    if ((uint32_t)id < a.n_blocks) {
        const T *k = reinterpret_cast<const T *>(a.k_base + (uint64_t)id * a.block_stride +
                                                 (uint64_t)(t & ((1 << a.block_shift) - 1)) * a.token_stride +
                                                 (uint64_t)c * a.head_stride);
        for (int i = 0; i < ql; ++i) {
            if (!sees(a, first + i, t)) continue;
            for (uint32_t h = c * a.group; h < (c + 1) * a.group; ++h) {
                const T *q = reinterpret_cast<const T *>(a.q + (uint64_t)(q0 + i) * a.q_token_stride + (uint64_t)h * a.q_head_stride);
                float x = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) x += to_f32(q[lane + 32 * e]) * to_f32(k[lane + 32 * e]);
                const float ls = lse[(uint64_t)(q0 + i) * a.n_heads + h];
                if (ls != neg_inf()) sum += exp2f((warp_sum(x) * a.scale - ls) * kLog2e);
            }
        }
    }
    if (lane == 0) a.w_out[at] = (a.w_in ? a.decay * a.w_in[at] : 0.f) + sum;
}

}  // namespace

#define GMS_BY_TYPE(K, ...)                                                           \
    do {                                                                              \
        if (dtype == GMS_DTYPE_BF16) {                                                \
            if (head_dim == 64) K<__nv_bfloat16, 64> __VA_ARGS__; else K<__nv_bfloat16, 128> __VA_ARGS__; \
        } else {                                                                      \
            if (head_dim == 64) K<__half, 64> __VA_ARGS__; else K<__half, 128> __VA_ARGS__; \
        }                                                                             \
    } while (0)

cudaError_t launch_kv_attention_rows(const AttnArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    const uint64_t rows = (uint64_t)a.total_q * a.n_heads;
    const uint32_t grid = (uint32_t)((rows + 3) / 4);
    if (grid == 0) return cudaSuccess;
    GMS_BY_TYPE(kv_attention_rows_kernel, <<<grid, 128, 0, s>>>(a));
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_kv_weights(const AttnArgs &a, const float *lse, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    const uint64_t warps = (uint64_t)a.n_seq * a.n_kv * a.max_kv;
    const uint32_t grid = (uint32_t)((warps + 3) / 4);
    if (grid == 0) return cudaSuccess;
    GMS_BY_TYPE(kv_weights_kernel, <<<grid, 128, 0, s>>>(a, lse));
    count_launches(1);
    return cudaGetLastError();
}

namespace {

int bad_pool(const gms_kv_pool *p)
{
    if (!p->base) return GMS_ERR_NULL;
    if (p->block_bytes == 0 || p->block_bytes % kBlockBytes) return GMS_ERR_ALIGN;
    if ((reinterpret_cast<uint64_t>(p->base) | p->plane_stride | p->block_stride) & 15u) return GMS_ERR_ALIGN;
    if (p->block_bytes > kMaxChunkBlocks * kBlockBytes || p->n_blocks == 0 || p->n_blocks > 0x7fffffffu) return GMS_ERR_ARG;
    if (p->block_stride < p->block_bytes && p->n_blocks > 1) return GMS_ERR_ARG;
    if (p->block_stride >> 40 || p->flags & ~GMS_KV_IMAGE_BY_ID) return GMS_ERR_ARG;
    if (p->n_planes > 1 && p->plane_stride < (uint64_t)(p->n_blocks - 1) * p->block_stride + p->block_bytes) return GMS_ERR_ARG;
    return GMS_OK;
}

int bad_layout(const gms_kv_pool *p, const gms_kv_layout *l)
{
    if ((l->token_stride | l->head_stride) & 15u) return GMS_ERR_ALIGN;
    if (l->dtype > GMS_DTYPE_F16 || (l->head_dim != 64 && l->head_dim != 128) || l->n_kv_heads == 0) return GMS_ERR_ARG;
    if (l->block_tokens < 16 || l->block_tokens > 1024 || l->block_tokens & (l->block_tokens - 1)) return GMS_ERR_ARG;
    if (l->k_plane >= p->n_planes || l->v_plane >= p->n_planes || l->k_plane == l->v_plane) return GMS_ERR_ARG;
    const uint64_t row = l->head_dim * 2, heads = l->n_kv_heads, tokens = l->block_tokens;
    const uint64_t ts = l->token_stride, hs = l->head_stride;
    if ((tokens - 1) * ts + (heads - 1) * hs + row > p->block_bytes) return GMS_ERR_ARG;
    const bool tokens_outside = (heads == 1 || hs >= row) && ts >= (heads - 1) * hs + row;
    const bool heads_outside = ts >= row && (heads == 1 || hs >= (tokens - 1) * ts + row);
    return tokens_outside || heads_outside ? GMS_OK : GMS_ERR_ARG;
}

uint32_t log2_of(uint32_t x) { return 31u - (uint32_t)__builtin_clz(x); }

// Checks everything a call is given and fills in the kernels' arguments.  `planning`: workspace pointers are not looked at.
int make_args(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *t, const gms_kv_weight *w,
              const gms_kv_prefix *x, AttnArgs *a)
{
    if (!pool || !layout || !t) return GMS_ERR_NULL;
    int rc = bad_pool(pool);
    if (rc == GMS_OK) rc = bad_layout(pool, layout);
    if (rc != GMS_OK) return rc;
    if (t->n_heads == 0 || t->n_heads % layout->n_kv_heads || !std::isfinite(t->scale)) return GMS_ERR_ARG;
    if (t->total_q > 0x7fffffffu || t->n_seq > 0x7fffffffu || t->max_kv > 0x7fffffffu || t->max_q > t->total_q) return GMS_ERR_ARG;
    if ((uint64_t)t->total_q * t->n_heads > 0x7fffffffull) return GMS_ERR_RANGE;
    if (!t->cu_q && (t->total_q != t->n_seq || (t->n_seq && t->max_q != 1))) return GMS_ERR_ARG;
    const bool work = t->n_seq && t->total_q;
    if (work && (!t->q || !t->out)) return GMS_ERR_NULL;
    if (t->n_seq && (!t->kv_lens || (t->max_kv && !t->block_table))) return GMS_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(t->q) | reinterpret_cast<uint64_t>(t->out) | t->q_token_stride | t->q_head_stride |
         t->out_token_stride | t->out_head_stride) & 15u)
        return GMS_ERR_ALIGN;
    if ((reinterpret_cast<uint64_t>(t->lse) | reinterpret_cast<uint64_t>(t->cu_q) | reinterpret_cast<uint64_t>(t->kv_lens) |
         reinterpret_cast<uint64_t>(t->block_table)) & 3u || reinterpret_cast<uint64_t>(t->status) & 7u ||
        reinterpret_cast<uint64_t>(t->workspace) & 255u)
        return GMS_ERR_ALIGN;
    if (t->table_stride > (1ull << 40) || t->table_stride * layout->block_tokens < t->max_kv) return GMS_ERR_RANGE;
    *a = {};
    a->k_base = static_cast<const uint8_t *>(pool->base) + layout->k_plane * pool->plane_stride;
    a->v_base = static_cast<const uint8_t *>(pool->base) + layout->v_plane * pool->plane_stride;
    a->block_stride = pool->block_stride;
    a->n_blocks = pool->n_blocks;
    a->token_stride = layout->token_stride;
    a->head_stride = layout->head_stride;
    a->block_shift = log2_of(layout->block_tokens);
    a->q = static_cast<const uint8_t *>(t->q);
    a->out = static_cast<uint8_t *>(t->out);
    a->lse = t->lse;
    a->cu_q = t->cu_q;
    a->kv_lens = t->kv_lens;
    a->table = t->block_table;
    a->table_stride = t->table_stride;
    a->q_token_stride = t->q_token_stride;
    a->q_head_stride = t->q_head_stride;
    a->out_token_stride = t->out_token_stride;
    a->out_head_stride = t->out_head_stride;
    a->n_seq = t->n_seq;
    a->n_heads = t->n_heads;
    a->n_kv = layout->n_kv_heads;
    a->group = t->n_heads / layout->n_kv_heads;
    a->total_q = t->total_q;
    a->max_q = t->max_q;
    a->max_kv = t->max_kv;
    a->window = t->window;
    a->sinks = t->sinks;
    a->scale = t->scale;
    a->status = reinterpret_cast<unsigned long long *>(t->status);
    if (w) {
        if (w->reserved) return GMS_ERR_ARG;
        if (t->n_seq && t->max_kv && !w->out) return GMS_ERR_NULL;
        if ((reinterpret_cast<uint64_t>(w->in) | reinterpret_cast<uint64_t>(w->out)) & 3u) return GMS_ERR_ALIGN;
        if (!std::isfinite(w->decay)) return GMS_ERR_ARG;
        if ((uint64_t)t->n_seq * layout->n_kv_heads * t->max_kv > (1ull << 32)) return GMS_ERR_RANGE;
        a->w_in = w->in;
        a->w_out = w->out;
        a->w_seq_stride = w->seq_stride;
        a->w_head_stride = w->head_stride;
        a->decay = w->decay;
    }
    if (x) {
        if (t->window || t->sinks || x->reserved || x->max_prefix > 0x7fffffffu || x->n_groups > t->n_seq || x->max_group_q > t->total_q)
            return GMS_ERR_ARG;
        if (x->n_groups && (!x->group_start || !x->prefix_lens || (x->max_prefix && !x->prefix_table))) return GMS_ERR_NULL;
        if ((reinterpret_cast<uint64_t>(x->group_start) | reinterpret_cast<uint64_t>(x->prefix_lens) |
             reinterpret_cast<uint64_t>(x->prefix_table)) & 3u)
            return GMS_ERR_ALIGN;
        if (x->prefix_stride > (1ull << 40) || (x->n_groups && x->prefix_stride * layout->block_tokens < x->max_prefix))
            return GMS_ERR_RANGE;
        a->group_start = x->group_start;
        a->prefix_lens = x->prefix_lens;
        a->prefix_table = x->prefix_table;
        a->prefix_stride = x->prefix_stride;
        a->n_groups = x->n_groups;
        a->max_prefix = x->max_prefix;
        a->max_group_q = x->max_group_q;
    }
    return GMS_OK;
}

uint64_t workspace_bytes(const AttnArgs &a)
{
    uint64_t n = 0;
    if (a.w_out && !a.lse) n += (uint64_t)a.total_q * a.n_heads * 4;  // the weights pass needs the log-sum-exps
    return (n + 255) / 256 * 256;
}

int attention_call(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *t, const gms_kv_weight *w,
                   const gms_kv_prefix *x, void *stream)
{
    AttnArgs a;
    const int rc = make_args(pool, layout, t, w, x, &a);
    if (rc != GMS_OK) return rc;
    const uint64_t need = workspace_bytes(a);
    if (need && !t->workspace) return GMS_ERR_NULL;
    if (need > t->workspace_bytes) return GMS_ERR_RANGE;
    if (a.n_seq == 0) return GMS_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (w && !a.lse) a.lse = static_cast<float *>(t->workspace);
    cudaError_t e = launch_kv_attention_rows(a, layout->dtype, layout->head_dim, s);
    if (e == cudaSuccess && w) e = launch_kv_weights(a, a.lse, layout->dtype, layout->head_dim, s);
    return e == cudaSuccess ? GMS_OK : report_cuda_error(e);
}

}  // namespace
}  // namespace gms

extern "C" {

int gms_kv_attention_workspace(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                               const gms_kv_weight *weight, uint64_t *nbytes)
{
    if (!nbytes) return GMS_ERR_NULL;
    gms::AttnArgs a;
    const int rc = gms::make_args(pool, layout, attn, weight, nullptr, &a);
    if (rc == GMS_OK) *nbytes = gms::workspace_bytes(a);
    return rc;
}

int gms_kv_attention(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn, const gms_kv_weight *weight,
                     void *stream)
{
    return gms::attention_call(pool, layout, attn, weight, nullptr, stream);
}

int gms_kv_attention_shared_workspace(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                                      const gms_kv_prefix *prefix, uint64_t *nbytes)
{
    if (!nbytes || !prefix) return GMS_ERR_NULL;
    gms::AttnArgs a;
    const int rc = gms::make_args(pool, layout, attn, nullptr, prefix, &a);
    if (rc == GMS_OK) *nbytes = gms::workspace_bytes(a);
    return rc;
}

int gms_kv_attention_shared(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                            const gms_kv_prefix *prefix, void *stream)
{
    if (!prefix) return GMS_ERR_NULL;
    return gms::attention_call(pool, layout, attn, nullptr, prefix, stream);
}

int gms_kv_evict(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_evict_args *t, void *stream)
{
    if (!pool || !layout || !t) return GMS_ERR_NULL;
    int rc = gms::bad_pool(pool);
    if (rc == GMS_OK) rc = gms::bad_layout(pool, layout);
    if (rc != GMS_OK) return rc;
    if (t->reserved || t->max_len > 0x7fffffffu || t->budget > 0x7fffffffu || (uint64_t)t->sinks + t->recent > t->budget)
        return GMS_ERR_ARG;
    if (t->n_layers) {
        const uint64_t last = (uint64_t)(t->n_layers - 1) * t->layer_planes;
        const uint32_t apart = layout->k_plane > layout->v_plane ? layout->k_plane - layout->v_plane : layout->v_plane - layout->k_plane;
        if (last + (layout->k_plane > layout->v_plane ? layout->k_plane : layout->v_plane) >= pool->n_planes) return GMS_ERR_ARG;
        // two layers must not share a plane
        if (t->n_layers > 1 && (t->layer_planes == 0 || (apart % t->layer_planes == 0 && apart / t->layer_planes < t->n_layers)))
            return GMS_ERR_ARG;
    }
    if ((reinterpret_cast<uint64_t>(t->weights) | reinterpret_cast<uint64_t>(t->weights_out) | reinterpret_cast<uint64_t>(t->lens) |
         reinterpret_cast<uint64_t>(t->lens_out) | reinterpret_cast<uint64_t>(t->src_table) | reinterpret_cast<uint64_t>(t->dst_table) |
         reinterpret_cast<uint64_t>(t->kept)) & 3u)
        return GMS_ERR_ALIGN;
    const uint64_t rows = (uint64_t)t->n_layers * t->n_seq * layout->n_kv_heads;
    const uint32_t most = t->max_len < t->budget ? t->max_len : t->budget;
    if (rows > 0x7fffffffull || rows * ((most + 63ull) / 64) > 0x7fffffffull) return GMS_ERR_RANGE;
    if (t->src_stride > (1ull << 40) || t->dst_stride > (1ull << 40) || t->src_stride * layout->block_tokens < t->max_len ||
        t->dst_stride * layout->block_tokens < most)
        return GMS_ERR_RANGE;
    if (rows == 0) return GMS_OK;
    if (!t->lens || (t->max_len && (!t->weights || !t->src_table)) || (t->budget && !t->kept) || (most && !t->dst_table))
        return GMS_ERR_NULL;
    if (t->weights_out && t->weights_out == t->weights) return GMS_ERR_ARG;
    gms::EvictArgs a = {};
    a.base = static_cast<uint8_t *>(pool->base);
    a.plane_stride = pool->plane_stride;
    a.block_stride = pool->block_stride;
    a.k_plane = layout->k_plane;
    a.v_plane = layout->v_plane;
    a.n_blocks = pool->n_blocks;
    a.token_stride = layout->token_stride;
    a.head_stride = layout->head_stride;
    a.block_shift = gms::log2_of(layout->block_tokens);
    a.row_bytes = layout->head_dim * 2;
    a.weights = t->weights;
    a.weights_out = t->weights_out;
    a.lens = t->lens;
    a.lens_out = t->lens_out;
    a.src_table = t->src_table;
    a.dst_table = t->dst_table;
    a.kept = t->kept;
    a.w_layer_stride = t->w_layer_stride;
    a.w_seq_stride = t->w_seq_stride;
    a.w_head_stride = t->w_head_stride;
    a.o_layer_stride = t->o_layer_stride;
    a.o_seq_stride = t->o_seq_stride;
    a.o_head_stride = t->o_head_stride;
    a.src_stride = t->src_stride;
    a.dst_stride = t->dst_stride;
    a.n_layers = t->n_layers;
    a.layer_planes = t->layer_planes;
    a.n_seq = t->n_seq;
    a.n_kv = layout->n_kv_heads;
    a.max_len = t->max_len;
    a.budget = t->budget;
    a.sinks = t->sinks;
    a.recent = t->recent;
    const cudaError_t e = gms::launch_kv_evict(a, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? GMS_OK : gms::report_cuda_error(e);
}

}  // extern "C"
