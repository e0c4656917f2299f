// Queries and keys normed and rotated, keys and values into the paged KV pool.
#include <cmath>

#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_ptx.h"

namespace gms {
namespace {

struct AppendArgs {
    const uint8_t *q, *k, *v;
    uint8_t *q_out, *k_base, *v_base;
    const int64_t *slots;
    const int32_t *positions, *n_rows;
    const float *inv_freq;
    const uint8_t *axes;
    const void *q_weight, *k_weight;
    uint64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head, block_stride, positions_stride;
    uint32_t token_stride, head_stride, block_shift, n_blocks;
    uint32_t rows, n_heads, n_kv, rotary, n_axes, pairs, weight_dtype;
    uint32_t parts, per_part;  // a row's q, k and v heads are cut into `parts` runs of `per_part`, a warp each
    float offset, eps, rope_scale;
};

template <class T>
__device__ __forceinline__ void unpack4(uint2 x, float *f)
{
    const T *e = reinterpret_cast<const T *>(&x);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = to_f32(e[i]);
}
template <class T>
__device__ __forceinline__ uint2 pack4(const float *f)
{
    return make_uint2(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()));
}
// Four weights from element e on.
__device__ __forceinline__ void load_weights(const AppendArgs &a, const void *w, uint32_t e, float *f)
{
    if (a.weight_dtype == GMS_DTYPE_F32) {
        const float4 x = reinterpret_cast<const float4 *>(w)[e / 4];
        f[0] = x.x, f[1] = x.y, f[2] = x.z, f[3] = x.w;
    } else {
        const uint2 x = reinterpret_cast<const uint2 *>(w)[e / 4];
        if (a.weight_dtype == GMS_DTYPE_BF16) unpack4<__nv_bfloat16>(x, f);
        else unpack4<__half>(x, f);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] += a.offset;
}

// D / 8 lanes hold a head's row, eight elements each: lane l the pairs of frequencies 4l .. 4l + 3 (both halves of them, so that
// nothing is exchanged), the lanes behind those the elements that are not rotated.  A warp takes a run of a token's heads, 32 / (D / 8)
// at a time, kUnroll loads in flight; angles are made once for all of them.
constexpr uint32_t kAppendThreads = 256, kUnroll = 4;

template <class T, int D>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr uint32_t L = D / 8, G = 32 / L;  // lanes a row, rows at a time
    const uint32_t lane = threadIdx.x & 31u, l = lane % L, sub = lane / L;
    const uint64_t item = (uint64_t)blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32;
    const uint32_t row = (uint32_t)(item / a.parts), part = (uint32_t)(item % a.parts);
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    if (row >= a.rows || (a.n_rows && (int64_t)row >= (int64_t)*a.n_rows)) return;
    const uint32_t groups = a.rotary / 8;
    const bool turned = l < groups;
    uint32_t e0, e1;  // the lane's two runs of four elements
    if (a.pairs == GMS_PAIR_NEIGHBOURS || !turned) e0 = 8 * l, e1 = e0 + 4;
    else e0 = 4 * l, e1 = e0 + a.rotary / 2;
    float c[4], s[4];
    if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t j = 4 * l + i, axis = a.axes ? min((uint32_t)a.axes[j], a.n_axes - 1) : 0;
            // in turns: what is left of them after the whole ones is exact enough in 32 bits, the product before is not
            const double turns = (double)a.positions[axis * a.positions_stride + row] * (double)a.inv_freq[j] * 0.15915494309189533577;
            float sn, cs;
            sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
            c[i] = cs * a.rope_scale;
            s[i] = sn * a.rope_scale;
        }
    }
    const uint32_t heads = a.n_heads + 2 * a.n_kv, h0 = part * a.per_part, h1 = min(h0 + a.per_part, heads);
    float wq[8], wk[8];
    if (a.q_weight && h0 < a.n_heads) load_weights(a, a.q_weight, e0, wq), load_weights(a, a.q_weight, e1, wq + 4);
    if (a.k_weight && h0 < a.n_heads + a.n_kv && h1 > a.n_heads) load_weights(a, a.k_weight, e0, wk), load_weights(a, a.k_weight, e1, wk + 4);
    uint64_t to = 0;
    bool kept = false;
    if (h1 > a.n_heads && a.n_kv) {
        const int64_t slot = a.slots[row];
        kept = slot >= 0 && (slot >> a.block_shift) < (int64_t)a.n_blocks;
        if (kept) to = (uint64_t)(slot >> a.block_shift) * a.block_stride + (uint64_t)(slot & ((1 << a.block_shift) - 1)) * a.token_stride;
    }
    for (uint32_t h = h0; h < h1; h += G * kUnroll) {
        uint2 x[kUnroll][2];
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            const uint32_t i = h + u * G + sub;
            if (i >= h1) continue;
            const uint8_t *p = i < a.n_heads ? a.q + row * a.q_token + i * a.q_head
                               : i < a.n_heads + a.n_kv ? a.k + row * a.k_token + (i - a.n_heads) * a.k_head
                                                        : a.v + row * a.v_token + (i - a.n_heads - a.n_kv) * a.v_head;
            x[u][0] = *reinterpret_cast<const uint2 *>(p + e0 * 2);
            x[u][1] = *reinterpret_cast<const uint2 *>(p + e1 * 2);
        }
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            const uint32_t i = h + u * G + sub;
            const bool in = i < h1, is_q = i < a.n_heads, is_v = i >= a.n_heads + a.n_kv;
            uint8_t *p = nullptr;
            if (in && is_q) p = a.q_out + row * a.o_token + i * a.o_head;
            else if (in && kept) p = is_v ? a.v_base + to + (uint64_t)(i - a.n_heads - a.n_kv) * a.head_stride
                                          : a.k_base + to + (uint64_t)(i - a.n_heads) * a.head_stride;
            if (__any_sync(0xffffffffu, in && !is_v)) {
                float f[8];
                unpack4<T>(x[u][0], f);
                unpack4<T>(x[u][1], f + 4);
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += f[e] * f[e];
#pragma unroll
                for (uint32_t o = L / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                const bool normed = is_q ? a.q_weight != nullptr : a.k_weight != nullptr;
                if (normed) {
                    const float r = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= r * (is_q ? wq[e] : wk[e]);
                }
                if (turned) {
                    if (a.pairs == GMS_PAIR_NEIGHBOURS) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x0 = f[2 * e], x1 = f[2 * e + 1];
                            f[2 * e] = x0 * c[e] - x1 * s[e];
                            f[2 * e + 1] = x1 * c[e] + x0 * s[e];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x0 = f[e], x1 = f[e + 4];
                            f[e] = x0 * c[e] - x1 * s[e];
                            f[e + 4] = x1 * c[e] + x0 * s[e];
                        }
                    }
                }
                if (!is_v) x[u][0] = pack4<T>(f), x[u][1] = pack4<T>(f + 4);
            }
            if (p) {
                *reinterpret_cast<uint2 *>(p + e0 * 2) = x[u][0];
                *reinterpret_cast<uint2 *>(p + e1 * 2) = x[u][1];
            }
        }
    }
}

template <class T>
cudaError_t launch_append(AppendArgs &a, uint32_t dim, cudaStream_t s)
{
    const uint32_t heads = a.n_heads + 2 * a.n_kv, at_once = (dim == 128 ? 2 : 4) * kUnroll;
    a.parts = (heads + at_once - 1) / at_once;
    a.per_part = at_once;
    const uint64_t warps = (uint64_t)a.rows * a.parts, grid = (warps + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    if (grid > 0x7fffffffull) return cudaErrorInvalidValue;
    return dim == 128 ? launch_dependent(kv_append_kernel<T, 128>, (uint32_t)grid, kAppendThreads, 0, s, a)
                      : launch_dependent(kv_append_kernel<T, 64>, (uint32_t)grid, kAppendThreads, 0, s, a);
}

}  // namespace
}  // namespace gms

extern "C" int gms_kv_append(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_append_args *t, void *stream)
{
    if (!pool || !layout || !t) return GMS_ERR_NULL;
    int rc = gms::bad_pool(pool);
    if (rc == GMS_OK) rc = gms::bad_layout(pool, layout);
    if (rc != GMS_OK) return rc;
    if (t->reserved || t->rotary_dim % 8 || t->rotary_dim > layout->head_dim || t->n_axes == 0 || t->n_axes > 8 || t->pairs > GMS_PAIR_NEIGHBOURS ||
        t->weight_dtype > GMS_DTYPE_F32)
        return GMS_ERR_ARG;
    if (!std::isfinite(t->weight_offset) || !std::isfinite(t->eps) || t->eps < 0.f || !std::isfinite(t->rope_scale)) return GMS_ERR_ARG;
    if (t->rows > 0x7fffffffu || t->n_heads > 65536u || layout->n_kv_heads > 65536u) return GMS_ERR_ARG;
    if ((t->q == nullptr) != (t->n_heads == 0) || (t->q == nullptr) != (t->q_out == nullptr) || (t->k == nullptr) != (t->v == nullptr))
        return GMS_ERR_NULL;
    if (t->k && t->rows && !t->slots) return GMS_ERR_NULL;
    if (t->rotary_dim && t->rows && (!t->positions || !t->inv_freq)) return GMS_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(t->q) | reinterpret_cast<uint64_t>(t->k) | reinterpret_cast<uint64_t>(t->v) |
         reinterpret_cast<uint64_t>(t->q_out) | reinterpret_cast<uint64_t>(t->q_weight) | reinterpret_cast<uint64_t>(t->k_weight) |
         t->q_token_stride | t->q_head_stride | t->k_token_stride | t->k_head_stride | t->v_token_stride | t->v_head_stride |
         t->out_token_stride | t->out_head_stride) & 15u)
        return GMS_ERR_ALIGN;
    if ((reinterpret_cast<uint64_t>(t->positions) | reinterpret_cast<uint64_t>(t->n_rows) | reinterpret_cast<uint64_t>(t->inv_freq)) & 3u ||
        reinterpret_cast<uint64_t>(t->slots) & 7u)
        return GMS_ERR_ALIGN;
    if (t->rotary_dim && (t->positions_stride < t->rows || t->positions_stride >> 40)) return GMS_ERR_RANGE;
    if (t->q && t->q == t->q_out && (t->q_token_stride != t->out_token_stride || t->q_head_stride != t->out_head_stride)) return GMS_ERR_ARG;
    const uint64_t heads = (uint64_t)t->n_heads + (t->k ? 2ull * layout->n_kv_heads : 0);
    if (t->rows * heads > 1ull << 36) return GMS_ERR_RANGE;
    if (t->rows == 0 || heads == 0) return GMS_OK;
    gms::AppendArgs a = {};
    a.q = static_cast<const uint8_t *>(t->q);
    a.k = static_cast<const uint8_t *>(t->k);
    a.v = static_cast<const uint8_t *>(t->v);
    a.q_out = static_cast<uint8_t *>(t->q_out);
    a.k_base = static_cast<uint8_t *>(pool->base) + layout->k_plane * pool->plane_stride;
    a.v_base = static_cast<uint8_t *>(pool->base) + layout->v_plane * pool->plane_stride;
    a.slots = t->slots;
    a.positions = t->positions;
    a.n_rows = t->n_rows;
    a.inv_freq = t->inv_freq;
    a.axes = t->axes;
    a.q_weight = t->q_weight;
    a.k_weight = t->k_weight;
    a.q_token = t->q_token_stride;
    a.q_head = t->q_head_stride;
    a.k_token = t->k_token_stride;
    a.k_head = t->k_head_stride;
    a.v_token = t->v_token_stride;
    a.v_head = t->v_head_stride;
    a.o_token = t->out_token_stride;
    a.o_head = t->out_head_stride;
    a.block_stride = pool->block_stride;
    a.positions_stride = t->positions_stride;
    a.token_stride = layout->token_stride;
    a.head_stride = layout->head_stride;
    a.block_shift = gms::log2_of(layout->block_tokens);
    a.n_blocks = pool->n_blocks;
    a.rows = t->rows;
    a.n_heads = t->n_heads;
    a.n_kv = t->k ? layout->n_kv_heads : 0;
    a.rotary = t->rotary_dim;
    a.n_axes = t->n_axes;
    a.pairs = t->pairs;
    a.weight_dtype = t->weight_dtype;
    a.offset = t->weight_offset;
    a.eps = t->eps;
    a.rope_scale = t->rope_scale;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = layout->dtype == GMS_DTYPE_BF16 ? gms::launch_append<__nv_bfloat16>(a, layout->head_dim, s)
                                                          : gms::launch_append<__half>(a, layout->head_dim, s);
    return e == cudaSuccess ? GMS_OK : gms::report_cuda_error(e);
}
