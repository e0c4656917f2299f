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
// nothing is exchanged), the lanes behind those the elements that are not rotated.  A warp takes a run of a row's heads, first the
// queries', then the keys', then the values', in batches of 4 x 32 / (D / 8), the next batch on its way while one is computed.
// Cosines and sines are made once for all of them, by all lanes.  Bound by memory where there are many rows, by latency where there
// are few (then a warp has one batch).
constexpr uint32_t kAppendThreads = 256, kUnroll = 4;

template <class T, int D>
__global__ void __launch_bounds__(kAppendThreads, 3) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr uint32_t L = D / 8, G = 32 / L, B = G * kUnroll;  // lanes a row, rows at a time, rows a batch
    const uint32_t lane = threadIdx.x & 31u, l = lane % L, sub = lane / L;
    const uint64_t item = (uint64_t)blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32;
    const uint32_t row = a.parts == 1 ? (uint32_t)item : (uint32_t)(item / a.parts), part = a.parts == 1 ? 0 : (uint32_t)(item % a.parts);
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    if (row >= a.rows) return;
    const uint32_t groups = a.rotary / 8;
    const bool turned = l < groups, halves = a.pairs == GMS_PAIR_HALVES;
    uint32_t e0, e1;  // the lane's two runs of four elements
    if (halves && turned) e0 = 4 * l, e1 = e0 + a.rotary / 2;
    else e0 = 8 * l, e1 = e0 + 4;
    const uint32_t apart = (e1 - e0) * 2;
    const uint8_t *q = a.q + row * a.q_token + e0 * 2, *k = a.k + row * a.k_token + e0 * 2, *v = a.v + row * a.v_token + e0 * 2;
    // the part's heads: queries h0 .. q_end - 1 and so on, in the order q, k, v
    const uint32_t heads = a.n_heads + 2 * a.n_kv, h0 = part * a.per_part, h1 = min(h0 + a.per_part, heads), k0 = a.n_heads, v0 = a.n_heads + a.n_kv;
    auto kind_end = [&](uint32_t h) { return min(h1, h < k0 ? k0 : h < v0 ? v0 : heads); };  // of the kind that head h has
    struct Batch {
        uint2 x[kUnroll][2];
    };
    auto load = [&](uint32_t h, Batch &x) {
        const uint32_t end = kind_end(h);
        const uint8_t *p = h < k0 ? q : h < v0 ? k : v;
        const uint64_t stride = h < k0 ? a.q_head : h < v0 ? a.k_head : a.v_head;
        p += (h - (h < k0 ? 0 : h < v0 ? k0 : v0) + sub) * stride;
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            if (h + u * G + sub < end) {
                x.x[u][0] = *reinterpret_cast<const uint2 *>(p);
                x.x[u][1] = *reinterpret_cast<const uint2 *>(p + apart);
            }
            p += G * stride;
        }
    };
    Batch x, y;
    load(h0, x);
    if (a.n_rows && (int64_t)row >= (int64_t)*a.n_rows) return;
    uint64_t to = 0;
    bool kept = false;
    if (h1 > k0 && a.n_kv) {
        const int64_t slot = a.slots[row];
        kept = slot >= 0 && (slot >> a.block_shift) < (int64_t)a.n_blocks;
        if (kept) to = (uint64_t)(slot >> a.block_shift) * a.block_stride + (uint64_t)(slot & ((1 << a.block_shift) - 1)) * a.token_stride + e0 * 2;
    }
    float c[4], s[4];
    if (groups && h0 < v0) {  // the G lanes that need the same four angles make 4 / G each
        constexpr uint32_t E = 4 / G;
        float mc[E], ms[E];
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) {
            const uint32_t j = min(4 * l + sub * E + i, a.rotary / 2 - 1), axis = a.axes ? min((uint32_t)a.axes[j], a.n_axes - 1) : 0;
            // in turns: what is left of them after the whole ones is exact enough in 32 bits, the product before is not
            const double turns = (double)a.positions[axis * a.positions_stride + row] * (double)a.inv_freq[j] * 0.15915494309189533577;
            float sn, cs;
            sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
            mc[i] = cs * a.rope_scale;
            ms[i] = sn * a.rope_scale;
        }
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            c[i] = __shfl_sync(0xffffffffu, mc[i % E], l + i / E * L);
            s[i] = __shfl_sync(0xffffffffu, ms[i % E], l + i / E * L);
        }
    }
    for (uint32_t h = h0; h < h1;) {
        const uint32_t end = kind_end(h), next = min(h + B, end);
        if (next < h1) load(next, y);
        const bool is_q = h < k0, is_v = h >= v0;
        if (!is_v) {
            const void *weight = is_q ? a.q_weight : a.k_weight;
            float w[8];
            if (weight) load_weights(a, weight, e0, w), load_weights(a, weight, e1, w + 4);
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u) {
                if (h + u * G >= end) break;
                float f[8];
                unpack4<T>(x.x[u][0], f);
                unpack4<T>(x.x[u][1], f + 4);
                if (weight) {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum += f[e] * f[e];
#pragma unroll
                    for (uint32_t o = L / 2; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    const float r = rsqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= r * w[e];
                }
                if (turned) {
                    if (halves) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x0 = f[e], x1 = f[e + 4];
                            f[e] = x0 * c[e] - x1 * s[e];
                            f[e + 4] = x1 * c[e] + x0 * s[e];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x0 = f[2 * e], x1 = f[2 * e + 1];
                            f[2 * e] = x0 * c[e] - x1 * s[e];
                            f[2 * e + 1] = x1 * c[e] + x0 * s[e];
                        }
                    }
                }
                x.x[u][0] = pack4<T>(f), x.x[u][1] = pack4<T>(f + 4);
            }
        }
        if (is_q || kept) {
            const uint64_t stride = is_q ? a.o_head : a.head_stride;
            uint8_t *p = is_q ? a.q_out + row * a.o_token + e0 * 2 : (is_v ? a.v_base : a.k_base) + to;
            p += (h - (is_q ? 0 : is_v ? v0 : k0) + sub) * stride;
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u) {
                if (h + u * G + sub < end) {
                    *reinterpret_cast<uint2 *>(p) = x.x[u][0];
                    *reinterpret_cast<uint2 *>(p + apart) = x.x[u][1];
                }
                p += G * stride;
            }
        }
        x = y;
        h = next;
    }
}

template <class T>
cudaError_t launch_append(AppendArgs &a, uint32_t dim, cudaStream_t s)
{
    const uint32_t heads = a.n_heads + 2 * a.n_kv, batch = (dim == 128 ? 2 : 4) * kUnroll;
    // A warp a row where that fills the GPU; with fewer rows they are cut, down to a batch a warp.
    const uint64_t fill = 148 * 24, batches = (heads + batch - 1) / batch;
    const uint64_t want = a.rows >= fill ? 1 : (fill + a.rows - 1) / a.rows, cuts = want < batches ? want : batches;
    a.per_part = (uint32_t)((batches + cuts - 1) / cuts) * batch;
    a.parts = (heads + a.per_part - 1) / a.per_part;
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
