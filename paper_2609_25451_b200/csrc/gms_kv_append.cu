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

// The two numbers in a word.
__device__ __forceinline__ float2 both(uint32_t x, __nv_bfloat16) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }
__device__ __forceinline__ float2 both(uint32_t x, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&x)); }

// Eight elements of a row, as the first and the second elements of four pairs: four neighbours each (HALVES, x: elements e0 .., y:
// elements e1 ..), or every other one of eight neighbours.
template <bool HALVES, class T>
__device__ __forceinline__ void pairs_of(const uint2 *x, float2 *a, float2 *b)
{
    const float2 p = both(x[0].x, T()), q = both(x[0].y, T()), r = both(x[1].x, T()), s = both(x[1].y, T());
    if (HALVES) a[0] = p, a[1] = q, b[0] = r, b[1] = s;
    else a[0] = make_float2(p.x, q.x), b[0] = make_float2(p.y, q.y), a[1] = make_float2(r.x, s.x), b[1] = make_float2(r.y, s.y);
}
template <bool HALVES, class T>
__device__ __forceinline__ void pack_pairs(const float2 *a, const float2 *b, uint2 *x)
{
    if (HALVES) {
        x[0] = make_uint2(pack2(a[0].x, a[0].y, T()), pack2(a[1].x, a[1].y, T()));
        x[1] = make_uint2(pack2(b[0].x, b[0].y, T()), pack2(b[1].x, b[1].y, T()));
    } else {
        x[0] = make_uint2(pack2(a[0].x, b[0].x, T()), pack2(a[0].y, b[0].y, T()));
        x[1] = make_uint2(pack2(a[1].x, b[1].x, T()), pack2(a[1].y, b[1].y, T()));
    }
}
// The weights of the same elements.
template <bool HALVES>
__device__ __forceinline__ void weights_of(const AppendArgs &a, const void *w, uint32_t e0, uint32_t e1, float2 *x, float2 *y)
{
    if (a.weight_dtype == GMS_DTYPE_F32) {
        const float4 p = reinterpret_cast<const float4 *>(w)[e0 / 4], q = reinterpret_cast<const float4 *>(w)[e1 / 4];
        if (HALVES) x[0] = make_float2(p.x, p.y), x[1] = make_float2(p.z, p.w), y[0] = make_float2(q.x, q.y), y[1] = make_float2(q.z, q.w);
        else x[0] = make_float2(p.x, p.z), y[0] = make_float2(p.y, p.w), x[1] = make_float2(q.x, q.z), y[1] = make_float2(q.y, q.w);
    } else {
        const uint2 p[2] = {reinterpret_cast<const uint2 *>(w)[e0 / 4], reinterpret_cast<const uint2 *>(w)[e1 / 4]};
        if (a.weight_dtype == GMS_DTYPE_BF16) pairs_of<HALVES, __nv_bfloat16>(p, x, y);
        else pairs_of<HALVES, __half>(p, x, y);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i].x += a.offset, x[i].y += a.offset, y[i].x += a.offset, y[i].y += a.offset;
}

// D / 8 lanes hold a head's row, eight elements each: lane l the pairs of frequencies 4l .. 4l + 3 (both halves of them, so that
// nothing is exchanged), the lanes behind those the elements that are not rotated.  A warp takes 256 / D neighbouring rows, and a
// run of their heads, first the queries', then the keys', then the values', kUnroll at a time, the next ones on their way while these
// are computed; what differs between the lanes (row, angles) stays the same for all of them.  Two pairs are computed an instruction.
// Bound by memory where there are many rows (52,367 of 32 / 8 heads of 64: 111 us, 5.8 TB/s, with 970 instructions a row; a
// warp with several heads of one row took 1,800 and 145 us), by latency where there are few (then a warp has kUnroll heads).  20
// warps an SM: with 24 and fewer registers, or 16, the same rows take 125 us; each a CTA of its own, so that none waits for others
// to end (in fours 115 us, and 6,776 rows of 16 / 4 heads of 128 21.0 us against 19.9).
constexpr uint32_t kAppendThreads = 32, kAppendCtas = 20, kUnroll = 4;

template <class T, int D, bool HALVES>
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr uint32_t L = D / 8, G = 32 / L;  // lanes a row, rows a warp
    const uint32_t lane = threadIdx.x & 31u, l = lane % L;
    const uint32_t item = blockIdx.x * (kAppendThreads / 32) + threadIdx.x / 32, part = a.parts == 1 ? 0 : item % a.parts;
    const uint64_t mine = (uint64_t)(a.parts == 1 ? item : item / a.parts) * G + lane / L;
    const uint32_t row = (uint32_t)min(mine, (uint64_t)a.rows - 1);  // (lanes without a row read the last one's and write nothing)
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    const uint32_t groups = a.rotary / 8;
    const bool turned = l < groups;
    uint32_t e0, e1;  // the lane's two runs of four elements
    if (HALVES && turned) e0 = 4 * l, e1 = e0 + a.rotary / 2;
    else e0 = 8 * l, e1 = e0 + 4;
    const uint32_t apart = (e1 - e0) * 2;
    // the part's heads, in the order q, k, v
    const uint32_t heads = a.n_heads + 2 * a.n_kv, h0 = part * a.per_part, h1 = min(h0 + a.per_part, heads), k0 = a.n_heads, v0 = a.n_heads + a.n_kv;
    using Batch = uint2[kUnroll][2];
    auto load = [&](Batch &x, const uint8_t *p, uint64_t step, uint32_t n) {
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            if (u < n) {
                x[u][0] = *reinterpret_cast<const uint2 *>(p);
                x[u][1] = *reinterpret_cast<const uint2 *>(p + apart);
            }
            p += step;
        }
    };
    auto store = [&](const Batch &x, uint8_t *p, uint64_t step, uint32_t n) {
#pragma unroll
        for (uint32_t u = 0; u < kUnroll; ++u) {
            if (u < n) {
                *reinterpret_cast<uint2 *>(p) = x[u][0];
                *reinterpret_cast<uint2 *>(p + apart) = x[u][1];
            }
            p += step;
        }
    };
    Batch x, y;
    const uint8_t *src = a.q + row * a.q_token + (uint64_t)h0 * a.q_head + e0 * 2;
    if (h0 < k0) load(x, src, a.q_head, min(h1, k0) - h0);
    const bool there = mine < a.rows && (!a.n_rows || (int64_t)mine < (int64_t)*a.n_rows);
    uint64_t to = 0;
    bool kept = false;
    if (h1 > k0 && a.n_kv) {
        const int64_t slot = a.slots[row];
        kept = there && slot >= 0 && (slot >> a.block_shift) < (int64_t)a.n_blocks;
        if (kept) to = (uint64_t)(slot >> a.block_shift) * a.block_stride + (uint64_t)(slot & ((1 << a.block_shift) - 1)) * a.token_stride + e0 * 2;
    }
    float2 c[2] = {}, s[2] = {}, sn[2] = {};
    if (turned && h0 < v0) {
        float gc[4], gs[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t j = 4 * l + i, axis = a.axes ? min((uint32_t)a.axes[j], a.n_axes - 1) : 0;
            // in turns: what is left of them after the whole ones is exact enough in 32 bits, the product before is not
            const double turns = (double)a.positions[axis * a.positions_stride + row] * (double)a.inv_freq[j] * 0.15915494309189533577;
            sincospif(2.f * (float)(turns - rint(turns)), &gs[i], &gc[i]);
            gc[i] *= a.rope_scale;
            gs[i] *= a.rope_scale;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) c[i] = make_float2(gc[2 * i], gc[2 * i + 1]), s[i] = make_float2(gs[2 * i], gs[2 * i + 1]), sn[i] = make_float2(-s[i].x, -s[i].y);
    }
#pragma unroll 1
    for (uint32_t kind = 0; kind < 2; ++kind) {
        const uint32_t k_first = kind ? max(k0, h0) - k0 : h0, k_end = kind ? min(v0, h1) - k0 : min(k0, h1);  // its heads
        if (kind ? h1 <= k0 || h0 >= v0 : h0 >= k0) continue;
        const uint64_t step = kind ? a.k_head : a.q_head, out_step = kind ? a.head_stride : a.o_head;
        uint8_t *dst = kind ? a.k_base + to + k_first * out_step : a.q_out + row * a.o_token + k_first * out_step + e0 * 2;
        const bool out = kind ? kept : there;
        if (kind) {
            src = a.k + row * a.k_token + k_first * step + e0 * 2;
            load(x, src, step, k_end - k_first);
        }
        const void *weight = kind ? a.k_weight : a.q_weight;
        float2 wa[2], wb[2];
        if (weight) weights_of<HALVES>(a, weight, e0, e1, wa, wb);
        auto turn = [&](Batch &x) {
#pragma unroll
            for (uint32_t u = 0; u < kUnroll; ++u) {
                float2 p[2], q[2];
                pairs_of<HALVES, T>(x[u], p, q);
                if (weight) {
                    float2 sum = ptx::mul2(p[0], p[0]);
                    sum = ptx::fma2(p[1], p[1], sum);
                    sum = ptx::fma2(q[0], q[0], sum);
                    sum = ptx::fma2(q[1], q[1], sum);
                    float all = sum.x + sum.y;
#pragma unroll
                    for (uint32_t o = L / 2; o; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
                    const float r = rsqrtf(all * (1.f / D) + a.eps);
                    const float2 rr = make_float2(r, r);
#pragma unroll
                    for (int i = 0; i < 2; ++i) p[i] = ptx::mul2(p[i], ptx::mul2(wa[i], rr)), q[i] = ptx::mul2(q[i], ptx::mul2(wb[i], rr));
                }
                float2 m[2], n[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    m[i] = ptx::fma2(q[i], sn[i], ptx::mul2(p[i], c[i]));
                    n[i] = ptx::fma2(p[i], s[i], ptx::mul2(q[i], c[i]));
                    // (elsewhere an element has nothing of its neighbour, whatever that holds)
                    p[i] = turned ? m[i] : p[i], q[i] = turned ? n[i] : q[i];
                }
                pack_pairs<HALVES, T>(p, q, x[u]);
            }
        };
        uint32_t left = k_end - k_first;
#pragma unroll 1
        for (;;) {
            const uint64_t far = kUnroll * step, out_far = kUnroll * out_step;
            if (left > kUnroll) load(y, src += far, step, left - kUnroll);
            turn(x);
            if (out) store(x, dst, out_step, left);
            if (left <= kUnroll) break;
            left -= kUnroll;
            dst += out_far;
            if (left > kUnroll) load(x, src += far, step, left - kUnroll);
            turn(y);
            if (out) store(y, dst, out_step, left);
            if (left <= kUnroll) break;
            left -= kUnroll;
            dst += out_far;
        }
    }
    if (h1 > v0 && kept) {
        const uint32_t first = max(v0, h0) - v0;
        const uint8_t *from = a.v + row * a.v_token + first * a.v_head + e0 * 2;
        uint8_t *dst = a.v_base + to + (uint64_t)first * a.head_stride;
#pragma unroll 1
        for (uint32_t left = h1 - v0 - first;;) {
            load(x, from, a.v_head, left);
            if (left > kUnroll) load(y, from + kUnroll * a.v_head, a.v_head, left - kUnroll);
            store(x, dst, a.head_stride, left);
            if (left > kUnroll) store(y, dst + (uint64_t)kUnroll * a.head_stride, a.head_stride, left - kUnroll);
            if (left <= 2 * kUnroll) break;
            left -= 2 * kUnroll;
            from += 2 * kUnroll * a.v_head;
            dst += 2 * kUnroll * (uint64_t)a.head_stride;
        }
    }
}

template <class T>
cudaError_t launch_append(AppendArgs &a, uint32_t dim, cudaStream_t s)
{
    // Four rows of 64 or two of 128 a warp, with all their heads where that fills the GPU twice; with fewer rows they are cut, down to
    // kUnroll heads a warp (6,776 rows of 16 / 4 heads of 128: 23.0 us where they fill it once, 21.5 twice or four times, 26.6 six
    // times, as more warps make the same angles; 52,367 rows of 32 / 8 heads of 64: 106 to 108 us in all of these).
    const uint32_t heads = a.n_heads + 2 * a.n_kv, together = dim == 128 ? 2 : 4;
    const uint64_t fill = 148 * 20 * 2, row_warps = (a.rows + together - 1) / together, batches = (heads + kUnroll - 1) / kUnroll;
    const uint64_t want = (fill + row_warps - 1) / row_warps, cuts = want < batches ? want : batches;
    a.per_part = (uint32_t)((batches + cuts - 1) / cuts) * kUnroll;
    a.parts = (heads + a.per_part - 1) / a.per_part;
    const uint64_t warps = row_warps * a.parts, grid = (warps + kAppendThreads / 32 - 1) / (kAppendThreads / 32);
    if (grid > 0x7fffffffull) return cudaErrorInvalidValue;
    if (a.pairs == GMS_PAIR_HALVES)
        return dim == 128 ? launch_dependent(kv_append_kernel<T, 128, true>, (uint32_t)grid, kAppendThreads, 0, s, a)
                          : launch_dependent(kv_append_kernel<T, 64, true>, (uint32_t)grid, kAppendThreads, 0, s, a);
    return dim == 128 ? launch_dependent(kv_append_kernel<T, 128, false>, (uint32_t)grid, kAppendThreads, 0, s, a)
                      : launch_dependent(kv_append_kernel<T, 64, false>, (uint32_t)grid, kAppendThreads, 0, s, a);
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
    if (t->rows * heads > 1ull << 33) return GMS_ERR_RANGE;
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
