// The gated delta rule on states in the pool: host entry points and the token-by-token kernel.
#include <cmath>

#include "gms_kv_delta.h"

namespace gms {
namespace {

constexpr uint32_t kRowThreads = 256, kRowWarps = kRowThreads / 32, kRowBatch = 8;

// A CTA has W value columns of one head's state in registers, four columns and D W / 1024 rows a thread, and goes through the
// sequence's rows one by one.  Both S^T k and S^T q are taken of the state before the row (S_new^T q = e^g S^T q + (k.q) d), so
// one exchange between the warps is all a row needs.  kRowBatch rows of q, k, v and gates are staged at a time.
template <class T, int D, int W>
__global__ void __launch_bounds__(kRowThreads) kv_delta_rows_kernel(const __grid_constant__ DeltaArgs a)
{
    constexpr int C = W / 4, R = kRowThreads / C, N = D / R;  // threads across, threads down, rows a thread
    constexpr int P = R / (32 / C);                           // partial sums that meet in shared memory (a warp has 32 / C threads down)
    static_assert(C <= 32 && N >= 1 && P == (int)kRowWarps, "");
    __shared__ float qs[kRowBatch][D], ks[kRowBatch][D], vs[kRowBatch][W], gate[kRowBatch], strength[kRowBatch], qk[kRowBatch];
    __shared__ float4 part[2][P][2][C];
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    const uint32_t slice = blockIdx.x % (D / W), h = blockIdx.x / (D / W) % a.n_heads, s = blockIdx.x / (D / W) / a.n_heads, c = h / a.group;
    const uint32_t col = tid % C, down = tid / C;
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    const int first = delta_begin(a, s), rows = delta_rows(a, s);
    if (delta_in_chunks(a, rows)) return;
    const bool fresh = a.past_lens && a.past_lens[s] <= 0;
    const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
    float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
    if (a.status && tid == 0 && ((!fresh && !from) || !to)) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
    const uint32_t at = (down * N) * D + slice * W + col * 4;
    float4 S[N];
#pragma unroll
    for (int i = 0; i < N; ++i) S[i] = from ? *reinterpret_cast<const float4 *>(from + at + i * D) : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r0 = 0; r0 < rows; r0 += kRowBatch) {
        const int n = min(rows - r0, (int)kRowBatch);
        __syncthreads();
        if ((int)warp < n) {  // a warp stages a row
            const uint64_t row = (uint64_t)(first + r0 + (int)warp);
            const T *qp = reinterpret_cast<const T *>(a.q + row * a.q_token + c * a.q_head), *kp = reinterpret_cast<const T *>(a.k + row * a.k_token + c * a.k_head);
            const T *vp = reinterpret_cast<const T *>(a.v + row * a.v_token + h * a.v_head) + slice * W;
            float x[D / 32], y[D / 32], xx = 0.f, yy = 0.f, xy = 0.f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                x[i] = to_f32(qp[lane + 32 * i]), y[i] = to_f32(kp[lane + 32 * i]);
                xx += x[i] * x[i], yy += y[i] * y[i], xy += x[i] * y[i];
            }
            xx = warp_sum(xx), yy = warp_sum(yy), xy = warp_sum(xy);
            const float fx = a.unit_qk ? rsqrtf(xx + a.unit_eps) : 1.f, fy = a.unit_qk ? rsqrtf(yy + a.unit_eps) : 1.f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) qs[warp][lane + 32 * i] = x[i] * fx, ks[warp][lane + 32 * i] = y[i] * fy;
            for (int i = lane; i < W; i += 32) vs[warp][i] = to_f32(vp[i]);
            if (lane == 0) {
                qk[warp] = xy * fx * fy;
                gate[warp] = a.g ? expf(a.g[row * a.g_stride + h]) : 1.f;
                strength[warp] = a.beta ? a.beta[row * a.beta_stride + h] : 1.f;
            }
        }
        __syncthreads();
        for (int r = 0; r < n; ++r) {
            float4 x = {}, y = {};  // S^T k, S^T q
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float kr = ks[r][down * N + i], qr = qs[r][down * N + i];
                x.x += kr * S[i].x, x.y += kr * S[i].y, x.z += kr * S[i].z, x.w += kr * S[i].w;
                y.x += qr * S[i].x, y.y += qr * S[i].y, y.z += qr * S[i].z, y.w += qr * S[i].w;
            }
#pragma unroll
            for (int o = C; o < 32; o <<= 1) {
                x.x += __shfl_xor_sync(0xffffffffu, x.x, o), x.y += __shfl_xor_sync(0xffffffffu, x.y, o);
                x.z += __shfl_xor_sync(0xffffffffu, x.z, o), x.w += __shfl_xor_sync(0xffffffffu, x.w, o);
                y.x += __shfl_xor_sync(0xffffffffu, y.x, o), y.y += __shfl_xor_sync(0xffffffffu, y.y, o);
                y.z += __shfl_xor_sync(0xffffffffu, y.z, o), y.w += __shfl_xor_sync(0xffffffffu, y.w, o);
            }
            if ((int)lane < C) part[r & 1][warp][0][col] = x, part[r & 1][warp][1][col] = y;
            __syncthreads();
            x = y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const float4 u = part[r & 1][p][0][col];
                x.x += u.x, x.y += u.y, x.z += u.z, x.w += u.w;
            }
            const float e = gate[r], b = strength[r];
            const float4 v = *reinterpret_cast<const float4 *>(&vs[r][col * 4]);
            const float4 d = make_float4(b * (v.x - e * x.x), b * (v.y - e * x.y), b * (v.z - e * x.z), b * (v.w - e * x.w));
            if (down == 0) {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float4 u = part[r & 1][p][1][col];
                    y.x += u.x, y.y += u.y, y.z += u.z, y.w += u.w;
                }
                const float z = qk[r];
                T *op = reinterpret_cast<T *>(a.out + (uint64_t)(first + r0 + r) * a.o_token + h * a.o_head) + slice * W + col * 4;
                *reinterpret_cast<uint2 *>(op) = make_uint2(pack2(a.scale * (e * y.x + z * d.x), a.scale * (e * y.y + z * d.y), T()),
                                                            pack2(a.scale * (e * y.z + z * d.z), a.scale * (e * y.w + z * d.w), T()));
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float kr = ks[r][down * N + i];
                S[i].x = e * S[i].x + kr * d.x, S[i].y = e * S[i].y + kr * d.y, S[i].z = e * S[i].z + kr * d.z, S[i].w = e * S[i].w + kr * d.w;
            }
        }
    }
    if (!to) return;
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<float4 *>(to + at + i * D) = S[i];
}

template <class T, int D>
cudaError_t launch_rows(const DeltaArgs &a, cudaStream_t s)
{
    constexpr int W = 32;
    return launch_dependent(kv_delta_rows_kernel<T, D, W>, a.n_seq * a.n_heads * (D / W), kRowThreads, 0, s, a);
}

int make_delta(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *t, DeltaArgs *a)
{
    if (!pool || !state || !t) return GMS_ERR_NULL;
    const int rc = bad_pool(pool);
    if (rc != GMS_OK) return rc;
    if (state->reserved || state->plane >= pool->n_planes || state->n_heads == 0 || state->n_heads > 65536u ||
        (state->head_dim != 64 && state->head_dim != 128))
        return GMS_ERR_ARG;
    const uint32_t bytes = 4 * state->head_dim * state->head_dim;
    if (pool->block_bytes < bytes) return GMS_ERR_ARG;
    if (t->n_key_heads == 0 || state->n_heads % t->n_key_heads || t->dtype > GMS_DTYPE_F16 || t->unit_qk > 1 || !std::isfinite(t->scale))
        return GMS_ERR_ARG;
    if (t->unit_qk && (!std::isfinite(t->unit_eps) || t->unit_eps < 0.f)) return GMS_ERR_ARG;
    if (t->total_q > 0x7fffffffu || t->n_seq > 0x7fffffffu || t->max_q > t->total_q) return GMS_ERR_ARG;
    if (!t->cu_q && (t->total_q != t->n_seq || (t->n_seq && t->max_q != 1))) return GMS_ERR_ARG;
    const uint64_t per_block = pool->block_bytes / bytes, blocks = (state->n_heads + per_block - 1) / per_block;
    if (t->n_seq && t->total_q && (!t->q || !t->k || !t->v || !t->out)) return GMS_ERR_NULL;
    if (t->n_seq && (!t->src_table || !t->dst_table)) return GMS_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(t->q) | reinterpret_cast<uint64_t>(t->k) | reinterpret_cast<uint64_t>(t->v) |
         reinterpret_cast<uint64_t>(t->out) | t->q_token_stride | t->q_head_stride | t->k_token_stride | t->k_head_stride |
         t->v_token_stride | t->v_head_stride | t->out_token_stride | t->out_head_stride) & 15u)
        return GMS_ERR_ALIGN;
    if ((reinterpret_cast<uint64_t>(t->g) | reinterpret_cast<uint64_t>(t->beta) | reinterpret_cast<uint64_t>(t->cu_q) |
         reinterpret_cast<uint64_t>(t->past_lens) | reinterpret_cast<uint64_t>(t->src_table) | reinterpret_cast<uint64_t>(t->dst_table)) & 3u ||
        reinterpret_cast<uint64_t>(t->status) & 7u || reinterpret_cast<uint64_t>(t->workspace) & 255u)
        return GMS_ERR_ALIGN;
    if (t->n_seq && (t->src_stride < blocks || t->dst_stride < blocks || t->src_stride >> 40 || t->dst_stride >> 40)) return GMS_ERR_RANGE;
    if (t->total_q && ((t->g && t->g_stride < state->n_heads) || (t->beta && t->beta_stride < state->n_heads))) return GMS_ERR_RANGE;
    if (((uint64_t)t->n_seq + t->total_q / kChunkRows) * state->n_heads > 1ull << 27) return GMS_ERR_RANGE;
    *a = {};
    a->q = static_cast<const uint8_t *>(t->q);
    a->k = static_cast<const uint8_t *>(t->k);
    a->v = static_cast<const uint8_t *>(t->v);
    a->out = static_cast<uint8_t *>(t->out);
    a->g = t->g;
    a->beta = t->beta;
    a->cu_q = t->cu_q;
    a->past_lens = t->past_lens;
    a->src_table = t->src_table;
    a->dst_table = t->dst_table;
    a->plane = static_cast<uint8_t *>(pool->base) + state->plane * pool->plane_stride;
    a->status = reinterpret_cast<unsigned long long *>(t->status);
    a->q_token = t->q_token_stride;
    a->q_head = t->q_head_stride;
    a->k_token = t->k_token_stride;
    a->k_head = t->k_head_stride;
    a->v_token = t->v_token_stride;
    a->v_head = t->v_head_stride;
    a->o_token = t->out_token_stride;
    a->o_head = t->out_head_stride;
    a->g_stride = t->g_stride;
    a->beta_stride = t->beta_stride;
    a->src_stride = t->src_stride;
    a->dst_stride = t->dst_stride;
    a->block_stride = pool->block_stride;
    a->n_blocks = pool->n_blocks;
    a->per_block = (uint32_t)per_block;
    a->n_seq = t->n_seq;
    a->n_heads = state->n_heads;
    a->group = state->n_heads / t->n_key_heads;
    a->total_q = t->total_q;
    a->max_q = t->max_q;
    a->unit_qk = t->unit_qk;
    a->unit_eps = t->unit_eps;
    a->scale = t->scale;
    return GMS_OK;
}

// Slots for every sequence's chunks, wherever its rows begin; 0: no sequence is long enough.
uint64_t chunk_slots(const DeltaArgs &a) { return a.max_q > kMostByRow ? a.total_q / kChunkRows + a.n_seq : 0; }

}  // namespace
}  // namespace gms

extern "C" {

int gms_kv_delta_workspace(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *args, uint64_t *nbytes)
{
    if (!nbytes) return GMS_ERR_NULL;
    gms::DeltaArgs a;
    const int rc = gms::make_delta(pool, state, args, &a);
    if (rc == GMS_OK) *nbytes = gms::chunk_slots(a) * a.n_heads * sizeof(gms::ChunkWork);
    return rc;
}

int gms_kv_delta(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *args, void *stream)
{
    gms::DeltaArgs a;
    const int rc = gms::make_delta(pool, state, args, &a);
    if (rc != GMS_OK) return rc;
    if (a.n_seq == 0) return GMS_OK;
    const uint64_t slots = gms::chunk_slots(a), need = slots * a.n_heads * sizeof(gms::ChunkWork);
    if (need && !args->workspace) return GMS_ERR_NULL;
    if (need > args->workspace_bytes) return GMS_ERR_RANGE;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = args->dtype == GMS_DTYPE_BF16;
    cudaError_t e = cudaSuccess;
    if (slots) {
        a.chunks = static_cast<uint8_t *>(args->workspace);
        a.n_slots = (uint32_t)slots;
        e = gms::launch_delta_chunks(a, args->dtype, state->head_dim, s);
        if (e != cudaSuccess) return gms::report_cuda_error(e);
    }
    if (state->head_dim == 128)
        e = bf16 ? gms::launch_rows<__nv_bfloat16, 128>(a, s) : gms::launch_rows<__half, 128>(a, s);
    else
        e = bf16 ? gms::launch_rows<__nv_bfloat16, 64>(a, s) : gms::launch_rows<__half, 64>(a, s);
    return e == cudaSuccess ? GMS_OK : gms::report_cuda_error(e);
}

}  // extern "C"
