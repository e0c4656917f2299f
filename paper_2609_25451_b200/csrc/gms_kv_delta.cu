// The gated delta rule on states in the pool: host entry points and the token-by-token kernel.
#include <cmath>

#include "gms_kv_delta.h"

namespace gms {
namespace {

constexpr uint32_t kRowThreads = 256, kRowWarps = kRowThreads / 32;

// W value columns of a head's state in a CTA's registers: four columns and D W / 1024 rows a thread.
template <int D, int W>
struct RowShape {
    static constexpr int C = W / 4, R = kRowThreads / C, N = D / R;  // threads across, threads down, rows a thread
    static_assert(C <= 32 && N % 2 == 0, "");
};
// B rows of q, k, v and gates, and what the warps tell each other.
template <int D, int W, int B>
struct RowSmem {
    float q[B][D], k[B][D], v[B][W], gate[B], strength[B], qk[B];
    float part[kRowWarps][2][W], d[W];
};

__device__ __forceinline__ void get4(float4 x, float2 *to) { to[0] = make_float2(x.x, x.y), to[1] = make_float2(x.z, x.w); }

// A row as a warp reads it, and puts it into shared memory.
template <class T, int D, int W>
struct Row1 {
    T q[D / 32], k[D / 32], v[(W + 31) / 32];
    float g, b;
};
template <class T, int D, int W>
__device__ __forceinline__ void read_row(const DeltaArgs &a, uint64_t row, uint32_t h, uint32_t slice, Row1<T, D, W> &x)
{
    const uint32_t lane = threadIdx.x & 31u, c = h / a.group;
    const T *qp = reinterpret_cast<const T *>(a.q + row * a.q_token + c * a.q_head), *kp = reinterpret_cast<const T *>(a.k + row * a.k_token + c * a.k_head);
    const T *vp = reinterpret_cast<const T *>(a.v + row * a.v_token + h * a.v_head) + slice * W;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) x.q[i] = qp[lane + 32 * i], x.k[i] = kp[lane + 32 * i];
#pragma unroll
    for (int i = 0; i < W / 32; ++i) x.v[i] = vp[lane + 32 * i];
    x.g = a.g ? a.g[row * a.g_stride + h] : 0.f;
    x.b = a.beta ? a.beta[row * a.beta_stride + h] : 1.f;
}
template <class T, int D, int W, int B>
__device__ __forceinline__ void put_row(const DeltaArgs &a, const Row1<T, D, W> &x, uint32_t to, RowSmem<D, W, B> &m)
{
    const uint32_t lane = threadIdx.x & 31u;
    float q[D / 32], k[D / 32], qq = 0.f, kk = 0.f, qk = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        q[i] = to_f32(x.q[i]), k[i] = to_f32(x.k[i]);
        qq += q[i] * q[i], kk += k[i] * k[i], qk += q[i] * k[i];
    }
    qq = warp_sum(qq), kk = warp_sum(kk), qk = warp_sum(qk);
    const float fq = a.unit_qk ? rsqrtf(qq + a.unit_eps) : 1.f, fk = a.unit_qk ? rsqrtf(kk + a.unit_eps) : 1.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) m.q[to][lane + 32 * i] = q[i] * fq, m.k[to][lane + 32 * i] = k[i] * fk;
#pragma unroll
    for (int i = 0; i < W / 32; ++i) m.v[to][lane + 32 * i] = to_f32(x.v[i]);
    if (lane == 0) m.qk[to] = qk * fq * fk, m.gate[to] = expf(x.g), m.strength[to] = x.b;
}

// Takes the state over n rows that are in shared memory (the first is row `first` of the call).  Both S^T k and S^T q are taken of the
// state before the row (S_new^T q = e^g S^T q + (k.q) d): the warps' parts of the two go through shared memory, each warp sums some
// columns of them and tells the others d.
template <class T, int D, int W, int B>
__device__ __forceinline__ void take_rows(const DeltaArgs &a, RowSmem<D, W, B> &m, int n, uint64_t first, uint32_t h, uint32_t slice,
                                          float2 (&S)[RowShape<D, W>::N][2])
{
    constexpr int C = RowShape<D, W>::C, N = RowShape<D, W>::N;
    constexpr uint32_t kMine = W / kRowWarps;  // columns that a warp sums
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32, col = threadIdx.x % C, down = threadIdx.x / C;
    for (int r = 0; r < n; ++r) {
        float k[N];
        float2 x0 = {}, x1 = {}, y0 = {}, y1 = {};
        auto twice = [](float f) { return make_float2(f, f); };
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const float2 kk = *reinterpret_cast<const float2 *>(&m.k[r][down * N + i]), qq = *reinterpret_cast<const float2 *>(&m.q[r][down * N + i]);
            k[i] = kk.x, k[i + 1] = kk.y;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float q = j ? qq.y : qq.x;
                x0 = ptx::fma2(twice(k[i + j]), S[i + j][0], x0), x1 = ptx::fma2(twice(k[i + j]), S[i + j][1], x1);
                y0 = ptx::fma2(twice(q), S[i + j][0], y0), y1 = ptx::fma2(twice(q), S[i + j][1], y1);
            }
        }
        float4 x = make_float4(x0.x, x0.y, x1.x, x1.y), y = make_float4(y0.x, y0.y, y1.x, y1.y);  // S^T k, S^T q
#pragma unroll
        for (int o = C; o < 32; o <<= 1) {
            x.x += __shfl_xor_sync(0xffffffffu, x.x, o), x.y += __shfl_xor_sync(0xffffffffu, x.y, o);
            x.z += __shfl_xor_sync(0xffffffffu, x.z, o), x.w += __shfl_xor_sync(0xffffffffu, x.w, o);
            y.x += __shfl_xor_sync(0xffffffffu, y.x, o), y.y += __shfl_xor_sync(0xffffffffu, y.y, o);
            y.z += __shfl_xor_sync(0xffffffffu, y.z, o), y.w += __shfl_xor_sync(0xffffffffu, y.w, o);
        }
        if ((int)lane < C) *reinterpret_cast<float4 *>(&m.part[warp][0][col * 4]) = x, *reinterpret_cast<float4 *>(&m.part[warp][1][col * 4]) = y;
        asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
        const float e = m.gate[r];
        {
            const uint32_t is_y = lane / kMine & 1u, c = warp * kMine + lane % kMine;  // (lanes beyond 2 kMine do the same again)
            float sum = 0.f;
#pragma unroll
            for (int p = 0; p < (int)kRowWarps; ++p) sum += m.part[p][is_y][c];
            const float d = m.strength[r] * (m.v[r][c] - e * sum), dd = __shfl_sync(0xffffffffu, d, lane % kMine);
            if (lane < kMine) m.d[c] = d;
            else if (lane < 2 * kMine)
                reinterpret_cast<T *>(a.out + (first + r) * a.o_token + h * a.o_head)[slice * W + c] = from_f32<T>(a.scale * (e * sum + m.qk[r] * dd));
        }
        asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
        const float4 d = *reinterpret_cast<const float4 *>(&m.d[col * 4]);
        const float2 d0 = make_float2(d.x, d.y), d1 = make_float2(d.z, d.w);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            S[i][0] = ptx::fma2(twice(k[i]), d0, ptx::mul2(twice(e), S[i][0]));
            S[i][1] = ptx::fma2(twice(k[i]), d1, ptx::mul2(twice(e), S[i][1]));
        }
    }
}

// Few states: W value columns of one a CTA.  Bound by latency.
template <class T, int D, int W>
__global__ void __launch_bounds__(kRowThreads) kv_delta_rows_kernel(const __grid_constant__ DeltaArgs a)
{
    constexpr int C = RowShape<D, W>::C, N = RowShape<D, W>::N;
    constexpr uint32_t B = kRowWarps;
    __shared__ RowSmem<D, W, B> m;
    const uint32_t tid = threadIdx.x, warp = tid / 32;
    const uint32_t slice = blockIdx.x % (D / W), h = blockIdx.x / (D / W) % a.n_heads, s = blockIdx.x / (D / W) / a.n_heads;
    // Beside the chunk kernels, which have waited for what was before them and have nothing to do with these sequences: what they leave
    // of the GPU is filled up.  The last CTA ends by waiting for them, so that nothing after this kernel starts before they have ended.
    if (!a.chunks) ptx::grid_wait();
    ptx::grid_launch_dependents();
    auto leave = [&] {
        if (a.chunks && blockIdx.x == gridDim.x - 1 && tid == 0) ptx::grid_wait();
    };
    const int first = delta_begin(a, s), rows = delta_rows(a, s);
    if (delta_in_chunks(a, rows)) return leave();
    const bool fresh = a.past_lens && a.past_lens[s] <= 0;
    const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
    float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
    if (a.status && tid == 0 && ((!fresh && !from) || !to)) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
    const uint32_t at = (tid / C * N) * D + slice * W + tid % C * 4;
    float2 S[N][2];
#pragma unroll
    for (int i = 0; i < N; ++i) get4(from ? *reinterpret_cast<const float4 *>(from + at + i * D) : make_float4(0.f, 0.f, 0.f, 0.f), S[i]);
    for (int r0 = 0; r0 < rows; r0 += B) {
        const int n = min(rows - r0, (int)B);
        __syncthreads();
        if ((int)warp < n) {  // a warp stages a row
            Row1<T, D, W> x;
            read_row<T, D, W>(a, (uint64_t)(first + r0 + (int)warp), h, slice, x);
            put_row<T, D, W>(a, x, warp, m);
        }
        __syncthreads();
        take_rows<T, D, W>(a, m, n, (uint64_t)(first + r0), h, slice, S);
    }
    if (!to) return leave();
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<float4 *>(to + at + i * D) = make_float4(S[i][0].x, S[i][0].y, S[i][1].x, S[i][1].y);
    leave();
}

template <int D>
struct StreamShape {
    static constexpr int kBuffers = D == 128 ? 3 : 4, kCtas = D == 128 ? 1 : 2, kRows = 8;  // rows at a time
};
template <int D>
struct StreamSmem {
    float state[StreamShape<D>::kBuffers][D * D];
    RowSmem<D, D, StreamShape<D>::kRows> rows;
    uint64_t full[StreamShape<D>::kBuffers], done[StreamShape<D>::kBuffers];
};
constexpr uint32_t kStreamThreads = kRowThreads + 32;

// Many states: whole ones through a ring of buffers, brought and taken away by bulk copies that one thread issues, two on their way while
// one is worked on, by CTAs that stay.  Bound by memory: 3.4 us a state of 64 KiB and SM, read and written, which is 5.6 TB/s on all
// of them, and 6 us to get going.  (64 sequences of 32 heads: 55 us, the kernel above with 32 or 128 columns a CTA 70 or 67.)
template <class T, int D>
__global__ void __launch_bounds__(kStreamThreads, StreamShape<D>::kCtas) kv_delta_stream_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(128) uint8_t raw[];
    StreamSmem<D> &m = *reinterpret_cast<StreamSmem<D> *>(raw);
    constexpr int C = RowShape<D, D>::C, N = RowShape<D, D>::N, NB = StreamShape<D>::kBuffers, B = StreamShape<D>::kRows;
    const uint32_t tid = threadIdx.x, warp = tid / 32, items = a.n_seq * a.n_heads;
    if (tid == 0) {
        for (int i = 0; i < NB; ++i) {
            ptx::mbar_init(ptx::smem_u32(&m.full[i]), 1);
            ptx::mbar_init(ptx::smem_u32(&m.done[i]), kRowWarps);
        }
        ptx::fence_mbar_init();
    }
    __syncthreads();
    if (!a.chunks) ptx::grid_wait();  // (as above)
    ptx::grid_launch_dependents();
    // A wait that runs out (it cannot, but for a fault in here) is told in the status word; everybody goes on without waiting.
    bool late = false;
    auto wait = [&](uint64_t *bar, uint32_t use) {
        if (late || ptx::mbar_wait(ptx::smem_u32(bar), use & 1u)) return;
        late = true;
        if (a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_TIMEOUT);
    };
    if (warp == kRowWarps) {
        if ((tid & 31u) != 0) return;
        auto rows_of = [&](uint32_t item) { return delta_rows(a, item / a.n_heads); };
        auto load = [&](uint32_t item, uint32_t k) {
            const uint32_t s = item / a.n_heads, h = item % a.n_heads, b = k % NB, bar = ptx::smem_u32(&m.full[b]);
            const bool fresh = a.past_lens && a.past_lens[s] <= 0;
            const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
            if (!from) {
                if (!fresh && a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
                ptx::mbar_arrive(bar);
                return;
            }
            ptx::mbar_expect(bar, D * D * 4);
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ptx::smem_u32(m.state[b])),
                         "l"(from), "r"(D * D * 4), "r"(bar)
                         : "memory");
        };
        auto store = [&](uint32_t item, uint32_t k) {
            const uint32_t s = item / a.n_heads, h = item % a.n_heads;
            float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
            if (to)
                asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(ptx::smem_u32(m.state[k % NB])), "r"(D * D * 4)
                             : "memory");
            else if (a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        };
        auto next = [&](uint32_t item) {  // of this CTA's items, those that are done here
            while (item < items && delta_in_chunks(a, rows_of(item))) item += gridDim.x;
            return item;
        };
        uint32_t ahead = next(blockIdx.x), k_ahead = 0;
        for (; k_ahead < NB - 1 && ahead < items; ++k_ahead, ahead = next(ahead + gridDim.x)) load(ahead, k_ahead);
        uint32_t k = 0;
        for (uint32_t item = next(blockIdx.x); item < items; item = next(item + gridDim.x), ++k) {
            wait(&m.done[k % NB], k / NB);
            store(item, k);
            if (ahead < items) {  // into the buffer of the state before, once that has been read
                asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                load(ahead, k_ahead);
                ++k_ahead, ahead = next(ahead + gridDim.x);
            }
        }
        if (late) {  // copies that may still be under way
            late = false;
            for (uint32_t i = k_ahead > NB ? k_ahead - NB : 0; i < k_ahead; ++i) wait(&m.full[i % NB], i / NB);
        }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        return;
    }
    // rows are read one state ahead
    Row1<T, D, D> row;
    auto first_rows = [&](uint32_t item) {
        while (item < items) {
            const int rows = delta_rows(a, item / a.n_heads);
            if (!delta_in_chunks(a, rows)) {
                if ((int)warp < min(rows, B)) read_row<T, D, D>(a, (uint64_t)(delta_begin(a, item / a.n_heads) + (int)warp), item % a.n_heads, 0, row);
                break;
            }
            item += gridDim.x;
        }
        return item;
    };
    uint32_t k = 0;
    for (uint32_t item = first_rows(blockIdx.x), next; item < items; item = next, ++k) {
        const uint32_t s = item / a.n_heads, h = item % a.n_heads, b = k % NB;
        const int first = delta_begin(a, s), rows = delta_rows(a, s);
        const bool zero = (a.past_lens && a.past_lens[s] <= 0) || !delta_state<D>(a, a.src_table, a.src_stride, s, h);
        if ((int)warp < min(rows, B)) put_row<T, D, D>(a, row, warp, m.rows);
        next = first_rows(item + gridDim.x);
        wait(&m.full[b], k / NB);
        float *state = m.state[b] + (tid / C * N) * D + tid % C * 4;
        float2 S[N][2];
#pragma unroll
        for (int i = 0; i < N; ++i) get4(zero ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4 *>(state + i * D), S[i]);
        asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
        take_rows<T, D, D>(a, m.rows, min(rows, B), (uint64_t)first, h, 0, S);
        for (int r0 = B; r0 < rows; r0 += B) {
            const int n = min(rows - r0, B);
            asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
            if ((int)warp < n) {
                Row1<T, D, D> x;
                read_row<T, D, D>(a, (uint64_t)(first + r0 + (int)warp), h, 0, x);
                put_row<T, D, D>(a, x, warp, m.rows);
            }
            asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
            take_rows<T, D, D>(a, m.rows, n, (uint64_t)(first + r0), h, 0, S);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) *reinterpret_cast<float4 *>(state + i * D) = make_float4(S[i][0].x, S[i][0].y, S[i][1].x, S[i][1].y);
        ptx::fence_proxy_async();
        asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");  // (the rows have been read, too)
        if ((tid & 31u) == 0) ptx::mbar_arrive(ptx::smem_u32(&m.done[b]));
    }
    if (a.chunks && blockIdx.x == gridDim.x - 1 && tid == 0) ptx::grid_wait();
}

template <class T, int D>
cudaError_t launch_rows(const DeltaArgs &a, cudaStream_t s)
{
    // Whole states pay from one and a half a CTA on: below that SMs stand idle or have two rounds to do (32 heads of 128, one row, us,
    // slices / whole states: 5 sequences 12.3 / 14.3, 8 14.3 / 14.3, 24 28.7 / 26.6; four rows: 5 16.4 / 16.4, 8 20.5 / 18.4, 24 43 / 35).
    // Beside the chunk kernels small CTAs fill up better, up to eight times as many states (the whole call, a long prompt and single
    // rows: 32 sequences 340 / 336, 64 233 / 235; 44 sequences of 9 to 51 rows, 24 heads 137 / 147).
    constexpr int W = 32;
    const uint64_t items = (uint64_t)a.n_seq * a.n_heads, held = 148 * StreamShape<D>::kCtas;
    if (2 * items <= (a.chunks ? 16 : 3) * held) return launch_dependent(kv_delta_rows_kernel<T, D, W>, (uint32_t)items * (D / W), kRowThreads, 0, s, a);
    static std::atomic<uint64_t> done;
    static_assert(sizeof(StreamSmem<D>) * StreamShape<D>::kCtas <= 231424, "");
    const cudaError_t e = allow_smem(kv_delta_stream_kernel<T, D>, sizeof(StreamSmem<D>), done);
    if (e != cudaSuccess) return e;
    return launch_dependent(kv_delta_stream_kernel<T, D>, (uint32_t)held, kStreamThreads, sizeof(StreamSmem<D>), s, a);
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

// Slots for every sequence's chunks, wherever its rows begin; 0: no sequence is long enough.  The smaller one of two numbers, each of
// which grows with the call: 255 single rows beside a prompt of 2,048, 32 heads, take 79 MB so, with a slot for each of them 210.
uint64_t chunk_slots(DeltaArgs &a)
{
    if (a.max_q <= kMostByRow) return 0;
    const uint64_t each = (uint64_t)a.total_q / kChunkRows + a.n_seq, by_begin = a.total_q / (kMostByRow + 1) + 1;
    a.by_begin = by_begin < each;
    return by_begin < each ? by_begin : each;
}
// They and the order of the sequences.
uint64_t work_bytes(DeltaArgs &a)
{
    const uint64_t slots = chunk_slots(a);
    return slots ? slots * a.n_heads * sizeof(ChunkWork) + ((uint64_t)a.n_seq * 4 + 255) / 256 * 256 : 0;
}

}  // namespace
}  // namespace gms

extern "C" {

int gms_kv_delta_workspace(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *args, uint64_t *nbytes)
{
    if (!nbytes) return GMS_ERR_NULL;
    gms::DeltaArgs a;
    const int rc = gms::make_delta(pool, state, args, &a);
    if (rc == GMS_OK) *nbytes = gms::work_bytes(a);
    return rc;
}

int gms_kv_delta(const gms_kv_pool *pool, const gms_kv_state *state, const gms_kv_delta_args *args, void *stream)
{
    gms::DeltaArgs a;
    const int rc = gms::make_delta(pool, state, args, &a);
    if (rc != GMS_OK) return rc;
    if (a.n_seq == 0) return GMS_OK;
    const uint64_t slots = gms::chunk_slots(a), need = gms::work_bytes(a);
    if (need && !args->workspace) return GMS_ERR_NULL;
    if (need > args->workspace_bytes) return GMS_ERR_RANGE;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool bf16 = args->dtype == GMS_DTYPE_BF16;
    cudaError_t e = cudaSuccess;
    if (slots) {
        a.chunks = static_cast<uint8_t *>(args->workspace);
        a.n_slots = (uint32_t)slots;
        a.order = reinterpret_cast<uint32_t *>(a.chunks + slots * a.n_heads * sizeof(gms::ChunkWork));
        e = gms::launch_delta_prep(a, args->dtype, state->head_dim, s);
        if (e == cudaSuccess) e = gms::launch_delta_chain(a, args->dtype, state->head_dim, s);
        if (e != cudaSuccess) return gms::report_cuda_error(e);
    }
    if (state->head_dim == 128)
        e = bf16 ? gms::launch_rows<__nv_bfloat16, 128>(a, s) : gms::launch_rows<__half, 128>(a, s);
    else
        e = bf16 ? gms::launch_rows<__nv_bfloat16, 64>(a, s) : gms::launch_rows<__half, 64>(a, s);
    return e == cudaSuccess ? GMS_OK : gms::report_cuda_error(e);
}

}  // extern "C"
