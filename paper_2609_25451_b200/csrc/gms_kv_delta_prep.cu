// The gated delta rule, 64 rows at a time: what a chunk's rows do to one another, then the chain of the states.
//
// With G the sum of the log gates from the chunk's first row on, r the keys' factors to unit length and S0 the state before the
// chunk (all of it row by row the same as the rule):
//   d = T (V - diag(f) K S0),            T = (I + A)^-1 diag(beta),  A_ij = beta_i r_i r_j (k_i.k_j) e^(G_i - G_j) for j < i, f = r e^G
//   out = diag(h) Q S0 + P d,            P_ij = scale s_i r_j (q_i.k_j) e^(G_i - G_j) for j <= i,  h = scale s e^G
//   S1 = e^G_last S0 + K^T diag(w) d,    w = r e^(G_last - G)
// T, P, f, h and w do not depend on the state: the first kernel makes them for all chunks at once.  The second goes through each
// sequence's chunks.  q, k and v enter the products as they are; differences of G are taken in 64 bits.
#include "gms_kv_delta.h"

namespace gms {
namespace {

constexpr float kMostNegative = -200.f;  // a gate of e^-200 is 0 in 32 bits, as is every product with it

using ptx::ldmatrix_x4;
using ptx::smem_u32;

// Which sequence and which of its chunks slot `id` stands for; false: none.
__device__ __forceinline__ bool find_chunk(const DeltaArgs &a, uint32_t id, uint32_t &s, uint32_t &chunk)
{
    uint32_t lo = 0, hi = a.n_seq;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (delta_slot(a, mid) <= id) lo = mid; else hi = mid;
    }
    s = lo;
    const uint32_t first = delta_slot(a, s);
    chunk = id - first;
    return id >= first;
}

constexpr uint32_t kPrepThreads = 128, kPrepHeads = 4, kRowPad = kChunkRows + 4;

template <int D>
struct PrepSmem {
    union {
        struct {
            uint8_t k[kChunkRows * D * 2], q[kChunkRows * D * 2];
        };
        struct {
            float a[kChunkRows][kRowPad], t[kChunkRows][kRowPad];  // A and the inverse of I + A, below their diagonals' 16 x 16 blocks
            uint8_t p[sizeof(ChunkWork::tile[0])];
        };
    };
    double sum[kPrepHeads][kChunkRows];  // G / ln 2
    float b[kPrepHeads][kChunkRows];
    float rk[kChunkRows], rq[kChunkRows];
    float top[2][4];
};

// Factors of products of two 32-bit matrices in shared memory, as two bf16 terms each: rows r0 + g (+ 8), columns c0 + t2 + {0, 1, 8, 9}
// of the first factor; rows k0 + t2 + {0, 1, 8, 9}, column n0 + g of the second.
struct Terms {
    uint32_t hi[4], lo[4];
};
__device__ __forceinline__ Terms first_factor(const float (*x)[kRowPad], uint32_t r, uint32_t c)
{
    Terms f;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) {
        const float2 v = *reinterpret_cast<const float2 *>(&x[r + (e & 1) * 8][c + (e & 2) * 4]);
        split2<__nv_bfloat16>(v.x, v.y, f.hi[e], f.lo[e]);
    }
    return f;
}
__device__ __forceinline__ void second_factor(const float (*x)[kRowPad], uint32_t k, uint32_t n, uint32_t *hi, uint32_t *lo)
{
#pragma unroll
    for (uint32_t e = 0; e < 2; ++e) split2<__nv_bfloat16>(x[k + 8 * e][n], x[k + 8 * e + 1][n], hi[e], lo[e]);
}
__device__ __forceinline__ void mma_terms(float *c, const Terms &f, const uint32_t *hi, const uint32_t *lo)
{
    mma16816(c, f.hi, hi[0], hi[1], __nv_bfloat16());
    mma16816(c, f.lo, hi[0], hi[1], __nv_bfloat16());
    mma16816(c, f.hi, lo[0], lo[1], __nv_bfloat16());
}
// -(X Y) Z with X 16 x 16 K, Y 16 K x 8 N, Z 8 N x 8 M; the first `used` of X's K tiles are not zero, nor are Z's rows from 16 `from` on.
// X Y stays in registers: an accumulator is, element for element, a first factor.
template <int K, int N, int M>
__device__ __forceinline__ void two_products(const float (*x)[kRowPad], uint32_t x_row, uint32_t x_col, const float (*y)[kRowPad], uint32_t y_row,
                                             uint32_t y_col, const float (*z)[kRowPad], uint32_t z_row, uint32_t z_col, uint32_t used, uint32_t from,
                                             float (*out)[4])
{
    const uint32_t lane = threadIdx.x & 31u, g = lane / 4, t2 = 2 * (lane & 3u);
    float mid[N][4] = {};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (k >= (int)used) break;
        const Terms f = first_factor(x, x_row + g, x_col + 16 * k + t2);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            uint32_t hi[2], lo[2];
            second_factor(y, y_row + 16 * k + t2, y_col + 8 * n + g, hi, lo);
            mma_terms(mid[n], f, hi, lo);
        }
    }
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        if (k < (int)from) continue;
        Terms f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            split2<__nv_bfloat16>(-mid[2 * k + e / 2][2 * (e & 1)], -mid[2 * k + e / 2][2 * (e & 1) + 1], f.hi[e], f.lo[e]);
#pragma unroll
        for (int n = 0; n < M; ++n) {
            uint32_t hi[2], lo[2];
            second_factor(z, z_row + 16 * k + t2, z_col + 8 * n + g, hi, lo);
            mma_terms(out[n], f, hi, lo);
        }
    }
}
__device__ __forceinline__ void put_tile(float (*t)[kRowPad], uint32_t r, uint32_t c, const float *x)
{
    const uint32_t lane = threadIdx.x & 31u, g = lane / 4, t2 = 2 * (lane & 3u);
    *reinterpret_cast<float2 *>(&t[r + g][c + t2]) = make_float2(x[0], x[1]);
    *reinterpret_cast<float2 *>(&t[r + g + 8][c + t2]) = make_float2(x[2], x[3]);
}

// One CTA per chunk and key head.  k_i.k_j and q_i.k_j on mma.sync (a warp has 16 rows i), then for each value head of the key
// head the decays, the inverse and what goes to the workspace.  The inverse of I + A: its diagonal blocks of 16 x 16 a warp each
// (a lane has a column and goes down it: x_i = -sum_(j<i) A_ij x_j), then, for blocks of 16 and of 32,
//   (X 0; Y Z)^-1 = (X^-1 0; -Z^-1 Y X^-1 Z^-1)
// in products of two-term factors (2^-16 relative, as T itself is handed on).
template <class T, int D>
__global__ void __launch_bounds__(kPrepThreads, 4) kv_delta_prep_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    PrepSmem<D> &m = *reinterpret_cast<PrepSmem<D> *>(raw);
    constexpr int C = kChunkRows, P = D / 8;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32, g = lane / 4, t2 = 2 * (lane & 3u);
    const uint32_t n_key = a.n_heads / a.group, kh = blockIdx.x % n_key, id = blockIdx.x / n_key;
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    uint32_t s, chunk;
    if (!find_chunk(a, id, s, chunk)) return;
    const int all_rows = delta_rows(a, s);
    if (!delta_in_chunks(a, all_rows) || chunk > (uint32_t)(all_rows - 1) / C) return;
    const int n = min(all_rows - (int)chunk * C, C), first = delta_begin(a, s) + (int)chunk * C;
#pragma unroll 4
    for (uint32_t i = tid; i < (uint32_t)(C * P); i += kPrepThreads) {
        const uint32_t r = i / P, c = i % P;
        const bool real = (int)r < n;
        const uint64_t row = (uint64_t)(first + (real ? (int)r : 0));
        cp16(smem_u32(m.k) + piece<P>(r, c), a.k + row * a.k_token + kh * a.k_head + c * 16, real);
        cp16(smem_u32(m.q) + piece<P>(r, c), a.q + row * a.q_token + kh * a.q_head + c * 16, real);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    // lengths: two threads a row
    uint32_t bad = 0;
    {
        const uint32_t r = tid / 2;
        float kk = 0.f, qq = 0.f;
#pragma unroll
        for (uint32_t c = 0; c < (uint32_t)P; c += 2) {
            const uint32_t at = piece<P>(r, c + (tid & 1u));
            const uint4 kv = *reinterpret_cast<const uint4 *>(m.k + at), qv = *reinterpret_cast<const uint4 *>(m.q + at);
            const T *ke = reinterpret_cast<const T *>(&kv), *qe = reinterpret_cast<const T *>(&qv);
#pragma unroll
            for (int e = 0; e < 8; ++e) kk += to_f32(ke[e]) * to_f32(ke[e]), qq += to_f32(qe[e]) * to_f32(qe[e]);
        }
        kk += __shfl_xor_sync(0xffffffffu, kk, 1);
        qq += __shfl_xor_sync(0xffffffffu, qq, 1);
        if (!(kk < kHuge) || !(qq < kHuge)) bad = 1;
        if ((tid & 1u) == 0) {
            m.rk[r] = a.unit_qk && (int)r < n ? rsqrtf(kk + a.unit_eps) : 1.f;
            m.rq[r] = a.unit_qk && (int)r < n ? rsqrtf(qq + a.unit_eps) : 1.f;
        }
    }
    // products of rows 16 warp .. with rows 0 .. of the keys
    float kk[C / 8][4] = {}, qk[C / 8][4] = {};
#pragma unroll
    for (int kt = 0; kt < D / 16; ++kt) {
        uint32_t ka[4], qa[4];
        const uint32_t at = piece<P>(16 * warp + (lane & 15u), 2 * kt + lane / 16);
        ldmatrix_x4(smem_u32(m.k) + at, ka);
        ldmatrix_x4(smem_u32(m.q) + at, qa);
#pragma unroll
        for (int nt = 0; nt < C / 8; nt += 2) {
            if (nt > 2 * (int)warp) break;
            uint32_t b[4];
            ldmatrix_x4(smem_u32(m.k) + piece<P>(8 * nt + (lane & 7u) + (lane & 16u) / 2, 2 * kt + (lane / 8 & 1u)), b);
            mma16816(kk[nt], ka, b[0], b[1], T());
            mma16816(kk[nt + 1], ka, b[2], b[3], T());
            mma16816(qk[nt], qa, b[0], b[1], T());
            mma16816(qk[nt + 1], qa, b[2], b[3], T());
        }
    }
    for (uint32_t j = 0; j < a.group; ++j) {
        ChunkWork *work = reinterpret_cast<ChunkWork *>(a.chunks + ((uint64_t)id * a.n_heads + kh * a.group + j) * sizeof(ChunkWork));
        const uint32_t jj = j % kPrepHeads;
        __syncthreads();  // the keys and queries, or the last head's matrices, have been read
        if (jj == 0 && j + warp < a.group) {  // gates of four heads, a warp each: two rows a lane, sums in 64 bits
            const uint32_t h = kh * a.group + j + warp;
            ChunkWork &w = work[warp];
            double x[2], sum_g = 0.;
            float beta[2], raw_g[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 2 * (int)lane + e;
                const uint64_t row = (uint64_t)(first + r);
                raw_g[e] = r < n && a.g ? a.g[row * a.g_stride + h] : 0.f;
                beta[e] = r < n ? a.beta ? a.beta[row * a.beta_stride + h] : 1.f : 0.f;
                if (!(raw_g[e] < kHuge) || !(fabsf(beta[e]) < kHuge)) bad = 1;
                sum_g += 1.4426950408889634 * (double)(raw_g[e] < kMostNegative ? kMostNegative : raw_g[e]);
                x[e] = sum_g;
            }
            double inc = sum_g;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= (uint32_t)o) inc += y;
            }
            const double last = __shfl_sync(0xffffffffu, inc, 31);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 2 * (int)lane + e;
                const double sum = inc - sum_g + x[e];
                const bool in = r < n;
                m.sum[warp][r] = sum;
                m.b[warp][r] = beta[e];
                const float gate = exp2f((float)sum), f = in ? m.rk[r] * gate : 0.f, hh = in ? a.scale * m.rq[r] * gate : 0.f,
                            ww = in ? m.rk[r] * exp2f((float)(last - sum)) : 0.f;
                w.f[r] = f, w.h[r] = hh, w.w[r] = ww;
                w.gate[r] = expf(raw_g[e]), w.beta[r] = beta[e], w.rk[r] = m.rk[r], w.rq[r] = m.rq[r];
                if (!(fabsf(f) < kHuge) || !(fabsf(hh) < kHuge) || !(fabsf(ww) < kHuge)) bad = 1;
            }
            const float all = exp2f((float)last);
            if (!(all < kHuge)) bad = 1;
            if (lane == 0) w.all = all;
        }
        __syncthreads();
        // A and P: rows i = 16 warp + g (+ 8), columns 8 nt + t2 + {0, 1}
        float pv[C / 8][4], top = 0.f;
        {
            const uint32_t i0 = 16 * warp + g;
            const double sum[2] = {m.sum[jj][i0], m.sum[jj][i0 + 8]};
            const float bk[2] = {m.b[jj][i0] * m.rk[i0], m.b[jj][i0 + 8] * m.rk[i0 + 8]};
            const float sq[2] = {(int)i0 < n ? a.scale * m.rq[i0] : 0.f, (int)i0 + 8 < n ? a.scale * m.rq[i0 + 8] : 0.f};
#pragma unroll
            for (int nt = 0; nt < C / 8; ++nt) {
                pv[nt][0] = pv[nt][1] = pv[nt][2] = pv[nt][3] = 0.f;
                if (nt > 2 * (int)warp + 1) continue;
                const uint32_t c0 = 8 * nt + t2;
                float av[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t i = i0 + (e & 2) * 4, c = c0 + (e & 1);
                    const float z = m.rk[c] * (c <= i ? ptx::ex2((float)(sum[e / 2] - m.sum[jj][c])) : 0.f);
                    av[e] = c < i ? bk[e / 2] * (kk[nt][e] * z) : 0.f;
                    pv[nt][e] = c <= i ? sq[e / 2] * (qk[nt][e] * z) : 0.f;
                    if (!(fabsf(av[e]) < kHuge) || !(fabsf(pv[nt][e]) < kHuge)) bad = 1;
                    top = fmaxf(top, fabsf(pv[nt][e]));
                }
                put_tile(m.a, 16 * warp, 8 * nt, av);
            }
        }
        float ps = 1.f;
        if (kHalf) {
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (lane == 0) m.top[0][warp] = top;
            __syncthreads();
            ps = range_scale(fmaxf(fmaxf(m.top[0][0], m.top[0][1]), fmaxf(m.top[0][2], m.top[0][3])));
            if (tid == 0) work->p_unit = flipped(ps);
        }
#pragma unroll
        for (int nt = 0; nt < C / 8; ++nt) {
            if (nt > 2 * (int)warp + 1) break;
            const uint32_t i = 16 * warp + g;
            *reinterpret_cast<uint32_t *>(m.p + block_piece(i, nt) + 2 * t2) = pack2(pv[nt][0] * ps, pv[nt][1] * ps, T());
            *reinterpret_cast<uint32_t *>(m.p + block_piece(i + 8, nt) + 2 * t2) = pack2(pv[nt][2] * ps, pv[nt][3] * ps, T());
        }
        __syncwarp();
        if (lane < 16) {  // the warp's own diagonal block
            const uint32_t d0 = 16 * warp;
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float sum = i == (int)lane ? 1.f : 0.f;
#pragma unroll
                for (int c = 0; c < i; c += 4) {
                    const float4 r = *reinterpret_cast<const float4 *>(&m.a[d0 + i][d0 + c]);
                    sum -= r.x * x[c];
                    if (c + 1 < i) sum -= r.y * x[c + 1];
                    if (c + 2 < i) sum -= r.z * x[c + 2];
                    if (c + 3 < i) sum -= r.w * x[c + 3];
                }
                x[i] = sum;
                m.t[d0 + i][d0 + lane] = sum;
            }
        }
        __syncthreads();
        if ((warp & 1u) == 0) {
            float o[2][4] = {};
            const uint32_t d0 = 16 * warp;
            two_products<1, 2, 2>(m.t, d0 + 16, d0 + 16, m.a, d0 + 16, d0, m.t, d0, d0, 1, 0, o);
            put_tile(m.t, d0 + 16, d0, o[0]);
            put_tile(m.t, d0 + 16, d0 + 8, o[1]);
        }
        __syncthreads();
        {
            const uint32_t r = 16 * (warp & 1u), c = 16 * (warp / 2);
            float o[2][4] = {};
            two_products<2, 4, 2>(m.t, 32 + r, 32, m.a, 32, 0, m.t, 0, c, (warp & 1u) + 1, warp / 2, o);
            put_tile(m.t, 32 + r, c, o[0]);
            put_tile(m.t, 32 + r, c + 8, o[1]);
        }
        __syncthreads();
        // T = inverse times diag(beta), eight neighbours a thread, below and in the diagonal blocks (nobody reads the rest)
        float x[3][8], most = 0.f;
        auto place = [&](uint32_t u, uint32_t &i, uint32_t &c) {  // piece u of 16 (2 + 4 + 6 + 8)
            const uint32_t block = u < 32 ? 0 : u < 96 ? 1 : u < 192 ? 2 : 3, in = u - 16 * block * (block + 1), width = 2 * block + 2;
            i = 16 * block + in / width, c = in % width;
        };
#pragma unroll
        for (uint32_t k = 0; k < 3; ++k) {
            const uint32_t u = k * kPrepThreads + tid;
            uint32_t i, c;
            place(u < 320 ? u : 0, i, c);
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(&m.t[i][8 * c + e]), b = *reinterpret_cast<const float4 *>(&m.b[jj][8 * c + e]);
                x[k][e] = v.x * b.x, x[k][e + 1] = v.y * b.y, x[k][e + 2] = v.z * b.z, x[k][e + 3] = v.w * b.w;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (8 * c + e > i) x[k][e] = 0.f;
                if (!(fabsf(x[k][e]) < kHuge)) bad = 1;
                most = fmaxf(most, fabsf(x[k][e]));
            }
        }
        float ts = 1.f;
        if (kHalf) {
#pragma unroll
            for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            if (lane == 0) m.top[1][warp] = most;
            __syncthreads();
            ts = range_scale(fmaxf(fmaxf(m.top[1][0], m.top[1][1]), fmaxf(m.top[1][2], m.top[1][3])));
            if (tid == 0) work->t_unit = flipped(ts);
        }
#pragma unroll
        for (uint32_t k = 0; k < 3; ++k) {
            const uint32_t u = k * kPrepThreads + tid;
            if (u >= 320) break;
            uint32_t i, c;
            place(u, i, c);
            uint4 hi, lo;
            split2<T>(x[k][0] * ts, x[k][1] * ts, hi.x, lo.x);
            split2<T>(x[k][2] * ts, x[k][3] * ts, hi.y, lo.y);
            split2<T>(x[k][4] * ts, x[k][5] * ts, hi.z, lo.z);
            split2<T>(x[k][6] * ts, x[k][7] * ts, hi.w, lo.w);
            *reinterpret_cast<uint4 *>(work->tile[0] + block_piece(i, c)) = hi;
            *reinterpret_cast<uint4 *>(work->tile[1] + block_piece(i, c)) = lo;
        }
        for (uint32_t i = tid; i < sizeof(m.p) / 16; i += kPrepThreads)
            reinterpret_cast<uint4 *>(work->tile[2])[i] = reinterpret_cast<const uint4 *>(m.p)[i];
        const bool any = __syncthreads_or(bad);
        if (tid == 0) work->by_row = any;
    }
}

template <class T, int D>
cudaError_t launch(const DeltaArgs &a, cudaStream_t s)
{
    static std::atomic<uint64_t> done;
    const cudaError_t e = allow_smem(kv_delta_prep_kernel<T, D>, sizeof(PrepSmem<D>), done);
    if (e != cudaSuccess) return e;
    return launch_dependent(kv_delta_prep_kernel<T, D>, a.n_slots * (a.n_heads / a.group), kPrepThreads, sizeof(PrepSmem<D>), s, a);
}

}  // namespace

cudaError_t launch_delta_prep(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    if (head_dim == 128) return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 128>(a, s) : launch<__half, 128>(a, s);
    return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 64>(a, s) : launch<__half, 64>(a, s);
}

}  // namespace gms
