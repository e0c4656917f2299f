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
using ptx::ldmatrix_x4_trans;
using ptx::smem_u32;

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// Byte offset of 16-byte piece c of row r in a tile of P pieces a row, so that eight neighbouring rows' pieces c lie in different banks.
template <int P>
__device__ __forceinline__ uint32_t piece(uint32_t r, uint32_t c)
{
    return (r * P + (P >= 8 ? c ^ (r & 7u) : c ^ ((r * P / 8) & (P - 1u)))) * 16;
}

// The same in a lower triangle's blocks of 16 x 16 16-bit numbers: piece c (of the 8 of a whole row), c / 2 <= r / 16.
__device__ __forceinline__ uint32_t block_piece(uint32_t r, uint32_t c)
{
    const uint32_t b = r / 16;
    return (b * (b + 1) / 2 + c / 2) * 512 + (r % 16 * 2 + ((c ^ (r / 4)) & 1u)) * 16;
}

// x = hi + lo with both of type T (2^-17 relative in bf16, the rest of f16's range aside).
template <class T>
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo)
{
    hi = pack2(x, y, T());
    const T *e = reinterpret_cast<const T *>(&hi);
    lo = pack2(x - to_f32(e[0]), y - to_f32(e[1]), T());
}

// A power of two by which a row of f16 terms is scaled so that its largest is below 2^12 (bf16 has the range of 32 bits); within
// 2^-30 .. 2^30, so that three such factors together stay far from the ends of 32 bits.
__device__ __forceinline__ float range_scale(float top)
{
    const int e = (int)(__float_as_uint(top) >> 23 & 255u) - 127;  // 2^e <= top
    return __uint_as_float((uint32_t)(127 + min(max(11 - e, -30), 30)) << 23);
}

// 1 / u for a power of two.
__device__ __forceinline__ float flipped(float u) { return __uint_as_float(0x7f000000u - __float_as_uint(u)); }

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
    cp_commit();
    cp_wait();
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

// Stage of the chain: a chunk's operands.  V is the columns of the CTA.
template <int D, int W>
struct Stage {
    uint8_t k[kChunkRows * D * 2], q[kChunkRows * D * 2], v[kChunkRows * W * 32];
    ChunkWork w;
};
// What the four warps of a slice tell each other: first factors of products, a lane's part of 16 x 16 of them each.
template <int D, bool UNITS>
struct Shared {
    uint4 s_hi[2][D / 16][32], s_lo[D / 16][32];  // S, in two terms; the first of this chunk and of the next
    uint4 x[4][2][32];                            // V - f X of the 16 rows of each warp, in two terms
    uint4 dw[4][2][32];                           // w d, in two terms
    uint4 d[4][32];
    float2 s_unit[2][UNITS ? 4 : 1][32], x_unit[UNITS ? 4 : 1][32], dw_unit[UNITS ? 4 : 1][32], d_unit[UNITS ? 4 : 1][32];  // f16: powers of
    uint32_t odd[4];                                                                                        // two that terms are multiples of
};
template <class T, int D, int W>
struct ChainSmem {
    static constexpr bool kUnits = std::is_same<T, __half>::value;
    static constexpr int kStages = D == 64 || W == 2 ? 3 : 2;  // that fit
    Stage<D, W> stage[kStages];
    Shared<D, kUnits> shared[W];
    uint64_t full[kStages], empty[kStages];
};
constexpr uint32_t kFetchWarps = 2, kFetchLanes = kFetchWarps * 32;

// A tile of 64 rows, PR pieces each; rows from n on are zeros.  A lane keeps to one piece of the rows that it copies.
template <int PR>
__device__ __forceinline__ void fetch_rows(uint32_t tile, uint32_t me, const uint8_t *src, uint64_t stride, int n)
{
    constexpr uint32_t kStep = kFetchLanes / PR, N = kChunkRows / kStep;
    const uint32_t c = me % PR, r0 = me / PR;
    src += r0 * stride + c * 16;
    if (n >= (int)kChunkRows) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            cp16(tile + piece<PR>(r0 + i * kStep, c), src, true);
            src += kStep * stride;
        }
    } else {
#pragma unroll 1
        for (uint32_t r = r0; r < (uint32_t)kChunkRows; r += kStep) {
            const bool real = (int)r < n;
            cp16(tile + piece<PR>(r, c), real ? src : src - r * stride, real);
            src += kStep * stride;
        }
    }
}
// Chunk `chunk` of a sequence; `full` is told when it has landed.
template <int D, int W>
__device__ __forceinline__ void fetch_chunk(const DeltaArgs &a, Stage<D, W> &st, uint32_t me, int chunk, int rows, int first, uint32_t kh, uint32_t h,
                                            uint32_t col0, uint32_t slot, uint32_t full)
{
    const int n = rows - chunk * (int)kChunkRows;
    const uint64_t row = (uint64_t)(first + chunk * (int)kChunkRows);
    const uint8_t *work = a.chunks + ((uint64_t)(slot + chunk) * a.n_heads + h) * sizeof(ChunkWork) + me * 16;
    const uint32_t to = smem_u32(&st.w) + me * 16;
    fetch_rows<D / 8>(smem_u32(st.k), me, a.k + row * a.k_token + kh * a.k_head, a.k_token, n);
    fetch_rows<W * 2>(smem_u32(st.v), me, a.v + row * a.v_token + h * a.v_head + col0 * 2, a.v_token, n);
    static_assert(sizeof(ChunkWork) % (16 * kFetchLanes) == 0, "");
#pragma unroll
    for (uint32_t i = 0; i < sizeof(ChunkWork) / (16 * kFetchLanes); ++i) cp16(to + i * 16 * kFetchLanes, work + i * 16 * kFetchLanes, true);
    fetch_rows<D / 8>(smem_u32(st.q), me, a.q + row * a.q_token + kh * a.q_head, a.q_token, n);
    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(full) : "memory");
}

// Four warps have 16 value columns of a head's state, transposed, as accumulators of mma.sync: each the columns of D / 4 keys for
// the state itself and 16 of the chunk's rows for everything that has rows.  What is an accumulator of one product is, element
// for element, a first factor of the next: S -> X = S K^T, Y = S Q^T -> d = (V - f X) T^T -> S, out.  Between those steps the warps
// hand their parts round through shared memory, three exchanges a chunk.  W such slices share a chunk's operands, which two more
// warps fetch one chunk ahead.
template <class T, int D, int W>
__global__ void __launch_bounds__((4 * W + kFetchWarps) * 32) kv_delta_chain_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    ChainSmem<T, D, W> &m = *reinterpret_cast<ChainSmem<T, D, W> *>(raw);
    constexpr int C = kChunkRows, P = D / 8, VP = W * 2, NT = D / 32, KQ = D / 64;  // tiles of 8 and of 16 keys that a warp has
    constexpr int kStages = ChainSmem<T, D, W>::kStages;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    constexpr uint32_t kSlices = D / (16 * W);
    const uint32_t part = blockIdx.x % kSlices, h = blockIdx.x / kSlices % a.n_heads, s = blockIdx.x / kSlices / a.n_heads, kh = h / a.group;
    const uint32_t col0 = part * W * 16;  // of the CTA
    ptx::grid_launch_dependents();
    ptx::grid_wait();
    const int rows = delta_rows(a, s), first = delta_begin(a, s);
    if (!delta_in_chunks(a, rows)) return;
    const int chunks = (rows + C - 1) / C;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            ptx::mbar_init(smem_u32(&m.full[i]), kFetchLanes);
            ptx::mbar_init(smem_u32(&m.empty[i]), 4 * W);
        }
        ptx::fence_mbar_init();
    }
    __syncthreads();
    // A wait that runs out (it cannot, but for a fault in here) is told in the status word; everybody goes on without waiting.
    bool late = false;
    auto wait = [&](uint64_t *bar, int use) {
        if (late || ptx::mbar_wait(smem_u32(bar), (uint32_t)(use & 1))) return;
        late = true;
        if (a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_TIMEOUT);
    };
    if (warp >= 4 * W) {  // the fetching warps
        const uint32_t me = (warp - 4 * W) * 32 + lane, slot = delta_slot(a, s);
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int i = chunk % kStages;
            if (chunk >= kStages) wait(&m.empty[i], chunk / kStages - 1);
            fetch_chunk<D, W>(a, m.stage[i], me, chunk, rows, first, kh, h, col0, slot, smem_u32(&m.full[i]));
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    // (the last rows have most to do: of two slices they go to different quarters of the SM)
    const uint32_t slice = warp / 4, mine = (warp & 3u) ^ (slice & 1u ? 3u : 0u);
    const bool fresh = a.past_lens && a.past_lens[s] <= 0;
    const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
    float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
    if (a.status && threadIdx.x == 0 && ((!fresh && !from) || !to)) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
    const uint32_t g = lane / 4, t2 = 2 * (lane & 3u);  // rows g and g + 8, columns 8 nt + t2 + {0, 1} of an accumulator
    const uint32_t at0 = (mine * (D / 4) + t2) * D + col0 + 16 * slice + g;
    const uint32_t row0 = 16 * mine, b_row = (lane & 7u) + (lane & 16u) / 2, b_piece = lane / 8 & 1u;  // of a lane's address for two second factors
    float S[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[nt][e] = from ? from[at0 + (8 * nt + (e & 1)) * D + (e & 2) * 4] : 0.f;
    auto &sh = m.shared[slice];
    auto together = [&] { asm volatile("bar.sync %0, 128;" ::"r"(slice + 1) : "memory"); };
    // Two terms of the 16 x 16 tile in accumulators x and y; f16: rows scaled by a power of two of their own, which goes to `unit`.
    auto top_of = [](const float *x, const float *y, int e) {
        float top = fmaxf(fmaxf(fabsf(x[2 * e]), fabsf(x[2 * e + 1])), fmaxf(fabsf(y[2 * e]), fabsf(y[2 * e + 1])));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        return fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    };
    auto put_terms = [&](uint4 *to_hi, uint4 *to_lo, const float *x, const float *y, float u0, float u1) {
        uint4 hi, lo;
        split2<T>(x[0] * u0, x[1] * u0, hi.x, lo.x);
        split2<T>(x[2] * u1, x[3] * u1, hi.y, lo.y);
        split2<T>(y[0] * u0, y[1] * u0, hi.z, lo.z);
        split2<T>(y[2] * u1, y[3] * u1, hi.w, lo.w);
        to_hi[lane] = hi, to_lo[lane] = lo;
    };
#pragma unroll 1
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int stage = chunk % kStages;
        Stage<D, W> &st = m.stage[stage];
        auto done = [&] {
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(smem_u32(&m.empty[stage]));
        };
        wait(&m.full[stage], chunk / kStages);
        const uint32_t turn = chunk & 1;
        const int n = min(rows - chunk * C, C);
        uint8_t *out = a.out + (uint64_t)(first + chunk * C) * a.o_token + h * a.o_head + (col0 + 16 * slice) * 2;
        float su[2] = {1.f, 1.f};
        if (kHalf) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = 0.f;
#pragma unroll
                for (int k = 0; k < KQ; ++k) top = fmaxf(top, top_of(S[2 * k], S[2 * k + 1], e));
                su[e] = range_scale(top);
            }
            sh.s_unit[turn][mine][lane] = make_float2(flipped(su[0]), flipped(su[1]));
        }
#pragma unroll
        for (int k = 0; k < KQ; ++k) put_terms(sh.s_hi[turn][mine * KQ + k], sh.s_lo[mine * KQ + k], S[2 * k], S[2 * k + 1], su[0], su[1]);
        // the rows' values, transposed like everything else
        uint32_t V[4];
        ldmatrix_x4_trans(smem_u32(st.v) + piece<VP>(row0 + b_row, 2 * slice + b_piece), V);
        constexpr uint32_t kOnes = kHalf ? 0x7c00u : 0x7f80u;
        uint32_t odd = st.w.by_row;
#pragma unroll
        for (int e = 0; e < 4; ++e) odd |= ((V[e] & kOnes) == kOnes) | ((V[e] >> 16 & kOnes) == kOnes);
        odd = __any_sync(0xffffffffu, odd);
        if (lane == 0) sh.odd[mine] = odd;
        uint32_t kb[D / 16][4];  // (what needs no news from the other warps is read before they meet)
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) ldmatrix_x4(smem_u32(st.k) + piece<P>(row0 + b_row, 2 * kt + b_piece), kb[kt]);
        together();
        if (sh.odd[0] | sh.odd[1] | sh.odd[2] | sh.odd[3]) {
            // row by row: something here is not finite, and in a product it would reach rows that come before it
            float4(*xy)[4][32] = reinterpret_cast<float4(*)[4][32]>(sh.x);  // [2][4][32], in the place of what is not needed
            float(*zs)[4][32] = reinterpret_cast<float(*)[4][32]>(sh.dw);
#pragma unroll 1
            for (int r = 0; r < n; ++r) {
                const float gate = st.w.gate[r], beta = st.w.beta[r], rk = st.w.rk[r], rq = st.w.rq[r];
                float x[2] = {}, y[2] = {}, z = 0.f, kv[2 * NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const T *kp = reinterpret_cast<const T *>(st.k + piece<P>(r, mine * NT + nt)) + t2;
                    const T *qp = reinterpret_cast<const T *>(st.q + piece<P>(r, mine * NT + nt)) + t2;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float k = to_f32(kp[e]) * rk, q = to_f32(qp[e]) * rq;
                        kv[2 * nt + e] = k;
                        z += k * q;
                        S[nt][e] *= gate, S[nt][2 + e] *= gate;
                        x[0] += S[nt][e] * k, x[1] += S[nt][2 + e] * k;
                        y[0] += S[nt][e] * q, y[1] += S[nt][2 + e] * q;
                    }
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    z += __shfl_xor_sync(0xffffffffu, z, o);
#pragma unroll
                    for (int e = 0; e < 2; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], o), y[e] += __shfl_xor_sync(0xffffffffu, y[e], o);
                }
                xy[r & 1][mine][lane] = make_float4(x[0], x[1], y[0], y[1]);
                zs[r & 1][mine][lane] = z;
                together();
                x[0] = x[1] = y[0] = y[1] = z = 0.f;
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    const float4 u = xy[r & 1][o][lane];
                    x[0] += u.x, x[1] += u.y, y[0] += u.z, y[1] += u.w;
                    z += zs[r & 1][o][lane];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float v = to_f32(*reinterpret_cast<const T *>(st.v + piece<VP>(r, 2 * slice + e) + g * 2));
                    const float d = beta * (v - x[e]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) S[nt][2 * e] += kv[2 * nt] * d, S[nt][2 * e + 1] += kv[2 * nt + 1] * d;
                    if (mine == 0 && (lane & 3u) == 0)
                        reinterpret_cast<T *>(out + (uint64_t)r * a.o_token)[g + 8 * e] = from_f32<T>(a.scale * (y[e] + z * d));
                }
            }
            done();
            continue;
        }
        // X = S K^T for the warp's rows
        float X[2][4] = {}, Xl[2][4] = {};
        float2 unit = make_float2(1.f, 1.f);
        // f16: accumulators go over to the unit of the next factors
        auto change = [&](float(*x)[4], float2 now, float2 next) {
            const float f0 = now.x * flipped(next.x), f1 = now.y * flipped(next.y);
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) x[nt][0] *= f0, x[nt][1] *= f0, x[nt][2] *= f1, x[nt][3] *= f1;
        };
        const float2 one = make_float2(1.f, 1.f);
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) {
            if (kHalf && kt % KQ == 0) {
                const float2 next = sh.s_unit[turn][kt / KQ][lane];
                if (kt) change(X, unit, next), change(Xl, unit, next);
                unit = next;
            }
            const uint4 hi = sh.s_hi[turn][kt][lane], lo = sh.s_lo[kt][lane];
            mma16816(X[0], &hi.x, kb[kt][0], kb[kt][1], T());
            mma16816(X[1], &hi.x, kb[kt][2], kb[kt][3], T());
            mma16816(Xl[0], &lo.x, kb[kt][0], kb[kt][1], T());
            mma16816(Xl[1], &lo.x, kb[kt][2], kb[kt][3], T());
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) X[nt][e] += Xl[nt][e];
        if (kHalf) change(X, unit, one);
        // what the values differ by from what the state says: X <- V - f X
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.f[row0 + 8 * nt + t2]);
            const T *va = reinterpret_cast<const T *>(&V[2 * nt]), *vb = reinterpret_cast<const T *>(&V[2 * nt + 1]);
            X[nt][0] = to_f32(va[0]) - f.x * X[nt][0];
            X[nt][1] = to_f32(va[1]) - f.y * X[nt][1];
            X[nt][2] = to_f32(vb[0]) - f.x * X[nt][2];
            X[nt][3] = to_f32(vb[1]) - f.y * X[nt][3];
        }
        float u0 = 1.f, u1 = 1.f;
        if (kHalf) {
            u0 = range_scale(top_of(X[0], X[1], 0)), u1 = range_scale(top_of(X[0], X[1], 1));
            sh.x_unit[mine][lane] = make_float2(flipped(u0), flipped(u1));
        }
        put_terms(sh.x[mine][0], sh.x[mine][1], X[0], X[1], u0, u1);
        uint32_t tb[2][C / 16][4];
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            if (kt > (int)mine) break;
            const uint32_t at = block_piece(row0 + b_row, 2 * kt + b_piece);
            ldmatrix_x4(smem_u32(st.w.tile[0]) + at, tb[0][kt]);
            ldmatrix_x4(smem_u32(st.w.tile[1]) + at, tb[1][kt]);
        }
        together();
        // d = X T^T: two terms each (the product of the small ones left out), from the rows up to the warp's own
        float d[2][4] = {}, dl[2][4] = {}, dt[2][4] = {};
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            if (kt > (int)mine) break;
            if (kHalf) {
                const float2 next = sh.x_unit[kt][lane];
                if (kt) change(d, unit, next), change(dl, unit, next), change(dt, unit, next);
                unit = next;
            }
            const uint4 hi = sh.x[kt][0][lane], lo = sh.x[kt][1][lane];
            const uint32_t *b = tb[0][kt], *c = tb[1][kt];
            mma16816(d[0], &hi.x, b[0], b[1], T());
            mma16816(d[1], &hi.x, b[2], b[3], T());
            mma16816(dl[0], &lo.x, b[0], b[1], T());
            mma16816(dl[1], &lo.x, b[2], b[3], T());
            mma16816(dt[0], &hi.x, c[0], c[1], T());
            mma16816(dt[1], &hi.x, c[2], c[3], T());
        }
        {
            const float f0 = kHalf ? st.w.t_unit * unit.x : 1.f, f1 = kHalf ? st.w.t_unit * unit.y : 1.f;
#pragma unroll
            for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) d[nt][e] = (d[nt][e] + (dl[nt][e] + dt[nt][e])) * (e & 2 ? f1 : f0);
        }
        if (kHalf) {
            u0 = range_scale(top_of(d[0], d[1], 0)), u1 = range_scale(top_of(d[0], d[1], 1));
            sh.d_unit[mine][lane] = make_float2(st.w.p_unit * flipped(u0), st.w.p_unit * flipped(u1));
        }
        sh.d[mine][lane] = make_uint4(pack2(d[0][0] * u0, d[0][1] * u0, T()), pack2(d[0][2] * u1, d[0][3] * u1, T()),
                                      pack2(d[1][0] * u0, d[1][1] * u0, T()), pack2(d[1][2] * u1, d[1][3] * u1, T()));
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.w[row0 + 8 * nt + t2]);
            d[nt][0] *= f.x, d[nt][1] *= f.y, d[nt][2] *= f.x, d[nt][3] *= f.y;
        }
        if (kHalf) {
            u0 = range_scale(top_of(d[0], d[1], 0)), u1 = range_scale(top_of(d[0], d[1], 1));
            sh.dw_unit[mine][lane] = make_float2(flipped(u0), flipped(u1));
        }
        put_terms(sh.dw[mine][0], sh.dw[mine][1], d[0], d[1], u0, u1);
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt)
#pragma unroll
            for (int nt = 0; nt < NT; nt += 2)
                ldmatrix_x4_trans(smem_u32(st.k) + piece<P>(16 * kt + (lane & 15u), mine * NT + nt + lane / 16), kb[kt * (NT / 2) + nt / 2]);
        together();
        // S <- e^G S + (w d) K for the warp's keys
        const float all = st.w.all;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[nt][e] *= all;
        unit = one;
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            if (kHalf) {
                const float2 next = sh.dw_unit[kt][lane];
#pragma unroll
                for (int nt = 0; nt < NT; nt += 2) change(S + nt, unit, next);
                unit = next;
            }
            const uint4 hi = sh.dw[kt][0][lane], lo = sh.dw[kt][1][lane];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    mma16816(S[nt], t ? &lo.x : &hi.x, kb[kt * (NT / 2) + nt / 2][2 * (nt & 1)], kb[kt * (NT / 2) + nt / 2][2 * (nt & 1) + 1], T());
        }
        if (kHalf) {
#pragma unroll
            for (int nt = 0; nt < NT; nt += 2) change(S + nt, unit, one);
        }
        // out = h Q S + P d for the warp's rows, with S before the chunk (one term each): nothing waits for it
        float Y[2][4] = {};
        unit = one;
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) {
            if (kHalf && kt % KQ == 0) {
                const float2 next = sh.s_unit[turn][kt / KQ][lane];
                if (kt) change(Y, unit, next);
                unit = next;
            }
            const uint4 hi = sh.s_hi[turn][kt][lane];
            uint32_t b[4];
            ldmatrix_x4(smem_u32(st.q) + piece<P>(row0 + b_row, 2 * kt + b_piece), b);
            mma16816(Y[0], &hi.x, b[0], b[1], T());
            mma16816(Y[1], &hi.x, b[2], b[3], T());
        }
        if (kHalf) change(Y, unit, one);
        unit = one;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.h[row0 + 8 * nt + t2]);
            Y[nt][0] *= f.x, Y[nt][1] *= f.y, Y[nt][2] *= f.x, Y[nt][3] *= f.y;
        }
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            if (kt > (int)mine) break;
            if (kHalf) {
                const float2 next = sh.d_unit[kt][lane];
                change(Y, unit, next);
                unit = next;
            }
            const uint4 x = sh.d[kt][lane];
            uint32_t b[4];
            ldmatrix_x4(smem_u32(st.w.tile[2]) + block_piece(row0 + b_row, 2 * kt + b_piece), b);
            mma16816(Y[0], &x.x, b[0], b[1], T());
            mma16816(Y[1], &x.x, b[2], b[3], T());
        }
        if (kHalf) change(Y, unit, one);
        // rows of 16 columns through the warp's own part of V's tile
        const uint32_t y[4] = {pack2(Y[0][0], Y[0][1], T()), pack2(Y[0][2], Y[0][3], T()), pack2(Y[1][0], Y[1][1], T()), pack2(Y[1][2], Y[1][3], T())};
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                         smem_u32(st.v) + piece<VP>(row0 + b_row, 2 * slice + b_piece)),
                     "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3])
                     : "memory");
        __syncwarp();
        const uint32_t r = row0 + lane / 2;
        const uint4 x = *reinterpret_cast<const uint4 *>(st.v + piece<VP>(r, 2 * slice + (lane & 1u)));
        if ((int)r < n) *reinterpret_cast<uint4 *>(out + (uint64_t)r * a.o_token + (lane & 1u) * 16) = x;
        done();
    }
    if (!to) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[at0 + (8 * nt + (e & 1)) * D + (e & 2) * 4] = S[nt][e];
}

template <class T, int D, int W>
cudaError_t launch_chain(const DeltaArgs &a, cudaStream_t s)
{
    static_assert(sizeof(ChainSmem<T, D, W>) <= 232448, "");
    static std::atomic<uint64_t> done;
    const cudaError_t e = allow_smem(kv_delta_chain_kernel<T, D, W>, sizeof(ChainSmem<T, D, W>), done);
    if (e != cudaSuccess) return e;
    return launch_dependent(kv_delta_chain_kernel<T, D, W>, a.n_seq * a.n_heads * (D / (16 * W)), (4 * W + kFetchWarps) * 32,
                            sizeof(ChainSmem<T, D, W>), s, a);
}

template <class T, int D>
cudaError_t launch(const DeltaArgs &a, cudaStream_t s)
{
    static std::atomic<uint64_t> done;
    cudaError_t e = allow_smem(kv_delta_prep_kernel<T, D>, sizeof(PrepSmem<D>), done);
    if (e == cudaSuccess)
        e = launch_dependent(kv_delta_prep_kernel<T, D>, a.n_slots * (a.n_heads / a.group), kPrepThreads, sizeof(PrepSmem<D>), s, a);
    if (e != cudaSuccess) return e;
    return (uint64_t)a.n_seq * a.n_heads * (D / 64) > 148 ? launch_chain<T, D, 4>(a, s) : launch_chain<T, D, 2>(a, s);
}

}  // namespace

cudaError_t launch_delta_chunks(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    if (head_dim == 128) return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 128>(a, s) : launch<__half, 128>(a, s);
    return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 64>(a, s) : launch<__half, 64>(a, s);
}

}  // namespace gms
