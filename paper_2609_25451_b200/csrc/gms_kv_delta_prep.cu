// The gated delta rule, 64 rows at a time: what a chunk's rows do to one another, then the chain of the states.
//
// With G the sum of the log gates from the chunk's first row on, r the keys' factors to unit length and S0 the state before the
// chunk (all of it row by row the same as the rule):
//   d = T (V - diag(f) K S0),            T = (I + A)^-1 diag(beta),  A_ij = beta_i r_i r_j (k_i.k_j) e^(G_i - G_j) for j < i, f = r e^G
//   out = diag(h) Q S0 + P d,            P_ij = scale s_i r_j (q_i.k_j) e^(G_i - G_j) for j <= i,  h = scale s e^G
//   S1 = e^G_last S0 + K^T diag(w) d,    w = r e^(G_last - G)
// T, P, f, h and w do not depend on the state: the first kernel makes them for all chunks at once.  The second goes through each
// sequence's chunks.  q, k and v enter the products as they are; differences of G are taken in 64 bits.  T, P and what they meet are
// terms of bf16 for both types: elements of one chunk lie as far apart as its decays do, and no scale would fit all of them into fp16.
#include "gms_kv_delta.h"

namespace gms {
namespace {

constexpr float kMostNegative = -200.f;  // a gate of e^-200 is 0 in 32 bits, as is every product with it

using ptx::ldmatrix_x4;
using ptx::ldmatrix_x4_trans;
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

constexpr uint32_t kPrepThreads = 128, kPrepHeads = 4;

// The sequences that are done in chunks, longest first (by their share of the longest possible, in 256 steps; which of two in the
// same step comes first is open, and no result depends on it): the chain's CTAs start in this order, so that short sequences fill up
// what the long ones leave.
__device__ void put_order(const DeltaArgs &a, uint32_t *count)
{
    const uint32_t tid = threadIdx.x;
    auto step_of = [&](int rows) { return 255u - (uint32_t)((uint64_t)(rows - 1) * 256 / a.max_q); };
    for (uint32_t i = tid; i < 256; i += kPrepThreads) count[i] = 0;
    __syncthreads();
    for (uint32_t s = tid; s < a.n_seq; s += kPrepThreads) {
        const int rows = delta_rows(a, s);
        if (delta_in_chunks(a, rows)) atomicAdd(&count[step_of(rows)], 1u);
    }
    __syncthreads();
    if (tid < 32) {
        uint32_t n[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) n[i] = count[8 * tid + i], sum += n[i];
        uint32_t before = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
            if (tid >= (uint32_t)o) before += x;
        }
        if (tid == 31) count[256] = before;
        before -= sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) count[8 * tid + i] = before, before += n[i];
    }
    __syncthreads();
    for (uint32_t s = tid; s < a.n_seq; s += kPrepThreads) {
        const int rows = delta_rows(a, s);
        if (delta_in_chunks(a, rows)) a.order[atomicAdd(&count[step_of(rows)], 1u)] = s;
        if (s >= count[256]) a.order[s] = kNone;
    }
}

// Blocks of 16 x 16, as two bf16 terms (2^-17 relative together).
template <int N>
struct Terms {
    uint8_t hi[N * 512], lo[N * 512];
};
struct View {
    uint8_t *hi, *lo;
};
template <int D>
struct PrepSmem {
    union {
        struct {
            uint8_t k[kChunkRows * D * 2], q[kChunkRows * D * 2];
        };
        struct {
            Terms<6> a;                  // A below its diagonal blocks
            Terms<5> inv;                // of I + A: the diagonal blocks' inverses and block (3, 2) of the inverse
            Terms<10> t;                 // the inverse times diag(beta)
            float diag[4][16][20];       // A's diagonal blocks
            Terms<10> p;
        };
    };
    float sum[kPrepHeads][2][kChunkRows];  // G / ln 2, as the sum of two
    float b[kPrepHeads][kChunkRows], rk[kChunkRows], rq[kChunkRows];
    float k2[kChunkRows];  // fp16: |k|^2
};

// Byte offset of block (i, j) in a triangle, in one without its diagonal, and of 16-byte piece c (0, 1) of row r in a block.
__device__ __forceinline__ uint32_t block_at(uint32_t i, uint32_t j) { return (i * (i + 1) / 2 + j) * 512; }
__device__ __forceinline__ uint32_t below_at(uint32_t i, uint32_t j) { return (i * (i - 1) / 2 + j) * 512; }
__device__ __forceinline__ uint32_t piece_in(uint32_t r, uint32_t c) { return (r * 2 + ((c ^ (r / 4)) & 1u)) * 16; }

// A block as a first factor; and c += x y with y a block: two terms each, the product of the small ones left out.
struct First {
    uint32_t hi[4], lo[4];
};
__device__ __forceinline__ First first_of(View x, uint32_t block)
{
    const uint32_t lane = threadIdx.x & 31u, at = block + piece_in(lane & 15u, lane / 16);
    First f;
    ldmatrix_x4(smem_u32(x.hi) + at, f.hi);
    ldmatrix_x4(smem_u32(x.lo) + at, f.lo);
    return f;
}
__device__ __forceinline__ First first_of(const float (*x)[4])  // minus the accumulators of a 16 x 16
{
    First f;
#pragma unroll
    for (int e = 0; e < 4; ++e) split2<__nv_bfloat16>(-x[e / 2][2 * (e & 1)], -x[e / 2][2 * (e & 1) + 1], f.hi[e], f.lo[e]);
    return f;
}
__device__ __forceinline__ void add_product(float (*c)[4], const First &x, View y, uint32_t block)
{
    const uint32_t lane = threadIdx.x & 31u, at = block + piece_in(lane & 15u, lane / 16);
    uint32_t hi[4], lo[4];
    ldmatrix_x4_trans(smem_u32(y.hi) + at, hi);
    ldmatrix_x4_trans(smem_u32(y.lo) + at, lo);
    const __nv_bfloat16 type{};
    mma16816(c[0], x.hi, hi[0], hi[1], type);
    mma16816(c[1], x.hi, hi[2], hi[3], type);
    mma16816(c[0], x.lo, hi[0], hi[1], type);
    mma16816(c[1], x.lo, hi[2], hi[3], type);
    mma16816(c[0], x.hi, lo[0], lo[1], type);
    mma16816(c[1], x.hi, lo[2], lo[3], type);
}
// Two neighbours of a row as two terms; a 16 x 16 of accumulators.
__device__ __forceinline__ void put_pair(View t, uint32_t at, float x, float y)
{
    uint32_t hi, lo;
    split2<__nv_bfloat16>(x, y, hi, lo);
    *reinterpret_cast<uint32_t *>(t.hi + at) = hi;
    *reinterpret_cast<uint32_t *>(t.lo + at) = lo;
}
__device__ __forceinline__ void put_block(View t, uint32_t block, const float (*x)[4], float &finite)
{
    const uint32_t lane = threadIdx.x & 31u, g = lane / 4, q = (lane & 3u) * 4;
#pragma unroll
    for (uint32_t nt = 0; nt < 2; ++nt) {
        put_pair(t, block + piece_in(g, nt) + q, x[nt][0], x[nt][1]);
        put_pair(t, block + piece_in(g + 8, nt) + q, x[nt][2], x[nt][3]);
#pragma unroll
        for (int e = 0; e < 4; ++e) finite = fmaf(x[nt][e], 0.f, finite);
    }
}

// One CTA per chunk and key head.  k_i.k_j and q_i.k_j on mma.sync (the diagonals are the rows' lengths), the ten blocks of the
// triangle shared out as three, two, three and two, then for each value head of the key head the decays, the inverse and what goes to
// the workspace.  The inverse of I + A: its diagonal blocks of 16 x 16 a warp each (a lane has a column and goes down it:
// x_i = -sum_(j<i) A_ij x_j), then, for blocks of 16 and of 32,
//   (X 0; Y Z)^-1 = (X^-1 0; -Z^-1 Y X^-1 Z^-1)
// in products of two-term factors (2^-16 relative, as T itself is handed on).  Bound by the issue of its 7,000 instructions a chunk and
// head and by its warps' waits for one another, which five CTAs an SM fill up (six, with fewer registers: 3 us more): 8,192 rows of 32
// heads of 128, bf16, 56 us (with P in one term 53; earlier steps: T, P and factors in 32 bits 172, blocks of two-term factors 62.5, with
// a warp for each 16 rows 59.5).
template <class T, int D>
__global__ void __launch_bounds__(kPrepThreads, 5) kv_delta_prep_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    PrepSmem<D> &m = *reinterpret_cast<PrepSmem<D> *>(raw);
    constexpr int C = kChunkRows, P = D / 8;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32, g = lane / 4, t2 = 2 * (lane & 3u);
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    if (blockIdx.x == 0) {
        put_order(a, reinterpret_cast<uint32_t *>(raw));
        return;
    }
    const uint32_t n_key = a.n_heads / a.group, kh = (blockIdx.x - 1) % n_key, id = (blockIdx.x - 1) / n_key;
    uint32_t s, chunk;
    if (!find_chunk(a, id, s, chunk)) return;
    const int all_rows = delta_rows(a, s);
    if (!delta_in_chunks(a, all_rows) || chunk > (uint32_t)(all_rows - 1) / C) return;
    const int n = min(all_rows - (int)chunk * C, C), first = delta_begin(a, s) + (int)chunk * C;
    {
        const uint32_t c = tid % P, r0 = tid / P;
        const uint8_t *kp = a.k + (uint64_t)first * a.k_token + kh * a.k_head + c * 16, *qp = a.q + (uint64_t)first * a.q_token + kh * a.q_head + c * 16;
#pragma unroll
        for (uint32_t i = 0; i < (uint32_t)(C * P) / kPrepThreads; ++i) {
            const uint32_t r = r0 + i * (kPrepThreads / P), real = (int)r < n ? r : 0;
            cp16(smem_u32(m.k) + piece<P>(r, c), kp + real * a.k_token, (int)r < n);
            cp16(smem_u32(m.q) + piece<P>(r, c), qp + real * a.q_token, (int)r < n);
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float finite = 0.f;  // NaN once something was not finite
    // products of keys and queries with keys, block by block: a warp has its diagonal block and one or two below (warp 0, two of the
    // last row of blocks), and of its queries with themselves
    const bool far = warp == 0;
    const int blocks = warp & 1u ? 2 : 3;
    auto row_of = [&](int b) { return b && far ? 3u : warp; };
    auto col_of = [&](int b) { return b == 0 ? warp : b == 2 ? 1u : warp == 3 ? 2u : 0u; };
    const uint32_t b_row = (lane & 7u) + (lane & 16u) / 2, b_piece = lane / 8 & 1u;
    float kk[3][2][4] = {}, qk[3][2][4] = {};
    {
        float qq[2][4] = {};
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) {
            uint32_t ka[4], qa[4], x[4];
            const uint32_t at = piece<P>(16 * warp + (lane & 15u), 2 * kt + lane / 16);
            ldmatrix_x4(smem_u32(m.k) + at, ka);
            ldmatrix_x4(smem_u32(m.q) + at, qa);
            ldmatrix_x4(smem_u32(m.q) + piece<P>(16 * warp + b_row, 2 * kt + b_piece), x);
            mma16816(qq[0], qa, x[0], x[1], T());
            mma16816(qq[1], qa, x[2], x[3], T());
#pragma unroll
            for (int b = 0; b < 3; ++b) {
                if (b >= blocks) break;
                if (b == 1 && far) {
                    const uint32_t last = piece<P>(48 + (lane & 15u), 2 * kt + lane / 16);
                    ldmatrix_x4(smem_u32(m.k) + last, ka);
                    ldmatrix_x4(smem_u32(m.q) + last, qa);
                }
                ldmatrix_x4(smem_u32(m.k) + piece<P>(16 * col_of(b) + b_row, 2 * kt + b_piece), x);
                mma16816(kk[b][0], ka, x[0], x[1], T());
                mma16816(kk[b][1], ka, x[2], x[3], T());
                mma16816(qk[b][0], qa, x[0], x[1], T());
                mma16816(qk[b][1], qa, x[2], x[3], T());
            }
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (8 * nt + t2 + (e & 1) == g + (e & 2) * 4) {  // on the diagonal
                    const uint32_t r = 16 * warp + g + (e & 2) * 4;
                    const float k2 = kk[0][nt][e], q2 = qq[nt][e];
                    if (kHalf) m.k2[r] = k2;
                    finite = fmaf(k2, 0.f, fmaf(q2, 0.f, finite));
                    m.rk[r] = a.unit_qk && (int)r < n ? rsqrtf(k2 + a.unit_eps) : 1.f;
                    m.rq[r] = a.unit_qk && (int)r < n ? rsqrtf(q2 + a.unit_eps) : 1.f;
                }
    }
    const View va = {m.a.hi, m.a.lo}, vi = {m.inv.hi, m.inv.lo}, vt = {m.t.hi, m.t.lo}, vp = {m.p.hi, m.p.lo};
    for (uint32_t j = 0; j < a.group; ++j) {
        ChunkWork *work = reinterpret_cast<ChunkWork *>(a.chunks + ((uint64_t)id * a.n_heads + kh * a.group + j) * sizeof(ChunkWork));
        const uint32_t jj = j % kPrepHeads;
        __syncthreads();  // the keys and queries, or the last head's matrices, have been read
        if (jj == 0) {
            if (j + warp < a.group) {  // gates of four heads, a warp each: two rows a lane, sums in 64 bits
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
                    if (!(raw_g[e] < kHuge)) finite = __int_as_float(0x7fffffff);  // (-infinity clears the state)
                    finite = fmaf(beta[e], 0.f, finite);
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
                // fp16: terms of w d have one scale for many rows, so an error of 2^-37 of the largest of them, which meets the longest key
                // where the shortest is the largest's own.  Keys more than 2^18 apart go row by row; those of zero, whose w may be any
                // size, add nothing
                float2 k2 = make_float2(1.f, 1.f);
                if (kHalf) {
                    k2 = *reinterpret_cast<const float2 *>(&m.k2[2 * lane]);
                    float most = fmaxf(k2.x, k2.y), least = fminf(k2.x > 0.f ? k2.x : kHuge, k2.y > 0.f ? k2.y : kHuge);
#pragma unroll
                    for (int o = 16; o; o >>= 1) {
                        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                        least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
                    }
                    if (most * 0x1p-36f > least) finite = __int_as_float(0x7fffffff);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 2 * (int)lane + e;
                    const double sum = inc - sum_g + x[e];
                    const bool in = r < n;
                    m.sum[warp][0][r] = (float)sum, m.sum[warp][1][r] = (float)(sum - (double)(float)sum);
                    m.b[warp][r] = beta[e];
                    const float gate = exp2f((float)sum), f = in ? m.rk[r] * gate : 0.f, hh = in ? a.scale * m.rq[r] * gate : 0.f,
                                ww = in && (e ? k2.y : k2.x) > 0.f ? m.rk[r] * exp2f((float)(last - sum)) : 0.f;
                    w.f[r] = f, w.h[r] = hh, w.w[r] = ww;
                    w.gate[r] = expf(raw_g[e]), w.beta[r] = beta[e], w.rk[r] = m.rk[r], w.rq[r] = m.rq[r];
                    finite = fmaf(f, 0.f, fmaf(hh, 0.f, fmaf(ww, 0.f, finite)));
                }
                const float all = exp2f((float)last);
                finite = fmaf(all, 0.f, finite);
                if (lane == 0) w.all = all;
            }
            __syncthreads();
        }
        // A and P: rows r0 and r0 + 8, columns c0 + {0, 1} and c0 + 8 + {0, 1} of a block (something in A that is not finite comes
        // through to T)
        const float2 minus = make_float2(-1.f, -1.f);
        auto twice = [](float x) { return make_float2(x, x); };
#pragma unroll
        for (int b = 0; b < 3; ++b) {
            if (b >= blocks) break;
            const uint32_t bi = row_of(b), bj = col_of(b), r0 = 16 * bi + g, c0 = 16 * bj + t2;
            float2 sh[2], sl[2], bk[2], sq[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t r = r0 + 8 * e;
                sh[e] = twice(m.sum[jj][0][r]), sl[e] = twice(m.sum[jj][1][r]);
                bk[e] = twice(m.b[jj][r] * m.rk[r]), sq[e] = twice((int)r < n ? a.scale * m.rq[r] : 0.f);
            }
#pragma unroll
            for (int nt = 0; nt < 2; ++nt) {
                const uint32_t c = c0 + 8 * nt;
                const float2 ch = *reinterpret_cast<const float2 *>(&m.sum[jj][0][c]), cl = *reinterpret_cast<const float2 *>(&m.sum[jj][1][c]);
                const float2 rc = *reinterpret_cast<const float2 *>(&m.rk[c]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float2 d = ptx::add2(ptx::fma2(ch, minus, sh[e]), ptx::fma2(cl, minus, sl[e]));
                    const float2 z = ptx::mul2(rc, make_float2(ptx::ex2(d.x), ptx::ex2(d.y)));
                    float2 av = ptx::mul2(bk[e], ptx::mul2(make_float2(kk[b][nt][2 * e], kk[b][nt][2 * e + 1]), z));
                    float2 pn = ptx::mul2(sq[e], ptx::mul2(make_float2(qk[b][nt][2 * e], qk[b][nt][2 * e + 1]), z));
                    if (b == 0) {
                        const uint32_t r = g + 8 * e, x = 8 * nt + t2;
                        if (x >= r) av.x = 0.f;
                        if (x + 1 >= r) av.y = 0.f;
                        if (x > r) pn.x = 0.f;
                        if (x + 1 > r) pn.y = 0.f;
                        *reinterpret_cast<float2 *>(&m.diag[warp][r][x]) = av;
                    } else {
                        put_pair(va, below_at(bi, bj) + piece_in(g + 8 * e, nt) + 2 * t2, av.x, av.y);
                    }
                    const float2 twofold = ptx::add2(pn, pn);  // (what rounds to an infinite term counts, too)
                    finite = fmaf(twofold.x, 0.f, fmaf(twofold.y, 0.f, finite));
                    put_pair(vp, block_at(bi, bj) + piece_in(g + 8 * e, nt) + 2 * t2, pn.x, pn.y);
                }
            }
        }
        __syncwarp();
        if (lane < 16) {  // the warp's own diagonal block
            float x[16];
            const float b = m.b[jj][16 * warp + lane];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float sum = i == (int)lane ? 1.f : 0.f;
#pragma unroll
                for (int c = 0; c < i; c += 4) {
                    const float4 r = *reinterpret_cast<const float4 *>(&m.diag[warp][i][c]);
                    sum -= r.x * x[c];
                    if (c + 1 < i) sum -= r.y * x[c + 1];
                    if (c + 2 < i) sum -= r.z * x[c + 2];
                    if (c + 3 < i) sum -= r.w * x[c + 3];
                }
                x[i] = sum;
            }
#pragma unroll
            for (int i = 0; i < 16; i += 2) {  // neighbouring lanes are neighbours of a row: each stores one row's pair of them
                const float other = __shfl_xor_sync(0xffffu, lane & 1u ? x[i] : x[i + 1], 1), ob = __shfl_xor_sync(0xffffu, b, 1);
                const float mine = lane & 1u ? x[i + 1] : x[i];
                const float l = lane & 1u ? other : mine, r = lane & 1u ? mine : other;
                const uint32_t at = piece_in(i + (lane & 1u), lane / 8) + (lane & 6u) * 2;
                put_pair(vi, warp * 512 + at, l, r);
                put_pair(vt, block_at(warp, warp) + at, l * (lane & 1u ? ob : b), r * (lane & 1u ? b : ob));
                finite = fmaf(x[i], 0.f, fmaf(x[i + 1], 0.f, finite));
            }
        }
        __syncthreads();
        constexpr uint32_t kInv32 = 4 * 512;  // where block (3, 2) of the inverse is
        if (warp != 1) {  // blocks (1, 0) and (3, 2) of T; (3, 2) of the inverse, too
            const uint32_t i = warp == 0 ? 0 : 2;
            float mid[2][4] = {}, o[2][4] = {};
            add_product(mid, first_of(vi, (i + 1) * 512), va, below_at(i + 1, i));
            add_product(o, first_of(mid), warp == 3 ? vi : vt, warp == 3 ? i * 512 : block_at(i, i));
            put_block(warp == 3 ? vi : vt, warp == 3 ? kInv32 : block_at(i + 1, i), o, finite);
        }
        __syncthreads();
        {  // blocks (2 .. 3, 0 .. 1) of T, one a warp
            const uint32_t i = 2 + (warp & 1u), c = warp / 2;
            float o[2][4] = {};
#pragma unroll
            for (uint32_t k = 0; k < 2; ++k) {
                if (k < c) continue;
                float mid[2][4] = {};
                add_product(mid, first_of(vi, i == 2 ? 2 * 512 : kInv32), va, below_at(2, k));
                if (i == 3) add_product(mid, first_of(vi, 3 * 512), va, below_at(3, k));
                add_product(o, first_of(mid), vt, block_at(k, c));
            }
            put_block(vt, block_at(i, c), o, finite);
        }
        __syncthreads();
        constexpr uint32_t kPieces = sizeof(m.p.hi) / 16;
        for (uint32_t u = tid; u < kPieces; u += kPrepThreads) {
            reinterpret_cast<uint4 *>(work->tile[0])[u] = reinterpret_cast<const uint4 *>(m.t.hi)[u];
            reinterpret_cast<uint4 *>(work->tile[1])[u] = reinterpret_cast<const uint4 *>(m.t.lo)[u];
            reinterpret_cast<uint4 *>(work->tile[2])[u] = reinterpret_cast<const uint4 *>(m.p.hi)[u];
            reinterpret_cast<uint4 *>(work->tile[3])[u] = reinterpret_cast<const uint4 *>(m.p.lo)[u];
        }
        const bool any = __syncthreads_or(finite != 0.f);
        if (tid == 0) work->by_row = any;
    }
}

template <class T, int D>
cudaError_t launch(const DeltaArgs &a, cudaStream_t s)
{
    static std::atomic<uint64_t> done;
    const cudaError_t e = allow_smem(kv_delta_prep_kernel<T, D>, sizeof(PrepSmem<D>), done);
    if (e != cudaSuccess) return e;
    return launch_dependent(kv_delta_prep_kernel<T, D>, a.n_slots * (a.n_heads / a.group) + 1, kPrepThreads, sizeof(PrepSmem<D>), s, a);
}

}  // namespace

cudaError_t launch_delta_prep(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    if (head_dim == 128) return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 128>(a, s) : launch<__half, 128>(a, s);
    return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 64>(a, s) : launch<__half, 64>(a, s);
}

}  // namespace gms
