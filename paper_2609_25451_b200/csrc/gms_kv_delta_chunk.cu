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

constexpr uint32_t kPrepThreads = 128;

template <int D>
struct PrepSmem {
    uint8_t k[kChunkRows * D * 2], q[kChunkRows * D * 2];
    float a[kChunkRows][kChunkRows + 4];
    uint8_t tile[3][kChunkRows * kChunkRows * 2];  // T hi, T lo, P, as they go to the workspace
    double sum[kChunkRows];                        // G
    float rk[kChunkRows], rq[kChunkRows], b[kChunkRows];
    float top[4];
    uint32_t bad;
};

// One CTA per chunk and key head.  k_i.k_j and q_i.k_j on mma.sync (a warp has 16 rows i), then for each value head of the key
// head the decays, the inverse (a thread has a column and goes down it: x_i = -sum_(j<i) A_ij x_j) and what goes to the workspace.
template <class T, int D>
__global__ void __launch_bounds__(kPrepThreads) kv_delta_prep_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    PrepSmem<D> &m = *reinterpret_cast<PrepSmem<D> *>(raw);
    constexpr int C = kChunkRows, P = D / 8;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    const uint32_t n_key = a.n_heads / a.group, kh = blockIdx.x % n_key, id = blockIdx.x / n_key;
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    uint32_t s, chunk;
    if (!find_chunk(a, id, s, chunk)) return;
    const int all_rows = delta_rows(a, s);
    if (!delta_in_chunks(a, all_rows) || chunk > (uint32_t)(all_rows - 1) / C) return;
    const int n = min(all_rows - (int)chunk * C, C), first = delta_begin(a, s) + (int)chunk * C;
    for (uint32_t i = tid; i < (uint32_t)(C * P); i += kPrepThreads) {
        const uint32_t r = i / P, c = i % P;
        const bool real = (int)r < n;
        const uint64_t row = (uint64_t)(first + (real ? (int)r : 0));
        cp16(smem_u32(m.k) + piece<P>(r, c), a.k + row * a.k_token + kh * a.k_head + c * 16, real);
        cp16(smem_u32(m.q) + piece<P>(r, c), a.q + row * a.q_token + kh * a.q_head + c * 16, real);
    }
    cp_commit();
    if (tid == 0) m.bad = 0;
    cp_wait();
    __syncthreads();
    // lengths: two threads a row
    uint32_t bad = 0;
    {
        const uint32_t r = tid / 2;
        float kk = 0.f, qq = 0.f;
        for (uint32_t c = tid & 1u; c < (uint32_t)P; c += 2) {
            const uint4 kv = *reinterpret_cast<const uint4 *>(m.k + piece<P>(r, c)), qv = *reinterpret_cast<const uint4 *>(m.q + piece<P>(r, c));
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
        const uint32_t h = kh * a.group + j;
        uint8_t *ws = a.chunks + ((uint64_t)id * a.n_heads + h) * sizeof(ChunkWork);
        ChunkWork &w = *reinterpret_cast<ChunkWork *>(ws);
        __syncthreads();
        if (warp == 0) {  // gates: two rows a lane, sums in 64 bits
            double x[2], g = 0.;
            float beta[2], raw_g[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 2 * (int)lane + e;
                const uint64_t row = (uint64_t)(first + r);
                raw_g[e] = r < n && a.g ? a.g[row * a.g_stride + h] : 0.f;
                beta[e] = r < n ? a.beta ? a.beta[row * a.beta_stride + h] : 1.f : 0.f;
                if (!(raw_g[e] < kHuge) || !(fabsf(beta[e]) < kHuge)) bad = 1;
                g += (double)(raw_g[e] < kMostNegative ? kMostNegative : raw_g[e]);
                x[e] = g;
            }
            double inc = g;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, inc, o);
                if (lane >= (uint32_t)o) inc += y;
            }
            const double last = __shfl_sync(0xffffffffu, inc, 31);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 2 * (int)lane + e;
                const double sum = inc - g + x[e];
                const bool in = r < n;
                m.sum[r] = sum;
                m.b[r] = beta[e];
                const float f = in ? m.rk[r] * expf((float)sum) : 0.f, hh = in ? a.scale * m.rq[r] * expf((float)sum) : 0.f,
                            ww = in ? m.rk[r] * expf((float)(last - sum)) : 0.f;
                w.f[r] = f, w.h[r] = hh, w.w[r] = ww;
                w.gate[r] = expf(raw_g[e]), w.beta[r] = beta[e], w.rk[r] = m.rk[r], w.rq[r] = m.rq[r];
                if (!(fabsf(f) < kHuge) || !(fabsf(hh) < kHuge) || !(fabsf(ww) < kHuge)) bad = 1;
            }
            const float all = expf((float)last);
            if (!(all < kHuge)) bad = 1;
            if (lane == 0) w.all = all;
        }
        __syncthreads();
        // A and P: row i = 16 warp + lane / 4 (+ 8), columns 8 nt + 2 (lane % 4) + {0, 1}
        float pv[C / 8][4], top = 0.f;
#pragma unroll
        for (int nt = 0; nt < C / 8; ++nt) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * (int)warp + (int)lane / 4 + (e & 2) * 4, c = 8 * nt + 2 * ((int)lane & 3) + (e & 1);
                const float decay = c <= i ? expf((float)(m.sum[i] - m.sum[c])) : 0.f;
                const float av = c < i ? m.b[i] * m.rk[i] * m.rk[c] * kk[nt][e] * decay : 0.f;
                pv[nt][e] = c <= i && i < n ? a.scale * m.rq[i] * m.rk[c] * qk[nt][e] * decay : 0.f;
                if (!(fabsf(av) < kHuge) || !(fabsf(pv[nt][e]) < kHuge)) bad = 1;
                top = fmaxf(top, fabsf(pv[nt][e]));
                m.a[i][c] = av;
            }
        }
        float ps = 1.f;
        if (kHalf) {
#pragma unroll
            for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            if (lane == 0) m.top[warp] = top;
            __syncthreads();
            ps = range_scale(fmaxf(fmaxf(m.top[0], m.top[1]), fmaxf(m.top[2], m.top[3])));
            if (tid == 0) w.p_unit = 1.f / ps;
        }
#pragma unroll
        for (int nt = 0; nt < C / 8; ++nt) {
            const uint32_t i = 16 * warp + lane / 4, c = 4 * (lane & 3u);
            *reinterpret_cast<uint32_t *>(m.tile[2] + piece<8>(i, nt) + c) = pack2(pv[nt][0] * ps, pv[nt][1] * ps, T());
            *reinterpret_cast<uint32_t *>(m.tile[2] + piece<8>(i + 8, nt) + c) = pack2(pv[nt][2] * ps, pv[nt][3] * ps, T());
        }
        __syncthreads();
        if (tid < (uint32_t)C) {
            float x[C];
            const float b = m.b[tid];
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                float sum = i == (int)tid ? 1.f : 0.f;
#pragma unroll
                for (int c = 0; c < i; c += 4) {
                    const float4 r = *reinterpret_cast<const float4 *>(&m.a[i][c]);
                    sum -= r.x * x[c];
                    if (c + 1 < i) sum -= r.y * x[c + 1];
                    if (c + 2 < i) sum -= r.z * x[c + 2];
                    if (c + 3 < i) sum -= r.w * x[c + 3];
                }
                x[i] = sum;
            }
#pragma unroll
            for (int i = 0; i < C; ++i) {
                x[i] *= b;
                if (!(fabsf(x[i]) < kHuge)) bad = 1;
                most = fmaxf(most, fabsf(x[i]));
            }
            float ts = 1.f;
            if (kHalf) {
#pragma unroll
                for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                if (lane == 0) m.top[warp] = most;
                asm volatile("bar.sync 1, 64;" ::: "memory");
                ts = range_scale(fmaxf(m.top[0], m.top[1]));
                if (tid == 0) w.t_unit = 1.f / ts;
            }
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const T hi = from_f32<T>(x[i] * ts), lo = from_f32<T>(x[i] * ts - to_f32(hi));
                const uint32_t at = piece<8>(i, tid / 8) + (tid & 7u) * 2;
                *reinterpret_cast<T *>(m.tile[0] + at) = hi;
                *reinterpret_cast<T *>(m.tile[1] + at) = lo;
            }
        }
        const bool any = __syncthreads_or(bad);
        if (tid == 0) w.by_row = any;
        const uint4 *from = reinterpret_cast<const uint4 *>(m.tile);
        uint4 *to = reinterpret_cast<uint4 *>(w.tile);
        for (uint32_t i = tid; i < sizeof(m.tile) / 16; i += kPrepThreads) to[i] = from[i];
    }
}

// Stage of the chain: a chunk's operands.  V is the columns of the CTA.
template <int D, int W>
struct Stage {
    uint8_t k[kChunkRows * D * 2], q[kChunkRows * D * 2], v[kChunkRows * W * 32];
    ChunkWork w;
};

// A warp has 16 value columns of a head's state, transposed, as accumulators of mma.sync (16 x D): what is an accumulator of one
// product is, element for element, the first factor of the next, so nothing leaves the registers between the products and the
// warps of a CTA (W of them, 16 W columns of one head) only share the operands that they read.  Chunks are fetched one ahead.
template <class T, int D, int W>
__global__ void __launch_bounds__(W * 32) kv_delta_chain_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    constexpr int C = kChunkRows, P = D / 8, VP = W * 2, NT = D / 8, CT = C / 8;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    using St = Stage<D, W>;
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    constexpr uint32_t kSlices = D / (16 * W);
    const uint32_t slice = blockIdx.x % kSlices, h = blockIdx.x / kSlices % a.n_heads, s = blockIdx.x / kSlices / a.n_heads, kh = h / a.group;
    const uint32_t col0 = slice * W * 16;  // of the CTA
    ptx::grid_launch_dependents();
    ptx::grid_wait();
    const int rows = delta_rows(a, s), first = delta_begin(a, s);
    if (!delta_in_chunks(a, rows)) return;
    const bool fresh = a.past_lens && a.past_lens[s] <= 0;
    const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
    float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
    if (a.status && tid == 0 && ((!fresh && !from) || !to)) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
    const uint32_t g = lane / 4, t2 = 2 * (lane & 3u);  // rows g and g + 8, columns 8 nt + t2 + {0, 1} of an accumulator
    const uint32_t v0 = col0 + 16 * warp + g;
    float S[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[nt][e] = from ? from[(uint64_t)(8 * nt + t2 + (e & 1)) * D + v0 + (e & 2) * 4] : 0.f;
    const int chunks = (rows + C - 1) / C;
    const uint32_t slot = delta_slot(a, s);
    auto fetch = [&](int chunk) {
        St &st = *reinterpret_cast<St *>(raw + (chunk & 1) * sizeof(St));
        const int r0 = chunk * C;
        for (uint32_t i = tid; i < (uint32_t)(C * P); i += W * 32) {
            const uint32_t r = i / P, c = i % P;
            const bool real = r0 + (int)r < rows;
            const uint64_t row = (uint64_t)(first + (real ? r0 + (int)r : 0));
            cp16(smem_u32(st.k) + piece<P>(r, c), a.k + row * a.k_token + kh * a.k_head + c * 16, real);
            cp16(smem_u32(st.q) + piece<P>(r, c), a.q + row * a.q_token + kh * a.q_head + c * 16, real);
        }
        for (uint32_t i = tid; i < (uint32_t)(C * VP); i += W * 32) {
            const uint32_t r = i / VP, c = i % VP;
            const bool real = r0 + (int)r < rows;
            const uint64_t row = (uint64_t)(first + (real ? r0 + (int)r : 0));
            cp16(smem_u32(st.v) + piece<VP>(r, c), a.v + row * a.v_token + h * a.v_head + col0 * 2 + c * 16, real);
        }
        const uint8_t *ws = a.chunks + ((uint64_t)(slot + chunk) * a.n_heads + h) * sizeof(ChunkWork);
        for (uint32_t i = tid; i < sizeof(ChunkWork) / 16; i += W * 32) cp16(smem_u32(&st.w) + i * 16, ws + i * 16, true);
        cp_commit();
    };
    if (chunks) fetch(0);
    for (int chunk = 0; chunk < chunks; ++chunk) {
        cp_wait();
        __syncthreads();  // the chunk is here, and nobody reads the stage of the last one any more
        if (chunk + 1 < chunks) fetch(chunk + 1);
        St &st = *reinterpret_cast<St *>(raw + (chunk & 1) * sizeof(St));
        const int n = min(rows - chunk * C, C);
        T *out = reinterpret_cast<T *>(a.out + (uint64_t)(first + chunk * C) * a.o_token + h * a.o_head);
        // the columns' values, transposed like everything else
        uint32_t V[CT][2];
        uint32_t odd = 0;
        constexpr uint32_t kOnes = kHalf ? 0x7c00u : 0x7f80u;
#pragma unroll
        for (int nt = 0; nt < CT; nt += 2) {
            uint32_t b[4];
            ldmatrix_x4_trans(smem_u32(st.v) + piece<VP>(8 * nt + (lane & 7u) + (lane & 16u) / 2, 2 * warp + (lane / 8 & 1u)), b);
            V[nt][0] = b[0], V[nt][1] = b[1], V[nt + 1][0] = b[2], V[nt + 1][1] = b[3];
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= ((b[e] & kOnes) == kOnes) | ((b[e] >> 16 & kOnes) == kOnes);
        }
        if (st.w.by_row || __any_sync(0xffffffffu, odd)) {
            // row by row: something here is not finite, and in a product it would reach rows that come before it
            for (int r = 0; r < n; ++r) {
                const float gate = st.w.gate[r], beta = st.w.beta[r], rk = st.w.rk[r], rq = st.w.rq[r];
                float x[2] = {}, y[2] = {}, z = 0.f, kv[2 * NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const T *kp = reinterpret_cast<const T *>(st.k + piece<P>(r, nt)) + t2, *qp = reinterpret_cast<const T *>(st.q + piece<P>(r, nt)) + t2;
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
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t c = 16 * warp + g + 8 * e;
                    const float v = to_f32(*reinterpret_cast<const T *>(st.v + piece<VP>(r, c / 8) + (c & 7u) * 2));
                    const float d = beta * (v - x[e]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) S[nt][2 * e] += kv[2 * nt] * d, S[nt][2 * e + 1] += kv[2 * nt + 1] * d;
                    if ((lane & 3u) == 0) {
                        T *op = reinterpret_cast<T *>(reinterpret_cast<uint8_t *>(out) + (uint64_t)r * a.o_token);
                        op[col0 + c] = from_f32<T>(a.scale * (y[e] + z * d));
                    }
                }
            }
            continue;
        }
        // f16: each of the warp's columns is scaled by a power of two of its own
        float su[2] = {1.f, 1.f}, si[2] = {1.f, 1.f};
        if (kHalf) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = 0.f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) top = fmaxf(top, fmaxf(fabsf(S[nt][2 * e]), fabsf(S[nt][2 * e + 1])));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                su[e] = range_scale(top), si[e] = 1.f / su[e];
            }
        }
        // X = S K^T (S in two terms), Y = S Q^T (one term: it goes into `out` alone)
        float X[CT][4] = {}, Y[CT][4] = {};
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) {
            uint32_t hi[4], lo[4];
            split2<T>(S[2 * kt][0] * su[0], S[2 * kt][1] * su[0], hi[0], lo[0]);
            split2<T>(S[2 * kt][2] * su[1], S[2 * kt][3] * su[1], hi[1], lo[1]);
            split2<T>(S[2 * kt + 1][0] * su[0], S[2 * kt + 1][1] * su[0], hi[2], lo[2]);
            split2<T>(S[2 * kt + 1][2] * su[1], S[2 * kt + 1][3] * su[1], hi[3], lo[3]);
            uint32_t b[CT][2];
#pragma unroll
            for (int nt = 0; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.k) + piece<P>(8 * nt + (lane & 7u) + (lane & 16u) / 2, 2 * kt + (lane / 8 & 1u)), x);
                b[nt][0] = x[0], b[nt][1] = x[1], b[nt + 1][0] = x[2], b[nt + 1][1] = x[3];
            }
#pragma unroll
            for (int nt = 0; nt < CT; ++nt) mma16816(X[nt], hi, b[nt][0], b[nt][1], T());
#pragma unroll
            for (int nt = 0; nt < CT; ++nt) mma16816(X[nt], lo, b[nt][0], b[nt][1], T());
#pragma unroll
            for (int nt = 0; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.q) + piece<P>(8 * nt + (lane & 7u) + (lane & 16u) / 2, 2 * kt + (lane / 8 & 1u)), x);
                mma16816(Y[nt], hi, x[0], x[1], T());
                mma16816(Y[nt + 1], hi, x[2], x[3], T());
            }
        }
        // what the values differ by from what the state says: X <- V - f X
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.f[8 * nt + t2]);
            const T *va = reinterpret_cast<const T *>(&V[nt][0]), *vb = reinterpret_cast<const T *>(&V[nt][1]);
            X[nt][0] = to_f32(va[0]) - f.x * (X[nt][0] * si[0]);
            X[nt][1] = to_f32(va[1]) - f.y * (X[nt][1] * si[0]);
            X[nt][2] = to_f32(vb[0]) - f.x * (X[nt][2] * si[1]);
            X[nt][3] = to_f32(vb[1]) - f.y * (X[nt][3] * si[1]);
        }
        float xu[2] = {1.f, 1.f}, xi[2] = {1.f, 1.f};
        if (kHalf) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = 0.f;
#pragma unroll
                for (int nt = 0; nt < CT; ++nt) top = fmaxf(top, fmaxf(fabsf(X[nt][2 * e]), fabsf(X[nt][2 * e + 1])));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                xu[e] = range_scale(top), xi[e] = st.w.t_unit / xu[e];
            }
        }
        // d = X T^T: two terms each (the product of the small ones left out); T's columns beyond a row's own are zero
        float d[CT][4] = {};
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            uint32_t hi[4], lo[4];
            split2<T>(X[2 * kt][0] * xu[0], X[2 * kt][1] * xu[0], hi[0], lo[0]);
            split2<T>(X[2 * kt][2] * xu[1], X[2 * kt][3] * xu[1], hi[1], lo[1]);
            split2<T>(X[2 * kt + 1][0] * xu[0], X[2 * kt + 1][1] * xu[0], hi[2], lo[2]);
            split2<T>(X[2 * kt + 1][2] * xu[1], X[2 * kt + 1][3] * xu[1], hi[3], lo[3]);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; nt += 2) {
                const uint32_t at = piece<8>(8 * nt + (lane & 7u) + (lane & 16u) / 2, 2 * kt + (lane / 8 & 1u));
                uint32_t x[4], y[4];
                ldmatrix_x4(smem_u32(st.w.tile[0]) + at, x);
                ldmatrix_x4(smem_u32(st.w.tile[1]) + at, y);
                mma16816(d[nt], hi, x[0], x[1], T());
                mma16816(d[nt + 1], hi, x[2], x[3], T());
                mma16816(d[nt], lo, x[0], x[1], T());
                mma16816(d[nt + 1], lo, x[2], x[3], T());
                mma16816(d[nt], hi, y[0], y[1], T());
                mma16816(d[nt + 1], hi, y[2], y[3], T());
            }
        }
        float du[2] = {1.f, 1.f}, di[2] = {1.f, 1.f};
        if (kHalf) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = 0.f;
#pragma unroll
                for (int nt = 0; nt < CT; ++nt) {
                    d[nt][2 * e] *= xi[e], d[nt][2 * e + 1] *= xi[e];
                    top = fmaxf(top, fmaxf(fabsf(d[nt][2 * e]), fabsf(d[nt][2 * e + 1])));
                }
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                du[e] = range_scale(top), di[e] = st.w.p_unit / du[e];
            }
        }
        // out = h Y + P d (one term each)
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.h[8 * nt + t2]);
            // (f16: in units of P and d)
            const float u0 = kHalf ? si[0] / di[0] : 1.f, u1 = kHalf ? si[1] / di[1] : 1.f;
            Y[nt][0] *= f.x * u0, Y[nt][1] *= f.y * u0, Y[nt][2] *= f.x * u1, Y[nt][3] *= f.y * u1;
        }
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            const uint32_t x[4] = {pack2(d[2 * kt][0] * du[0], d[2 * kt][1] * du[0], T()), pack2(d[2 * kt][2] * du[1], d[2 * kt][3] * du[1], T()),
                                   pack2(d[2 * kt + 1][0] * du[0], d[2 * kt + 1][1] * du[0], T()),
                                   pack2(d[2 * kt + 1][2] * du[1], d[2 * kt + 1][3] * du[1], T())};
#pragma unroll
            for (int nt = 2 * kt; nt < CT; nt += 2) {
                uint32_t b[4];
                ldmatrix_x4(smem_u32(st.w.tile[2]) + piece<8>(8 * nt + (lane & 7u) + (lane & 16u) / 2, 2 * kt + (lane / 8 & 1u)), b);
                mma16816(Y[nt], x, b[0], b[1], T());
                mma16816(Y[nt + 1], x, b[2], b[3], T());
            }
        }
        // S <- e^G S + (w d) K, w d in two terms (f16: S in units of the terms' scale meanwhile)
        const float all = st.w.all;
        float dw[2] = {1.f, 1.f};
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.w[8 * nt + t2]);
            d[nt][0] *= f.x, d[nt][1] *= f.y, d[nt][2] *= f.x, d[nt][3] *= f.y;
        }
        if (kHalf) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float top = 0.f;
#pragma unroll
                for (int nt = 0; nt < CT; ++nt) top = fmaxf(top, fmaxf(fabsf(d[nt][2 * e]), fabsf(d[nt][2 * e + 1])));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                dw[e] = range_scale(top);
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) S[nt][0] *= all * dw[0], S[nt][1] *= all * dw[0], S[nt][2] *= all * dw[1], S[nt][3] *= all * dw[1];
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            uint32_t hi[4], lo[4];
            split2<T>(d[2 * kt][0] * dw[0], d[2 * kt][1] * dw[0], hi[0], lo[0]);
            split2<T>(d[2 * kt][2] * dw[1], d[2 * kt][3] * dw[1], hi[1], lo[1]);
            split2<T>(d[2 * kt + 1][0] * dw[0], d[2 * kt + 1][1] * dw[0], hi[2], lo[2]);
            split2<T>(d[2 * kt + 1][2] * dw[1], d[2 * kt + 1][3] * dw[1], hi[3], lo[3]);
#pragma unroll
            for (int nt = 0; nt < NT; nt += 4) {
                uint32_t x[4], y[4];
                ldmatrix_x4_trans(smem_u32(st.k) + piece<P>(16 * kt + (lane & 15u), nt + lane / 16), x);
                ldmatrix_x4_trans(smem_u32(st.k) + piece<P>(16 * kt + (lane & 15u), nt + 2 + lane / 16), y);
                mma16816(S[nt], hi, x[0], x[1], T());
                mma16816(S[nt + 1], hi, x[2], x[3], T());
                mma16816(S[nt + 2], hi, y[0], y[1], T());
                mma16816(S[nt + 3], hi, y[2], y[3], T());
                mma16816(S[nt], lo, x[0], x[1], T());
                mma16816(S[nt + 1], lo, x[2], x[3], T());
                mma16816(S[nt + 2], lo, y[0], y[1], T());
                mma16816(S[nt + 3], lo, y[2], y[3], T());
            }
        }
        if (kHalf) {
            const float u0 = 1.f / dw[0], u1 = 1.f / dw[1];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) S[nt][0] *= u0, S[nt][1] *= u0, S[nt][2] *= u1, S[nt][3] *= u1;
        }
        // rows of 16 columns through the warp's own part of V's tile (its columns have been read)
        __syncwarp();
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const uint32_t lo = pack2(Y[nt][0] * di[0], Y[nt][1] * di[0], T()), hi = pack2(Y[nt][2] * di[1], Y[nt][3] * di[1], T());
            const uint32_t at = smem_u32(st.v) + piece<VP>(8 * nt + (lane & 7u), 2 * warp + (lane / 8 & 1u));
            asm volatile("stmatrix.sync.aligned.m8n8.x2.trans.shared.b16 [%0], {%1, %2};" ::"r"(at), "r"(lo), "r"(hi) : "memory");
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < C / 16; ++i) {
            const int r = 16 * i + (int)lane / 2;
            const uint4 x = *reinterpret_cast<const uint4 *>(st.v + piece<VP>(r, 2 * warp + (lane & 1u)));
            if (r < n)
                *reinterpret_cast<uint4 *>(reinterpret_cast<uint8_t *>(out) + (uint64_t)r * a.o_token + (col0 + 16 * warp) * 2 + (lane & 1u) * 16) = x;
        }
    }
    if (!to) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[(uint64_t)(8 * nt + t2 + (e & 1)) * D + v0 + (e & 2) * 4] = S[nt][e];
}

template <class T, int D>
cudaError_t launch(const DeltaArgs &a, cudaStream_t s)
{
    constexpr int W = D == 128 ? 2 : 2;
    static std::atomic<uint64_t> done[2];
    cudaError_t e = allow_smem(kv_delta_prep_kernel<T, D>, sizeof(PrepSmem<D>), done[0]);
    if (e == cudaSuccess) e = allow_smem(kv_delta_chain_kernel<T, D, W>, 2 * sizeof(Stage<D, W>), done[1]);
    if (e == cudaSuccess)
        e = launch_dependent(kv_delta_prep_kernel<T, D>, a.n_slots * (a.n_heads / a.group), kPrepThreads, sizeof(PrepSmem<D>), s, a);
    if (e == cudaSuccess)
        e = launch_dependent(kv_delta_chain_kernel<T, D, W>, a.n_seq * a.n_heads * (D / (16 * W)), W * 32, 2 * sizeof(Stage<D, W>), s, a);
    return e;
}

}  // namespace

cudaError_t launch_delta_chunks(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    if (head_dim == 128) return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 128>(a, s) : launch<__half, 128>(a, s);
    return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 64>(a, s) : launch<__half, 64>(a, s);
}

}  // namespace gms
