// Accumulated attention weights where the logits were not kept (many query rows): a second pass over the keys alone.
//
//   out[t] = decay * in[t] + sum over rows r that see t of 2^(c q_r.k_t - lse2_r)
//
// A CTA owns every so many 128-token chunk of one sequence and KV head: every warp keeps 32 tokens' keys in registers as matrix
// fragments and walks all query rows, 128 at a time through shared memory (S^T = K Q^T, so a token's sum stays in a quad of
// lanes); the next chunk's keys are on their way meanwhile, and up to 128 rows stay in shared memory for all chunks.  Each sum
// has one owner and one order: no atomics, equal calls give equal bits.  Bound by the exponentials and the matrix unit for
// many rows, by latency and reading K for few.  (32 queries over 16,001 tokens with their weights, 8 KV heads x 128 rows of 64:
// 57 us with one chunk a CTA, 53 us so; 919 us with one warp a token.)
#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_ptx.h"

namespace gms {
namespace {

using namespace ptx;

constexpr int kWarps = 4, kThreads = kWarps * 32, kTokens = kWarps * 32, kRows = kTokens;

template <class T, int D>
__global__ void __launch_bounds__(kThreads) kv_weights_kernel(const __grid_constant__ AttnArgs a, const float *lse, uint32_t parts,
                                                               uint32_t behind)
{
    if (!behind) grid_wait();  // else the attention kernels ahead have waited, and only their log-sum-exps are waited for below
    constexpr int kPieces = D / 8, kStride = D * 2 + 16;  // 16-byte pieces of a row; bytes between rows (no bank conflicts)
    constexpr int kLoads = kTokens * kPieces / kThreads;
    extern __shared__ __align__(16) uint8_t smem[];
    uint8_t *const k_sh = smem, *const q_sh = smem + kTokens * kStride;
    float *const lse_sh = reinterpret_cast<float *>(q_sh + kRows * kStride);
    int *const pos_sh = reinterpret_cast<int *>(lse_sh + kRows);
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    const uint32_t item = blockIdx.x / parts, c = item % a.n_kv, s = item / a.n_kv;
    const int n = seq_kv_len(a, s), q0 = seq_q_begin(a, s), q_len = seq_q_len(a, s), rows = q_len * (int)a.group, first = seq_first(a, s);
    const int32_t *const table = a.table + s * a.table_stride;
    const float c2 = a.scale * kLog2e;
    auto held = [&](int t) { return t < n && (uint32_t)table[(uint32_t)t >> a.block_shift] < a.n_blocks; };
    uint4 next[kLoads];
    auto fetch = [&](int t0) {  // tokens that nobody can see are zero
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = i * kThreads + (int)tid, t = t0 + x / kPieces;
            const int id = t < n ? table[(uint32_t)t >> a.block_shift] : -1;
            next[i] = make_uint4(0, 0, 0, 0);
            if ((uint32_t)id < a.n_blocks)
                next[i] = *reinterpret_cast<const uint4 *>(a.k_base + (uint64_t)id * a.block_stride +
                                                           (uint64_t)((uint32_t)t & ((1u << a.block_shift) - 1u)) * a.token_stride +
                                                           (uint64_t)c * a.head_stride + x % kPieces * 16);
        }
    };
    bool ready = false;  // the queries (when they fit) are in shared memory
    int t0 = (int)(blockIdx.x % parts) * kTokens;
    if (t0 < n) fetch(t0);
    grid_wait();  // the log-sum-exps are there
#pragma unroll 1
    for (; t0 < n; t0 += (int)parts * kTokens) {
        __syncthreads();  // the last chunk's keys have been read
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int x = i * kThreads + (int)tid;
            *reinterpret_cast<uint4 *>(k_sh + x / kPieces * kStride + x % kPieces * 16) = next[i];
        }
        __syncthreads();
        // keys of tokens base + lane/4 + 8 i, i < 4, as two 16-row fragments
        const int base = t0 + (int)warp * 32 + (int)lane / 4;
        uint32_t k[2][D / 16][4];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
                ldmatrix_x4(smem_u32(k_sh) + (warp * 32 + m * 16 + (lane & 15u)) * kStride + (kk * 2 + (lane >> 4)) * 16, k[m][kk]);
        uint32_t seen = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) seen |= held(base + 8 * i) ? 1u << i : 0u;
        if (t0 + (int)parts * kTokens < n) fetch(t0 + (int)parts * kTokens);
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
        const int t_last = min(t0 + kTokens, n) - 1;
        for (int r0 = 0; r0 < rows; r0 += kRows) {
            const int here = min(kRows, rows - r0), p_min = first + r0 / (int)a.group, p_max = first + (r0 + here - 1) / (int)a.group;
            if (p_max < t0) continue;  // all of these rows come before all of these tokens
            if (a.window && p_min >= 0 && (uint32_t)p_min >= a.window && t_last <= p_min - (int)a.window && (uint32_t)t0 >= a.sinks) continue;
            if (!ready) {
                __syncthreads();
#pragma unroll 8
                for (int i = 0; i < kRows * kPieces / kThreads; ++i) {
                    const int x = i * kThreads + (int)tid, r = x / kPieces, ch = x % kPieces, row = r0 + r;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (r < here)
                        v = *reinterpret_cast<const uint4 *>(a.q + (uint64_t)(q0 + row / (int)a.group) * a.q_token_stride +
                                                             (uint64_t)(c * a.group + (uint32_t)row % a.group) * a.q_head_stride + ch * 16);
                    *reinterpret_cast<uint4 *>(q_sh + r * kStride + ch * 16) = v;
                }
                if (tid < kRows) {
                    const int row = r0 + (int)tid;
                    float x = __int_as_float(0x7f800000);  // rows that do not exist or see nothing: weight 0
                    if ((int)tid < here) x = lse[(uint64_t)(q0 + row / (int)a.group) * a.n_heads + c * a.group + (uint32_t)row % a.group] * kLog2e;
                    lse_sh[tid] = x == neg_inf() ? -x : x;
                    pos_sh[tid] = first + row / (int)a.group;
                }
                __syncthreads();
                ready = rows <= kRows;
            }
            const bool whole = t_last <= p_min && seen == 15u &&
                               (a.window == 0 || p_max < 0 || (uint32_t)p_max < a.window || t0 > p_max - (int)a.window || (uint32_t)t_last < a.sinks);
            const bool all_whole = __all_sync(0xffffffffu, whole);
            for (int j = 0; j < here; j += 8) {
                float acc[2][4];
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[m][e] = 0.f;
#pragma unroll
                for (int kk = 0; kk < D / 16; kk += 2) {
                    uint32_t b[4];
                    ldmatrix_x4(smem_u32(q_sh) + (j + (lane & 7u)) * kStride + (kk * 2 + (lane >> 3)) * 16, b);
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        mma16816(acc[m], k[m][kk], b[0], b[1], T());
                        mma16816(acc[m], k[m][kk + 1], b[2], b[3], T());
                    }
                }
                const int r = j + (int)(lane & 3u) * 2;
                const float l0 = lse_sh[r], l1 = lse_sh[r + 1];
                // the rows that fill up the last eight go the masked way: their zeros times a key that holds an infinity are NaN
                if (all_whole && j + 8 <= here) {
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        sum[2 * m] += ex2(fmaf(acc[m][0], c2, -l0)) + ex2(fmaf(acc[m][1], c2, -l1));
                        sum[2 * m + 1] += ex2(fmaf(acc[m][2], c2, -l0)) + ex2(fmaf(acc[m][3], c2, -l1));
                    }
                } else {
                    const int p0 = pos_sh[r], p1 = pos_sh[r + 1];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = base + 8 * i;
                        if (!(seen >> i & 1u)) continue;
                        if (r < here && sees(a, p0, t)) sum[i] += ex2(fmaf(acc[i / 2][(i % 2) * 2], c2, -l0));
                        if (r + 1 < here && sees(a, p1, t)) sum[i] += ex2(fmaf(acc[i / 2][(i % 2) * 2 + 1], c2, -l1));
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
            sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
            const int t = base + 8 * i;
            if ((lane & 3u) == (uint32_t)i && t < n) {
                const uint64_t at = s * a.w_seq_stride + c * a.w_head_stride + t;
                a.w_out[at] = (a.w_in ? a.decay * a.w_in[at] : 0.f) + sum[i];
            }
        }
    }
}

template <class T, int D>
cudaError_t launch(const AttnArgs &a, const float *lse, uint64_t grid, uint32_t parts, uint32_t behind, cudaStream_t s)
{
    constexpr uint32_t smem = (kTokens + kRows) * (D * 2 + 16) + kRows * 8;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(kv_weights_kernel<T, D>, smem, done);
    if (e != cudaSuccess) return e;
    return launch_dependent(kv_weights_kernel<T, D>, (uint32_t)grid, kThreads, smem, s, a, lse, parts, behind);
}

}  // namespace

cudaError_t launch_kv_weights(const AttnArgs &a, const float *lse, bool behind, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    const uint64_t items = (uint64_t)a.n_seq * a.n_kv, chunks = (a.max_kv + kTokens - 1) / kTokens;
    if (items == 0 || chunks == 0) return cudaSuccess;
    // as many CTAs as the SMs hold at once (four an SM at dim 64, two at 128), each with equally many chunks of the longest row
    const uint64_t resident = 148 * (head_dim == 64 ? 4 : 2), rounds = (items * chunks + resident - 1) / resident;
    const uint32_t parts = (uint32_t)((chunks + rounds - 1) / rounds), behind_word = behind;
    if (dtype == GMS_DTYPE_BF16)
        return head_dim == 64 ? launch<__nv_bfloat16, 64>(a, lse, items * parts, parts, behind_word, s)
                              : launch<__nv_bfloat16, 128>(a, lse, items * parts, parts, behind_word, s);
    return head_dim == 64 ? launch<__half, 64>(a, lse, items * parts, parts, behind_word, s)
                          : launch<__half, 128>(a, lse, items * parts, parts, behind_word, s);
}

}  // namespace gms
