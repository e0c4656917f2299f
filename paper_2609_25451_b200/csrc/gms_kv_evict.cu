// Eviction from the paged KV pool: which tokens stay, and moving them together.
#include "gms_internal.h"
#include "gms_kv_attn.h"

namespace gms {
namespace {

constexpr uint32_t kSelThreads = 256;

// Order-preserving integer of a weight: NaN below everything, -0 equal to +0.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// One CTA per (layer, sequence, KV head).  The weight that separates what stays from what goes is found byte by byte
// from the top (four passes of a 256-bin histogram); then one pass in token order writes the kept positions.
__global__ void __launch_bounds__(kSelThreads) kv_evict_select_kernel(EvictArgs a)
{
    __shared__ uint32_t hist[256], wsum[kSelThreads / 32], sh[2];
    const uint32_t row = blockIdx.x, tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    const uint32_t c = row % a.n_kv, s = row / a.n_kv % a.n_seq, l = row / a.n_kv / a.n_seq;
    const uint32_t n = (uint32_t)min(max(a.lens[s], 0), (int)a.max_len), keep = min(n, a.budget);
    const float *w = a.weights + l * a.w_layer_stride + s * a.w_seq_stride + c * a.w_head_stride;
    float *wo = a.weights_out ? a.weights_out + l * a.o_layer_stride + s * a.o_seq_stride + c * a.o_head_stride : nullptr;
    int32_t *kept = a.kept + (uint64_t)row * a.budget;
    if (l == 0 && c == 0 && tid == 0 && a.lens_out) a.lens_out[s] = (int32_t)keep;
    const uint32_t lo = a.sinks, hi = n > keep ? n - a.recent : 0;  // the tokens that compete (n > keep only)
    uint32_t limit = 0xffffffffu, take = 0;                        // kept: key > limit, and the first `take` equal to it
    if (n > keep && keep > a.sinks + a.recent) {
        uint32_t want = keep - a.sinks - a.recent, prefix = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            hist[tid] = 0;
            __syncthreads();
            for (uint32_t t = lo + tid; t < hi; t += kSelThreads) {
                const uint32_t k = weight_key(w[t]);
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                uint32_t b = 255, left = want;
                while (hist[b] < left) left -= hist[b--];  // terminates: the bins hold at least `want` keys
                sh[0] = b;
                sh[1] = left;
            }
            __syncthreads();
            prefix |= sh[0] << shift;
            want = sh[1];
            __syncthreads();
        }
        limit = prefix;
        take = want;
    }
    uint32_t above = 0, equal = 0;  // kept for sure / equal to the limit, before this run of tokens
    for (uint32_t t0 = 0; t0 < n; t0 += kSelThreads) {
        const uint32_t t = t0 + tid;
        uint32_t is_above = 0, is_equal = 0;
        float x = 0.f;
        if (t < n) {
            x = w[t];
            if (n <= keep || t < lo || t >= hi) {
                is_above = 1;
            } else {
                const uint32_t k = weight_key(x);
                is_above = k > limit;
                is_equal = k == limit;
            }
        }
        const uint32_t ba = __ballot_sync(0xffffffffu, is_above), be = __ballot_sync(0xffffffffu, is_equal);
        if (lane == 0) wsum[warp] = __popc(ba) | __popc(be) << 16;
        __syncthreads();
        uint32_t before = 0, all = 0;
#pragma unroll
        for (uint32_t i = 0; i < kSelThreads / 32; ++i) {
            const uint32_t v = wsum[i];
            if (i < warp) before += v;
            all += v;
        }
        const uint32_t lt = (1u << lane) - 1u;
        const uint32_t eq = equal + (before >> 16) + __popc(be & lt), pos = above + (before & 0xffffu) + __popc(ba & lt) + min(eq, take);
        if (is_above || (is_equal && eq < take)) {
            kept[pos] = (int32_t)t;
            if (wo) wo[pos] = x;
        }
        above += all & 0xffffu;
        equal += all >> 16;
        __syncthreads();
    }
    for (uint32_t j = keep + tid; j < a.budget; j += kSelThreads) kept[j] = -1;
}

// Copies the kept rows: a CTA moves 64 tokens of one (layer, sequence, KV head), 16 bytes a lane.
__global__ void __launch_bounds__(256) kv_evict_move_kernel(EvictArgs a, uint32_t chunks)
{
    const uint32_t row = blockIdx.x / chunks, j0 = blockIdx.x % chunks * 64;
    const uint32_t c = row % a.n_kv, s = row / a.n_kv % a.n_seq, l = row / a.n_kv / a.n_seq;
    const uint32_t keep = min((uint32_t)min(max(a.lens[s], 0), (int)a.max_len), a.budget);
    const uint32_t per_row = a.row_bytes / 16, part = threadIdx.x % per_row, mask = (1u << a.block_shift) - 1u;
    const int32_t *kept = a.kept + (uint64_t)row * a.budget;
    uint8_t *kp = a.base + (uint64_t)(a.k_plane + l * a.layer_planes) * a.plane_stride;
    uint8_t *vp = a.base + (uint64_t)(a.v_plane + l * a.layer_planes) * a.plane_stride;
    for (uint32_t j = j0 + threadIdx.x / per_row; j < min(j0 + 64, keep); j += 256 / per_row) {
        const uint32_t t = (uint32_t)kept[j];
        const int from = a.src_table[s * a.src_stride + (t >> a.block_shift)], to = a.dst_table[s * a.dst_stride + (j >> a.block_shift)];
        if ((uint32_t)from >= a.n_blocks || (uint32_t)to >= a.n_blocks) continue;
        const uint64_t head = (uint64_t)c * a.head_stride + part * 16;
        const uint64_t so = (uint64_t)from * a.block_stride + (uint64_t)(t & mask) * a.token_stride + head;
        const uint64_t to_off = (uint64_t)to * a.block_stride + (uint64_t)(j & mask) * a.token_stride + head;
        const uint4 k = *reinterpret_cast<const uint4 *>(kp + so), v = *reinterpret_cast<const uint4 *>(vp + so);
        *reinterpret_cast<uint4 *>(kp + to_off) = k;
        *reinterpret_cast<uint4 *>(vp + to_off) = v;
    }
}

}  // namespace

cudaError_t launch_kv_evict(const EvictArgs &a, cudaStream_t s)
{
    const uint32_t rows = a.n_layers * a.n_seq * a.n_kv, chunks = (min(a.max_len, a.budget) + 63) / 64;
    kv_evict_select_kernel<<<rows, kSelThreads, 0, s>>>(a);
    count_launches(1);
    if (chunks) {
        kv_evict_move_kernel<<<rows * chunks, 256, 0, s>>>(a, chunks);
        count_launches(1);
    }
    return cudaGetLastError();
}

}  // namespace gms
