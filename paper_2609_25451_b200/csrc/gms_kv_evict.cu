// Eviction from the paged KV pool: which tokens stay, and moving them together.
#include "gms_internal.h"
#include "gms_kv_attn.h"

namespace gms {
namespace {

constexpr uint32_t kSelThreads = 512, kSelWarps = kSelThreads / 32, kBins = 2048, kHeldKeys = 9984;  // with the histogram within 48 KB

// Order-preserving integer of a weight: NaN below everything, -0 equal to +0.
__device__ __forceinline__ uint32_t weight_key(float w)
{
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// Sum over the threads before this one; `sh` has a word a warp and is free again after the caller's next barrier.
__device__ __forceinline__ uint32_t block_before(uint32_t x, uint32_t *sh, uint32_t *all)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    uint32_t inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= (uint32_t)o) inc += y;
    }
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    uint32_t w = lane < kSelWarps ? sh[lane] : 0;
#pragma unroll
    for (int o = 1; o < (int)kSelWarps; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= (uint32_t)o) w += y;
    }
    *all = __shfl_sync(0xffffffffu, w, kSelWarps - 1);
    const uint32_t warps = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
    return inc - x + (warp ? warps : 0);
}

// One CTA per (layer, sequence, KV head).  The weight that separates what stays from what goes is found in three passes from
// the top (11, 11 and 10 bits of an order-preserving integer, a histogram each); then one pass in token order, four tokens a
// thread, writes the kept positions.  The keys are held in shared memory (HELD: rows of up to 9,984 tokens; longer rows are
// read again, from L2 mostly).  Latency counts: a row is a few thousand words, and one sequence has few rows (601 tokens, 8 rows:
// 8 us; with four 8-bit passes and one thread searching the bins 20 us).
template <bool HELD>
__global__ void __launch_bounds__(kSelThreads) kv_evict_select_kernel(const __grid_constant__ EvictArgs a)
{
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[kBins], wsum[2][kSelWarps], sh[2];
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    const uint32_t c = row % a.n_kv, s = row / a.n_kv % a.n_seq, l = row / a.n_kv / a.n_seq;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t n = (uint32_t)min(max(a.lens[s], 0), (int)a.max_len), keep = min(n, a.budget);
    const float *w = a.weights + l * a.w_layer_stride + s * a.w_seq_stride + c * a.w_head_stride;
    float *wo = a.weights_out ? a.weights_out + l * a.o_layer_stride + s * a.o_seq_stride + c * a.o_head_stride : nullptr;
    int32_t *kept = a.kept + (uint64_t)row * a.budget;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // lens_out may be lens itself: the other CTAs of the sequence read it here, so the next kernel writes it.  Without one
    // (budget or max_len 0) keep is 0 whatever they read.
    if (min(a.max_len, a.budget) == 0 && l == 0 && c == 0 && tid == 0 && a.lens_out) a.lens_out[s] = 0;
    const uint32_t lo = a.sinks, hi = n > keep ? n - a.recent : 0;  // the tokens that compete (n > keep only)
    uint32_t limit = 0xffffffffu, take = 0;                        // kept: key > limit, and the first `take` equal to it
    auto key = [&](uint32_t t) { return HELD ? keys[t - lo] : weight_key(w[t]); };
    if (n > keep && keep > a.sinks + a.recent) {
        uint32_t want = keep - a.sinks - a.recent, prefix = 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
#pragma unroll
            for (uint32_t i = 0; i < kBins / kSelThreads; ++i) hist[i * kSelThreads + tid] = 0;
            __syncthreads();
            for (uint32_t t = lo + tid; t < hi; t += kSelThreads) {
                uint32_t k;
                if (HELD && pass == 0) keys[t - lo] = k = weight_key(w[t]);
                else k = key(t);
                if (pass == 0 || (k >> (shift + bits)) == (prefix >> (shift + bits))) atomicAdd(&hist[(k >> shift) & ((1u << bits) - 1u)], 1u);
            }
            __syncthreads();
            uint32_t mine = 0, all, top = kBins - 1 - tid * 4;  // bins from the top, four a thread (empty ones above 2^bits)
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) mine += hist[top - i];
            uint32_t before = block_before(mine, wsum[0], &all);
            if (before < want && want <= before + mine) {
                while (before + hist[top] < want) before += hist[top--];
                sh[0] = top;
                sh[1] = want - before;
            }
            __syncthreads();
            prefix |= sh[0] << shift;
            want = sh[1];
        }
        limit = prefix;
        take = want;
    }
    uint32_t above = 0, equal = 0, turn = 0;  // kept for sure / equal to the limit, before this run of tokens
    for (uint32_t t0 = 0; t0 < n; t0 += kSelThreads * 4, turn ^= 1) {
        uint32_t kind = 0, count = 0;  // two bits a token: 1 above, 2 equal; above in the low half, equal in the high half
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t t = t0 + tid * 4 + i;
            if (t >= n) continue;
            uint32_t is = 1;
            if (n > keep && t >= lo && t < hi) {
                // limit 0xffffffff: nothing between sinks and recent stays
                const uint32_t k = limit == 0xffffffffu ? 0u : key(t);
                is = k > limit ? 1u : k == limit ? 2u : 0u;
            }
            kind |= is << (2 * i);
            count += is == 1 ? 1u : is == 2 ? 0x10000u : 0u;
        }
        uint32_t all;
        const uint32_t before = block_before(count, wsum[turn], &all);
        uint32_t ab = above + (before & 0xffffu), eq = equal + (before >> 16);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t is = kind >> (2 * i) & 3u, t = t0 + tid * 4 + i;
            if (is == 1 || (is == 2 && eq < take)) {
                const uint32_t pos = ab + min(eq, take);
                kept[pos] = (int32_t)t;
                if (wo) wo[pos] = w[t];
            }
            ab += is == 1;
            eq += is == 2;
        }
        above += all & 0xffffu;
        equal += all >> 16;
    }
    for (uint32_t j = keep + tid; j < a.budget; j += kSelThreads) kept[j] = -1;
}

// Copies the kept rows: a CTA moves 64 tokens of one (layer, sequence, KV head), 16 bytes a lane; every row is read once and
// written once, in whole 128- or 256-byte pieces.  Bound by memory: 4 sequences, 32 layers, 8 heads, 8k -> 2k tokens (2.15 GB):
// 325 us = 6.6 TB/s of the call's 371 us.
__global__ void __launch_bounds__(256) kv_evict_move_kernel(const __grid_constant__ EvictArgs a, uint32_t chunks)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t row = blockIdx.x / chunks, j0 = blockIdx.x % chunks * 64;
    const uint32_t c = row % a.n_kv, s = row / a.n_kv % a.n_seq, l = row / a.n_kv / a.n_seq;
    // whether this reads the length from before the call or the one that another CTA has just written over it, keep is the same
    const uint32_t keep = min((uint32_t)min(max(a.lens[s], 0), (int)a.max_len), a.budget);
    if (l == 0 && c == 0 && j0 == 0 && threadIdx.x == 0 && a.lens_out) a.lens_out[s] = (int32_t)keep;
    const uint32_t per_row = a.row_bytes / 16, part = threadIdx.x % per_row, mask = (1u << a.block_shift) - 1u;
    const int32_t *kept = a.kept + (uint64_t)row * a.budget;
    uint8_t *kp = a.base + (uint64_t)(a.k_plane + l * a.layer_planes) * a.plane_stride;
    uint8_t *vp = a.base + (uint64_t)(a.v_plane + l * a.layer_planes) * a.plane_stride;
    for (uint32_t j = j0 + threadIdx.x / per_row; j < min(j0 + 64, keep); j += 256 / per_row) {
        const uint32_t t = (uint32_t)kept[j];
        const int from = a.src_table[s * a.src_stride + (t >> a.block_shift)], to = a.dst_table[s * a.dst_stride + (j >> a.block_shift)];
        if ((uint32_t)from >= a.n_blocks || (uint32_t)to >= a.n_blocks) {
            if (a.status && part == 0) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
            continue;
        }
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
    const bool held = a.max_len <= kHeldKeys;
    const cudaError_t e = held ? launch_dependent(kv_evict_select_kernel<true>, rows, kSelThreads, min(a.max_len, kHeldKeys) * 4, s, a)
                               : launch_dependent(kv_evict_select_kernel<false>, rows, kSelThreads, 0, s, a);
    if (e != cudaSuccess || chunks == 0) return e;
    return launch_dependent(kv_evict_move_kernel, rows * chunks, 256, 0, s, a, chunks);
}

}  // namespace gms
