// Internal declarations of the gated delta rule's kernels.
#pragma once
#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_ptx.h"

namespace gms {

struct DeltaArgs {
    const uint8_t *q, *k, *v;
    uint8_t *out;
    const float *g, *beta;
    const int32_t *cu_q, *past_lens, *src_table, *dst_table;
    uint8_t *plane;
    unsigned long long *status;
    uint64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head, g_stride, beta_stride, src_stride, dst_stride, block_stride;
    uint32_t n_blocks, per_block;        // states a block holds
    uint32_t n_seq, n_heads, group;      // group = n_heads / n_key_heads
    uint32_t total_q, max_q, unit_qk;
    float unit_eps, scale;
    uint8_t *chunks;                     // workspace: ChunkWork [n_slots][n_heads]; null: no sequence is done in chunks
    uint32_t n_slots, by_begin;
    uint32_t *order;                     // workspace: the sequences done in chunks, longest first, then kNone
};

// Sequences of more rows than kMostByRow are done kChunkRows at a time (us, in chunks / row by row, 32 heads of 128, bf16: 1 sequence of
// 20 rows 21.5 / 20.5, of 24 21.5 / 22.5; 8 of 16 46 / 34, of 20 47 / 40, of 24 47 / 44, of 32 48 / 55; 32 of 20 128 / 117, of 24 129 / 131; 44 of
// 9 to 51 rows, 24 heads, in chunks from 21 rows on 138, from 25 on 157).
constexpr uint32_t kChunkRows = 64, kMostByRow = 20, kNone = 0xffffffffu;

// What the first of the two chunk kernels leaves for the second.
struct alignas(256) ChunkWork {
    uint8_t tile[4][10 * 512];  // T, P, two bf16 terms each: blocks of 16 x 16 in and below the diagonal, laid out as `block_piece` says
    float f[kChunkRows], w[kChunkRows], h[kChunkRows];
    float gate[kChunkRows], beta[kChunkRows], rk[kChunkRows], rq[kChunkRows];  // for chunks that are done row by row
    float all;                                     // e^G of the chunk
    uint32_t by_row;
};

// What comes before the states' chain, for all chunks at once; the chain.
cudaError_t launch_delta_prep(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s);
cudaError_t launch_delta_chain(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s);

#ifdef __CUDACC__
__device__ __forceinline__ int delta_begin(const DeltaArgs &a, uint32_t s) { return a.cu_q ? min(max(a.cu_q[s], 0), (int)a.total_q) : (int)s; }
__device__ __forceinline__ int delta_rows(const DeltaArgs &a, uint32_t s)
{
    if (!a.cu_q) return 1;
    return min(max(min(a.cu_q[s + 1], (int)a.total_q) - delta_begin(a, s), 0), (int)a.max_q);
}
__device__ __forceinline__ bool delta_in_chunks(const DeltaArgs &a, int rows) { return a.chunks && rows > (int)kMostByRow; }
// First slot of a sequence in the workspace.  A sequence of n rows has n / 64 + 1 slots at least, whatever comes before it; or, where
// many are short, n / 21 if it is done in chunks (no fewer than its chunks, and sequences that are not may have none).
__device__ __forceinline__ uint32_t delta_slot(const DeltaArgs &a, uint32_t s)
{
    const uint32_t begin = (uint32_t)delta_begin(a, s);
    return a.by_begin ? begin / (kMostByRow + 1) : begin / kChunkRows + s;
}
// Where a head's state lies; null: in a hole.
template <int D>
__device__ __forceinline__ float *delta_state(const DeltaArgs &a, const int32_t *table, uint64_t stride, uint32_t s, uint32_t h)
{
    const int id = table[s * stride + h / a.per_block];
    if ((uint32_t)id >= a.n_blocks) return nullptr;
    return reinterpret_cast<float *>(a.plane + (uint64_t)id * a.block_stride) + (uint64_t)(h % a.per_block) * D * D;
}

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}

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
// 2^-30 .. 2^74.  (A state may have decayed far below what a later gate above 0 brings it back to.)
__device__ __forceinline__ float range_scale(float top)
{
    const int e = (int)(__float_as_uint(top) >> 23 & 255u) - 127;  // 2^e <= top
    return __uint_as_float((uint32_t)(127 + min(max(11 - e, -30), 74)) << 23);
}

// What the largest numbers are not scaled down to: differences from 2^41 on; states from 2^25 on, so that what part of one gives an
// output (terms below 2^12, queries below 2^16, 128 of each) may go over to another part's unit: 2^35 2^14 2^74 < 2^127.
__device__ __forceinline__ bool beyond_scale(float u) { return u <= 0x1p-30f; }
__device__ __forceinline__ bool state_beyond_scale(float u) { return u <= 0x1p-14f; }

// 1 / u for a power of two.
__device__ __forceinline__ float flipped(float u) { return __uint_as_float(0x7f000000u - __float_as_uint(u)); }
#endif

}  // namespace gms
