// Joining the pieces of attention items that were cut across workers, and the two passes of a shared-prefix call.
//
// Pieces carry a running maximum m (base 2), a sum l and unnormalised values o:  M = max m_i,  L = sum l_i 2^(m_i - M),
// out = sum o_i 2^(m_i - M) / L,  in the order of the pieces, so equal calls give equal bits.  One warp a row; the pieces
// are a few MB at most and still in L2.
#include <cmath>
#include <type_traits>

#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_ptx.h"

namespace gms {
namespace {

using namespace ptx;

constexpr uint32_t kWarps = 8, kLookers = 2 * 148;

// Adds pieces first, first + step, ... < n; piece i lies at slot(i) of ml and o.  Eight loads of o are in flight.
template <int D, class F>
__device__ __forceinline__ void add_pieces(Row<D> &x, const float2 *ml, const float *o, uint32_t first, uint32_t step, uint32_t n, F slot)
{
    using V = typename std::conditional<D == 128, float4, float2>::type;
    const uint32_t lane = threadIdx.x & 31u;
    for (uint32_t i0 = first; i0 < n; i0 += 32 * step) {
        const uint32_t me = i0 + lane * step;
        float2 mine = make_float2(neg_inf(), 0.f);
        if (me < n) mine = ml[slot(me)];
        float top = fmaxf(x.m, mine.x);
#pragma unroll
        for (int k = 16; k; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
        const float f = x.m == top ? 1.f : ex2(x.m - top), g = mine.x == top ? 1.f : ex2(mine.x - top);
        x.m = top;
        x.l = x.l * f + warp_sum(mine.y * g);
#pragma unroll
        for (int e = 0; e < D / 32; ++e) x.o[e] *= f;
        const uint32_t left = min(32u, (n - i0 + step - 1) / step);
        for (uint32_t b = 0; b < left; b += 8) {
            V v[8];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) v[j] = reinterpret_cast<const V *>(o + slot(i0 + min(b + j, left - 1) * step) * D)[lane];
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                const float gi = __shfl_sync(0xffffffffu, g, (b + j) & 31u), li = __shfl_sync(0xffffffffu, mine.y, (b + j) & 31u);
                if (b + j >= left || li == 0.f) continue;  // nothing seen there
                const float *vf = reinterpret_cast<const float *>(&v[j]);
#pragma unroll
                for (int e = 0; e < D / 32; ++e) x.o[e] += vf[e] * gi;
            }
        }
    }
}

// Rows of finished items that came out non-finite (a cut item's words are zero): a word has 32 rows, four for each warp, and
// neighbouring words go to different blocks of the first ones.  (With all blocks looking, each wave of them paid for a load from
// L2: windowed prompt 247 us, so 242.)  A lane's word in its block's turn.
__device__ __forceinline__ uint32_t redo_word(const AttnArgs &a, const Pass &p, uint32_t turn)
{
    const uint64_t w = blockIdx.x + ((uint64_t)turn * 32 + (threadIdx.x & 31u)) * min(gridDim.x, kLookers);
    return p.redo && blockIdx.x < kLookers && w < (uint64_t)p.n_units * a.n_kv * 8 ? p.redo[w] : 0u;
}
// What a warp does again: rows row, row + 8, ... of the cut item (KV head c) that are marked in `bad`, and its share of the rows
// that are marked in the block's words (`rows`: the first turn's).  Kept out of the join's own code, which is short of registers.
template <class T, int D, int ROWS, int TILE>
__device__ __noinline__ void redo(const AttnArgs &a, const Pass &p, int q0, int row, uint32_t c, uint32_t bad, uint32_t rows)
{
    __syncwarp();
    for (; bad; bad &= bad - 1) {
        const int r = row + (__ffs(bad) - 1) * (int)kWarps;
        attend_row<T, D>(a, q0 + r / (int)a.group, c * a.group + (uint32_t)r % a.group);
    }
    if (!p.redo || blockIdx.x >= kLookers) return;
    for (uint32_t turn = 0;; rows = redo_word(a, p, ++turn)) {
        const uint64_t lookers = min(gridDim.x, kLookers), first = blockIdx.x + turn * 32 * lookers;
        if (first >= (uint64_t)p.n_units * a.n_kv * 8) return;
        for (uint32_t some = __ballot_sync(0xffffffffu, rows != 0); some; some &= some - 1) {
            const uint64_t word = first + (__ffs(some) - 1) * lookers, item = word / 8;
            const uint32_t unit = (uint32_t)(item / a.n_kv);
            uint32_t left = __shfl_sync(0xffffffffu, rows, __ffs(some) - 1);
            const Unit u = get_unit<ROWS, TILE>(a, p, unit / p.n_rt, unit % p.n_rt);
            if (u.tiles == 0) continue;  // sees nothing: no words were written
            for (uint32_t k = 0; left; ++k, left &= left - 1) {
                if (k % kWarps != threadIdx.x / 32) continue;
                const int r = (int)(word % 8) * 32 + __ffs(left) - 1;
                attend_row<T, D>(a, unit_tok(a, u, r), unit_head(a, u, (uint32_t)(item % a.n_kv), r));
            }
        }
    }
}

// A block does `rows_a_block` rows (part `part` of them) of one cut item: of item i (by_item: fewer items than borders), or of
// the item into which the border before worker i + 1 falls, if that is its first border.  Also: rows of units that see
// nothing are zero, their log-sum-exps -infinity; and (AGAIN) rows to be done again are.
template <class T, int D, int ROWS, int TILE, bool AGAIN>
__global__ void __launch_bounds__(kWarps * 32, D == 64 ? 4 : 3) kv_attn_join_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Pass p,
                                                                                    uint32_t parts, uint32_t rows_a_block, uint32_t by_item)
{
    grid_launch_dependents();
    for (uint32_t x = blockIdx.x; x < p.n_units; x += gridDim.x) {  // while the attention kernel still runs
        const Unit u = get_unit<ROWS, TILE>(a, p, x / p.n_rt, x % p.n_rt);
        if (u.rows == 0 || u.tiles != 0) continue;
        for (uint32_t k = threadIdx.x; k < u.rows * a.n_kv; k += kWarps * 32) {
            const int r = k % u.rows;
            const uint32_t h = unit_head(a, u, k / u.rows, r);
            const uint64_t tok = unit_tok(a, u, r);
            uint4 *op = reinterpret_cast<uint4 *>(a.out + tok * a.out_token_stride + h * a.out_head_stride);
            for (int d = 0; d < D / 8; ++d) op[d] = make_uint4(0, 0, 0, 0);
            if (a.lse) a.lse[tok * a.n_heads + h] = neg_inf();
        }
    }
    grid_wait();
    const uint32_t i = blockIdx.x / parts, row_first = blockIdx.x % parts * rows_a_block, warp = threadIdx.x / 32, lane = threadIdx.x & 31u;
    const uint32_t rows = AGAIN ? redo_word(a, p, 0) : 0;  // on its way while the pieces are joined
    Cut x = {};
    uint32_t bad = 0;  // bit k: row warp + 8 k of the block came out non-finite
    __shared__ float m_sh[kWarps], l_sh[kWarps];
    __shared__ float o_sh[kWarps][D];
    auto done = [&](const Row<D> &sum, uint32_t r) {
        const int row = x.row0 + (int)(row_first + r);
        if (finish<T, D>(a, sum, x.q0 + row / (int)a.group, x.c * a.group + (uint32_t)row % a.group)) bad |= 1u << (r / kWarps);
    };
    auto join = [&] {
        if (by_item) {
            const uint32_t unit = i / a.n_kv, first_tile = p.begin[unit], all = p.begin[unit + 1] - first_tile, total = p.begin[p.n_units];
            if (all == 0) return;
            const uint32_t n = used_workers(total, p.workers), per = total / n, more = total - per * n, size = all / a.n_kv, extra = item_extra<TILE>();
            x.c = i % a.n_kv;
            x.c0 = tile_owner(first_tile + x.c * size + extra, per, more);
            x.c1 = tile_owner(first_tile + x.c * size + size - 1, per, more);
            if (x.c0 == x.c1) return;
            const Unit u = get_unit<ROWS, TILE>(a, p, unit / p.n_rt, unit % p.n_rt);
            x.q0 = u.q0, x.row0 = u.row0, x.rows = u.rows;
        } else {
            if (i + 1 >= p.workers) return;
            x = p.cuts[i + 1];
            if (x.c1 == 0 || x.c0 != i) return;  // the border lies between two items, or is not the item's first
        }
        // few rows: several warps share a row's pieces
        const uint32_t here = min((uint32_t)max(x.rows - (int)row_first, 0), rows_a_block);  // rows of this block
        const uint32_t share = here == 0 || here >= kWarps ? 1 : kWarps / here;
        if (share > 1) {
            Row<D> sum;
            const uint32_t r = warp % here, g = warp / here;
            if (g < share)
                add_pieces<D>(sum, p.part_ml, p.part_o, g, share, x.c1 - x.c0 + 1,
                              [&](uint32_t k) { return ((uint64_t)(x.c0 + k) * 2 + (k == 0)) * p.slot_rows + row_first + r; });
            if (lane == 0) m_sh[warp] = sum.m, l_sh[warp] = sum.l;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) o_sh[warp][lane * (D / 32) + e] = sum.o[e];
            __syncthreads();
            if (warp >= here) return;
            for (uint32_t k = 1; k < share; ++k) {
                const uint32_t other = warp + k * here;
                const float m2 = m_sh[other], top = fmaxf(sum.m, m2), f1 = sum.m == top ? 1.f : ex2(sum.m - top), f2 = m2 == top ? 1.f : ex2(m2 - top);
                sum.m = top;
                sum.l = sum.l * f1 + l_sh[other] * f2;
#pragma unroll
                for (int e = 0; e < D / 32; ++e) sum.o[e] = sum.o[e] * f1 + o_sh[other][lane * (D / 32) + e] * f2;
            }
            done(sum, warp);
            return;
        }
        for (uint32_t r = warp; r < here; r += kWarps) {
            Row<D> sum;
            add_pieces<D>(sum, p.part_ml, p.part_o, 0, 1, x.c1 - x.c0 + 1,
                          [&](uint32_t k) { return ((uint64_t)(x.c0 + k) * 2 + (k == 0)) * p.slot_rows + row_first + r; });
            done(sum, r);
        }
    };
    join();
    if (AGAIN) {
        const bool more = p.redo && blockIdx.x < kLookers && (uint64_t)p.n_units * a.n_kv * 8 > 32 * kLookers;  // turns to come
        if (more || __any_sync(0xffffffffu, bad | rows)) redo<T, D, ROWS, TILE>(a, p, x.q0, x.row0 + (int)(row_first + warp), x.c, bad, rows);
    }
}

// Adds what a pass has for one (query row, head); s: sequence, or group in the prefix pass.  False: the pass has left the row out
// (max_group_q).
template <int D, int ROWS, int TILE>
__device__ bool add_pass(const AttnArgs &a, const Pass &p, Row<D> &x, uint32_t s, int tok, uint32_t h)
{
    const uint64_t row = (uint64_t)tok * a.n_heads + h;
    const uint32_t c = h / a.group;
    Unit u = get_unit<ROWS, TILE>(a, p, s, 0);
    const uint32_t in = (uint32_t)(tok - u.q0) * a.group + h % a.group, rt = in / ROWS, r = in % ROWS;
    if (rt >= p.n_rt) return false;
    if (rt) u = get_unit<ROWS, TILE>(a, p, s, rt);
    if ((int)r >= u.rows) return false;
    if (u.tiles == 0) return true;
    if (p.team) {
        add_pieces<D>(x, p.row_ml, p.row_o, 0, 1, 1, [&](uint32_t) { return row; });
        return true;
    }
    const uint32_t total = p.begin[p.n_units], first = p.begin[s * p.n_rt + rt] + c * item_cost<TILE>(u.tiles) + item_extra<TILE>();
    const uint32_t n = used_workers(total, p.workers), per = total / n, more = total % n;
    const uint32_t c0 = tile_owner(first, per, more), c1 = tile_owner(first + u.tiles - 1, per, more);
    if (c0 == c1) add_pieces<D>(x, p.row_ml, p.row_o, 0, 1, 1, [&](uint32_t) { return row; });
    else
        add_pieces<D>(x, p.part_ml, p.part_o, 0, 1, c1 - c0 + 1, [&](uint32_t k) { return ((uint64_t)(c0 + k) * 2 + (k == 0)) * p.slot_rows + r; });
    return true;
}

template <class T, int D>
__global__ void __launch_bounds__(kWarps * 32) kv_attn_join_shared_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Pass pre,
                                                                          const __grid_constant__ Pass own)
{
    const uint64_t row = (uint64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    grid_wait();
    if (row >= (uint64_t)a.total_q * a.n_heads) return;
    const int tok = (int)(row / a.n_heads);
    const uint32_t h = (uint32_t)(row % a.n_heads), s = owner_of_row(a, tok);
    if (s >= a.n_seq) return;
    Row<D> x;
    const uint32_t g = group_of_seq(a, s);
    if (g < a.n_groups) {
        if (!(pre.rows == kTcRows ? add_pass<D, kTcRows, kTcTile>(a, pre, x, g, tok, h) : add_pass<D, kFewRows, kFewTile>(a, pre, x, g, tok, h)))
            return;
    }
    if (own.rows == kTcRows) add_pass<D, kTcRows, kTcTile>(a, own, x, s, tok, h);
    else add_pass<D, kFewRows, kFewTile>(a, own, x, s, tok, h);
    if (finish<T, D>(a, x, tok, h) && own.again) {
        __syncwarp();
        attend_row<T, D>(a, tok, h);
    }
}

}  // namespace

#define GMS_BY_TYPE(CALL)                                                               \
    do {                                                                                \
        if (dtype == GMS_DTYPE_BF16) {                                                  \
            using T = __nv_bfloat16;                                                    \
            if (head_dim == 64) { constexpr int D = 64; return CALL; }                  \
            constexpr int D = 128;                                                      \
            return CALL;                                                                \
        }                                                                               \
        using T = __half;                                                               \
        if (head_dim == 64) { constexpr int D = 64; return CALL; }                      \
        constexpr int D = 128;                                                          \
        return CALL;                                                                    \
    } while (0)

cudaError_t launch_kv_attn_join(const AttnArgs &a, const Pass &p, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    const uint32_t borders = p.workers < 2 ? 1 : p.workers - 1;
    const uint64_t items = (uint64_t)p.n_units * a.n_kv;
    const uint32_t by_item = items <= borders;
    // sixteen rows a block; fewer, their pieces spread over the warps, where few items are in many pieces each
    const uint32_t rows_a_block = !by_item || p.workers / items < 16 ? kFewRows : p.slot_rows <= kFewRows ? 1 : 4;
    const uint32_t parts = (p.slot_rows + rows_a_block - 1) / rows_a_block, grid = (by_item ? (uint32_t)items : borders) * parts;
#define GMS_JOIN(ROWS, TILE, AGAIN) \
    GMS_BY_TYPE((launch_dependent(kv_attn_join_kernel<T, D, ROWS, TILE, AGAIN>, grid, kWarps * 32, 0, s, a, p, parts, rows_a_block, by_item)))
    if (p.rows == kTcRows) {
        if (p.again) GMS_JOIN(kTcRows, kTcTile, true);
        GMS_JOIN(kTcRows, kTcTile, false);
    }
    if (p.again) GMS_JOIN(kFewRows, kFewTile, true);
    GMS_JOIN(kFewRows, kFewTile, false);
#undef GMS_JOIN
}

cudaError_t launch_kv_attn_join_shared(const AttnArgs &a, const Pass &pre, const Pass &own, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    const uint32_t grid = (uint32_t)(((uint64_t)a.total_q * a.n_heads + kWarps - 1) / kWarps);
    GMS_BY_TYPE((launch_dependent(kv_attn_join_shared_kernel<T, D>, grid, kWarps * 32, 0, s, a, pre, own)));
}

}  // namespace gms
