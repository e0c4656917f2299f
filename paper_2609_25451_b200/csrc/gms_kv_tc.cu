// Attention of many query rows (prompts, chunks, batches behind one prefix) over the paged pool, on tcgen05.
//
// A unit is 256 query rows (tokens x the heads that share a KV head), two slots of 128.  Per step of 64 tokens and slot
//   S = Q K^T      (128 x 64 x D, both operands in shared memory, S in tensor memory)
//   P = 2^(S c - m), rounded to the pool's type, written over S in tensor memory; l += sum P in 32 bits
//   O += P V       (128 x D x 64, P from tensor memory, V as it lies in the pool: token rows, "MN-major" operand)
// Each slot has two S buffers, so that the product for its next step is done while its softmax works on this one, and the two
// slots take turns at the tensor core; a buffer is written again once P V of the step that used it is complete.
// (128-token steps with one buffer a slot: 976 us for 2,048 new tokens over 16k, the softmax waiting 40 % of the time.)
// O stays in tensor memory for the whole item; it is rescaled only when a row's maximum has grown by more than 2^8 (weights
// are then at most 256 times too large against a stale maximum, which 16-bit P and 32-bit l and O hold without loss).
// Warps 0-3 and 4-7: softmax of slots 0 and 1, one thread a row (no shuffles), 200 registers a thread.  Warps 8 and 11 issue
// the products of slots 0 and 1.  Warp 9 issues the TMA loads: one box of 64 elements x up to 128 tokens of one block, all ids
// of a tile at once, one lane a box; Q as boxes of 64 elements x heads x tokens where 128 rows are whole tokens (else the
// softmax threads copy it).  Warp 10 deals out the items (a ring of descriptors in shared memory).
// Bound: the softmax, by instruction latency: a step takes 2,250 cycles for both slots where the special-function unit needs
// 1,024 and the tensor core 1,280 (64-column scores read both operands from shared memory at 1.5 times the cycles); tensor pipe
// 47 % active.  Taking a part of the exponentials on the multiply-add units, loading the next S ahead, and making the slots
// take turns were each slower.  2,048 + 2 new sequences over 16k cached tokens, 32 / 8 heads of 128, bf16, 728 GFLOP: 780 us
// back to back (0.93 PFLOP/s), 870 to 890 us among other work.  8,192 tokens under a window of 1,024, f16: 238 us.
// Tensor memory: 2 x 2 S buffers of 64 columns, O0 O1 (D each) = 512 columns at D = 128, hence P over S.
// Shared memory: Q 2 x 128 x D, then a ring of K and V tiles.
#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_tcgen05.h"

namespace gms {
namespace {

using namespace ptx;

constexpr int kThreads = 384, kRows = (int)kTcRows, kTile = (int)kTcTile;
constexpr float kLag = 8.f;  // log2 of how far a maximum may have grown before O is rescaled
// log2 of how much larger P is kept: with the lag the most that fp16 holds.  Else weights below 2^-25 of the maximum were nothing
// to the product with V, however many there are, and counted in l all the same.
template <class T> constexpr float kUp = std::is_same<T, __half>::value ? 7.f : 0.f;

// A run of tiles of one item, as the roles read it from shared memory.  k0 == k1: no more.
struct Segment {
    const int32_t *table;
    int q0, row0, rows, n, first, pos_min, pos_max, n_sink_tiles, first_tile, tiles, k0, k1;
    uint32_t c, item, whole, holes;
};
constexpr uint32_t kSegments = 4;

template <int D>
struct Tc {
    static constexpr int kHalves = D / 64;
    static constexpr uint32_t kHalfBytes = 128 * 128;             // 128 rows x 64 elements
    static constexpr uint32_t kTileBytes = kHalves * kHalfBytes;  // a K, V or Q tile
    static constexpr int kStages = D == 128 ? 4 : 8;
    static constexpr uint32_t kBars = (2 * kStages + 2 + 2 + 4 + 4 + 4 + 1 + 3 * kSegments) * 8;
    static constexpr uint32_t kOutBytes = 8 * 4096;               // 32 rows x 128 bytes a softmax warp, for coalesced stores
    static constexpr uint32_t kSmem = (2 + kStages) * kTileBytes + kOutBytes + kBars + 128 + kSegments * sizeof(Segment) + 1024;
    static constexpr uint32_t kO = 256;                            // first column of O0
    static constexpr uint32_t kCols = 512;
};

__device__ __forceinline__ bool next_segment(const AttnArgs &a, const Pass &p, Walk &w, Segment &g, bool first)
{
    Unit u = {};
    uint32_t at = 0;
    g.c = 0, g.k0 = g.k1 = 0;
    const bool more = walk_next<kRows, kTile>(a, p, w, u, g.c, g.k0, g.k1, at, g.item);
    if (!more) g.k0 = g.k1 = 0;
    if (first && (threadIdx.x & 31u) == 0) write_cut(p, blockIdx.x, w, u, g.c, g.k0, at);
    g.table = u.table;
    g.q0 = u.q0, g.row0 = u.row0, g.rows = u.rows, g.n = u.n, g.first = u.first, g.pos_min = u.pos_min, g.pos_max = u.pos_max;
    g.n_sink_tiles = u.n_sink_tiles, g.first_tile = u.first_tile, g.tiles = u.tiles, g.whole = u.whole;
    return more;
}
__device__ __forceinline__ int seg_tile(const Segment &g, int k)
{
    return k < g.n_sink_tiles ? k : g.first_tile + k - g.n_sink_tiles;
}

template <class T> struct IsBf16 { static constexpr bool value = false; };
template <> struct IsBf16<__nv_bfloat16> { static constexpr bool value = true; };

// Changes the sign of (or clears) two packed 16-bit values.
__device__ __forceinline__ uint4 with_sign(uint4 v, uint32_t flip, uint32_t keep)
{
    return make_uint4((v.x ^ flip) & keep, (v.y ^ flip) & keep, (v.z ^ flip) & keep, (v.w ^ flip) & keep);
}

// The lowest n bits (n may lie outside 0 .. 32).
__device__ __forceinline__ uint32_t first_bits(int n) { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; }

// A wait that every role uses: bounded, and cut short when another role has given up.
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, volatile uint32_t *abort, unsigned long long *status)
{
    const uint64_t end = now_ns() + kWaitLimitNs;
    for (uint32_t n = 0; n < (1u << 24) && now_ns() <= end; ++n) {
        if (mbar_spin(bar, parity, 256)) return true;
        if (*abort) return false;
    }
    *abort = 1;
    if (status) atomicOr(status, (unsigned long long)GMS_DEV_TIMEOUT);
    return false;
}
__device__ __forceinline__ bool wait_or_abort(uint32_t bar, uint32_t parity, volatile uint32_t *abort, unsigned long long *status)
{
    return mbar_spin(bar, parity, 4096) || wait_slow(bar, parity, abort, status);
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) kv_attn_tc_kernel(const __grid_constant__ CUtensorMap kmap,
                                                                 const __grid_constant__ CUtensorMap vmap,
                                                                 const __grid_constant__ CUtensorMap qmap,
                                                                 const __grid_constant__ AttnArgs a, const __grid_constant__ Pass p,
                                                                 uint32_t box_tokens, uint32_t q_tma)
{
    using F = Tc<D>;
    constexpr int NS = F::kStages;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *sm = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t q_smem = base, ring = base + 2 * F::kTileBytes;
    uint64_t *bars = reinterpret_cast<uint64_t *>(sm + (2 + NS) * F::kTileBytes + F::kOutBytes);
    const uint32_t full = smem_u32(bars), empty = full + 8 * NS, q_full = empty + 8 * NS, q_empty = q_full + 16, s_full = q_empty + 16,
                   p_full = s_full + 32, o_done = p_full + 32, drain = o_done + 32, seg_full = drain + 8, seg_empty = seg_full + 8 * kSegments,
                   seg_holes = seg_empty + 8 * kSegments;
    uint32_t *plan = reinterpret_cast<uint32_t *>(bars + 2 * NS + 17 + 3 * kSegments);
    volatile uint32_t *shared_words = plan + 16;  // behind the plan's 14  // [0] tensor memory, [1] abort
    volatile uint32_t *abort = shared_words + 1;
    Segment *const segs = reinterpret_cast<Segment *>(const_cast<uint32_t *>(shared_words) + 4);
    if (tid == 0) {
        for (int i = 0; i < NS; ++i) mbar_init(full + 8 * i, 1), mbar_init(empty + 8 * i, 2);  // both product warps
        for (int i = 0; i < 2; ++i) {
            mbar_init(q_full + 8 * i, q_tma ? 1 : 128);
            mbar_init(q_empty + 8 * i, 1);
            for (int b = 0; b < 2; ++b) {  // one of each a buffer: no one is ever two phases behind
                mbar_init(s_full + 8 * (2 * i + b), 1);
                mbar_init(p_full + 8 * (2 * i + b), 128);
                mbar_init(o_done + 8 * (2 * i + b), 1);
            }
        }
        mbar_init(drain, 2);
        for (uint32_t i = 0; i < kSegments; ++i) {
            mbar_init(seg_full + 8 * i, 1);
            mbar_init(seg_holes + 8 * i, 1);
            mbar_init(seg_empty + 8 * i, 11);  // 8 softmax warps, 3 more
        }
        *abort = 0;
        fence_mbar_init();
        tma_prefetch_map(&kmap);
        tma_prefetch_map(&vmap);
        if (q_tma) tma_prefetch_map(&qmap);
    }
    if (warp == 8) tmem_alloc(smem_u32(const_cast<uint32_t *>(shared_words)), F::kCols);
    if (!p.behind) grid_wait();
    grid_launch_dependents();
    tc_fence_before();
    Walk w = plan_walk<kRows, kTile, kThreads, 1>(a, p, plan);  // ends with __syncthreads
    tc_fence_after();
    const uint32_t tmem = shared_words[0];

    // 384 threads x 168 registers = 128 x 104 + 256 x 200
    uint32_t seg = 0;  // segments seen
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (warp == 10) {
            // ------------------------------------------------------------------ items
            for (bool more = true; more; ++seg) {
                const uint32_t at = seg % kSegments;
                if (!__all_sync(0xffffffffu, wait_or_abort(seg_empty + 8 * at, ((seg / kSegments) & 1u) ^ 1u, abort, a.status))) break;
                Segment g;
                more = next_segment(a, p, w, g, seg == 0);
                if (lane == 0) {
                    segs[at] = g;
                    mbar_arrive(seg_full + 8 * at);
                }
                if (more) {  // whether any id of its tiles lies outside the pool (then the softmax looks at every tile's)
                    bool hole = false;
                    const int t_end = min(g.n, (seg_tile(g, g.k1 - 1) + 1) * kTile), step = 1 << a.block_shift;
                    for (int k = g.k0; k < min(g.k1, g.n_sink_tiles); ++k)
                        for (int t = k * kTile + (int)lane * step; t < (k + 1) * kTile; t += 32 * step)
                            hole |= (uint32_t)g.table[(uint32_t)t >> a.block_shift] >= a.n_blocks;
                    for (int t = (seg_tile(g, max(g.k0, g.n_sink_tiles)) * kTile & ~(step - 1)) + (int)lane * step; t < t_end; t += 32 * step)
                        hole |= (uint32_t)g.table[(uint32_t)t >> a.block_shift] >= a.n_blocks;
                    hole = __any_sync(0xffffffffu, hole);
                    if (lane == 0) {
                        segs[at].holes = hole;
                        mbar_arrive(seg_holes + 8 * at);
                    }
                }
            }
            __syncwarp();
        } else if (warp == 9) {
            // ------------------------------------------------------------------ loads
            const int per = kTile / (int)box_tokens, boxes = per * F::kHalves;  // boxes a tile: at most 16
            const int half = (int)lane % F::kHalves, part = (int)lane / F::kHalves;
            const uint32_t tok_mask = (1u << a.block_shift) - 1u;
            uint32_t n = 0, q_n[2] = {0, 0};  // stages filled; times each slot's Q was
            bool ok = true;
            // K and V that one row tile reads go first in L2; those that several read stay
            const uint64_t policy = p.n_rt == 1 ? policy_evict_first() : policy_evict_normal();
            for (;; ++seg) {
                ok = __all_sync(0xffffffffu, ok && wait_or_abort(seg_full + 8 * (seg % kSegments), (seg / kSegments) & 1u, abort, a.status));
                if (!ok) break;
                const Segment &g = segs[seg % kSegments];
                if (g.k0 == g.k1) break;
                const int32_t *table = g.table;
                const int len = g.n, k1 = g.k1, head = (int)g.c;
                // A hole, nothing left to read, or nothing that any row sees (what has left the window and lies in a sinks' tile or
                // in the first one behind may belong to someone else by now): out of range, zeros arrive.
                const int last = min(len - 1, g.pos_max), past = g.whole ? 0 : max(g.pos_min, 0) - (int)min(a.window - 1u, 0x7fffffffu);
                auto block_of = [&](int k) -> int {
                    const int t = seg_tile(g, k) * kTile + part * (int)box_tokens;
                    int id = -1;
                    if ((int)lane < boxes && t <= last && (t + (int)box_tokens > past || (uint32_t)t < a.sinks)) id = table[(uint32_t)t >> a.block_shift];
                    return (uint32_t)id < a.n_blocks ? id : (int)a.n_blocks;
                };
                int next = block_of(g.k0);
                if (q_tma) {
#pragma unroll
                    for (int slot = 0; slot < 2; ++slot) {
                        if (!ok || slot * 128 >= g.rows) continue;
                        ok = __all_sync(0xffffffffu, wait_or_abort(q_empty + 8 * slot, (q_n[slot] & 1u) ^ 1u, abort, a.status));
                        if (!ok) continue;
                        if (lane == 0) {
                            mbar_expect(q_full + 8 * slot, F::kTileBytes);
                            for (int h = 0; h < F::kHalves; ++h)
                                tma_load_3d(q_smem + slot * F::kTileBytes + h * F::kHalfBytes, &qmap, h * 64, head * (int)a.group,
                                            g.q0 + (g.row0 + slot * 128) / (int)a.group, q_full + 8 * slot);
                        }
                        ++q_n[slot];
                    }
                }
                for (int k = g.k0; ok && k < k1; ++k) {
                    const int blk = next, t = seg_tile(g, k) * kTile + part * (int)box_tokens;
                    if (k + 1 < k1) next = block_of(k + 1);
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint32_t st = n % NS;
                        ok = __all_sync(0xffffffffu, wait_or_abort(empty + 8 * st, ((n / NS) & 1u) ^ 1u, abort, a.status));
                        if (!ok) break;
                        if (lane == 0) mbar_expect(full + 8 * st, F::kTileBytes);
                        __syncwarp();
                        if ((int)lane < boxes)
                            tma_load_4d(ring + st * F::kTileBytes + half * F::kHalfBytes + part * box_tokens * 128, v ? &vmap : &kmap, half * 64,
                                        (int)((uint32_t)t & tok_mask), head, blk, full + 8 * st, policy);
                        ++n;
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(seg_empty + 8 * (seg % kSegments));
            }
            if (!ok)  // give up: wait (bounded) for what is still on its way into this CTA's shared memory
                for (uint32_t i = n > (uint32_t)NS ? n - NS : 0; i < n; ++i) (void)mbar_wait(full + 8 * (i % NS), (i / NS) & 1u);
            for (int slot = 0; !ok && slot < 2; ++slot)
                if (q_n[slot]) (void)mbar_wait(q_full + 8 * slot, (q_n[slot] - 1) & 1u);
        } else {
            // ------------------------------------------------------------------ products of one slot (warp 8: slot 0, warp 11: slot 1)
            constexpr uint32_t id_s = f16_idesc(128, 64, IsBf16<T>::value, false), id_o = f16_idesc(128, D, IsBf16<T>::value, true);
            // Straight-line code a tile: these warps compete for issue with two softmax warps each, every instruction counts.
#define GMS_WAIT(bar, parity)                                                             \
        if (!__all_sync(0xffffffffu, mbar_spin(bar, parity, 4096)) &&                         \
            !__all_sync(0xffffffffu, wait_slow(bar, parity, abort, a.status)))                \
            goto products_done
            const uint32_t on = one_lane(), slot = warp == 8 ? 0u : 1u;
            constexpr uint32_t hi = desc_hi(1024), half_k = 64 * 128 >> 4, half_v = 4 * 2048 >> 4;
            const uint32_t q_lo = desc_lo(q_smem + slot * F::kTileBytes, 16), k_lo = desc_lo(ring, 16), v_lo = desc_lo(ring, F::kHalfBytes);
            const uint32_t s_tm = tmem + slot * 128, o_tm = tmem + F::kO + slot * D;
            const uint32_t my_s = s_full + 16 * slot, my_p = p_full + 16 * slot, my_o = o_done + 16 * slot, my_q = 8 * slot;
            // S of one half of a K tile (k: its descriptor) into buffer b
            auto scores = [&](uint32_t b, uint32_t k) {
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t off = ((kk / 4) * F::kHalfBytes + (kk % 4) * 32) >> 4;
                    mma_ss(on, s_tm + b * 64, q_lo + off, k + b * half_k + off, hi, id_s, kk > 0);
                }
                tc_commit(on, my_s + 8 * b);
            };
            auto values = [&](uint32_t b, uint32_t v, bool add) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) mma_ts(on, o_tm, s_tm + b * 64 + kk * 8, v + b * half_v + (kk * 2048 >> 4), hi, id_o, add || kk > 0);
                tc_commit(on, my_o + 8 * b);
            };
            uint32_t ks = 0, kph = 0;       // stage of the next K tile (V follows it) and its phase
            uint32_t tiles = 0, items = 0;  // of this slot so far (low bits count)
            for (;; ++seg) {
                GMS_WAIT(seg_full + 8 * (seg % kSegments), (seg / kSegments) & 1u);
                const Segment &g = segs[seg % kSegments];
                const bool mine = slot == 0 || __shfl_sync(0xffffffffu, g.rows, 0) > 128;
                const int nt = __shfl_sync(0xffffffffu, g.k1 - g.k0, 0);
                __syncwarp();
                if (lane == 0) mbar_arrive(seg_empty + 8 * (seg % kSegments));
                if (nt == 0) break;
                if (!mine) {  // no rows here: only hand the stages back
                    for (int j = 0; j < 2 * nt; ++j) {
                        GMS_WAIT(full + 8 * ks, kph);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(empty + 8 * ks);
                        if (++ks == NS) ks = 0, kph ^= 1u;
                    }
                    continue;
                }
                uint32_t k = k_lo + (ks * F::kTileBytes >> 4);
                GMS_WAIT(full + 8 * ks, kph);
                GMS_WAIT(q_full + my_q, items & 1u);
                GMS_WAIT(my_o, (tiles & 1u) ^ 1u);  // P V of the last item: its buffers are free
                GMS_WAIT(my_o + 8, (tiles & 1u) ^ 1u);
                tc_fence_after();
#pragma unroll 1
                for (uint32_t b = 0; b < 2; ++b) scores(b, k);
                tc_commit(on, empty + 8 * ks);
                if (nt == 1) tc_commit(on, q_empty + my_q);
                for (int j = 0; j < nt; ++j) {
                    const uint32_t vs = ks + 1, v = v_lo + (vs * F::kTileBytes >> 4);
                    const bool more = j + 1 < nt;
                    GMS_WAIT(full + 8 * vs, kph);
                    ks += 2;
                    if (ks == NS) ks = 0, kph ^= 1u;
                    k = k_lo + (ks * F::kTileBytes >> 4);
#pragma unroll 1
                    for (uint32_t b = 0; b < 2; ++b) {
                        GMS_WAIT(my_p + 8 * b, tiles & 1u);
                        tc_fence_after();
                        values(b, v, j > 0 || b > 0);
                        if (more) {
                            if (b == 0) GMS_WAIT(full + 8 * ks, kph);
                            GMS_WAIT(my_o + 8 * b, tiles & 1u);  // P lies over S
                            tc_fence_after();
                            scores(b, k);
                        }
                    }
                    tc_commit(on, empty + 8 * vs);
                    if (more) tc_commit(on, empty + 8 * ks);
                    if (j + 2 == nt) tc_commit(on, q_empty + my_q);
                    ++tiles;
                }
                ++items;
            }
        products_done:
#undef GMS_WAIT
            tc_commit(on, drain);  // nothing of this warp's is in flight when the CTA ends
            (void)mbar_wait(drain, 0);
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // ------------------------------------------------------------------ softmax, one thread a row
        const int slot = (int)warp / 4, row_in = (int)(warp % 4) * 32 + (int)lane, row = slot * 128 + row_in;
        const uint32_t lanes = ((warp % 4) * 32) << 16;
        const uint32_t s_col = tmem + lanes + slot * 128, o_col = tmem + lanes + F::kO + slot * D;
        const float scale2 = a.scale * kLog2e, c2 = a.scale == 0.f ? 1.f : fabsf(scale2);
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, keep = a.scale == 0.f ? 0u : 0xffffffffu;
        uint32_t n = 0, tiles = 0;  // tiles of all segments so far; of this slot
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity) {
            if (!__all_sync(0xffffffffu, mbar_spin(bar, parity, 4096)))  // the warp goes on, or gives up, as one
                ok = __all_sync(0xffffffffu, wait_slow(bar, parity, abort, a.status));
            return ok;
        };
        for (;; ++seg) {
            if (!wait(seg_full + 8 * (seg % kSegments), (seg / kSegments) & 1u)) break;
            const Segment &g = segs[seg % kSegments];
            const int k0 = g.k0, k1 = g.k1, rows = g.rows, row0 = g.row0, q0 = g.q0, len = g.n;
            if (k0 == k1) break;
            const uint32_t head0 = g.c * a.group;
            const bool all = g.whole != 0;
            if (slot == 1 && rows <= 128) {
                n += (uint32_t)(k1 - k0);
                __syncwarp();
                if (lane == 0) mbar_arrive(seg_empty + 8 * (seg % kSegments));
                continue;
            }
            auto tok_of = [&](int r) { return q0 + (row0 + r) / (int)a.group; };
            auto head_of = [&](int r) { return head0 + (uint32_t)(row0 + r) % a.group; };
            auto pos_of = [&](int r) { return all ? len - 1 : g.first + (row0 + r) / (int)a.group; };
            if (!q_tma) {  // 16-byte pieces, a row's in neighbouring lanes; rows that do not exist are zero
#pragma unroll 4
                for (int i = 0; i < D / 8; ++i) {
                    const int idx = i * 128 + row_in, r = idx / (D / 8), ch = idx % (D / 8);
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (slot * 128 + r < rows)
                        v = with_sign(*reinterpret_cast<const uint4 *>(a.q + (uint64_t)tok_of(slot * 128 + r) * a.q_token_stride +
                                                                       (uint64_t)head_of(slot * 128 + r) * a.q_head_stride + ch * 16),
                                      flip, keep);
                    *reinterpret_cast<uint4 *>(sm + slot * F::kTileBytes + (ch / 8) * F::kHalfBytes + r * 128 + (((ch % 8) ^ (r & 7)) << 4)) = v;
                }
                fence_proxy_async();
                mbar_arrive(q_full + 8 * slot);
            }

            const bool live = row < rows, busy = slot * 128 + (int)(warp % 4) * 32 < rows;  // a warp without rows computes nothing
            const int pos_own = pos_of(live ? row : rows - 1), pos_hi = pos_of(min(slot * 128 + 127, rows - 1));
            const int pos = min(pos_own, len - 1), pos_lo = min(pos_of(slot * 128), len - 1);  // the newest token seen, of the row and at least
            const int32_t *table = g.table;
            // the row's window starts at low; low_hi: the latest start among the slot's rows; sink: tokens always seen
            auto low_of = [&](int ps) { return all || a.window == 0 || (uint32_t)max(ps, 0) < a.window ? 0 : ps - (int)a.window + 1; };
            const int low = low_of(pos_own), low_hi = low_of(pos_hi), sink = (int)min(a.sinks, 0x7fffffffu);
            float m = neg_inf(), l = 0.f;
            const int n_sink_tiles = g.n_sink_tiles, past_sinks = g.first_tile - n_sink_tiles;
            if (!wait(seg_holes + 8 * (seg % kSegments), (seg / kSegments) & 1u)) break;
            const bool holes = g.holes != 0;
            // One step: 64 columns of S to P.  (In the code once: first runs are bound by fetching instructions.)
            auto step = [&](const int half, const bool edge, int k, int t0, uint32_t valid) {
                if (!wait(s_full + 8 * (2 * slot + half), tiles & 1u)) return;
                tc_fence_after();
                if (busy) {
                    uint32_t s[2][32];
                    tmem_ld32(s_col + half * 64, s[0]);
                    tmem_ld32(s_col + half * 64 + 32, s[1]);
                    tmem_wait32(s[0]);
                    tmem_wait32(s[1]);
                    if (edge) {
                        const uint32_t v4 = valid >> (4 * half);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int c0 = t0 + half * 64 + i * 32;
                            const uint32_t held = ((v4 >> (2 * i) & 1u) ? 0xffffu : 0u) | ((v4 >> (2 * i + 1) & 1u) ? 0xffff0000u : 0u);
                            const uint32_t on = held & first_bits(pos + 1 - c0) & (~first_bits(low - c0) | first_bits(sink - c0));
                            if (__all_sync(0xffffffffu, on == 0xffffffffu)) continue;
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!(on >> j & 1u)) s[i][j] = 0xff800000u;
                        }
                    }
                    float tops[4];  // four chains
#pragma unroll
                    for (int i = 0; i < 4; ++i) tops[i] = __uint_as_float(s[i / 2][(i % 2) * 16]);
#pragma unroll
                    for (int j = 1; j < 15; j += 2)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            tops[i] = fmaxf(fmaxf(tops[i], __uint_as_float(s[i / 2][(i % 2) * 16 + j])),
                                            __uint_as_float(s[i / 2][(i % 2) * 16 + j + 1]));
#pragma unroll
                    for (int i = 0; i < 4; ++i) tops[i] = fmaxf(tops[i], __uint_as_float(s[i / 2][(i % 2) * 16 + 15]));
                    const float top = fmaxf(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])), neg_inf()) * c2;
                    const bool grow = top > m + kLag || (m == neg_inf() && top != m);
                    if (__any_sync(0xffffffffu, grow)) {
                        const float f = grow ? (m == neg_inf() ? 0.f : ex2(m - top)) : 1.f;
                        if (grow) m = top;
                        l *= f;
                        if (k != k0 || half) {  // O is at rest between the last step's product and this step's handing over
                            if (!wait(o_done + 8 * (2 * slot + (half ^ 1)), (tiles + (half ^ 1)) & 1u)) return;
                            tc_fence_after();
#pragma unroll 1
                            for (int i = 0; i < D / 32; ++i) {
                                uint32_t o[32];
                                tmem_ld32(o_col + i * 32, o);
                                tmem_wait32(o);
#pragma unroll
                                for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                tmem_st32(o_col + i * 32, o);
                            }
                        }
                    }
                    const float z = m == neg_inf() ? 0.f : m - kUp<T>;
                    const float2 cc = make_float2(c2, c2), zz = make_float2(-z, -z);
                    float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    uint32_t pk[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        float2 x = make_float2(__uint_as_float(s[j / 16][(j * 2) % 32]), __uint_as_float(s[j / 16][(j * 2 + 1) % 32]));
                        x = fma2(x, cc, zz);
                        x.x = ex2(x.x);
                        x.y = ex2(x.y);
                        part[j & 1] = add2(part[j & 1], x);
                        pk[j] = pack2(x.x, x.y, T());
                    }
                    tmem_st32(s_col + half * 64, pk);
                    part[0] = add2(part[0], part[1]);
                    l += part[0].x + part[0].y;
                }
                // Values of tokens that do not exist must not meet the product, whatever bits they are; nor those that no row
                // of the unit sees, where rows are not done again.  Thread r of each slot clears token r of the tile before
                // its slot's first half is handed over (the other slot may clear it too: the same zeros).
                if (half == 0 && edge) {
                    const int t = t0 + row_in;
                    const bool none = t >= len || (!p.again && (t > g.pos_max || (!all && !sees(a, max(g.pos_min, t), t))));
                    if (__any_sync(0xffffffffu, none)) {
                        const uint32_t vs = 2 * n + 1;
                        if (!wait(full + 8 * (vs % NS), (vs / NS) & 1u)) return;
                        if (none)
#pragma unroll
                            for (int h = 0; h < F::kHalves; ++h)
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    st_shared_zero16(ring + (vs % NS) * F::kTileBytes + h * F::kHalfBytes + row_in * 128 +
                                                     ((e ^ (lane & 7)) << 4));
                        fence_proxy_async();
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(p_full + 8 * (2 * slot + half));
            };
            for (int k = k0; ok && k < k1; ++k) {
                const int t0 = (k < n_sink_tiles ? k : past_sinks + k) * kTile;
                uint32_t valid = 0xffu;
                if (holes) {  // the block of each 16 tokens of the tile, one lane each
                    const int t = t0 + (int)lane * 16;
                    const int id = lane < 8 && t < len ? table[(uint32_t)t >> a.block_shift] : -1;
                    valid = __ballot_sync(0xffffffffu, (uint32_t)id < a.n_blocks) & 0xffu;
                }
                const bool whole = valid == 0xffu && t0 + kTile - 1 <= pos_lo && (t0 >= low_hi || t0 + kTile - 1 < sink);
#pragma unroll 1
                for (int half = 0; ok && half < 2; ++half) step(half, !whole, k, t0, valid);
                ++n;
                ++tiles;
            }
            if (!ok) break;
            m -= kUp<T>;  // what O and l stand against
            // the item's rows (or this CTA's piece of them)
            if (!wait(o_done + 16 * slot, (tiles - 1) & 1u) || !wait(o_done + 16 * slot + 8, (tiles - 1) & 1u)) break;
            tc_fence_after();
            const uint64_t tok = tok_of(live ? row : 0);
            const uint32_t h = head_of(live ? row : 0);
            const bool starts = k0 == 0, mine = starts && k1 == g.tiles, finished = mine && !p.row_o;
            const float inv = l == 0.f ? 0.f : 1.f / l;
            bool bad = false;
            if (finished) {
                // through shared memory, so that four lanes write 64 bytes of a row at a time
                const uint64_t at = tok * a.out_token_stride + h * a.out_head_stride;
                uint8_t *stage = sm + (2 + NS) * F::kTileBytes + warp * 4096;
                if (live && a.lse) a.lse[tok * a.n_heads + h] = l == 0.f ? neg_inf() : (m + log2f(l)) * kLn2;
                const uint32_t rows_here = (uint32_t)max(0, min(32, rows - slot * 128 - (int)(warp % 4) * 32));
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    tmem_ld32(o_col + i * 32, o);
                    tmem_wait32(o);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float lo = __uint_as_float(o[j * 8 + 2 * e]) * inv, hi = __uint_as_float(o[j * 8 + 2 * e + 1]) * inv;
                            if (l == 0.f) lo = hi = 0.f;
                            bad |= !(fabsf(lo) < kHuge && fabsf(hi) < kHuge);
                            v[e] = pack2(lo, hi, T());
                        }
                        *reinterpret_cast<uint4 *>(stage + lane * 64 + ((j ^ (lane >> 1 & 3)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t r = e * 8 + lane / 4, ch = lane & 3u;
                        const uint64_t to = __shfl_sync(0xffffffffu, at, r);
                        const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * 64 + ((ch ^ (r >> 1 & 3)) << 4));
                        if (r < rows_here) *reinterpret_cast<uint4 *>(a.out + to + i * 64 + ch * 16) = v;
                    }
                    __syncwarp();
                }
            } else {
                const uint64_t at = mine ? tok * a.n_heads + h : ((uint64_t)blockIdx.x * 2 + (starts ? 1 : 0)) * p.slot_rows + row;
                float *dst = mine ? p.row_o : p.part_o;
                uint8_t *stage = sm + (2 + NS) * F::kTileBytes + warp * 4096;
                if (live) (mine ? p.row_ml : p.part_ml)[at] = make_float2(m, l);
                const uint32_t rows_here = (uint32_t)max(0, min(32, rows - slot * 128 - (int)(warp % 4) * 32));
#pragma unroll 1
                for (int i = 0; i < D / 32; ++i) {
                    uint32_t o[32];
                    tmem_ld32(o_col + i * 32, o);
                    tmem_wait32(o);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4 *>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                            make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint32_t r = e * 4 + lane / 8, ch = lane & 7u;
                        const uint64_t to = __shfl_sync(0xffffffffu, at, r);
                        const uint4 v = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((ch ^ (r & 7)) << 4));
                        if (r < rows_here) *reinterpret_cast<uint4 *>(dst + to * D + i * 32 + ch * 4) = v;
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            if (p.redo) {  // which of the warp's rows the join has to do again
                const uint32_t again = __ballot_sync(0xffffffffu, live && bad);
                if (lane == 0) p.redo[(uint64_t)g.item * 8 + warp] = again;
                if (rows <= 128 && lane == 1) p.redo[(uint64_t)g.item * 8 + 4 + warp] = 0;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(seg_empty + 8 * (seg % kSegments));
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_free(tmem, F::kCols);
    }
    if (p.behind) grid_wait();  // this kernel's end stands for both
}

template <class T, int D>
cudaError_t launch(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, const CUtensorMap *qmap,
                   uint32_t box_tokens, cudaStream_t s)
{
    constexpr uint32_t smem = Tc<D>::kSmem;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(kv_attn_tc_kernel<T, D>, smem, done);
    if (e != cudaSuccess) return e;
    const CUtensorMap &qm = qmap ? *qmap : kmap;
    const uint32_t q_tma = qmap != nullptr;
    return launch_dependent(kv_attn_tc_kernel<T, D>, p.workers, kThreads, smem, s, kmap, vmap, qm, a, p, box_tokens, q_tma);
}

}  // namespace

cudaError_t launch_kv_attn_tc(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, const CUtensorMap *qmap,
                              uint32_t box_tokens, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    if (dtype == GMS_DTYPE_BF16)
        return head_dim == 64 ? launch<__nv_bfloat16, 64>(a, p, kmap, vmap, qmap, box_tokens, s)
                              : launch<__nv_bfloat16, 128>(a, p, kmap, vmap, qmap, box_tokens, s);
    return head_dim == 64 ? launch<__half, 64>(a, p, kmap, vmap, qmap, box_tokens, s) : launch<__half, 128>(a, p, kmap, vmap, qmap, box_tokens, s);
}

}  // namespace gms
