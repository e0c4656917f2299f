// Internal declarations of the attention and eviction kernels on the paged KV pool.
#pragma once
#include <atomic>
#include <cstdint>

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cmath>
#include <type_traits>

#include "gms.h"

namespace gms {

void count_launches(uint32_t n);

// GMS_OK, or what is wrong with a pool or with a layout in it.
int bad_pool(const gms_kv_pool *p);
int bad_layout(const gms_kv_pool *p, const gms_kv_layout *l);
inline uint32_t log2_of(uint32_t x) { return 31u - (uint32_t)__builtin_clz(x); }

// What every attention kernel gets (by value).  Strides of pool and of q / out are in bytes.
struct AttnArgs {
    const uint8_t *k_base, *v_base;  // planes of this layer
    uint64_t block_stride;
    uint32_t n_blocks, token_stride, head_stride, block_shift;  // block_tokens = 1 << block_shift
    const uint8_t *q;
    uint8_t *out;
    float *lse;
    const int32_t *cu_q, *kv_lens, *table;
    uint64_t table_stride;
    uint64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;
    uint32_t n_seq, n_heads, n_kv, group;  // group = n_heads / n_kv
    uint32_t total_q, max_q, max_kv, window, sinks;
    float scale;
    // shared prefixes (n_groups = 0: none)
    const int32_t *group_start, *prefix_lens, *prefix_table;
    uint64_t prefix_stride;
    uint32_t n_groups, max_prefix, max_group_q;
    // accumulated weights (w_out = null: none)
    const float *w_in;
    float *w_out;
    uint64_t w_seq_stride, w_head_stride;
    float decay;
    unsigned long long *status;  // may be null
};

// How a pass over cached tokens is cut.  A unit is a run of up to ROWS query rows (token-major, the heads of one KV head
// inside a token) of one sequence (or, in a prefix pass, of one group); an item is a unit for one KV head; an item's work
// is the list of token tiles that at least one of its rows sees.  All items' tiles, one after the other, are dealt out
// evenly: worker i of n (n = workers, or T if that is less) gets T / n or T / n + 1 tiles, whatever items they fall into, so
// ragged lengths cost no balance.  (Of the many-row kernel's items each counts kTcExtra tiles more, which stand for loading Q
// and writing the result: without them the worker with 38 short items of a windowed prompt took 1.2 times the others' time.)
// A worker is a CTA of the many-row kernel, a warp of the few-row kernel.  An item that one
// worker has whole is finished there; the at most two pieces a worker has of others go to its two slots of part_o / part_ml
// and are joined by kv_attn_join.
struct Cut {               // the item into which the border before worker i falls (c1 = 0: the border lies between items)
    int q0, row0, rows;
    uint32_t c, c0, c1;    // KV head; first and last worker that has a piece
    uint32_t pad[2];
};
struct Pass {
    uint32_t prefix;       // 1: units are groups' query rows over their prefix, all of it seen
    uint32_t behind;       // 1: launched behind the prefix pass of the same call, on which it does not depend
    uint32_t n_units, n_rt, workers;  // n_rt units a sequence (group)
    uint32_t rows, tile;   // rows a unit, tokens a tile
    uint32_t slot_rows;    // rows a slot of part_o has room for (at most `rows`)
    uint32_t *begin;       // [n_units + 1] tiles before each unit (written by CTA 0 for the join)
    Cut *cuts;             // [workers], written by worker i for its own border
    float *part_o;         // [2 * workers][slot_rows][head_dim], not normalised
    float2 *part_ml;       // [2 * workers][slot_rows]: running maximum (base 2) and sum
    float *row_o;          // null: finished rows go to out / lse; else [total_q * n_heads][head_dim], not normalised
    float2 *row_ml;        // [total_q * n_heads]
    float *logits;         // null, or [n_units * n_kv][max_q * group][logit_stride], base 2, in tile list order (few-row pass only)
    uint32_t logit_stride;
    uint32_t team;         // 1: few-row pass, a CTA an item: its warps share the tiles and join in shared memory, nothing is cut
    uint32_t again;        // 1: rows that come out non-finite are done again (attend_row)
    uint32_t *redo;        // many-row pass: null, or [n_units * n_kv][8], a bit for each such row of a finished item
};

struct EvictArgs {
    uint8_t *base;
    uint64_t plane_stride, block_stride;
    uint32_t k_plane, v_plane, n_blocks, token_stride, head_stride, block_shift, row_bytes;
    const float *weights;
    float *weights_out;
    const int32_t *lens;
    int32_t *lens_out;
    const int32_t *src_table, *dst_table;
    int32_t *kept;
    uint64_t w_layer_stride, w_seq_stride, w_head_stride, o_layer_stride, o_seq_stride, o_head_stride, src_stride, dst_stride;
    uint32_t n_layers, layer_planes, n_seq, n_kv, max_len, budget, sinks, recent;
    unsigned long long *status;  // may be null
};

// behind: the attention kernels of the same call have been launched.
cudaError_t launch_kv_weights(const AttnArgs &a, const float *lse, bool behind, uint32_t dtype, uint32_t head_dim, cudaStream_t s);
// Joins the two passes of a shared-prefix call, row by row.
cudaError_t launch_kv_attn_join_shared(const AttnArgs &a, const Pass &prefix, const Pass &own, uint32_t dtype, uint32_t head_dim,
                                       cudaStream_t s);
// Few query rows a unit (at most 16): kv_attn_few; many: kv_attn_tc.
constexpr uint32_t kFewRows = 16, kFewTile = 16, kFewWarps = 4, kFewMaxWorkers = 2 * 148 * kFewWarps;
cudaError_t launch_kv_attn_few(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, uint32_t dtype,
                               uint32_t head_dim, cudaStream_t s);
// Many query rows a unit; box_tokens: tokens a TMA box of the maps holds; qmap: null, or boxes of 64 elements x group heads
// x 128 / group tokens of the queries.
constexpr uint32_t kTcRows = 256, kTcTile = 128, kTcMaxWorkers = 148, kTcExtra = 2;
cudaError_t launch_kv_attn_tc(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, const CUtensorMap *qmap,
                              uint32_t box_tokens, uint32_t dtype, uint32_t head_dim, cudaStream_t s);
cudaError_t launch_kv_attn_join(const AttnArgs &a, const Pass &p, uint32_t dtype, uint32_t head_dim, cudaStream_t s);
cudaError_t launch_kv_few_weights(const AttnArgs &a, const Pass &p, cudaStream_t s);
cudaError_t launch_kv_evict(const EvictArgs &a, cudaStream_t s);

// Lets a kernel have more than 48 KB of shared memory, once a device (`done` has a bit for each).
template <class K>
cudaError_t allow_smem(K kernel, uint32_t smem, std::atomic<uint64_t> &done)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && done.load(std::memory_order_relaxed) >> dev & 1u)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

// Launches a kernel that may start before the one ahead of it in the stream has drained.  What keeps that in order:
//  - The first kernel of a call (an attention kernel, the selecting kernel of an eviction) waits for the one ahead before it
//    touches anything, and lets the next one start only after that wait.  So whatever was there before the call is complete for
//    every kernel of the call, waiting or not.
//  - Each further kernel of the call (the own pass of a shared call, joins, weights, the moving kernel) may let its successor
//    start at once and, before its own wait, read what was there before the call and write what no other kernel of the call
//    touches, nothing more.
//  - Every kernel waits for the one ahead at some time, so a kernel's end stands for all that were launched before it.
template <class K, class... A>
cudaError_t launch_dependent(K kernel, uint32_t grid, uint32_t block, uint32_t smem, cudaStream_t s, const A &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at = {};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

#ifdef __CUDACC__
// ------------------------------------------------------------------ device helpers
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f, kHuge = 3.4e38f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }
template <class T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32(float x) { return __float2half_rn(x); }

// Query rows and cached tokens of one sequence, clamped to what the host announced (so that no index leaves a buffer
// whatever the device arrays hold).  Positions go by the lengths themselves: what is left out shifts nothing.
__device__ __forceinline__ int seq_q_begin(const AttnArgs &a, uint32_t s)
{
    return a.cu_q ? min(max(a.cu_q[s], 0), (int)a.total_q) : (int)s;
}
__device__ __forceinline__ int seq_q_len(const AttnArgs &a, uint32_t s)
{
    if (!a.cu_q) return 1;
    const int b = seq_q_begin(a, s);
    return min(max(min(a.cu_q[s + 1], (int)a.total_q) - b, 0), (int)a.max_q);
}
__device__ __forceinline__ int seq_kv_len(const AttnArgs &a, uint32_t s) { return min(max(a.kv_lens[s], 0), (int)a.max_kv); }
// Position of a sequence's first query.
__device__ __forceinline__ int seq_first(const AttnArgs &a, uint32_t s)
{
    return max(a.kv_lens[s], 0) - (a.cu_q ? max(min(a.cu_q[s + 1], (int)a.total_q) - seq_q_begin(a, s), 0) : 1);
}
__device__ __forceinline__ int prefix_len(const AttnArgs &a, uint32_t g)
{
    return min(max(a.prefix_lens[g], 0), (int)a.max_prefix);
}
// Whether the query at position `pos` sees token t.
__device__ __forceinline__ bool sees(const AttnArgs &a, int pos, int t)
{
    return t <= pos && (a.window == 0 || (long long)t > (long long)pos - (long long)a.window || (uint32_t)t < a.sinks);
}
// Last index i in [0, n) with v[i] <= x (v ascending, v[0] <= x).
__device__ __forceinline__ uint32_t last_not_above(const int32_t *v, uint32_t n, int x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (v[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
// Sequence that owns query row `tok`, or n_seq.  Equal offsets (empty sequences) resolve to the last of them.
__device__ __forceinline__ uint32_t owner_of_row(const AttnArgs &a, int tok)
{
    if (!a.cu_q) return (uint32_t)tok < a.n_seq ? (uint32_t)tok : a.n_seq;
    if (tok < a.cu_q[0] || tok >= a.cu_q[a.n_seq]) return a.n_seq;
    const uint32_t s = last_not_above(a.cu_q, a.n_seq, tok);
    return tok - seq_q_begin(a, s) < seq_q_len(a, s) ? s : a.n_seq;
}
// Group of a sequence, or n_groups.
__device__ __forceinline__ uint32_t group_of_seq(const AttnArgs &a, uint32_t s)
{
    if (a.n_groups == 0 || (int)s < a.group_start[0] || (int)s >= a.group_start[a.n_groups]) return a.n_groups;
    return last_not_above(a.group_start, a.n_groups, (int)s);
}
struct Unit {
    const int32_t *table;
    int q0, row0, rows;      // first query row of the sequence (group); first row of the unit and their number
    int n, first;            // cached tokens; position of the sequence's first query
    int pos_min, pos_max;    // of the unit's rows (at n or beyond it where the call leaves out the newest tokens)
    int n_sink_tiles, first_tile, tiles;  // tile list: 0 .. n_sink_tiles-1, then first_tile ..; `tiles` in all
    bool whole;              // every row sees every token
};
__device__ __forceinline__ int unit_tile(const Unit &u, int k) { return k < u.n_sink_tiles ? k : u.first_tile + k - u.n_sink_tiles; }
__device__ __forceinline__ int unit_row_pos(const AttnArgs &a, const Unit &u, int r)
{
    return u.whole ? u.n - 1 : u.first + (u.row0 + r) / (int)a.group;
}
// Query row and head of row r of a unit.
__device__ __forceinline__ int unit_tok(const AttnArgs &a, const Unit &u, int r) { return u.q0 + (u.row0 + r) / (int)a.group; }
__device__ __forceinline__ uint32_t unit_head(const AttnArgs &a, const Unit &u, uint32_t c, int r)
{
    return c * a.group + (uint32_t)(u.row0 + r) % a.group;
}
// `s`: sequence or group, `rt`: row tile of it.
template <int ROWS, int TILE>
__device__ __forceinline__ Unit get_unit(const AttnArgs &a, const Pass &p, uint32_t s, uint32_t rt)
{
    Unit u;
    int q_len;
    if (p.prefix) {
        const int s0 = min(max(a.group_start[s], 0), (int)a.n_seq), s1 = min(max(a.group_start[s + 1], s0), (int)a.n_seq);
        u.q0 = a.cu_q ? min(max(a.cu_q[s0], 0), (int)a.total_q) : s0;
        const int end = a.cu_q ? min(max(a.cu_q[s1], u.q0), (int)a.total_q) : s1;
        q_len = min(end - u.q0, (int)a.max_group_q);
        u.n = prefix_len(a, s);
        u.table = a.prefix_table + s * a.prefix_stride;
        u.whole = true;
        u.first = u.n - q_len;
    } else {
        u.q0 = seq_q_begin(a, s);
        q_len = seq_q_len(a, s);
        u.n = seq_kv_len(a, s);
        u.table = a.table + s * a.table_stride;
        u.whole = false;
        u.first = seq_first(a, s);
    }
    u.row0 = (int)rt * ROWS;
    u.rows = max(min(q_len * (int)a.group - u.row0, ROWS), 0);  // total_q * n_heads < 2^31
    u.n_sink_tiles = u.first_tile = u.tiles = 0;
    u.pos_min = u.pos_max = u.n - 1;
    if (u.rows > 0) {
        if (!u.whole) {
            u.pos_min = u.first;
            u.pos_max = u.first + q_len - 1;
            if (p.n_rt > 1) {
                u.pos_min += u.row0 / (int)a.group;
                u.pos_max = u.first + (u.row0 + u.rows - 1) / (int)a.group;
            }
        }
        const int last = min(u.pos_max, u.n - 1);
        if (last >= 0) {
            if (!u.whole && a.window != 0 && u.pos_min >= 0 && (uint32_t)u.pos_min >= a.window) {
                u.first_tile = min((u.pos_min - (int)a.window + 1) / TILE, last / TILE + 1);
                u.n_sink_tiles = (int)min((uint32_t)u.first_tile, a.sinks / TILE + (a.sinks % TILE != 0));
            }
            u.tiles = u.n_sink_tiles + last / TILE + 1 - u.first_tile;
        }
    }
    return u;
}
// What an item counts in the deal: its tiles come after kTcExtra (many-row kernel) that stand for its fixed cost.
template <int TILE>
__device__ __forceinline__ uint32_t item_extra() { return TILE == (int)kTcTile ? kTcExtra : 0; }
template <int TILE>
__device__ __forceinline__ uint32_t item_cost(int tiles) { return tiles ? (uint32_t)tiles + item_extra<TILE>() : 0; }
// The part of the work that a worker has, item by item.
struct Walk {
    uint32_t pos, end;   // tiles still to do, in the order over all items
    uint32_t base;       // tiles before the current unit
    uint32_t s, rt;
    uint32_t total, per, more;  // tiles in all; every share has `per`, the first `more` shares one more
};
// Workers that get work: no share is empty, so a piece lies in every slot that the join looks at.
__device__ __forceinline__ uint32_t used_workers(uint32_t total, uint32_t workers) { return min(total, workers); }
// Which worker's share holds tile t.
__device__ __forceinline__ uint32_t tile_owner(uint32_t t, uint32_t per, uint32_t more)
{
    const uint32_t high = more * (per + 1);
    return t < high ? t / (per + 1) : more + (t - high) / per;
}
// Scans all units (fewer than 2^31 tiles in all) and finds the share of the caller's worker.  A CTA is WORKERS workers
// (1, or one a warp); every thread calls it.  `sh` is 4 * (warps + 2 * WORKERS) bytes of shared memory.
template <int ROWS, int TILE, int THREADS, int WORKERS>
__device__ __forceinline__ Walk plan_walk(const AttnArgs &a, const Pass &p, uint32_t *sh)
{
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32, worker = WORKERS > 1 ? warp : 0;
    const uint32_t per = (p.n_units + THREADS - 1) / THREADS, u0 = min(tid * per, p.n_units), u1 = min(u0 + per, p.n_units);
    auto tiles_of = [&](uint32_t u) {
        return item_cost<TILE>(get_unit<ROWS, TILE>(a, p, p.n_rt > 1 ? u / p.n_rt : u, p.n_rt > 1 ? u % p.n_rt : 0).tiles) * a.n_kv;
    };
    uint32_t mine = 0;
#pragma unroll 1
    for (uint32_t u = u0; u < u1; ++u) mine += tiles_of(u);
    uint32_t inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= (uint32_t)o) inc += x;
    }
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    uint32_t before = inc - mine, total = 0;
#pragma unroll
    for (uint32_t i = 0; i < THREADS / 32; ++i) {
        if (i < warp) before += sh[i];
        total += sh[i];
    }
    const uint32_t n = used_workers(total, p.workers);
    Walk w;
    w.total = total;
    w.per = n ? total / n : 0;
    w.more = total - w.per * n;
    w.pos = w.end = total;
    uint32_t at[WORKERS];  // where each worker's share begins
#pragma unroll
    for (uint32_t k = 0; k < WORKERS; ++k) {
        const uint32_t i = blockIdx.x * WORKERS + k;
        at[k] = i < n ? i * w.per + min(i, w.more) : total;
        if (k == worker && i < n) {
            w.pos = at[k];
            w.end = at[k] + w.per + (i < w.more);
        }
    }
    if (blockIdx.x == 0 && tid == 0) p.begin[p.n_units] = total;
#pragma unroll 1
    for (uint32_t u = u0, b = before; u < u1; ++u) {
        const uint32_t t = per > 1 ? tiles_of(u) : mine;
        if (blockIdx.x == 0) p.begin[u] = b;
#pragma unroll
        for (uint32_t k = 0; k < WORKERS; ++k)
            if (at[k] - b < t) {  // b <= at < b + t
                sh[THREADS / 32 + 2 * k] = b;
                sh[THREADS / 32 + 2 * k + 1] = u;
            }
        b += t;
    }
    __syncthreads();
    w.base = w.s = w.rt = 0;
    if (w.pos < w.end) {
        w.base = sh[THREADS / 32 + 2 * worker];
        const uint32_t u = sh[THREADS / 32 + 2 * worker + 1];
        w.s = p.n_rt > 1 ? u / p.n_rt : u;
        w.rt = p.n_rt > 1 ? u % p.n_rt : 0;
    }
    return w;
}
// The next run of tiles k0 .. k1-1 of one item (unit u, KV head c) that is the worker's; false: no more.  `at` is the place of
// the item's tile 0 in the order over all items.
template <int ROWS, int TILE>
__device__ __forceinline__ bool walk_next(const AttnArgs &a, const Pass &p, Walk &w, Unit &u, uint32_t &c, int &k0, int &k1, uint32_t &at,
                                          uint32_t &item)
{
    constexpr int E = TILE == (int)kTcTile ? (int)kTcExtra : 0;
    while (w.pos < w.end) {
        uint32_t size;
        for (;;) {
            u = get_unit<ROWS, TILE>(a, p, w.s, w.rt);
            size = item_cost<TILE>(u.tiles);
            if (w.pos < w.base + size * a.n_kv) break;
            w.base += size * a.n_kv;
            if (++w.rt == p.n_rt) w.rt = 0, ++w.s;
        }
        const uint32_t in = w.pos - w.base;
        c = a.n_kv > 1 ? in / size : 0;
        const uint32_t from = in - c * size, to = min(size, from + (w.end - w.pos));
        at = w.pos - from + E;
        item = (w.s * p.n_rt + w.rt) * a.n_kv + c;
        w.pos += to - from;
        k0 = max((int)from - E, 0);
        k1 = (int)to - E;
        if (k1 > k0) return true;
    }
    return false;
}
// One thread of a worker, for the border before its share (its first run of tiles): what the join needs to know.
__device__ __forceinline__ void write_cut(const Pass &p, uint32_t worker, const Walk &w, const Unit &u, uint32_t c, int k0, uint32_t at)
{
    Cut x = {};
    if (k0 > 0) {
        x.q0 = u.q0, x.row0 = u.row0, x.rows = u.rows, x.c = c;
        x.c0 = tile_owner(at, w.per, w.more);
        x.c1 = tile_owner(at + u.tiles - 1, w.per, w.more);
    }
    p.cuts[worker] = x;
}
// c += a b: one 16 x 8 x 16 product a warp; the last argument only names the type.
__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

__device__ __forceinline__ float warp_sum(float x)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A lane's D / 32 neighbouring elements of a row.
template <int D> using RowPiece = typename std::conditional<D == 128, uint2, uint32_t>::type;

// One warp adds tokens from .. to - 1, all of them seen, to one (query row, head) in 32 bits: the definition, written down, newest
// token first and four at a time (so that their loads are in flight together).  Lanes split the head dimension; the running
// maximum m, sum l and weighted values o are rescaled when the maximum moves.  `bad`: the lane's columns whose value is in
// question; true once all of them are known not to be finite.
template <class T, int D>
__device__ __noinline__ bool attend_tokens(const AttnArgs &a, const float *q, uint32_t c, const int32_t *table, int from, int to,
                                           uint32_t bad, float &m, float &l, float *o)
{
    constexpr int E = D / 32, N = 4;
    using V = RowPiece<D>;
    const uint64_t head = (uint64_t)c * a.head_stride + (threadIdx.x & 31u) * sizeof(V);
    const uint32_t mask = (1u << a.block_shift) - 1u;
#pragma unroll 1
    for (int t1 = to - 1; t1 >= from; t1 -= N) {
        int id[N];
        V piece[N];
#pragma unroll
        for (int j = 0; j < N; ++j) id[j] = t1 - j >= from ? table[(t1 - j) >> a.block_shift] : -1;
        auto row = [&](int j) { return (uint64_t)id[j] * a.block_stride + (uint64_t)((uint32_t)(t1 - j) & mask) * a.token_stride + head; };
        auto held = [&](int j) { return (uint32_t)id[j] < a.n_blocks; };
#pragma unroll
        for (int j = 0; j < N; ++j) piece[j] = held(j) ? *reinterpret_cast<const V *>(a.k_base + row(j)) : V{};
        float x[N], top = m;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const T *k = reinterpret_cast<const T *>(&piece[j]);
            x[j] = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) x[j] += q[e] * to_f32(k[e]);
            x[j] = warp_sum(x[j]) * a.scale * kLog2e;
            if (!held(j)) x[j] = neg_inf();
            top = fmaxf(top, x[j]);
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (held(j)) piece[j] = *reinterpret_cast<const V *>(a.v_base + row(j));
        const float z = top == neg_inf() ? 0.f : top, f = m == top ? 1.f : exp2f(m - z);
        m = top;
        l *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (!held(j)) continue;
            const T *v = reinterpret_cast<const T *>(&piece[j]);
            const float p = exp2f(x[j] - z);
            l += p;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += p * to_f32(v[e]);
        }
        bool open = false;
#pragma unroll
        for (int e = 0; e < E; ++e) open |= (bad >> e & 1u) && fabsf(o[e]) < INFINITY;
        if (!__any_sync(0xffffffffu, open)) return true;
    }
    return false;
}
// Whether one of the tokens from .. to - 1 has a value that is not finite (called by a whole warp).
template <class T, int D>
__device__ __noinline__ bool any_not_finite(const AttnArgs &a, uint32_t c, const int32_t *table, int from, int to)
{
    constexpr uint32_t kOnes = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;  // the exponent of infinities and NaN
    constexpr int kPieces = D / 8;
    bool found = false;
#pragma unroll 4
    for (int i = (int)(threadIdx.x & 31u); i < (to - from) * kPieces; i += 32) {
        const int t = from + i / kPieces, id = table[t >> a.block_shift];
        if ((uint32_t)id >= a.n_blocks) continue;
        const uint4 v = *reinterpret_cast<const uint4 *>(a.v_base + (uint64_t)id * a.block_stride +
                                                         (uint64_t)(t & ((1 << a.block_shift) - 1)) * a.token_stride +
                                                         (uint64_t)c * a.head_stride + i % kPieces * 16);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) found |= (w[e] & kOnes) == kOnes || (w[e] >> 16 & kOnes) == kOnes;
    }
    return __any_sync(0xffffffffu, found);
}
// The matrix-product kernels multiply a weight of 0 with the values of tokens that some rows of a unit see and others do
// not; where such a value is NaN or infinite the product is NaN.  Rows that come out non-finite are therefore looked at again
// by this, which never touches what a row does not see (called by a whole warp).  Two things keep the cost down where values
// that a row does see make it non-finite, as the definition has it: nothing is done unless a token close to those that the row
// sees (behind it, before its window, after the sinks) holds a non-finite value, and a row is given up as soon as everything in
// it that was non-finite is known to be so.  One infinite value that 2,048 queries over 16k tokens see (32 / 8 heads, 0.6 ms
// without it): 1.4 ms, with all rows done again 5.2 s.  Infinities from the newest 300 tokens on, which some rows of a unit
// see and others do not: 40 ms.
template <class T, int D>
__device__ __noinline__ void attend_row(const AttnArgs &a, int tok, uint32_t h)
{
    constexpr int E = D / 32;
    using V = RowPiece<D>;
    const uint32_t lane = threadIdx.x & 31u, c = h / a.group, s = owner_of_row(a, tok);
    if (s >= a.n_seq) return;
    const int32_t *table = a.table + s * a.table_stride;
    const int n = seq_kv_len(a, s), pos = seq_first(a, s) + tok - seq_q_begin(a, s), last = min(pos, n - 1);
    const int low = a.window && pos >= 0 && (uint32_t)pos >= a.window ? pos - (int)a.window + 1 : 0;
    // how far from what the row sees its unit's tiles go, at most: positions lie (rows - 1) / group + 1 apart, and tiles are whole
    const int reach = (int)((kTcRows - 1) / a.group + kTcTile);
    const int low_end = min(low, last + 1), past = (int)min((long long)pos + 1 + reach, (long long)n);
    const int sinks = (int)min(a.sinks, (uint32_t)max(low_end, 0)), tail = min((sinks + (int)kTcTile - 1) / (int)kTcTile * (int)kTcTile, low_end);
    if (!any_not_finite<T, D>(a, c, table, max(last + 1, 0), past) && !any_not_finite<T, D>(a, c, table, max(low_end - reach, 0), low_end) &&
        !any_not_finite<T, D>(a, c, table, sinks, tail))
        return;
    V *op = reinterpret_cast<V *>(a.out + (uint64_t)tok * a.out_token_stride + (uint64_t)h * a.out_head_stride) + lane;
    const V qv = reinterpret_cast<const V *>(a.q + (uint64_t)tok * a.q_token_stride + (uint64_t)h * a.q_head_stride)[lane];
    V ov = *op;
    float q[E], o[E], m = neg_inf(), l = 0.f;
    uint32_t bad = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] = to_f32(reinterpret_cast<const T *>(&qv)[e]), o[e] = 0.f;
        bad |= fabsf(to_f32(reinterpret_cast<const T *>(&ov)[e])) < INFINITY ? 0u : 1u << e;
    }
    if (attend_tokens<T, D>(a, q, c, table, low, last + 1, bad, m, l, o)) return;
    if (attend_tokens<T, D>(a, q, c, table, 0, sinks, bad, m, l, o)) return;
    const uint32_t g = group_of_seq(a, s);
    if (g < a.n_groups && attend_tokens<T, D>(a, q, c, a.prefix_table + g * a.prefix_stride, 0, prefix_len(a, g), bad, m, l, o)) return;
#pragma unroll
    for (int e = 0; e < E; ++e) reinterpret_cast<T *>(&ov)[e] = from_f32<T>(l == 0.f ? 0.f : o[e] / l);
    *op = ov;
}

// A row's values spread over a warp (lane: D / 32 neighbouring ones), not normalised; maximum (base 2) and sum.
template <int D>
struct Row {
    float m = -INFINITY, l = 0.f, o[D / 32] = {};
};

// Writes a finished row; whether it has a value that is not finite.
template <class T, int D>
__device__ __forceinline__ bool finish(const AttnArgs &a, const Row<D> &x, int tok, uint32_t h)
{
    const uint32_t lane = threadIdx.x & 31u;
    T *op = reinterpret_cast<T *>(a.out + (uint64_t)tok * a.out_token_stride + (uint64_t)h * a.out_head_stride) + lane * (D / 32);
    const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
    bool bad = false;
    T v[D / 32];
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
        const float y = x.l == 0.f ? 0.f : x.o[e] * inv;
        bad |= !(fabsf(y) < kHuge);
        v[e] = from_f32<T>(y);
    }
    if (D == 128) *reinterpret_cast<uint2 *>(op) = *reinterpret_cast<const uint2 *>(v);
    else *reinterpret_cast<uint32_t *>(op) = *reinterpret_cast<const uint32_t *>(v);
    if (a.lse && lane == 0) a.lse[(uint64_t)tok * a.n_heads + h] = x.l == 0.f ? neg_inf() : (x.m + log2f(x.l)) * kLn2;
    return __any_sync(0xffffffffu, bad);
}
#endif

}  // namespace gms
