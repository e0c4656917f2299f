// Attention over the paged KV pool: host entry points and the plan of a call.
#include <cmath>

#include "gms_internal.h"
#include "gms_kv_attn.h"

namespace gms {
namespace {

int bad_pool(const gms_kv_pool *p)
{
    if (!p->base) return GMS_ERR_NULL;
    if (p->block_bytes == 0 || p->block_bytes % kBlockBytes) return GMS_ERR_ALIGN;
    if ((reinterpret_cast<uint64_t>(p->base) | p->plane_stride | p->block_stride) & 15u) return GMS_ERR_ALIGN;
    if (p->block_bytes > kMaxChunkBlocks * kBlockBytes || p->n_blocks == 0 || p->n_blocks > 0x7fffffffu) return GMS_ERR_ARG;
    if (p->block_stride < p->block_bytes && p->n_blocks > 1) return GMS_ERR_ARG;
    if (p->block_stride >> 40 || p->flags & ~GMS_KV_IMAGE_BY_ID) return GMS_ERR_ARG;
    if (p->n_planes > 1 && p->plane_stride < (uint64_t)(p->n_blocks - 1) * p->block_stride + p->block_bytes) return GMS_ERR_ARG;
    return GMS_OK;
}

int bad_layout(const gms_kv_pool *p, const gms_kv_layout *l)
{
    if ((l->token_stride | l->head_stride) & 15u) return GMS_ERR_ALIGN;
    if (l->dtype > GMS_DTYPE_F16 || (l->head_dim != 64 && l->head_dim != 128) || l->n_kv_heads == 0) return GMS_ERR_ARG;
    if (l->block_tokens < 16 || l->block_tokens > 1024 || l->block_tokens & (l->block_tokens - 1)) return GMS_ERR_ARG;
    if (l->k_plane >= p->n_planes || l->v_plane >= p->n_planes || l->k_plane == l->v_plane) return GMS_ERR_ARG;
    const uint64_t row = l->head_dim * 2, heads = l->n_kv_heads, tokens = l->block_tokens;
    const uint64_t ts = l->token_stride, hs = l->head_stride;
    if ((tokens - 1) * ts + (heads - 1) * hs + row > p->block_bytes) return GMS_ERR_ARG;
    const bool tokens_outside = (heads == 1 || hs >= row) && ts >= (heads - 1) * hs + row;
    const bool heads_outside = ts >= row && (heads == 1 || hs >= (tokens - 1) * ts + row);
    return tokens_outside || heads_outside ? GMS_OK : GMS_ERR_ARG;
}

uint32_t log2_of(uint32_t x) { return 31u - (uint32_t)__builtin_clz(x); }

// Checks everything a call is given and fills in the kernels' arguments.  `planning`: workspace pointers are not looked at.
int make_args(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *t, const gms_kv_weight *w,
              const gms_kv_prefix *x, AttnArgs *a)
{
    if (!pool || !layout || !t) return GMS_ERR_NULL;
    int rc = bad_pool(pool);
    if (rc == GMS_OK) rc = bad_layout(pool, layout);
    if (rc != GMS_OK) return rc;
    if (t->n_heads == 0 || t->n_heads % layout->n_kv_heads || !std::isfinite(t->scale)) return GMS_ERR_ARG;
    if (t->total_q > 0x7fffffffu || t->n_seq > 0x7fffffffu || t->max_kv > 1u << 30 || t->max_q > t->total_q) return GMS_ERR_ARG;
    if ((uint64_t)t->total_q * t->n_heads > 0x7fffffffull) return GMS_ERR_RANGE;
    if (!t->cu_q && (t->total_q != t->n_seq || (t->n_seq && t->max_q != 1))) return GMS_ERR_ARG;
    const bool work = t->n_seq && t->total_q;
    if (work && (!t->q || !t->out)) return GMS_ERR_NULL;
    if (t->n_seq && (!t->kv_lens || (t->max_kv && !t->block_table))) return GMS_ERR_NULL;
    if ((reinterpret_cast<uint64_t>(t->q) | reinterpret_cast<uint64_t>(t->out) | t->q_token_stride | t->q_head_stride |
         t->out_token_stride | t->out_head_stride) & 15u)
        return GMS_ERR_ALIGN;
    if ((reinterpret_cast<uint64_t>(t->lse) | reinterpret_cast<uint64_t>(t->cu_q) | reinterpret_cast<uint64_t>(t->kv_lens) |
         reinterpret_cast<uint64_t>(t->block_table)) & 3u || reinterpret_cast<uint64_t>(t->status) & 7u ||
        reinterpret_cast<uint64_t>(t->workspace) & 255u)
        return GMS_ERR_ALIGN;
    if (t->table_stride > (1ull << 40) || t->table_stride * layout->block_tokens < t->max_kv) return GMS_ERR_RANGE;
    *a = {};
    a->k_base = static_cast<const uint8_t *>(pool->base) + layout->k_plane * pool->plane_stride;
    a->v_base = static_cast<const uint8_t *>(pool->base) + layout->v_plane * pool->plane_stride;
    a->block_stride = pool->block_stride;
    a->n_blocks = pool->n_blocks;
    a->token_stride = layout->token_stride;
    a->head_stride = layout->head_stride;
    a->block_shift = log2_of(layout->block_tokens);
    a->q = static_cast<const uint8_t *>(t->q);
    a->out = static_cast<uint8_t *>(t->out);
    a->lse = t->lse;
    a->cu_q = t->cu_q;
    a->kv_lens = t->kv_lens;
    a->table = t->block_table;
    a->table_stride = t->table_stride;
    a->q_token_stride = t->q_token_stride;
    a->q_head_stride = t->q_head_stride;
    a->out_token_stride = t->out_token_stride;
    a->out_head_stride = t->out_head_stride;
    a->n_seq = t->n_seq;
    a->n_heads = t->n_heads;
    a->n_kv = layout->n_kv_heads;
    a->group = t->n_heads / layout->n_kv_heads;
    a->total_q = t->total_q;
    a->max_q = t->max_q;
    a->max_kv = t->max_kv;
    a->window = t->window;
    a->sinks = t->sinks;
    a->scale = t->scale;
    a->status = reinterpret_cast<unsigned long long *>(t->status);
    if (w) {
        if (w->reserved) return GMS_ERR_ARG;
        if (t->n_seq && t->max_kv && !w->out) return GMS_ERR_NULL;
        if ((reinterpret_cast<uint64_t>(w->in) | reinterpret_cast<uint64_t>(w->out)) & 3u) return GMS_ERR_ALIGN;
        if (!std::isfinite(w->decay)) return GMS_ERR_ARG;
        if ((uint64_t)t->n_seq * layout->n_kv_heads * t->max_kv > (1ull << 32)) return GMS_ERR_RANGE;
        a->w_in = w->in;
        a->w_out = w->out;
        a->w_seq_stride = w->seq_stride;
        a->w_head_stride = w->head_stride;
        a->decay = w->decay;
    }
    if (x) {
        if (t->window || t->sinks || x->reserved || x->max_prefix > 1u << 30 || x->n_groups > t->n_seq || x->max_group_q > t->total_q)
            return GMS_ERR_ARG;
        if (x->n_groups && (!x->group_start || !x->prefix_lens || (x->max_prefix && !x->prefix_table))) return GMS_ERR_NULL;
        if ((reinterpret_cast<uint64_t>(x->group_start) | reinterpret_cast<uint64_t>(x->prefix_lens) |
             reinterpret_cast<uint64_t>(x->prefix_table)) & 3u)
            return GMS_ERR_ALIGN;
        if (x->prefix_stride > (1ull << 40) || (x->n_groups && x->prefix_stride * layout->block_tokens < x->max_prefix))
            return GMS_ERR_RANGE;
        a->group_start = x->group_start;
        a->prefix_lens = x->prefix_lens;
        a->prefix_table = x->prefix_table;
        a->prefix_stride = x->prefix_stride;
        a->n_groups = x->n_groups;
        a->max_prefix = x->max_prefix;
        a->max_group_q = x->max_group_q;
    }
    return GMS_OK;
}

using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                            const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                            CUtensorMapFloatOOBfill);
Encode encoder()
{
    static const Encode encode = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<Encode>(p);
    }();
    return encode;
}
int encode_map(CUtensorMap *m, uint32_t dtype, uint32_t rank, const void *base, const cuuint64_t *dims, const cuuint64_t *strides,
               const cuuint32_t *box)
{
    const Encode encode = encoder();
    if (!encode) return report_cuda_error(cudaErrorNotSupported);
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(m, dtype == GMS_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank,
                              const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? GMS_OK : report_cuda_error(cudaErrorInvalidValue);
}
// One layer's keys or values.  For the many-row kernel (d, token of block, head, block), boxes of 64 elements x `box_tokens`
// tokens; for the few-row kernel (d mod 64, token of block, d / 64, head, block), boxes of whole rows.
int encode_pool(CUtensorMap *m, const gms_kv_pool *pool, const gms_kv_layout *l, uint32_t plane, uint32_t box_tokens, bool whole_rows)
{
    // a stride along a dimension of one element is never used, but has to be a legal one
    const cuuint64_t head = l->n_kv_heads > 1 ? l->head_stride : l->token_stride;
    const cuuint64_t block = pool->n_blocks > 1 ? pool->block_stride : pool->block_bytes;
    const uint8_t *base = static_cast<const uint8_t *>(pool->base) + plane * pool->plane_stride;
    if (whole_rows) {
        const cuuint64_t dims[5] = {64, l->block_tokens, l->head_dim / 64, l->n_kv_heads, pool->n_blocks};
        const cuuint64_t strides[4] = {l->token_stride, 128, head, block};
        const cuuint32_t box[5] = {64, box_tokens, l->head_dim / 64, 1, 1};
        return encode_map(m, l->dtype, 5, base, dims, strides, box);
    }
    const cuuint64_t dims[4] = {l->head_dim, l->block_tokens, l->n_kv_heads, pool->n_blocks};
    const cuuint64_t strides[3] = {l->token_stride, head, block};
    const cuuint32_t box[4] = {64, box_tokens, 1, 1};
    return encode_map(m, l->dtype, 4, base, dims, strides, box);
}
// The queries as (d, head, token): 128 rows are the `group` heads of 128 / group tokens.  False where that does not come out even,
// where the strides are not a tensor map's (heads or tokens that share bytes), or where the scale's sign has to go into Q.
bool q_boxes(const AttnArgs &a, uint32_t head_dim)
{
    return a.scale > 0.f && 128 % a.group == 0 && a.q_head_stride >= head_dim * 2 && a.q_token_stride >= head_dim * 2 &&
           a.q_head_stride < (1ull << 40) && a.q_token_stride < (1ull << 40);
}
int encode_q(CUtensorMap *m, const AttnArgs &a, uint32_t dtype, uint32_t head_dim)
{
    const cuuint64_t dims[3] = {head_dim, a.n_heads, a.total_q}, strides[2] = {a.q_head_stride, a.q_token_stride};
    const cuuint32_t box[3] = {64, a.group, 128 / a.group};
    return encode_map(m, dtype, 3, a.q, dims, strides, box);
}

struct Carve {  // hands out 256-byte aligned pieces of the workspace; with a null base it only counts
    uint8_t *base;
    uint64_t used = 0;
    template <class T> T *take(uint64_t n)
    {
        T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
        used += (n * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

struct Plan {
    Pass own, prefix;
    bool shared, logits;
    float *lse;  // where the weights pass finds the log-sum-exps
};

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Most tiles an item can have, from what the host knows; most tiles of a pass.
uint64_t item_tiles(const AttnArgs &a, const Pass &p)
{
    uint64_t span = p.prefix ? a.max_prefix : a.max_kv;
    if (!p.prefix && a.window) {
        const uint64_t seen = (uint64_t)a.window + a.sinks + 2 * p.tile + (p.rows - 1) / a.group;
        if (seen < span) span = seen;
    }
    return ceil_div(span, p.tile) + (p.tile == kTcTile ? kTcExtra : 0);
}
uint64_t most_tiles(const AttnArgs &a, const Pass &p)
{
    return p.n_units >= 1u << 30 ? 1ull << 31 : p.n_units * (uint64_t)a.n_kv * item_tiles(a, p);
}

uint64_t pass_rows(const AttnArgs &a, bool prefix) { return (uint64_t)(prefix ? a.max_group_q : a.max_q) * a.group; }
void cut_pass(const AttnArgs &a, bool prefix, bool tc, uint64_t rows, Pass *p)
{
    p->prefix = prefix;
    p->rows = tc ? kTcRows : kFewRows;
    p->tile = tc ? kTcTile : kFewTile;
    p->n_rt = (uint32_t)ceil_div(rows, p->rows);
    if (p->n_rt == 0) p->n_rt = 1;
    const uint64_t units = (uint64_t)(prefix ? a.n_groups : a.n_seq) * p->n_rt;
    p->n_units = (uint32_t)(units < 0xffffffffull ? units : 0xffffffffull);  // too many: most_tiles refuses them
    // as many workers as the SMs hold; fewer where they would have fewer than two tiles
    const uint64_t want = ceil_div(most_tiles(a, *p), 2), most = tc ? kTcMaxWorkers : kFewMaxWorkers;
    p->workers = (uint32_t)(want < 1 ? 1 : want < most ? want : most);
    p->slot_rows = rows < p->rows ? (uint32_t)(rows < 1 ? 1 : rows) : p->rows;
}

// Few-row kernel: whether a CTA takes a whole item (its four warps share the tiles; no plan, no pieces, one kernel) or all tiles
// are dealt out evenly.  Measured, us a call, 32 / 8 heads of 128, lengths n/2 .. n (even deal / CTA an item):
//   sequences   n = 64       260          512          1,024        2,048
//       1       9.6 / 5.1    12.5 / 9.4   10.6 / 11.0  10.8 / 17.9
//      16      13.8 / 7.5    14.9 / 9.8   17.6 / 13.3  21.3 / 20.4  29.6 / 34.1
//      32      14.5 / 6.9    17.7 / 12.6  21.2 / 16.2  29.1 / 24.0  44.7 / 41.3
//      48      14.8 / 11.7   20.4 / 20.0  24.8 / 25.2  37.2 / 37.9  60.2 / 63.9
//      64      17.8 / 12.4   24.5 / 21.4  32.5 / 27.3  48.3 / 43.7  79.9 / 74.4
//     256      27.8 / 41.4   54.0 / 64.1  85.1 / 86.4  148 / 136    272 / 244
// A CTA an item loses where few items leave SMs idle for long, where one wave of CTAs is a little more than full, and where
// very many items are very short; beyond 128 tiles (2,048 tokens) the even deal's balance is worth its join.
// The rule takes the slower side at five of these points: 64 sequences of 64 tokens (17.8 for 12.4), and four that lose 2 to 4 %
// (1 of 512, 16 of 1,024, 48 of 512, 256 of 512).  It goes by max_kv: a call that announces far more than its sequences have (a
// graph captured once for all lengths) is dealt evenly.
bool team_deal(uint64_t items, uint64_t tiles)
{
    const uint64_t held = kFewMaxWorkers / kFewWarps;  // CTAs that the SMs hold at once
    if (tiles > 128) return false;
    if (items <= held) return tiles * (held - items) <= 32 * (held - 8);
    return items < 512 ? tiles <= 32 : 64 * tiles >= items;
}

constexpr uint64_t kFewMostRows = 64;  // of a unit that goes to the few-row kernel

void plan_pass(const AttnArgs &a, uint32_t head_dim, bool prefix, bool rows_out, Carve *c, Pass *p)
{
    *p = {};
    const uint64_t rows = pass_rows(a, prefix);
    // Up to 16 rows a KV head: the few-row kernel, which reads K and V once.  More: the tensor-core kernel reads them once for
    // 256 rows, but takes 8 us longer to get going (its Q, descriptors and tensor memory; 16 us against 8 us for one tile), so
    // short calls of up to 64 rows go to the few-row kernel all the same, 16 rows at a time: where no warp gets more than four
    // of its tiles (three suffixes of 40 behind a prefix of 129 tokens, 24 rows: 15 us against 23 us).
    bool tc = rows > kFewRows;
    cut_pass(a, prefix, false, rows, p);
    if (tc && rows <= kFewMostRows && most_tiles(a, *p) <= 4ull * kFewMaxWorkers) tc = false;
    if (tc) cut_pass(a, prefix, true, rows, p);
    if (!tc) p->team = team_deal((uint64_t)p->n_units * a.n_kv, item_tiles(a, *p));
    if (p->team) p->workers = 1;
    p->begin = c->take<uint32_t>((uint64_t)p->n_units + 1);
    p->cuts = c->take<Cut>(p->workers);
    p->part_ml = c->take<float2>(2ull * p->workers * p->slot_rows);
    p->part_o = c->take<float>(2ull * p->workers * p->slot_rows * head_dim);
    if (rows_out) {
        p->row_ml = c->take<float2>((uint64_t)a.total_q * a.n_heads);
        p->row_o = c->take<float>((uint64_t)a.total_q * a.n_heads * head_dim);
    }
    p->again = a.max_q > 1;  // with one query a sequence, what its rows do not see is cleared before the product
    if (tc && p->again && !rows_out) p->redo = c->take<uint32_t>((uint64_t)p->n_units * a.n_kv * (kTcRows / 32));
}

// What the plan above takes at most, for this call and for every one with no larger numbers: a smaller call may be cut in a
// way that takes more than this one's (items dealt out instead of a CTA each, the other kernel, logits kept).  Every term grows
// with n_seq, max_q, max_kv, total_q and a prefix's numbers alone.
void most_of_pass(const AttnArgs &a, uint32_t head_dim, bool prefix, bool rows_out, Carve *c)
{
    const uint64_t rows = pass_rows(a, prefix);
    Pass few = {}, many = {};
    cut_pass(a, prefix, false, rows < kFewMostRows ? rows : kFewMostRows, &few);
    if (rows > kFewRows) cut_pass(a, prefix, true, rows, &many);
    auto larger = [](uint64_t x, uint64_t y) { return x > y ? x : y; };
    const uint64_t slots = 2 * larger((uint64_t)few.workers * few.slot_rows, (uint64_t)many.workers * many.slot_rows);
    c->take<uint32_t>(larger(few.n_units, many.n_units) + 1);
    c->take<Cut>(larger(few.workers, many.workers));
    c->take<float2>(slots);
    c->take<float>(slots * head_dim);
    if (rows_out) {
        c->take<float2>((uint64_t)a.total_q * a.n_heads);
        c->take<float>((uint64_t)a.total_q * a.n_heads * head_dim);
    } else if (a.max_q > 1) {
        c->take<uint32_t>((uint64_t)many.n_units * a.n_kv * (kTcRows / 32));
    }
}
// Logits are kept tile by tile as the few-row kernel takes them, so under a window only for what it reaches.
uint64_t logit_stride(const AttnArgs &a)
{
    Pass p = {};
    p.rows = kFewRows, p.tile = kFewTile;
    return item_tiles(a, p) * kFewTile;
}
uint64_t most_of_call(const AttnArgs &a, uint32_t head_dim, bool shared)
{
    Carve c{nullptr};
    most_of_pass(a, head_dim, false, shared, &c);
    if (shared) most_of_pass(a, head_dim, true, true, &c);
    if (a.w_out) {
        if (!a.lse) c.take<float>((uint64_t)a.total_q * a.n_heads);
        const uint32_t kept = kFewRows / a.group;  // queries whose logits are kept
        c.take<float>((uint64_t)a.n_seq * a.n_heads * (a.max_q < kept ? a.max_q : kept) * logit_stride(a));
    }
    return c.used;
}

int plan_call(const AttnArgs &a, uint32_t head_dim, bool shared, void *workspace, Plan *pl, uint64_t *bytes)
{
    *pl = {};
    Carve c{static_cast<uint8_t *>(workspace)};
    pl->shared = shared;
    plan_pass(a, head_dim, false, shared, &c, &pl->own);
    if (shared) plan_pass(a, head_dim, true, true, &c, &pl->prefix);
    pl->lse = a.lse;
    if (a.w_out) {
        if (!a.lse) pl->lse = c.take<float>((uint64_t)a.total_q * a.n_heads);
        if (pl->own.rows == kFewRows && pl->own.n_rt == 1) {
            pl->logits = true;
            pl->own.logit_stride = (uint32_t)logit_stride(a);
            pl->own.logits = c.take<float>((uint64_t)a.n_seq * a.n_heads * a.max_q * pl->own.logit_stride);
        }
    }
    const uint64_t most = most_of_call(a, head_dim, shared);
    *bytes = c.used > most ? c.used : most;
    // the kernels count tiles in 31 bits
    const bool fits = most_tiles(a, pl->own) >> 31 == 0 && (!shared || most_tiles(a, pl->prefix) >> 31 == 0);
    return fits ? GMS_OK : GMS_ERR_RANGE;
}

int attention_call(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *t, const gms_kv_weight *w,
                   const gms_kv_prefix *x, void *stream)
{
    AttnArgs a;
    int rc = make_args(pool, layout, t, w, x, &a);
    if (rc != GMS_OK) return rc;
    Plan pl;
    uint64_t need = 0;
    rc = plan_call(a, layout->head_dim, x != nullptr, t->workspace, &pl, &need);
    if (rc != GMS_OK) return rc;
    if (a.n_seq == 0) return GMS_OK;
    if (!t->workspace) return GMS_ERR_NULL;
    if (need > t->workspace_bytes) return GMS_ERR_RANGE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint32_t dtype = layout->dtype, dim = layout->head_dim;
    cudaError_t e = cudaSuccess;
    if (a.total_q) {
        AttnArgs b = a;
        b.lse = pl.lse;
        CUtensorMap kmap[2], vmap[2];  // boxes of the few-row and of the many-row kernel
        const uint32_t box = layout->block_tokens < kTcTile ? layout->block_tokens : kTcTile;
        const bool prefix = pl.shared && pl.prefix.n_units;
        pl.own.behind = prefix;
        for (int i = 0; i < 2; ++i) {
            const uint32_t rows = i ? kTcRows : kFewRows;
            if (pl.own.rows != rows && !(prefix && pl.prefix.rows == rows)) continue;
            rc = encode_pool(&kmap[i], pool, layout, layout->k_plane, i ? box : kFewTile, i == 0);
            if (rc == GMS_OK) rc = encode_pool(&vmap[i], pool, layout, layout->v_plane, i ? box : kFewTile, i == 0);
            if (rc != GMS_OK) return rc;
        }
        CUtensorMap qmap;
        const bool tc = pl.own.rows == kTcRows || (prefix && pl.prefix.rows == kTcRows), q_tma = tc && q_boxes(a, dim);
        if (q_tma) rc = encode_q(&qmap, a, dtype, dim);
        if (rc != GMS_OK) return rc;
        auto launch = [&](const Pass &p) {
            return p.rows == kTcRows ? launch_kv_attn_tc(b, p, kmap[1], vmap[1], q_tma ? &qmap : nullptr, box, dtype, dim, s)
                                     : launch_kv_attn_few(b, p, kmap[0], vmap[0], dtype, dim, s);
        };
        if (prefix) e = launch(pl.prefix);
        if (e == cudaSuccess) e = launch(pl.own);
        if (e == cudaSuccess)
            e = pl.shared ? launch_kv_attn_join_shared(b, pl.prefix, pl.own, dtype, dim, s)
                          : pl.own.team ? cudaSuccess : launch_kv_attn_join(b, pl.own, dtype, dim, s);
        if (e == cudaSuccess && w && pl.logits) e = launch_kv_few_weights(b, pl.own, s);
    }
    if (e == cudaSuccess && w && !(a.total_q && pl.logits)) e = launch_kv_weights(a, pl.lse, a.total_q != 0, dtype, dim, s);
    return e == cudaSuccess ? GMS_OK : report_cuda_error(e);
}

}  // namespace
}  // namespace gms

extern "C" {

int gms_kv_attention_workspace(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                               const gms_kv_weight *weight, uint64_t *nbytes)
{
    if (!nbytes) return GMS_ERR_NULL;
    gms::AttnArgs a;
    int rc = gms::make_args(pool, layout, attn, weight, nullptr, &a);
    gms::Plan plan;
    if (rc == GMS_OK) rc = gms::plan_call(a, layout->head_dim, false, nullptr, &plan, nbytes);
    return rc;
}

int gms_kv_attention(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn, const gms_kv_weight *weight,
                     void *stream)
{
    return gms::attention_call(pool, layout, attn, weight, nullptr, stream);
}

int gms_kv_attention_shared_workspace(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                                      const gms_kv_prefix *prefix, uint64_t *nbytes)
{
    if (!nbytes || !prefix) return GMS_ERR_NULL;
    gms::AttnArgs a;
    int rc = gms::make_args(pool, layout, attn, nullptr, prefix, &a);
    gms::Plan plan;
    if (rc == GMS_OK) rc = gms::plan_call(a, layout->head_dim, true, nullptr, &plan, nbytes);
    return rc;
}

int gms_kv_attention_shared(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_attn *attn,
                            const gms_kv_prefix *prefix, void *stream)
{
    if (!prefix) return GMS_ERR_NULL;
    return gms::attention_call(pool, layout, attn, nullptr, prefix, stream);
}

int gms_kv_evict(const gms_kv_pool *pool, const gms_kv_layout *layout, const gms_kv_evict_args *t, void *stream)
{
    if (!pool || !layout || !t) return GMS_ERR_NULL;
    int rc = gms::bad_pool(pool);
    if (rc == GMS_OK) rc = gms::bad_layout(pool, layout);
    if (rc != GMS_OK) return rc;
    if (t->reserved || t->max_len > 1u << 30 || t->budget > 1u << 30 || (uint64_t)t->sinks + t->recent > t->budget)
        return GMS_ERR_ARG;
    if (t->n_layers) {
        const uint64_t last = (uint64_t)(t->n_layers - 1) * t->layer_planes;
        const uint32_t apart = layout->k_plane > layout->v_plane ? layout->k_plane - layout->v_plane : layout->v_plane - layout->k_plane;
        if (last + (layout->k_plane > layout->v_plane ? layout->k_plane : layout->v_plane) >= pool->n_planes) return GMS_ERR_ARG;
        // two layers must not share a plane
        if (t->n_layers > 1 && (t->layer_planes == 0 || (apart % t->layer_planes == 0 && apart / t->layer_planes < t->n_layers)))
            return GMS_ERR_ARG;
    }
    if ((reinterpret_cast<uint64_t>(t->weights) | reinterpret_cast<uint64_t>(t->weights_out) | reinterpret_cast<uint64_t>(t->lens) |
         reinterpret_cast<uint64_t>(t->lens_out) | reinterpret_cast<uint64_t>(t->src_table) | reinterpret_cast<uint64_t>(t->dst_table) |
         reinterpret_cast<uint64_t>(t->kept)) & 3u || reinterpret_cast<uint64_t>(t->status) & 7u)
        return GMS_ERR_ALIGN;
    const uint64_t rows = (uint64_t)t->n_layers * t->n_seq * layout->n_kv_heads;
    const uint32_t most = t->max_len < t->budget ? t->max_len : t->budget;
    if (rows > 0x7fffffffull || rows * ((most + 63ull) / 64) > 0x7fffffffull) return GMS_ERR_RANGE;
    if (t->src_stride > (1ull << 40) || t->dst_stride > (1ull << 40) || t->src_stride * layout->block_tokens < t->max_len ||
        t->dst_stride * layout->block_tokens < most)
        return GMS_ERR_RANGE;
    if (rows == 0) return GMS_OK;
    if (!t->lens || (t->max_len && (!t->weights || !t->src_table)) || (t->budget && !t->kept) || (most && !t->dst_table))
        return GMS_ERR_NULL;
    if (t->weights_out && t->weights_out == t->weights) return GMS_ERR_ARG;
    if (t->lens_out && t->lens_out != t->lens && t->lens_out < t->lens + t->n_seq && t->lens < t->lens_out + t->n_seq) return GMS_ERR_ARG;
    gms::EvictArgs a = {};
    a.base = static_cast<uint8_t *>(pool->base);
    a.plane_stride = pool->plane_stride;
    a.block_stride = pool->block_stride;
    a.k_plane = layout->k_plane;
    a.v_plane = layout->v_plane;
    a.n_blocks = pool->n_blocks;
    a.token_stride = layout->token_stride;
    a.head_stride = layout->head_stride;
    a.block_shift = gms::log2_of(layout->block_tokens);
    a.row_bytes = layout->head_dim * 2;
    a.weights = t->weights;
    a.weights_out = t->weights_out;
    a.lens = t->lens;
    a.lens_out = t->lens_out;
    a.src_table = t->src_table;
    a.dst_table = t->dst_table;
    a.kept = t->kept;
    a.w_layer_stride = t->w_layer_stride;
    a.w_seq_stride = t->w_seq_stride;
    a.w_head_stride = t->w_head_stride;
    a.o_layer_stride = t->o_layer_stride;
    a.o_seq_stride = t->o_seq_stride;
    a.o_head_stride = t->o_head_stride;
    a.src_stride = t->src_stride;
    a.dst_stride = t->dst_stride;
    a.n_layers = t->n_layers;
    a.layer_planes = t->layer_planes;
    a.n_seq = t->n_seq;
    a.n_kv = layout->n_kv_heads;
    a.max_len = t->max_len;
    a.budget = t->budget;
    a.sinks = t->sinks;
    a.recent = t->recent;
    a.status = reinterpret_cast<unsigned long long *>(t->status);
    const cudaError_t e = gms::launch_kv_evict(a, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? GMS_OK : gms::report_cuda_error(e);
}

}  // extern "C"
