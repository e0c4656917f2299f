// Attention of few query rows (at most 16 a KV head: one token of a grouped-query model, or a few) over the paged pool.
//
// Bound: memory.  Every visible K and V row is read once; 16 rows of mma.sync per 256-byte row are far below the tensor
// rate, so the legacy matrix instruction is enough and what counts is bytes in flight and an even deal (see Pass).
// Every warp is a worker of its own, as in the streaming kernels: tiles of 16 tokens come by TMA through the block table into
// the warp's ring (K and V of one KV head, one box of whole rows each, 128-byte swizzle, so that ldmatrix has no bank
// conflicts), and no warp waits for another.  S = Q K^T, the online softmax and O += P V stay in registers.
// For short items (TEAM) a CTA takes a whole item: its warps share the tiles and join at the end, there is no plan and no second
// kernel.  The rule and both sides' times stand where the call is planned.
// The loads carry an evict-first hint: K and V are read once, and the kernels' own code, fetched again for every launch, stays
// in L2 (64 suffixes behind a prefix of 8,192: 86 us without, 74 us with it).
// Measured: 48 sequences of up to 12,001 tokens, 2,048 + 4 visible, 32 / 8 heads of 128, bf16: 73 us for 360 MB = 4.9 TB/s,
// about 8 us of it launch, plan and first tiles; DRAM reads 364 MB, nothing is read twice.  8 x 65k tokens on one KV head: 43 us.
// One sequence under a window of 256 and 4 sinks: 10 us, three of them launch and the first code fetches.
#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_ptx.h"

namespace gms {
namespace {

using namespace ptx;

constexpr int kWarps = (int)kFewWarps, kThreads = kWarps * 32;

// A run of tiles of one item, from the issue side to the arithmetic side of a warp (which may be several short items behind).
struct Run {
    int q0, row0, rows, n, first, pos_min, pos_max, n_sink_tiles, first_tile, tiles, k0, k1;
    uint32_t c, seq, whole, pad;
};
constexpr uint32_t kRuns = 8;  // more than stages

template <int D>
struct Few {
    static constexpr int kHalves = D / 64;
    static constexpr uint32_t kStageBytes = 2 * kHalves * 2048;          // K then V, 16 tokens x 128 bytes a half
    static constexpr int kStages = D == 128 ? 3 : 6;                      // so that two CTAs share an SM
    static constexpr uint32_t kRing = kStages * kStageBytes;             // a warp's
    static constexpr uint32_t kSmem = kWarps * kRing + kWarps * (kStages * 8 + kRuns * sizeof(Run)) + 4 * (kWarps + 2 * kWarps) + 1024;
};

// Registers of a warp's running softmax over its share of an item.
template <int D>
struct Acc {
    float o[D / 8][4], m[2], l[2];
};

// HI: the units have more than 8 rows (the upper half of the 16-row fragments is in use).  TEAM: see Pass.
template <class T, int D, bool HI, bool TEAM>
__global__ void __launch_bounds__(kThreads, 2) kv_attn_few_kernel(const __grid_constant__ CUtensorMap kmap,
                                                                  const __grid_constant__ CUtensorMap vmap,
                                                                  const __grid_constant__ AttnArgs a, const __grid_constant__ Pass p)
{
    using F = Few<D>;
    constexpr int S = F::kStages, NJ = D / 8;
    // fp16 weights are kept 2^15 times larger, the largest that fits: else those below 2^-25 of the maximum were nothing to the
    // product with V, however many there are, and counted in l all the same
    constexpr float kUp = std::is_same<T, __half>::value ? 15.f : 0.f;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid / 32;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *sm = smem_raw + (base - smem_u32(smem_raw));
    const uint32_t ring = base + warp * F::kRing;
    uint64_t *bars = reinterpret_cast<uint64_t *>(sm + kWarps * F::kRing);
    Run *runs = reinterpret_cast<Run *>(bars + kWarps * S) + warp * kRuns;
    uint32_t *plan = reinterpret_cast<uint32_t *>(reinterpret_cast<Run *>(bars + kWarps * S) + kWarps * kRuns);
    const uint32_t bar = smem_u32(bars + warp * S);
    if (lane == 0) {
        for (int i = 0; i < S; ++i) mbar_init(bar + 8 * i, 1);
        fence_mbar_init();
        if (warp == 0) {
            tma_prefetch_map(&kmap);
            tma_prefetch_map(&vmap);
        }
    }
    if (!p.behind) grid_wait();
    grid_launch_dependents();
    Walk w = {};
    if (!TEAM) w = plan_walk<kFewRows, kFewTile, kThreads, kWarps>(a, p, plan);
    const uint32_t worker = blockIdx.x * kWarps + warp;

    const float c2 = a.scale * kLog2e;
    const uint32_t tok_mask = (1u << a.block_shift) - 1u;
    // K and V are read once by the call (more row tiles: several times): they go first, and code, tables and pieces stay in L2
    const uint64_t policy = p.n_rt == 1 ? policy_evict_first() : policy_evict_normal();
    const int r0 = (int)lane / 4, r1 = r0 + 8;
    uint32_t put = 0, got = 0;   // stages issued / consumed
    uint32_t ahead = 0, cur = 0; // runs seen by the issue side / by the arithmetic
    uint32_t holes = 0;          // a bit for each stage that holds a hole
    // issue side: tiles ik .. ik1-1 of its run, block ids of tiles ibase + lane
    const int32_t *itable = nullptr;
    int ik = 0, ik1 = 0, isink = 0, ishift = 0, ibase = 0, ids = 0;
    uint32_t ic = 0;
    bool more = true;
    // arithmetic side
    Run run = {};
    int ck = 0;
    uint32_t q[D / 16][4];
    int p0 = 0, p1 = 0;
    Acc<D> x = {};
    x.m[0] = x.m[1] = neg_inf();
    // Every part of the loop stands in the code once: a short call is bound by fetching instructions.
#pragma unroll 1
    for (;;) {
#pragma unroll 1
        while (put - got < (uint32_t)S) {
            if (ik == ik1) {
                if (!more) break;
                Unit un = {};
                int k0 = 0, k1 = 0;
                uint32_t at = 0, item = 0;
                if (TEAM) {
                    item = blockIdx.x;
                    un = get_unit<kFewRows, kFewTile>(a, p, item / a.n_kv / p.n_rt, item / a.n_kv % p.n_rt);
                    ic = item % a.n_kv;
                    k0 = un.tiles * (int)warp / kWarps;
                    k1 = un.tiles * (int)(warp + 1) / kWarps;
                    more = ahead == 0 && k1 > k0;
                } else {
                    more = walk_next<kFewRows, kFewTile>(a, p, w, un, ic, k0, k1, at, item);
                    if (ahead == 0 && lane == 0 && worker < p.workers) write_cut(p, worker, w, un, ic, more ? k0 : 0, at);
                }
                if (!more) break;
                if (lane == 0) {
                    Run &r = runs[ahead % kRuns];
                    r.q0 = un.q0, r.row0 = un.row0, r.rows = un.rows, r.n = un.n, r.first = un.first, r.pos_min = un.pos_min, r.pos_max = un.pos_max;
                    r.n_sink_tiles = un.n_sink_tiles, r.first_tile = un.first_tile, r.tiles = un.tiles, r.k0 = k0, r.k1 = k1;
                    r.c = ic, r.seq = item / a.n_kv, r.whole = un.whole;
                }
                __syncwarp();
                ++ahead;
                itable = un.table, isink = un.n_sink_tiles, ishift = un.first_tile - un.n_sink_tiles;
                ik = k0, ik1 = k1, ibase = k0 - 32;
            }
            if (ik - ibase == 32) {
                ibase = ik;
                const int k = ik + (int)lane;
                ids = k < ik1 ? itable[(uint32_t)((k < isink ? k : k + ishift) * kFewTile) >> a.block_shift] : -1;
            }
            const int id = __shfl_sync(0xffffffffu, ids, ik - ibase);
            const uint32_t st = put % S;
            const bool hole = (uint32_t)id >= a.n_blocks;
            holes = hole ? holes | 1u << st : holes & ~(1u << st);
            if (lane == 0) {
                const uint32_t dst = ring + st * F::kStageBytes, b = bar + 8 * st;
                const int y = (int)((uint32_t)((ik < isink ? ik : ik + ishift) * kFewTile) & tok_mask);
                const int blk = hole ? (int)a.n_blocks : id;  // a hole: out of range, zeros arrive
                mbar_expect(b, F::kStageBytes);
                tma_load_5d(dst, &kmap, 0, y, 0, (int)ic, blk, b, policy);
                tma_load_5d(dst + F::kHalves * 2048, &vmap, 0, y, 0, (int)ic, blk, b, policy);
            }
            ++ik;
            ++put;
        }
        if (got == put) break;
        if (ck == run.k1) {  // the next run: its query rows as matrix fragments (rows that do not exist are zero)
            run = runs[cur % kRuns];
            ++cur;
            ck = run.k0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = i ? r1 : r0;
                const bool on = r < run.rows;
                const int row = run.row0 + (on ? r : 0);
                const uint32_t h = run.c * a.group + (uint32_t)row % a.group;
                const int tok = run.q0 + row / (int)a.group;
                const uint32_t *qp = reinterpret_cast<const uint32_t *>(a.q + (uint64_t)tok * a.q_token_stride + h * a.q_head_stride) + (lane & 3u);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    q[kk][i] = on ? qp[kk * 8] : 0u;
                    q[kk][i + 2] = on ? qp[kk * 8 + 4] : 0u;
                }
                (i ? p1 : p0) = run.whole ? run.n - 1 : run.first + (run.row0 + r) / (int)a.group;
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) x.o[j][e] = 0.f;
            x.m[0] = x.m[1] = neg_inf();
            x.l[0] = x.l[1] = 0.f;
        }
        {
            const uint32_t st = got % S, kt = ring + st * F::kStageBytes, vt = kt + F::kHalves * 2048;
            if (!__all_sync(0xffffffffu, mbar_wait(bar + 8 * st, (got / S) & 1u))) {
                // give up: no more copies; those in flight are waited for (bounded)
                if (lane == 0 && a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_TIMEOUT);
                for (; got != put; ++got) (void)mbar_wait(bar + 8 * (got % S), (got / S) & 1u);
                break;
            }
            const int t0 = (ck < run.n_sink_tiles ? ck : run.first_tile + ck - run.n_sink_tiles) * kFewTile;
            const bool hole = holes >> st & 1u;
            float s[2][4];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[j][e] = 0.f;
            const uint32_t krow = (lane & 7u) + ((lane >> 4) << 3);  // token of this lane's ldmatrix row
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t ch = (kk & 3) * 2 + ((lane >> 3) & 1u);
                uint32_t b[4];
                ldmatrix_x4(kt + (kk / 4) * 2048 + krow * 128 + ((ch ^ (krow & 7u)) << 4), b);
                mma16816(s[0], q[kk], b[0], b[1], T());
                mma16816(s[1], q[kk], b[2], b[3], T());
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[j][e] *= c2;
            const int t1 = t0 + kFewTile - 1;
            const bool full = !hole && t1 <= run.pos_min && t1 < run.n &&
                              (run.whole || a.window == 0 || (long long)t0 > (long long)run.pos_max - (long long)a.window || (uint32_t)t1 < a.sinks);
            if (!full) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int t = t0 + j * 8 + (int)(lane & 3u) * 2 + (e & 1);
                        const bool on = !hole && t < run.n && (run.whole || sees(a, e < 2 ? p0 : p1, t));
                        if (!on) s[j][e] = neg_inf();
                    }
                // values that no row sees must not meet the matrix product, whatever bits they are
                if (lane < kFewTile) {
                    const int t = t0 + (int)lane;
                    const bool none = t >= run.n || t > run.pos_max || (!run.whole && !sees(a, max(run.pos_min, t), t));
                    if (none)
#pragma unroll
                        for (int h = 0; h < F::kHalves; ++h)
#pragma unroll
                            for (int e = 0; e < 8; ++e) st_shared_zero16(vt + h * 2048 + lane * 128 + e * 16);
                }
                fence_proxy_async();  // before a later copy lands in this slot
                __syncwarp();
            }
            if (p.logits) {
                float *lp = p.logits + ((uint64_t)run.seq * a.n_kv + run.c) * a.max_q * a.group * p.logit_stride;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t t = ck * kFewTile + j * 8 + (lane & 3u) * 2;
                    if (r0 < run.rows) *reinterpret_cast<float2 *>(lp + (uint64_t)r0 * p.logit_stride + t) = make_float2(s[j][0], s[j][1]);
                    if (HI && r1 < run.rows) *reinterpret_cast<float2 *>(lp + (uint64_t)r1 * p.logit_stride + t) = make_float2(s[j][2], s[j][3]);
                }
            }
            // online softmax; a row's 16 logits lie in the four lanes of a quad
            float mn[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float v = fmaxf(fmaxf(s[0][r * 2], s[0][r * 2 + 1]), fmaxf(s[1][r * 2], s[1][r * 2 + 1]));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
                v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
                mn[r] = fmaxf(x.m[r], v);
            }
            if (__any_sync(0xffffffffu, mn[0] != x.m[0] || mn[1] != x.m[1])) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float f = x.m[r] == mn[r] ? 1.f : ex2(x.m[r] - mn[r]);
                    x.m[r] = mn[r];
                    x.l[r] *= f;
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        x.o[j][r * 2] *= f;
                        x.o[j][r * 2 + 1] *= f;
                    }
                }
            }
            const float z0 = x.m[0] == neg_inf() ? 0.f : x.m[0] - kUp, z1 = x.m[1] == neg_inf() ? 0.f : x.m[1] - kUp;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[j][e] = (HI || e < 2) ? ex2(s[j][e] - (e < 2 ? z0 : z1)) : 0.f;
                    x.l[e / 2] += s[j][e];
                }
            // P is rounded to the pool's type, because the matrix instruction takes both factors in one type and V is in that one;
            // the sums l keep the unrounded weights (summing the rounded ones would cost a conversion back for each)
            const uint32_t pa[4] = {pack2(s[0][0], s[0][1], T()), pack2(s[0][2], s[0][3], T()), pack2(s[1][0], s[1][1], T()),
                                    pack2(s[1][2], s[1][3], T())};
            const uint32_t vrow = (lane & 7u) + ((lane >> 3) & 1u) * 8;
#pragma unroll
            for (int j = 0; j < NJ; j += 2) {
                const uint32_t ch = (j & 7) + (lane >> 4);
                uint32_t b[4];
                ldmatrix_x4_trans(vt + (j / 8) * 2048 + vrow * 128 + ((ch ^ (vrow & 7u)) << 4), b);
                mma16816(x.o[j], pa, b[0], b[1], T());
                mma16816(x.o[j + 1], pa, b[2], b[3], T());
            }
            __syncwarp();  // every lane has read the slot
        }
        ++got;
        if (++ck != run.k1) continue;
        // the end of the run
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            x.l[r] += __shfl_xor_sync(0xffffffffu, x.l[r], 1);
            x.l[r] += __shfl_xor_sync(0xffffffffu, x.l[r], 2);
        }
        if (TEAM) continue;
        const bool starts = run.k0 == 0, ends = run.k1 == run.tiles;
        uint32_t again = 0;  // finished rows to be done once more
#pragma unroll
        for (int r = 0; r < (HI ? 2 : 1); ++r) {
            const int row = r ? r1 : r0;
            if (row >= run.rows) continue;
            const uint64_t tok = run.q0 + (run.row0 + row) / (int)a.group;
            const uint32_t h = run.c * a.group + (uint32_t)(run.row0 + row) % a.group;
            const float m = x.m[r] - kUp, l = x.l[r];  // what o and l stand against
            if (starts && ends && !p.row_o) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                uint32_t *op = reinterpret_cast<uint32_t *>(a.out + tok * a.out_token_stride + h * a.out_head_stride) + (lane & 3u);
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const float lo = x.o[j][r * 2] * inv, hi = x.o[j][r * 2 + 1] * inv;
                    again |= !(fabsf(lo) < kHuge && fabsf(hi) < kHuge) ? 1u << r : 0u;
                    op[j * 4] = l == 0.f ? 0u : pack2(lo, hi, T());
                }
                if (a.lse && (lane & 3u) == 0) a.lse[tok * a.n_heads + h] = l == 0.f ? neg_inf() : (m + log2f(l)) * kLn2;
            } else {
                uint64_t at;
                float *po;
                if (starts && ends) {
                    at = tok * a.n_heads + h;
                    po = p.row_o + at * D;
                    if ((lane & 3u) == 0) p.row_ml[at] = make_float2(m, l);
                } else {
                    at = ((uint64_t)worker * 2 + (starts ? 1 : 0)) * p.slot_rows + row;
                    po = p.part_o + at * D;
                    if ((lane & 3u) == 0) p.part_ml[at] = make_float2(m, l);
                }
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    *reinterpret_cast<float2 *>(po + j * 8 + (lane & 3u) * 2) = make_float2(x.o[j][r * 2], x.o[j][r * 2 + 1]);
            }
        }
        if (p.again) {
            for (int r = 0; r < 2; ++r) {
                const uint32_t rows = __ballot_sync(0xffffffffu, again >> r & 1u);
                for (int row = 0; row < 8; ++row)
                    if (rows >> (row * 4) & 15u) {
                        __syncwarp();
                        const int at = run.row0 + row + 8 * r;
                        attend_row<T, D>(a, run.q0 + at / (int)a.group, run.c * a.group + (uint32_t)at % a.group);
                    }
            }
        }
    }
    if (TEAM) {  // the warps' shares, through the rings, which are idle now
        constexpr int R = HI ? 2 : 1;
        float *const jo = reinterpret_cast<float *>(sm), *const jm = jo + kWarps * NJ * R * 2 * 32, *const jl = jm + kWarps * R * 32;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            jm[(warp * R + i) * 32 + lane] = x.m[i] - kUp;
            jl[(warp * R + i) * 32 + lane] = x.l[i];
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) jo[(((warp * NJ + j) * R + i) * 2 + e) * 32 + lane] = x.o[j][i * 2 + e];
        }
        const uint32_t unit = blockIdx.x / a.n_kv;
        const Unit un = get_unit<kFewRows, kFewTile>(a, p, unit / p.n_rt, unit % p.n_rt);
        __syncthreads();
        constexpr int E = D / 32;  // neighbouring values a lane
#pragma unroll 1
        for (int r = (int)warp; r < un.rows; r += kWarps) {
            const int i = r / 8, quad = r % 8 * 4;
            Row<D> sum;
#pragma unroll
            for (int k = 0; k < kWarps; ++k) sum.m = fmaxf(sum.m, jm[(k * R + i) * 32 + quad]);
#pragma unroll
            for (int k = 0; k < kWarps; ++k) {
                const float m = jm[(k * R + i) * 32 + quad], f = m == sum.m ? 1.f : ex2(m - sum.m);
                sum.l += jl[(k * R + i) * 32 + quad] * f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int d = (int)lane * E + e;
                    sum.o[e] += jo[(((k * NJ + d / 8) * R + i) * 2 + d % 2) * 32 + quad + d % 8 / 2] * f;
                }
            }
            const int tok = unit_tok(a, un, r);
            const uint32_t h = unit_head(a, un, blockIdx.x % a.n_kv, r);
            if (!p.row_o) {
                if (finish<T, D>(a, sum, tok, h) && p.again) {
                    __syncwarp();
                    attend_row<T, D>(a, tok, h);
                }
                continue;
            }
            const uint64_t at = (uint64_t)tok * a.n_heads + h;
            if (lane == 0) p.row_ml[at] = make_float2(sum.m, sum.l);
#pragma unroll
            for (int e = 0; e < E; ++e) p.row_o[at * D + lane * E + e] = sum.o[e];
        }
    }
    if (p.behind) grid_wait();  // this kernel's end stands for both
}

template <class T, int D, bool HI, bool TEAM>
cudaError_t launch_few(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, cudaStream_t s)
{
    constexpr uint32_t smem = Few<D>::kSmem;
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(kv_attn_few_kernel<T, D, HI, TEAM>, smem, done);
    if (e != cudaSuccess) return e;
    const uint32_t grid = TEAM ? p.n_units * a.n_kv : (p.workers + kWarps - 1) / kWarps;
    return launch_dependent(kv_attn_few_kernel<T, D, HI, TEAM>, grid, kThreads, smem, s, kmap, vmap, a, p);
}
template <class T, int D, bool HI>
cudaError_t launch(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, cudaStream_t s)
{
    return p.team ? launch_few<T, D, HI, true>(a, p, kmap, vmap, s) : launch_few<T, D, HI, false>(a, p, kmap, vmap, s);
}

// One thread four tokens: the logits that the attention kernel left, against the finished log-sum-exps, rows in order.
__global__ void __launch_bounds__(256) kv_few_weights_kernel(const __grid_constant__ AttnArgs a, const __grid_constant__ Pass p, uint32_t chunks)
{
    __shared__ float lse[kFewRows];
    const uint32_t item = blockIdx.x / chunks, s = item / a.n_kv, c = item % a.n_kv;
    const Unit u = get_unit<kFewRows, kFewTile>(a, p, s, 0);
    grid_wait();
    if ((int)threadIdx.x < u.rows)
        lse[threadIdx.x] = a.lse[(uint64_t)(u.q0 + threadIdx.x / a.group) * a.n_heads + c * a.group + threadIdx.x % a.group] * kLog2e;
    __syncthreads();
    const int t = (int)(blockIdx.x % chunks * 1024 + threadIdx.x * 4);
    if (t >= u.n) return;
    const uint64_t at = s * a.w_seq_stride + c * a.w_head_stride + t;
    const int left = min(u.n - t, 4), tile = t / (int)kFewTile;
    float in[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) in[e] = a.w_in && e < left ? a.w_in[at + e] : 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    // tiles that nobody sees have no logits; in those of the list a token that a row does not see has -infinity
    const int k = tile < u.n_sink_tiles ? tile : tile - u.first_tile + u.n_sink_tiles;  // place in the list
    if (u.rows > 0 && (tile < u.n_sink_tiles || (tile >= u.first_tile && k < u.tiles))) {
        const float4 *lp = reinterpret_cast<const float4 *>(p.logits + (uint64_t)item * a.max_q * a.group * p.logit_stride + k * (int)kFewTile +
                                                            t % (int)kFewTile);
#pragma unroll 4
        for (int r = 0; r < u.rows; ++r) {
            const float4 x = lp[(uint64_t)r * (p.logit_stride / 4)];
            const float l = lse[r] == neg_inf() ? 0.f : lse[r];
            sum.x += ex2(x.x - l);
            sum.y += ex2(x.y - l);
            sum.z += ex2(x.z - l);
            sum.w += ex2(x.w - l);
        }
    }
    const float add[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) a.w_out[at + e] = a.decay * in[e] + add[e];
}

}  // namespace

cudaError_t launch_kv_attn_few(const AttnArgs &a, const Pass &p, const CUtensorMap &kmap, const CUtensorMap &vmap, uint32_t dtype,
                               uint32_t head_dim, cudaStream_t s)
{
    const bool hi = (p.prefix ? a.max_group_q : a.max_q) * a.group > 8;
    if (dtype == GMS_DTYPE_BF16) {
        if (head_dim == 64)
            return hi ? launch<__nv_bfloat16, 64, true>(a, p, kmap, vmap, s) : launch<__nv_bfloat16, 64, false>(a, p, kmap, vmap, s);
        return hi ? launch<__nv_bfloat16, 128, true>(a, p, kmap, vmap, s) : launch<__nv_bfloat16, 128, false>(a, p, kmap, vmap, s);
    }
    if (head_dim == 64) return hi ? launch<__half, 64, true>(a, p, kmap, vmap, s) : launch<__half, 64, false>(a, p, kmap, vmap, s);
    return hi ? launch<__half, 128, true>(a, p, kmap, vmap, s) : launch<__half, 128, false>(a, p, kmap, vmap, s);
}

cudaError_t launch_kv_few_weights(const AttnArgs &a, const Pass &p, cudaStream_t s)
{
    const uint32_t chunks = (a.max_kv + 1023) / 1024;
    if (chunks == 0) return cudaSuccess;
    return launch_dependent(kv_few_weights_kernel, a.n_seq * a.n_kv * chunks, 256, 0, s, a, p, chunks);
}

}  // namespace gms
