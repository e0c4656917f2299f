// The gated delta rule in chunks: the chain of the states (what its operands are stands at the kernel that makes them).
#include <cmath>

#include "gms_kv_delta.h"

namespace gms {
namespace {

using ptx::ldmatrix_x4;
using ptx::ldmatrix_x4_trans;
using ptx::smem_u32;

constexpr __nv_bfloat16 kWide{};  // the type of terms that have 32 bits' range

// A chunk's operands.  V is the columns of the CTA, 16 for each of its W slices.
template <int D, int W>
struct Stage {
    uint8_t k[kChunkRows * D * 2], q[kChunkRows * D * 2], v[kChunkRows * W * 32];
    ChunkWork w;
};

// A tile of 64 rows, PR pieces each; rows from n on are zeros.  A lane keeps to one piece of the rows that it copies.
template <int PR, uint32_t kFetchLanes>
__device__ __forceinline__ void fetch_rows(uint32_t tile, uint32_t me, const uint8_t *src, uint64_t stride, int n)
{
    constexpr uint32_t kStep = kFetchLanes / PR, N = kChunkRows / kStep;
    static_assert(kStep * PR == kFetchLanes, "");
    const uint32_t c = me % PR, r0 = me / PR;
    src += r0 * stride + c * 16;
    if (n >= (int)kChunkRows) {
#pragma unroll
        for (uint32_t i = 0; i < N; ++i) {
            cp16(tile + piece<PR>(r0 + i * kStep, c), src, true);
            src += kStep * stride;
        }
    } else {
#pragma unroll 1
        for (uint32_t r = r0; r < (uint32_t)kChunkRows; r += kStep) {
            const bool real = (int)r < n;
            cp16(tile + piece<PR>(r, c), real ? src : src - r * stride, real);
            src += kStep * stride;
        }
    }
}
// Chunk `chunk` of a sequence; `full` is told when it has landed.
template <int D, int W, uint32_t kLanes>
__device__ __forceinline__ void fetch_chunk(const DeltaArgs &a, Stage<D, W> &st, uint32_t me, int chunk, int rows, int first, uint32_t kh, uint32_t h,
                                            uint32_t col0, uint32_t slot, uint32_t full)
{
    const int n = rows - chunk * (int)kChunkRows;
    const uint64_t row = (uint64_t)(first + chunk * (int)kChunkRows);
    const uint8_t *work = a.chunks + ((uint64_t)(slot + chunk) * a.n_heads + h) * sizeof(ChunkWork) + me * 16;
    const uint32_t to = smem_u32(&st.w) + me * 16;
    fetch_rows<D / 8, kLanes>(smem_u32(st.k), me, a.k + row * a.k_token + kh * a.k_head, a.k_token, n);
    fetch_rows<W * 2, kLanes>(smem_u32(st.v), me, a.v + row * a.v_token + h * a.v_head + col0 * 2, a.v_token, n);
    constexpr uint32_t kPieces = sizeof(ChunkWork) / 16;
#pragma unroll
    for (uint32_t i = 0; i < kPieces / kLanes; ++i) cp16(to + i * 16 * kLanes, work + i * 16 * kLanes, true);
    if (kPieces % kLanes && me < kPieces % kLanes) cp16(to + kPieces / kLanes * 16 * kLanes, work + kPieces / kLanes * 16 * kLanes, true);
    fetch_rows<D / 8, kLanes>(smem_u32(st.q), me, a.q + row * a.q_token + kh * a.q_head, a.q_token, n);
    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(full) : "memory");
}

// ------------------------------------------------------------------------------------------------ few states
// What the warps of a slice tell each other: accumulators, and first factors of products (a lane's part of 16 x 16).
template <int D>
struct Talk {
    uint4 s[D / 16][32];       // S before the chunk, the first of its two terms
    union {
        float4 sum[4][3][2][32];  // [to][from the others]: what X is the sum of
        uint4 d[4][2][32];        // d, in two terms, once all sums have been read (and gone before the next ones are written)
    };
    uint4 x[4][2][32];         // V - f X of the 16 rows of each warp, in two terms
    uint4 dw[4][2][32];        // w d, the same
    float2 s_unit[4][8], dw_unit[4][8];  // f16: powers of two that rows' terms are multiples of
    uint32_t odd[4];           // the chunk is done row by row
};
template <int D, int W>
struct RelayShape {
    static constexpr int kStages = 3;
    static constexpr uint32_t kOuts = W == 1 ? 2 : 1;  // warps of a slice that make `out`
    static constexpr uint32_t kFetchWarps = 2, kFetchLanes = kFetchWarps * 32, kWorkers = (4 + kOuts) * W, kThreads = (kWorkers + kFetchWarps) * 32;
};
template <int D, int W>
struct RelaySmem {
    Stage<D, W> stage[3];
    Talk<D> talk[W];
    uint64_t full[3], empty[3], ready[W], taken[W];
    uint32_t nth;  // of the items that a CTA goes through (no register is free for it)
};

// A slice, 16 value columns of a head's state, has four warps that carry the state on and one or two that make `out`.  The state lies,
// transposed, in accumulators of mma.sync, the columns of D / 4 keys a warp; what is an accumulator of one product is, element for
// element, a first factor of the next: S -> X = S K^T (each warp its keys' part, for all rows) -> d = (V - f X) T^T -> S, each warp
// 16 of the rows in between, with three exchanges through shared memory a chunk.  The others get S and d handed and work beside the
// next chunk: of two slices one each, which leaves 168 registers a thread (two each, of 14 warps, 128); of one slice two, which one
// alone would hold up (8,192 rows of 4 heads of 128 235 us, so 243).  W slices share a chunk's operands, which two more warps fetch
// ahead.  Bound by the latency of that sequence of small products and exchanges: 8,192 rows of 32 heads of 128, two slices a CTA, 280 us
// or 4,060 cycles a chunk (one: 3,190), in which the products take 45 % of the tensor cores' cycles and loads, stores and exchanges
// 69 % of shared memory's.  `out` could have S in two terms, too: 64 products a slice and chunk more, on the warp that has most, and
// 386 us instead of 335 for that call (one slice a CTA 241 instead of 233), for an error of 1.65 instead of 1.78 thousandths in bf16.
template <class T, int D, int W>
__device__ __forceinline__ void relay(const DeltaArgs &a, RelaySmem<D, W> &m, uint32_t s, uint32_t h, uint32_t part, bool &late)
{
    constexpr int C = kChunkRows, P = D / 8, VP = W * 2, NT = D / 32, KQ = D / 64;  // tiles of 8 and of 16 keys that a warp has
    constexpr int kStages = RelayShape<D, W>::kStages;
    constexpr uint32_t kOuts = RelayShape<D, W>::kOuts, kWorkers = RelayShape<D, W>::kWorkers;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    const uint32_t kh = h / a.group, col0 = part * W * 16;  // of the CTA
    const int rows = delta_rows(a, s), first = delta_begin(a, s);
    const int chunks = (rows + C - 1) / C;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            ptx::mbar_init(smem_u32(&m.full[i]), RelayShape<D, W>::kFetchLanes);
            ptx::mbar_init(smem_u32(&m.empty[i]), kWorkers);
        }
        for (int i = 0; i < W; ++i) {
            ptx::mbar_init(smem_u32(&m.ready[i]), 4);
            ptx::mbar_init(smem_u32(&m.taken[i]), kOuts);
        }
        ptx::fence_mbar_init();
    }
    __syncthreads();
    // A wait that runs out (it cannot, but for a fault in here) is told in the status word; everybody goes on without waiting.
    auto wait = [&](uint64_t *bar, int use) {
        if (late || ptx::mbar_wait(smem_u32(bar), (uint32_t)(use & 1))) return;
        late = true;
        if (a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_TIMEOUT);
    };
    auto arrive = [&](uint64_t *bar) {  // of a warp
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(smem_u32(bar));
    };
    if (warp >= kWorkers) {  // the fetching warps
        const uint32_t me = (warp - kWorkers) * 32 + lane, slot = delta_slot(a, s);
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int i = chunk % kStages;
            if (chunk >= kStages) wait(&m.empty[i], chunk / kStages - 1);
            fetch_chunk<D, W, RelayShape<D, W>::kFetchLanes>(a, m.stage[i], me, chunk, rows, first, kh, h, col0, slot, smem_u32(&m.full[i]));
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    const uint32_t g = lane / 4, t2 = 2 * (lane & 3u);  // rows g and g + 8, columns 8 nt + t2 + {0, 1} of an accumulator
    const uint32_t b_row = (lane & 7u) + (lane & 16u) / 2, b_piece = lane / 8 & 1u;  // of a lane's address for two second factors
    const float2 one = make_float2(1.f, 1.f);
    // f16: accumulators go over to the unit of the next factors
    auto change = [](float(*x)[4], float2 now, float2 next) {
        const float f0 = now.x * flipped(next.x), f1 = now.y * flipped(next.y);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) x[nt][0] *= f0, x[nt][1] *= f0, x[nt][2] *= f1, x[nt][3] *= f1;
    };
    // or, in a unit of their own, are added to others (units may lie too far apart for both)
    auto add_in = [](float(*x)[4], const float(*part)[4], float2 unit) {
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            x[nt][0] = fmaf(part[nt][0], unit.x, x[nt][0]), x[nt][1] = fmaf(part[nt][1], unit.x, x[nt][1]);
            x[nt][2] = fmaf(part[nt][2], unit.y, x[nt][2]), x[nt][3] = fmaf(part[nt][3], unit.y, x[nt][3]);
        }
    };
    if (warp >= 4 * W) {
        // out = h Q S + P d, with S before the chunk (one term of S, two of P and d without the product of the small ones), two tiles of
        // 16 rows at a time: the first and the last, then, or by another warp, those between them
        const uint32_t slice = (warp - 4 * W) / kOuts;
        Talk<D> &talk = m.talk[slice];
#pragma unroll 1
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int stage = chunk % kStages, n = min(rows - chunk * C, C);
            Stage<D, W> &st = m.stage[stage];
            uint8_t *out = a.out + (uint64_t)(first + chunk * C) * a.o_token + h * a.o_head + (col0 + 16 * slice) * 2;
            wait(&m.full[stage], chunk / kStages);
            wait(&m.ready[slice], chunk);
            const bool by_row = talk.odd[0] | talk.odd[1] | talk.odd[2] | talk.odd[3];
            uint4 sf[D / 16], df[4][2];
            float2 su[4];
#pragma unroll
            for (int kt = 0; kt < D / 16; ++kt) sf[kt] = talk.s[kt][lane];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                df[kt][0] = talk.d[kt][0][lane], df[kt][1] = talk.d[kt][1][lane];
                if (kHalf) su[kt] = talk.s_unit[kt][g];
            }
            arrive(&m.taken[slice]);
            if (!by_row) {
#pragma unroll
                for (uint32_t pair = 0; pair < 2 / kOuts; ++pair) {
                    const bool inner = kOuts == 1 ? pair : warp & 1u;
                    const int tile[2] = {inner ? 1 : 0, inner ? 2 : 3};
                    float Y[2][2][4] = {};
                    float2 unit = one;
#pragma unroll
                    for (int kt = 0; kt < D / 16; ++kt) {
                        if (kHalf && kt % KQ == 0) {
                            const float2 next = su[kt / KQ];
                            if (kt) change(Y[0], unit, next), change(Y[1], unit, next);
                            unit = next;
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t b[4];
                            ldmatrix_x4(smem_u32(st.q) + piece<P>(16 * tile[i] + b_row, 2 * kt + b_piece), b);
                            mma16816(Y[i][0], &sf[kt].x, b[0], b[1], T());
                            mma16816(Y[i][1], &sf[kt].x, b[2], b[3], T());
                        }
                    }
                    if (kHalf) change(Y[0], unit, one), change(Y[1], unit, one);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
#pragma unroll
                        for (int nt = 0; nt < 2; ++nt) {
                            const float2 f = *reinterpret_cast<const float2 *>(&st.w.h[16 * tile[i] + 8 * nt + t2]);
                            Y[i][nt][0] *= f.x, Y[i][nt][1] *= f.y, Y[i][nt][2] *= f.x, Y[i][nt][3] *= f.y;
                        }
                    }
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if (kt > tile[i]) continue;
                            uint32_t b[2][4];
#pragma unroll
                            for (int t = 0; t < 2; ++t) ldmatrix_x4(smem_u32(st.w.tile[2 + t]) + block_piece(16 * tile[i] + b_row, 2 * kt + b_piece), b[t]);
#pragma unroll
                            for (int t = 0; t < 3; ++t) {  // d's terms with P's first one, d's first one with P's second
                                mma16816(Y[i][0], &df[kt][t & 1].x, b[t / 2][0], b[t / 2][1], kWide);
                                mma16816(Y[i][1], &df[kt][t & 1].x, b[t / 2][2], b[t / 2][3], kWide);
                            }
                        }
                    // (through the slice's part of V's tile, which the other warps have read)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                                         smem_u32(st.v) + piece<VP>(16 * tile[i] + b_row, 2 * slice + b_piece)),
                                     "r"(pack2(Y[i][0][0], Y[i][0][1], T())), "r"(pack2(Y[i][0][2], Y[i][0][3], T())),
                                     "r"(pack2(Y[i][1][0], Y[i][1][1], T())), "r"(pack2(Y[i][1][2], Y[i][1][3], T()))
                                     : "memory");
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int r = 16 * tile[i] + (int)lane / 2;
                        const uint4 x = *reinterpret_cast<const uint4 *>(st.v + piece<VP>(r, 2 * slice + (lane & 1u)));
                        if (r < n) *reinterpret_cast<uint4 *>(out + (uint64_t)r * a.o_token + (lane & 1u) * 16) = x;
                    }
                }
            }
            arrive(&m.empty[stage]);
        }
        return;
    }
    // (the last rows have most to do: of two slices they go to different quarters of the SM)
    const uint32_t slice = warp / 4, mine = (warp & 3u) ^ (slice & 1u ? 3u : 0u), row0 = 16 * mine;
    Talk<D> &talk = m.talk[slice];
    const bool fresh = a.past_lens && a.past_lens[s] <= 0;
    const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
    float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
    if (a.status && threadIdx.x == 0 && ((!fresh && !from) || !to)) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
    const uint32_t at0 = (mine * (D / 4) + t2) * D + col0 + 16 * slice + g;
    float S[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[nt][e] = from ? from[at0 + (8 * nt + (e & 1)) * D + (e & 2) * 4] : 0.f;
    auto together = [&] { asm volatile("bar.sync %0, 128;" ::"r"(slice + 1) : "memory"); };
    auto seat = [](uint32_t to, uint32_t from) { return from < to ? from : from - 1; };  // the place that one of four has among the other three
    // f16: the scales of a lane's two rows of the 16 x 16 in accumulators x and y
    auto top_of = [](const float *x, const float *y, int e) {
        float top = fmaxf(fmaxf(fabsf(x[2 * e]), fabsf(x[2 * e + 1])), fmaxf(fabsf(y[2 * e]), fabsf(y[2 * e + 1])));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        return fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    };
    auto scales = [&](const float *x, const float *y) { return make_float2(range_scale(top_of(x, y, 0)), range_scale(top_of(x, y, 1))); };
    auto inverse = [](float2 u) { return make_float2(flipped(u.x), flipped(u.y)); };
    auto tell = [&](float2 *unit, float2 u) {
        if ((lane & 3u) == 0) unit[g] = u;
    };
    auto terms = [](auto type, const float *x, const float *y, float2 u, uint4 &hi, uint4 &lo) {
        using Term = decltype(type);
        split2<Term>(x[0] * u.x, x[1] * u.x, hi.x, lo.x);
        split2<Term>(x[2] * u.y, x[3] * u.y, hi.y, lo.y);
        split2<Term>(y[0] * u.x, y[1] * u.x, hi.z, lo.z);
        split2<Term>(y[2] * u.y, y[3] * u.y, hi.w, lo.w);
    };
#pragma unroll 1
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int stage = chunk % kStages, n = min(rows - chunk * C, C);
        Stage<D, W> &st = m.stage[stage];
        wait(&m.full[stage], chunk / kStages);
        // what needs no news from the other warps is read before they meet
        uint32_t kb[4][KQ][4], V[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < KQ; ++k) ldmatrix_x4(smem_u32(st.k) + piece<P>(16 * i + b_row, 2 * (mine * KQ + k) + b_piece), kb[i][k]);
        ldmatrix_x4_trans(smem_u32(st.v) + piece<VP>(row0 + b_row, 2 * slice + b_piece), V);
        if (chunk) wait(&m.taken[slice], chunk - 1);
        // S in two terms
        uint4 hi[KQ], lo[KQ];
        float2 su = one;
        if (kHalf) {
            su = scales(S[0], S[1]);
#pragma unroll
            for (int k = 1; k < KQ; ++k) {
                const float2 u = scales(S[2 * k], S[2 * k + 1]);
                su = make_float2(fminf(su.x, u.x), fminf(su.y, u.y));
            }
            tell(talk.s_unit[mine], inverse(su));
        }
        uint32_t odd = kHalf && (state_beyond_scale(su.x) || state_beyond_scale(su.y));
#pragma unroll
        for (int k = 0; k < KQ; ++k) {
            terms(T(), S[2 * k], S[2 * k + 1], su, hi[k], lo[k]);
            talk.s[mine * KQ + k][lane] = hi[k];
        }
        // its part of X = S K^T for all rows
        float x[4][2][4] = {};
#pragma unroll
        for (int k = 0; k < KQ; ++k)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    mma16816(x[i][0], t ? &lo[k].x : &hi[k].x, kb[i][k][0], kb[i][k][1], T());
                    mma16816(x[i][1], t ? &lo[k].x : &hi[k].x, kb[i][k][2], kb[i][k][3], T());
                }
        float X[2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kHalf) {
                const float2 u = inverse(su);
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) x[i][nt][0] *= u.x, x[i][nt][1] *= u.x, x[i][nt][2] *= u.y, x[i][nt][3] *= u.y;
            }
            if (i == (int)mine) {
#pragma unroll
                for (int e = 0; e < 4; ++e) X[0][e] = x[i][0][e], X[1][e] = x[i][1][e];
            } else {
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) talk.sum[i][seat(i, mine)][nt][lane] = make_float4(x[i][nt][0], x[i][nt][1], x[i][nt][2], x[i][nt][3]);
            }
        }
        uint32_t tb[2][C / 16][4];
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            if (kt > (int)mine) break;
            const uint32_t at = block_piece(row0 + b_row, 2 * kt + b_piece);
            ldmatrix_x4(smem_u32(st.w.tile[0]) + at, tb[0][kt]);
            ldmatrix_x4(smem_u32(st.w.tile[1]) + at, tb[1][kt]);
        }
        together();
        // what the values differ by from what the state says: X <- V - f X, for the warp's rows
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
            for (int o = 0; o < 3; ++o) {
                const float4 u = talk.sum[mine][o][nt][lane];
                X[nt][0] += u.x, X[nt][1] += u.y, X[nt][2] += u.z, X[nt][3] += u.w;
            }
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.f[row0 + 8 * nt + t2]);
            const T *va = reinterpret_cast<const T *>(&V[2 * nt]), *vb = reinterpret_cast<const T *>(&V[2 * nt + 1]);
            X[nt][0] = to_f32(va[0]) - f.x * X[nt][0];
            X[nt][1] = to_f32(va[1]) - f.y * X[nt][1];
            X[nt][2] = to_f32(vb[0]) - f.x * X[nt][2];
            X[nt][3] = to_f32(vb[1]) - f.y * X[nt][3];
        }
        uint4 own_hi, own_lo;
        terms(kWide, X[0], X[1], one, own_hi, own_lo);
        talk.x[mine][0][lane] = own_hi, talk.x[mine][1][lane] = own_lo;
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt)
#pragma unroll
            for (int k = 0; k < KQ; ++k)
                ldmatrix_x4_trans(smem_u32(st.k) + piece<P>(16 * kt + (lane & 15u), mine * NT + 2 * k + lane / 16), kb[kt][k]);
        together();
        // d = X T^T: two terms each (the product of the small ones left out), of bf16, which has the range, from the rows up to the
        // warp's own
        float d[2][4] = {}, dl[2][4] = {}, dt[2][4] = {};
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            if (kt > (int)mine) break;
            const uint4 p = kt == (int)mine ? own_hi : talk.x[kt][0][lane], q = kt == (int)mine ? own_lo : talk.x[kt][1][lane];
            mma16816(d[0], &p.x, tb[0][kt][0], tb[0][kt][1], kWide);
            mma16816(d[1], &p.x, tb[0][kt][2], tb[0][kt][3], kWide);
            mma16816(dl[0], &q.x, tb[0][kt][0], tb[0][kt][1], kWide);
            mma16816(dl[1], &q.x, tb[0][kt][2], tb[0][kt][3], kWide);
            mma16816(dt[0], &p.x, tb[1][kt][0], tb[1][kt][1], kWide);
            mma16816(dt[1], &p.x, tb[1][kt][2], tb[1][kt][3], kWide);
        }
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[nt][e] += dl[nt][e] + dt[nt][e];
        float size = 0.f;  // (infinite from 2^64 on, NaN with one in d or what it was made of)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) size = fmaf(d[nt][e], d[nt][e], size);
        terms(kWide, d[0], d[1], one, own_hi, own_lo);
        talk.d[mine][0][lane] = own_hi, talk.d[mine][1][lane] = own_lo;
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.w[row0 + 8 * nt + t2]);
            d[nt][0] *= f.x, d[nt][1] *= f.y, d[nt][2] *= f.x, d[nt][3] *= f.y;
        }
        float2 u = one;
        if (kHalf) {
            u = scales(d[0], d[1]);
            tell(talk.dw_unit[mine], inverse(u));
        }
        terms(T(), d[0], d[1], u, own_hi, own_lo);
        talk.dw[mine][0][lane] = own_hi, talk.dw[mine][1][lane] = own_lo;
        odd |= st.w.by_row | !(size < INFINITY) | (kHalf && (beyond_scale(u.x) || beyond_scale(u.y)));
        odd = __any_sync(0xffffffffu, odd);
        if (lane == 0) talk.odd[mine] = odd;
        arrive(&m.ready[slice]);
        together();
        if (talk.odd[0] | talk.odd[1] | talk.odd[2] | talk.odd[3]) {
            // row by row, from the state as it was: something here is not finite, or far from it, and in a product would reach rows before it
            uint8_t *out = a.out + (uint64_t)(first + chunk * C) * a.o_token + h * a.o_head + (col0 + 16 * slice) * 2;
            float4(*xy)[4][32] = reinterpret_cast<float4(*)[4][32]>(talk.x);  // [2][4][32], in the place of what is not needed
            float(*zs)[4][32] = reinterpret_cast<float(*)[4][32]>(talk.dw);
#pragma unroll 1
            for (int r = 0; r < n; ++r) {
                const float gate = st.w.gate[r], beta = st.w.beta[r], rk = st.w.rk[r], rq = st.w.rq[r];
                float p[2] = {}, y[2] = {}, z = 0.f, kv[2 * NT];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const T *kp = reinterpret_cast<const T *>(st.k + piece<P>(r, mine * NT + nt)) + t2;
                    const T *qp = reinterpret_cast<const T *>(st.q + piece<P>(r, mine * NT + nt)) + t2;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float k = to_f32(kp[e]) * rk, q = to_f32(qp[e]) * rq;
                        kv[2 * nt + e] = k;
                        z += k * q;
                        S[nt][e] *= gate, S[nt][2 + e] *= gate;
                        p[0] += S[nt][e] * k, p[1] += S[nt][2 + e] * k;
                        y[0] += S[nt][e] * q, y[1] += S[nt][2 + e] * q;
                    }
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    z += __shfl_xor_sync(0xffffffffu, z, o);
#pragma unroll
                    for (int e = 0; e < 2; ++e) p[e] += __shfl_xor_sync(0xffffffffu, p[e], o), y[e] += __shfl_xor_sync(0xffffffffu, y[e], o);
                }
                xy[r & 1][mine][lane] = make_float4(p[0], p[1], y[0], y[1]);
                zs[r & 1][mine][lane] = z;
                together();
                p[0] = p[1] = y[0] = y[1] = z = 0.f;
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    const float4 u = xy[r & 1][o][lane];
                    p[0] += u.x, p[1] += u.y, y[0] += u.z, y[1] += u.w;
                    z += zs[r & 1][o][lane];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float v = to_f32(*reinterpret_cast<const T *>(st.v + piece<VP>(r, 2 * slice + e) + g * 2));
                    const float d = beta * (v - p[e]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) S[nt][2 * e] += kv[2 * nt] * d, S[nt][2 * e + 1] += kv[2 * nt + 1] * d;
                    if (mine == 0 && (lane & 3u) == 0)
                        reinterpret_cast<T *>(out + (uint64_t)r * a.o_token)[g + 8 * e] = from_f32<T>(a.scale * (y[e] + z * d));
                }
            }
            arrive(&m.empty[stage]);
            continue;
        }
        // S <- e^G S + (w d) K for the warp's keys
        const float all = st.w.all;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 4; ++e) S[nt][e] *= all;
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            const uint4 p = kt == (int)mine ? own_hi : talk.dw[kt][0][lane], q = kt == (int)mine ? own_lo : talk.dw[kt][1][lane];
            float part[NT][4] = {};
            float(*to)[4] = kHalf ? part : S;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma16816(to[nt], t ? &q.x : &p.x, kb[kt][nt / 2][2 * (nt & 1)], kb[kt][nt / 2][2 * (nt & 1) + 1], T());
            if (kHalf) {
                const float2 unit = talk.dw_unit[kt][g];
#pragma unroll
                for (int nt = 0; nt < NT; nt += 2) add_in(S + nt, part + nt, unit);
            }
        }
        arrive(&m.empty[stage]);
    }
    if (!to) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[at0 + (8 * nt + (e & 1)) * D + (e & 2) * 4] = S[nt][e];
}

// Most items of a batch in which few sequences are long are none: they come last.  Where there are many for each SM, CTAs go through
// several (AGAIN) instead of being started for each (us, one CTA an item / so: a prompt of 2,048 rows among 255 single rows, 32 heads of
// 128 368 / 296, of 64 212 / 144; of 4,096 among 95 265 / 257; of 8,192 among 31, 4,096 items, 337 / 364, as the loop costs registers).
constexpr uint32_t kMany = 148 * 32;
template <class T, int D, int W, bool AGAIN>
__global__ void __launch_bounds__(RelayShape<D, W>::kThreads) kv_delta_relay_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    RelaySmem<D, W> &m = *reinterpret_cast<RelaySmem<D, W> *>(raw);
    constexpr uint32_t kParts = D / (16 * W);
    bool late = false;  // a wait has run out
    ptx::grid_launch_dependents();
    ptx::grid_wait();
    volatile uint32_t &nth = m.nth;
    if (AGAIN) {
        if (threadIdx.x == 0) nth = 0;
        __syncthreads();
    }
    for (;;) {
        const uint32_t item = blockIdx.x + (AGAIN ? nth * gridDim.x : 0);
        if (item >= a.n_seq * a.n_heads * kParts) return;
        const uint32_t s = a.order[item / kParts / a.n_heads];
        if (s >= a.n_seq) return;
        relay<T, D, W>(a, m, s, item / kParts % a.n_heads, item % kParts, late);
        if (!AGAIN) return;
        __syncthreads();
        if (threadIdx.x == 0) {  // (made anew for the next item)
            for (int i = 0; i < RelayShape<D, W>::kStages; ++i) ptx::mbar_inval(smem_u32(&m.full[i])), ptx::mbar_inval(smem_u32(&m.empty[i]));
            for (int i = 0; i < W; ++i) ptx::mbar_inval(smem_u32(&m.ready[i])), ptx::mbar_inval(smem_u32(&m.taken[i]));
            nth = nth + 1;
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ many states
// W warps with states, and warps that fetch.
template <int D, int W>
struct SoloShape {
    static constexpr int kStages = D == 64 && W == 4 ? 2 : 3;  // that fit (two CTAs an SM there)
    static constexpr uint32_t kFetchWarps = 2, kFetchLanes = kFetchWarps * 32, kThreads = (W + kFetchWarps) * 32;
    static constexpr uint32_t kCtas = D == 64 && W == 4 ? 2 : 1;
};
template <int D, int W>
struct SoloSmem {
    Stage<D, W> stage[SoloShape<D, W>::kStages];
    uint64_t full[3], empty[3];
};

// A warp has 16 value columns of a head's state, transposed, as accumulators of mma.sync (16 x D): what is an accumulator of one
// product is, element for element, a first factor of the next, S -> X = S K^T, Y = S Q^T -> d = (V - f X) T^T -> S, out, so nothing
// leaves the registers between the products and no warp waits for another.  W of them (16 W columns of a head) share a chunk's
// operands, which further warps fetch ahead.  Bound by the rate of the products, 440 of them a chunk and warp at 128 keys, 8.3 cycles
// each, and what a warp alone on its quarter of an SM does not hide of their latencies: 5,800 cycles a chunk (64 keys: 280, 7,600 with
// two CTAs an SM).
template <class T, int D, int W>
__device__ __forceinline__ void solo(const DeltaArgs &a, SoloSmem<D, W> &m, uint32_t s, uint32_t h, uint32_t part, bool &late)
{
    constexpr int C = kChunkRows, P = D / 8, VP = W * 2, NT = D / 8, CT = C / 8;
    constexpr int kStages = SoloShape<D, W>::kStages;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    const uint32_t kh = h / a.group, col0 = part * W * 16;  // of the CTA
    const int rows = delta_rows(a, s), first = delta_begin(a, s);
    const int chunks = (rows + C - 1) / C;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            ptx::mbar_init(smem_u32(&m.full[i]), SoloShape<D, W>::kFetchLanes);
            ptx::mbar_init(smem_u32(&m.empty[i]), W);
        }
        ptx::fence_mbar_init();
    }
    __syncthreads();
    // A wait that runs out (it cannot, but for a fault in here) is told in the status word; everybody goes on without waiting.
    auto wait = [&](uint64_t *bar, int use) {
        if (late || ptx::mbar_wait(smem_u32(bar), (uint32_t)(use & 1))) return;
        late = true;
        if (a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_TIMEOUT);
    };
    if (warp >= W) {  // the fetching warps
        const uint32_t me = (warp - W) * 32 + lane, slot = delta_slot(a, s);
        for (int chunk = 0; chunk < chunks; ++chunk) {
            const int i = chunk % kStages;
            if (chunk >= kStages) wait(&m.empty[i], chunk / kStages - 1);
            fetch_chunk<D, W, SoloShape<D, W>::kFetchLanes>(a, m.stage[i], me, chunk, rows, first, kh, h, col0, slot, smem_u32(&m.full[i]));
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        return;
    }
    const bool fresh = a.past_lens && a.past_lens[s] <= 0;
    const float *from = fresh ? nullptr : delta_state<D>(a, a.src_table, a.src_stride, s, h);
    float *to = delta_state<D>(a, a.dst_table, a.dst_stride, s, h);
    if (a.status && threadIdx.x == 0 && ((!fresh && !from) || !to)) atomicOr(a.status, (unsigned long long)GMS_DEV_HOLE);
    const uint32_t g = lane / 4, t2 = 2 * (lane & 3u);  // rows g and g + 8, columns 8 nt + t2 + {0, 1} of an accumulator
    const uint32_t at0 = t2 * D + col0 + 16 * warp + g;
    const uint32_t b_row = (lane & 7u) + (lane & 16u) / 2, b_piece = lane / 8 & 1u;  // of a lane's address for two second factors
    float S[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) S[nt][e] = from ? from[at0 + (8 * nt + (e & 1)) * D + (e & 2) * 4] : 0.f;
    auto times = [](float *x, float2 f, float2 g) {  // rows g and g + 8 of an accumulator
        const float2 a = ptx::mul2(make_float2(x[0], x[1]), f), b = ptx::mul2(make_float2(x[2], x[3]), g);
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
    };
    // f16: rows (e = 0, 1: g and g + 8) are scaled by powers of two of their own before they are rounded
    auto top_of = [](const float(*x)[4], int tiles, int e) {
        float top = 0.f;
#pragma unroll
        for (int nt = 0; nt < tiles; ++nt) top = fmaxf(top, fmaxf(fabsf(x[nt][2 * e]), fabsf(x[nt][2 * e + 1])));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        return fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    };
    auto terms = [](auto type, const float(*x)[4], float u0, float u1, uint32_t *hi, uint32_t *lo) {  // of the 16 x 16 in accumulators x[0] and x[1]
        using Term = decltype(type);
        split2<Term>(x[0][0] * u0, x[0][1] * u0, hi[0], lo[0]);
        split2<Term>(x[0][2] * u1, x[0][3] * u1, hi[1], lo[1]);
        split2<Term>(x[1][0] * u0, x[1][1] * u0, hi[2], lo[2]);
        split2<Term>(x[1][2] * u1, x[1][3] * u1, hi[3], lo[3]);
    };
#pragma unroll 1
    for (int chunk = 0; chunk < chunks; ++chunk) {
        const int stage = chunk % kStages;
        Stage<D, W> &st = m.stage[stage];
        const int n = min(rows - chunk * C, C);
        uint8_t *out = a.out + (uint64_t)(first + chunk * C) * a.o_token + h * a.o_head + (col0 + 16 * warp) * 2;
        auto done = [&] {
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(smem_u32(&m.empty[stage]));
        };
        wait(&m.full[stage], chunk / kStages);
        // the columns' values, transposed like everything else
        uint32_t V[CT][2];
        const uint32_t by_row = st.w.by_row;
#pragma unroll
        for (int nt = 0; nt < CT; nt += 2) {
            uint32_t b[4];
            ldmatrix_x4_trans(smem_u32(st.v) + piece<VP>(8 * nt + b_row, 2 * warp + b_piece), b);
            V[nt][0] = b[0], V[nt][1] = b[1], V[nt + 1][0] = b[2], V[nt + 1][1] = b[3];
        }
        // X = S K^T (S in two terms), Y = S Q^T (one term: it goes into `out` alone)
        float X[CT][4] = {}, Y[CT][4] = {};
        float u0 = 1.f, u1 = 1.f;
        uint32_t odd = by_row;  // the chunk is done row by row
        if (kHalf) {
            u0 = range_scale(top_of(S, NT, 0)), u1 = range_scale(top_of(S, NT, 1));
            odd |= state_beyond_scale(u0) || state_beyond_scale(u1);
        }
#pragma unroll
        for (int kt = 0; kt < D / 16; ++kt) {
            uint32_t hi[4], lo[4], b[CT][2], c[CT][2];
#pragma unroll
            for (int nt = 0; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.k) + piece<P>(8 * nt + b_row, 2 * kt + b_piece), x);
                b[nt][0] = x[0], b[nt][1] = x[1], b[nt + 1][0] = x[2], b[nt + 1][1] = x[3];
            }
            terms(T(), S + 2 * kt, u0, u1, hi, lo);
#pragma unroll
            for (int nt = 0; nt < CT; ++nt) mma16816(X[nt], hi, b[nt][0], b[nt][1], T());
#pragma unroll
            for (int nt = 0; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.q) + piece<P>(8 * nt + b_row, 2 * kt + b_piece), x);
                c[nt][0] = x[0], c[nt][1] = x[1], c[nt + 1][0] = x[2], c[nt + 1][1] = x[3];
            }
#pragma unroll
            for (int nt = 0; nt < CT; ++nt) mma16816(X[nt], lo, b[nt][0], b[nt][1], T());
#pragma unroll
            for (int nt = 0; nt < CT; ++nt) mma16816(Y[nt], hi, c[nt][0], c[nt][1], T());
        }
        // what the values differ by from what the state says: X <- V - f X
        const float si0 = flipped(u0), si1 = flipped(u1);
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.f[8 * nt + t2]);
            const T *va = reinterpret_cast<const T *>(&V[nt][0]), *vb = reinterpret_cast<const T *>(&V[nt][1]);
            const float2 m0 = kHalf ? ptx::mul2(f, make_float2(-si0, -si0)) : make_float2(-f.x, -f.y), m1 = kHalf ? ptx::mul2(f, make_float2(-si1, -si1)) : m0;
            const float2 x0 = ptx::fma2(m0, make_float2(X[nt][0], X[nt][1]), make_float2(to_f32(va[0]), to_f32(va[1])));
            const float2 x1 = ptx::fma2(m1, make_float2(X[nt][2], X[nt][3]), make_float2(to_f32(vb[0]), to_f32(vb[1])));
            X[nt][0] = x0.x, X[nt][1] = x0.y, X[nt][2] = x1.x, X[nt][3] = x1.y;
        }
        // d = X T^T: two terms each (the product of the small ones left out), of bf16, which has the range; T's columns beyond a row's
        // own are zero
        float d[CT][4] = {};
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            uint32_t hi[4], lo[4], b[CT][2];
#pragma unroll
            for (int nt = 2 * kt; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.w.tile[0]) + block_piece(8 * nt + b_row, 2 * kt + b_piece), x);
                b[nt][0] = x[0], b[nt][1] = x[1], b[nt + 1][0] = x[2], b[nt + 1][1] = x[3];
            }
            terms(kWide, X + 2 * kt, 1.f, 1.f, hi, lo);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; ++nt) mma16816(d[nt], hi, b[nt][0], b[nt][1], kWide);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; ++nt) mma16816(d[nt], lo, b[nt][0], b[nt][1], kWide);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.w.tile[1]) + block_piece(8 * nt + b_row, 2 * kt + b_piece), x);
                mma16816(d[nt], hi, x[0], x[1], kWide);
                mma16816(d[nt + 1], hi, x[2], x[3], kWide);
            }
        }
        float2 size = make_float2(0.f, 0.f);  // (infinite from 2^64 on, NaN with one in d or what it was made of)
#pragma unroll
        for (int nt = 0; nt < CT; ++nt)
            size = ptx::fma2(make_float2(d[nt][0], d[nt][1]), make_float2(d[nt][0], d[nt][1]),
                             ptx::fma2(make_float2(d[nt][2], d[nt][3]), make_float2(d[nt][2], d[nt][3]), size));
        odd |= !(size.x + size.y < INFINITY);
        // out = h Y + P d (two terms each without the product of the small ones)
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.h[8 * nt + t2]);
            times(Y[nt], kHalf ? ptx::mul2(f, make_float2(si0, si0)) : f, kHalf ? ptx::mul2(f, make_float2(si1, si1)) : f);
        }
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            uint32_t hi[4], lo[4], b[CT][2];
#pragma unroll
            for (int nt = 2 * kt; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.w.tile[2]) + block_piece(8 * nt + b_row, 2 * kt + b_piece), x);
                b[nt][0] = x[0], b[nt][1] = x[1], b[nt + 1][0] = x[2], b[nt + 1][1] = x[3];
            }
            terms(kWide, d + 2 * kt, 1.f, 1.f, hi, lo);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; ++nt) mma16816(Y[nt], hi, b[nt][0], b[nt][1], kWide);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; ++nt) mma16816(Y[nt], lo, b[nt][0], b[nt][1], kWide);
#pragma unroll
            for (int nt = 2 * kt; nt < CT; nt += 2) {
                uint32_t x[4];
                ldmatrix_x4(smem_u32(st.w.tile[3]) + block_piece(8 * nt + b_row, 2 * kt + b_piece), x);
                mma16816(Y[nt], hi, x[0], x[1], kWide);
                mma16816(Y[nt + 1], hi, x[2], x[3], kWide);
            }
        }
        // S <- e^G S + (w d) K, w d in two terms (f16: S in units of the terms meanwhile)
#pragma unroll
        for (int nt = 0; nt < CT; ++nt) {
            const float2 f = *reinterpret_cast<const float2 *>(&st.w.w[8 * nt + t2]);
            times(d[nt], f, f);
        }
        if (kHalf) {
            // (the state's part, below 2^12 all / its own scale, may be up to 2^20 larger in that unit)
            u0 = range_scale(fmaxf(top_of(d, CT, 0), st.w.all * si0 * 0x1p-8f)), u1 = range_scale(fmaxf(top_of(d, CT, 1), st.w.all * si1 * 0x1p-8f));
            odd |= beyond_scale(u0) || beyond_scale(u1);
        }
        if (__any_sync(0xffffffffu, odd)) {
            // row by row: something here is not finite, or far from it, and in a product would reach rows before it
#pragma unroll 1
            for (int r = 0; r < n; ++r) {
                const float gate = st.w.gate[r], beta = st.w.beta[r], rk = st.w.rk[r], rq = st.w.rq[r];
                float x[2] = {}, y[2] = {}, z = 0.f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const T *kp = reinterpret_cast<const T *>(st.k + piece<P>(r, nt)) + t2, *qp = reinterpret_cast<const T *>(st.q + piece<P>(r, nt)) + t2;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float k = to_f32(kp[e]) * rk, q = to_f32(qp[e]) * rq;
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
                float d[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    d[e] = beta * (to_f32(*reinterpret_cast<const T *>(st.v + piece<VP>(r, 2 * warp + e) + g * 2)) - x[e]);
                    if ((lane & 3u) == 0) reinterpret_cast<T *>(out + (uint64_t)r * a.o_token)[g + 8 * e] = from_f32<T>(a.scale * (y[e] + z * d[e]));
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const T *kp = reinterpret_cast<const T *>(st.k + piece<P>(r, nt)) + t2;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float k = to_f32(kp[e]) * rk;
                        S[nt][e] += k * d[0], S[nt][2 + e] += k * d[1];
                    }
                }
            }
            done();
            continue;
        }
        const float all0 = st.w.all * u0, all1 = st.w.all * u1;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) times(S[nt], make_float2(all0, all0), make_float2(all1, all1));
#pragma unroll
        for (int kt = 0; kt < C / 16; ++kt) {
            uint32_t hi[4], lo[4];
            terms(T(), d + 2 * kt, u0, u1, hi, lo);
#pragma unroll
            for (int n0 = 0; n0 < NT; n0 += 8) {
                uint32_t b[8][2];
#pragma unroll
                for (int nt = 0; nt < 8; nt += 2) {
                    uint32_t x[4];
                    ldmatrix_x4_trans(smem_u32(st.k) + piece<P>(16 * kt + (lane & 15u), n0 + nt + lane / 16), x);
                    b[nt][0] = x[0], b[nt][1] = x[1], b[nt + 1][0] = x[2], b[nt + 1][1] = x[3];
                }
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) mma16816(S[n0 + nt], hi, b[nt][0], b[nt][1], T());
#pragma unroll
                for (int nt = 0; nt < 8; ++nt) mma16816(S[n0 + nt], lo, b[nt][0], b[nt][1], T());
            }
        }
        if (kHalf) {
            const float i0 = flipped(u0), i1 = flipped(u1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) times(S[nt], make_float2(i0, i0), make_float2(i1, i1));
        }
        // rows of 16 columns through the warp's own part of V's tile
#pragma unroll
        for (int nt = 0; nt < CT; nt += 2)
            asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(
                             smem_u32(st.v) + piece<VP>(8 * nt + b_row, 2 * warp + b_piece)),
                         "r"(pack2(Y[nt][0], Y[nt][1], T())), "r"(pack2(Y[nt][2], Y[nt][3], T())),
                         "r"(pack2(Y[nt + 1][0], Y[nt + 1][1], T())), "r"(pack2(Y[nt + 1][2], Y[nt + 1][3], T()))
                         : "memory");
        __syncwarp();
#pragma unroll
        for (int i = 0; i < C / 16; ++i) {
            const int r = 16 * i + (int)lane / 2;
            const uint4 x = *reinterpret_cast<const uint4 *>(st.v + piece<VP>(r, 2 * warp + (lane & 1u)));
            if (r < n) *reinterpret_cast<uint4 *>(out + (uint64_t)r * a.o_token + (lane & 1u) * 16) = x;
        }
        done();
    }
    if (!to) return;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) to[at0 + (8 * nt + (e & 1)) * D + (e & 2) * 4] = S[nt][e];
}

template <class T, int D, int W, bool AGAIN>
__global__ void __launch_bounds__(SoloShape<D, W>::kThreads, SoloShape<D, W>::kCtas) kv_delta_solo_kernel(const __grid_constant__ DeltaArgs a)
{
    extern __shared__ __align__(16) uint8_t raw[];
    SoloSmem<D, W> &m = *reinterpret_cast<SoloSmem<D, W> *>(raw);
    constexpr uint32_t kParts = D / (16 * W);
    // Where some SMs have a second CTA from the start, they are those of the first CTAs, which therefore take the shorter sequences of
    // the first 148 (13 sequences of up to 2,001 rows, 16 heads of 64, us without / with: f16 154.7 / 146.5, bf16 150.5 / 142.4).
    constexpr uint32_t kSms = 148;
    const bool turned = SoloShape<D, W>::kCtas == 2 && gridDim.x > kSms && gridDim.x <= 2 * kSms && blockIdx.x < kSms;
    bool late = false;  // a wait has run out
    ptx::grid_launch_dependents();
    ptx::grid_wait();
    for (uint32_t item = turned ? kSms - 1 - blockIdx.x : blockIdx.x; item < a.n_seq * a.n_heads * kParts; item += gridDim.x) {
        const uint32_t s = a.order[item / kParts / a.n_heads];
        if (s >= a.n_seq) return;
        solo<T, D, W>(a, m, s, item / kParts % a.n_heads, item % kParts, late);
        if (!AGAIN) return;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int i = 0; i < SoloShape<D, W>::kStages; ++i) ptx::mbar_inval(smem_u32(&m.full[i])), ptx::mbar_inval(smem_u32(&m.empty[i]));
        }
    }
}

// More than half of an SM's shared memory: while the kernel ahead drains, two CTAs would come to share the first SMs that are free.
constexpr uint32_t kOneAnSm = 118784;

template <class T, int D, int W, bool AGAIN>
cudaError_t launch_relay(const DeltaArgs &a, uint32_t ctas, cudaStream_t s)
{
    static_assert(sizeof(RelaySmem<D, W>) <= 232448, "");
    static std::atomic<uint64_t> done;
    const cudaError_t e = allow_smem(kv_delta_relay_kernel<T, D, W, AGAIN>, 232448, done);
    if (e != cudaSuccess) return e;
    const uint32_t smem = sizeof(RelaySmem<D, W>) > kOneAnSm ? sizeof(RelaySmem<D, W>) : kOneAnSm;
    return launch_dependent(kv_delta_relay_kernel<T, D, W, AGAIN>, ctas, RelayShape<D, W>::kThreads, smem, s, a);
}
template <class T, int D, int W>
cudaError_t launch_relay(const DeltaArgs &a, cudaStream_t s)
{
    const uint32_t items = a.n_seq * a.n_heads * (D / (16 * W));
    return items <= kMany ? launch_relay<T, D, W, false>(a, items, s) : launch_relay<T, D, W, true>(a, 148 * 4, s);
}
template <class T, int D, int W, bool AGAIN>
cudaError_t launch_solo(const DeltaArgs &a, uint32_t ctas, cudaStream_t s)
{
    static_assert(sizeof(SoloSmem<D, W>) <= 232448, "");
    static std::atomic<uint64_t> done;
    const cudaError_t e = allow_smem(kv_delta_solo_kernel<T, D, W, AGAIN>, 232448, done);
    if (e != cudaSuccess) return e;
    const uint32_t threads = SoloShape<D, W>::kThreads, smem = sizeof(SoloSmem<D, W>);
    if (SoloShape<D, W>::kCtas == 1) return launch_dependent(kv_delta_solo_kernel<T, D, W, AGAIN>, ctas, threads, smem, s, a);
    // Two an SM: they start when the kernel ahead has ended, or the first two, the longest, come to share the first SM that is free
    // (13 sequences of up to 2,001 rows, 16 heads of 64: 179 us so, 142 us waiting; fp16 185 and 146 us).
    kv_delta_solo_kernel<T, D, W, AGAIN><<<ctas, threads, smem, s>>>(a);
    const cudaError_t f = cudaGetLastError();
    if (f == cudaSuccess) count_launches(1);
    return f;
}
template <class T, int D, int W>
cudaError_t launch_solo(const DeltaArgs &a, cudaStream_t s)
{
    const uint32_t items = a.n_seq * a.n_heads * (D / (16 * W));
    return items <= kMany ? launch_solo<T, D, W, false>(a, items, s) : launch_solo<T, D, W, true>(a, 148 * 8 * SoloShape<D, W>::kCtas, s);
}
// The lengths are on the device: where there are more than two sequences for every max_q rows, as many count as have max_q rows, the
// others being short.  While an SM each is enough for their slices (a pair of slices each), relays are faster, beyond that solos (us,
// the first kernel included, relay / solo, bf16: 1 sequence of 8,192 rows, 4 heads of 128 235 / 398, 32 heads of 128 335 / 443; 8 of
// 1,232 to 2,632, 6 heads of 64 116 / 128; 2 of 4,000, 32 heads of 128 331 / 253; 8 of 1,000 321 / 271; 4 of 100 to 4,000 411 / 366;
// 1 of 8,192, 32 heads of 64, one slice an SM 239, two 296, solo 337).
template <class T, int D>
cudaError_t launch(const DeltaArgs &a, cudaStream_t s)
{
    const uint64_t alike = ((uint64_t)a.total_q + a.max_q / 2) / a.max_q;
    const uint64_t slices = (a.n_seq <= 2 * alike ? a.n_seq : alike) * a.n_heads * (D / 16);
    if (slices <= 148) return launch_relay<T, D, 1>(a, s);
    return slices <= 2 * 148 ? launch_relay<T, D, 2>(a, s) : launch_solo<T, D, 4>(a, s);
}

}  // namespace

cudaError_t launch_delta_chain(const DeltaArgs &a, uint32_t dtype, uint32_t head_dim, cudaStream_t s)
{
    if (head_dim == 128) return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 128>(a, s) : launch<__half, 128>(a, s);
    return dtype == GMS_DTYPE_BF16 ? launch<__nv_bfloat16, 64>(a, s) : launch<__half, 64>(a, s);
}

}  // namespace gms
