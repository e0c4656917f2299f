// Block tables and slot maps from request lengths.
#include "gms_internal.h"
#include "gms_kv_attn.h"
#include "gms_ptx.h"

namespace gms {
namespace {

struct PlanArgs {
    const int32_t *lens, *new_lens, *drop_lens;
    int32_t *lens_out, *table, *free_ids;
    const int32_t *free_state;
    int32_t *free_state_out, *cu_q;
    int64_t *slots;
    int32_t *positions;
    unsigned long long *status;
    uint64_t table_stride;
    uint32_t n_seq, total_rows, table_blocks, free_cap, n_blocks, block_shift;
};

constexpr uint32_t kPlanTile = 2048;  // sequences
constexpr uint32_t kPlanCtas = 8;     // of a cluster
constexpr int32_t kMostTokens = 1 << 30;
constexpr uint32_t kKept = 1024;      // ids that come back, a warp

// Sum over the threads before this one; `sh` has a word a warp and is free again after the caller's next two barriers.
template <uint32_t WARPS>
__device__ __forceinline__ uint64_t sum_before(uint64_t x, uint64_t *sh, uint64_t *all)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x / 32;
    uint64_t inc = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= (uint32_t)o) inc += y;
    }
    if (lane == 31) sh[warp] = inc;
    __syncthreads();
    uint64_t w = lane < WARPS ? sh[lane] : 0;
#pragma unroll
    for (uint32_t o = 1; o < WARPS; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
    }
    *all = __shfl_sync(0xffffffffu, w, WARPS - 1);
    const uint64_t warps = __shfl_sync(0xffffffffu, w, warp ? warp - 1 : 0);
    return inc - x + (warp ? warps : 0);
}

// What a tile's sequences have, for whoever looks for the owner of a row or of a block.
struct Tile {
    uint32_t row[kPlanTile + 1];   // first row
    uint32_t base[kPlanTile];      // position of that row
    uint32_t had[kPlanTile];       // blocks from before
    uint32_t rank[kPlanTile + 1];  // blocks that the ring gives to the sequences before (from the tile's first): at most 2^31
    uint32_t back[kPlanTile + 1];  // blocks that come back from the sequences before (from the tile's first)
};
// Last i < n with v[i] <= x (v ascending, v[0] <= x).
__device__ __forceinline__ uint32_t owner(const uint32_t *v, uint32_t n, uint32_t x)
{
    uint32_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (v[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ uint32_t blocks_of(uint32_t tokens, const PlanArgs &a)
{
    return min((tokens + (1u << a.block_shift) - 1u) >> a.block_shift, a.table_blocks);
}
__device__ __forceinline__ uint32_t clamped(int32_t x) { return (uint32_t)min(max(x, 0), kMostTokens); }

template <bool CLUSTER>
__device__ __forceinline__ void all_here()
{
    if (CLUSTER)
        asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    else
        __syncthreads();
}

// A word to the same place in every CTA of the cluster (a lane each).
template <bool CLUSTER>
__device__ __forceinline__ void tell_all(uint32_t *place, uint32_t x)
{
    const uint32_t lane = threadIdx.x & 31u;
    if (!CLUSTER) {
        if (lane == 0) *place = x;
    } else if (lane < kPlanCtas) {
        asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.u32 [a], %2;\n\t}" ::"r"(ptx::smem_u32(place)),
                     "r"(lane), "r"(x)
                     : "memory");
    }
}

// One CTA, or a cluster of eight that all scan the lengths for themselves and share rows and blocks out (a captured step costs one
// launch either way; the last CTA writes what is one word a sequence).  Nothing that one CTA reads is written by another: taken
// and returned places of the ring are different ones, so are entries that are looked up and entries that are new; lengths and the
// ring's state, which may be updated in place, are written behind a barrier.  Blocks that come back are looked at twice, a run of
// them a warp: how many are blocks, then, when all warps know what the others have, where they go; runs up to kKept come into shared
// memory at once (511 rows turning over, 179k such blocks: 17.2 us with both looks at the table, 15.3 us).  Bound by latency: four
// lengths a sequence, a scan, one or two words a row.
template <bool CLUSTER>
__global__ void __launch_bounds__(CLUSTER ? 1024 : 512) kv_plan_kernel(const __grid_constant__ PlanArgs a)
{
    constexpr uint32_t kPlanThreads = CLUSTER ? 1024 : 512, kPlanWarps = kPlanThreads / 32, kPlanEach = kPlanTile / kPlanThreads;
    constexpr uint32_t kAllWarps = (CLUSTER ? kPlanCtas : 1) * kPlanWarps, kLook = 8, kRows = 4;
    __shared__ uint32_t found[kAllWarps];  // blocks that each warp's run has
    extern __shared__ uint8_t raw[];
    Tile &t = *reinterpret_cast<Tile *>(raw);
    int32_t *keep = reinterpret_cast<int32_t *>(raw + sizeof(Tile));  // kKept for each warp
    __shared__ uint64_t sums[2][kPlanWarps];
    const uint32_t tid = threadIdx.x, n_cta = CLUSTER ? kPlanCtas : 1, cta = CLUSTER ? blockIdx.x : 0;
    const bool leader = cta == n_cta - 1;
    const uint32_t at = cta * kPlanThreads + tid, step = n_cta * kPlanThreads;
    ptx::grid_wait();
    ptx::grid_launch_dependents();
    const uint32_t cap = a.free_cap;
    const uint32_t head = cap ? (uint32_t)a.free_state[0] % cap : 0, count = cap ? (uint32_t)min(max(a.free_state[1], 0), (int)cap) : 0;
    uint64_t rows_before = 0, rank_before = 0;  // of all tiles before
    uint32_t returned = 0;                      // blocks that have come back so far
    const uint64_t most = a.total_rows;
    bool full = false;
    if (leader && tid == 0) a.cu_q[0] = 0;
    for (uint32_t s0 = 0; s0 < a.n_seq; s0 += kPlanTile) {
        const uint32_t n = min(a.n_seq - s0, kPlanTile), first = tid * kPlanEach;
        uint32_t len[kPlanEach], base[kPlanEach], rows[kPlanEach];
        uint64_t mine = 0;
#pragma unroll
        for (uint32_t i = 0; i < kPlanEach; ++i) {
            len[i] = base[i] = rows[i] = 0;
            if (first + i >= n) continue;
            const uint32_t s = s0 + first + i;
            len[i] = clamped(a.lens[s]);
            base[i] = a.drop_lens ? len[i] - min(len[i], clamped(a.drop_lens[s])) : len[i];
            rows[i] = clamped(a.new_lens[s]);
            mine += rows[i];
        }
        uint64_t all_rows;
        uint64_t row = rows_before + sum_before<kPlanWarps>(mine, sums[0], &all_rows);
        uint64_t moved[kPlanEach], mine_moved = 0;  // blocks taken in the low half, given back in the high half: at most 2^31 of a tile's each
#pragma unroll
        for (uint32_t i = 0; i < kPlanEach; ++i) {
            const uint64_t end = row + rows[i];
            if (end > a.total_rows) {
                full |= rows[i] != 0;
                rows[i] = row < a.total_rows ? (uint32_t)(a.total_rows - row) : 0;
            }
            const uint32_t had = blocks_of(len[i], a), need = blocks_of(base[i] + rows[i], a);
            moved[i] = need > had ? need - had : (uint64_t)(had - need) << 32;
            mine_moved += moved[i];
            if (first + i < n) {
                t.row[first + i] = (uint32_t)min(row, most);
                t.base[first + i] = base[i];
                t.had[first + i] = had;
            }
            row = end;
        }
        uint64_t all_moved;
        uint64_t before = sum_before<kPlanWarps>(mine_moved, sums[1], &all_moved);
#pragma unroll
        for (uint32_t i = 0; i < kPlanEach; ++i) {
            if (first + i < n) {
                t.rank[first + i] = (uint32_t)before;
                t.back[first + i] = (uint32_t)(before >> 32);
            }
            before += moved[i];
        }
        const uint32_t row0 = (uint32_t)min(rows_before, most), row1 = (uint32_t)min(rows_before + all_rows, most);
        if (tid == 0) {
            t.row[n] = row1;
            t.rank[n] = (uint32_t)all_moved;
            t.back[n] = (uint32_t)(all_moved >> 32);
        }
        all_here<CLUSTER>();  // the tile is there, and nobody reads the lengths any more
        if (leader) {
#pragma unroll
            for (uint32_t i = 0; i < kPlanEach; ++i) {
                if (first + i >= n) continue;
                a.lens_out[s0 + first + i] = (int32_t)(base[i] + rows[i]);
                a.cu_q[s0 + first + i + 1] = (int32_t)(t.row[first + i] + rows[i]);
            }
        }
        // where the ring's r-th block (from the tile's first) stands; null when it is empty
        auto place = [&](uint32_t r) -> const int32_t * {
            const uint64_t k = rank_before + r;
            if (k >= count) return nullptr;
            const uint32_t p = head + (uint32_t)k;
            return a.free_ids + (p < cap ? p : p - cap);
        };
        for (uint32_t r = at; r < t.rank[n]; r += step) {
            const uint32_t i = owner(t.rank, n, r);
            const int32_t *from = place(r);
            const int32_t id = from ? *from : -1;
            full |= !from;
            a.table[(uint64_t)(s0 + i) * a.table_stride + t.had[i] + (r - t.rank[i])] = id;
        }
        for (uint64_t x0 = row0 + at; x0 < row1; x0 += kRows * (uint64_t)step) {  // kRows look-ups a thread under way at once
            const int32_t *where[kRows];
            uint32_t pos[kRows];
            int32_t id[kRows];
#pragma unroll
            for (uint32_t k = 0; k < kRows; ++k) {
                const uint64_t x = x0 + k * (uint64_t)step;
                where[k] = nullptr;
                if (x >= row1) continue;
                const uint32_t i = owner(t.row, n, (uint32_t)x), had = t.had[i];
                pos[k] = t.base[i] + ((uint32_t)x - t.row[i]);
                const uint32_t b = pos[k] >> a.block_shift;
                if (b < had) where[k] = a.table + (uint64_t)(s0 + i) * a.table_stride + b;
                else if (b < a.table_blocks) where[k] = place(t.rank[i] + (b - had));
                else full = true;
            }
#pragma unroll
            for (uint32_t k = 0; k < kRows; ++k) id[k] = where[k] ? *where[k] : -1;
#pragma unroll
            for (uint32_t k = 0; k < kRows; ++k) {
                const uint64_t x = x0 + k * (uint64_t)step;
                if (x >= row1) continue;
                a.slots[x] = (uint32_t)id[k] < a.n_blocks ? ((int64_t)id[k] << a.block_shift) + (pos[k] & ((1u << a.block_shift) - 1u)) : -1;
                if (a.positions) a.positions[x] = (int32_t)pos[k];
            }
        }
        if (t.back[n]) {
            const uint32_t lane = tid & 31u, warp = cta * kPlanWarps + tid / 32, room = cap - count;
            const uint32_t run = (t.back[n] + kAllWarps * 32 - 1) / (kAllWarps * 32) * 32, r0 = min(warp * run, t.back[n]), r1 = min(r0 + run, t.back[n]);
            uint32_t i = 0;
            const uint32_t first_owner = r0 + lane < r1 ? owner(t.back, n, r0 + lane) : 0;
            // runs that shared memory has room for are fetched all at once
            const bool kept = run <= kKept;
            int32_t *mine = keep + tid / 32 * kKept;
            if (kept && r0 + lane < r1) {
                uint32_t o = first_owner, end = t.back[o + 1];
                const int32_t *p = a.table + ((int64_t)((uint64_t)(s0 + o) * a.table_stride + t.had[o]) - (int64_t)end);
                for (uint32_t r = r0 + lane; r < r1; r += 32) {
                    while (r >= end) {
                        end = t.back[++o + 1];
                        p = a.table + ((int64_t)((uint64_t)(s0 + o) * a.table_stride + t.had[o]) - (int64_t)end);
                    }
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(ptx::smem_u32(mine + (r - r0))), "l"(p + r) : "memory");
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
            }
            // the ids of up to kLook x 32 entries of the run from r on (a lane reads what it has fetched); owners go up with r
            auto look = [&](uint32_t r, int32_t *id) {
                if (kept) {
#pragma unroll
                    for (uint32_t k = 0; k < kLook; ++k) id[k] = r + 32 * k + lane < r1 ? mine[r + 32 * k + lane - r0] : -1;
                    return;
                }
                const uint32_t o = __shfl_sync(0xffffffffu, i, 0), end = t.back[o + 1];  // (lane 0 has the lowest owner)
                if (r + 32 * kLook <= min(end, r1)) {  // all of one sequence
                    const int32_t *p = a.table + (uint64_t)(s0 + o) * a.table_stride + t.had[o] - (end - r) + lane;
#pragma unroll
                    for (uint32_t k = 0; k < kLook; ++k) id[k] = p[32 * k];
                    i = o;
                    return;
                }
                uint32_t at[kLook];
#pragma unroll
                for (uint32_t k = 0; k < kLook; ++k) {
                    at[k] = r + 32 * k + lane;
                    id[k] = -1;
                    if (at[k] >= r1) continue;
                    while (t.back[i + 1] <= at[k]) ++i;
                    id[k] = a.table[(uint64_t)(s0 + i) * a.table_stride + t.had[i] - (t.back[i + 1] - at[k])];
                }
            };
            uint32_t mine_found = 0;
            i = first_owner;
            for (uint32_t r = r0; r < r1; r += 32 * kLook) {
                int32_t id[kLook];
                look(r, id);
#pragma unroll
                for (uint32_t k = 0; k < kLook; ++k) mine_found += __popc(__ballot_sync(0xffffffffu, (uint32_t)id[k] < a.n_blocks));
            }
            tell_all<CLUSTER>(&found[warp], mine_found);
            all_here<CLUSTER>();
            uint32_t before = 0, all = 0;
            for (uint32_t w = lane; w < kAllWarps; w += 32) {
                all += found[w];
                if (w < warp) before += found[w];
            }
            before = returned + __reduce_add_sync(0xffffffffu, before);
            all = __reduce_add_sync(0xffffffffu, all);
            i = first_owner;
            for (uint32_t r = r0; r < r1; r += 32 * kLook) {
                int32_t id[kLook];
                look(r, id);
#pragma unroll
                for (uint32_t k = 0; k < kLook; ++k) {
                    const bool is = (uint32_t)id[k] < a.n_blocks;
                    const uint32_t which = __ballot_sync(0xffffffffu, is), to = before + __popc(which & ((1u << lane) - 1u));
                    before += __popc(which);
                    if (is && to < room) {
                        const uint32_t p = head + count, q = (p >= cap ? p - cap : p) + to;
                        a.free_ids[q >= cap ? q - cap : q] = id[k];
                    } else {
                        full |= is;
                    }
                }
            }
            returned = min(returned + all, room);
        }
        rows_before += all_rows;
        rank_before += (uint32_t)all_moved;
        __syncthreads();  // the tile and the sums may be written again
    }
    for (uint64_t x = min(rows_before, most) + at; x < a.total_rows; x += step) {
        a.slots[x] = -1;
        if (a.positions) a.positions[x] = 0;
    }
    if (a.n_seq == 0) all_here<CLUSTER>();  // (with sequences the barriers above stand between the reads and this)
    if (leader && tid == 0) {
        const uint32_t out = (uint32_t)min(rank_before, (uint64_t)count);
        const uint32_t p = head + out;
        a.free_state_out[0] = (int32_t)(cap && p >= cap ? p - cap : p);
        a.free_state_out[1] = (int32_t)(count - out + returned);
    }
    if (full && a.status) atomicOr(a.status, (unsigned long long)GMS_DEV_FULL);
}

cudaError_t launch_plan(const PlanArgs &a, cudaStream_t s)
{
    static std::atomic<uint64_t> done[2];
    // Eight CTAs pay where there is more to do than a second start and their exchange cost (us, one CTA / eight; rows a sequence x sequences:
    // 1 x 512 4.9 / 5.8, 1 x 1,024 6.3 / 6.4, 1 x 2,048 9.1 / 6.7, 16 x 128 6.4 / 5.7, 2,000 x 1 4.2 / 4.8, 4,000 x 1 5.3 / 4.8,
    // 1,000 x 8 9.8 / 5.2, 64 x 511 53.8 / 8.9).
    const bool cluster = (uint64_t)a.total_rows + a.n_seq > 2048;
    const uint32_t threads = cluster ? 1024 : 512, smem = sizeof(Tile) + threads / 32 * kKept * 4;
    cudaError_t e = cluster ? allow_smem(kv_plan_kernel<true>, smem, done[1]) : allow_smem(kv_plan_kernel<false>, smem, done[0]);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster ? kPlanCtas : 1);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = kPlanCtas;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster ? 2 : 1;
    e = cluster ? cudaLaunchKernelEx(&cfg, kv_plan_kernel<true>, a) : cudaLaunchKernelEx(&cfg, kv_plan_kernel<false>, a);
    if (e == cudaSuccess) count_launches(1);
    return e;
}

}  // namespace
}  // namespace gms

extern "C" int gms_kv_plan(const gms_kv_plan_args *t, void *stream)
{
    if (!t) return GMS_ERR_NULL;
    if (t->block_tokens < 16 || t->block_tokens > 1024 || t->block_tokens & (t->block_tokens - 1)) return GMS_ERR_ARG;
    if (t->n_blocks == 0 || t->n_blocks > 0x7fffffffu || t->total_rows > 0x7fffffffu || t->n_seq > 0x7fffffffu || t->free_cap > 0x7fffffffu)
        return GMS_ERR_ARG;
    // (blocks are counted in 32 bits over the sequences of a tile)
    if (t->table_stride > 1ull << 40 || t->table_blocks > t->table_stride || t->table_blocks > 1u << 20) return GMS_ERR_RANGE;
    if ((reinterpret_cast<uint64_t>(t->lens) | reinterpret_cast<uint64_t>(t->new_lens) | reinterpret_cast<uint64_t>(t->drop_lens) |
         reinterpret_cast<uint64_t>(t->lens_out) | reinterpret_cast<uint64_t>(t->block_table) | reinterpret_cast<uint64_t>(t->free_ids) |
         reinterpret_cast<uint64_t>(t->free_state) | reinterpret_cast<uint64_t>(t->free_state_out) | reinterpret_cast<uint64_t>(t->cu_q) |
         reinterpret_cast<uint64_t>(t->positions)) & 3u ||
        (reinterpret_cast<uint64_t>(t->slots) | reinterpret_cast<uint64_t>(t->status)) & 7u)
        return GMS_ERR_ALIGN;
    if (!t->free_state || !t->free_state_out || !t->cu_q || (t->free_cap && !t->free_ids) || (t->total_rows && !t->slots)) return GMS_ERR_NULL;
    if (t->n_seq && (!t->lens || !t->new_lens || !t->lens_out || (t->table_blocks && !t->block_table))) return GMS_ERR_NULL;
    auto meet = [](const void *x, uint64_t nx, const void *y, uint64_t ny) {
        const uint64_t p = reinterpret_cast<uint64_t>(x), q = reinterpret_cast<uint64_t>(y);
        return p < q + ny && q < p + nx;
    };
    const uint64_t words = 4ull * t->n_seq;
    if (t->lens_out != t->lens && meet(t->lens_out, words, t->lens, words)) return GMS_ERR_ARG;
    if (meet(t->lens_out, words, t->new_lens, words) || (t->drop_lens && meet(t->lens_out, words, t->drop_lens, words))) return GMS_ERR_ARG;
    if (t->free_state_out != t->free_state && meet(t->free_state_out, 8, t->free_state, 8)) return GMS_ERR_ARG;
    gms::PlanArgs a = {};
    a.lens = t->lens;
    a.new_lens = t->new_lens;
    a.drop_lens = t->drop_lens;
    a.lens_out = t->lens_out;
    a.table = t->block_table;
    a.free_ids = t->free_ids;
    a.free_state = t->free_state;
    a.free_state_out = t->free_state_out;
    a.cu_q = t->cu_q;
    a.slots = t->slots;
    a.positions = t->positions;
    a.status = reinterpret_cast<unsigned long long *>(t->status);
    a.table_stride = t->table_stride;
    a.n_seq = t->n_seq;
    a.total_rows = t->total_rows;
    a.table_blocks = t->table_blocks;
    a.free_cap = t->free_cap;
    a.n_blocks = t->n_blocks;
    a.block_shift = gms::log2_of(t->block_tokens);
    const cudaError_t e = gms::launch_plan(a, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? GMS_OK : gms::report_cuda_error(e);
}
