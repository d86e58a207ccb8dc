// The plan of a serving step on the GPU (spd_plan_batch): row offsets, positions, slots and next lengths from the requests' lengths,
// pages of finished requests back to the pool, new pages out of it into the block tables.
//
// Everything is a prefix sum over the requests: of pages given back (they extend the pool in the requests' order), of pages and rows
// wanted (a request is served while neither sum passes what there is), of the rows served.  Rows then find their request by a search
// in the offsets.
//
// Bound: latency, of a few dependent steps (lengths, sums, pages given back, table entries); the bytes take well under a microsecond.  So
// one launch: a cluster of up to eight thread blocks, each of which forms all sums for itself from the lengths (cheaper
// than an exchange), gives back its share of the pages, and after a cluster barrier writes its share of the rows.
// 256 single tokens 4.6 us; 2048 requests, 81 thousand rows, 100 of them finished 22.7 (sums 6, pages given back 7, rows 8; with 16 blocks, which not
// every GPU can place, 3 less; sums of 64 bits and a search per row took 48).
#include "../../include/spd.h"
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace spd {

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32, PLAN_MAX_CLUSTER = 8;
constexpr int PLAN_MAX_B = 16384; // two words of shared memory each
constexpr int PLAN_MAX_TOKENS = 1 << 30; // row numbers and strides between them stay within 32 bits

struct PlanArgs {
    const int32_t *lens, *news, *n_free;
    int32_t *table, *free_pages, *n_free_next, *cu, *positions, *slots, *next_lens;
    int B, max_pages, page, n_pages, n_tokens;
    int *err;
};

// Sums that stop at the largest number: what is wanted may be more than there is by any amount.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { const uint32_t s = a + b; return s < a ? 0xffffffffu : s; }
__device__ __forceinline__ uint2 add_sat(uint2 a, uint2 b) { return make_uint2(add_sat(a.x, b.x), add_sat(a.y, b.y)); }

// Exclusive prefix sums of two numbers over the block's threads; the totals in `all`.
__device__ __forceinline__ uint2 block_scan(uint2 v, uint2 &all, uint2 *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto before = [&](uint2 x) { // inclusive sums over the lanes, then one lane up
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint2 y = make_uint2(__shfl_up_sync(0xffffffffu, x.x, o), __shfl_up_sync(0xffffffffu, x.y, o));
            if (lane >= o) x = add_sat(x, y);
        }
        return x;
    };
    const uint2 x = before(v);
    if (lane == 31) part[warp] = x;
    __syncthreads();
    const uint2 w = before(part[lane]);
    all = make_uint2(__shfl_sync(0xffffffffu, w.x, 31), __shfl_sync(0xffffffffu, w.y, 31));
    const uint2 warps = make_uint2(__shfl_sync(0xffffffffu, w.x, (warp + 31) & 31), __shfl_sync(0xffffffffu, w.y, (warp + 31) & 31));
    const uint2 lanes = make_uint2(__shfl_up_sync(0xffffffffu, x.x, 1), __shfl_up_sync(0xffffffffu, x.y, 1));
    __syncthreads(); // `part` may be written again
    const uint2 zero = make_uint2(0, 0);
    return add_sat(warp ? warps : zero, lane ? lanes : zero);
}
static_assert(PLAN_WARPS == 32, "a lane per warp");

// Positions and slots of the rows, entries of the tables' new pages.  cu: row offsets; at: places of the requests' first new pages among those taken.
// A warp takes GROUPS x 32 consecutive rows: one search for the first one's request, then, 32 rows at a time, the next 32 offsets in the lanes.  (A search
// per row, or one per thread with four rows each, whose stores then lie apart: 13 us of a mixed step's 26.)
struct Fill {
    const int *cu, *at;
    int served, top, lg;
    __device__ __forceinline__ int page_of(int pos, int page) const { return lg >= 0 ? pos >> lg : pos / page; }
    template <int GROUPS> __device__ __forceinline__ void rows(const PlanArgs &a, int rank, int ranks) const
    {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
        for (int w0 = (rank * PLAN_WARPS + warp) * 32 * GROUPS; w0 < a.n_tokens; w0 += ranks * PLAN_THREADS * GROUPS) {
            int b[GROUPS], id[GROUPS], pos[GROUPS], j[GROUPS];
            if (w0 < served) {
                int lo = 0, end = a.B; // cu[lo] <= w0 < cu[end]; the same for the warp
                while (end - lo > 1) {
                    const int mid = (lo + end) >> 1;
                    if (cu[mid] <= w0) lo = mid; else end = mid;
                }
#pragma unroll
                for (int i = 0; i < GROUPS; ++i) {
                    const int r = w0 + 32 * i + lane, last = min(w0 + 32 * i + 31, served - 1);
                    while (true) { // lanes' requests: lo and how many of the next 32 start at or before the row
                        const int start = lo + 1 + lane < a.B ? cu[lo + 1 + lane] : served;
                        int n = 0;
                        if (__shfl_sync(0xffffffffu, start, 0) <= last) {
#pragma unroll
                            for (int step = 16; step > 0; step >>= 1) n += __shfl_sync(0xffffffffu, start, n + step - 1) <= r ? step : 0;
                            n += __shfl_sync(0xffffffffu, start, n) <= r;
                        }
                        if (cu[lo] <= r) b[i] = lo + n; // always so in the first turn
                        // all 32 start within the group: there may be more
                        if (__shfl_sync(0xffffffffu, start, 31) > last) break;
                        lo += 32;
                    }
                    lo = __shfl_sync(0xffffffffu, b[i], last - (w0 + 32 * i) < 0 ? 0 : last - (w0 + 32 * i)); // the last row's, for the next group
                }
            }
            // the loads of all rows at once, one kind after the other
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) pos[i] = w0 + 32 * i + lane < served ? a.lens[b[i]] : 0;
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                const int r = w0 + 32 * i + lane;
                id[i] = j[i] = -1;
                if (r >= served) continue;
                const int have = pos[i] ? page_of(pos[i] - 1, a.page) + 1 : 0;
                pos[i] += r - cu[b[i]];
                j[i] = page_of(pos[i], a.page);
                id[i] = j[i] < have ? a.table[(long)b[i] * a.max_pages + j[i]] : __ldcg(a.free_pages + (top - 1 - (at[b[i]] + j[i] - have)));
                if (j[i] < have) j[i] |= 0x80000000; // not a new page
            }
#pragma unroll
            for (int i = 0; i < GROUPS; ++i) {
                const int r = w0 + 32 * i + lane, in_page = pos[i] - (j[i] & 0x7fffffff) * a.page;
                if (r >= a.n_tokens) break;
                const bool mine = r < served, good = mine && (uint32_t)id[i] < (uint32_t)a.n_pages;
                if (mine && in_page == 0 && j[i] >= 0) a.table[(long)b[i] * a.max_pages + j[i]] = id[i]; // a new page's first row is always a new one
                if (mine && !good) atomicOr(a.err, ERR_PAGE_RANGE);
                a.positions[r] = mine ? pos[i] : -1;
                a.slots[r] = good ? id[i] * a.page + in_page : -1;
            }
        }
    }
};

__global__ void __launch_bounds__(PLAN_THREADS, 1) plan_batch_kernel(const __grid_constant__ PlanArgs a)
{
    extern __shared__ int plan_sm[];
    int *cu = plan_sm, *at = cu + a.B + 1; // row offsets; a request's place among the pages given back or taken
    int *list = cu; // before the row offsets are made: finished requests that this block looks after
    __shared__ uint2 part[PLAN_WARPS];
    __shared__ int n_done;
    __shared__ volatile int any_bad;
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, rank = blockIdx.x, ranks = gridDim.x, warp = tid >> 5;
    const long capacity = (long)a.max_pages * a.page;
    const int lg = a.page & (a.page - 1) ? -1 : __ffs(a.page) - 1; // page sizes are mostly powers of two
    auto page_of = [&](int pos) { return lg >= 0 ? pos >> lg : pos / a.page; };
    auto pages_of = [&](int n) { return n ? page_of(n - 1) + 1 : 0; };
    auto flag = [&](int bit) { atomicOr(a.err, bit); };
    auto set_flag = [&](int block) { // any_bad of a block of the cluster
        const uint32_t mine = tc::smem_u32((const void *)&any_bad);
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(ranks > 1 ? tc::mapa_shared(mine, block) : mine), "r"(1) : "memory");
    };

    int n_free = *a.n_free;
    if (n_free < 0 || n_free > a.n_pages) {
        n_free = n_free < 0 ? 0 : a.n_pages;
        if (rank == 0 && tid == 0) flag(ERR_CAPACITY);
    }
    // Finished requests: their pages join the pool.  Once as if all their entries named pages (then how many there are is known from the lengths);
    // if that is not so, once more with entries outside the cache passed over.
    if (tid == 0) n_done = any_bad = 0;
    __syncthreads();
    // every block has read the pool's size and set its flag to 0: waited for where that matters
    if (ranks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    auto all_started = [&] {
        if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        __syncthreads();
    };
    bool some = false;
    for (int b = tid; b < a.B; b += PLAN_THREADS) {
        at[b] = 0;
        if (a.news[b] >= 0) continue;
        some = true;
        const int len = a.lens[b];
        if (len >= 0 && len <= capacity) at[b] = pages_of(len);
        else if (rank == 0) flag(ERR_CAPACITY);
        if (b % ranks == rank) list[atomicAdd(&n_done, 1)] = b; // this block's; their order does not matter
    }
    const bool any_done = __syncthreads_or(some);
    int top = n_free; // pages in the pool once all have been given back
    for (bool again = false; any_done; again = true) {
        if (again) { // pages that exist
            for (int b = warp; b < a.B; b += PLAN_WARPS) {
                if (a.news[b] >= 0) continue;
                const int len = a.lens[b], have = len >= 0 && len <= capacity ? pages_of(len) : 0;
                int count = 0;
                for (int j = lane; j < have; j += 32) count += (uint32_t)a.table[(long)b * a.max_pages + j] < (uint32_t)a.n_pages;
                count = __reduce_add_sync(0xffffffffu, count);
                if (lane == 0) at[b] = count;
            }
            __syncthreads();
        }
        uint32_t sum = n_free;
        for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
            const int b = b0 + tid;
            uint2 all;
            const uint2 before = block_scan(make_uint2(b < a.B && a.news[b] < 0 ? at[b] : 0, 0), all, part);
            if (b < a.B) at[b] = (int)min(add_sat(sum, before.x), (uint32_t)a.n_pages);
            sum = add_sat(sum, all.x);
        }
        top = (int)min(sum, (uint32_t)a.n_pages);
        if (again) __syncthreads(); else all_started(); // the places are there, and the other blocks' flags may be raised
        for (int k = warp; k < n_done; k += PLAN_WARPS) {
            const int b = list[k], len = a.lens[b], have = len >= 0 && len <= capacity ? pages_of(len) : 0;
            int to = at[b];
#pragma unroll 4
            for (int j0 = 0; j0 < have; j0 += 32) {
                const int id = j0 + lane < have ? a.table[(long)b * a.max_pages + j0 + lane] : 0;
                const bool good = j0 + lane < have && (uint32_t)id < (uint32_t)a.n_pages;
                const unsigned all = __ballot_sync(0xffffffffu, good);
                const int place = again ? to + __popc(all & ((1u << lane) - 1)) : to + lane;
                if (good && place < top) a.free_pages[place] = id;
                if (!again && j0 + lane < have && !good) {
                    flag(ERR_PAGE_RANGE);
                    for (int c = 0; c < ranks; ++c) set_flag(c);
                }
                to += again ? __popc(all) : 32;
            }
        }
        // Pages given back are in the pool.
        if (ranks > 1) tc::cluster_sync(); else __syncthreads();
        if (again || !any_bad) {
            if (sum > (uint32_t)a.n_pages && rank == 0 && tid == 0) flag(ERR_CAPACITY); // more pages than there are: some came back twice
            break;
        }
    }

    // Requests with new tokens: pages and rows wanted up to each, then the rows of those that are served.
    uint32_t wanted = 0, rows = 0;
    int served = 0, taken = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        int len = 0, n = 0, take = 0;
        bool done = false, bad = false;
        if (b < a.B) {
            len = a.lens[b];
            n = a.news[b];
            done = n < 0;
            if (done) n = 0;
            else if (len < 0 || len > capacity - n) { bad = true; n = 0; }
            if (n > 0) take = pages_of(len + n) - pages_of(len);
        }
        uint2 all, mine;
        const uint2 before = block_scan(make_uint2(take, n), all, part);
        const uint32_t take_to = add_sat(add_sat(wanted, before.x), take), rows_to = add_sat(add_sat(rows, before.y), n);
        const bool ok = (take == 0 || take_to <= (uint32_t)top) && rows_to <= (uint32_t)a.n_tokens;
        const int n_ok = ok ? n : 0, take_ok = ok ? take : 0;
        uint2 got = before;
        if (__syncthreads_and(ok)) mine = all; // the usual case: all of them are served
        else got = block_scan(make_uint2(take_ok, n_ok), mine, part);
        if (b < a.B) {
            cu[b] = served + (int)got.y;
            if (!done) at[b] = taken + (int)got.x;
            if (b % ranks == rank) {
                a.cu[b] = cu[b];
                a.next_lens[b] = done ? 0 : len + n_ok;
                if (bad || !ok) flag(ERR_CAPACITY);
            }
        }
        wanted = add_sat(wanted, all.x);
        rows = add_sat(rows, all.y);
        served += (int)mine.y;
        taken += (int)mine.x;
    }
    if (tid == 0) {
        cu[a.B] = served;
        if (rank == 0) a.cu[a.B] = served;
    }
    if (any_done) __syncthreads(); else all_started(); // the offsets are there, and every block has read the pool's size
    if (rank == 0 && tid == 0) *a.n_free_next = top - taken;

    // where the rows are many, four groups of them share a search and the waiting for their loads
    const Fill f{cu, at, served, top, lg};
    if (a.n_tokens > ranks * PLAN_THREADS) f.rows<4>(a, rank, ranks);
    else f.rows<1>(a, rank, ranks);
}

} // namespace

} // namespace spd

using namespace spd;

extern "C" int spd_plan_batch(const spd_page_pool *pool, const int32_t *seq_lens, const int32_t *new_lens, int32_t B, int32_t *block_table,
                              int32_t max_pages, int32_t n_tokens, int32_t *cu_new, int32_t *positions, int32_t *slots, int32_t *next_lens,
                              int32_t *err_flag, void *stream)
{
    if (!pool) return SPD_ENULL;
    if (pool->n_pages < 1 || pool->kv_block_size < 1 || (int64_t)pool->n_pages * pool->kv_block_size > 0x7fffffffLL) return SPD_EINVAL;
    if (B < 0 || B > PLAN_MAX_B || max_pages < 1 || n_tokens < 0 || n_tokens > PLAN_MAX_TOKENS || (int64_t)max_pages * pool->kv_block_size > 0x7fffffffLL) return SPD_EINVAL;
    if (!pool->free_pages || !pool->n_free || !pool->n_free_next || !cu_new || !err_flag) return SPD_ENULL;
    if (B && (!seq_lens || !new_lens || !block_table || !next_lens)) return SPD_ENULL;
    if (n_tokens && (!positions || !slots)) return SPD_ENULL;
    if (B && (next_lens == seq_lens || next_lens == new_lens)) return SPD_EINVAL; // still read while they are written
    const PlanArgs a{seq_lens, new_lens, pool->n_free, block_table, pool->free_pages, pool->n_free_next, cu_new, positions, slots, next_lens, B,
                     max_pages, pool->kv_block_size, pool->n_pages, n_tokens, err_flag};
    static SmemLimit limit;
    cudaError_t e = limit.raise((const void *)plan_batch_kernel, (2 * PLAN_MAX_B + 1) * 4);
    // a block per 1024 rows: one alone needs no cluster
    int ranks = 1;
    while (ranks < PLAN_MAX_CLUSTER && (long)ranks * PLAN_THREADS < n_tokens) ranks *= 2;
    if (e == cudaSuccess) e = launch_kernel(plan_batch_kernel, dim3(ranks), dim3(PLAN_THREADS), (2 * (size_t)B + 1) * 4, (cudaStream_t)stream, ranks, a);
    if (e != cudaSuccess) { note_cuda_error(e); return SPD_ECUDA; }
    return SPD_OK;
}
