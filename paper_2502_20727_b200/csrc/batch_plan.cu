// The plan of a serving step on the GPU (spd_plan_batch): row offsets, positions, slots and next lengths from the requests' lengths,
// pages of finished requests back to the pool, new pages out of it into the block tables.
//
// Everything is a prefix sum over the requests: of pages given back (they extend the pool in the requests' order), of pages and rows
// wanted (a request is served while neither sum passes what there is), of the rows served.  Rows then find their request by a
// binary search in the offsets.
//
// Bound: latency, of a few dependent steps (lengths, sums, pages given back, table entries); the bytes take well under a microsecond.  So
// one launch: a cluster of up to eight thread blocks, each of which forms all sums for itself from the lengths (cheaper
// than an exchange), gives back its share of the pages, and after one cluster barrier writes its share of the rows.
#include "../../include/spd.h"
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace spd {

namespace {

constexpr int PLAN_THREADS = 1024, PLAN_WARPS = PLAN_THREADS / 32, PLAN_MAX_CLUSTER = 8;
constexpr int PLAN_MAX_B = 16384; // two words of shared memory each

struct PlanArgs {
    const int32_t *lens, *news, *n_free;
    int32_t *table, *free_pages, *n_free_next, *cu, *positions, *slots, *next_lens;
    int B, max_pages, page, n_pages, n_tokens;
    int *err;
};

// Exclusive prefix sums of two numbers over the block's threads; the totals in `all`.
__device__ __forceinline__ longlong2 block_scan(longlong2 v, longlong2 &all, longlong2 *part)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    longlong2 x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, x.x, o), b = __shfl_up_sync(0xffffffffu, x.y, o);
        if (lane >= o) { x.x += a; x.y += b; }
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    longlong2 w = lane < PLAN_WARPS ? part[lane] : make_longlong2(0, 0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, w.x, o), b = __shfl_up_sync(0xffffffffu, w.y, o);
        if (lane >= o) { w.x += a; w.y += b; }
    }
    all = make_longlong2(__shfl_sync(0xffffffffu, w.x, 31), __shfl_sync(0xffffffffu, w.y, 31));
    const int before = warp ? warp - 1 : 0;
    const long long bx = __shfl_sync(0xffffffffu, w.x, before), by = __shfl_sync(0xffffffffu, w.y, before);
    __syncthreads(); // `part` may be written again
    return make_longlong2(x.x - v.x + (warp ? bx : 0), x.y - v.y + (warp ? by : 0));
}

__global__ void __launch_bounds__(PLAN_THREADS) plan_batch_kernel(const __grid_constant__ PlanArgs a)
{
    extern __shared__ int plan_sm[];
    int *cu = plan_sm, *at = cu + a.B + 1; // row offsets; a request's place among the pages given back or taken
    __shared__ longlong2 part[PLAN_WARPS];
    __shared__ int any_done;
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, rank = blockIdx.x, ranks = gridDim.x, warp = tid >> 5;
    const long capacity = (long)a.max_pages * a.page;
    auto pages_of = [&](long n) { return (int)((n + a.page - 1) / a.page); };
    auto flag = [&](int bit) { atomicOr(a.err, bit); };

    int n_free = *a.n_free;
    if (n_free < 0 || n_free > a.n_pages) {
        n_free = n_free < 0 ? 0 : a.n_pages;
        if (rank == 0 && tid == 0) flag(ERR_CAPACITY);
    }
    if (tid == 0) any_done = 0;
    __syncthreads();
    // Finished requests: their pages are counted (by a warp each, as entries outside the cache are passed over), placed, and given back by the
    // block whose turn it is.
    for (int b = tid; b < a.B; b += PLAN_THREADS) {
        const bool done = a.news[b] < 0;
        at[b] = done ? -1 : 0;
        if (done) any_done = 1;
    }
    __syncthreads();
    int top = n_free; // pages in the pool once all have been given back
    if (any_done) {
        for (int b = warp; b < a.B; b += PLAN_WARPS) {
            if (at[b] == 0) continue; // the same for the whole warp
            const long len = a.lens[b];
            int count = 0;
            if (len >= 0 && len <= capacity) {
                const int have = pages_of(len);
                for (int j0 = 0; j0 < have; j0 += 32) {
                    const int id = j0 + lane < have ? a.table[(long)b * a.max_pages + j0 + lane] : -1;
                    const bool good = id >= 0 && id < a.n_pages;
                    if (rank == 0 && !good && j0 + lane < have) flag(ERR_PAGE_RANGE);
                    count += __popc(__ballot_sync(0xffffffffu, good));
                }
            } else if (rank == 0 && lane == 0)
                flag(ERR_CAPACITY);
            __syncwarp();
            if (lane == 0) at[b] = count;
        }
        __syncthreads();
        long long sum = n_free;
        for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
            const int b = b0 + tid;
            longlong2 all;
            const longlong2 before = block_scan(make_longlong2(b < a.B ? at[b] : 0, 0), all, part);
            if (b < a.B) at[b] = (int)(sum + before.x < a.n_pages ? sum + before.x : a.n_pages);
            sum += all.x;
        }
        if (sum > a.n_pages) { // more pages than there are: some came back twice
            if (rank == 0 && tid == 0) flag(ERR_CAPACITY);
            sum = a.n_pages;
        }
        top = (int)sum;
        __syncthreads();
        for (int b = warp * ranks + rank; b < a.B; b += PLAN_WARPS * ranks) {
            if (a.news[b] >= 0) continue;
            const long len = a.lens[b];
            if (len < 0 || len > capacity) continue;
            const int have = pages_of(len);
            int to = at[b];
            for (int j0 = 0; j0 < have; j0 += 32) {
                const int id = j0 + lane < have ? a.table[(long)b * a.max_pages + j0 + lane] : -1;
                const unsigned good = __ballot_sync(0xffffffffu, id >= 0 && id < a.n_pages);
                const int place = to + __popc(good & ((1u << lane) - 1));
                if ((good >> lane & 1) && place < top) a.free_pages[place] = id;
                to += __popc(good);
            }
        }
    }

    // Requests with new tokens: pages and rows wanted up to each, then the rows of those that are served.
    long long wanted = 0, rows = 0;
    int served = 0, taken = 0;
    for (int b0 = 0; b0 < a.B; b0 += PLAN_THREADS) {
        const int b = b0 + tid;
        long len = 0, n = 0;
        int take = 0;
        bool done = false, bad = false;
        if (b < a.B) {
            len = a.lens[b];
            n = a.news[b];
            done = n < 0;
            if (done) n = 0;
            else if (len < 0 || len > capacity - n) { bad = true; n = 0; }
            if (n > 0) take = pages_of(len + n) - pages_of(len);
        }
        longlong2 all, mine;
        const longlong2 before = block_scan(make_longlong2(take, n), all, part);
        const long long take_to = wanted + before.x + take, rows_to = rows + before.y + n;
        const bool ok = (take == 0 || take_to <= top) && rows_to <= a.n_tokens;
        const int n_ok = ok ? (int)n : 0, take_ok = ok ? take : 0;
        const longlong2 got_before = block_scan(make_longlong2(n_ok, take_ok), mine, part);
        if (b < a.B) {
            cu[b] = served + (int)got_before.x;
            if (!done) at[b] = taken + (int)got_before.y;
            if (b % ranks == rank) {
                a.cu[b] = cu[b];
                a.next_lens[b] = done ? 0 : (int)len + n_ok;
                if (bad || !ok) flag(ERR_CAPACITY);
            }
        }
        wanted += all.x;
        rows += all.y;
        served += (int)mine.x;
        taken += (int)mine.y;
    }
    if (tid == 0) {
        cu[a.B] = served;
        if (rank == 0) a.cu[a.B] = served;
    }
    // Pages given back are in the pool, and every block has read its size.
    if (ranks > 1) tc::cluster_sync(); else __syncthreads();
    if (rank == 0 && tid == 0) *a.n_free_next = top - taken;

    for (int r = rank * PLAN_THREADS + tid; r < a.n_tokens; r += ranks * PLAN_THREADS) {
        int pos = -1, slot = -1;
        if (r < served) {
            int b = 0, end = a.B; // cu[b] <= r < cu[end]
            while (end - b > 1) {
                const int mid = (b + end) >> 1;
                if (cu[mid] <= r) b = mid; else end = mid;
            }
            const int len = a.lens[b];
            pos = len + (r - cu[b]);
            const int j = pos / a.page, in_page = pos - j * a.page, have = pages_of(len);
            int id;
            if (j < have) id = a.table[(long)b * a.max_pages + j];
            else {
                id = __ldcg(a.free_pages + (top - 1 - (at[b] + j - have)));
                if (in_page == 0) a.table[(long)b * a.max_pages + j] = id; // a new page's first row is always a new one
            }
            if (id < 0 || id >= a.n_pages) flag(ERR_PAGE_RANGE);
            else slot = id * a.page + in_page;
        }
        a.positions[r] = pos;
        a.slots[r] = slot;
    }
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
    if (B < 0 || B > PLAN_MAX_B || max_pages < 1 || n_tokens < 0 || (int64_t)max_pages * pool->kv_block_size > 0x7fffffffLL) return SPD_EINVAL;
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
