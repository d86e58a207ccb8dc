// Attention of a chunk of new tokens per sequence over a paged K/V cache (spd_paged_attention): checks, choice of kernel,
// the kernel that serves every type, and the merge of key ranges.
//
// Query i of sequence b sits at position p = lens[b] + i and sees the keys t <= p with t > p - window or t < sinks
// (window 0: all t <= p):  out = sum_t softmax_t(scale q . k_t) v_t.  It always sees itself, so no row is empty.
#include "../../include/spd.h"
#include "paged.cuh"

#include <math.h>

namespace spd {

namespace {

// Every type (float32 queries, head_dim 32; not float32 over 4-bit pages of head_dim 64 and 128): CUDA cores, float32 throughout.  A thread block takes 16 RPT packed rows (row r = new
// token r / group, query head r % group, so that a group shares the K/V tiles) and walks tiles of 64 keys, widened to float32
// in shared memory.  Thread (tx, ty) computes the scores of rows ty RPT .. and keys tx + 16 j, four head dims at a time (eight
// products per 16-byte shared-memory load), the row maxima and sums over its half warp, and the output columns 4 tx + 64 j.
// Bound: for chunks shared-memory loads beside the FMAs and the blocks of the longest sequences, for few rows (RPT 1) the cache
// reads, which are cut into key ranges over thread blocks.
// One warp per row, without tiles, took 259 us for 4 ragged chunks of up to 256 tokens where this takes 30 (head_dim 64).
constexpr int GK = 64, G_THREADS = 256;

// float32 caches: the next tile is on its way (cp.async) while this one is computed
template <int FMT, int D, int RPT> struct GenCfg {
    static constexpr int RT = 16 * RPT, LD = D + 4, LP = GK + 4, BUFS = FMT == KV_F32 ? 2 : 1;
    static constexpr int SMEM = (RT * LD + BUFS * 2 * GK * LD + RT * LP) * 4;
};

__device__ __forceinline__ void cp16(void *dst, const void *src, bool valid)
{
    const int n = valid ? 16 : 0; // 0 source bytes: zero fill
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(n) : "memory");
}

template <int FMT> __device__ __forceinline__ float4 cache4(const PagedKv &kv, const void *pages, const float *scales, long row, int D, int c)
{
    if (FMT == KV_F32) return *(const float4 *)((const float *)pages + row * D + c * 4);
    if (FMT == KV_BF16) {
        const uint2 u = *(const uint2 *)((const bf16 *)pages + row * D + c * 4);
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
    }
    if constexpr (FMT == KV_INT4) { // four dims of one half
        const bool high = c * 4 >= D / 2;
        const uint32_t w = *(const uint32_t *)((const uint8_t *)pages + row * (D / 2) + (high ? c * 4 - D / 2 : c * 4)) >> (high ? 4 : 0);
        const uint2 p = kv4_params(scales, row);
        const float s = kv4_scale(high ? p.y : p.x), m = kv4_min(high ? p.y : p.x);
        return make_float4(fmaf((float)(w & 15), s, m), fmaf((float)(w >> 8 & 15), s, m), fmaf((float)(w >> 16 & 15), s, m),
                           fmaf((float)(w >> 24 & 15), s, m));
    }
    typedef typename KvElem<FMT>::type E;
    const uint32_t w = *(const uint32_t *)((const uint8_t *)pages + row * D + c * 4);
    const float s = scales[row];
    if constexpr (FMT == KV_E4M3 || FMT == KV_INT8)
        return make_float4(kv_value<FMT>((E)w) * s, kv_value<FMT>((E)(w >> 8)) * s, kv_value<FMT>((E)(w >> 16)) * s, kv_value<FMT>((E)(w >> 24)) * s);
    return make_float4(0.f, 0.f, 0.f, 0.f);
}

template <typename T, int FMT, int D, int RPT>
__global__ void __launch_bounds__(G_THREADS) paged_attention_general_kernel(const __grid_constant__ PagedAttnArgs a)
{
    using C = GenCfg<FMT, D, RPT>;
    constexpr int RT = C::RT, LD = C::LD, LP = C::LP, OC = D < 64 ? 1 : D / 64; // groups of 4 output columns per thread (D 32: half the threads)
    extern __shared__ __align__(16) float gsm[];
    float *sQ = gsm, *sKV = sQ + RT * LD, *sP = sKV + C::BUFS * 2 * GK * LD;
    if (threadIdx.x == 0) stamp_entry(a.stamp);
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.z / a.splits, split = blockIdx.z % a.splits, kvh = blockIdx.y;
    int row0, n_new, len;
    if (!batch_row(a.rb, b, a.max_new, a.max_context, row0, n_new, len, a.err)) return;
    const int r0 = blockIdx.x * RT, all_rows = n_new * a.group;
    if (r0 >= all_rows) return;
    const int rows = min(RT, all_rows - r0), tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int pos_first = len + r0 / a.group, pos_last = len + (r0 + rows - 1) / a.group, kv_len = pos_last + 1;
    // tiles of 64 keys that hold a key some row sees: sinks, then the window of the first row onwards
    const int lo_min = a.window ? max(0, pos_first - a.window + 1) : 0, first = lo_min / GK;
    const int n_sink = min((min(a.sinks, lo_min) + GK - 1) / GK, first);
    const int n_all = n_sink + (kv_len + GK - 1) / GK - first;
    const int j_begin = (int)((long)n_all * split / a.splits), j_end = (int)((long)n_all * (split + 1) / a.splits);
    const int32_t *bt = a.rb.table + (long)b * a.rb.max_pages;

    for (int i = tid; i < RT * (D / 4); i += G_THREADS) {
        const int r = i / (D / 4), c = i % (D / 4), rr = r0 + r;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) {
            const T *p = (const T *)a.q + (long)(row0 + rr / a.group) * a.q_stride + (long)(kvh * a.group + rr % a.group) * D + c * 4;
            x = make_float4(to_f<T>(p[0]), to_f<T>(p[1]), to_f<T>(p[2]), to_f<T>(p[3]));
        }
        *(float4 *)(sQ + r * LD + c * 4) = x;
    }
    float o[RPT][OC][4], m[RPT], l[RPT];
    int pos[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int r = ty * RPT + i;
        pos[i] = r < rows ? len + (r0 + r) / a.group : -1;
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int k = 0; k < OC; ++k) o[i][k][0] = o[i][k][1] = o[i][k][2] = o[i][k][3] = 0.f;
    }
    auto key0 = [&](int j) { return (j < n_sink ? j : first + (j - n_sink)) * GK; };
    auto load_tile = [&](int j) {
        float *dK = sKV + (C::BUFS == 2 ? (j - j_begin) & 1 : 0) * 2 * GK * LD, *dV = dK + GK * LD;
        const int t0 = key0(j);
#pragma unroll 4
        for (int i = tid; i < GK * (D / 4); i += G_THREADS) {
            const int r = i / (D / 4), c = i % (D / 4), t = t0 + r;
            long row = -1;
            if (t < kv_len && (t >= lo_min || t < a.sinks)) { // keys that no row sees come as zeros
                const int pi = t / a.kv.page, page = bt[pi];
                if (page < 0 || page >= a.kv.n_pages) atomicOr(a.err, ERR_PAGE_RANGE);
                else row = ((long)page * a.kv.nkv + kvh) * a.kv.page + (t - pi * a.kv.page);
            }
            if (FMT == KV_F32) {
                const long off = row >= 0 ? row * D + c * 4 : 0;
                cp16(dK + r * LD + c * 4, (const float *)a.kv.k + off, row >= 0);
                cp16(dV + r * LD + c * 4, (const float *)a.kv.v + off, row >= 0);
            } else {
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
                if (row >= 0) { x = cache4<FMT>(a.kv, a.kv.k, a.kv.ks, row, D, c); y = cache4<FMT>(a.kv, a.kv.v, a.kv.vs, row, D, c); }
                *(float4 *)(dK + r * LD + c * 4) = x;
                *(float4 *)(dV + r * LD + c * 4) = y;
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (C::BUFS == 2 && j_begin < j_end) load_tile(j_begin);
    for (int j = j_begin; j < j_end; ++j) {
        const int t0 = key0(j);
        if (C::BUFS == 2) {
            if (j + 1 < j_end) load_tile(j + 1); else asm volatile("cp.async.commit_group;" ::: "memory");
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else
            load_tile(j);
        __syncthreads();
        const float *sK = sKV + (C::BUFS == 2 ? (j - j_begin) & 1 : 0) * 2 * GK * LD, *sV = sK + GK * LD;
        float s[RPT][4];
#pragma unroll
        for (int i = 0; i < RPT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll 4
        for (int c = 0; c < D / 4; ++c) {
            float4 k4[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) k4[e] = *(const float4 *)(sK + (tx + 16 * e) * LD + c * 4);
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const float4 q4 = *(const float4 *)(sQ + (ty * RPT + i) * LD + c * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[i][e] = fmaf(q4.w, k4[e].w, fmaf(q4.z, k4[e].z, fmaf(q4.y, k4[e].y, fmaf(q4.x, k4[e].x, s[i][e]))));
            }
        }
        // some row does not see some key of the tile
        const bool masked = !(t0 + GK - 1 <= pos_first && (!a.window || t0 > pos_last - a.window || t0 + GK - 1 < a.sinks)) || rows < RT;
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            float mx = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = t0 + tx + 16 * e;
                s[i][e] *= a.scale_log2;
                if (masked && (t > pos[i] || (a.window && t <= pos[i] - a.window && t >= a.sinks))) s[i][e] = -INFINITY;
                mx = fmaxf(mx, s[i][e]);
            }
#pragma unroll
            for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
            const float nm = fmaxf(m[i], mx), base = nm == -INFINITY ? 0.f : nm, f = m[i] == -INFINITY ? 0.f : exp2f(m[i] - base);
            m[i] = nm;
            l[i] *= f;
#pragma unroll
            for (int k = 0; k < OC; ++k) { o[i][k][0] *= f; o[i][k][1] *= f; o[i][k][2] *= f; o[i][k][3] *= f; }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = s[i][e] == -INFINITY ? 0.f : exp2f(s[i][e] - base);
                l[i] += p;
                sP[(ty * RPT + i) * LP + tx + 16 * e] = p;
            }
        }
        __syncwarp(); // a row's weights come from its own half warp
        if (D >= 64 || tx < D / 4) {
#pragma unroll 2
            for (int t = 0; t < GK; t += 4) {
                float4 p4[RPT];
#pragma unroll
                for (int i = 0; i < RPT; ++i) p4[i] = *(const float4 *)(sP + (ty * RPT + i) * LP + t);
#pragma unroll
                for (int h = 0; h < 4; ++h) {
#pragma unroll
                    for (int k = 0; k < OC; ++k) {
                        const float4 v = *(const float4 *)(sV + (t + h) * LD + tx * 4 + 64 * k);
#pragma unroll
                        for (int i = 0; i < RPT; ++i) {
                            const float p = h == 0 ? p4[i].x : h == 1 ? p4[i].y : h == 2 ? p4[i].z : p4[i].w;
                            if (masked && p == 0.f) continue; // an unseen key's values may be anything
                            o[i][k][0] = fmaf(p, v.x, o[i][k][0]);
                            o[i][k][1] = fmaf(p, v.y, o[i][k][1]);
                            o[i][k][2] = fmaf(p, v.z, o[i][k][2]);
                            o[i][k][3] = fmaf(p, v.w, o[i][k][3]);
                        }
                    }
                }
            }
        }
        __syncthreads(); // the tile has been read
    }
    const long plane = (long)a.rb.n_tokens * a.nq;
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int r = ty * RPT + i;
#pragma unroll
        for (int w = 8; w > 0; w >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        if (r >= rows) continue;
        const int rr = r0 + r, head = kvh * a.group + rr % a.group;
        const long token = row0 + rr / a.group, w = (long)split * plane + token * a.nq + head;
        if (l[i] != l[i]) m[i] = fmaxf(m[i], 0.f); // scores that are all NaN leave no maximum
        if (a.part_o && tx == 0) { a.part_ml[w * 2] = m[i]; a.part_ml[w * 2 + 1] = l[i]; }
        if (D < 64 && tx >= D / 4) continue;
        const float inv = a.part_o ? 1.f : inverse_sum(l[i]);
#pragma unroll
        for (int k = 0; k < OC; ++k) {
            const int c = tx * 4 + 64 * k;
            const float4 x = make_float4(o[i][k][0] * inv, o[i][k][1] * inv, o[i][k][2] * inv, o[i][k][3] * inv);
            if (a.part_o) *(float4 *)(a.part_o + w * D + c) = x;
            else {
                T *dst = (T *)a.out + token * a.o_stride + (long)head * D + c;
                dst[0] = from_f<T>(x.x); dst[1] = from_f<T>(x.y); dst[2] = from_f<T>(x.z); dst[3] = from_f<T>(x.w);
            }
        }
    }
    if (threadIdx.x == 0) stamp_exit(a.stamp);
}

template <typename T, int FMT, int D, int RPT> cudaError_t launch_general(const PagedAttnArgs &a, cudaStream_t st)
{
    using C = GenCfg<FMT, D, RPT>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise((const void *)paged_attention_general_kernel<T, FMT, D, RPT>, C::SMEM);
    if (e != cudaSuccess) return e;
    const long tiles = row_tiles(a, C::RT);
    return launch_kernel(paged_attention_general_kernel<T, FMT, D, RPT>, dim3((unsigned)tiles, a.kv.nkv, a.rb.B * a.splits), dim3(G_THREADS), C::SMEM, st, 0, a);
}
template <typename T, int FMT, int D> cudaError_t general_by_rows(const PagedAttnArgs &a, cudaStream_t st)
{
    switch (a.row_tile) {
    case 16: return launch_general<T, FMT, D, 1>(a, st);
    default: return launch_general<T, FMT, D, 4>(a, st);
    }
}
template <int FMT> cudaError_t general_f32(const PagedAttnArgs &a, cudaStream_t st)
{
    switch (a.kv.d) {
    case 32: return general_by_rows<float, FMT, 32>(a, st);
    case 64: return general_by_rows<float, FMT, 64>(a, st);
    case 128: return general_by_rows<float, FMT, 128>(a, st);
    default: return cudaErrorInvalidValue;
    }
}

} // namespace

cudaError_t launch_paged_attention_general(const PagedAttnArgs &a, int q_bf16, cudaStream_t st)
{
    if (q_bf16) {
        if (a.kv.d != 32) return cudaErrorInvalidValue; // 64 and 128: the tensor-core kernels
        switch (a.kv.fmt) {
        case KV_BF16: return general_by_rows<bf16, KV_BF16, 32>(a, st);
        case KV_E4M3: return general_by_rows<bf16, KV_E4M3, 32>(a, st);
        case KV_INT8: return general_by_rows<bf16, KV_INT8, 32>(a, st);
        case KV_INT4: return general_by_rows<bf16, KV_INT4, 32>(a, st);
        default: return cudaErrorInvalidValue;
        }
    }
    switch (a.kv.fmt) {
    case KV_F32: return general_f32<KV_F32>(a, st);
    case KV_E4M3: return general_f32<KV_E4M3>(a, st);
    case KV_INT8: return general_f32<KV_INT8>(a, st);
    case KV_INT4: return a.kv.d == 32 ? general_by_rows<float, KV_INT4, 32>(a, st) : cudaErrorInvalidValue; // others: paged_attention_rows4.cu
    default: return cudaErrorInvalidValue;
    }
}

namespace {

enum AttnKernel { ATTN_GENERAL, ATTN_ROWS, ATTN_STREAM, ATTN_TC };
struct AttnPlan { AttnKernel kernel; int splits; size_t workspace; int row_tile; };

// tcgen05 over 4-bit pages: ranges by a model of the time, in units of 50 ns: a key tile takes 2.2 us in a thread block with an SM to itself, 3.6 in each of
// two; partial rows and their sum 5 us and 0.35 per thousand rows and range.  The model takes all sequences for as long as the bound.  Several are mostly not,
// and thread blocks beyond one per SM even that out by themselves: there ranges have to gain 15 %, and beyond those that run at a time there are none.  At most four
// times as many blocks as run at a time (79 MB of partial rows of 128 on 148 SMs), which keeps the launch within its limits, too.  rows: by the bounds, not the tokens at hand, so that
// a workspace for a step of many tokens serves one of fewer.  Measured, us in one range
// and by this rule, 64 heads on 8 unless said: one sequence, 128 tokens on 14000 keys (64 blocks) 236, 112; 300 on 16000 (152) 388, 285; 600 (304) 610, 515; 700 (352) 618, 552; 2000
// on 8000, 8 heads on 8 (128) 170, 148; 16 sequences, up to 8 tokens on 2000 to 8000 keys (128) 133, 90; 20, five tokens on 8000 (160) 199, 156; 24, on 2000 to 8000 (192) 154,
// 110.  Where there are none, us in one range and in two or three: one sequence, 1024 tokens on 14336 keys (512) 698, 698; 2048 (1024) 1258, 1408; 40 sequences, five tokens on 2000
// to 8000 keys (320) 162, 165; 100 to 128 tokens on 500 to 4000 keys, 40 heads on 40, 4 sequences (160) 74, 90; 8 (320) 112, 168.
int tc4_splits(long blocks, long tiles, long rows, int B)
{
    const long sms = sm_count(), two = 2 * sms; // two: blocks that run at a time
    if (B > 1 && blocks > two) return 1;
    auto pace = [=](long n) { return n / two * 72 + (n % two == 0 ? 0 : n % two <= sms ? 44 : 72); }; // time of a key tile in each of n blocks
    long best = tiles * pace(blocks) * (B == 1 ? 95 : blocks > sms ? 85 : 100) / 100;
    int splits = 1;
    for (int s = 2; s <= 64 && s <= tiles && blocks * s <= 4 * two; ++s) {
        const long cost = (tiles + s - 1) / s * pace(blocks * s) + 100 + rows * s * 7 / 1000;
        if (cost < best) { best = cost; splits = s; }
    }
    return splits;
}

// Ranges (s, a cluster) that `tiles` row tiles over 4-bit pages are cut into, or fewer where not all clusters would find their SMs at once: these lie in
// groups of unequal size.  places: clusters of 1 .. 8 thread blocks that a B200 holds with 1, 2 and 3 blocks per SM, as the runtime says.  One cluster too
// many waits for all the others: single tokens on 2300 keys, 64 heads on 8, 2 sequences as 16 clusters of 8 15 us, of 6 8.3; 6 as 48 of 3 18, of 2 11.6.
long clusters_that_fit(long s, long tiles, int resident)
{
    static const int places[3][PAGED_MAX_CLUSTER] = {{148, 74, 45, 33, 26, 22, 15, 15}, {296, 148, 93, 71, 56, 45, 37, 33}, {444, 222, 142, 104, 82, 71, 56, 48}};
    const int per_sm = tiles * s <= sm_count() ? 1 : resident;
    if (s <= PAGED_MAX_CLUSTER && tiles * s <= (long)per_sm * sm_count())
        while (s > 1 && tiles > places[per_sm - 1][s - 1]) --s;
    return s;
}

// Which kernel serves a call, and into how many ranges the keys of its row tiles are cut.
AttnPlan plan_attention(int fmt, int d, int nkv, int dtype, int nq, int B, long n_tokens, int max_new, int max_context, int window, int sinks)
{
    AttnPlan p{ATTN_GENERAL, 1, 0, 0};
    if (max_new > max_context) max_new = max_context;
    const long rows = (long)max_new * (nq / nkv);
    long keys = max_context;
    if (window && keys > (long)window + max_new + sinks) keys = (long)window + max_new + sinks;
    const long tiles16 = (rows + 15) / 16 * nkv * (B > 0 ? B : 1);
    if (fmt == KV_INT4 && dtype == 0 && d != 32) {
        // tiles of 8 rows; ranges of the keys, joined in a cluster, where the tiles do not fill the GPU, none under 256 keys
        p.kernel = ATTN_ROWS;
        const long blocks = (rows + 7) / 8 * nkv * (B > 0 ? B : 1), sms = sm_count();
        long s = sms / blocks >= 2 ? sms / blocks : 2 * sms / blocks;
        if (s > (keys + 255) / 256) s = (keys + 255) / 256;
        p.splits = (int)(s < 1 ? 1 : clusters_that_fit(s > PAGED_MAX_CLUSTER ? PAGED_MAX_CLUSTER : s, blocks, 2));
    } else if (dtype != 1 || d == 32) {
        // 64-row tiles do the most products per shared-memory load (four chunks of up to 512 rows, head_dim 64, with ranges of four
        // tiles or more: 64 rows 38.7 us, 32 rows 57; with the finer ranges below 64 rows take 30); ranges where the tiles do not give every SM four thread blocks, of at least two tiles of 64 keys
        const long pairs = (long)nkv * (B > 0 ? B : 1);
        p.row_tile = rows <= 32 ? 16 : 64;
        long s = 4L * sm_count() / ((rows + p.row_tile - 1) / p.row_tile * pairs);
        if (s > (keys + 127) / 128) s = (keys + 127) / 128;
        p.splits = (int)(s < 1 ? 1 : s > 64 ? 64 : s);
    } else if (fmt == KV_INT4 && rows <= PAGED_MAX_FEW_ROWS && keys >= 2048 && B <= STREAM_MAX_B &&
               (long)B * nkv * (keys / 32) >= (rows <= 8 ? 32L * stream4_workers(1) : 24L * stream4_workers(2)) &&
               (long)B * nkv * ((keys + max_new) / 32 + 4) < (1L << 30)) { // steps of 32 keys: numbers of 32 bits
        // Dealt out evenly where the sequences are not short and every warp has 32 (16 rows: 24) steps or more by the bounds: below that the second kernel and
        // the warps' new starts cost more than the balance gains.  Measured, single tokens, 64 heads on 8, us this way and as thread blocks per sequence: 18 steps
        // (128 sequences of 129 to 1023 keys) 36, 31; 27 (32 of 1000 to 6000) 49, 38; 36 (32 of 4000 to 8000) 61, 69; 54 (32 of 3000 to 12000) 66, 79; 67 (16 of
        // 20000 to 30000) 101, 118; on 16 heads 56 steps (200 of 100 to 1000) 87, 79.  128 heads on 8: 30 (24 of 1000 to 6000) 45, 53; 31 (100 of 300 to 1500) 59,
        // 50; 54 (16 of 4000 to 16000) 69, 99.
        p.kernel = ATTN_STREAM;
        p.workspace = stream4_workspace((int)rows, d);
        return p;
    } else if (rows <= PAGED_MAX_FEW_ROWS ||
               (fmt == KV_INT4 && rows <= 2 * PAGED_MAX_FEW_ROWS && (long)B * nkv <= sm_count() && (keys <= 4096 || 4L * B * nkv >= sm_count())) ||
               (fmt == KV_INT4 && tiles16 <= sm_count() && keys <= 4096 && tiles16 * keys <= 2048L * sm_count())) {
        // 4 bits: up to 32 rows as two tiles of 16, except for more (sequence, KV head) pairs than SMs and on long contexts of few pairs.  Measured, 64 heads on
        // 8, us this way and on tcgen05: 4 tokens, 500 to 2300 keys, 4 sequences 14, 19, 8: 21, 28, 16: 36, 39, 32: 62, 50, 64: 118, 83; 4 tokens on 8000 keys
        // 28, 22; five tokens (40 rows), 32 sequences 82, 50.  More rows where their tiles of 16 find an SM each and the contexts are short; one sequence, 64 heads
        // on 8: 8 tokens on 200 keys 7, 11, on 2300: 13, 17; 35 tokens on 1000 keys 15, 19, on 3900 (not here) 31, 28.
        p.kernel = ATTN_ROWS;
        // Ranges enough to give every SM one (wide) thread block, or, where there are many (sequence, KV head) pairs, to fill
        // the resident ones; at least one per 2048 keys, which evens out sequences of unequal length; none under 256 keys.
        // More than a cluster's worth cost a second kernel (about 2 us) and pay from 512 keys each.  Measured, 8 KV heads of
        // 8 query heads, bf16, us by ranges: 1 x 4096 keys 8: 11.2, 20: 12.8; 1 x 16384 8: 24.9, 20: 22.4; 4 x 4096 2: 24.7,
        // 4: 18.9, 8: 19.1; 16 x 4096 2: 49, 8: 61.
        const long pairs = (long)(B > 0 ? B : 1) * nkv * ((rows + 15) / 16), sms = sm_count();
        const int resident = fmt == KV_INT4 ? (rows <= 8 ? 3 : 2) : fmt != KV_BF16 && rows <= 8 ? 4 : 3;
        long s = sms / pairs >= 2 ? sms / pairs : resident * sms / pairs;
        if (s > (keys + 255) / 256) s = (keys + 255) / 256;
        if (s < (keys + 2047) / 2048) s = (keys + 2047) / 2048;
        if (s > PAGED_MAX_CLUSTER) {
            if (s > keys / 512) s = keys / 512;
            if (s > 64) s = 64;
            if (s < 12) s = PAGED_MAX_CLUSTER;
        }
        if (fmt == KV_INT4) s = clusters_that_fit(s, pairs, resident);
        p.splits = (int)(s < 1 ? 1 : s);
    } else {
        // two thread blocks per SM: ranges where the row tiles leave some idle, of at least four tiles of 128 keys
        p.kernel = ATTN_TC;
        const long blocks = (rows + 127) / 128 * nkv * (B > 0 ? B : 1);
        long s = 2L * sm_count() / blocks;
        if (s > (keys + 511) / 512) s = (keys + 511) / 512;
        p.splits = (int)(s < 1 ? 1 : s > 64 ? 64 : s);
        if (fmt == KV_INT4) p.splits = tc4_splits(blocks, (keys + 127) / 128, (long)(B > 0 ? B : 1) * max_new * nq, B);
    }
    if (p.kernel == ATTN_ROWS ? p.splits > PAGED_MAX_CLUSTER : p.splits > 1) p.workspace = (size_t)p.splits * n_tokens * nq * (d + 2) * sizeof(float);
    return p;
}

} // namespace

cudaError_t run_paged_attention(PagedAttnArgs &a, int q_bf16, int part_splits, cudaStream_t st)
{
    AttnPlan p = plan_attention(a.kv.fmt, a.kv.d, a.kv.nkv, q_bf16, a.nq, a.rb.B, a.rb.n_tokens, a.max_new, a.max_context, a.window, a.sinks);
    if (p.workspace && p.splits > part_splits) {
        const int own = p.kernel == ATTN_ROWS ? PAGED_MAX_CLUSTER : 1; // ranges that need no workspace
        p.splits = part_splits > own ? part_splits : own;
        p.workspace = p.splits > own;
    }
    a.splits = p.splits;
    a.row_tile = p.row_tile;
    if (a.kv.fmt == KV_INT4 && a.rb.B <= ORDER_MAX_B && (p.kernel == ATTN_ROWS || p.kernel == ATTN_TC)) {
        // Sequences by length where their blocks are about as many as run at a time: 64 single tokens on 129 to 1023 keys 22.5 -> 19.6 us (all of one
        // length 22.4 -> 23.2), five tokens, 32 sequences of 500 to 2300 keys 62 -> 50.  Not for several tiles of rows per sequence, whose short blocks pay
        // the 0.4 us for nothing (ragged chunks 162 -> 161, in float32 12.0 -> 12.6).
        const long rows = (long)a.max_new * a.group, blocks = (long)a.kv.nkv * a.rb.B * p.splits;
        a.longest_first = rows <= (p.kernel == ATTN_TC ? 128 : q_bf16 ? 2 * PAGED_MAX_FEW_ROWS : 8) && blocks > sm_count() && blocks <= 8 * sm_count();
    }
    if (!p.workspace) a.part_o = a.part_ml = nullptr;
    cudaError_t e = cudaSuccess;
    switch (p.kernel) {
    case ATTN_GENERAL: e = launch_paged_attention_general(a, q_bf16, st); break;
    case ATTN_ROWS: e = a.kv.fmt == KV_INT4 ? launch_paged_attention_rows4(a, q_bf16, false, st) : launch_paged_attention_rows(a, st); break;
    case ATTN_STREAM: return launch_paged_attention_rows4(a, q_bf16, true, st);
    case ATTN_TC: e = launch_paged_attention_tc(a, st); break;
    }
    if (e == cudaSuccess && p.workspace) e = launch_paged_merge(a, q_bf16, st);
    return e;
}

int check_cache(const spd_kv_cache *c, const spd_ragged *r, PagedKv *kv, RaggedBatch *rb); // kv_cache.cu
bool known_format(int f);
bool rows_ok(const void *p, int64_t stride, int heads, int d, int dtype);

} // namespace spd

using namespace spd;

extern "C" int spd_paged_attention(const spd_kv_cache *cache, const spd_ragged *batch, const void *q, int64_t q_stride, void *out,
                                   int64_t out_stride, int32_t dtype, int32_t n_q_heads, int32_t max_new, int32_t max_context, float scale,
                                   int32_t window, int32_t sinks, void *workspace, size_t workspace_bytes, int32_t *err_flag, void *stream)
{
    PagedAttnArgs a{};
    const int rc = check_cache(cache, batch, &a.kv, &a.rb);
    if (rc) return rc;
    if (!err_flag) return SPD_ENULL;
    if ((dtype != 0 && dtype != 1) || n_q_heads < 1 || n_q_heads > 65535 || n_q_heads % a.kv.nkv || a.rb.B > 65535) return SPD_EINVAL;
    if ((a.kv.fmt == KV_F32 && dtype != 0) || (a.kv.fmt == KV_BF16 && dtype != 1)) return SPD_EINVAL;
    if (max_new < 1 || max_context < 1 || max_context > PAGED_MAX_CONTEXT || window < 0 || sinks < 0 || !(scale > 0.f) || !isfinite(scale)) return SPD_EINVAL;
    if ((int64_t)a.rb.max_pages * a.kv.page < max_context) return SPD_ECAPACITY;
    if (a.rb.B == 0 || a.rb.n_tokens == 0) return SPD_OK;
    if (!q || !out) return SPD_ENULL;
    if (!rows_ok(q, q_stride, n_q_heads, a.kv.d, dtype) || !rows_ok(out, out_stride, n_q_heads, a.kv.d, dtype)) return SPD_EINVAL;
    if (q == out) return SPD_EINVAL;
    a.q = q; a.out = out; a.q_stride = q_stride; a.o_stride = out_stride;
    a.nq = n_q_heads; a.group = n_q_heads / a.kv.nkv; a.max_new = max_new < max_context ? max_new : max_context; a.max_context = max_context;
    a.window = window; a.sinks = window ? sinks : 0;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.err = err_flag;
    const AttnPlan p = plan_attention(a.kv.fmt, a.kv.d, a.kv.nkv, dtype, a.nq, a.rb.B, a.rb.n_tokens, max_new, max_context, a.window, a.sinks);
    if (p.workspace && (!workspace || workspace_bytes < p.workspace || ((uintptr_t)workspace & 255))) return SPD_EWORKSPACE;
    if (p.workspace) {
        a.part_o = (float *)workspace;
        a.part_ml = a.part_o + (size_t)p.splits * a.rb.n_tokens * a.nq * a.kv.d;
    }
    const cudaError_t e = run_paged_attention(a, dtype, p.workspace ? p.splits : 0, (cudaStream_t)stream);
    if (e != cudaSuccess) { note_cuda_error(e); return SPD_ECUDA; }
    return SPD_OK;
}

extern "C" int spd_paged_attention_workspace_bytes(const spd_kv_cache *cache, int32_t B, int32_t n_tokens, int32_t dtype, int32_t n_q_heads,
                                                   int32_t max_new, int32_t max_context, int32_t window, int32_t sinks, size_t *out_bytes)
{
    if (!cache || !out_bytes) return SPD_ENULL;
    if (B < 0 || n_tokens < 0 || (dtype != 0 && dtype != 1) || cache->n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % cache->n_kv_heads || max_new < 1 || max_context < 1 || window < 0 || sinks < 0) return SPD_EINVAL;
    if (!known_format(cache->format)) return SPD_EINVAL;
    *out_bytes = plan_attention(cache->format, cache->head_dim, cache->n_kv_heads, dtype, n_q_heads, B, n_tokens, max_new, max_context, window,
                                window ? sinks : 0).workspace;
    return SPD_OK;
}
