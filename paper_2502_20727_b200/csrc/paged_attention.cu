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

// One warp per (new token, query head); lane l owns dims [l * VEC, (l + 1) * VEC).  Online softmax in base 2 and fp32;
// keys are visited one by one, first the sinks that lie before the window, then the window.
template <typename T, int FMT, int VEC>
__global__ void __launch_bounds__(128) paged_attention_simt_kernel(PagedAttnArgs a)
{
    constexpr int D = 32 * VEC;
    typedef typename KvElem<FMT>::type E;
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y, b = blockIdx.z;
    int row0, n_new, len;
    if (!batch_row(a.rb, b, a.max_new, a.max_context, row0, n_new, len, a.err)) return;
    const int i = blockIdx.x * 4 + warp;
    if (i >= n_new) return;
    const int kvh = h / a.group, pos = len + i;
    const int lo = a.window ? max(0, pos - a.window + 1) : 0, n_sink = min(a.sinks, lo);
    float q[VEC], o[VEC];
    const T *qp = (const T *)a.q + (long)(row0 + i) * a.q_stride + (long)h * D + lane * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) { q[e] = to_f<T>(qp[e]) * a.scale_log2; o[e] = 0.f; }
    float mx = -INFINITY, den = 0.f;
    const int32_t *bt = a.rb.table + (long)b * a.rb.max_pages;
    const int n_keys = n_sink + pos + 1 - lo;
    for (int j = 0; j < n_keys; ++j) {
        const int t = j < n_sink ? j : lo + (j - n_sink), pi = t / a.kv.page;
        if (pi >= a.rb.max_pages) { atomicOr(a.err, ERR_CAPACITY); break; }
        const int page = bt[pi];
        if (page < 0 || page >= a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); continue; }
        const long row = ((long)page * a.kv.nkv + kvh) * a.kv.page + t % a.kv.page;
        const E *kp = (const E *)a.kv.k + row * D + lane * VEC, *vp = (const E *)a.kv.v + row * D + lane * VEC;
        float s = 0.f, vs = 1.f;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s = fmaf(q[e], kv_value<FMT>(kp[e]), s);
        s = warp_sum(s);
        if (FMT >= KV_E4M3) { s *= a.kv.ks[row]; vs = a.kv.vs[row]; }
        const float nm = fmaxf(mx, s), base = nm == -INFINITY ? 0.f : nm;
        const float corr = exp2f(mx - base), p = exp2f(s - base);
        den = den * corr + p;
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = fmaf(o[e], corr, p * (vs * kv_value<FMT>(vp[e])));
        mx = nm;
    }
    T *op = (T *)a.out + (long)(row0 + i) * a.o_stride + (long)h * D + lane * VEC;
    const float inv = den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
#pragma unroll
    for (int e = 0; e < VEC; ++e) op[e] = from_f<T>(o[e] * inv);
}

template <typename T, int FMT> cudaError_t simt_by_dim(const PagedAttnArgs &a, cudaStream_t st)
{
    const dim3 grid((a.max_new + 3) / 4, a.nq, a.rb.B);
    switch (a.kv.d) {
    case 32: return launch_kernel(paged_attention_simt_kernel<T, FMT, 1>, grid, dim3(128), 0, st, 0, a);
    case 64: return launch_kernel(paged_attention_simt_kernel<T, FMT, 2>, grid, dim3(128), 0, st, 0, a);
    case 128: return launch_kernel(paged_attention_simt_kernel<T, FMT, 4>, grid, dim3(128), 0, st, 0, a);
    default: return cudaErrorInvalidValue;
    }
}
template <typename T> cudaError_t simt_by_format(const PagedAttnArgs &a, cudaStream_t st)
{
    switch (a.kv.fmt) {
    case KV_F32: return simt_by_dim<T, KV_F32>(a, st);
    case KV_BF16: return simt_by_dim<T, KV_BF16>(a, st);
    case KV_E4M3: return simt_by_dim<T, KV_E4M3>(a, st);
    case KV_INT8: return simt_by_dim<T, KV_INT8>(a, st);
    default: return cudaErrorInvalidValue;
    }
}

} // namespace

cudaError_t launch_paged_attention_simt(const PagedAttnArgs &a, int q_bf16, cudaStream_t st)
{
    return q_bf16 ? simt_by_format<bf16>(a, st) : simt_by_format<float>(a, st);
}

namespace {

enum AttnKernel { ATTN_SIMT, ATTN_ROWS, ATTN_TC };
struct AttnPlan { AttnKernel kernel; int splits; size_t workspace; };

// Which kernel serves a call, and into how many ranges the keys of its row tiles are cut.
AttnPlan plan_attention(int fmt, int d, int nkv, int dtype, int nq, int B, long n_tokens, int max_new, int max_context, int window, int sinks)
{
    AttnPlan p{ATTN_SIMT, 1, 0};
    if (dtype != 1 || (d != 64 && d != 128)) return p;
    if (max_new > max_context) max_new = max_context;
    const long rows = (long)max_new * (nq / nkv);
    long keys = max_context;
    if (window && keys > (long)window + max_new + sinks) keys = (long)window + max_new + sinks;
    if (rows <= 16) {
        p.kernel = ATTN_ROWS;
        // Ranges enough to give every SM one (wide) thread block, or, where there are many (sequence, KV head) pairs, to fill
        // the resident ones; at least one per 2048 keys, which evens out sequences of unequal length; none under 256 keys.
        // More than a cluster's worth cost a second kernel (about 2 us) and pay from 512 keys each.  Measured, 8 KV heads of
        // 8 query heads, bf16, us by ranges: 1 x 4096 keys 8: 11.2, 20: 12.8; 1 x 16384 8: 24.9, 20: 22.4; 4 x 4096 2: 24.7,
        // 4: 18.9, 8: 19.1; 16 x 4096 2: 49, 8: 61.
        const long pairs = (long)(B > 0 ? B : 1) * nkv, sms = sm_count(), resident = fmt != KV_BF16 && rows <= 8 ? 4 : 3;
        long s = sms / pairs >= 2 ? sms / pairs : resident * sms / pairs;
        if (s > (keys + 255) / 256) s = (keys + 255) / 256;
        if (s < (keys + 2047) / 2048) s = (keys + 2047) / 2048;
        if (s > PAGED_MAX_CLUSTER) {
            if (s > keys / 512) s = keys / 512;
            if (s > 64) s = 64;
            if (s < 12) s = PAGED_MAX_CLUSTER;
        }
        p.splits = (int)(s < 1 ? 1 : s);
    }
    else {
        // one thread block per SM: ranges where the row tiles leave SMs idle, of at least four tiles of 128 keys
        p.kernel = ATTN_TC;
        const long blocks = (rows + (rows > 128 ? 255 : 127)) / (rows > 128 ? 256 : 128) * nkv * (B > 0 ? B : 1);
        long s = sm_count() / blocks;
        if (s > (keys + 511) / 512) s = (keys + 511) / 512;
        p.splits = (int)(s < 1 ? 1 : s > 64 ? 64 : s);
    }
    if (p.kernel == ATTN_TC ? p.splits > 1 : p.splits > PAGED_MAX_CLUSTER) p.workspace = (size_t)p.splits * n_tokens * nq * (d + 2) * sizeof(float);
    return p;
}

} // namespace

int check_cache(const spd_kv_cache *c, const spd_ragged *r, PagedKv *kv, RaggedBatch *rb); // kv_cache.cu
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
    if (max_new < 1 || max_context < 1 || window < 0 || sinks < 0 || !(scale > 0.f) || !isfinite(scale)) return SPD_EINVAL;
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
    a.splits = p.splits;
    if (p.workspace) {
        a.part_o = (float *)workspace;
        a.part_ml = a.part_o + (size_t)p.splits * a.rb.n_tokens * a.nq * a.kv.d;
    }
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    switch (p.kernel) {
    case ATTN_SIMT: e = launch_paged_attention_simt(a, dtype, st); break;
    case ATTN_ROWS: e = launch_paged_attention_rows(a, st); break;
    case ATTN_TC: e = launch_paged_attention_tc(a, st); break;
    }
    if (e == cudaSuccess && p.workspace) e = launch_paged_merge(a, dtype, st);
    if (e != cudaSuccess) { note_cuda_error(e); return SPD_ECUDA; }
    return SPD_OK;
}

extern "C" int spd_paged_attention_workspace_bytes(const spd_kv_cache *cache, int32_t B, int32_t n_tokens, int32_t dtype, int32_t n_q_heads,
                                                   int32_t max_new, int32_t max_context, int32_t window, int32_t sinks, size_t *out_bytes)
{
    if (!cache || !out_bytes) return SPD_ENULL;
    if (B < 0 || n_tokens < 0 || (dtype != 0 && dtype != 1) || cache->n_kv_heads < 1 || n_q_heads < 1 || n_q_heads % cache->n_kv_heads || max_new < 1 || max_context < 1 || window < 0 || sinks < 0) return SPD_EINVAL;
    if (cache->format < SPD_KV_F32 || cache->format > SPD_KV_INT8) return SPD_EINVAL;
    *out_bytes = plan_attention(cache->format, cache->head_dim, cache->n_kv_heads, dtype, n_q_heads, B, n_tokens, max_new, max_context, window,
                                window ? sinks : 0).workspace;
    return SPD_OK;
}
