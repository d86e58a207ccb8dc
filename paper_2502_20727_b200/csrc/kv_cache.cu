// Appending rows to a paged K/V cache and reading them back, for plain and 8-bit caches.
//
// A cached row is the head_dim values of one token of one KV head.  In the 8-bit formats it has one float32 scale s:
//   e4m3 : s = the smallest power of two with max|x| <= 448 s; code = x / s rounded to e4m3.  The division is exact, so
//          the only rounding is e4m3's (relative 2^-4 at most, absolute s 2^-10 below the normal range), and code * s
//          is exact in bfloat16 too.
//   int8 : s = max|x| / 127; code = x * (127 / max|x|) rounded to the nearest integer, half to even.
// A row of zeros has s = 1; s is at least 2^-126; a row that holds a NaN or an infinity gets s = NaN and codes 0, so that
// reading it gives NaN everywhere and nothing else is touched.
//
// Bound: memory.  Eight elements per lane, so that a bf16 row of 128 is half a warp's 16-byte loads; a warp serves rows
// of one token (the K and V rows of consecutive heads), finds the token's sequence once, and has ROWS_PER_LANE loads in
// flight before it needs the first.
#include "../../include/spd.h"
#include "paged.cuh"

namespace spd {

namespace {

constexpr int KV_THREADS = 256, ROWS_PER_LANE = 4;

// Sequence of token row t: the last b with cu[b] <= t (warp-wide, coalesced).  -1: t lies outside every sequence.
__device__ __forceinline__ int find_sequence(const RaggedBatch &rb, int t)
{
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int i0 = 0; i0 <= rb.B; i0 += 32) {
        const int i = i0 + lane;
        const unsigned m = __ballot_sync(0xffffffffu, i <= rb.B && rb.cu[i] <= t);
        before += __popc(m);
        if (m != 0xffffffffu) break;
    }
    return before >= 1 && before <= rb.B ? before - 1 : -1;
}

// Element offset of row 0 of (page of position pos, head 0) plus the row inside the page; negative: not to be touched.
__device__ __forceinline__ bool locate_row(const PagedKv &kv, const RaggedBatch &rb, int b, long pos, long &page, int &slot, int *err)
{
    if (pos < 0 || pos / kv.page >= rb.max_pages) { atomicOr(err, ERR_CAPACITY); return false; }
    page = rb.table[(long)b * rb.max_pages + pos / kv.page];
    slot = (int)(pos % kv.page);
    if (page < 0 || page >= kv.n_pages) { atomicOr(err, ERR_PAGE_RANGE); return false; }
    return true;
}

template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&x)[8])
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<bf16>(const bf16 *p, float (&x)[8])
{
    const uint4 u = *(const uint4 *)p;
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<float>(float *p, const float (&x)[8])
{
    *(float4 *)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4 *)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store8<bf16>(bf16 *p, const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *(const uint32_t *)&h;
    }
    *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ uint32_t e4m3_x4(float a, float b, float c, float d)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ uint32_t int8_x4(const float *x, float inv)
{
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int c = __float2int_rn(x[i] * inv);
        c = min(127, max(-127, c));
        w |= (uint32_t)(c & 255) << (8 * i);
    }
    return w;
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(PagedKv kv, RaggedBatch rb, const T *k, const T *v, long k_stride, long v_stride,
                                                              int warps_per_token, int *err)
{
    constexpr int LPR = D / 8, RPW = 32 / LPR; // lanes per row, rows a warp instruction covers
    typedef typename KvElem<FMT>::type E;
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, sub = lane / LPR, li = lane % LPR;
    const long w = (long)blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5);
    const long t = w / warps_per_token;
    if (t >= rb.n_tokens) return;
    const int r0 = (int)(w % warps_per_token) * RPW * ROWS_PER_LANE; // row 2h: K of head h, 2h + 1: V
    float x[ROWS_PER_LANE][8];
#pragma unroll
    for (int i = 0; i < ROWS_PER_LANE; ++i) {
        const int r = r0 + i * RPW + sub, h = r >> 1;
        if (h < kv.nkv) load8<T>((r & 1 ? v + t * v_stride : k + t * k_stride) + (long)h * D + li * 8, x[i]);
    }
    const int b = find_sequence(rb, (int)t);
    if (b < 0) return; // rows behind the last sequence
    long page;
    int slot;
    if (!locate_row(kv, rb, b, (long)rb.lens[b] + (t - rb.cu[b]), page, slot, err)) return;
#pragma unroll
    for (int i = 0; i < ROWS_PER_LANE; ++i) {
        const int r = r0 + i * RPW + sub, h = r >> 1;
        const long row = (page * kv.nkv + h) * kv.page + slot;
        if constexpr (FMT == KV_F32 || FMT == KV_BF16) {
            if (h < kv.nkv) store8<E>((E *)(r & 1 ? kv.v : kv.k) + row * D + li * 8, x[i]);
            continue;
        }
        // largest magnitude of the row; a NaN wins (comparisons on the bit patterns of |x|)
        uint32_t m = 0;
        if (h < kv.nkv) {
#pragma unroll
            for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[i][e]) & 0x7fffffffu);
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float amax = __uint_as_float(m);
        if (h >= kv.nkv) continue;
        float s = 1.f;
        uint2 codes = make_uint2(0, 0);
        if (m >= 0x7f800000u) s = __uint_as_float(0x7fc00000u);
        else if (m) {
            if (FMT == KV_E4M3) {
                // amax = f 2^ex with f in [1, 2); 448 = 1.75 * 2^8.  Denormal amax: the clamp decides.
                int ex = (int)(m >> 23) - 127 - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
                ex = max(ex, -126);
                s = __uint_as_float((uint32_t)(ex + 127) << 23);
                const float inv = __uint_as_float((uint32_t)(127 - ex) << 23); // ex <= 120: a normal number
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = x[i][e] * inv;
                if (ex == 120) { // 256 s would be 2^128: the last code that still reads as a finite float is 240
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = fminf(240.f, fmaxf(-240.f, y[e]));
                }
                codes = make_uint2(e4m3_x4(y[0], y[1], y[2], y[3]), e4m3_x4(y[4], y[5], y[6], y[7]));
            } else {
                s = fmaxf(__fdiv_rn(amax, 127.f), 1.17549435e-38f);
                const float inv = __fdiv_rn(127.f, fmaxf(amax, 127.f * 1.17549435e-38f));
                codes = make_uint2(int8_x4(x[i], inv), int8_x4(x[i] + 4, inv));
            }
        }
        *(uint2 *)((uint8_t *)(r & 1 ? kv.v : kv.k) + row * D + li * 8) = codes;
        if (li == 0) (r & 1 ? kv.vs : kv.ks)[row] = s;
    }
}

template <typename T, int FMT, int D>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(PagedKv kv, RaggedBatch rb, T *k, T *v, long k_stride, long v_stride,
                                                             int warps_per_token, int *err)
{
    constexpr int LPR = D / 8, RPW = 32 / LPR;
    typedef typename KvElem<FMT>::type E;
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31, sub = lane / LPR, li = lane % LPR;
    const long w = (long)blockIdx.x * (KV_THREADS / 32) + (threadIdx.x >> 5);
    const long t = w / warps_per_token;
    if (t >= rb.n_tokens) return;
    const int r0 = (int)(w % warps_per_token) * RPW * ROWS_PER_LANE;
    const int b = find_sequence(rb, (int)t);
    if (b < 0) return;
    long page;
    int slot;
    if (!locate_row(kv, rb, b, (long)rb.lens[b] + (t - rb.cu[b]), page, slot, err)) return;
    float x[ROWS_PER_LANE][8];
#pragma unroll
    for (int i = 0; i < ROWS_PER_LANE; ++i) {
        const int r = r0 + i * RPW + sub, h = r >> 1;
        if (h >= kv.nkv) continue;
        const long row = (page * kv.nkv + h) * kv.page + slot;
        const E *src = (const E *)(r & 1 ? kv.v : kv.k) + row * D + li * 8;
        if constexpr (FMT == KV_F32 || FMT == KV_BF16) load8<E>(src, x[i]);
        else {
            const uint2 c = *(const uint2 *)src;
            const float s = (r & 1 ? kv.vs : kv.ks)[row];
            const uint32_t cw[2] = {c.x, c.y};
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = kv_value<FMT>((E)(cw[e >> 2] >> (8 * (e & 3)))) * s;
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS_PER_LANE; ++i) {
        const int r = r0 + i * RPW + sub, h = r >> 1;
        if (h < kv.nkv) store8<T>((r & 1 ? v + t * v_stride : k + t * k_stride) + (long)h * D + li * 8, x[i]);
    }
}

template <bool WRITE, typename T, int FMT, int D>
cudaError_t launch(const PagedKv &kv, const RaggedBatch &rb, const void *k, const void *v, long ks, long vs, int *err, cudaStream_t st)
{
    const int rows_per_warp = 32 / (D / 8) * ROWS_PER_LANE;
    const int wpt = (2 * kv.nkv + rows_per_warp - 1) / rows_per_warp;
    const long blocks = ((long)rb.n_tokens * wpt + KV_THREADS / 32 - 1) / (KV_THREADS / 32);
    if (blocks <= 0) return cudaSuccess;
    if (blocks > 0x7fffffffL) return cudaErrorInvalidValue;
    if (WRITE)
        return launch_kernel(kv_write_kernel<T, FMT, D>, dim3((unsigned)blocks), dim3(KV_THREADS), 0, st, 0, kv, rb, (const T *)k, (const T *)v, ks, vs, wpt, err);
    return launch_kernel(kv_read_kernel<T, FMT, D>, dim3((unsigned)blocks), dim3(KV_THREADS), 0, st, 0, kv, rb, (T *)k, (T *)v, ks, vs, wpt, err);
}

template <bool WRITE, typename T, int FMT>
cudaError_t by_dim(const PagedKv &kv, const RaggedBatch &rb, const void *k, const void *v, long ks, long vs, int *err, cudaStream_t st)
{
    switch (kv.d) {
    case 32: return launch<WRITE, T, FMT, 32>(kv, rb, k, v, ks, vs, err, st);
    case 64: return launch<WRITE, T, FMT, 64>(kv, rb, k, v, ks, vs, err, st);
    case 128: return launch<WRITE, T, FMT, 128>(kv, rb, k, v, ks, vs, err, st);
    default: return cudaErrorInvalidValue;
    }
}

template <bool WRITE, typename T>
cudaError_t by_format(const PagedKv &kv, const RaggedBatch &rb, const void *k, const void *v, long ks, long vs, int *err, cudaStream_t st)
{
    switch (kv.fmt) {
    case KV_F32: return by_dim<WRITE, T, KV_F32>(kv, rb, k, v, ks, vs, err, st);
    case KV_BF16: return by_dim<WRITE, T, KV_BF16>(kv, rb, k, v, ks, vs, err, st);
    case KV_E4M3: return by_dim<WRITE, T, KV_E4M3>(kv, rb, k, v, ks, vs, err, st);
    case KV_INT8: return by_dim<WRITE, T, KV_INT8>(kv, rb, k, v, ks, vs, err, st);
    default: return cudaErrorInvalidValue;
    }
}

} // namespace

cudaError_t launch_kv_write(const PagedKv &kv, const RaggedBatch &rb, const void *k, const void *v, long ks, long vs, int in_bf16, int *err,
                            cudaStream_t st)
{
    return in_bf16 ? by_format<true, bf16>(kv, rb, k, v, ks, vs, err, st) : by_format<true, float>(kv, rb, k, v, ks, vs, err, st);
}
cudaError_t launch_kv_read(const PagedKv &kv, const RaggedBatch &rb, void *k, void *v, long ks, long vs, int out_bf16, int *err,
                           cudaStream_t st)
{
    return out_bf16 ? by_format<false, bf16>(kv, rb, k, v, ks, vs, err, st) : by_format<false, float>(kv, rb, k, v, ks, vs, err, st);
}

} // namespace spd

using namespace spd;

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

} // namespace

namespace spd {

// Checks shared by the cache operators; fills the internal descriptions.
int check_cache(const spd_kv_cache *c, const spd_ragged *r, PagedKv *kv, RaggedBatch *rb)
{
    if (!c || !r) return SPD_ENULL;
    if (c->format < SPD_KV_F32 || c->format > SPD_KV_INT8) return SPD_EINVAL;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return SPD_EINVAL;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->kv_block_size < 1) return SPD_EINVAL;
    if (r->B < 0 || r->n_tokens < 0 || r->max_pages < 1) return SPD_EINVAL;
    if (!c->k_pages || !c->v_pages || (c->format >= SPD_KV_E4M3 && (!c->k_scales || !c->v_scales))) return SPD_ENULL;
    if (!r->cu_new || !r->seq_lens || !r->block_table) return SPD_ENULL;
    if (!aligned16(c->k_pages) || !aligned16(c->v_pages) || ((uintptr_t)c->k_scales & 3) || ((uintptr_t)c->v_scales & 3)) return SPD_EINVAL;
    *kv = PagedKv{c->k_pages, c->v_pages, c->k_scales, c->v_scales, c->n_pages, c->n_kv_heads, c->kv_block_size, c->head_dim, c->format};
    *rb = RaggedBatch{r->cu_new, r->seq_lens, r->block_table, r->B, r->max_pages, r->n_tokens};
    return SPD_OK;
}

// rows of `heads` heads, `stride` elements apart, 16-byte aligned
bool rows_ok(const void *p, int64_t stride, int heads, int d, int dtype)
{
    const int es = dtype ? 2 : 4;
    return aligned16(p) && stride >= (int64_t)heads * d && (stride * es) % 16 == 0;
}

} // namespace spd

extern "C" int spd_kv_write(const spd_kv_cache *cache, const spd_ragged *batch, const void *k, const void *v, int64_t k_stride,
                            int64_t v_stride, int32_t dtype, int32_t *err_flag, void *stream)
{
    PagedKv kv;
    RaggedBatch rb;
    const int rc = check_cache(cache, batch, &kv, &rb);
    if (rc) return rc;
    if (!err_flag) return SPD_ENULL;
    if (dtype != 0 && dtype != 1) return SPD_EINVAL;
    if (rb.B == 0 || rb.n_tokens == 0) return SPD_OK;
    if (!k || !v) return SPD_ENULL;
    if (!rows_ok(k, k_stride, kv.nkv, kv.d, dtype) || !rows_ok(v, v_stride, kv.nkv, kv.d, dtype)) return SPD_EINVAL;
    const cudaError_t e = launch_kv_write(kv, rb, k, v, k_stride, v_stride, dtype, err_flag, (cudaStream_t)stream);
    if (e != cudaSuccess) { note_cuda_error(e); return SPD_ECUDA; }
    return SPD_OK;
}

extern "C" int spd_kv_read(const spd_kv_cache *cache, const spd_ragged *batch, void *k, void *v, int64_t k_stride, int64_t v_stride,
                           int32_t dtype, int32_t *err_flag, void *stream)
{
    PagedKv kv;
    RaggedBatch rb;
    const int rc = check_cache(cache, batch, &kv, &rb);
    if (rc) return rc;
    if (!err_flag) return SPD_ENULL;
    if (dtype != 0 && dtype != 1) return SPD_EINVAL;
    if (rb.B == 0 || rb.n_tokens == 0) return SPD_OK;
    if (!k || !v) return SPD_ENULL;
    if (!rows_ok(k, k_stride, kv.nkv, kv.d, dtype) || !rows_ok(v, v_stride, kv.nkv, kv.d, dtype)) return SPD_EINVAL;
    const cudaError_t e = launch_kv_read(kv, rb, k, v, k_stride, v_stride, dtype, err_flag, (cudaStream_t)stream);
    if (e != cudaSuccess) { note_cuda_error(e); return SPD_ECUDA; }
    return SPD_OK;
}
