// Appending rows to a paged K/V cache and reading them back, for plain, 8-bit and 4-bit caches.
//
// A cached row is the head_dim values of one token of one KV head.  In the 8-bit formats it has one float32 scale s:
//   e4m3 : s = the smallest power of two with max|x| <= 448 s; code = x / s rounded to e4m3.  The division is exact, so
//          the only rounding is e4m3's (relative 2^-4 at most, absolute s 2^-10 below the normal range), and code * s
//          is exact in bfloat16 too.
//   int8 : s = max|x| / 127; code = x * (127 * (1 / max|x|)) rounded to the nearest integer, half to even; quotient, reciprocal and
//          products are rounded to float32, which moves values within 2^-22 of a border between two codes at most.
// A row of zeros has s = 1; s is at least 2^-126; a row that holds a NaN or an infinity gets s = NaN and codes 0, so that
// reading it gives NaN everywhere and nothing else is touched.
//   int4 : two halves of the head dims, each with its smallest value m rounded down to bf16 and a scale s = (max - m) / 15 rounded to
//          bf16, at least 2^-60; code = (x - m) / s rounded to the nearest integer, half to even.  The quotients are the correctly
//          rounded ones (from the rounded reciprocal with one residual correction, Markstein 1990), so that ties, which are common among
//          bf16 values, fall as they do in exact arithmetic.  m <= x, and s is off by 2^-9 at most, so codes end at 15 by themselves.
//          16 prompts of about 1024 tokens, 40 heads, stored and read back: 131 us (5.4 TB/s; storing is bound by its instructions: with
//          eight elements a lane in place of 16 155 us at 78 % of the issue slots).
//
// Bound: memory.  A thread block serves a few consecutive tokens and 16 cached rows (K and V of eight heads) of each; one warp
// finds the tokens' sequences and pages for all of them, then every lane moves eight elements of UNITS rows with all loads in
// flight at once (a bf16 row of 128 is half a warp's 16-byte accesses).  The chain of dependent loads before the data -
// sequence bounds, length and page id - is paid once per block: with one per warp the same copies ran at 3.1 TB/s.
#include "../../include/spd.h"
#include "paged.cuh"

#include <type_traits>

namespace spd {

namespace {

constexpr int KV_THREADS = 256, ROWS = 16; // rows of a token a block serves

// Where the block's tokens t0 .. t0 + TT - 1 are cached: the row of (page, head 0, slot), or -1 where a token is nobody's or does
// not fit (error bit).  Warp 0; lane k < TT takes token k.  Sequence of token t: the last b with cu[b] <= t.
template <int TT> __device__ __forceinline__ void locate_tokens(const PagedKv &kv, const RaggedBatch &rb, const int32_t *slots, int t0, long (&base)[TT], int *err)
{
    const int lane = threadIdx.x & 31;
    if (slots) { // the caller knows: one load in place of the search and the table
        if (lane >= TT) return;
        const int slot = t0 + lane < rb.n_tokens ? slots[t0 + lane] : -1;
        const int page = slot < 0 ? 0 : slot / kv.page;
        if (slot >= 0 && page >= kv.n_pages) atomicOr(err, ERR_PAGE_RANGE);
        base[lane] = slot >= 0 && page < kv.n_pages ? (long)page * kv.nkv * kv.page + (slot - page * kv.page) : -1;
        return;
    }
    int before[TT];
#pragma unroll
    for (int k = 0; k < TT; ++k) before[k] = 0;
    for (int i0 = 0; i0 <= rb.B; i0 += 32) {
        const int i = i0 + lane, c = i <= rb.B ? rb.cu[i] : 0x7fffffff;
        unsigned last = 0;
#pragma unroll
        for (int k = 0; k < TT; ++k) {
            last = __ballot_sync(0xffffffffu, c <= t0 + k && i <= rb.B);
            before[k] += __popc(last);
        }
        if (last != 0xffffffffu) break;
    }
    int mine = 0;
#pragma unroll
    for (int k = 0; k < TT; ++k)
        if (lane == k) mine = before[k];
    if (lane >= TT) return;
    long where = -1;
    if (t0 + lane < rb.n_tokens && mine >= 1 && mine <= rb.B) {
        const int b = mine - 1;
        const long pos = (long)rb.lens[b] + (t0 + lane - rb.cu[b]);
        if (pos < 0 || pos / kv.page >= rb.max_pages) atomicOr(err, ERR_CAPACITY);
        else {
            const int page = rb.table[(long)b * rb.max_pages + pos / kv.page];
            if (page < 0 || page >= kv.n_pages) atomicOr(err, ERR_PAGE_RANGE);
            else where = (long)page * kv.nkv * kv.page + pos % kv.page;
        }
    }
    base[lane] = where;
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

// The values of eight bytes of a 4-bit row: eight dims of the first half and eight of the second.  code * scale + smallest is rounded once: to float32,
// or, by a product in bf16x2, to bf16.  A code is exact under the exponent of 2^23 (2^7 in bf16), less that.
__device__ __forceinline__ void values4(uint2 w, uint2 par, float *low, float *high)
{
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t p = half ? par.y : par.x;
        const float s = kv4_scale(p), m = kv4_min(p);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fmaf(__uint_as_float(0x4b000000u | ((i < 4 ? w.x : w.y) >> (8 * (i & 3) + 4 * half) & 15u)) - 8388608.f, s, m);
        store8<float>(half ? high : low, x);
    }
}
__device__ __forceinline__ void values4(uint2 w, uint2 par, bf16 *low, bf16 *high)
{
    const uint32_t c128 = widen_const();
    const uint32_t b[4] = {__byte_perm(w.x, 0, 0x4140), __byte_perm(w.x, 0, 0x4342), __byte_perm(w.y, 0, 0x4140), __byte_perm(w.y, 0, 0x4342)};
    const auto h = [](uint32_t x) { return *(const __nv_bfloat162 *)&x; };
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const uint32_t p = half ? par.y : par.x, s = __byte_perm(p, 0, 0x1010), m = __byte_perm(p, 0, 0x3232);
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 v = __hfma2(__hsub2(h(and_or(b[i] >> (4 * half), 0x000f000fu, c128)), h(c128)), h(s), h(m));
            x[i] = *(const uint32_t *)&v;
        }
        *(uint4 *)(half ? high : low) = make_uint4(x[0], x[1], x[2], x[3]);
    }
}

__device__ __forceinline__ uint32_t e4m3_x4(float a, float b, float c, float d)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
// Four codes x * inv rounded to nearest, half to even, |x * inv| < 127.5: adding 1.5 * 2^23 leaves the integer in the sum's low
// byte (two instructions a code where a float-to-integer conversion takes a slot of a quarter-rate pipe).
__device__ __forceinline__ uint32_t int8_x4(const float *x, float inv)
{
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__fadd_rn(__fmul_rn(x[i], inv), 12582912.f));
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

// eight elements as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<bf16> { uint4 u; };
template <> struct Raw8<float> { float4 a, b; };
template <> struct Raw8<uint8_t> { uint2 u; };
template <> struct Raw8<int8_t> { uint2 u; };
__device__ __forceinline__ void get(const Raw8<bf16> &r, float (&x)[8])
{
    const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void get(const Raw8<float> &r, float (&x)[8])
{
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
__device__ __forceinline__ void get(const Raw8<uint8_t> &r, float (&x)[8]) // e4m3
{
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = kv_value<KV_E4M3>((uint8_t)((e < 4 ? r.u.x : r.u.y) >> (8 * (e & 3))));
}
__device__ __forceinline__ void get(const Raw8<int8_t> &r, float (&x)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = kv_value<KV_INT8>((int8_t)((e < 4 ? r.u.x : r.u.y) >> (8 * (e & 3))));
}

// bits of the largest magnitude
__device__ __forceinline__ uint32_t top_of(const Raw8<bf16> &r)
{
    const uint32_t m = __vmaxu2(__vmaxu2(r.u.x & 0x7fff7fffu, r.u.y & 0x7fff7fffu), __vmaxu2(r.u.z & 0x7fff7fffu, r.u.w & 0x7fff7fffu));
    return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t top_of(const Raw8<float> &r)
{
    const uint32_t a = max(__float_as_uint(r.a.x) & 0x7fffffffu, __float_as_uint(r.a.y) & 0x7fffffffu);
    const uint32_t b = max(__float_as_uint(r.a.z) & 0x7fffffffu, __float_as_uint(r.a.w) & 0x7fffffffu);
    const uint32_t c = max(__float_as_uint(r.b.x) & 0x7fffffffu, __float_as_uint(r.b.y) & 0x7fffffffu);
    const uint32_t d = max(__float_as_uint(r.b.z) & 0x7fffffffu, __float_as_uint(r.b.w) & 0x7fffffffu);
    return max(max(a, b), max(c, d));
}

__device__ __forceinline__ float min_nan(float a, float b) // NaN if either is
{
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// Smallest and largest element of the 16 x LANES elements of a group of lanes, NaN if one is.
template <int LANES> __device__ __forceinline__ float2 range_of(const Raw8<bf16> (&r)[2])
{
    const uint4 u = r[0].u, v = r[1].u;
    const auto h = [](uint32_t w) { return *(const __nv_bfloat162 *)&w; };
    const auto w = [](__nv_bfloat162 v) { return *(const uint32_t *)&v; };
    const auto least = [&](uint4 a) { return __hmin2_nan(__hmin2_nan(h(a.x), h(a.y)), __hmin2_nan(h(a.z), h(a.w))); };
    const auto most = [&](uint4 a) { return __hmax2_nan(__hmax2_nan(h(a.x), h(a.y)), __hmax2_nan(h(a.z), h(a.w))); };
    const uint32_t lo = w(__hmin2_nan(least(u), least(v))), hi = w(__hmax2_nan(most(u), most(v))) ^ 0x80008000u;
    __nv_bfloat162 x = __hmin2_nan(h(__byte_perm(lo, hi, 0x5410)), h(__byte_perm(lo, hi, 0x7632))); // (smallest, minus the largest)
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) x = __hmin2_nan(x, h(__shfl_xor_sync(0xffffffffu, w(x), o)));
    return make_float2(__uint_as_float(w(x) << 16), __uint_as_float((w(x) & 0xffff0000u) ^ 0x80000000u));
}
template <int LANES> __device__ __forceinline__ float2 range_of(const Raw8<float> (&r)[2])
{
    const auto least = [](const Raw8<float> &q) {
        return min_nan(min_nan(min_nan(q.a.x, q.a.y), min_nan(q.a.z, q.a.w)), min_nan(min_nan(q.b.x, q.b.y), min_nan(q.b.z, q.b.w)));
    };
    const auto most = [](const Raw8<float> &q) {
        return max_nan(max_nan(max_nan(q.a.x, q.a.y), max_nan(q.a.z, q.a.w)), max_nan(max_nan(q.b.x, q.b.y), max_nan(q.b.z, q.b.w)));
    };
    float lo = min_nan(least(r[0]), least(r[1])), hi = max_nan(most(r[0]), most(r[1]));
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    return make_float2(lo, hi);
}
// 1 / s, rounded to nearest, for a bf16 number s from 2^-60 on: one Newton step from the approximate reciprocal (the correctly rounded
// quotient for every such s: all of them were compared with the division's)
__device__ __forceinline__ float reciprocal(float s)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s));
    return fmaf(fmaf(-s, y, 1.f), y, y);
}
// Four 4-bit codes, one per byte, of x >= m: (x - m) / s by its correctly rounded quotient, the integer as in int8_x4; two at a time
__device__ __forceinline__ uint32_t int4_x4(const float *x, float m, float s, float inv)
{
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const float2 d = add2(make_float2(x[i], x[i + 1]), make_float2(-m, -m)), q = mul2(d, make_float2(inv, inv));
        const float2 c = add2(fma2(fma2(q, make_float2(-s, -s), d), make_float2(inv, inv), q), make_float2(12582912.f, 12582912.f));
        b[i] = __float_as_uint(c.x);
        b[i + 1] = __float_as_uint(c.y);
    }
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

// Rows a lane has in flight, tokens of a block.  FEW: few rows in all, which then spread over more blocks.
// 4 bits: a lane has 16 elements of a row (read: eight bytes, eight elements of either half; written: of one half, two Raw8) of four rows, so that what is
// done once per half row is done by half as many lanes.
template <typename T, int D, bool FEW, bool INT4> struct KvShape {
    static constexpr int LPR = D / (INT4 ? 16 : 8), PER_PASS = KV_THREADS / LPR; // lanes per row, rows per pass of the block
    static constexpr int TT = (FEW ? 1 : (sizeof(T) == 4 ? 4 : 8) / (INT4 ? 2 : 1)) * PER_PASS / ROWS, UNITS = TT * ROWS / PER_PASS;
};

template <typename T, int FMT, int D, bool FEW>
__global__ void __launch_bounds__(KV_THREADS) kv_write_kernel(PagedKv kv, RaggedBatch rb, const int32_t *slots, const T *k, const T *v, long k_stride, long v_stride, int *err)
{
    using S = KvShape<T, D, FEW, FMT == KV_INT4>;
    constexpr int LPR = S::LPR, TT = S::TT, UNITS = S::UNITS, PARTS = FMT == KV_INT4 ? 2 : 1; // Raw8s of a lane and row
    typedef typename KvElem<FMT>::type E;
    __shared__ long base[TT];
    pdl_launch_dependents();
    pdl_wait();
    const int t0 = blockIdx.x * TT, r0 = blockIdx.y * ROWS, li = threadIdx.x % LPR, g = threadIdx.x / LPR;
    Raw8<T> raw[UNITS][PARTS];
#pragma unroll
    for (int i = 0; i < UNITS; ++i) { // row 2h: K of head h, 2h + 1: V
        const int id = i * S::PER_PASS + g, t = t0 + id / ROWS, r = r0 + id % ROWS;
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            raw[i][q] = Raw8<T>{};
            if (t < rb.n_tokens && (r >> 1) < kv.nkv)
                raw[i][q] = *(const Raw8<T> *)((r & 1 ? v + (long)t * v_stride : k + (long)t * k_stride) + (long)(r >> 1) * D + (li * PARTS + q) * 8);
        }
    }
    if (threadIdx.x < 32) locate_tokens<TT>(kv, rb, slots, t0, base, err);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int id = i * S::PER_PASS + g, r = r0 + id % ROWS, h = r >> 1;
        const long where = base[id / ROWS], row = where + (long)h * kv.page;
        const bool ok = where >= 0 && h < kv.nkv;
        float x[8];
        get(raw[i][0], x);
        if constexpr (FMT == KV_F32 || FMT == KV_BF16) {
            if (ok) store8<E>((E *)(r & 1 ? kv.v : kv.k) + row * D + li * 8, x);
            continue;
        }
        if constexpr (FMT == KV_INT4) {
            // lanes li and li ^ LPR / 2 have the same bytes' low and high codes
            constexpr int HALF = LPR / 2;
            const bool high = li >= HALF;
            const float2 range = range_of<HALF>(raw[i]);
            // down to bf16: towards zero, or away from it where negative
            const uint32_t bits = __float_as_uint(range.x), mb = (range.x < 0.f ? bits + 0xffffu : bits) & 0xffff0000u;
            const float m = __uint_as_float(mb), spread = __fsub_rn(range.y, m);
            // spread / 15 as amax / 127 below
            const float q0 = spread * (1.f / 15.f), step = fmaf(fmaf(-q0, 15.f, spread), 1.f / 15.f, q0);
            const float s = fmaxf(__bfloat162float(__float2bfloat16_rn(step)), 0x1p-60f), inv = reciprocal(s);
            const bool bad = !(spread < INFINITY); // a NaN or an infinity in the half, or a spread that is no float
            float y[8];
            get(raw[i][1], y);
            uint2 own = make_uint2(int4_x4(x, m, s, inv), int4_x4(x + 4, m, s, inv)), other = make_uint2(int4_x4(y, m, s, inv), int4_x4(y + 4, m, s, inv));
            // this lane keeps the first eight dims (low half) or the last eight (high half); bit 7 of the others' codes: `bad`
            if (high) { const uint2 t = own; own = other; other = t; }
            other = make_uint2(__shfl_xor_sync(0xffffffffu, bad ? 0x80u : other.x, HALF), __shfl_xor_sync(0xffffffffu, other.y, HALF));
            const bool row_bad = bad || (other.x & 0x80u);
            if (!ok) continue;
            const uint2 lo = high ? other : own, hi = high ? own : other;
            *(uint2 *)((uint8_t *)(r & 1 ? kv.v : kv.k) + row * (D / 2) + (li & (HALF - 1)) * 16 + high * 8) =
                row_bad ? make_uint2(0, 0) : make_uint2(lo.x | (hi.x << 4), lo.y | (hi.y << 4));
            if ((li & (HALF - 1)) == 0)
                ((uint32_t *)(r & 1 ? kv.vs : kv.ks))[2 * row + high] = row_bad ? 0x7fc07fc0u : (__float_as_uint(s) >> 16) | mb;
            continue;
        }
        // largest magnitude of the row; a NaN wins (comparisons on the bit patterns of |x|)
        uint32_t m = top_of(raw[i][0]);
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        const float amax = __uint_as_float(m);
        float s;
        uint2 codes;
        if (FMT == KV_E4M3) {
            // amax = f 2^ex with f in [1, 2); 448 = 1.75 * 2^8.  Denormal amax (and 0): the clamp decides.
            const int ex = max((int)(m >> 23) - 127 - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
            s = __uint_as_float((uint32_t)(ex + 127) << 23);
            const float inv = __uint_as_float((uint32_t)(127 - min(ex, 120)) << 23); // ex <= 120 where amax is finite: a normal number
            const float top = ex == 120 ? 240.f : 448.f; // 256 * 2^120 would be 2^128: the last code that still reads as a finite float is 240
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = fminf(top, fmaxf(-top, x[e] * inv));
            codes = make_uint2(e4m3_x4(x[0], x[1], x[2], x[3]), e4m3_x4(x[4], x[5], x[6], x[7]));
        } else {
            // amax / 127 by a product with the rounded reciprocal and one residual correction, which gives the rounded quotient
            // (Markstein 1990); the codes' factor is the rounded reciprocal times 127, rounded: the same bits wherever a row is quantised
            const float q0 = amax * (1.f / 127.f);
            s = fmaxf(fmaf(fmaf(-q0, 127.f, amax), 1.f / 127.f, q0), 1.17549435e-38f);
            const float inv = __fmul_rn(__frcp_rn(fmaxf(amax, 127.f * 1.17549435e-38f)), 127.f);
            codes = make_uint2(int8_x4(x, inv), int8_x4(x + 4, inv));
        }
        if (m == 0) s = 1.f;
        if (m >= 0x7f800000u) { s = __uint_as_float(0x7fc00000u); codes = make_uint2(0, 0); }
        if (!ok) continue;
        *(uint2 *)((uint8_t *)(r & 1 ? kv.v : kv.k) + row * D + li * 8) = codes;
        if (li == 0) (r & 1 ? kv.vs : kv.ks)[row] = s;
    }
}

template <typename T, int FMT, int D, bool FEW>
__global__ void __launch_bounds__(KV_THREADS) kv_read_kernel(PagedKv kv, RaggedBatch rb, T *k, T *v, long k_stride, long v_stride, int *err)
{
    typedef typename KvElem<FMT>::type E;
    using S = KvShape<E, D, FEW, FMT == KV_INT4>;
    constexpr int LPR = S::LPR, TT = S::TT, UNITS = S::UNITS;
    __shared__ long base[TT];
    pdl_launch_dependents();
    pdl_wait();
    const int t0 = blockIdx.x * TT, r0 = blockIdx.y * ROWS, li = threadIdx.x % LPR, g = threadIdx.x / LPR;
    if (threadIdx.x < 32) locate_tokens<TT>(kv, rb, nullptr, t0, base, err);
    __syncthreads();
    if constexpr (FMT == KV_INT4) {
        uint2 codes[UNITS], par[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int id = i * S::PER_PASS + g, r = r0 + id % ROWS, h = r >> 1;
            const long where = base[id / ROWS], row = where + (long)h * kv.page;
            codes[i] = par[i] = make_uint2(0, 0);
            if (where >= 0 && h < kv.nkv) {
                codes[i] = *(const uint2 *)((const uint8_t *)(r & 1 ? kv.v : kv.k) + row * (D / 2) + li * 8);
                par[i] = kv4_params(r & 1 ? kv.vs : kv.ks, row);
            }
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int id = i * S::PER_PASS + g, t = t0 + id / ROWS, r = r0 + id % ROWS, h = r >> 1;
            if (base[id / ROWS] < 0 || h >= kv.nkv) continue;
            T *dst = (r & 1 ? v + (long)t * v_stride : k + (long)t * k_stride) + (long)h * D + li * 8;
            values4(codes[i], par[i], dst, dst + D / 2);
        }
    } else {
        Raw8<E> raw[UNITS];
        float s[UNITS];
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int id = i * S::PER_PASS + g, r = r0 + id % ROWS, h = r >> 1;
            const long where = base[id / ROWS], row = where + (long)h * kv.page;
            raw[i] = Raw8<E>{};
            s[i] = 1.f;
            if (where >= 0 && h < kv.nkv) {
                raw[i] = *(const Raw8<E> *)((const E *)(r & 1 ? kv.v : kv.k) + row * D + li * 8);
                if (sizeof(E) == 1) s[i] = (r & 1 ? kv.vs : kv.ks)[row];
            }
        }
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int id = i * S::PER_PASS + g, t = t0 + id / ROWS, r = r0 + id % ROWS, h = r >> 1;
            if (base[id / ROWS] < 0 || h >= kv.nkv) continue;
            float x[8];
            get(raw[i], x);
            if (sizeof(E) == 1) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] *= s[i];
            }
            store8<T>((r & 1 ? v + (long)t * v_stride : k + (long)t * k_stride) + (long)h * D + li * 8, x);
        }
    }
}

template <bool WRITE, typename T, int FMT, int D>
cudaError_t launch(const PagedKv &kv, const RaggedBatch &rb, const int32_t *slots, const void *k, const void *v, long ks, long vs, int *err, cudaStream_t st)
{
    typedef typename std::conditional<WRITE, T, typename KvElem<FMT>::type>::type In;
    auto grid = [&](int tt) { return dim3((unsigned)((rb.n_tokens + tt - 1) / tt), (unsigned)((2 * kv.nkv + ROWS - 1) / ROWS)); };
    // under one block per SM the copy is a matter of latency (64 tokens x 16 rows appended and read back: 9.5 -> 7.2 us)
    const dim3 full = grid(KvShape<In, D, false, FMT == KV_INT4>::TT);
    if ((long)full.x * full.y < sm_count()) {
        const dim3 few = grid(KvShape<In, D, true, FMT == KV_INT4>::TT);
        if (WRITE) return launch_kernel(kv_write_kernel<T, FMT, D, true>, few, dim3(KV_THREADS), 0, st, 0, kv, rb, slots, (const T *)k, (const T *)v, ks, vs, err);
        return launch_kernel(kv_read_kernel<T, FMT, D, true>, few, dim3(KV_THREADS), 0, st, 0, kv, rb, (T *)k, (T *)v, ks, vs, err);
    }
    if (WRITE) return launch_kernel(kv_write_kernel<T, FMT, D, false>, full, dim3(KV_THREADS), 0, st, 0, kv, rb, slots, (const T *)k, (const T *)v, ks, vs, err);
    return launch_kernel(kv_read_kernel<T, FMT, D, false>, full, dim3(KV_THREADS), 0, st, 0, kv, rb, (T *)k, (T *)v, ks, vs, err);
}

template <bool WRITE, typename T, int FMT>
cudaError_t by_dim(const PagedKv &kv, const RaggedBatch &rb, const int32_t *slots, const void *k, const void *v, long ks, long vs, int *err, cudaStream_t st)
{
    switch (kv.d) {
    case 32: return launch<WRITE, T, FMT, 32>(kv, rb, slots, k, v, ks, vs, err, st);
    case 64: return launch<WRITE, T, FMT, 64>(kv, rb, slots, k, v, ks, vs, err, st);
    case 128: return launch<WRITE, T, FMT, 128>(kv, rb, slots, k, v, ks, vs, err, st);
    default: return cudaErrorInvalidValue;
    }
}

template <bool WRITE, typename T>
cudaError_t by_format(const PagedKv &kv, const RaggedBatch &rb, const int32_t *slots, const void *k, const void *v, long ks, long vs, int *err, cudaStream_t st)
{
    switch (kv.fmt) {
    case KV_F32: return by_dim<WRITE, T, KV_F32>(kv, rb, slots, k, v, ks, vs, err, st);
    case KV_BF16: return by_dim<WRITE, T, KV_BF16>(kv, rb, slots, k, v, ks, vs, err, st);
    case KV_E4M3: return by_dim<WRITE, T, KV_E4M3>(kv, rb, slots, k, v, ks, vs, err, st);
    case KV_INT8: return by_dim<WRITE, T, KV_INT8>(kv, rb, slots, k, v, ks, vs, err, st);
    case KV_INT4: return by_dim<WRITE, T, KV_INT4>(kv, rb, slots, k, v, ks, vs, err, st);
    default: return cudaErrorInvalidValue;
    }
}

} // namespace

cudaError_t launch_kv_write(const PagedKv &kv, const RaggedBatch &rb, const int32_t *slots, const void *k, const void *v, long ks, long vs, int in_bf16,
                            int *err, cudaStream_t st)
{
    return in_bf16 ? by_format<true, bf16>(kv, rb, slots, k, v, ks, vs, err, st) : by_format<true, float>(kv, rb, slots, k, v, ks, vs, err, st);
}
cudaError_t launch_kv_read(const PagedKv &kv, const RaggedBatch &rb, void *k, void *v, long ks, long vs, int out_bf16, int *err,
                           cudaStream_t st)
{
    return out_bf16 ? by_format<false, bf16>(kv, rb, nullptr, k, v, ks, vs, err, st) : by_format<false, float>(kv, rb, nullptr, k, v, ks, vs, err, st);
}

} // namespace spd

using namespace spd;

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

} // namespace

namespace spd {

bool known_format(int f) { return (f >= SPD_KV_F32 && f <= SPD_KV_INT8) || f == SPD_KV_INT4; }

// Checks shared by the cache operators; fills the internal descriptions.
int check_cache(const spd_kv_cache *c, const spd_ragged *r, PagedKv *kv, RaggedBatch *rb)
{
    if (!c || !r) return SPD_ENULL;
    if (!known_format(c->format)) return SPD_EINVAL;
    if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) return SPD_EINVAL;
    if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 65535 || c->kv_block_size < 1) return SPD_EINVAL;
    if (r->B < 0 || r->n_tokens < 0 || r->max_pages < 1) return SPD_EINVAL;
    if (!c->k_pages || !c->v_pages || (c->format >= SPD_KV_E4M3 && (!c->k_scales || !c->v_scales))) return SPD_ENULL;
    if (r->B && (!r->cu_new || !r->seq_lens || !r->block_table)) return SPD_ENULL; // arrays of no elements may be null
    if (!aligned16(c->k_pages) || !aligned16(c->v_pages) || (((uintptr_t)c->k_scales | (uintptr_t)c->v_scales) & (c->format == SPD_KV_INT4 ? 7 : 3)))
        return SPD_EINVAL;
    *kv = PagedKv{c->k_pages, c->v_pages, c->k_scales, c->v_scales, c->n_pages, c->n_kv_heads, c->kv_block_size, c->head_dim, c->format};
    *rb = RaggedBatch{r->cu_new, r->seq_lens, r->block_table, r->B, r->max_pages, r->n_tokens, 0, 0};
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
    const cudaError_t e = launch_kv_write(kv, rb, nullptr, k, v, k_stride, v_stride, dtype, err_flag, (cudaStream_t)stream);
    if (e != cudaSuccess) { note_cuda_error(e); return SPD_ECUDA; }
    return SPD_OK;
}

extern "C" int spd_kv_write_slots(const spd_kv_cache *cache, const int32_t *slots, int32_t n_tokens, const void *k, const void *v, int64_t k_stride,
                                  int64_t v_stride, int32_t dtype, int32_t *err_flag, void *stream)
{
    PagedKv kv;
    RaggedBatch rb;
    const spd_ragged rows{nullptr, nullptr, nullptr, 0, 1, n_tokens};
    const int rc = check_cache(cache, &rows, &kv, &rb);
    if (rc) return rc;
    if (!err_flag) return SPD_ENULL;
    if (dtype != 0 && dtype != 1) return SPD_EINVAL;
    if (n_tokens == 0) return SPD_OK;
    if (!slots || !k || !v) return SPD_ENULL;
    if (!rows_ok(k, k_stride, kv.nkv, kv.d, dtype) || !rows_ok(v, v_stride, kv.nkv, kv.d, dtype)) return SPD_EINVAL;
    const cudaError_t e = launch_kv_write(kv, rb, slots, k, v, k_stride, v_stride, dtype, err_flag, (cudaStream_t)stream);
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
