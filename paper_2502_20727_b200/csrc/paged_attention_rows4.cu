// Paged attention for few query rows over 4-bit pages (bf16 queries: up to 32 rows, more in small calls; float32: any number, in tiles of 8): the arrangement of
// paged_attention_rows.cu - keys and head dims as rows of m16n8k16 MMAs, 8 or 16 query rows as their columns, a private ring of key
// tiles per warp, key ranges joined through a cluster - with what 4 bits change:
//   - the cache stream is a quarter of bf16's, so that instructions bound the kernel, the unpacking of codes before all.  Codes are float16
//     operands without arithmetic: one in the lowest bits of a float16 is the subnormal number code * 2^-24, one in bits 4-7 is 16 times
//     that, and the tensor cores' products with subnormals are exact.  A word of eight codes costs four masks and a shift;
//   - q . k = sum over the halves of s (q . codes) + m sum(q), and sum p v = sum (p s) codes + sum p m: scales and smallest values meet the
//     products in float32.  Q is float16, scaled per row by a power of two (see paged_attention_rows.cu);
//   - p s has to be float16 beside the codes, and s may be anything.  The score of a key therefore carries the exponent e of its V row's largest
//     parameter: x = 2^(score + e - max) <= 2^8, weights x (s 2^-e), the key's share in the softmax x 2^-e.  What float16 leaves out of a
//     weight is then small beside the largest contribution to the output, not beside the largest softmax weight;
//   - a warp takes 32 keys a step (two MMA tiles): one wait, one maximum and one check of it for both, and each lane turns one key's
//     parameters into the factors that all lanes read;
//   - tiles come by cp.async: a page's 16 keys are 64 chunks of 16 bytes, two instructions for the warp; as TMA boxes they were two boxes and
//     two bulk copies from one lane, at several times the instructions;
//   - float32 queries: Q and the weights in two float16s each (22 bits), codes less 8 so that sums do not cancel, the maximum followed at once; the tensor cores add up
//     16 products at a time, float32 additions the rest: their own longer sums are cut off at every step (errors of 3.6e-7 to 1.5e-6 relative to
//     float64 in place of 1.5e-7 to 3.6e-7, and 3 to 10 % less time).
// 32 sequences of 9 to 16 thousand tokens, 64 heads on 8 (475 MB), us by step: 16 keys a step by TMA, a thread block per range 188; 32 keys a step by
// cp.async 145; keys dealt out evenly to the resident warps (below) 132; two float32 operations per instruction, factors without bank
// conflicts, V by transposing matrix loads 124; 168 registers and three stages in place of 128 and two 107; warp numbers that the
// compiler knows to be the same in all lanes 105 (4.5 TB/s, 69 % of a copy's; about 500 instructions a step, of which 176 unpack).
// Not kept: shifts as products' high words on the FMA pipe (slower issue), the next step's first products under this one's softmax (113).
#include "paged_rows.cuh"

#include <type_traits>

namespace spd {

namespace {

using namespace few;

constexpr int STEP = 32; // keys a warp takes at a time

template <int D> struct Step4 {
    static constexpr int RB = D / 2, TILE = STEP * RB;                      // bytes of a row; of K or V of a step
    static constexpr int STAGE = 2 * TILE + 2 * STEP * 8;                   // tiles and parameters
    static constexpr int FACTORS = STEP * 80;                               // a step's factors, each twice: a pair of columns is one operand
};
// Thread blocks of RW warps for one (sequence, KV head) and key range
template <int D, int RW> struct Rows4Cfg : Step4<D> {
    static constexpr int STAGES = RW == 8 || D == 64 ? 4 : 3;
    static constexpr int RING = RW * STAGES * Step4<D>::STAGE, MERGE = RW * 16 * (D + 4) * 4;
    static constexpr int OFF_FACTORS = RING > MERGE ? RING : MERGE, OFF_JOIN = OFF_FACTORS + RW * Step4<D>::FACTORS;
    static constexpr int SMEM = OFF_JOIN + join_bytes(RW) + 128;            // + alignment slack
};

__device__ __forceinline__ void cp8(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 8 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
struct Pairs { float2 a, b; };
__device__ __forceinline__ Pairs lds_pairs(uint32_t p)
{
    const uint4 u = lds128(p);
    return Pairs{make_float2(__uint_as_float(u.x), __uint_as_float(u.y)), make_float2(__uint_as_float(u.z), __uint_as_float(u.w))};
}
__device__ __forceinline__ void sts_f4(uint32_t p, float x, float y) // x, x, y, y
{
    asm volatile("st.shared.v4.f32 [%0], {%1,%1,%2,%2};" ::"r"(p), "f"(x), "f"(y) : "memory");
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *(const uint32_t *)&v;
}
// codes of bytes 0 and 2 of a word (shifted right by 8: bytes 1 and 3) as float16x2, in units of 2^-24 and 2^-20
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0x00f000f0u; }
// float32 queries: code - 8 and 16 (code - 8), so that sums of weighted codes do not cancel against weighted smallest values
__device__ __forceinline__ uint32_t centred(uint32_t w, uint32_t mask, uint32_t c1024, uint32_t minus)
{
    const uint32_t x = and_or(w, mask, c1024);
    const __half2 v = __hsub2(*(const __half2 *)&x, *(const __half2 *)&minus);
    return *(const uint32_t *)&v;
}
// What a float16 leaves of a float32 operand is a second float16: 22 bits, in products of their own
__device__ __forceinline__ void split_half(float x, float y, uint32_t &high, uint32_t &low)
{
    const __half2 h = __floats2half2_rn(x, y);
    high = *(const uint32_t *)&h;
    low = pack_half(x - __low2float(h), y - __high2float(h));
}
template <typename T> struct Code4 { // the operands' units; what the weights are scaled by, and how far the maximum may be exceeded (powers of two)
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr float LOW = F32 ? 1.f : 0x1p24f, HIGH = F32 ? 0x1p-4f : 0x1p20f, WEIGHT = F32 ? 0x1p12f : 1.f, SLACK = F32 ? 0.f : 8.f;
};

// What a warp has of NR groups of 8 query rows: sums over its keys of weights times codes (tiles 0 .. MT / 2 - 1: first half of the head, in units of
// 2^-24; the others 2^-20), of weights times smallest values, of weights; the maxima they are relative to.
template <int D, int NR> struct Partial {
    float o[NR][D / 16][4];
    float2 m_used[NR], l[NR], om[NR][2]; // of this lane's columns 2 t4 and 2 t4 + 1
};

// The query rows of a (sequence, KV head) and the keys they see
struct Rows {
    int b, kvh, row0, r0, rows, len, kv_len; // packed rows r0 .. r0 + rows - 1: row r = new token r / group, query head r % group; len: the first one's position
    int lo_min, first, n_sink, n_steps; // steps of 32 keys that hold a key some row sees: sinks, then the window of the first query onwards
    // the `most` rows from `from` on, of n_new tokens behind the cached ones in `len`
    __device__ __forceinline__ void keys(const PagedAttnArgs &a, int n_new, int from = 0, int most = 0x7fffffff)
    {
        r0 = from;
        rows = min(n_new * a.group - from, most);
        kv_len = len + (from + rows - 1) / a.group + 1;
        len += from / a.group;
        lo_min = a.window ? max(0, len - a.window + 1) : 0;
        first = lo_min / STEP;
        n_sink = min((min(a.sinks, lo_min) + STEP - 1) / STEP, first);
        n_steps = n_sink + (kv_len + STEP - 1) / STEP - first;
    }
};

// One warp: steps j0, j0 + stride, ..., n_mine of them.  ring: its ST stages, fk: its factors' place.
// PAGES: page sizes 16, 32, 64, ... with less than 2^31 bytes of codes per page; else any.
template <typename T, int D, int NR, int ST, bool PAGES>
__device__ __forceinline__ void walk(const PagedAttnArgs &a, const Rows &q, int j0, int n_mine, int stride, uint32_t ring, uint32_t fk, Partial<D, NR> &acc_out)
{
    using C = Step4<D>;
    using U = Code4<T>;
    constexpr bool F32 = U::F32;
    constexpr int MT = D / 16, RB = C::RB, W = D / 32; // W: words of a lane per row
    const int lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    constexpr uint32_t F = STEP * 16; // factors: K scales, K smallest values, V scales, V smallest values, (exponent, unit)
    const int rows = q.rows, row0 = q.row0, len = q.len, kv_len = q.kv_len, kvh = q.kvh, pos_max = kv_len - 1, lo_min = q.lo_min;
    const int32_t *bt = a.rb.table + (long)q.b * a.rb.max_pages;
    const int gap = q.first - q.n_sink;
    auto key0 = [&](int i) { const int j = j0 + i * stride; return (j + (j < q.n_sink ? 0 : gap)) * STEP; };
    // steps that may hold keys which no row sees
    auto edge = [&](int i) { const int j = j0 + i * stride; return j == q.n_steps - 1 || (unsigned)(j - q.n_sink + 1) < 2u; };
    // every row sees every key of the 32 from t0 on
    auto seen_by_all = [&](int t0) { return t0 + STEP - 1 <= len && (!a.window || t0 > pos_max - a.window || t0 + STEP - 1 < a.sinks); };
    // 16-byte chunk c of row r of a tile
    auto at = [&](int r, int c) -> uint32_t { return RB == 64 ? r * 64 + ((c ^ ((r >> 1) & 3)) << 4) : r * 32 + ((c ^ ((r >> 2) & 1)) << 4); };
    constexpr int CPR = RB / 16, RPI = 32 / CPR; // chunks per row, rows per copy instruction
    const uint32_t lane_dst = at(lane / CPR, lane % CPR);
    // PAGES: ids of the pages of keys 0 and 16 of a step, asked for a step ahead (nothing looks at them before the copies); else the id of this
    // lane's key's page.
    struct Ids { int p[2]; };
    const int lg = __ffs(a.kv.page) - 1;
    auto needed = [&](int t, int n) { return t < kv_len && (t + n - 1 >= lo_min || t < a.sinks); }; // one of the keys t .. t + n - 1 is seen
    auto ask = [&](int i) {
        Ids w{{0, 0}};
        const int t0 = key0(i);
        if (PAGES) {
            const bool some = edge(i);
            if (!some || needed(t0, 16)) w.p[0] = bt[t0 >> lg];
            if (!some || needed(t0 + 16, 16)) w.p[1] = bt[(t0 + 16) >> lg];
        } else if (needed(t0 + lane, 1))
            w.p[0] = bt[(t0 + lane) / a.kv.page];
        return w;
    };
    // this lane's first chunk and parameters in page 0
    const int in_row = PAGES ? lane / CPR % 16 : 0;
    const uint8_t *k0 = (const uint8_t *)a.kv.k + ((long)kvh * a.kv.page + in_row) * RB + lane % CPR * 16;
    const uint8_t *v0 = (const uint8_t *)a.kv.v + ((long)kvh * a.kv.page + in_row) * RB + lane % CPR * 16;
    const uint2 *kp0 = (const uint2 *)a.kv.ks + (long)kvh * a.kv.page + (PAGES ? lane & 15 : 0), *vp0 = (const uint2 *)a.kv.vs + (long)kvh * a.kv.page + (PAGES ? lane & 15 : 0);
    const typename std::conditional<PAGES, uint32_t, unsigned long long>::type page_rows = (unsigned long long)a.kv.nkv * a.kv.page;
    auto load = [&](int stage, int i, const Ids &w) {
        const uint32_t dst = ring + stage * C::STAGE + lane_dst, dst_p = ring + stage * C::STAGE + 2 * C::TILE + lane * 8;
        const int t0 = key0(i);
        if (PAGES) {
            const uint32_t in0 = (uint32_t)t0 & (a.kv.page - 1), in1 = (uint32_t)(t0 + 16) & (a.kv.page - 1); // rows in the pages
            auto copy = [&](int h, bool valid) {
                const unsigned long long by = (unsigned long long)(uint32_t)w.p[h] * (page_rows * RB) + (h ? in1 : in0) * RB;
                const uint8_t *k = valid ? k0 + by : k0, *v = valid ? v0 + by : v0;
#pragma unroll
                for (int c = 0; c < 16 / RPI; ++c) {
                    cp16(dst + h * 16 * RB + c * RPI * RB, k + c * RPI * RB, valid);
                    cp16(dst + C::TILE + h * 16 * RB + c * RPI * RB, v + c * RPI * RB, valid);
                }
            };
            auto copy_params = [&](bool valid) {
                const unsigned long long by = (unsigned long long)(uint32_t)(lane < 16 ? w.p[0] : w.p[1]) * page_rows + (lane < 16 ? in0 : in1);
                cp8(dst_p, valid ? kp0 + by : kp0, valid);
                cp8(dst_p + STEP * 8, valid ? vp0 + by : vp0, valid);
            };
            if (max((uint32_t)w.p[0], (uint32_t)w.p[1]) < (uint32_t)a.kv.n_pages && !edge(i)) {
                copy(0, true);
                copy(1, true);
                copy_params(true);
            } else {
                bool valid[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    valid[h] = needed(t0 + 16 * h, 16);
                    if (valid[h] && (uint32_t)w.p[h] >= (uint32_t)a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); valid[h] = false; }
                    copy(h, valid[h]);
                }
                copy_params(lane < 16 ? valid[0] : valid[1]);
            }
        } else {
            const int t = t0 + lane;
            bool valid = needed(t, 1);
            if (valid && (uint32_t)w.p[0] >= (uint32_t)a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); valid = false; }
            const long row = valid ? (long)(w.p[0] * page_rows) + t % a.kv.page : -1; // from (page 0, this KV head, row 0)
#pragma unroll
            for (int k = 0; k < STEP / RPI; ++k) {
                const long r = __shfl_sync(0xffffffffu, row, k * RPI + lane / CPR);
                cp16(dst + k * RPI * RB, k0 + (r >= 0 ? r * RB : 0), r >= 0);
                cp16(dst + C::TILE + k * RPI * RB, v0 + (r >= 0 ? r * RB : 0), r >= 0);
            }
            cp8(dst_p, kp0 + (valid ? row : 0), valid);
            cp8(dst_p + STEP * 8, vp0 + (valid ? row : 0), valid);
        }
    };

#pragma unroll
    for (int s = 0; s < ST; ++s) {
        if (s < n_mine) load(s, s, ask(s));
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    Ids next{{0, 0}};
    if (ST < n_mine) next = ask(ST);

    // Q fragments (column g of a group of 8 rows), in the order of the codes; rows beyond the last are zero.  A lane's dims: D / 8 of either half.
    uint32_t qf[NR][2 * W][2], ql[F32 ? NR : 1][2 * W][2]; // ql: what float16 leaves of float32
    float2 qs[NR], qsum[NR][2]; // of this lane's columns 2 t4 and 2 t4 + 1: to base-2 units; sums of the halves in those
    int pos[NR][2];
    const int first_in_group = q.r0 % a.group; // the rows' tokens are counted from the first row's
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int r = g + 8 * n;
        const bool live = r < rows;
        const int i = live ? (q.r0 + r) / a.group : 0, head = live ? q.r0 + r - i * a.group : 0;
        const T *qp = (const T *)a.q + (long)(row0 + i) * a.q_stride + (long)(kvh * a.group + head) * D;
        float x[W][8];
        uint32_t top = 0; // largest magnitude's bits (float32's)
#pragma unroll
        for (int m = 0; m < W; ++m) {
            const T *src = qp + (D / 2) * (m / (W / 2)) + (D / 8) * t4 + 8 * (m % (W / 2));
            if constexpr (F32) {
                const float4 u = live ? *(const float4 *)src : make_float4(0.f, 0.f, 0.f, 0.f), v = live ? *(const float4 *)(src + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
                x[m][0] = u.x; x[m][1] = u.y; x[m][2] = u.z; x[m][3] = u.w; x[m][4] = v.x; x[m][5] = v.y; x[m][6] = v.z; x[m][7] = v.w;
            } else {
                const uint4 u = live ? *(const uint4 *)src : make_uint4(0, 0, 0, 0);
                const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) { x[m][2 * e] = __uint_as_float(w[e] << 16); x[m][2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[m][e]) & 0x7fffffffu);
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int ex = max((int)(top >> 23), 27) - 127;                   // 2^ex <= largest < 2^(ex + 1), ex >= -100
        const float f = __uint_as_float((uint32_t)(127 + 14 - ex) << 23); // to [2^14, 2^15)
        const float my_qs = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + ex) << 23);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int m = 0; m < W; ++m) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a0 = x[m][2 * e] * f, a1 = x[m][2 * e + 1] * f;
                if (F32) {
                    split_half(a0, a1, hi[e], lo[e]);
                    sum[m / (W / 2)] += a0 + a1;
                } else {
                    hi[e] = pack_half(a0, a1);
                    const __half2 v = *(const __half2 *)&hi[e];
                    sum[m / (W / 2)] += __low2float(v) + __high2float(v);
                }
            }
            qf[n][2 * m][0] = __byte_perm(hi[0], hi[1], 0x5410); qf[n][2 * m][1] = __byte_perm(hi[0], hi[1], 0x7632);
            qf[n][2 * m + 1][0] = __byte_perm(hi[2], hi[3], 0x5410); qf[n][2 * m + 1][1] = __byte_perm(hi[2], hi[3], 0x7632);
            if constexpr (F32) {
                ql[n][2 * m][0] = __byte_perm(lo[0], lo[1], 0x5410); ql[n][2 * m][1] = __byte_perm(lo[0], lo[1], 0x7632);
                ql[n][2 * m + 1][0] = __byte_perm(lo[2], lo[3], 0x5410); ql[n][2 * m + 1][1] = __byte_perm(lo[2], lo[3], 0x7632);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = 8 * n + 2 * t4 + e;
            pos[n][e] = c < rows ? len + (first_in_group + c) / a.group : -1;
        }
        qs[n] = make_float2(__shfl_sync(0xffffffffu, my_qs, 2 * t4 * 4), __shfl_sync(0xffffffffu, my_qs, (2 * t4 + 1) * 4));
#pragma unroll
        for (int h = 0; h < 2; ++h)
            qsum[n][h] = mul2(make_float2(__shfl_sync(0xffffffffu, sum[h], 2 * t4 * 4), __shfl_sync(0xffffffffu, sum[h], (2 * t4 + 1) * 4)), qs[n]);
    }

    // where this lane reads in a tile: K rows g (and 8, 16, 24 further on), the factors of these keys; V by transposing matrix loads of 8 keys x 16
    // bytes, which give a lane bytes 2 g and 2 g + 1 of keys 2 t4 and 2 t4 + 1.
    const uint32_t lane_k = RB == 64 ? at(g, t4) : at(g, t4 >> 1) + (t4 & 1) * 8, my_factors = fk + g * 16;
    const uint32_t lane_v = at(lane & 15, lane >> 4); // matrices: keys 0-7 and 8-15 of chunk 0, of chunk 1
    uint32_t c1024 = 0, c1032 = 0, c1152 = 0; // float16x2, in registers
    if (F32) asm volatile("mov.b32 %0, 0x64006400;\n\tmov.b32 %1, 0x64086408;\n\tmov.b32 %2, 0x64806480;" : "=r"(c1024), "=r"(c1032), "=r"(c1152));
    auto low = [&](uint32_t w) { return F32 ? centred(w, 0x000f000fu, c1024, c1032) : low_codes(w); };
    auto high = [&](uint32_t w) { return F32 ? centred(w, 0x00f000f0u, c1024, c1152) : high_codes(w); };
    auto &o = acc_out.o;
    auto &m_used = acc_out.m_used;
    auto &l = acc_out.l;
    auto &om = acc_out.om;
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int i = 0; i < MT; ++i) { o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f; }
        m_used[n] = make_float2(-INFINITY, -INFINITY);
        l[n] = om[n][0] = om[n][1] = make_float2(0.f, 0.f);
    }

    float2 limit[NR], minus[NR]; // maxima beyond which the sums follow; what is added to a score
#pragma unroll
    for (int n = 0; n < NR; ++n) { limit[n] = make_float2(-INFINITY, -INFINITY); minus[n] = make_float2(3e38f, 3e38f); }
    int stage = 0;
    for (int it = 0; it < n_mine; ++it) {
        asm volatile("cp.async.wait_group %0;" ::"n"(ST - 1) : "memory");
        __syncwarp();
        const uint32_t sK = ring + stage * C::STAGE, sV = sK + C::TILE, sP = sV + C::TILE;
        const int t0 = key0(it);
        { // the factors of key `lane`
            const uint2 kp = lds64(sP + lane * 8), vp = lds64(sP + STEP * 8 + lane * 8);
            const uint32_t km = __vmaxu2(kp.x & 0x7fff7fffu, kp.y & 0x7fff7fffu), vm = __vmaxu2(vp.x & 0x7fff7fffu, vp.y & 0x7fff7fffu);
            // a row that is not finite is a NaN for those who see its key, and nothing for the others
            const bool k_bad = ((km + 0x00800080u) & 0x80008000u) != 0;
            const float ks = k_bad ? __uint_as_float(0x7fc00000u) : kv4_scale(kp.x) * U::LOW;
            sts_f4(fk + lane * 16, ks, kv4_scale(kp.y) * U::HIGH);
            auto middle = [](uint32_t p) { return F32 ? fmaf(8.f, kv4_scale(p), kv4_min(p)) : kv4_min(p); }; // what a code of 0, float32: of 8, stands for
            sts_f4(fk + F + lane * 16, middle(kp.x), middle(kp.y));
            const uint32_t top = max(vm & 0xffffu, vm >> 16);
            const bool v_bad = top >= 0x7f80u;
            const int ex = min(max((int)(top >> 7), 127 - 60), 127 + 100);
            const float unit = __uint_as_float((uint32_t)(254 - ex) << 23), f = v_bad ? 0.f : unit;
            const float ev = v_bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(0x4b000000u | ex) - (8388608.f + 127.f); // 2^23 + ex
            const uint2 q = v_bad ? make_uint2(0, 0) : vp;
            sts_f4(fk + 2 * F + lane * 16, kv4_scale(q.x) * (f * U::WEIGHT), kv4_scale(q.y) * (f * U::WEIGHT));
            // the power of two first: 8 s of a finite row that nobody sees may be no float, and its weight of 0 would make a NaN of that
            auto scaled_middle = [f](uint32_t p) { return F32 ? fmaf(8.f, kv4_scale(p) * f, kv4_min(p) * f) : kv4_min(p) * f; };
            sts_f4(fk + 3 * F + lane * 16, scaled_middle(q.x), scaled_middle(q.y));
            sts_f4(fk + 4 * F + lane * 16, ev, unit);
        }
        float2 s[2][NR][2], unit[2][2]; // scores in base-2 units; [tile][rows g and g + 8]
        float acc[2][2][NR][4];        // q . codes [tile][half]
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint32_t p = sK + lane_k + u * 16 * RB;
            uint32_t w0[W], w1[W]; // rows g and g + 8
            if (W == 4) {
                const uint4 x = lds128(p), y = lds128(p + 8 * RB);
                w0[0] = x.x; w0[1] = x.y; w0[2 % W] = x.z; w0[3 % W] = x.w;
                w1[0] = y.x; w1[1] = y.y; w1[2 % W] = y.z; w1[3 % W] = y.w;
            } else {
                const uint2 x = lds64(p), y = lds64(p + 8 * RB);
                w0[0] = x.x; w0[1] = x.y; w1[0] = y.x; w1[1] = y.y;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint32_t y0 = w0[i] >> 8, y1 = w1[i] >> 8;
                const uint32_t l0 = low(w0[i]), l1 = low(w1[i]), l2 = low(y0), l3 = low(y1), h0 = high(w0[i]), h1 = high(w1[i]), h2 = high(y0), h3 = high(y1);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    if constexpr (F32) {
                        // sums of 16 products at a time, added in float32: a longer chain in the tensor cores is cut off, not rounded, at every step
                        float c0[4], c1[4], d0[4], d1[4];
                        mma16816_zero(c0, l0, l1, l2, l3, qf[n][i][0], qf[n][i][1]);
                        mma16816_zero(c1, h0, h1, h2, h3, qf[n][W + i][0], qf[n][W + i][1]);
                        mma16816_zero(d0, l0, l1, l2, l3, ql[n][i][0], ql[n][i][1]);
                        mma16816_zero(d1, h0, h1, h2, h3, ql[n][W + i][0], ql[n][W + i][1]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            acc[u][0][n][e] = (i ? acc[u][0][n][e] : 0.f) + (c0[e] + d0[e]);
                            acc[u][1][n][e] = (i ? acc[u][1][n][e] : 0.f) + (c1[e] + d1[e]);
                        }
                    } else if (i == 0) {
                        mma16816_zero(acc[u][0][n], l0, l1, l2, l3, qf[n][i][0], qf[n][i][1]);
                        mma16816_zero(acc[u][1][n], h0, h1, h2, h3, qf[n][W + i][0], qf[n][W + i][1]);
                    } else {
                        mma16816<true>(acc[u][0][n], l0, l1, l2, l3, qf[n][i][0], qf[n][i][1]);
                        mma16816<true>(acc[u][1][n], h0, h1, h2, h3, qf[n][W + i][0], qf[n][W + i][1]);
                    }
                }
            }
        }
        __syncwarp(); // the factors
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t p = my_factors + (16 * u + 8 * h) * 16;
                const Pairs k = lds_pairs(p), km = lds_pairs(p + F), eu = lds_pairs(p + 4 * F);
                unit[u][h] = eu.b;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const float2 c0 = make_float2(acc[u][0][n][2 * h], acc[u][0][n][2 * h + 1]), c1 = make_float2(acc[u][1][n][2 * h], acc[u][1][n][2 * h + 1]);
                    s[u][n][h] = fma2(fma2(k.b, c1, mul2(k.a, c0)), qs[n], fma2(km.b, qsum[n][1], fma2(km.a, qsum[n][0], eu.a)));
                }
            }
        }
        if (!seen_by_all(t0)) { // masked scores are -inf whatever was computed
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int t = t0 + 16 * u + 8 * h + g;
                        if (!sees(t, pos[n][0], a.window, a.sinks)) s[u][n][h].x = -INFINITY;
                        if (!sees(t, pos[n][1], a.window, a.sinks)) s[u][n][h].y = -INFINITY;
                    }
        }
        float2 mx[NR];
        bool grow = false;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            auto over_rows = [](float m) {
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                return fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
            };
            mx[n].x = over_rows(fmaxf(fmaxf(s[0][n][0].x, s[0][n][1].x), fmaxf(s[1][n][0].x, s[1][n][1].x)));
            mx[n].y = over_rows(fmaxf(fmaxf(s[0][n][0].y, s[0][n][1].y), fmaxf(s[1][n][0].y, s[1][n][1].y)));
            grow |= mx[n].x > limit[n].x || mx[n].y > limit[n].y; // first keys of a row included (-inf)
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const float2 nm = make_float2(fmaxf(m_used[n].x, mx[n].x), fmaxf(m_used[n].y, mx[n].y));
                const float2 f = make_float2(m_used[n].x == -INFINITY ? 0.f : ex2(m_used[n].x - nm.x), m_used[n].y == -INFINITY ? 0.f : ex2(m_used[n].y - nm.y));
                m_used[n] = nm;
                limit[n] = make_float2(nm.x + U::SLACK, nm.y + U::SLACK);
                minus[n] = make_float2(fminf(-nm.x, 3e38f), fminf(-nm.y, 3e38f)); // no key seen so far: the weights are 2^-inf whatever this is
                l[n] = mul2(l[n], f);
                om[n][0] = mul2(om[n][0], f);
                om[n][1] = mul2(om[n][1], f);
#pragma unroll
                for (int i = 0; i < MT; ++i) { o[n][i][0] *= f.x; o[n][i][1] *= f.y; o[n][i][2] *= f.x; o[n][i][3] *= f.y; }
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t pf[2][NR][2], pl[2][F32 ? NR : 1][2]; // weights [half], and what float16 leaves of them
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t p = my_factors + (16 * u + 8 * h) * 16;
                const Pairs vs = lds_pairs(p + 2 * F), vm = lds_pairs(p + 3 * F);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const float2 y = add2(s[u][n][h], minus[n]), x = make_float2(ex2(y.x), ex2(y.y));
                    l[n] = fma2(x, unit[u][h], l[n]);
                    om[n][0] = fma2(x, vm.a, om[n][0]);
                    om[n][1] = fma2(x, vm.b, om[n][1]);
                    const float2 w0 = mul2(x, vs.a), w1 = mul2(x, vs.b);
                    if constexpr (F32) {
                        uint32_t hi, lo;
                        split_half(w0.x, w0.y, hi, lo);
                        pf[0][n][h] = transpose8x8(hi);
                        pl[0][n][h] = transpose8x8(lo);
                        split_half(w1.x, w1.y, hi, lo);
                        pf[1][n][h] = transpose8x8(hi);
                        pl[1][n][h] = transpose8x8(lo);
                    } else {
                        pf[0][n][h] = transpose8x8(pack_half(w0.x, w0.y));
                        pf[1][n][h] = transpose8x8(pack_half(w1.x, w1.y));
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < RB / 16; c += 2) { // 16-byte chunks: dims 16 c + 2 g and 16 c + 2 g + 1 of either half are MMA rows g and g + 8
                uint32_t v[4];
                ldsm4t(v, (sV + lane_v + u * 16 * RB) ^ (c << 4));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t x0 = v[2 * i], x1 = v[2 * i + 1], y0 = x0 >> 8, y1 = x1 >> 8;
                    const uint32_t l0 = low(x0), l1 = low(y0), l2 = low(x1), l3 = low(y1), h0 = high(x0), h1 = high(y0), h2 = high(x1), h3 = high(y1);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        if constexpr (F32) {
                            float c0[4], c1[4];
                            mma16816_zero(c0, l0, l1, l2, l3, pl[0][n][0], pl[0][n][1]);
                            mma16816_zero(c1, h0, h1, h2, h3, pl[1][n][0], pl[1][n][1]);
                            mma16816<true>(c0, l0, l1, l2, l3, pf[0][n][0], pf[0][n][1]);
                            mma16816<true>(c1, h0, h1, h2, h3, pf[1][n][0], pf[1][n][1]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) { o[n][c + i][e] += c0[e]; o[n][W + c + i][e] += c1[e]; }
                        } else {
                            mma16816<true>(o[n][c + i], l0, l1, l2, l3, pf[0][n][0], pf[0][n][1]);
                            mma16816<true>(o[n][W + c + i], h0, h1, h2, h3, pf[1][n][0], pf[1][n][1]);
                        }
                    }
                }
            }
        }
        __syncwarp(); // every lane has read the stage and the factors
        if (it + ST < n_mine) {
            load(stage, it + ST, next);
            if (it + ST + 1 < n_mine) next = ask(it + ST + 1);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage == ST) stage = 0;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // over the warp's lanes
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) {
            auto other = [&](float2 v) { return add2(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, x), __shfl_xor_sync(0xffffffffu, v.y, x))); };
            l[n] = other(l[n]);
            om[n][0] = other(om[n][0]);
            om[n][1] = other(om[n][1]);
        }
    }
}

__device__ __forceinline__ float column(float2 v, int e) { return e ? v.y : v.x; }

template <typename T, int D, int NR, int RW, bool PAGES>
__global__ void __launch_bounds__(32 * RW, RW == 8 ? 1 : NR == 1 && sizeof(T) == 2 ? 3 : 2) paged_attention_rows4_kernel(const __grid_constant__ PagedAttnArgs a)
{
    using C = Rows4Cfg<D, RW>;
    constexpr int MT = D / 16, W = D / 32;
    extern __shared__ uint8_t rows4_raw[];
    uint8_t *gen = rows4_raw + ((128u - (tc::smem_u32(rows4_raw) & 127u)) & 127u);
    const uint32_t base = tc::smem_u32(gen);
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3; // the same in all lanes, for the compiler too
    if (threadIdx.x == 0) stamp_entry(a.stamp);
    pdl_launch_dependents();
    pdl_wait();
    const int split = blockIdx.z;
    Rows q;
    int n_new;
    const int tile = blockIdx.x / a.kv.nkv; // of 8 NR rows
    q.kvh = blockIdx.x - tile * a.kv.nkv;
    q.b = blockIdx.y;
    const bool fits = a.longest_first ? batch_row_by_length(a.rb, q.b, a.max_new, a.max_context, q.b, q.row0, n_new, q.len, a.err, (uint32_t *)(gen + C::OFF_JOIN))
                                      : batch_row(a.rb, q.b, a.max_new, a.max_context, q.row0, n_new, q.len, a.err); // OFF_JOIN: written again after the walk
    if (!fits || n_new * a.group <= tile * 8 * NR) return; // the same for a whole cluster
    q.keys(a, n_new, tile * 8 * NR, 8 * NR);
    // short sequences are cut into fewer ranges, of at least 4 steps
    const int splits = min(a.splits, (q.n_steps + 3) / 4);
    const int per = splits > 1 ? q.n_steps / splits : q.n_steps, extra = q.n_steps - per * splits; // the first `extra` ranges get one more
    const int j_begin = split < splits ? split * per + min(split, extra) : 0;
    const int j_end = split < splits ? j_begin + per + (split < extra ? 1 : 0) : 0;
    Partial<D, NR> p;
    walk<T, D, NR, C::STAGES, PAGES>(a, q, j_begin + warp, (j_end - j_begin - warp + RW - 1) / RW, RW, base + warp * C::STAGES * C::STAGE,
                                  base + C::OFF_FACTORS + warp * C::FACTORS, p);
    __syncthreads(); // the partial rows go over the rings
    float *mo = (float *)gen, *ml = mo + RW * 16 * (D + 2); // [warp][16][D + 2], [warp][16][2]
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * t4 + e;
            if (r < q.rows) {
                float *dst = mo + (warp * 16 + r) * (D + 2) + 2 * g;
#pragma unroll
                for (int i = 0; i < MT; ++i) { // MMA row g: dim 16 i + 2 g of the tile's half, row g + 8: + 1
                    const int h = i / W;
                    const float x = (h ? Code4<T>::HIGH : Code4<T>::LOW) / Code4<T>::WEIGHT, y = column(p.om[n][h], e);
                    *(float2 *)(dst + h * (D / 2) + 16 * (i % W)) = make_float2(fmaf(p.o[n][i][e], x, y), fmaf(p.o[n][i][2 + e], x, y));
                }
                if (g == 0) { ml[(warp * 16 + r) * 2] = column(p.m_used[n], e); ml[(warp * 16 + r) * 2 + 1] = column(p.l[n], e); }
            }
        }
    }
    join_rows<T, D, RW>(a, gen, C::OFF_JOIN, q.rows, q.row0, q.r0, q.kvh, split, splits, [](int, int, float &, float &) {});
    if (threadIdx.x == 0) stamp_exit(a.stamp);
}

// ---- Many sequences: the steps of all (sequence, KV head) pairs, one after the other, are dealt out evenly to the warps that the GPU holds at a time.
// A pair whose steps lie with one warp is finished by it; what a warp has of another pair goes to one of its two places in the workspace
// (it can have the end of one and the start of another), and a second kernel adds those up.
constexpr int STREAM_WARPS = 4;
template <int D> struct StreamCfg : Step4<D> {
    static constexpr int STAGES = D == 64 ? 4 : 3;
    static constexpr int OFF_FACTORS = STREAM_WARPS * STAGES * Step4<D>::STAGE, OFF_STARTS = OFF_FACTORS + STREAM_WARPS * Step4<D>::FACTORS;
    static constexpr int SMEM = OFF_STARTS + (STREAM_MAX_B + 1) * 4 + 128; // + alignment slack
};

// First step of every sequence's pairs in the order of all, [B + 1], in shared memory; by the whole block.
__device__ __forceinline__ void stream_starts(const PagedAttnArgs &a, int *starts, int *part)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = blockDim.x;
    int total = 0;
    for (int b0 = 0; b0 < a.rb.B; b0 += n) {
        const int b = b0 + tid;
        int x = 0;
        if (b < a.rb.B) {
            Rows q;
            int n_new;
            if (batch_row(a.rb, b, a.max_new, a.max_context, q.row0, n_new, q.len, a.err)) {
                q.keys(a, n_new);
                x = q.n_steps * a.kv.nkv;
            }
        }
        int y = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, y, o);
            if (lane >= o) y += z;
        }
        if (lane == 31) part[warp] = y;
        __syncthreads();
        int before = total, all = 0;
        for (int w = 0; w < n / 32; ++w) {
            if (w < warp) before += part[w];
            all += part[w];
        }
        if (b < a.rb.B) starts[b] = before + y - x;
        total += all;
        __syncthreads();
    }
    if (tid == 0) starts[a.rb.B] = total;
    __syncthreads();
}
// The last sequence that starts at or before step x and has steps
__device__ __forceinline__ int stream_find(const int *starts, int B, int x)
{
    int lo = 0, hi = B; // starts[lo] <= x < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
// How `total` steps are dealt out: no more workers than steps, the first `extra` of them one more than the others.
struct Deal {
    int workers, per, extra;
    __device__ __forceinline__ Deal(int total, int warps)
    {
        workers = min(warps, total);
        per = total / max(workers, 1);
        extra = total - per * workers;
    }
    __device__ __forceinline__ int begin(int w) const { return w * per + min(w, extra); }
    __device__ __forceinline__ int worker_of(int x) const { return x < extra * (per + 1) ? x / (per + 1) : extra + (x - extra * (per + 1)) / per; }
};

template <int D, int NR, bool PAGES>
__global__ void __launch_bounds__(32 * STREAM_WARPS, NR == 1 ? 3 : 2) paged_attention_stream4_kernel(const __grid_constant__ PagedAttnArgs a, int *starts_out)
{
    using C = StreamCfg<D>;
    constexpr int W = D / 32;
    extern __shared__ uint8_t rows4_raw[];
    uint8_t *gen = rows4_raw + ((128u - (tc::smem_u32(rows4_raw) & 127u)) & 127u);
    const uint32_t base = tc::smem_u32(gen);
    __shared__ int part[STREAM_WARPS];
    int *starts = (int *)(gen + C::OFF_STARTS);
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3; // the same in all lanes, for the compiler too
    if (threadIdx.x == 0) stamp_entry(a.stamp);
    pdl_launch_dependents();
    pdl_wait();
    stream_starts(a, starts, part);
    for (int b = threadIdx.x; blockIdx.x == 0 && b <= a.rb.B; b += 32 * STREAM_WARPS) starts_out[b] = starts[b]; // for the second kernel
    const Deal deal(starts[a.rb.B], gridDim.x * STREAM_WARPS);
    const int me = blockIdx.x * STREAM_WARPS + warp;
    if (me >= deal.workers) return;
    int x = deal.begin(me);
    const int x_end = deal.begin(me + 1);
    while (x < x_end) {
        Rows q;
        int n_new;
        q.b = stream_find(starts, a.rb.B, x);
        batch_row(a.rb, q.b, a.max_new, a.max_context, q.row0, n_new, q.len, a.err);
        q.keys(a, n_new);
        const int in_seq = x - starts[q.b];
        q.kvh = in_seq / q.n_steps;
        const int j0 = in_seq - q.kvh * q.n_steps, n = min(q.n_steps - j0, x_end - x);
        Partial<D, NR> p;
        walk<bf16, D, NR, C::STAGES, PAGES>(a, q, j0, n, 1, base + warp * C::STAGES * C::STAGE, base + C::OFF_FACTORS + warp * C::FACTORS, p);
        x += n;
        const bool whole = n == q.n_steps;
        const long slot = 2L * me + (j0 == 0);
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = 8 * nr + 2 * t4 + e;
                if (r >= q.rows) continue;
                float inv = 1.f;
                if (whole) inv = inverse_sum(column(p.l[nr], e));
                const int i = r / a.group, head = q.kvh * a.group + r - i * a.group;
#pragma unroll
                for (int t = 0; t < 2 * W; ++t) { // dims 16 (t % W) + 2 g and the next of half t / W
                    const float unit = t < W ? Code4<bf16>::LOW : Code4<bf16>::HIGH, low = column(p.om[nr][t / W], e);
                    const float y0 = fmaf(p.o[nr][t][e], unit, low) * inv, y1 = fmaf(p.o[nr][t][2 + e], unit, low) * inv;
                    const int dim = t / W * (D / 2) + 16 * (t % W) + 2 * g;
                    if (whole) *(uint32_t *)((bf16 *)a.out + (long)(q.row0 + i) * a.o_stride + (long)head * D + dim) = pack(y0, y1);
                    else *(float2 *)(a.part_o + (slot * (8 * NR) + r) * D + dim) = make_float2(y0, y1);
                }
                if (!whole && g == 0) {
                    const float m = column(p.l[nr], e) != column(p.l[nr], e) ? fmaxf(column(p.m_used[nr], e), 0.f) : column(p.m_used[nr], e); // scores that are all NaN leave no maximum
                    *(float2 *)(a.part_ml + (slot * (8 * NR) + r) * 2) = make_float2(m, column(p.l[nr], e));
                }
            }
        }
    }
    if (threadIdx.x == 0) stamp_exit(a.stamp);
}

// Adds up what several warps have of a pair: a warp per query row.
template <int D, int NR>
__global__ void __launch_bounds__(128) paged_merge_stream4_kernel(const __grid_constant__ PagedAttnArgs a, int warps, const int *starts)
{
    constexpr int VEC = D / 32;
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, r = blockIdx.z * 4 + (threadIdx.x >> 5);
    pdl_wait();
    Rows q;
    int n_new;
    q.kvh = blockIdx.x;
    q.b = blockIdx.y;
    const int start = __ldcg(starts + q.b), total = __ldcg(starts + a.rb.B);
    if (!batch_row(a.rb, q.b, a.max_new, a.max_context, q.row0, n_new, q.len, a.err)) return;
    q.keys(a, n_new);
    if (r >= q.rows) return;
    const Deal deal(total, warps);
    const int x0 = start + q.kvh * q.n_steps, w0 = deal.worker_of(x0), w1 = deal.worker_of(x0 + q.n_steps - 1);
    if (w0 == w1) return; // finished by its warp
    float m = -INFINITY, den = 0.f, o[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[e] = 0.f;
    for (int wb = w0; wb <= w1; wb += 32) { // maxima and sums in the lanes, then eight workers' rows at a time
        const int w = wb + lane, n = min(32, w1 - wb + 1);
        const int slot = 2 * w + (deal.begin(w) <= x0);
        const float2 ml = lane < n ? __ldcg((const float2 *)(a.part_ml + ((long)slot * (8 * NR) + r) * 2)) : make_float2(-INFINITY, 0.f);
        float v[8][VEC];
        auto fetch = [&](int k0) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float *src = a.part_o + ((long)__shfl_sync(0xffffffffu, slot, (k0 + k) & 31) * (8 * NR) + r) * D + lane * VEC;
#pragma unroll
                for (int e = 0; e < VEC; e += 2) {
                    const float2 x = k0 + k < n ? __ldcg((const float2 *)(src + e)) : make_float2(0.f, 0.f);
                    v[k][e] = x.x; v[k][e + 1] = x.y;
                }
            }
        };
        fetch(0);
        const float nm = fmaxf(m, warp_max(ml.x)), f = m == -INFINITY ? 0.f : ex2(m - nm), mine = ml.x == -INFINITY ? 0.f : ex2(ml.x - nm);
        m = nm;
        den = fmaf(den, f, warp_sum(ml.y * mine));
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] *= f;
        for (int k0 = 0; k0 < n; k0 += 8) {
            if (k0) fetch(k0);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float wt = __shfl_sync(0xffffffffu, mine, (k0 + k) & 31);
#pragma unroll
                for (int e = 0; e < VEC; ++e) o[e] = fmaf(v[k][e], wt, o[e]);
            }
        }
    }
    const float inv = inverse_sum(den);
    const int i = r / a.group, head = q.kvh * a.group + r - i * a.group;
    bf16 *dst = (bf16 *)a.out + (long)(q.row0 + i) * a.o_stride + (long)head * D + lane * VEC;
#pragma unroll
    for (int e = 0; e < VEC; e += 2) *(uint32_t *)(dst + e) = pack(o[e] * inv, o[e + 1] * inv);
}

template <typename T, int D, int NR, int RW, bool PAGES> cudaError_t launch_rows4(const PagedAttnArgs &a, cudaStream_t st)
{
    using C = Rows4Cfg<D, RW>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise((const void *)paged_attention_rows4_kernel<T, D, NR, RW, PAGES>, C::SMEM);
    if (e != cudaSuccess) return e;
    const long tiles = row_tiles(a, 8 * NR);
    return launch_kernel_z(paged_attention_rows4_kernel<T, D, NR, RW, PAGES>, dim3((unsigned)(a.kv.nkv * tiles), a.rb.B, a.splits), dim3(32 * RW), C::SMEM, st, a.part_o ? 1 : a.splits, a);
}
template <int D, int NR, bool PAGES> cudaError_t launch_stream4(PagedAttnArgs a, cudaStream_t st)
{
    using C = StreamCfg<D>;
    static SmemLimit limit;
    cudaError_t e = limit.raise((const void *)paged_attention_stream4_kernel<D, NR, PAGES>, C::SMEM);
    if (e != cudaSuccess) return e;
    const int workers = stream4_workers(NR);
    a.part_ml = a.part_o + (size_t)workers * 2 * 8 * NR * D;
    int *starts = (int *)(a.part_ml + (size_t)workers * 2 * 8 * NR * 2);
    e = launch_kernel(paged_attention_stream4_kernel<D, NR, PAGES>, dim3(workers / STREAM_WARPS), dim3(32 * STREAM_WARPS), C::SMEM, st, 0, a, starts);
    if (e != cudaSuccess) return e;
    const int rows = a.max_new * a.group;
    return launch_kernel(paged_merge_stream4_kernel<D, NR>, dim3(a.kv.nkv, a.rb.B, (rows + 3) / 4), dim3(128), 0, st, 0, a, workers, starts);
}
template <typename T, int D, int NR> cudaError_t rows4_by_page(const PagedAttnArgs &a, bool stream, cudaStream_t st)
{
    const bool pages = a.kv.page >= 16 && !(a.kv.page & (a.kv.page - 1)) && (long)a.kv.nkv * a.kv.page * (D / 2) <= 0x7fffffffL;
    if constexpr (sizeof(T) == 2)
        if (stream) return pages ? launch_stream4<D, NR, true>(a, st) : launch_stream4<D, NR, false>(a, st);
    if (!pages) return launch_rows4<T, D, NR, 4, false>(a, st);
    if ((long)a.kv.nkv * a.rb.B * a.splits * row_tiles(a, 8 * NR) <= sm_count()) return launch_rows4<T, D, NR, 8, true>(a, st);
    return launch_rows4<T, D, NR, 4, true>(a, st);
}
template <int D> cudaError_t rows4_by_type(const PagedAttnArgs &a, int q_bf16, bool stream, cudaStream_t st)
{
    if (!q_bf16) return rows4_by_page<float, D, 1>(a, false, st);
    return a.max_new * a.group <= 8 ? rows4_by_page<bf16, D, 1>(a, stream, st) : rows4_by_page<bf16, D, 2>(a, stream, st);
}

} // namespace

int stream4_workers(int nr) { return sm_count() * (nr == 1 ? 3 : 2) * STREAM_WARPS; }
size_t stream4_workspace(int rows, int d) { return (size_t)stream4_workers(rows <= 8 ? 1 : 2) * 2 * (rows <= 8 ? 8 : 16) * (d + 2) * sizeof(float) + (STREAM_MAX_B + 1) * sizeof(int); }

cudaError_t launch_paged_attention_rows4(const PagedAttnArgs &a, int q_bf16, bool stream, cudaStream_t st)
{
    if (a.kv.d == 128) return rows4_by_type<128>(a, q_bf16, stream, st);
    if (a.kv.d == 64) return rows4_by_type<64>(a, q_bf16, stream, st);
    return cudaErrorInvalidValue;
}

} // namespace spd
