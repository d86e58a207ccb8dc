// Paged attention for few query rows (bf16) over 4-bit pages: the arrangement of paged_attention_rows.cu - keys and head dims as rows of
// m16n8k16 MMAs, the 8 or 16 query rows as their columns, a private ring of key tiles per warp, key ranges joined through a cluster or the
// workspace - with what 4 bits change:
//   - the cache stream is a quarter of bf16's, so that instructions bound the kernel, the unpacking of codes before all.  Codes are float16
//     operands without arithmetic: one in the lowest bits of a float16 is the subnormal number code * 2^-24, one in bits 4-7 is 16 times
//     that, and the tensor cores' products with subnormals are exact.  A word of eight codes costs four masks and a shift;
//   - q . k = sum over the halves of s (q . codes) + m sum(q), and sum p v = sum (p s) codes + sum p m: scales and smallest values meet the
//     products in float32.  Q is float16, scaled per row by a power of two (see paged_attention_rows.cu);
//   - p s has to be float16 beside the codes, and s may be anything.  The score of a key therefore carries the exponent e of its V row's largest
//     parameter: x = 2^(score + e - max) <= 2^8, weights x (s 2^-e), the key's share in the softmax x 2^-e.  What float16 leaves out of a
//     weight is then small beside the largest contribution to the output, not beside the largest softmax weight;
//   - a warp takes 32 keys a step (two MMA tiles): one wait, one maximum and one check of it for both, and each lane turns one key's
//     parameters into the factors that all lanes read (every lane for its own rows: 16 more instructions per key and lane);
//   - tiles come by cp.async: a page's 16 keys are 64 chunks of 16 bytes, two instructions for the warp; as TMA boxes they were two boxes and
//     two bulk copies from one lane, at several times the instructions.
// Measured, 32 sequences of 9 to 16 thousand tokens, 64 heads on 8: 190 us with 16 keys a step by TMA; REPLACED.
#include "paged_rows.cuh"

namespace spd {

namespace {

using namespace few;

constexpr int STEP = 32; // keys a warp takes at a time

template <int D, int RW> struct Rows4Cfg {
    static constexpr int RB = D / 2, TILE = STEP * RB;                      // bytes of a row; of K or V of a step
    static constexpr int STAGE = 2 * TILE + 2 * STEP * 8;                   // tiles and parameters
    static constexpr int STAGES = RW == 8 ? 4 : D == 128 ? 2 : 4;
    static constexpr int FACTORS = STEP * 40;                               // a step's factors: K float4, V float4, (exponent, unit)
    static constexpr int RING = RW * STAGES * STAGE, MERGE = RW * 16 * (D + 4) * 4;
    static constexpr int OFF_FACTORS = RING > MERGE ? RING : MERGE, OFF_JOIN = OFF_FACTORS + RW * FACTORS;
    static constexpr int SMEM = OFF_JOIN + join_bytes(RW) + 128;            // + alignment slack
};

__device__ __forceinline__ void cp8(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 8 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float4 lds_f4(uint32_t a)
{
    const uint4 u = lds128(a);
    return make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
}
__device__ __forceinline__ void sts_f4(uint32_t a, float x, float y, float z, float w)
{
    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(a), "f"(x), "f"(y), "f"(z), "f"(w) : "memory");
}
__device__ __forceinline__ void sts_f2(uint32_t a, float x, float y)
{
    asm volatile("st.shared.v2.f32 [%0], {%1,%2};" ::"r"(a), "f"(x), "f"(y) : "memory");
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *(const uint32_t *)&v;
}
// codes of bytes 0 and 2 of a word (shifted right by 8: bytes 1 and 3) as float16x2, in units of 2^-24 and 2^-20
__device__ __forceinline__ uint32_t low_codes(uint32_t w) { return w & 0x000f000fu; }
__device__ __forceinline__ uint32_t high_codes(uint32_t w) { return w & 0x00f000f0u; }
constexpr float LOW_UNIT = 0x1p24f, HIGH_UNIT = 0x1p20f;

// NR: groups of 8 query rows.  PAGE16: 16 keys lie in one page.
template <int D, int NR, int RW, bool PAGE16>
__global__ void __launch_bounds__(32 * RW, RW == 8 ? 1 : NR == 1 ? 4 : 3) paged_attention_rows4_kernel(const __grid_constant__ PagedAttnArgs a)
{
    using C = Rows4Cfg<D, RW>;
    constexpr int MT = D / 16, ST = C::STAGES, RB = C::RB, W = D / 32; // W: words of a lane per row
    extern __shared__ uint8_t rows4_raw[];
    uint8_t *gen = rows4_raw + ((128u - (tc::smem_u32(rows4_raw) & 127u)) & 127u);
    const uint32_t base = tc::smem_u32(gen);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const uint32_t ring = base + warp * ST * C::STAGE, fk = base + C::OFF_FACTORS + warp * C::FACTORS, fv = fk + STEP * 16, fe = fv + STEP * 16;
    if (threadIdx.x == 0) stamp_entry(a.stamp);
    pdl_launch_dependents();
    pdl_wait();
    const int kvh = blockIdx.x, b = blockIdx.y, split = blockIdx.z;
    int row0, n_new, len;
    if (!batch_row(a.rb, b, a.max_new, a.max_context, row0, n_new, len, a.err)) return; // the same for a whole cluster
    const int rows = n_new * a.group; // <= 8 NR
    const int kv_len = len + n_new, pos_max = kv_len - 1;
    // steps of 32 keys that hold a key some row sees: sinks, then the window of the first query onwards
    const int lo_min = a.window ? max(0, len - a.window + 1) : 0, first = lo_min / STEP;
    const int n_sink = min((min(a.sinks, lo_min) + STEP - 1) / STEP, first);
    const int n_steps = n_sink + (kv_len + STEP - 1) / STEP - first;
    // short sequences are cut into fewer ranges, of at least 4 steps
    const int splits = min(a.splits, (n_steps + 3) / 4);
    const int per = splits > 1 ? n_steps / splits : n_steps, extra = n_steps - per * splits; // the first `extra` ranges get one more
    const int j_begin = split < splits ? split * per + min(split, extra) : 0;
    const int j_end = split < splits ? j_begin + per + (split < extra ? 1 : 0) : 0;
    const int n_mine = (j_end - j_begin - warp + RW - 1) / RW; // steps j_begin + warp, + RW, ...

    const int32_t *bt = a.rb.table + (long)b * a.rb.max_pages;
    const int bpp = a.kv.page / 16; // PAGE16: blocks of 16 keys per page
    auto key0 = [&](int i) { const int j = j_begin + warp + i * RW; return (j < n_sink ? j : first + (j - n_sink)) * STEP; };
    // every row sees every key of the 32 from t0 on
    auto seen_by_all = [&](int t0) { return t0 + STEP - 1 <= len && (!a.window || t0 > pos_max - a.window || t0 + STEP - 1 < a.sinks); };
    auto row_in = [&](int page, int in_page) -> long {
        if (page < 0 || page >= a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); return -1; }
        return ((long)page * a.kv.nkv + kvh) * a.kv.page + in_page;
    };
    // PAGE16: cached rows of the step's keys 0 and 16; else (the first only) of this lane's key.  -1: no row needs them, or a bad page id.
    struct Where { long r[2]; };
    auto lookup = [&](int i) {
        Where w{{-1, -1}};
        const int t0 = key0(i);
        if (PAGE16) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = t0 + 16 * h, blk = t >> 4;
                if (t < kv_len && (t + 15 >= lo_min || t < a.sinks)) w.r[h] = bpp == 1 ? row_in(bt[blk], 0) : row_in(bt[blk / bpp], blk % bpp * 16);
            }
        } else {
            const int t = t0 + lane;
            if (t < kv_len && (t >= lo_min || t < a.sinks)) w.r[0] = row_in(bt[t / a.kv.page], t % a.kv.page);
        }
        return w;
    };
    // 16-byte chunk c of row r of a tile
    auto at = [&](int r, int c) -> uint32_t { return RB == 64 ? r * 64 + ((c ^ ((r >> 1) & 3)) << 4) : r * 32 + ((c ^ ((r >> 2) & 1)) << 4); };
    constexpr int CPR = RB / 16, RPI = 32 / CPR; // chunks per row, rows per copy instruction
    const uint32_t lane_dst = at(lane / CPR, lane % CPR);
    auto load = [&](int stage, const Where &w) {
        const uint32_t dst = ring + stage * C::STAGE;
#pragma unroll
        for (int i = 0; i < STEP / RPI; ++i) {
            const int r = i * RPI + lane / CPR;
            const long row = PAGE16 ? w.r[i * RPI / 16] + (r & 15) : __shfl_sync(0xffffffffu, w.r[0], r);
            const bool valid = PAGE16 ? w.r[i * RPI / 16] >= 0 : row >= 0;
            const long off = valid ? row * RB + (lane % CPR) * 16 : 0;
            cp16(dst + lane_dst + i * RPI * RB, (const uint8_t *)a.kv.k + off, valid);
            cp16(dst + C::TILE + lane_dst + i * RPI * RB, (const uint8_t *)a.kv.v + off, valid);
        }
        const long mine = PAGE16 ? (lane < 16 ? w.r[0] : w.r[1]) : w.r[0];
        const bool valid = mine >= 0;
        const long off = valid ? mine + (PAGE16 ? lane & 15 : 0) : 0;
        cp8(dst + 2 * C::TILE + lane * 8, (const uint2 *)a.kv.ks + off, valid);
        cp8(dst + 2 * C::TILE + STEP * 8 + lane * 8, (const uint2 *)a.kv.vs + off, valid);
    };

#pragma unroll
    for (int s = 0; s < ST; ++s) {
        if (s < n_mine) load(s, lookup(s));
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    Where next{{-1, -1}};
    if (ST < n_mine) next = lookup(ST);

    // Q fragments (column g of a group of 8 rows), in the order of the codes; rows beyond the last are zero.  A lane's dims: D / 8 of either half.
    uint32_t qf[NR][2 * W][2];
    float qs[NR][2], qsum[NR][2][2]; // of this lane's columns 2 t4 and 2 t4 + 1: to base-2 units; sums of the halves in those
    int pos[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int r = g + 8 * n;
        const bool live = r < rows;
        const int i = live ? r / a.group : 0, head = live ? r - i * a.group : 0;
        const bf16 *qp = (const bf16 *)a.q + (long)(row0 + i) * a.q_stride + (long)(kvh * a.group + head) * D;
        uint4 u[W];
        uint32_t top = 0; // largest magnitude's bits
#pragma unroll
        for (int m = 0; m < W; ++m) {
            u[m] = live ? *(const uint4 *)(qp + (D / 2) * (m / (W / 2)) + (D / 8) * t4 + 8 * (m % (W / 2))) : make_uint4(0, 0, 0, 0);
            const uint32_t x = __vmaxu2(__vmaxu2(u[m].x & 0x7fff7fffu, u[m].y & 0x7fff7fffu), __vmaxu2(u[m].z & 0x7fff7fffu, u[m].w & 0x7fff7fffu));
            top = max(top, max(x & 0xffffu, x >> 16));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int ex = max((int)(top >> 7), 27) - 127;                    // 2^ex <= largest < 2^(ex + 1), ex >= -100
        const float f = __uint_as_float((uint32_t)(127 + 14 - ex) << 23); // to [2^14, 2^15)
        const float my_qs = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + ex) << 23);
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int m = 0; m < W; ++m) {
            const uint32_t w[4] = {u[m].x, u[m].y, u[m].z, u[m].w};
            uint32_t x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __half2 v = __floats2half2_rn(__uint_as_float(w[e] << 16) * f, __uint_as_float(w[e] & 0xffff0000u) * f);
                x[e] = *(const uint32_t *)&v;
                sum[m / (W / 2)] += __low2float(v) + __high2float(v);
            }
            qf[n][2 * m][0] = __byte_perm(x[0], x[1], 0x5410); qf[n][2 * m][1] = __byte_perm(x[0], x[1], 0x7632);
            qf[n][2 * m + 1][0] = __byte_perm(x[2], x[3], 0x5410); qf[n][2 * m + 1][1] = __byte_perm(x[2], x[3], 0x7632);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 1);
            sum[h] += __shfl_xor_sync(0xffffffffu, sum[h], 2);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = 8 * n + 2 * t4 + e;
            pos[n][e] = c < rows ? len + c / a.group : -1;
            qs[n][e] = __shfl_sync(0xffffffffu, my_qs, (2 * t4 + e) * 4);
#pragma unroll
            for (int h = 0; h < 2; ++h) qsum[n][e][h] = __shfl_sync(0xffffffffu, sum[h], (2 * t4 + e) * 4) * qs[n][e];
        }
    }

    // where this lane reads in a tile; the second eight and sixteen rows are a fixed distance away
    const uint32_t lane_k = RB == 64 ? at(key_of(g), t4) : at(key_of(g), t4 >> 1) + (t4 & 1) * 8;
    auto v_at = [&](int r) { return RB == 64 ? at(r, g >> 1) + (g & 1) * 8 : at(r, g >> 2) + (g & 3) * 4; };
    const uint32_t lane_v0 = v_at(key_of(2 * t4)), lane_v1 = v_at(key_of(2 * t4 + 1));
    const int my_key = key_of(g);

    float o[NR][MT][4]; // tiles 0 .. MT / 2 - 1: first half of the head, in units of 2^-24; the others 2^-20
    float m_used[NR][2], l[NR][2], om[NR][2][2]; // om: weighted sums of the halves' smallest values, as l over this lane's keys
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int i = 0; i < MT; ++i) { o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f; }
#pragma unroll
        for (int e = 0; e < 2; ++e) { m_used[n][e] = -INFINITY; l[n][e] = om[n][e][0] = om[n][e][1] = 0.f; }
    }

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
            sts_f4(fk + lane * 16, k_bad ? __uint_as_float(0x7fc00000u) : kv4_scale(kp.x) * LOW_UNIT, kv4_scale(kp.y) * HIGH_UNIT, kv4_min(kp.x), kv4_min(kp.y));
            const uint32_t top = max(vm & 0xffffu, vm >> 16);
            const bool v_bad = top >= 0x7f80u;
            const int ex = min(max((int)(top >> 7), 127 - 60), 127 + 30);
            const float unit = __uint_as_float((uint32_t)(254 - ex) << 23), f = v_bad ? 0.f : unit;
            const float ev = v_bad ? __uint_as_float(0x7fc00000u) : __uint_as_float(0x4b000000u | ex) - (8388608.f + 127.f); // 2^23 + ex
            const uint2 q = v_bad ? make_uint2(0, 0) : vp;
            sts_f4(fv + lane * 16, kv4_scale(q.x) * f, kv4_scale(q.y) * f, kv4_min(q.x) * f, kv4_min(q.y) * f);
            sts_f2(fe + lane * 8, ev, unit);
        }
        float s[2][NR][4], unit[2][2]; // scores in base-2 units; [tile][rows g and g + 8]
        float acc[2][2][NR][4];        // q . codes [tile][half]
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < NR; ++n) acc[u][h][n][0] = acc[u][h][n][1] = acc[u][h][n][2] = acc[u][h][n][3] = 0.f;
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
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    mma16816<true>(acc[u][0][n], low_codes(w0[i]), low_codes(w1[i]), low_codes(y0), low_codes(y1), qf[n][i][0], qf[n][i][1]);
                    mma16816<true>(acc[u][1][n], high_codes(w0[i]), high_codes(w1[i]), high_codes(y0), high_codes(y1), qf[n][W + i][0], qf[n][W + i][1]);
                }
            }
        }
        __syncwarp(); // the factors
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int key = 16 * u + 8 * h + my_key;
                const float4 k = lds_f4(fk + key * 16);
                const uint2 eu = lds64(fe + key * 8);
                unit[u][h] = __uint_as_float(eu.y);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float shift = fmaf(k.w, qsum[n][e][1], fmaf(k.z, qsum[n][e][0], __uint_as_float(eu.x)));
                        s[u][n][2 * h + e] = fmaf(fmaf(k.y, acc[u][1][n][2 * h + e], k.x * acc[u][0][n][2 * h + e]), qs[n][e], shift);
                    }
                }
            }
        }
        if (!seen_by_all(t0)) { // masked scores are -inf whatever was computed
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!sees(t0 + 16 * u + 8 * (e >> 1) + my_key, pos[n][e & 1], a.window, a.sinks)) s[u][n][e] = -INFINITY;
        }
        float mx[NR][2];
        bool grow = false;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float m = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e]));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                mx[n][e] = m;
                grow |= m > m_used[n][e] + 8.f; // first keys of a row included (-inf)
            }
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                float f[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float nm = fmaxf(m_used[n][e], mx[n][e]);
                    f[e] = m_used[n][e] == -INFINITY ? 0.f : ex2(m_used[n][e] - nm);
                    m_used[n][e] = nm;
                    l[n][e] *= f[e];
                    om[n][e][0] *= f[e];
                    om[n][e][1] *= f[e];
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) { o[n][i][0] *= f[0]; o[n][i][1] *= f[1]; o[n][i][2] *= f[0]; o[n][i][3] *= f[1]; }
            }
        }
        float mb[NR][2]; // no key seen so far: the weights are 2^-inf whatever this is
#pragma unroll
        for (int n = 0; n < NR; ++n) { mb[n][0] = fmaxf(m_used[n][0], -3e38f); mb[n][1] = fmaxf(m_used[n][1], -3e38f); }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            uint32_t pf[2][NR][2]; // [half]
            float w[2][NR][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 v = lds_f4(fv + (16 * u + 8 * h + my_key) * 16);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float x = ex2(s[u][n][2 * h + e] - mb[n][e]);
                        l[n][e] = fmaf(x, unit[u][h], l[n][e]);
                        om[n][e][0] = fmaf(x, v.z, om[n][e][0]);
                        om[n][e][1] = fmaf(x, v.w, om[n][e][1]);
                        w[0][n][2 * h + e] = x * v.x;
                        w[1][n][2 * h + e] = x * v.y;
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    pf[q][n][0] = transpose8x8(pack_half(w[q][n][0], w[q][n][1]));
                    pf[q][n][1] = transpose8x8(pack_half(w[q][n][2], w[q][n][3]));
                }
            }
            // bytes g D / 16 .. of four keys: dims from there on in either half
            uint32_t v[4][W / 2];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t p = sV + (q & 1 ? lane_v1 : lane_v0) + ((q >> 1) * 8 + u * 16) * RB;
                if (W == 4) {
                    const uint2 x = lds64(p);
                    v[q][0] = x.x; v[q][W / 2 - 1] = x.y;
                } else
                    v[q][0] = lds32(p);
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                // bytes (k0.2j, k0.2j+1, k1.2j, k1.2j+1), j = i & 1
                const uint32_t sel = i & 1 ? 0x7632 : 0x5410;
                const uint32_t x0 = __byte_perm(v[0][i >> 1], v[1][i >> 1], sel), x1 = __byte_perm(v[2][i >> 1], v[3][i >> 1], sel);
                const uint32_t y0 = x0 >> 8, y1 = x1 >> 8;
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    mma16816<true>(o[n][i], low_codes(x0), low_codes(y0), low_codes(x1), low_codes(y1), pf[0][n][0], pf[0][n][1]);
                    mma16816<true>(o[n][W + i], high_codes(x0), high_codes(y0), high_codes(x1), high_codes(y1), pf[1][n][0], pf[1][n][1]);
                }
            }
        }
        __syncwarp(); // every lane has read the stage and the factors
        if (it + ST < n_mine) {
            load(stage, next);
            if (it + ST + 1 < n_mine) next = lookup(it + ST + 1);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage == ST) stage = 0;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // the warps' partial rows, over the rings
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) {
                l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], x);
                om[n][e][0] += __shfl_xor_sync(0xffffffffu, om[n][e][0], x);
                om[n][e][1] += __shfl_xor_sync(0xffffffffu, om[n][e][1], x);
            }
        }
    }
    __syncthreads();
    float *mo = (float *)gen, *ml = mo + RW * 16 * (D + 2); // [warp][16][D + 2], [warp][16][2]
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * t4 + e;
            if (r < rows) {
                float *dst = mo + (warp * 16 + r) * (D + 2) + g * (D / 16);
#pragma unroll
                for (int i = 0; i < MT; ++i) { // MMA row g: dim g D/16 + 2i of the tile's half, row g + 8: + 1
                    const int h = i / W;
                    const float x = h ? HIGH_UNIT : LOW_UNIT;
                    *(float2 *)(dst + h * (D / 2) + 2 * (i % W)) = make_float2(fmaf(o[n][i][e], x, om[n][e][h]), fmaf(o[n][i][2 + e], x, om[n][e][h]));
                }
                if (g == 0) { ml[(warp * 16 + r) * 2] = m_used[n][e]; ml[(warp * 16 + r) * 2 + 1] = l[n][e]; }
            }
        }
    }
    join_rows<D, RW>(a, gen, C::OFF_JOIN, rows, row0, len, kvh, split, splits, [](int, int, float &, float &) {});
    if (threadIdx.x == 0) stamp_exit(a.stamp);
}

template <int D, int NR, int RW, bool PAGE16> cudaError_t launch_rows4(const PagedAttnArgs &a, cudaStream_t st)
{
    using C = Rows4Cfg<D, RW>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise((const void *)paged_attention_rows4_kernel<D, NR, RW, PAGE16>, C::SMEM);
    if (e != cudaSuccess) return e;
    return launch_kernel_z(paged_attention_rows4_kernel<D, NR, RW, PAGE16>, dim3(a.kv.nkv, a.rb.B, a.splits), dim3(32 * RW), C::SMEM, st, a.part_o ? 1 : a.splits, a);
}
template <int D, int NR> cudaError_t rows4_by_page(const PagedAttnArgs &a, cudaStream_t st)
{
    if (a.kv.page % 16) return launch_rows4<D, NR, 4, false>(a, st);
    if ((long)a.kv.nkv * a.rb.B * a.splits <= sm_count()) return launch_rows4<D, NR, 8, true>(a, st);
    return launch_rows4<D, NR, 4, true>(a, st);
}
template <int D> cudaError_t rows4_by_count(const PagedAttnArgs &a, cudaStream_t st)
{
    return a.max_new * a.group <= 8 ? rows4_by_page<D, 1>(a, st) : rows4_by_page<D, 2>(a, st);
}

} // namespace

cudaError_t launch_paged_attention_rows4(const PagedAttnArgs &a, cudaStream_t st)
{
    if (a.kv.d == 128) return rows4_by_count<128>(a, st);
    if (a.kv.d == 64) return rows4_by_count<64>(a, st);
    return cudaErrorInvalidValue;
}

} // namespace spd
