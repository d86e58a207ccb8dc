// Paged attention for few query rows (bf16): all rows of a (sequence, KV head) - new tokens times query heads per KV head -
// fit the 16 rows of one m16n8k16 MMA tile, as in single-token steps and short drafts.
//
// Bound: the cache stream.  Per 16 cached keys a warp loads two 16 x head_dim tiles and issues 2 * head_dim / 8 MMAs, a
// small part of an SM's issue slots at the rate HBM delivers the tiles, so the simple tensor path (mma.sync, registers) is
// enough and the rest serves the loads:
//   - every warp works on its own 16-key blocks (j, j + 4, ...) with a private ring of cp.async stages: no block-wide
//     barrier between the first load and the merge, and about 100 KB in flight per SM (2 thread blocks);
//   - the keys of a (sequence, KV head) are cut into ranges over thread blocks where there are few of them (grid z), the
//     ranges' partial rows are added up by paged_merge_kernel;
//   - 8-bit caches stay 8-bit up to the fragment registers.  A 16-byte shared-memory load gives a lane 16 consecutive head
//     dims of one key; any assignment of dims to the MMA's k index is right as long as Q uses the same one, so the even and
//     the odd bytes of a 32-bit word become the two B registers of one MMA without a shuffle.  V is loaded as 16 dims of four
//     keys, whose bytes are interleaved by key pairs; the output columns come out permuted and are stored where they belong.
//     Row scales multiply the fp32 scores (K) and the softmax weights before they are rounded (V).
//   - e4m3 -> bf16: sign, exponent and mantissa moved to their places give the value times 2^-120, one bf16x2 product puts
//     the exponent right (exact, subnormals too).  int8 -> bf16: the low 7 bits over the exponent of 128 give 128 + low, and
//     128 (or 256 where the sign bit is set) is subtracted (exact).
// Softmax: base 2, fp32, per warp; the accumulators follow the running maximum lazily (they are rescaled when it has grown by
// more than 2^8: weights stay below 2^8, where bf16 rounds as finely as at 1).
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace spd {

namespace {

constexpr int RW = 4, R_THREADS = 32 * RW, BK16 = 16;

template <int FMT, int D> struct RowsCfg {
    static constexpr int ES = FMT == KV_BF16 ? 2 : 1;
    static constexpr int RB = D * ES;                      // bytes of a cached row
    static constexpr int CPR = RB / 16;                    // 16-byte chunks of it
    static constexpr int SC = FMT == KV_BF16 ? 0 : 128;    // 16 K scales, 16 V scales
    static constexpr int STAGE = 2 * BK16 * RB + SC;
    static constexpr int STAGES = FMT == KV_BF16 && D == 128 ? 3 : 6;
    static constexpr int RING = RW * STAGES * STAGE;
    static constexpr int MERGE = RW * 16 * (D + 4) * 4;
    static constexpr int SMEM = (RING > MERGE ? RING : MERGE);
};

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 16 : 0; // 0 source bytes: zero fill
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ float2 lds_f2(uint32_t a)
{
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t *)&v;
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// keys t of a row at position pos (-1: no row) that it sees
__device__ __forceinline__ bool sees(int t, int pos, int window, int sinks) { return t <= pos && (!window || t > pos - window || t < sinks); }

// P16: the page size is a multiple of 16, so a 16-key block lies in one page
template <int FMT, int D, bool P16>
__global__ void __launch_bounds__(R_THREADS, 2) paged_attention_rows_kernel(const __grid_constant__ PagedAttnArgs a)
{
    using C = RowsCfg<FMT, D>;
    constexpr bool Q8 = FMT != KV_BF16;
    constexpr int NT = D / 8, KS = D / 16;
    extern __shared__ __align__(128) uint8_t rows_smem[];
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const int kvh = blockIdx.x, b = blockIdx.y, split = blockIdx.z;
    int row0, n_new, len;
    if (!batch_row(a.rb, b, a.max_new, a.max_context, row0, n_new, len, a.err)) return;
    const int rows = n_new * a.group; // <= 16
    const int kv_len = len + n_new;
    // blocks of 16 keys that hold a key some row sees: sinks, then the window of the first query onwards
    const int lo_min = a.window ? max(0, len - a.window + 1) : 0, first = lo_min / BK16;
    const int n_sink = min((min(a.sinks, lo_min) + BK16 - 1) / BK16, first);
    const int n_blocks = n_sink + (kv_len + BK16 - 1) / BK16 - first;
    // short sequences are cut into fewer ranges, of at least 8 blocks
    const int splits = min(a.splits, (n_blocks + 7) / 8);
    const int j_begin = split < splits ? (int)((long)n_blocks * split / splits) : 0;
    const int j_end = split < splits ? (int)((long)n_blocks * (split + 1) / splits) : 0;

    const uint32_t ring = tc::smem_u32(rows_smem) + warp * C::STAGES * C::STAGE;
    const int32_t *bt = a.rb.table + (long)b * a.rb.max_pages;
    auto block_of = [&](int j) { return j < n_sink ? j : first + (j - n_sink); };
    auto row_valid = [&](int t) { return t < kv_len && (t >= lo_min || t < a.sinks); };
    auto lookup = [&](int t) { // cached row of key t, or -1
        const int pi = t / a.kv.page, page = bt[pi];
        if (page < 0 || page >= a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); return -1L; }
        return ((long)page * a.kv.nkv + kvh) * a.kv.page + (t - pi * a.kv.page);
    };
    // cached row of this lane's key (lane & 15) of block j - P16: of the block's first key
    auto lookup_block = [&](int j) -> long {
        const int t0 = block_of(j) * BK16;
        if (P16) return lookup(t0);
        const int t = t0 + (lane & 15);
        return row_valid(t) ? lookup(t) : -1L;
    };
    auto load_block = [&](int j, int stage, long where) {
        const uint32_t sK = ring + stage * C::STAGE, sV = sK + BK16 * C::RB;
        const int t0 = block_of(j) * BK16;
        constexpr int RPI = 32 / C::CPR; // rows per instruction
        const int c = lane % C::CPR;
#pragma unroll
        for (int i = 0; i < BK16 / RPI; ++i) {
            const int r = i * RPI + lane / C::CPR;
            long row;
            bool ok;
            if (P16) { row = where + r; ok = where >= 0 && row_valid(t0 + r); }
            else { row = __shfl_sync(0xffffffffu, where, r); ok = row >= 0; }
            const long off = ok ? row * C::RB + c * 16 : 0;
            const int ck = C::CPR >= 8 ? c ^ ((r & 1) << 2) : c;
            const int cv = Q8 ? (C::CPR == 8 ? c ^ (r & 6) : c ^ (r & 2)) : c ^ (r & 7);
            cp16(sK + r * C::RB + ck * 16, (const uint8_t *)a.kv.k + off, ok);
            cp16(sV + r * C::RB + cv * 16, (const uint8_t *)a.kv.v + off, ok);
        }
        if (Q8) {
            const int r = lane & 15;
            const long row = P16 ? where + r : where;
            const bool ok = P16 ? where >= 0 && row_valid(t0 + r) : where >= 0;
            cp4(sV + BK16 * C::RB + lane * 4, (lane < 16 ? a.kv.ks : a.kv.vs) + (ok ? row : 0), ok);
        }
    };

    // Q fragments; rows beyond the tile's are zero
    uint32_t qf[KS][4];
    int pos[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h;
        const bool live = r < rows;
        const int i = live ? r / a.group : 0, head = live ? r % a.group : 0;
        pos[h] = live ? len + i : -1;
        const bf16 *qp = (const bf16 *)a.q + (long)(row0 + i) * a.q_stride + (long)(kvh * a.group + head) * D;
        if (!Q8) {
#pragma unroll
            for (int m = 0; m < D / 32; ++m) {
                const uint4 u = live ? *(const uint4 *)(qp + 32 * m + 8 * t4) : make_uint4(0, 0, 0, 0);
                qf[2 * m][h] = u.x; qf[2 * m][2 + h] = u.y; qf[2 * m + 1][h] = u.z; qf[2 * m + 1][2 + h] = u.w;
            }
        } else {
#pragma unroll
            for (int m = 0; m < D / 64; ++m) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint4 u = live ? *(const uint4 *)(qp + 64 * m + 16 * t4 + 8 * half) : make_uint4(0, 0, 0, 0);
                    // dims (0, 2) and (1, 3) of every four: the even and the odd bytes of a cached word
                    qf[4 * m + 2 * half][h] = __byte_perm(u.x, u.y, 0x5410);
                    qf[4 * m + 2 * half][2 + h] = __byte_perm(u.x, u.y, 0x7632);
                    qf[4 * m + 2 * half + 1][h] = __byte_perm(u.z, u.w, 0x5410);
                    qf[4 * m + 2 * half + 1][2 + h] = __byte_perm(u.z, u.w, 0x7632);
                }
            }
        }
    }
    const int pos_max = kv_len - 1;
    // every row sees every key of the 16 from t0 on
    auto seen_by_all = [&](int t0) { return t0 + 15 <= len && (!a.window || t0 > pos_max - a.window || t0 + 15 < a.sinks); };

    float o[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) { o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f; }
    float m_used[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    bool dirty = false; // a NaN or infinity of V was taken out of a block that not every row sees

    const int n_mine = (j_end - j_begin - warp + RW - 1) / RW; // blocks j_begin + warp, + RW, ...
    long where = 0;
    for (int s = 0; s < C::STAGES - 1; ++s) {
        if (s < n_mine) load_block(j_begin + warp + s * RW, s, lookup_block(j_begin + warp + s * RW));
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (C::STAGES - 1 < n_mine) where = lookup_block(j_begin + warp + (C::STAGES - 1) * RW);
    int stage = 0;
    for (int it = 0; it < n_mine; ++it) {
        asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 2) : "memory");
        __syncwarp();
        {   // refill the stage read in the previous iteration (STAGES - 1 ahead), page lookups another one ahead
            const int nx = it + C::STAGES - 1;
            if (nx < n_mine) load_block(j_begin + warp + nx * RW, stage == 0 ? C::STAGES - 1 : stage - 1, where);
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (nx + 1 < n_mine) where = lookup_block(j_begin + warp + (nx + 1) * RW);
        }
        const uint32_t sK = ring + stage * C::STAGE, sV = sK + BK16 * C::RB, sS = sV + BK16 * C::RB;
        const int t0 = block_of(j_begin + warp + it * RW) * BK16;
        float s[2][4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
            const int r = nt * 8 + g;
            if (!Q8) {
#pragma unroll
                for (int m = 0; m < D / 32; ++m) {
                    const uint4 u = lds128(sK + r * C::RB + (((4 * m + t4) ^ ((r & 1) << 2)) << 4));
                    mma16816(s[nt], qf[2 * m][0], qf[2 * m][1], qf[2 * m][2], qf[2 * m][3], u.x, u.y);
                    mma16816(s[nt], qf[2 * m + 1][0], qf[2 * m + 1][1], qf[2 * m + 1][2], qf[2 * m + 1][3], u.z, u.w);
                }
            } else {
#pragma unroll
                for (int m = 0; m < D / 64; ++m) {
                    const uint4 u = lds128(sK + r * C::RB + ((C::CPR >= 8 ? (4 * m + t4) ^ ((r & 1) << 2) : t4) << 4));
                    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = 4 * m + i;
                        mma16816(s[nt], qf[k][0], qf[k][1], qf[k][2], qf[k][3], even2<FMT>(w[i]), odd2<FMT>(w[i]));
                    }
                }
            }
        }
        // scores in base 2; masked ones -inf whatever was computed
        const bool all_seen = seen_by_all(t0);
        float mx[2] = {-INFINITY, -INFINITY};
        float2 kscale[2], vscale[2];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            if (Q8) { kscale[nt] = lds_f2(sS + (nt * 8 + 2 * t4) * 4); vscale[nt] = lds_f2(sS + 64 + (nt * 8 + 2 * t4) * 4); }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = t0 + nt * 8 + 2 * t4 + (e & 1), h = e >> 1;
                float v = s[nt][e] * a.scale_log2;
                if (Q8) v *= (e & 1) ? kscale[nt].y : kscale[nt].x;
                if (!all_seen && !sees(t, pos[h], a.window, a.sinks)) v = -INFINITY;
                s[nt][e] = v;
                mx[h] = fmaxf(mx[h], v);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
        }
        const bool grow = mx[0] > m_used[0] + 8.f || mx[1] > m_used[1] + 8.f; // first keys of a row included (-inf)
        if (__any_sync(0xffffffffu, grow)) {
            float f[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float nm = fmaxf(m_used[h], mx[h]);
                f[h] = m_used[h] == -INFINITY ? 0.f : ex2(m_used[h] - nm);
                m_used[h] = nm;
                l[h] *= f[h];
            }
#pragma unroll
            for (int i = 0; i < NT; ++i) { o[i][0] *= f[0]; o[i][1] *= f[0]; o[i][2] *= f[1]; o[i][3] *= f[1]; }
        }
        const float base[2] = {m_used[0] == -INFINITY ? 0.f : m_used[0], m_used[1] == -INFINITY ? 0.f : m_used[1]};
        uint32_t pf[4];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[e] = ex2(s[nt][e] - base[e >> 1]);
                l[e >> 1] += p[e];
                if (Q8) { // a masked key's scale may be anything
                    const float w = p[e] * ((e & 1) ? vscale[nt].y : vscale[nt].x);
                    p[e] = s[nt][e] == -INFINITY ? 0.f : w;
                }
            }
            pf[2 * nt] = pack(p[0], p[1]);
            pf[2 * nt + 1] = pack(p[2], p[3]);
        }
        if (!Q8) {
            if (!all_seen) {
                // 0 * NaN would reach rows that do not see the key: take non-finite values out here, give them back at the end
                constexpr int RPI = 32 / C::CPR;
#pragma unroll
                for (int i = 0; i < BK16 / RPI; ++i) {
                    const uint32_t at = sV + (i * RPI + lane / C::CPR) * C::RB + (lane % C::CPR) * 16;
                    uint4 u = lds128(at);
                    uint32_t w[4] = {u.x, u.y, u.z, u.w};
                    bool bad = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; bad = true; }
                        if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; bad = true; }
                    }
                    if (bad) { sts128(at, make_uint4(w[0], w[1], w[2], w[3])); dirty = true; }
                }
                __syncwarp();
            }
#pragma unroll
            for (int dp = 0; dp < D / 16; ++dp) {
                uint32_t vf[4];
                const int r = (lane & 7) + (((lane >> 3) & 1) << 3), c = dp * 2 + (lane >> 4);
                ldsm4t(vf, sV + r * C::RB + ((c ^ (r & 7)) << 4));
                mma16816(o[2 * dp], pf[0], pf[1], pf[2], pf[3], vf[0], vf[1]);
                mma16816(o[2 * dp + 1], pf[0], pf[1], pf[2], pf[3], vf[2], vf[3]);
            }
        } else {
            constexpr int W = D / 32; // words per key and lane
            uint32_t v[4][W];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = 2 * t4 + (q & 1) + (q >> 1) * 8;
                if (W == 4) {
                    const uint4 u = lds128(sV + r * C::RB + ((g ^ (r & 6)) << 4));
                    v[q][0] = u.x; v[q][1] = u.y; v[q][2 % W] = u.z; v[q][3 % W] = u.w;
                } else {
                    const uint2 u = lds64(sV + r * C::RB + (((g >> 1) ^ (r & 2)) << 4) + (g & 1) * 8);
                    v[q][0] = u.x; v[q][1] = u.y;
                }
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                // bytes (k0.0, k0.1, k1.0, k1.1): even bytes = column 0 of keys (k0, k1), odd bytes = column 1
                const uint32_t x0 = __byte_perm(v[0][w], v[1][w], 0x5410), x1 = __byte_perm(v[2][w], v[3][w], 0x5410);
                const uint32_t y0 = __byte_perm(v[0][w], v[1][w], 0x7632), y1 = __byte_perm(v[2][w], v[3][w], 0x7632);
                mma16816(o[4 * w], pf[0], pf[1], pf[2], pf[3], even2<FMT>(x0), even2<FMT>(x1));
                mma16816(o[4 * w + 1], pf[0], pf[1], pf[2], pf[3], odd2<FMT>(x0), odd2<FMT>(x1));
                mma16816(o[4 * w + 2], pf[0], pf[1], pf[2], pf[3], even2<FMT>(y0), even2<FMT>(y1));
                mma16816(o[4 * w + 3], pf[0], pf[1], pf[2], pf[3], odd2<FMT>(y0), odd2<FMT>(y1));
            }
        }
        stage = stage + 1 == C::STAGES ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");

    // the four warps' partial rows, merged through shared memory (the rings are done with)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    }
    const int any_dirty = __syncthreads_or(dirty);
    float *mo = (float *)rows_smem, *ml = mo + RW * 16 * (D + 2); // [warp][16][D + 2], [warp][16][2]
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int r = g + 8 * h;
        if (r < rows) {
            float *dst = mo + (warp * 16 + r) * (D + 2);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                if (!Q8) *(float2 *)(dst + nt * 8 + 2 * t4) = make_float2(o[nt][2 * h], o[nt][2 * h + 1]);
                else { // column n of MMA nt = dim n * D / 8 + nt
                    dst[(2 * t4) * (D / 8) + nt] = o[nt][2 * h];
                    dst[(2 * t4 + 1) * (D / 8) + nt] = o[nt][2 * h + 1];
                }
            }
            if (t4 == 0) { ml[(warp * 16 + r) * 2] = m_used[h]; ml[(warp * 16 + r) * 2 + 1] = l[h]; }
        }
    }
    __syncthreads();
    const long plane = (long)a.rb.n_tokens * a.nq;
    for (int idx = threadIdx.x; idx < rows * (D / 2); idx += R_THREADS) {
        const int r = idx / (D / 2), c = idx % (D / 2) * 2;
        float m = -INFINITY, den = 0.f, x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < RW; ++w) m = fmaxf(m, ml[(w * 16 + r) * 2]);
#pragma unroll
        for (int w = 0; w < RW; ++w) {
            const float mw = ml[(w * 16 + r) * 2], f = mw == -INFINITY ? 0.f : ex2(mw - m);
            den = fmaf(ml[(w * 16 + r) * 2 + 1], f, den);
            const float2 v = *(const float2 *)(mo + (w * 16 + r) * (D + 2) + c);
            x = fmaf(v.x, f, x);
            y = fmaf(v.y, f, y);
        }
        const int i = r / a.group, head = kvh * a.group + r % a.group;
        if (!Q8 && any_dirty) { // the values taken out above, for the rows that see them
            const int p = len + i;
            for (int j = j_begin; j < j_end; ++j) {
                const int t0 = block_of(j) * BK16;
                for (int t = t0; t < t0 + BK16 && !seen_by_all(t0); ++t) {
                    if (!sees(t, p, a.window, a.sinks)) continue;
                    const long row = lookup(t);
                    if (row < 0) continue;
                    const __nv_bfloat162 v = *(const __nv_bfloat162 *)((const bf16 *)a.kv.v + row * D + c);
                    const float vx = __bfloat162float(v.x), vy = __bfloat162float(v.y);
                    if (!isfinite(vx)) x += vx;
                    if (!isfinite(vy)) y += vy;
                }
            }
        }
        if (a.splits == 1) {
            const float inv = den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
            *(uint32_t *)((bf16 *)a.out + (long)(row0 + i) * a.o_stride + (long)head * D + c) = pack(x * inv, y * inv);
        } else {
            const long at = (long)split * plane + (long)(row0 + i) * a.nq + head;
            if (den != den) m = fmaxf(m, 0.f); // scores that are all NaN leave no maximum: not an empty range
            if (m != -INFINITY) *(float2 *)(a.part_o + at * D + c) = make_float2(x, y);
            if (c == 0) { a.part_ml[at * 2] = m; a.part_ml[at * 2 + 1] = den; }
        }
    }
}

// Adds up the key ranges of a split launch: one warp per (token, query head), the ranges' weights in its lanes.
template <typename T, int D>
__global__ void __launch_bounds__(128) paged_merge_kernel(const __grid_constant__ PagedAttnArgs a)
{
    constexpr int VEC = D / 32;
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const long w = (long)blockIdx.x * 4 + (threadIdx.x >> 5), plane = (long)a.rb.n_tokens * a.nq;
    if (w >= plane) return;
    const int t = (int)(w / a.nq), head = (int)(w % a.nq);
    int before = 0;
    for (int i0 = 0; i0 <= a.rb.B; i0 += 32) {
        const unsigned mk = __ballot_sync(0xffffffffu, i0 + lane <= a.rb.B && a.rb.cu[i0 + lane] <= t);
        before += __popc(mk);
        if (mk != 0xffffffffu) break;
    }
    if (before < 1 || before > a.rb.B) return;
    int row0, n_new, len;
    if (!batch_row(a.rb, before - 1, a.max_new, a.max_context, row0, n_new, len, a.err)) return;
    float m = -INFINITY;
    for (int s = lane; s < a.splits; s += 32) m = fmaxf(m, __ldcg(a.part_ml + ((long)s * plane + w) * 2));
    m = warp_max(m);
    float o[VEC], den = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[e] = 0.f;
    for (int s = 0; s < a.splits; ++s) {
        const long at = (long)s * plane + w;
        const float ms = __ldcg(a.part_ml + at * 2);
        if (ms == -INFINITY) continue; // an empty range: nothing was written
        const float f = ex2(ms - m);
        den = fmaf(__ldcg(a.part_ml + at * 2 + 1), f, den);
#pragma unroll
        for (int e = 0; e < VEC; ++e) o[e] = fmaf(__ldcg(a.part_o + at * D + lane * VEC + e), f, o[e]);
    }
    const float inv = den > 0.f ? 1.f / den : (den == 0.f ? 0.f : den);
    T *dst = (T *)a.out + (long)t * a.o_stride + (long)head * D + lane * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) dst[e] = from_f<T>(o[e] * inv);
}

template <int FMT, int D, bool P16> cudaError_t launch_rows(const PagedAttnArgs &a, cudaStream_t st)
{
    using C = RowsCfg<FMT, D>;
    static SmemLimit limit;
    const cudaError_t e = limit.raise((const void *)paged_attention_rows_kernel<FMT, D, P16>, C::SMEM);
    if (e != cudaSuccess) return e;
    return launch_kernel(paged_attention_rows_kernel<FMT, D, P16>, dim3(a.kv.nkv, a.rb.B, a.splits), dim3(R_THREADS), C::SMEM, st, 0, a);
}
template <int FMT> cudaError_t rows_by_dim(const PagedAttnArgs &a, cudaStream_t st)
{
    const bool p16 = a.kv.page % 16 == 0;
    if (a.kv.d == 128) return p16 ? launch_rows<FMT, 128, true>(a, st) : launch_rows<FMT, 128, false>(a, st);
    if (a.kv.d == 64) return p16 ? launch_rows<FMT, 64, true>(a, st) : launch_rows<FMT, 64, false>(a, st);
    return cudaErrorInvalidValue;
}

} // namespace

cudaError_t launch_paged_attention_rows(const PagedAttnArgs &a, cudaStream_t st)
{
    switch (a.kv.fmt) {
    case KV_BF16: return rows_by_dim<KV_BF16>(a, st);
    case KV_E4M3: return rows_by_dim<KV_E4M3>(a, st);
    case KV_INT8: return rows_by_dim<KV_INT8>(a, st);
    default: return cudaErrorInvalidValue;
    }
}

cudaError_t launch_paged_merge(const PagedAttnArgs &a, int q_bf16, cudaStream_t st)
{
    const dim3 grid((unsigned)(((long)a.rb.n_tokens * a.nq + 3) / 4));
    if (q_bf16 && a.kv.d == 128) return launch_kernel(paged_merge_kernel<bf16, 128>, grid, dim3(128), 0, st, 0, a);
    if (q_bf16 && a.kv.d == 64) return launch_kernel(paged_merge_kernel<bf16, 64>, grid, dim3(128), 0, st, 0, a);
    return cudaErrorInvalidValue;
}

} // namespace spd
