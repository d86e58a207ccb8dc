// Paged attention for few query rows (bf16): all rows of a (sequence, KV head) - new tokens times query heads per KV head -
// are the 8 or 16 columns of m16n8k16 MMAs, as in single-token steps and short drafts.
//
// Bound: the cache stream.  Keys and head dims are the MMA rows (S^T = K Q^T, O^T = V^T P^T), so that 8 query rows cost no
// padding: per 16 cached keys a warp issues head_dim / 8 MMAs for 8 query rows, a small part of an SM's issue slots at the
// rate HBM delivers the keys.  mma.sync and registers are enough, and the rest serves the loads and, for 8-bit caches, the
// widening of the codes:
//   - every warp works on its own 16-key blocks (j, j + 4, ..., or j + 8 in thread blocks of eight warps) with a private ring of
//     tiles, one TMA box each for K and V (page sizes that are multiples of 16; cp.async otherwise, into the same swizzled
//     layout): no block-wide barrier between the first load and the merge;
//   - the keys of a (sequence, KV head) are cut into ranges over thread blocks where there are few of them.  Up to 8 ranges
//     are one thread-block cluster that adds up its partial rows through shared memory; more go through the workspace and
//     paged_merge_kernel;
//   - the weights leave the first product with keys as rows and enter the second with keys as its k index: one 8 x 8
//     transpose (movmatrix) per 8 keys;
//   - 8-bit caches stay 8-bit up to the fragment registers.  A 16-byte shared-memory load gives a lane 16 consecutive head
//     dims of one key; any assignment of dims to the MMA's k index is right as long as Q uses the same one.  Likewise any
//     assignment of keys to score rows is right as long as V uses the same one: row 2i of eight keys is key 2i, row 2i + 1 is
//     key (2i) ^ 5, with which both the K loads (lanes = rows) and the V loads (lanes = row pairs) meet every shared-memory
//     bank once under the swizzle.
//   - K codes become float16 (exact, e4m3 up to a power of two; see half_of) and so does Q, scaled per row by a power of two to
//     below 2^15: the scaled row keeps bf16's 8 bits for everything down to 2^-29 of its largest value.  V codes become bfloat16
//     (exact), because the weights they meet carry the V scales and reach from 1 to where they vanish, a range that float16 does
//     not cover: e4m3 by moving sign, exponent and mantissa to bf16's places (the value times 2^-120) and one product, int8 as
//     128 + low 7 bits minus 128 or 256;
//   - weights are rounded to bf16.  With int8 scales, which are not powers of two, even a row's only weight is off, and the errors
//     came to 1.5 times that of the output's own rounding: there the rest of each weight is a second bf16 with products of its own
//     (32 sequences of 9 to 16 thousand tokens: 192 us, 182 without; the same for the other formats cost 2 to 8 % and
//     would take errors of 1.05 to 1.3 times to 1).
// Softmax: base 2, fp32, per warp; the accumulators follow the running maximum lazily (they are rescaled when it has grown by
// more than 2^8: weights stay below 2^8, where bf16 rounds as finely as at 1).
#include "gemm_tc.cuh"
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace spd {

namespace {

constexpr int BK16 = 16;

// RW warps per thread block; `stages` tiles per warp (TMA: as many as the launch has shared memory for)
template <int FMT, int D, int RW> struct RowsCfg {
    static constexpr bool Q8 = FMT != KV_BF16;
    static constexpr int RB = D * (Q8 ? 1 : 2);            // bytes of a cached row
    static constexpr int TR = RB > 128 ? 128 : RB;         // bytes of a tile row; 256-byte rows are two tiles
    static constexpr int TILE = BK16 * RB;                 // K or V of one block
    static constexpr int STAGES = RB == 256 ? 2 : RB == 128 ? 3 : 6; // with the most thread blocks resident
    static constexpr int MAX_STAGES = 8;
    static constexpr int MERGE = RW * 16 * (D + 4) * 4;    // the warps' partial rows, over the tiles
    // after the tiles: 16 K scales, 16 V scales per stage; a barrier per stage; abort flag; merged [16][2], weights [16][RW], rows' places [16], ranges' weights [16][8]
    static constexpr int off_sc(int st) { return RW * st * 2 * TILE > MERGE ? RW * st * 2 * TILE : (MERGE + 1023) / 1024 * 1024; }
    static constexpr int off_bar(int st) { return off_sc(st) + (Q8 ? RW * st * 128 : 0); }
    static constexpr int off_pml(int st) { return (off_bar(st) + RW * st * 8 + 16 + 15) / 16 * 16; }
    static constexpr int smem(int st) { return off_pml(st) + 128 + 16 * RW * 4 + 128 + 16 * PAGED_MAX_CLUSTER * 4 + 1024; } // + alignment slack
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
// 64 bytes, both sides 16-byte aligned
__device__ __forceinline__ void bulk64(uint32_t dst, const void *src, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 64, [%2];" ::"r"(dst), "l"(src), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a)
{
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ float lds_f(uint32_t a)
{
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool F16>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
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

// Two K codes of a word -> float16x2.  int8: codes with the sign bit flipped (code + 128), bytes 0, 1 or (SECOND) 2, 3, under the
// exponent of 1024, minus 1152.  e4m3: bytes 0, 2 or 1, 3, sign, exponent and mantissa moved to float16's places: the value
// times E4M3_UNIT = 2^-8, exactly (64 sequences of ragged lengths: 33.3 us, with a conversion instruction per pair 34.1).
constexpr float E4M3_UNIT = 0x1p-8f;
template <int FMT, bool SECOND> __device__ __forceinline__ uint32_t half_of(uint32_t w)
{
    if (FMT == KV_E4M3) return SECOND ? ((w >> 1) & 0x3f803f80u) | (w & 0x80008000u) : ((w << 7) & 0x3f803f80u) | ((w << 8) & 0x80008000u);
    const uint32_t x = __byte_perm(w, 0x64646464u, SECOND ? 0x4342 : 0x4140);
    const __half2 v = __hsub2(*(const __half2 *)&x, __half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480)));
    return *(const uint32_t *)&v;
}

// keys t that a row at position pos (-1: no row) sees
__device__ __forceinline__ bool sees(int t, int pos, int window, int sinks) { return t <= pos && (!window || t > pos - window || t < sinks); }

// key of score row c (0-7) of eight
__device__ __forceinline__ int key_of(int c) { return c & 1 ? (c & 6) ^ 5 : c; }

// NR: groups of 8 query rows
template <int FMT, int D, int NR, int RW, bool TMA>
__global__ void __launch_bounds__(32 * RW, RW == 8 ? 1 : NR == 1 && FMT != KV_BF16 ? 4 : 3) paged_attention_rows_kernel(const __grid_constant__ TcMap k_map, const __grid_constant__ TcMap v_map,
                                                                            const __grid_constant__ PagedAttnArgs a)
{
    using C = RowsCfg<FMT, D, RW>;
    constexpr bool Q8 = C::Q8;
    constexpr int MT = D / 16, KS = D / 16, R_THREADS = 32 * RW;
    const int ST = TMA ? a.stages : C::STAGES;
    extern __shared__ uint8_t rows_raw[];
    uint8_t *gen = rows_raw + ((1024u - (tc::smem_u32(rows_raw) & 1023u)) & 1023u);
    const uint32_t base = tc::smem_u32(gen);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
    const uint32_t ring = base + warp * ST * 2 * C::TILE, ring_sc = base + C::off_sc(ST) + warp * ST * 128, bars = base + C::off_bar(ST) + warp * ST * 8;
    volatile int *abort_flag = (volatile int *)(gen + C::off_bar(ST) + RW * ST * 8);
    if (threadIdx.x == 0) stamp_entry(a.stamp);
    pdl_launch_dependents();
    if (TMA) {
        if (lane == 0) {
            for (int s = 0; s < ST; ++s) tc::mbar_init(bars + 8 * s, 1);
            if (warp == 0) *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
        }
        __syncthreads();
    }
    pdl_wait();
    const int kvh = blockIdx.x, b = blockIdx.y, split = blockIdx.z;
    int row0, n_new, len;
    if (!batch_row(a.rb, b, a.max_new, a.max_context, row0, n_new, len, a.err)) return; // the same for a whole cluster
    const int rows = n_new * a.group; // <= 8 NR
    const int kv_len = len + n_new, pos_max = kv_len - 1;
    // blocks of 16 keys that hold a key some row sees: sinks, then the window of the first query onwards
    const int lo_min = a.window ? max(0, len - a.window + 1) : 0, first = lo_min / BK16;
    const int n_sink = min((min(a.sinks, lo_min) + BK16 - 1) / BK16, first);
    const int n_blocks = n_sink + (kv_len + BK16 - 1) / BK16 - first;
    // short sequences are cut into fewer ranges, of at least 8 blocks
    const int splits = min(a.splits, (n_blocks + 7) / 8);
    const int per = splits > 1 ? n_blocks / splits : n_blocks, extra = n_blocks - per * splits; // the first `extra` ranges get one more
    const int j_begin = split < splits ? split * per + min(split, extra) : 0;
    const int j_end = split < splits ? j_begin + per + (split < extra ? 1 : 0) : 0;

    const int32_t *bt = a.rb.table + (long)b * a.rb.max_pages;
    const int bpp = a.kv.page / BK16; // TMA: blocks per page
    auto block_of = [&](int j) { return j < n_sink ? j : first + (j - n_sink); };
    auto row_valid = [&](int t) { return t < kv_len && (t >= lo_min || t < a.sinks); };
    // every row sees every key of the 16 from t0 on
    auto seen_by_all = [&](int t0) { return t0 + 15 <= len && (!a.window || t0 > pos_max - a.window || t0 + 15 < a.sinks); };
    auto lookup = [&](int t) { // cached row of key t, or -1
        const int pi = t / a.kv.page, page = bt[pi];
        if (page < 0 || page >= a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); return -1L; }
        return ((long)page * a.kv.nkv + kvh) * a.kv.page + (t - pi * a.kv.page);
    };
    // TMA: cached row of the first key of block j (a bad page id: page 0, with the error bit); else of this lane's key (lane & 15), or -1
    auto row_of = [&](int blk, int page) -> long {
        if (page < 0 || page >= a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); page = 0; }
        return ((long)page * a.kv.nkv + kvh) * a.kv.page + (bpp == 1 ? 0 : blk % bpp * BK16);
    };
    auto lookup_block = [&](int j) -> long {
        const int blk = block_of(j);
        if (TMA) return row_of(blk, bt[bpp == 1 ? blk : blk / bpp]);
        const int t = blk * BK16 + (lane & 15);
        return row_valid(t) ? lookup(t) : -1L;
    };
    // 16-byte chunk c of row r of a tile pair / tile, where the copies put it
    auto at = [&](int r, int c) -> uint32_t {
        if (C::RB == 256) return (c >> 3) * (BK16 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
        if (C::RB == 128) return r * 128 + ((c ^ (r & 7)) << 4);
        return r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
    };
    auto load_block = [&](int stage, long where) {
        const uint32_t sK = ring + stage * 2 * C::TILE, sV = sK + C::TILE, sS = ring_sc + stage * 128;
        if (TMA) {
            if (lane == 0) {
                const uint32_t bar = bars + 8 * stage;
                tc::mbar_expect_tx(bar, 2 * C::TILE + (Q8 ? 128 : 0));
                tc::tma_load_3d(sK, (const CUtensorMap *)&k_map, 0, (int)where, 0, bar);
                tc::tma_load_3d(sV, (const CUtensorMap *)&v_map, 0, (int)where, 0, bar);
                if (Q8) { bulk64(sS, a.kv.ks + where, bar); bulk64(sS + 64, a.kv.vs + where, bar); }
            }
        } else {
            constexpr int CPR = C::RB / 16, RPI = 32 / CPR; // chunks per row, rows per instruction
            const int c = lane % CPR;
#pragma unroll
            for (int i = 0; i < BK16 / RPI; ++i) {
                const int r = i * RPI + lane / CPR;
                const long row = __shfl_sync(0xffffffffu, where, r);
                const long off = row >= 0 ? row * C::RB + c * 16 : 0;
                cp16(sK + at(r, c), (const uint8_t *)a.kv.k + off, row >= 0);
                cp16(sV + at(r, c), (const uint8_t *)a.kv.v + off, row >= 0);
            }
            if (Q8) cp4(sS + lane * 4, (lane < 16 ? a.kv.ks : a.kv.vs) + (where >= 0 ? where : 0), where >= 0);
        }
    };

    const int n_mine = (j_end - j_begin - warp + RW - 1) / RW; // blocks j_begin + warp, + RW, ...
    auto mine = [&](int i) { return j_begin + warp + i * RW; };
    // The tiles and Q are asked for together: page ids of the first tiles (one lane each), Q as it lies, then the tiles.
    int first_page = 0;
    if (TMA) {
        const int blk = block_of(j_begin + warp + lane * RW);
        if (lane < ST && lane < n_mine) first_page = bt[bpp == 1 ? blk : blk / bpp];
    }
    uint4 q_raw[NR][D / 32];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const int r = g + 8 * n;
        const bool live = r < rows;
        const int i = live ? r / a.group : 0, head = live ? r - i * a.group : 0;
        const bf16 *qp = (const bf16 *)a.q + (long)(row0 + i) * a.q_stride + (long)(kvh * a.group + head) * D;
#pragma unroll
        for (int m = 0; m < D / 32; ++m) { // a 16-byte K chunk is 8 dims (bf16) or 16 (codes)
            const int dim = Q8 ? 64 * (m >> 1) + 16 * t4 + 8 * (m & 1) : 32 * m + 8 * t4;
            q_raw[n][m] = live ? *(const uint4 *)(qp + dim) : make_uint4(0, 0, 0, 0);
        }
    }
    for (int s = 0; s < ST; ++s) {
        if (TMA) {
            const int page = __shfl_sync(0xffffffffu, first_page, s & 31);
            if (s < n_mine) load_block(s, row_of(block_of(mine(s)), page));
        } else {
            if (s < n_mine) load_block(s, lookup_block(mine(s)));
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    }
    long where = ST < n_mine ? lookup_block(mine(ST)) : 0;

    // Q fragments (column g of a group of 8 rows); rows beyond the tile's are zero.  qs: what turns the scores of this lane's
    // columns 2 t4 and 2 t4 + 1 into base-2 units
    uint32_t qf[NR][KS][2];
    float qs[NR][2];
    int pos[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        uint4 (&u)[D / 32] = q_raw[n];
        float my_qs = a.scale_log2;
        if (Q8) {
            uint32_t top = 0; // largest magnitude's bits
#pragma unroll
            for (int m = 0; m < D / 32; ++m) {
                const uint32_t w[4] = {u[m].x, u[m].y, u[m].z, u[m].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max(top, max(w[e] & 0x7fffu, (w[e] >> 16) & 0x7fffu));
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int ex = max((int)(top >> 7), 27) - 127;                         // 2^ex <= largest < 2^(ex + 1), ex >= -100
            const float f = __uint_as_float((uint32_t)(127 + 14 - ex) << 23);      // to [2^14, 2^15)
            my_qs *= __uint_as_float((uint32_t)(127 - 14 + ex) << 23) * (FMT == KV_E4M3 ? 1.f / E4M3_UNIT : 1.f);
#pragma unroll
            for (int m = 0; m < D / 32; ++m) {
                const uint32_t w[4] = {u[m].x, u[m].y, u[m].z, u[m].w};
                uint32_t x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __half2 v = __floats2half2_rn(__uint_as_float(w[e] << 16) * f, __uint_as_float(w[e] & 0xffff0000u) * f);
                    x[e] = *(const uint32_t *)&v;
                }
                u[m] = make_uint4(x[0], x[1], x[2], x[3]);
            }
        }
#pragma unroll
        for (int m = 0; m < D / 32; ++m) {
            if (FMT == KV_E4M3) { // as half_of pairs the codes
                qf[n][2 * m][0] = __byte_perm(u[m].x, u[m].y, 0x5410); qf[n][2 * m][1] = __byte_perm(u[m].x, u[m].y, 0x7632);
                qf[n][2 * m + 1][0] = __byte_perm(u[m].z, u[m].w, 0x5410); qf[n][2 * m + 1][1] = __byte_perm(u[m].z, u[m].w, 0x7632);
            } else {
                qf[n][2 * m][0] = u[m].x; qf[n][2 * m][1] = u[m].y; qf[n][2 * m + 1][0] = u[m].z; qf[n][2 * m + 1][1] = u[m].w;
            }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = 8 * n + 2 * t4 + e;
            pos[n][e] = c < rows ? len + c / a.group : -1;
            qs[n][e] = __shfl_sync(0xffffffffu, my_qs, (2 * t4 + e) * 4);
        }
    }

    // where this lane reads in a stage; chunk bits above the lane's own are XORs, rows + 8 a fixed distance
    const uint32_t lane_k = at(key_of(g), t4);
    const int vc = lane & 7;
    const uint32_t lane_v0 = Q8 ? (D == 128 ? at(key_of(2 * t4), g) : at(key_of(2 * t4), g >> 1) + (g & 1) * 8) : at(key_of(vc) + (lane & 8), lane >> 4);
    const uint32_t lane_v1 = Q8 ? (D == 128 ? at(key_of(2 * t4 + 1), g) : at(key_of(2 * t4 + 1), g >> 1) + (g & 1) * 8) : 0u;
    const uint32_t lane_s = key_of(g) * 4, c128 = widen_const();

    float o[NR][MT][4];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int i = 0; i < MT; ++i) { o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f; }
    }
    float m_used[NR][2], l[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) { m_used[n][0] = m_used[n][1] = -INFINITY; l[n][0] = l[n][1] = 0.f; }
    bool dirty = false; // a NaN or infinity of V was taken out of a block that not every row sees
    bool ok = true;
    int stage = 0, phase = 0;
    for (int it = 0; it < n_mine; ++it) {
        if (TMA) {
            ok = tc::mbar_wait(bars + 8 * stage, phase, a.err, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
        } else {
            asm volatile("cp.async.wait_group %0;" ::"n"(C::STAGES - 1) : "memory");
            __syncwarp();
        }
        const uint32_t sK = ring + stage * 2 * C::TILE, sV = sK + C::TILE, sS = ring_sc + stage * 128;
        const int t0 = block_of(mine(it)) * BK16;
        float s[NR][4], ks[2], vs[2]; // rows g and g + 8
#pragma unroll
        for (int n = 0; n < NR; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
        if (!Q8) {
#pragma unroll
            for (int m = 0; m < D / 32; ++m) {
                const uint32_t p = ((sK + lane_k) ^ ((m & 1) << 6)) + (m >> 1) * (BK16 * 128);
                const uint4 u = lds128(p), w = lds128(p + 8 * C::TR);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    mma16816<false>(s[n], u.x, w.x, u.y, w.y, qf[n][2 * m][0], qf[n][2 * m][1]);
                    mma16816<false>(s[n], u.z, w.z, u.w, w.w, qf[n][2 * m + 1][0], qf[n][2 * m + 1][1]);
                }
            }
        } else {
#pragma unroll
            for (int m = 0; m < D / 64; ++m) {
                const uint32_t p = (sK + lane_k) ^ (m << 6);
                const uint4 u0 = lds128(p), u1 = lds128(p + 8 * C::TR);
                const uint32_t w0[4] = {u0.x, u0.y, u0.z, u0.w}, w1[4] = {u1.x, u1.y, u1.z, u1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t x0 = FMT == KV_INT8 ? w0[i] ^ 0x80808080u : w0[i], x1 = FMT == KV_INT8 ? w1[i] ^ 0x80808080u : w1[i];
                    const uint32_t a0 = half_of<FMT, false>(x0), a1 = half_of<FMT, false>(x1), a2 = half_of<FMT, true>(x0), a3 = half_of<FMT, true>(x1);
#pragma unroll
                    for (int n = 0; n < NR; ++n) mma16816<true>(s[n], a0, a1, a2, a3, qf[n][4 * m + i][0], qf[n][4 * m + i][1]);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) { ks[h] = lds_f(sS + lane_s + h * 32); vs[h] = lds_f(sS + lane_s + 64 + h * 32); }
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] *= ks[e >> 1];
            }
        }
        const bool all_seen = seen_by_all(t0);
        if (!all_seen) { // masked scores are -inf whatever was computed
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (!sees(t0 + 8 * (e >> 1) + key_of(g), pos[n][e & 1], a.window, a.sinks)) s[n][e] = -INFINITY;
            }
        }
        float mx[NR][2];
        bool grow = false;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float m = fmaxf(s[n][e], s[n][2 + e]);
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                mx[n][e] = m * qs[n][e];
                grow |= mx[n][e] > m_used[n][e] + 8.f; // first keys of a row included (-inf)
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
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) { o[n][i][0] *= f[0]; o[n][i][1] *= f[1]; o[n][i][2] *= f[0]; o[n][i][3] *= f[1]; }
            }
        }
        uint32_t pf[NR][2], pl[NR][2]; // pl: what rounding left, int8
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float mb = m_used[n][e & 1] == -INFINITY ? 0.f : m_used[n][e & 1];
                p[e] = ex2(fmaf(s[n][e], qs[n][e & 1], -mb));
                l[n][e & 1] += p[e];
                if (Q8) p[e] *= vs[e >> 1];
            }
            if (Q8 && !all_seen) { // 0 times the scale of a masked key, which may be anything
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (s[n][e] == -INFINITY) p[e] = 0.f;
            }
            pf[n][0] = transpose8x8(pack(p[0], p[1]));
            pf[n][1] = transpose8x8(pack(p[2], p[3]));
            if (FMT == KV_INT8) {
                auto left = [](float lo, float hi) { // lo, hi minus their bf16s
                    const uint32_t w = pack(lo, hi);
                    return pack(lo - __uint_as_float(w << 16), hi - __uint_as_float(w & 0xffff0000u));
                };
                pl[n][0] = transpose8x8(left(p[0], p[1]));
                pl[n][1] = transpose8x8(left(p[2], p[3]));
            }
        }
        if constexpr (!Q8) {
            if (!all_seen) {
                // 0 * NaN would reach rows that do not see the key: take non-finite values out here, give them back at the end
#pragma unroll
                for (int i = 0; i < C::TILE / 512; ++i) {
                    const uint32_t p = sV + (i * 32 + lane) * 16;
                    const uint4 u = lds128(p);
                    uint32_t w[4] = {u.x, u.y, u.z, u.w};
                    bool bad = false;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; bad = true; }
                        if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; bad = true; }
                    }
                    if (bad) { sts128(p, make_uint4(w[0], w[1], w[2], w[3])); dirty = true; }
                }
                tc::fence_proxy_async(); // the tile is refilled by the async proxy
                __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                uint32_t vf[4]; // (keys 0-7, dims 0-7), (keys 8-15, dims 0-7), (keys 0-7, dims 8-15), (keys 8-15, dims 8-15)
                ldsm4t(vf, ((sV + lane_v0) ^ ((i & 3) << 5)) + (i >> 2) * (BK16 * 128));
#pragma unroll
                for (int n = 0; n < NR; ++n) mma16816<false>(o[n][i], vf[0], vf[2], vf[1], vf[3], pf[n][0], pf[n][1]);
            }
        } else {
            constexpr int W = D / 32; // words per key and lane: dims g * D / 8 ..
            uint32_t v[4][W];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t p = sV + (q & 1 ? lane_v1 : lane_v0) + (q >> 1) * 8 * C::TR;
                if (W == 4) {
                    const uint4 u = lds128(p);
                    v[q][0] = u.x; v[q][1] = u.y; v[q][2 % W] = u.z; v[q][3 % W] = u.w;
                } else {
                    const uint2 u = lds64(p);
                    v[q][0] = u.x; v[q][1] = u.y;
                }
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                // bytes (k0.0, k0.1, k1.0, k1.1): even bytes = dim 0 of keys (k0, k1), odd bytes = dim 1
                const uint32_t x0 = __byte_perm(v[0][w], v[1][w], 0x5410), x1 = __byte_perm(v[2][w], v[3][w], 0x5410);
                const uint32_t y0 = __byte_perm(v[0][w], v[1][w], 0x7632), y1 = __byte_perm(v[2][w], v[3][w], 0x7632);
                const uint32_t a0 = even2<FMT>(x0, c128), a1 = odd2<FMT>(x0, c128), a2 = even2<FMT>(x1, c128), a3 = odd2<FMT>(x1, c128);
                const uint32_t b0 = even2<FMT>(y0, c128), b1 = odd2<FMT>(y0, c128), b2 = even2<FMT>(y1, c128), b3 = odd2<FMT>(y1, c128);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    mma16816<false>(o[n][2 * w], a0, a1, a2, a3, pf[n][0], pf[n][1]);
                    mma16816<false>(o[n][2 * w + 1], b0, b1, b2, b3, pf[n][0], pf[n][1]);
                    if (FMT == KV_INT8) {
                        mma16816<false>(o[n][2 * w], a0, a1, a2, a3, pl[n][0], pl[n][1]);
                        mma16816<false>(o[n][2 * w + 1], b0, b1, b2, b3, pl[n][0], pl[n][1]);
                    }
                }
            }
        }
        __syncwarp(); // every lane has read the stage
        if (it + ST < n_mine) {
            load_block(stage, where);
            if (it + ST + 1 < n_mine) where = lookup_block(mine(it + ST + 1));
        }
        if (!TMA) asm volatile("cp.async.commit_group;" ::: "memory");
        if (++stage == ST) { stage = 0; phase ^= 1; }
    }
    if (!TMA) asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (TMA && !ok) { // gave up: the copies still in flight must land before the memory is reused
        for (int it = 0; it < ST; ++it) {
            const long long t_end = clock64() + tc::WAIT_LIMIT_CYCLES;
            while (!tc::mbar_try_wait(bars + 8 * stage, phase) && clock64() < t_end) {}
            if (++stage == ST) { stage = 0; phase ^= 1; }
        }
    }

    // the warps' partial rows, merged through shared memory (the rings are done with)
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 4);
            l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 8);
            l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 16);
        }
    }
    const int any_dirty = __syncthreads_or(dirty);
    float *mo = (float *)gen, *ml = mo + RW * 16 * (D + 2); // [warp][16][D + 2], [warp][16][2]
    float *pml = (float *)(gen + C::off_pml(ST));
#pragma unroll
    for (int n = 0; n < NR; ++n) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = 8 * n + 2 * t4 + e;
            if (r < rows) {
                float *dst = mo + (warp * 16 + r) * (D + 2);
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    if (!Q8) { dst[16 * i + g] = o[n][i][e]; dst[16 * i + 8 + g] = o[n][i][2 + e]; }
                    else *(float2 *)(dst + g * (D / 8) + 2 * i) = make_float2(o[n][i][e], o[n][i][2 + e]); // MMA row g: dims g D/8 + 2i, row g + 8: + 1
                }
                if (g == 0) { ml[(warp * 16 + r) * 2] = m_used[n][e]; ml[(warp * 16 + r) * 2 + 1] = l[n][e]; }
            }
        }
    }
    __syncthreads();
    // per row: the warps' weights relative to the block's maximum, its maximum and sum, where the row goes
    const bool clustered = a.splits > 1 && !a.part_o;
    const long plane = (long)a.rb.n_tokens * a.nq;
    float *wt = pml + 32;                // [16][RW]
    long *dst_of = (long *)(wt + 16 * RW); // [16]
    float *cw = (float *)(dst_of + 16);    // [16][ranges of a cluster]
    if (threadIdx.x < rows) {
        const int r = threadIdx.x, i = r / a.group, head = kvh * a.group + r - i * a.group;
        float m = -INFINITY, den = 0.f;
#pragma unroll
        for (int w = 0; w < RW; ++w) m = fmaxf(m, ml[(w * 16 + r) * 2]);
#pragma unroll
        for (int w = 0; w < RW; ++w) {
            const float mw = ml[(w * 16 + r) * 2], f = mw == -INFINITY ? 0.f : ex2(mw - m);
            wt[r * RW + w] = f;
            den = fmaf(ml[(w * 16 + r) * 2 + 1], f, den);
        }
        if (den != den) m = fmaxf(m, 0.f); // scores that are all NaN leave no maximum: not an empty range
        pml[2 * r] = m;
        pml[2 * r + 1] = den;
        dst_of[r] = a.part_o ? (long)split * plane + (long)(row0 + i) * a.nq + head : (long)(row0 + i) * a.o_stride + (long)head * D;
    }
    __syncthreads();
#pragma unroll 4
    for (int idx = threadIdx.x; idx < rows * (D / 2); idx += R_THREADS) {
        const int r = idx / (D / 2), c = idx % (D / 2) * 2;
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int w = 0; w < RW; ++w) {
            const float f = wt[r * RW + w];
            const float2 v = *(const float2 *)(mo + (w * 16 + r) * (D + 2) + c);
            x = fmaf(v.x, f, x);
            y = fmaf(v.y, f, y);
        }
        if (!Q8 && any_dirty) { // the values taken out above, for the rows that see them
            const int p = len + r / a.group;
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
            const float inv = inverse_sum(pml[2 * r + 1]);
            *(uint32_t *)((bf16 *)a.out + dst_of[r] + c) = pack(x * inv, y * inv);
        } else if (clustered) // only this thread reads (r, c) of the warps' partials: the first one's place keeps the sum
            *(float2 *)(mo + r * (D + 2) + c) = make_float2(x, y);
        else {
            const float m = pml[2 * r];
            if (m != -INFINITY) *(float2 *)(a.part_o + dst_of[r] * D + c) = make_float2(x, y);
            if (c == 0) *(float2 *)(a.part_ml + dst_of[r] * 2) = make_float2(m, pml[2 * r + 1]);
        }
    }
    if (clustered) {
        tc::cluster_sync();
        const uint32_t mo_addr = base, pml_addr = base + C::off_pml(ST);
        auto peer2 = [](uint32_t addr, int rank) {
            float2 v;
            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(tc::mapa_shared(addr, rank)) : "memory");
            return v;
        };
        // per row: the ranges' weights, with the sum's reciprocal in them (over the warps' weights, which have been used)
        if (threadIdx.x < rows) {
            const int r = threadIdx.x;
            float2 q[PAGED_MAX_CLUSTER];
            float m = -INFINITY, den = 0.f;
#pragma unroll
            for (int s = 0; s < PAGED_MAX_CLUSTER; ++s) q[s] = s < splits ? peer2(pml_addr + 8 * r, s) : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int s = 0; s < PAGED_MAX_CLUSTER; ++s) m = fmaxf(m, q[s].x);
#pragma unroll
            for (int s = 0; s < PAGED_MAX_CLUSTER; ++s) {
                q[s].x = q[s].x == -INFINITY ? 0.f : ex2(q[s].x - m);
                den = fmaf(q[s].y, q[s].x, den);
            }
            const float inv = inverse_sum(den);
#pragma unroll
            for (int s = 0; s < PAGED_MAX_CLUSTER; ++s)
                if (s < splits) cw[r * PAGED_MAX_CLUSTER + s] = q[s].x * inv;
        }
        __syncthreads();
        for (int idx = split + a.splits * (int)threadIdx.x; idx < rows * (D / 2); idx += a.splits * R_THREADS) {
            const int r = idx / (D / 2), c = idx % (D / 2) * 2;
            float2 v[PAGED_MAX_CLUSTER];
            float x = 0.f, y = 0.f;
#pragma unroll
            for (int s = 0; s < PAGED_MAX_CLUSTER; ++s) v[s] = s < splits ? peer2(mo_addr + (r * (D + 2) + c) * 4, s) : make_float2(0.f, 0.f);
#pragma unroll
            for (int s = 0; s < PAGED_MAX_CLUSTER; ++s) {
                const float f = s < splits ? cw[r * PAGED_MAX_CLUSTER + s] : 0.f;
                x = fmaf(v[s].x, f, x);
                y = fmaf(v[s].y, f, y);
            }
            *(uint32_t *)((bf16 *)a.out + dst_of[r] + c) = pack(x, y);
        }
        tc::cluster_sync(); // no block exits while a peer still reads its shared memory
    }
    if (threadIdx.x == 0) stamp_exit(a.stamp);
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
    int before = a.rb.cu ? 0 : t / a.rb.uniform + 1;
    for (int i0 = 0; a.rb.cu && i0 <= a.rb.B; i0 += 32) {
        const unsigned mk = __ballot_sync(0xffffffffu, i0 + lane <= a.rb.B && a.rb.cu[i0 + lane] <= t);
        before += __popc(mk);
        if (mk != 0xffffffffu) break;
    }
    if (before < 1 || before > a.rb.B) return;
    int row0, n_new, len;
    if (!batch_row(a.rb, before - 1, a.max_new, a.max_context, row0, n_new, len, a.err)) return;
    // the ranges' maxima and sums in the lanes (two each), then their rows eight at a time
    float mr[2], wr[2], den = 0.f;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int s = lane + 32 * k;
        const float2 v = s < a.splits ? __ldcg((const float2 *)(a.part_ml + ((long)s * plane + w) * 2)) : make_float2(-INFINITY, 0.f);
        mr[k] = v.x; wr[k] = v.y;
    }
    const float m = warp_max(fmaxf(mr[0], mr[1]));
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float f = mr[k] == -INFINITY ? 0.f : ex2(mr[k] - m); // an empty range has no rows
        den = fmaf(wr[k], f, den);
        wr[k] = f;
    }
    den = warp_sum(den);
    float o[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) o[e] = 0.f;
    for (int s0 = 0; s0 < a.splits; s0 += 8) {
        float v[8][VEC], f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int s = s0 + k;
            f[k] = __shfl_sync(0xffffffffu, s < 32 ? wr[0] : wr[1], s & 31);
            const bool empty = __shfl_sync(0xffffffffu, s < 32 ? mr[0] : mr[1], s & 31) == -INFINITY || s >= a.splits;
            const float *p = a.part_o + ((long)(empty ? 0 : s) * plane + w) * D + lane * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[k][e] = empty ? 0.f : __ldcg(p + e);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) o[e] = fmaf(v[k][e], f[k], o[e]);
        }
    }
    const float inv = inverse_sum(den);
    T *dst = (T *)a.out + (long)t * a.o_stride + (long)head * D + lane * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) dst[e] = from_f<T>(o[e] * inv);
    if (lane == 0) stamp_exit(a.stamp); // the slot's start is the ranges' launch
}

template <int FMT, int D, int NR, int RW, bool TMA>
cudaError_t launch_rows(PagedAttnArgs a, const TcMap &km, const TcMap &vm, cudaStream_t st)
{
    using C = RowsCfg<FMT, D, RW>;
    static SmemLimit limit;
    // deep rings where few thread blocks share an SM
    a.stages = C::STAGES;
    const long per_sm = ((long)a.kv.nkv * a.rb.B * a.splits + sm_count() - 1) / sm_count();
    while (TMA && a.stages < C::MAX_STAGES && C::smem(a.stages + 1) * per_sm <= 220 * 1024) ++a.stages;
    cudaError_t e = limit.raise((const void *)paged_attention_rows_kernel<FMT, D, NR, RW, TMA>,
                                C::smem(C::MAX_STAGES) < 227 * 1024 ? C::smem(C::MAX_STAGES) : 227 * 1024);
    if (e != cudaSuccess) return e;
    return launch_kernel_z(paged_attention_rows_kernel<FMT, D, NR, RW, TMA>, dim3(a.kv.nkv, a.rb.B, a.splits), dim3(32 * RW), C::smem(a.stages), st,
                           a.part_o ? 1 : a.splits, km, vm, a);
}
template <int FMT, int D, int NR> cudaError_t rows_by_copy(const PagedAttnArgs &a, cudaStream_t st)
{
    // 16-key blocks as TMA boxes: they lie in one page, row numbers fit a coordinate, scales start on 16 bytes
    TcMap km{}, vm{};
    const long rows = (long)a.kv.n_pages * a.kv.nkv * a.kv.page;
    const int es = FMT == KV_BF16 ? 2 : 1;
    if (a.kv.page % BK16 == 0 && rows <= 0x7fffffffL && !(((uintptr_t)a.kv.ks | (uintptr_t)a.kv.vs) & 15) &&
        make_cache_map(&km, a.kv.k, rows, D, es) == 0 && make_cache_map(&vm, a.kv.v, rows, D, es) == 0) {
        if ((long)a.kv.nkv * a.rb.B * a.splits <= sm_count()) return launch_rows<FMT, D, NR, 8, true>(a, km, vm, st);
        return launch_rows<FMT, D, NR, 4, true>(a, km, vm, st);
    }
    return launch_rows<FMT, D, 2, 4, false>(a, km, vm, st);
}
template <int FMT, int D> cudaError_t rows_by_count(const PagedAttnArgs &a, cudaStream_t st)
{
    return a.max_new * a.group <= 8 ? rows_by_copy<FMT, D, 1>(a, st) : rows_by_copy<FMT, D, 2>(a, st);
}
template <int FMT> cudaError_t rows_by_dim(const PagedAttnArgs &a, cudaStream_t st)
{
    if (a.kv.d == 128) return rows_by_count<FMT, 128>(a, st);
    if (a.kv.d == 64) return rows_by_count<FMT, 64>(a, st);
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
    switch (a.kv.d) {
    case 128: return q_bf16 ? launch_kernel(paged_merge_kernel<bf16, 128>, grid, dim3(128), 0, st, 0, a) : launch_kernel(paged_merge_kernel<float, 128>, grid, dim3(128), 0, st, 0, a);
    case 64: return q_bf16 ? launch_kernel(paged_merge_kernel<bf16, 64>, grid, dim3(128), 0, st, 0, a) : launch_kernel(paged_merge_kernel<float, 64>, grid, dim3(128), 0, st, 0, a);
    case 32: return q_bf16 ? launch_kernel(paged_merge_kernel<bf16, 32>, grid, dim3(128), 0, st, 0, a) : launch_kernel(paged_merge_kernel<float, 32>, grid, dim3(128), 0, st, 0, a);
    default: return cudaErrorInvalidValue;
    }
}

} // namespace spd
