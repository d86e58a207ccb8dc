// Paged attention for many query rows (bf16, head_dim 64 or 128) on the tcgen05 tensor cores: chunks of prompts on a cached
// context, drafts of many tokens, grouped-query batches.
//
// The rows of a (sequence, KV head) are packed: row r = new token r / group, query head r % group of the KV head, so that the
// query heads of a group share every K/V tile.  A thread block serves one tile of 128 rows, and two blocks share an SM (each 256
// columns of tensor memory and 110 KB of shared memory): one's products run under the other's softmax, start and end.  One block
// with two tiles that shared their K/V tiles and took turns waited for itself at both ends of short contexts (window of 1024: 181
// against 141 us); on long ones the two forms are within what the clock changes (2048 tokens on 14336, 64 heads: 1168 us against 1041
// when they were compared, and 1090 to 1190 since for the form that was kept).
// Per tile of 128 keys and 128 rows:
//   S = Q K^T      tcgen05.mma, Q and K as K-major 128B-swizzled tiles, accumulator in tensor memory
//   P = softmax    thread = row and half of the keys: maximum (joined with the other half's), then the weights, which go back
//                  to tensor memory as bf16 over the scores already read
//   O += P V       tcgen05.mma with P read from tensor memory and V as the MN-major operand ([key][dim] rows as they are
//                  stored); O stays in tensor memory and is rescaled there only when the row maximum has grown by more than 2^8
// Tensor memory: S and P at column 0, O at 128.
// Warps: 0-7 softmax (two threads per row: one per row left the schedulers waiting on their own instructions' latencies), then the
// load warps, then one that issues the MMAs.  There is one K and one V slot; K is free once S is computed.  bf16 pages of a multiple
// of 16 tokens arrive by TMA, one box per 16 keys and 64 dims (a second load warp looks after V, see below); bf16 pages of other
// sizes by four load warps; 8-bit pages by eight (four took 212 us where eight take 187), which widen the
// codes to bf16 on the way into shared memory.  The pairs that widening a 32-bit word gives are (0, 2) and (1, 3) of its four
// codes: the head dims of Q, K and V all sit in that order, and the output is put right when it is stored.  Row scales multiply
// the scores (K) and the weights (V) in fp32.  A weight that carries an int8 row's scale is off by up to 2^-8 even where it is the
// row's only one, and such errors came to 1.5 times the output's own rounding: there what rounding left is a second bf16 with a
// product of its own (ragged chunks of up to 700 tokens on up to 1000, 40 heads: 243 us; e4m3, whose scales are powers of two and
// whose weights are single bf16s, 187; bf16 124).
// A key that only some of the rows see may hold anything in V: tiles with such keys have their NaNs and infinities taken out of
// shared memory before the product, and rows that do see them get them back at the end.
// Key tiles can be cut into ranges over thread blocks (fp32 partial rows in the workspace, paged_merge_kernel).
#include "gemm_tc.cuh"
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace spd {

namespace {

using namespace tc;

constexpr int TQ = 128, TK = 128, HALF = 128 * 128; // bytes of [128 rows][64 bf16]
// named barriers: each always with the same number of threads, and no arrival left over
enum { BAR_OUT = 1, BAR_LOAD = 2, BAR_PAIR = 4 }; // BAR_PAIR .. + 3

template <int D> struct TcCfg {
    static constexpr int TILE = 128 * D * 2;
    static constexpr int OFF_Q = 0, OFF_K = TILE, OFF_V = OFF_K + TILE;
    static constexpr int OFF_SC = OFF_V + TILE;                //  [8][256] K and V scales of a tile
    static constexpr int OFF_ROW = OFF_SC + 8 * 1024;          // [2][128] cached rows of a tile's keys
    static constexpr int OFF_BAR = OFF_ROW + 2 * 1024;
    static constexpr int OFF_RED = OFF_BAR + 512;              // [2 parities][2 halves][128] maxima; sums at the end
    static constexpr int SMEM = OFF_RED + 2048 + 1024;         // + alignment slack
};

// Shared-memory descriptors in two words: 128B-swizzled tiles, 8-row groups 1024 bytes apart.  Word 0 holds the address / 16 (and,
// for the MN-major V tile, the distance of its 64-dim blocks), so a step inside a tile is an addition to it.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lead) { return ((addr & 0x3FFFFu) >> 4) | (lead << 16); }
// The products are issued by one elected lane of a converged warp whose operands are the same in all lanes: they then live in
// uniform registers, and the issue loop keeps ahead of the tensor cores (with a single-lane branch it did not).
// D[tmem] (+)= A[shared] B[shared]
__device__ __forceinline__ void umma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 da, db;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(DESC_HI) : "memory");
}
// D[tmem] (+)= A[tmem] B[shared]
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc)
{
    asm volatile("{\n\t.reg .pred p, e;\n\t.reg .b64 db;\n\tmov.b64 db, {%2, %5};\n\t"
                 "elect.sync _|e, 0xffffffff;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "r"(DESC_HI) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// 32 columns of the warp's lanes, without a wait: the registers may be read after tmem_wait32 on them only.
__device__ __forceinline__ void tmem_ask32(uint32_t ta, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(ta) : "memory");
}
__device__ __forceinline__ void tmem_wait32(uint32_t (&r)[32]) // the registers pass through, so that no use of them moves before the wait
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t ta, const uint32_t *v)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(ta), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
                   "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_ld16u(uint32_t ta, uint32_t (&r)[16])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(ta) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
template <int ID, int N> __device__ __forceinline__ void named_bar() { asm volatile("bar.sync %0, %1;" ::"n"(ID), "n"(N) : "memory"); }
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t *)&v;
}
__device__ __forceinline__ float max_nan(float a, float b) // NaN if either is
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// two fp32 operations per instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(*(unsigned long long *)&d)
        : "l"(*(const unsigned long long *)&a), "l"(*(const unsigned long long *)&b), "l"(*(const unsigned long long *)&c));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*(unsigned long long *)&d) : "l"(*(const unsigned long long *)&a), "l"(*(const unsigned long long *)&b));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(*(unsigned long long *)&d) : "l"(*(const unsigned long long *)&a), "l"(*(const unsigned long long *)&b));
    return d;
}
// 2^t of two values on the FMA pipes, for t <= 127 (t below -126 counts as -126): t = n + f with n = round(t), |f| <= 1/2; a
// polynomial of degree 4 for 2^f (least maximum relative error over the interval by a Lawson iteration: 2.6e-6) whose exponent
// field n is added to.
__device__ __forceinline__ float2 exp2_poly2(float2 t)
{
    const float2 magic = make_float2(12582912.f, 12582912.f); // 1.5 * 2^23: the sum's low bits are n
    t = make_float2(fmaxf(t.x, -126.f), fmaxf(t.y, -126.f));
    const float2 z = add2(t, magic), n = add2(z, make_float2(-12582912.f, -12582912.f));
    const float2 f = fma2(n, make_float2(-1.f, -1.f), t);
    float2 p = fma2(make_float2(0.009570102207362652f, 0.009570102207362652f), f, make_float2(0.05591785907745361f, 0.05591785907745361f));
    p = fma2(p, f, make_float2(0.240247443318367f, 0.240247443318367f));
    p = fma2(p, f, make_float2(0.6931217908859253f, 0.6931217908859253f));
    p = fma2(p, f, make_float2(0.9999992847442627f, 0.9999992847442627f));
    p = make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(z.x) << 23)), __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(z.y) << 23)));
    // at -126 the polynomial gives just under 1, hence a subnormal number here: flushed, so that -inf gives 0
    float2 d;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(*(unsigned long long *)&d) : "l"(*(const unsigned long long *)&p), "l"(0x3f8000003f800000ull));
    return d;
}
// Waits a bounded time whatever the abort flag says: copies and products in flight before the memory is given up.
__device__ __forceinline__ void settle(uint32_t bar, uint32_t parity)
{
    const long long t_end = clock64() + WAIT_LIMIT_CYCLES;
    while (!mbar_try_wait(bar, parity) && clock64() < t_end) {}
}
__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// byte offset of 16-byte chunk c (8 dims) of row r in a K-major tile of 64-dim halves
__device__ __forceinline__ uint32_t tile_at(int r, int c) { return (uint32_t)((c >> 3) * HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }

__device__ __forceinline__ bool clean16(uint4 &u) // takes NaNs and infinities out; true: there were some
{
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if ((w[e] & 0x7f80u) == 0x7f80u) { w[e] &= 0xffff0000u; bad = true; }
        if ((w[e] & 0x7f800000u) == 0x7f800000u) { w[e] &= 0xffffu; bad = true; }
    }
    u = make_uint4(w[0], w[1], w[2], w[3]);
    return bad;
}

// Column (from the unit's first) of the weights of keys k, k + 1: each 32 keys' go over columns of their own half's scores, the
// second 32 over the last 16, so that the first 32 scores can be read again after them.
__device__ __forceinline__ constexpr uint32_t weight_column(int k) { return (uint32_t)((k >> 6) * 64 + (k & 32 ? 48 : 0) + ((k & 31) >> 1)); }
// ... and of what rounding left of it (int8): the rest of those scores' columns
__device__ __forceinline__ constexpr uint32_t rest_column(int k) { return (uint32_t)((k >> 6) * 64 + (k & 32 ? 32 : 16) + ((k & 31) >> 1)); }
constexpr int load_warps(bool tma, bool q8) { return tma ? 2 : q8 ? 8 : 4; }
constexpr int SOFT_WARPS = 8, SOFT_THREADS = 32 * SOFT_WARPS;
constexpr int tc_threads(bool tma, bool q8) { return SOFT_THREADS + 32 * (load_warps(tma, q8) + 1); } // two blocks: 80 registers a thread, 72 or 56
// 8-bit caches: the load warps' way from one tile to the next is the longest, so there are eight of them, and of the 56 registers a thread
// that 17 warps leave they give 16 to the softmax warps: 8 x 72 + 8 x 40 + 56 = 17 x 56.  (ptxas spills 4 to 72 bytes a thread in all variants
// of this kernel but one.)
constexpr int Q8_LAUNCH_REGS = 56, Q8_SOFT_REGS = 72, Q8_LOAD_REGS = 40;
static_assert(8 * Q8_SOFT_REGS + 8 * Q8_LOAD_REGS + Q8_LAUNCH_REGS <= 17 * Q8_LAUNCH_REGS);

template <int FMT, int D, bool TMA>
__global__ void __launch_bounds__(tc_threads(TMA, FMT != KV_BF16), 2) paged_attention_tc_kernel(const __grid_constant__ TcMap k_map, const __grid_constant__ TcMap v_map,
                                                                          const __grid_constant__ PagedAttnArgs a)
{
    using C = TcCfg<D>;
    constexpr bool Q8 = FMT != KV_BF16;
    constexpr uint32_t T_COLS = 256, T_O = 128;
    constexpr int W_LOAD = SOFT_WARPS, W_MMA = SOFT_WARPS + load_warps(TMA, Q8), LT = 32 * load_warps(TMA, Q8);
    extern __shared__ uint8_t tc_raw[];
    uint8_t *gen = tc_raw + ((1024u - (smem_u32(tc_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(gen), bars = base + C::OFF_BAR;
    const uint32_t q_full = bars, k_full = bars + 8, k_empty = bars + 16, v_full = bars + 24, v_empty = bars + 32, v_clean = bars + 40, s_full = bars + 48;
    const uint32_t p_ready = bars + 56, p_rest = bars + 64; // weights of a tile's first 64 keys, of the others
    const uint32_t o_done = bars + 72, drain = bars + 80;
    auto sc_full = [&](int s) { return bars + 8u * (11 + s); };
    uint32_t *tmem_slot = (uint32_t *)(gen + C::OFF_BAR + 8 * 40);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    volatile int *dirty = (volatile int *)(tmem_slot + 2);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) stamp_entry(a.stamp);
    pdl_wait(); // pdl_launch_dependents: below, once the block owns its tensor memory
    const int b = blockIdx.z / a.splits, split = blockIdx.z % a.splits, kvh = blockIdx.y;
    int row0, n_new, len;
    if (!batch_row(a.rb, b, a.max_new, a.max_context, row0, n_new, len, a.err)) return;
    constexpr int ROWS = TQ;
    const int all_rows = n_new * a.group;
    const int tile = (int)gridDim.x - 1 - (int)blockIdx.x; // the longest rows first
    const int r0 = tile * ROWS;
    if (r0 >= all_rows) return;
    const int rows = min(ROWS, all_rows - r0);
    // new token and head of the tiles' row r.  A quotient of small numbers by way of their floats: (n + 1/2) / group is off by less
    // than the 1 / (2 group) that could change it while n < 2^22, and n < group + 256
    const int tok0 = r0 / a.group, head0 = r0 - tok0 * a.group;
    const float inv_group = 1.f / (float)a.group;
    auto token_of = [&](int r) { return (int)(((float)(head0 + r) + 0.5f) * inv_group); }; // after tok0
    auto head_of = [&](int r, int token) { return head0 + r - token * a.group; };
    const int pos_first = len + r0 / a.group, pos_last = len + (r0 + rows - 1) / a.group;
    const int kv_len = pos_last + 1;
    // tiles of 128 keys that hold a key some row sees: sinks, then the window of the first row onwards
    const int lo_min = a.window ? max(0, pos_first - a.window + 1) : 0, first = lo_min / TK;
    const int n_sink = min((min(a.sinks, lo_min) + TK - 1) / TK, first);
    const int n_all = n_sink + (kv_len + TK - 1) / TK - first;
    const int j_begin = (int)((long)n_all * split / a.splits), n_tiles = (int)((long)n_all * (split + 1) / a.splits) - j_begin;
    auto key0 = [&](int j) { return ((j_begin + j) < n_sink ? (j_begin + j) : first + (j_begin + j) - n_sink) * TK; };
    auto key_needed = [&](int t) { return t < kv_len && (t >= lo_min || t < a.sinks); };
    // some row does not see some key of the tile
    auto partial = [&](int t0) { return !(t0 + TK - 1 <= pos_first && (!a.window || t0 > pos_last - a.window || t0 + TK - 1 < a.sinks)); };
    const int32_t *bt = a.rb.table + (long)b * a.rb.max_pages;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        *dirty = 0;
        mbar_init(q_full, SOFT_THREADS);
        mbar_init(k_full, TMA ? 1 : LT);
        mbar_init(v_full, TMA ? 1 : LT);
        mbar_init(k_empty, 1);
        mbar_init(v_empty, 1);
        mbar_init(v_clean, 1);
        mbar_init(s_full, 1);
        mbar_init(p_ready, 4);
        mbar_init(p_rest, 4);
        mbar_init(o_done, 1);
        mbar_init(drain, 1);
        for (int s = 0; s < 8; ++s) mbar_init(sc_full(s), 128);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == W_MMA) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(T_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_launch_dependents();
    if (warp >= W_LOAD && warp < W_MMA) {
        if (Q8) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Q8_LOAD_REGS));
        const int tid = threadIdx.x - 32 * W_LOAD;
        // one box = 16 keys x 64 dims; lane = (16 keys, half of the head); 16 keys that no row needs come as zeros (a row beyond the map)
        constexpr int BOXES = 8 * (D / 64);
        auto tma_tile = [&](int j, bool is_v) {
            const uint32_t full = is_v ? v_full : k_full;
            const int t = key0(j) + (lane & 7) * 16, h = lane >> 3;
            long row = (long)a.kv.n_pages * a.kv.nkv * a.kv.page;
            if (t < kv_len && (t + 15 >= lo_min || t < a.sinks)) {
                const int pi = t / a.kv.page;
                int page = bt[pi];
                if (page < 0 || page >= a.kv.n_pages) { atomicOr(a.err, ERR_PAGE_RANGE); page = 0; }
                row = ((long)page * a.kv.nkv + kvh) * a.kv.page + (t - pi * a.kv.page);
            }
            bool ok = true;
            if (j > 0) ok = mbar_wait(is_v ? v_empty : k_empty, (j - 1) & 1, a.err, abort_flag);
            if (!__all_sync(0xffffffffu, ok)) return false;
            if (lane == 0) mbar_expect_tx(full, C::TILE);
            __syncwarp();
            if (lane < BOXES)
                tma_load_3d(base + (is_v ? C::OFF_V : C::OFF_K) + h * HALF + (lane & 7) * 2048, (const CUtensorMap *)(is_v ? &v_map : &k_map),
                            h * 64, (int)row, 0, full);
            return true;
        };
        bool ok = true;
        if (TMA) {
            // The first warp asks for the K tiles, the second for the V tiles.  It also passes them on to the MMA warps: those with
            // keys that not every row sees without the values that 0 would not cancel.
            if (warp == W_LOAD) {
                int in = 0;
                for (; ok && in < n_tiles; in += ok) ok = tma_tile(in, false);
                if (!ok && in > 0) settle(k_full, (in - 1) & 1); // a copy in flight lands before the block ends
            } else {
                int in = 0;
                for (; ok && in < n_tiles; ) {
                    ok = tma_tile(in, true);
                    if (!ok) break;
                    const int j = in++;
                    ok = mbar_wait(v_full, j & 1, a.err, abort_flag);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (partial(key0(j))) {
                        const uint32_t v = base + C::OFF_V + lane * 16;
                        uint32_t top = 0; // largest magnitude bits of either half
#pragma unroll 16
                        for (int i = 0; i < C::TILE / 512; ++i) {
                            const uint4 x = lds128(v + i * 512);
                            top = __vmaxu2(top, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
                        }
                        if ((top & 0xffffu) >= 0x7f80u || (top >> 16) >= 0x7f80u) {
                            for (int i = 0; i < C::TILE / 512; ++i) {
                                uint4 x = lds128(v + i * 512);
                                if (clean16(x)) sts128(v + i * 512, x);
                            }
                            *dirty = 1;
                        }
                        fence_proxy_async();
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive(v_clean);
                }
                if (!ok && in > 0) settle(v_full, (in - 1) & 1);
            }
        } else {
            long *rowoff = (long *)(gen + C::OFF_ROW);
            float *sc = (float *)(gen + C::OFF_SC);
            auto rows_of = [&](int j) { // cached rows (-1: no row needs the key) and scales of the tile's keys
                if (LT > 128 && tid >= 128) {
                    named_bar<BAR_LOAD, LT>();
                    return;
                }
                const int t = key0(j) + tid;
                long row = -1;
                if (key_needed(t)) {
                    const int pi = t / a.kv.page, page = bt[pi];
                    if (page < 0 || page >= a.kv.n_pages) atomicOr(a.err, ERR_PAGE_RANGE);
                    else row = ((long)page * a.kv.nkv + kvh) * a.kv.page + (t - pi * a.kv.page);
                }
                rowoff[(j & 1) * 128 + tid] = row;
                if (Q8) {
                    sc[(j & 7) * 256 + tid] = row >= 0 ? a.kv.ks[row] : 0.f;
                    sc[(j & 7) * 256 + 128 + tid] = row >= 0 ? a.kv.vs[row] : 0.f;
                    mbar_arrive(sc_full(j & 7)); // eight tiles later the slot's scores have long been weighted
                }
                named_bar<BAR_LOAD, LT>();
            };
            if constexpr (Q8) {
                constexpr int CPR = D / 16, N = 64 * CPR / LT; // 16-code chunks per row; per thread and half a tile (64 keys)
                const uint32_t c128 = widen_const();
                const int c = tid % CPR;
                auto fetch = [&](int j, int h, const void *pages, uint4 (&x)[N]) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const long row = rowoff[(j & 1) * 128 + h * 64 + i * (LT / CPR) + tid / CPR];
                        x[i] = row >= 0 ? *(const uint4 *)((const uint8_t *)pages + row * D + c * 16) : make_uint4(0, 0, 0, 0);
                    }
                };
                auto widen = [&](uint32_t tile_base, int h, const uint4 (&x)[N]) {
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int r = h * 64 + i * (LT / CPR) + tid / CPR;
                        const uint4 lo = make_uint4(even2<FMT>(x[i].x, c128), odd2<FMT>(x[i].x, c128), even2<FMT>(x[i].y, c128), odd2<FMT>(x[i].y, c128));
                        const uint4 hi = make_uint4(even2<FMT>(x[i].z, c128), odd2<FMT>(x[i].z, c128), even2<FMT>(x[i].w, c128), odd2<FMT>(x[i].w, c128));
                        const bool swap = (c >> 2) & 1; // the two halves of the head in turn: other banks
                        sts128(tile_base + tile_at(r, 2 * c + swap), swap ? hi : lo);
                        sts128(tile_base + tile_at(r, 2 * c + !swap), swap ? lo : hi);
                    }
                };
                uint4 x0[N], x1[N]; // one batch is on its way while the other is widened
                if (n_tiles > 0) { rows_of(0); fetch(0, 0, a.kv.k, x0); }
                for (int j = 0; j < n_tiles; ++j) {
                    fetch(j, 1, a.kv.k, x1);
                    if (j > 0) mbar_wait(k_empty, (j - 1) & 1, a.err, abort_flag);
                    widen(base + C::OFF_K, 0, x0);
                    fetch(j, 0, a.kv.v, x0);
                    widen(base + C::OFF_K, 1, x1);
                    fence_proxy_async();
                    mbar_arrive(k_full);
                    fetch(j, 1, a.kv.v, x1);
                    if (j > 0) mbar_wait(v_empty, (j - 1) & 1, a.err, abort_flag);
                    widen(base + C::OFF_V, 0, x0);
                    if (j + 1 < n_tiles) { rows_of(j + 1); fetch(j + 1, 0, a.kv.k, x0); }
                    widen(base + C::OFF_V, 1, x1);
                    fence_proxy_async();
                    mbar_arrive(v_full);
                }
            } else {
                // cp.async, one operand tile behind
                constexpr int CH = D / 8;
                auto copy = [&](int j, const void *pages, uint32_t tile_base) {
                    for (int i = tid; i < 128 * CH; i += 128) {
                        const int r = i / CH, c = i % CH;
                        const long row = rowoff[(j & 1) * 128 + r];
                        cp16(tile_base + tile_at(r, c), (const bf16 *)pages + (row >= 0 ? row * D + c * 8 : 0), row >= 0);
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                };
                auto landed_v = [&](int j) {
                    if (partial(key0(j))) { // this thread's own chunks
                        bool bad = false;
                        for (int i = tid; i < 128 * CH; i += 128) {
                            const uint32_t p = base + C::OFF_V + tile_at(i / CH, i % CH);
                            uint4 u = lds128(p);
                            if (clean16(u)) { sts128(p, u); bad = true; }
                        }
                        if (bad) *dirty = 1;
                    }
                    fence_proxy_async();
                    mbar_arrive(v_full);
                };
                for (int j = 0; j < n_tiles; ++j) {
                    rows_of(j);
                    if (j > 0) mbar_wait(k_empty, (j - 1) & 1, a.err, abort_flag);
                    copy(j, a.kv.k, base + C::OFF_K);
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    if (j) landed_v(j - 1);
                    if (j > 0) mbar_wait(v_empty, (j - 1) & 1, a.err, abort_flag);
                    copy(j, a.kv.v, base + C::OFF_V);
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    fence_proxy_async();
                    mbar_arrive(k_full);
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                if (n_tiles) landed_v(n_tiles - 1);
            }
        }
    } else if (warp >= W_MMA) {
        // A wait that gives up raises the abort flag, after which every wait returns at once: the loops run out on whatever is there,
        // and the block ends with the error bit set.
        constexpr uint32_t idesc_s = make_idesc(TK), idesc_o = make_idesc(D) | (1u << 16); // V: MN-major
        const uint32_t q_lo = desc_lo(base + C::OFF_Q, 1), k_lo = desc_lo(base + C::OFF_K, 1), v_lo = desc_lo(base + C::OFF_V, HALF >> 4);
        auto wait = [&](uint32_t bar, int parity) {
            mbar_wait(bar, parity, a.err, abort_flag);
            __syncwarp();
            fence_after();
        };
        auto issue_s = [&] {
#pragma unroll
            for (int kk = 0; kk < D / UMMA_K; ++kk)
                umma_ss(tmem, q_lo + (kk >> 2) * (HALF >> 4) + (kk & 3) * 2, k_lo + (kk >> 2) * (HALF >> 4) + (kk & 3) * 2, idesc_s, kk > 0);
            commit(s_full);
            commit(k_empty);
        };
        auto issue_o = [&](int kk0, bool acc) { // 64 keys
#pragma unroll
            for (int kk = kk0; kk < kk0 + 64 / UMMA_K; ++kk)
                umma_ts(tmem + T_O, tmem + weight_column(16 * kk), v_lo + kk * (UMMA_K * 128 >> 4), idesc_o, acc || kk > 0);
            if (FMT == KV_INT8) {
#pragma unroll
                for (int kk = kk0; kk < kk0 + 64 / UMMA_K; ++kk)
                    umma_ts(tmem + T_O, tmem + rest_column(16 * kk), v_lo + kk * (UMMA_K * 128 >> 4), idesc_o, 1);
            }
        };
        if (n_tiles > 0) {
            wait(q_full, 0);
            wait(k_full, 0);
            issue_s();
        }
        for (int j = 0; j < n_tiles; ++j) {
            wait(TMA ? v_clean : v_full, j & 1);
            wait(p_ready, j & 1);
            issue_o(0, j > 0);
            wait(p_rest, j & 1);
            issue_o(64 / UMMA_K, true);
            commit(v_empty);
            if (j + 1 < n_tiles) {
                wait(k_full, (j + 1) & 1);
                issue_s();
            } else
                commit(o_done);
        }
        // one answer for the warp: another warp may raise the flag at this moment
        if (__any_sync(0xffffffffu, *abort_flag) && n_tiles > 0) { // products in flight end before tensor memory is freed
            commit(drain);
            settle(drain, 0);
        }
        __syncwarp();
    } else {
        if (Q8) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Q8_SOFT_REGS));
        const int half = warp >> 2, row = (warp & 3) * 32 + lane, pair_bar = BAR_PAIR + (warp & 3);
        // Q: rows of the tiles, zeros beyond the last; codes' dim order where the cache is 8-bit
        {
            constexpr int CH = D / 8, N = ROWS * CH / SOFT_THREADS;
            uint4 x[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int idx = k * SOFT_THREADS + threadIdx.x, r = idx / CH, c = idx % CH, t = token_of(r);
                x[k] = make_uint4(0, 0, 0, 0);
                if (r < rows) x[k] = *(const uint4 *)((const bf16 *)a.q + (long)(row0 + tok0 + t) * a.q_stride + (long)(kvh * a.group + head_of(r, t)) * D + c * 8);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int idx = k * SOFT_THREADS + threadIdx.x, r = idx / CH, c = idx % CH;
                const uint4 y = x[k];
                sts128(base + C::OFF_Q + tile_at(r, c),
                       Q8 ? make_uint4(__byte_perm(y.x, y.y, 0x5410), __byte_perm(y.x, y.y, 0x7632), __byte_perm(y.z, y.w, 0x5410), __byte_perm(y.z, y.w, 0x7632)) : y);
            }
            fence_proxy_async();
            mbar_arrive(q_full);
        }
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + half * 64u; // this thread's scores: 64 columns; its weights: the first 32 of them
        const uint32_t t_o = tmem + lanes + T_O + half * (D / 2);
        const int my_token = token_of(row);
        const bool live = row < rows;
        const int pos = live ? len + tok0 + my_token : -1;
        const float qs = a.scale_log2;
        const float *sc = (const float *)(gen + C::OFF_SC);
        float *red = (float *)(gen + C::OFF_RED);
        float m_used = -INFINITY, l = 0.f;
        for (int j = 0; j < n_tiles; ++j) {
            const int t0 = key0(j) + half * 64;
            mbar_wait(s_full, j & 1, a.err, abort_flag); // see the MMA warp about waits that give up
            if (Q8) mbar_wait(sc_full(j & 7), (j >> 3) & 1, a.err, abort_flag);
            __syncwarp();
            fence_after();
            const bool masked = partial(key0(j));
            unsigned long long seen = ~0ull; // this thread's columns whose keys the row sees: c <= pos - t0 with c >= lo or c < sinks - t0
            if (masked) {
                auto below = [](int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; };
                seen = below(pos - t0 + 1);
                if (a.window) seen &= ~below(pos - a.window + 1 - t0) | below(a.sinks - t0);
            }
            const float *ks = sc + (j & 7) * 256 + half * 64, *vs = ks + 128;
            // 32 scores (as read) in columns c0 ..: scaled by the keys' scales, -inf where the row does not see the key
            auto finish = [&](int c0, uint32_t (&r)[32]) {
                if (Q8) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 k4 = *(const float4 *)(ks + c0 + e);
                        const float2 x = mul2(make_float2(__uint_as_float(r[e]), __uint_as_float(r[e + 1])), make_float2(k4.x, k4.y));
                        const float2 y = mul2(make_float2(__uint_as_float(r[e + 2]), __uint_as_float(r[e + 3])), make_float2(k4.z, k4.w));
                        r[e] = __float_as_uint(x.x); r[e + 1] = __float_as_uint(x.y); r[e + 2] = __float_as_uint(y.x); r[e + 3] = __float_as_uint(y.y);
                    }
                }
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!((uint32_t)(seen >> c0) & (1u << e))) r[e] = 0xff800000u;
                }
            };
            auto max_of = [&](const uint32_t (&r)[32]) {
                float x0 = -INFINITY, x1 = -INFINITY, x2 = -INFINITY, x3 = -INFINITY;
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    x0 = max_nan(max_nan(x0, __uint_as_float(r[e])), __uint_as_float(r[e + 1]));
                    x1 = max_nan(max_nan(x1, __uint_as_float(r[e + 2])), __uint_as_float(r[e + 3]));
                    x2 = max_nan(max_nan(x2, __uint_as_float(r[e + 4])), __uint_as_float(r[e + 5]));
                    x3 = max_nan(max_nan(x3, __uint_as_float(r[e + 6])), __uint_as_float(r[e + 7]));
                }
                return max_nan(max_nan(x0, x1), max_nan(x2, x3));
            };
            uint32_t ra[32], rb[32]; // the first 32 scores are read twice: 64 would not stay in the registers of two blocks
            float mx;
            tmem_ask32(t_s, ra);
            tmem_wait32(ra);
            finish(0, ra);
            mx = max_of(ra);
            tmem_ask32(t_s + 32, rb);
            tmem_wait32(rb);
            finish(32, rb);
            mx = max_nan(mx, max_of(rb)) * qs;
            // join with the other half's maximum: both threads of a row then take the same decision
            float *rm = red + (j & 1) * 256 + row;
            rm[half * 128] = mx;
            asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
            mx = max_nan(mx, rm[(half ^ 1) * 128]);
            // A NaN or +inf among the scores: no softmax.  Said here, because exp2_poly2 would make a weight of 0 of the NaN or inf - inf
            // that is its argument then.
            if (!(mx < INFINITY)) l = __uint_as_float(0x7fc00000u);
            const bool up = mx > m_used + 8.f; // -inf: a row's first keys
            if (__any_sync(0xffffffffu, up)) {
                // all rows of the warp follow, so that rows whose first keys were few or low do not come one by one
                float f = 1.f;
                if (mx > m_used) { f = m_used == -INFINITY ? 1.f : ex2(m_used - mx); m_used = mx; l *= f; }
                if (j > 0 && __any_sync(0xffffffffu, f != 1.f)) {
                    // every product so far is complete: S of this tile was issued after them
#pragma unroll 1
                    for (int d0 = 0; d0 < D / 2; d0 += 16) {
                        uint32_t x[16];
                        tmem_ld16u(t_o + d0, x);
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
                        tmem_st16(t_o + d0, x);
                    }
                    tmem_st_wait();
                    fence_before();
                    asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory"); // the other half's columns too
                }
            }
            const float mb = m_used == -INFINITY ? 0.f : m_used;
            const float2 q2 = make_float2(qs, qs), m2 = make_float2(-mb, -mb);
            float2 ls = make_float2(0.f, 0.f);
            auto weigh = [&](int c0, uint32_t (&r)[32]) {
                uint32_t w[16];
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const float2 t = fma2(make_float2(__uint_as_float(r[2 * k]), __uint_as_float(r[2 * k + 1])), q2, m2);
                    // every second pair (bf16 pages by TMA) or every fourth on the FMA pipes, which the exponentials otherwise leave idle
                    float2 p = (TMA ? k % 2 == 1 : k % 4 == 3) ? exp2_poly2(t) : make_float2(ex2(t.x), ex2(t.y));
                    ls = add2(ls, p);
                    if (Q8) p = mul2(p, *(const float2 *)(vs + c0 + 2 * k));
                    w[k] = pack(p.x, p.y);
                    if (FMT == KV_INT8) { r[2 * k] = __float_as_uint(p.x); r[2 * k + 1] = __float_as_uint(p.y); }
                }
                if (Q8 && masked) { // 0 times the scale of an unseen key, which may be anything
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        if (!((uint32_t)(seen >> c0) & (1u << (2 * k)))) w[k] &= 0xffff0000u;
                        if (!((uint32_t)(seen >> c0) & (2u << (2 * k)))) w[k] &= 0xffffu;
                    }
                }
                tmem_st16(t_s + weight_column(c0), w);
                if (FMT == KV_INT8) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        w[k] = pack(__uint_as_float(r[2 * k]) - __uint_as_float(w[k] << 16), __uint_as_float(r[2 * k + 1]) - __uint_as_float(w[k] & 0xffff0000u));
                        if (masked) {
                            if (!((uint32_t)(seen >> c0) & (1u << (2 * k)))) w[k] &= 0xffff0000u;
                            if (!((uint32_t)(seen >> c0) & (2u << (2 * k)))) w[k] &= 0xffffu;
                        }
                    }
                    tmem_st16(t_s + rest_column(c0), w);
                }
            };
            weigh(32, rb);
            tmem_ask32(t_s, ra);
            tmem_wait32(ra);
            finish(0, ra);
            weigh(0, ra);
            l += ls.x + ls.y;
            tmem_st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(half ? p_rest : p_ready);
        }
        bool ok = true;
        if (n_tiles > 0) {
            ok = mbar_wait(o_done, 0, a.err, abort_flag);
            ok = __all_sync(0xffffffffu, ok);
            fence_after();
        }
        // the sums of a row's two threads
        asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory"); // the maxima have been read
        red[half * 128 + row] = l;
        asm volatile("bar.sync %0, 64;" ::"r"(pair_bar) : "memory");
        {
            const float den = l + red[(half ^ 1) * 128 + row];
            float m = m_used;
            if (den != den) m = fmaxf(m, 0.f); // scores that are all NaN leave no maximum
            const float inv = a.part_o ? 1.f : inverse_sum(den);
            const int head = kvh * a.group + head_of(row, my_token);
            const long token = row0 + tok0 + my_token;
            const long w = (long)split * ((long)a.rb.n_tokens * a.nq) + token * a.nq + head;
            if (a.part_o && live && half == 0) { a.part_ml[w * 2] = m; a.part_ml[w * 2 + 1] = den; }
            const bool give_back = !Q8 && *dirty;
#pragma unroll 1
            for (int c0 = half * (D / 2); c0 < (half + 1) * (D / 2) && n_tiles > 0 && ok; c0 += 16) {
                uint32_t y[16];
                float v[16], x[16];
                __syncwarp(); // the load is the whole warp's; rows take their own ways below
                tmem_ld16u(tmem + lanes + T_O + c0, y);
                if (live) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(y[e]);
                    if (give_back) {
                        for (int j = 0; j < n_tiles; ++j) {
                            const int t0 = key0(j);
                            for (int t = t0; t < t0 + TK && partial(t0); ++t) {
                                if (t > pos || (a.window && t <= pos - a.window && t >= a.sinks)) continue;
                                const int pi = t / a.kv.page, page = bt[pi];
                                if (page < 0 || page >= a.kv.n_pages) continue;
                                const bf16 *src = (const bf16 *)a.kv.v + (((long)page * a.kv.nkv + kvh) * a.kv.page + (t - pi * a.kv.page)) * D + c0;
#pragma unroll 1
                                for (int e = 0; e < 16; ++e) {
                                    const float z = __bfloat162float(src[e]);
                                    if (!isfinite(z)) {
#pragma unroll
                                        for (int k = 0; k < 16; ++k)
                                            if (k == e) v[k] += z;
                                    }
                                }
                            }
                        }
                    }
                    // columns of an 8-bit cache are in the order (0, 2, 1, 3) of every four
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[Q8 ? (e & ~3) | ((e & 1) << 1) | ((e >> 1) & 1) : e] = v[e] * inv;
                    if (a.part_o) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) *(float4 *)(a.part_o + w * D + c0 + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                    } else { // through the Q tile, so that whole rows leave together
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            sts128(base + C::OFF_Q + tile_at(row, (c0 + e) >> 3),
                                   make_uint4(pack(x[e], x[e + 1]), pack(x[e + 2], x[e + 3]), pack(x[e + 4], x[e + 5]), pack(x[e + 6], x[e + 7])));
                    }
                }
            }
            if (!a.part_o && n_tiles > 0) {
                named_bar<BAR_OUT, SOFT_THREADS>();
                constexpr int CH = D / 8;
#pragma unroll 4
                for (int idx = threadIdx.x; idx < 128 * CH; idx += SOFT_THREADS) {
                    const int r = idx / CH, c = idx % CH, t = token_of(r);
                    if (r >= rows || !ok) continue;
                    *(uint4 *)((bf16 *)a.out + (long)(row0 + tok0 + t) * a.o_stride + (long)(kvh * a.group + head_of(r, t)) * D + c * 8) =
                        lds128(base + C::OFF_Q + tile_at(r, c));
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (warp == W_MMA) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(T_COLS) : "memory");
    }
    if (threadIdx.x == 0) stamp_exit(a.stamp);
}

template <int FMT, int D, bool TMA> cudaError_t launch_tc(const PagedAttnArgs &a, const TcMap &km, const TcMap &vm, cudaStream_t st)
{
    static SmemLimit limit;
    if (FMT != KV_BF16) { // the registers that the warps pass on have to be there
        static const cudaError_t fits = [] {
            cudaFuncAttributes f{};
            const cudaError_t e = cudaFuncGetAttributes(&f, (const void *)paged_attention_tc_kernel<FMT, D, TMA>);
            return e != cudaSuccess ? e : f.numRegs == Q8_LAUNCH_REGS ? cudaSuccess : cudaErrorInvalidKernelImage;
        }();
        if (fits != cudaSuccess) return fits;
    }
    const cudaError_t e = limit.raise((const void *)paged_attention_tc_kernel<FMT, D, TMA>, TcCfg<D>::SMEM);
    if (e != cudaSuccess) return e;
    const long tiles = ((long)a.max_new * a.group + TQ - 1) / TQ;
    return launch_kernel(paged_attention_tc_kernel<FMT, D, TMA>, dim3((unsigned)tiles, a.kv.nkv, a.rb.B * a.splits), dim3(tc_threads(TMA, FMT != KV_BF16)),
                         TcCfg<D>::SMEM, st, 0, km, vm, a);
}
template <int FMT, int D> cudaError_t tc_by_copy(const PagedAttnArgs &a, cudaStream_t st)
{
    TcMap km{}, vm{};
    if constexpr (FMT == KV_BF16) {
        const long rows = (long)a.kv.n_pages * a.kv.nkv * a.kv.page;
        if (a.kv.page % 16 == 0 && rows < 0x7fffff00L && make_operand_map(&km, a.kv.k, D, rows, 1, D, 0, 16) == 0 &&
            make_operand_map(&vm, a.kv.v, D, rows, 1, D, 0, 16) == 0)
            return launch_tc<FMT, D, true>(a, km, vm, st);
    }
    return launch_tc<FMT, D, false>(a, km, vm, st);
}
template <int FMT> cudaError_t tc_by_dim(const PagedAttnArgs &a, cudaStream_t st)
{
    if (a.kv.d == 128) return tc_by_copy<FMT, 128>(a, st);
    if (a.kv.d == 64) return tc_by_copy<FMT, 64>(a, st);
    return cudaErrorInvalidValue;
}

} // namespace

cudaError_t launch_paged_attention_tc(const PagedAttnArgs &a, cudaStream_t st)
{
    switch (a.kv.fmt) {
    case KV_BF16: return tc_by_dim<KV_BF16>(a, st);
    case KV_E4M3: return tc_by_dim<KV_E4M3>(a, st);
    case KV_INT8: return tc_by_dim<KV_INT8>(a, st);
    default: return cudaErrorInvalidValue;
    }
}

} // namespace spd
