// What the kernels for few query rows share (paged_attention_rows.cu, paged_attention_rows4.cu): loads, MMAs, which keys a row sees, and how
// the partial rows of a thread block's warps, of a cluster's blocks and of the key ranges become the output.
#pragma once
#include "paged.cuh"
#include "tc_ptx.cuh"

namespace spd {
namespace few {

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool valid)
{
    const int n = valid ? 16 : 0; // 0 source bytes: zero fill
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
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
// the first of a chain, float16: nothing to add to
__device__ __forceinline__ void mma16816_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
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

// keys t that a row at position pos (-1: no row) sees
__device__ __forceinline__ bool sees(int t, int pos, int window, int sinks) { return t <= pos && (!window || t > pos - window || t < sinks); }

// key of score row c (0-7) of eight
__device__ __forceinline__ int key_of(int c) { return c & 1 ? (c & 6) ^ 5 : c; }

__device__ __forceinline__ void store2(bf16 *p, float x, float y) { *(uint32_t *)p = pack(x, y); }
__device__ __forceinline__ void store2(float *p, float x, float y) { *(float2 *)p = make_float2(x, y); }

// Shared memory behind the partial rows, from `off_pml` on: merged [16][2], weights [16][RW], rows' places [16], ranges' weights [16][8].
constexpr int join_bytes(int RW) { return 128 + 16 * RW * 4 + 128 + 16 * PAGED_MAX_CLUSTER * 4; }

// The warps' partial rows (packed rows r0 .. r0 + rows - 1 of the sequence) lie at gen: [warp][16][D + 2] sums, then [warp][16][2] maxima and weights' sums.  extra(r, c, x, y): called for columns
// c and c + 1 of row r once their warps' sums are added up in x and y.
template <typename T, int D, int RW, typename Extra>
__device__ __forceinline__ void join_rows(const PagedAttnArgs &a, uint8_t *gen, int off_pml, int rows, int row0, int r0, int kvh, int split, int splits, Extra extra)
{
    constexpr int R_THREADS = 32 * RW;
    const uint32_t base = tc::smem_u32(gen);
    float *mo = (float *)gen, *ml = mo + RW * 16 * (D + 2), *pml = (float *)(gen + off_pml);
    __syncthreads();
    // per row: the warps' weights relative to the block's maximum, its maximum and sum, where the row goes
    const bool clustered = a.splits > 1 && !a.part_o;
    const long plane = (long)a.rb.n_tokens * a.nq;
    float *wt = pml + 32;                // [16][RW]
    long *dst_of = (long *)(wt + 16 * RW); // [16]
    float *cw = (float *)(dst_of + 16);    // [16][ranges of a cluster]
    if (threadIdx.x < rows) {
        const int r = threadIdx.x, i = (r0 + r) / a.group, head = kvh * a.group + r0 + r - i * a.group;
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
        extra(r, c, x, y);
        if (a.splits == 1) {
            const float inv = inverse_sum(pml[2 * r + 1]);
            store2((T *)a.out + dst_of[r] + c, x * inv, y * inv);
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
        const uint32_t mo_addr = base, pml_addr = base + off_pml;
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
            store2((T *)a.out + dst_of[r] + c, x, y);
        }
        tc::cluster_sync(); // no block exits while a peer still reads its shared memory
    }
}

} // namespace few
} // namespace spd
