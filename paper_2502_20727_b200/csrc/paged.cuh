// Paged K/V cache operators: the cache's storage formats, where rows of a ragged batch sit in their sequences and
// pages, and the launchers of kv_cache.cu, paged_attention.cu, paged_attention_rows.cu, paged_attention_rows4.cu and paged_attention_tc.cu.
#pragma once
#include "common.cuh"

#include <atomic>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

namespace spd {

enum KvFormat : int { KV_F32 = 0, KV_BF16 = 1, KV_E4M3 = 2, KV_INT8 = 3, KV_INT4 = 5 };

// [n_pages, n_kv_heads, page, head_dim] elements; 8-bit formats: one float32 scale per (page, head, row).  4 bits: head_dim / 2 bytes per
// row, and instead of a scale two words, one per half of the head dims: a bfloat16 scale (low bits) and a bfloat16 smallest value.
struct PagedKv {
    void *k, *v;
    float *ks, *vs;
    int n_pages, nkv, page, d, fmt;
};

// New rows of B sequences, one sequence after the other: sequence b has rows cu[b] .. cu[b+1]-1 at positions
// lens[b], lens[b]+1, ...  The stack's own batches (attention only): cu null = `uniform` rows each; lens null = 0; plus `first`.
struct RaggedBatch {
    const int32_t *cu, *lens, *table;
    int B, max_pages, n_tokens;
    int uniform, first;
};

struct PagedAttnArgs {
    PagedKv kv;
    RaggedBatch rb;
    const void *q;
    void *out;
    long q_stride, o_stride;      // elements between token rows
    int nq, group;                // query heads; query heads per KV head
    int max_new, max_context;     // host bounds on new and on cached + new tokens of a sequence
    int window, sinks;            // window 0: everything before the query
    float scale_log2;             // softmax scale times log2(e)
    int splits;                   // ranges the keys of a row tile are cut into
    int row_tile;                 // general kernel: rows of a thread block (16 or 64)
    int stages;                   // paged_attention_rows.cu: set by its launcher
    int longest_first;            // 4-bit caches: thread blocks take the sequences by length (batch_row_by_length)
    float *part_o, *part_ml;      // ranges that no cluster adds up (else null): fp32 [splits][n_tokens * nq][d], [splits][n_tokens * nq][2]
    int *err;
    unsigned long long *stamp;    // the stack's launch timeline, or null
};

template <int FMT> struct KvElem;
template <> struct KvElem<KV_F32> { typedef float type; };
template <> struct KvElem<KV_BF16> { typedef bf16 type; };
template <> struct KvElem<KV_E4M3> { typedef uint8_t type; };
template <> struct KvElem<KV_INT8> { typedef int8_t type; };
template <> struct KvElem<KV_INT4> { typedef uint8_t type; };

// code -> the value it stands for before the row's scale
template <int FMT> __device__ __forceinline__ float kv_value(typename KvElem<FMT>::type c);
template <> __device__ __forceinline__ float kv_value<KV_F32>(float c) { return c; }
template <> __device__ __forceinline__ float kv_value<KV_BF16>(bf16 c) { return __bfloat162float(c); }
template <> __device__ __forceinline__ float kv_value<KV_E4M3>(uint8_t c)
{
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(c, __NV_E4M3)));
}
template <> __device__ __forceinline__ float kv_value<KV_INT8>(int8_t c) { return (float)c; }

// 4-bit rows: byte i holds the code of dim i (low bits) and of dim i + head_dim / 2; value = code * scale + smallest of the dim's half.
__device__ __forceinline__ float kv4_scale(uint32_t half) { return __uint_as_float(half << 16); }
__device__ __forceinline__ float kv4_min(uint32_t half) { return __uint_as_float(half & 0xffff0000u); }
// A row's parameters; all four are NaN where one of them is not finite.
__device__ __forceinline__ uint2 kv4_params(const float *params, long row)
{
    const uint2 p = *(const uint2 *)(params + 2 * row);
    const uint32_t bad = (((p.x & 0x7f807f80u) + 0x00800080u) | ((p.y & 0x7f807f80u) + 0x00800080u)) & 0x80008000u;
    return bad ? make_uint2(0x7fc07fc0u, 0x7fc07fc0u) : p;
}

// Two 8-bit codes of a word -> bf16x2 of the values they stand for, exactly: bytes 0 and 2 (even), bytes 1 and 3 (odd).
// c128: widen_const(), kept in a register by the caller.
template <int FMT> __device__ __forceinline__ uint32_t even2(uint32_t w, uint32_t c128);
template <int FMT> __device__ __forceinline__ uint32_t odd2(uint32_t w, uint32_t c128);
__device__ __forceinline__ uint32_t widen_const() // bf16x2 of 128, which the compiler does not turn back into a literal
{
    uint32_t c;
    asm volatile("mov.b32 %0, 0x43004300;" : "=r"(c));
    return c;
}
__device__ __forceinline__ uint32_t e4m3_fix(uint32_t x) // sign | 4 exponent bits | 3 mantissa bits in bf16's places: times 2^120
{
    const __nv_bfloat162 v = __hmul2(*(const __nv_bfloat162 *)&x, __nv_bfloat162(__ushort_as_bfloat16(0x7b80), __ushort_as_bfloat16(0x7b80)));
    return *(const uint32_t *)&v;
}
// (a & b) | c in one instruction: with two literals the compiler takes two
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t int8_fix(uint32_t w, uint32_t c128) // codes in bits 0-7 and 16-23
{
    const uint32_t x = and_or(w, 0x007f007fu, c128), y = and_or(w, 0x00800080u, c128);
    const __nv_bfloat162 v = __hsub2(*(const __nv_bfloat162 *)&x, *(const __nv_bfloat162 *)&y);
    return *(const uint32_t *)&v;
}
template <> __device__ __forceinline__ uint32_t even2<KV_E4M3>(uint32_t w, uint32_t) { return e4m3_fix(((w << 4) & 0x07f007f0u) | ((w << 8) & 0x80008000u)); }
template <> __device__ __forceinline__ uint32_t odd2<KV_E4M3>(uint32_t w, uint32_t) { return e4m3_fix(((w >> 4) & 0x07f007f0u) | (w & 0x80008000u)); }
template <> __device__ __forceinline__ uint32_t even2<KV_INT8>(uint32_t w, uint32_t c128) { return int8_fix(w, c128); }
template <> __device__ __forceinline__ uint32_t odd2<KV_INT8>(uint32_t w, uint32_t c128) { return int8_fix(w >> 8, c128); }

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

// What a sequence's batch row says, checked once: false (and an error bit) where it does not fit the call.
__device__ __forceinline__ bool batch_row_fits(const RaggedBatch &rb, int max_new, int max_context, int row0, int &n_new, int len, int *err)
{
    if (n_new == 0) return false;
    if (row0 < 0 || n_new < 0 || n_new > rb.n_tokens - row0 || n_new > max_new || len < 0 || len > max_context - n_new) {
        atomicOr(err, ERR_CAPACITY);
        n_new = 0;
        return false;
    }
    return true;
}
__device__ __forceinline__ bool batch_row(const RaggedBatch &rb, int b, int max_new, int max_context, int &row0, int &n_new, int &len, int *err)
{
    row0 = rb.cu ? rb.cu[b] : b * rb.uniform;
    n_new = rb.cu ? rb.cu[b + 1] - row0 : rb.uniform;
    len = (rb.lens ? rb.lens[b] : 0) + rb.first;
    return batch_row_fits(rb, max_new, max_context, row0, n_new, len, err);
}
// The same for the sequence b with `place` longer ones: thread blocks start in the order of their numbers, and long sequences that start last are what a
// launch ends with.  By the whole block (128 threads or more), of a batch with cu and lens of at most ORDER_MAX_B sequences; sm: ORDER_MAX_B + 4 words,
// 16-byte aligned.  Lengths count up to 2^24, sequences of one length go by their numbers; whatever the lengths hold, every sequence has one place.
constexpr int ORDER_MAX_B = 128;
__device__ __forceinline__ bool batch_row_by_length(const RaggedBatch &rb, int place, int max_new, int max_context, int &b, int &row0, int &n_new, int &len, int *err, uint32_t *sm)
{
    const int i = threadIdx.x;
    uint32_t mine = ORDER_MAX_B - 1 - i;
    if (i < ORDER_MAX_B) {
        if (i < rb.B) {
            row0 = rb.cu[i];
            n_new = rb.cu[i + 1] - row0;
            len = rb.lens[i];
            mine |= min((uint32_t)len + (uint32_t)n_new, 0xffffffu) << 7;
        }
        sm[i] = mine; // behind the last sequence: less than any
    }
    __syncthreads();
    if (i < rb.B) {
        int longer = 0;
        for (int k0 = 0; k0 < rb.B; k0 += 32) {
            uint4 u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = *(const uint4 *)(sm + k0 + 4 * k);
#pragma unroll
            for (int k = 0; k < 8; ++k) longer += (u[k].x > mine) + (u[k].y > mine) + (u[k].z > mine) + (u[k].w > mine);
        }
        if (longer == place) *(int4 *)(sm + ORDER_MAX_B) = make_int4(i, row0, n_new, len);
    }
    __syncthreads();
    const int4 row = *(const int4 *)(sm + ORDER_MAX_B);
    b = row.x; row0 = row.y; n_new = row.z; len = row.w;
    return batch_row_fits(rb, max_new, max_context, row0, n_new, len, err);
}

// Tiles of `per` packed rows that a sequence can have.  max_new is a host bound of up to 2^30, but no sequence has more rows than the tensors, which fit the
// GPU: in a launch of this many tiles the rows' numbers stay within 32 bits.
inline long row_tiles(const PagedAttnArgs &a, int per)
{
    return ((long)(a.max_new < a.rb.n_tokens ? a.max_new : a.rb.n_tokens) * a.group + per - 1) / per;
}

// What the weighted sum of a row is multiplied by.  Every query sees its own key, so a sum of 0 (all its scores -inf) has no softmax,
// and neither has one of NaN.
__device__ __forceinline__ float inverse_sum(float den) { return den > 0.f ? 1.f / den : __uint_as_float(0x7fc00000u); }

// A kernel's dynamic shared-memory limit, raised once per device (by any thread; twice does no harm).
struct SmemLimit {
    std::atomic<bool> done[64] = {};
    cudaError_t raise(const void *kernel, int bytes)
    {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess || (dev >= 0 && dev < 64 && done[dev])) return e;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
        return e;
    }
};

// slots non-null: row t goes to slot slots[t] = page id * page + row of the page (negative: nobody's), whatever rb says
cudaError_t launch_kv_write(const PagedKv &kv, const RaggedBatch &rb, const int32_t *slots, const void *k, const void *v, long k_stride,
                            long v_stride, int in_bf16, int *err, cudaStream_t st);
cudaError_t launch_kv_read(const PagedKv &kv, const RaggedBatch &rb, void *k, void *v, long k_stride, long v_stride, int out_bf16,
                           int *err, cudaStream_t st);

// float32 queries, or bf16 ones with head_dim 32
cudaError_t launch_paged_attention_general(const PagedAttnArgs &a, int q_bf16, cudaStream_t st);
// Key ranges that one thread-block cluster adds up in shared memory; more go through the workspace.
constexpr int PAGED_MAX_CLUSTER = 8;
// Longest sequence: positions and what is added to them (windows' ends, tiles) stay within 32 bits.
constexpr int PAGED_MAX_CONTEXT = 1 << 30;
// bf16 queries, head_dim 64 or 128, few rows (new tokens x query heads per KV head) per sequence and KV head
constexpr int PAGED_MAX_FEW_ROWS = 16;
cudaError_t launch_paged_attention_rows(const PagedAttnArgs &a, cudaStream_t st);
// The same over 4-bit pages, any number of rows.  stream: all sequences' keys dealt out evenly to the warps that fit the GPU, through part_o (stream4_workspace bytes).
cudaError_t launch_paged_attention_rows4(const PagedAttnArgs &a, int q_bf16, bool stream, cudaStream_t st);
constexpr int STREAM_MAX_B = 512; // sequences of such a call: every block sums up their lengths
int stream4_workers(int groups_of_8_rows);
size_t stream4_workspace(int rows, int head_dim);
// bf16 queries, head_dim 64 or 128, any number of rows
cudaError_t launch_paged_attention_tc(const PagedAttnArgs &a, cudaStream_t st);
// Chooses a kernel and launches it (and the merge).  part_o / part_ml: room for `part_splits` ranges of partial rows, or null and 0;
// more ranges than that are not made (a cluster's worth needs none).
cudaError_t run_paged_attention(PagedAttnArgs &a, int q_bf16, int part_splits, cudaStream_t st);
// Adds up the key ranges of a split launch.
cudaError_t launch_paged_merge(const PagedAttnArgs &a, int q_bf16, cudaStream_t st);

} // namespace spd
