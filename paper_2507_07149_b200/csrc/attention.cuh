// What the attention kernels and their entry points share.
#pragma once
#include <cuda.h>

#include "common.cuh"

namespace daf {

// [batch, sequence, head, element] with the last one contiguous; strides in elements.
struct AttnTensor {
    void *p;
    uint64_t sb, ss, sh;
};

// Division by a number known on the host, by a product and a shift (Granlund and Montgomery, PLDI'94): n < 2^31.
struct FastDiv {
    uint32_t d, mul, shift;
    __host__ void set(uint32_t by)
    {
        d = by;
        shift = 0;
        while ((1ull << shift) < by) shift++;
        mul = (uint32_t)((((1ull << shift) - by) << 32) / by) + 1u;
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};

struct AttnArgs {
    AttnTensor q, k, v, out, grad_out, dq, dk, dv;
    float *lse;                  // [B, H, Sq]: natural logarithm of each row's sum of exponentials, -inf for a row that sees no key
    const int32_t *lengths;      // keys of each sequence, or null
    float *row_nl2, *row_ndelta; // backward workspace, [B, H, rows_padded]: see attention_rows_kernel
    // float16 backward: squared norms of the rows of grad_out, [B, H, rows_padded], and [B, Hkv] each their maximum over the rows
    // that meet a key head and a bound of v's
    float *row_norm2, *grad_max, *value_max;
    unsigned int *device_status; // see record_error
    uint32_t B, Sq, Sk, H, Hkv, D, group, causal, rows_padded;
    float scale, scale_log2;     // scale_log2 = scale * log2(e)
};

// Keys of sequence b.
__device__ __forceinline__ uint32_t attn_length(const AttnArgs &a, uint32_t b)
{
    if (!a.lengths) return a.Sk;
    const int n = __ldg(a.lengths + b);
    return n < 0 ? 0u : (uint32_t)n < a.Sk ? (uint32_t)n : a.Sk;
}
// Keys [0, limit) are visible to query i of a sequence with n keys.
__device__ __forceinline__ int attn_limit(const AttnArgs &a, uint32_t n, int i)
{
    if (!a.causal) return (int)n;
    const int c = i + 1 + (int)a.Sk - (int)a.Sq;
    return c < (int)n ? c : (int)n;
}

__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// binary32 inputs in three bfloat16 planes (at `planes_at`, attn_planes_workspace bytes)
uint64_t attn_planes_workspace(const AttnArgs &a, bool backward);
daf_status attn_forward_planes(const AttnArgs &a, char *planes_at, WorkspaceHeader *header, cudaStream_t s);
daf_status attn_backward_planes(const AttnArgs &a, char *planes_at, WorkspaceHeader *header, cudaStream_t s);
// float16 backward: P is held 2^8 times its size, so that probabilities down to 2^-22 keep their bits.
constexpr float kHalfLift = 8.0f;
daf_status attn_rows(uint32_t dtype, const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s);
daf_status attn_zero(uint32_t dtype, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D, cudaStream_t s);
// Into how many runs of key blocks a 16-bit forward call cuts each of its row tiles: 1, or as many as fill a B200 where the
// tiles alone leave half of it idle and eight blocks or more are walked.  (4 x 43 queries over 4740 keys, one head of 72: 65.5 us
// on 4 CTAs, 21.5 on 148.)
uint32_t attn_splits(const AttnArgs &a);
template <typename T> daf_status attn_forward_tc(const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s);

// Map of a tensor for copies of `rows` rows times 64 elements of one head; false if the driver refuses it.
bool attn_tensor_map(CUtensorMap *map, bool bf16, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D, uint32_t rows);
// The same for storing 32 rows times 32 elements.
bool attn_store_map(CUtensorMap *map, bool bf16, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D);

template <typename T> daf_status attn_backward_tc(const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s);

}  // namespace daf
