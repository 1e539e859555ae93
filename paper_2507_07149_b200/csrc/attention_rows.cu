// What attention's backward kernels of every type share: the row statistics they start from, and gradients that are zero.
#include "attention.cuh"

namespace daf {

constexpr int kRowThreads = 256;
constexpr uint32_t kRowsPerCta = 128;            // what the workspace's rows are padded to

// eight elements from a 16-byte boundary
template <typename T> __device__ __forceinline__ void load8_any(const void *p, float (&x)[8])
{
    const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p));
    Elem<T>::widen8(u, x);
    if (Elem<T>::kBytes == 4) {
        const float4 w = __ldg(reinterpret_cast<const float4 *>(p) + 1);
        x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    }
}

// What the backward kernels need of each row, D / 8 lanes (rounded up to a power of two) per row, 128 rows of a head per
// CTA: -lse in units of log2, -inf for rows that see nothing and for the padding (their probabilities then come out as
// exp2(-inf) = 0), and -delta = -sum(grad_out * out).  float16 also notes |grad_out|^2 of the row and the largest one of a key
// head's readers, rows that see nothing left out, and a bound of a key head's |v|^2, D times the largest square (maxima of
// non-negative floats by their bits: the order of the atomics changes nothing).  Reading v for that costs float16 calls 1 to 4 %
// (16 x 509 tokens, 16 heads of 80: 145 -> 148 us); CTAs of their own for v 8 %.
template <typename T> __global__ void __launch_bounds__(kRowThreads) attention_rows_kernel(const __grid_constant__ AttnArgs a, uint32_t lanes, WorkspaceHeader *header)
{
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) header->status = 0u;
    const uint32_t lane = threadIdx.x % lanes, per = kRowThreads / lanes, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H;
    const uint32_t first = blockIdx.x * kRowsPerCta;
    const bool reads = lane * 8u < a.D;
    constexpr bool F16 = __is_same(T, __half);
    float most = 0.0f;
    // the same rows of v, by the first of the query heads that read them
    if (F16 && first < a.Sk && h % a.group == 0) {
        const uint32_t n = attn_length(a, b), head = b * a.Hkv + h / a.group;
        const T *const v = reinterpret_cast<const T *>(a.v.p) + a.v.sb * b + a.v.sh * (h / a.group) + lane * 8u;
        uint32_t two = 0u;                                         // the largest |v|, by the bits, in each half
#pragma unroll 8
        for (uint32_t r = first + threadIdx.x / lanes; r < first + kRowsPerCta; r += per)
            if (r < n && reads) {
                const uint4 u = __ldg(reinterpret_cast<const uint4 *>(v + a.v.ss * r));
                two = __vmaxu2(__vmaxu2(two, u.x & 0x7FFF7FFFu), u.y & 0x7FFF7FFFu);
                two = __vmaxu2(__vmaxu2(two, u.z & 0x7FFF7FFFu), u.w & 0x7FFF7FFFu);
            }
        const uint32_t top = __reduce_max_sync(0xffffffffu, __vmaxu2(two, two >> 16) & 0xFFFFu);
        const float largest = __half2float(__ushort_as_half((unsigned short)top));
        if ((threadIdx.x & 31u) == 0) atomicMax(reinterpret_cast<uint32_t *>(a.value_max) + head, __float_as_uint((float)a.D * largest * largest));
    }
    if (F16 && first >= a.rows_padded) return;
    const T *const o = reinterpret_cast<const T *>(a.out.p) + a.out.sb * b + a.out.sh * h + lane * 8u;
    const T *const g = reinterpret_cast<const T *>(a.grad_out.p) + a.grad_out.sb * b + a.grad_out.sh * h + lane * 8u;
#pragma unroll 4
    for (uint32_t r = threadIdx.x / lanes; r < kRowsPerCta; r += per) {        // whole warps leave together
        const uint32_t i = first + r;
        float nl2 = -INFINITY, delta = 0.0f, norm = 0.0f;
        if (i < a.Sq) {
            const float l = a.lse[(uint64_t)bh * a.Sq + i];
            if (l != -INFINITY) nl2 = -l * 1.4426950408889634f + (F16 ? kHalfLift : 0.0f);
            if (reads) {
                float x[8], y[8];
                load8_any<T>(o + a.out.ss * i, x);
                load8_any<T>(g + a.grad_out.ss * i, y);
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    delta = __fmaf_rn(x[e], y[e], delta);
                    if (F16) norm = __fmaf_rn(y[e], y[e], norm);
                }
            }
        }
        for (uint32_t d = lanes >> 1; d; d >>= 1) {
            delta += __shfl_xor_sync(0xffffffffu, delta, d);
            if (F16) norm += __shfl_xor_sync(0xffffffffu, norm, d);
        }
        if (F16 && nl2 == -INFINITY) norm = 0.0f;
        most = fmaxf(most, norm);
        if (lane == 0) {
            if (F16) a.row_norm2[(uint64_t)bh * a.rows_padded + i] = norm;
            a.row_nl2[(uint64_t)bh * a.rows_padded + i] = nl2;
            a.row_ndelta[(uint64_t)bh * a.rows_padded + i] = -delta;
        }
    }
    if (F16) {
        const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
        if ((threadIdx.x & 31u) == 0) atomicMax(reinterpret_cast<uint32_t *>(a.grad_max) + b * a.Hkv + h / a.group, top);
    }
}

daf_status attn_rows(uint32_t dtype, const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s)
{
    uint32_t lanes = 1;
    while (lanes * 8u < a.D) lanes *= 2u;
    const uint32_t tiles = a.rows_padded / kRowsPerCta, key_tiles = dtype == DAF_F16 ? (a.Sk + kRowsPerCta - 1u) / kRowsPerCta : 0u;
    const dim3 grid(tiles > key_tiles ? tiles : key_tiles, a.B * a.H);
    if (dtype == DAF_F32) attention_rows_kernel<float><<<grid, kRowThreads, 0, s>>>(a, lanes, header);
    else if (dtype == DAF_F16) attention_rows_kernel<__half><<<grid, kRowThreads, 0, s>>>(a, lanes, header);
    else attention_rows_kernel<__nv_bfloat16><<<grid, kRowThreads, 0, s>>>(a, lanes, header);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

// Gradients of a call without queries (dk, dv) or without keys (dq): zero.
__global__ void __launch_bounds__(kRowThreads) attention_zero_kernel(AttnTensor t, uint32_t S, uint32_t H, uint32_t row_bytes, uint32_t elem_bytes, uint64_t units)
{
    const uint32_t per_row = row_bytes / 16u;
    for (uint64_t u = (uint64_t)blockIdx.x * kRowThreads + threadIdx.x; u < units; u += (uint64_t)gridDim.x * kRowThreads) {
        const uint64_t r = u / per_row, h = r % H, i = r / H % S, b = r / H / S;
        *reinterpret_cast<uint4 *>(reinterpret_cast<char *>(t.p) + (t.sb * b + t.ss * i + t.sh * h) * elem_bytes + (u - r * per_row) * 16u) = make_uint4(0u, 0u, 0u, 0u);
    }
}
daf_status attn_zero(uint32_t dtype, const AttnTensor &t, uint32_t B, uint32_t S, uint32_t H, uint32_t D, cudaStream_t s)
{
    const uint32_t bytes = dtype == DAF_F32 ? 4u : 2u;
    const uint64_t units = (uint64_t)B * S * H * D * bytes / 16u, grid = (units + kRowThreads - 1u) / kRowThreads;
    if (!units) return DAF_OK;
    attention_zero_kernel<<<(uint32_t)(grid < 4096u ? grid : 4096u), kRowThreads, 0, s>>>(t, S, H, D * bytes, bytes, units);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

}  // namespace daf
