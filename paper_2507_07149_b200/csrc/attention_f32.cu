// Attention for binary32 inputs, forward and the backward pass that recomputes the probabilities; and, for every type, the
// row statistics the backward pass starts from.
//
//   S = scale q k^T over the visible keys,  P = exp(S - L) with L = log sum exp S,  out = P v
//   delta = sum(grad_out * out),  dS = P (grad_out v^T - delta) scale
//   dq = dS k,  dk = dS^T q,  dv = P^T grad_out   (dk, dv summed over the query heads of a key head)
//
// One CTA per 64 rows of the tensor it produces: the forward and dq kernels hold 64 queries and walk the keys, the dk / dv
// kernel holds 64 keys of a key head and walks the queries of every head that reads it, so no sum crosses CTAs.  A thread
// owns 4 x 4 scores and 4 x (D / 16) outputs.  Products are binary32 fused multiply-adds: three TF32 products on the tensor
// cores (mma.sync) in their place came out 5 to 15 % faster, but carry 22 bits of each factor instead of 24.
// Bound: shared-memory reads (8 of 16 bytes per 64 multiply-adds of a thread) and, at D = 128, the eight warps per SM that
// its tiles leave room for: 25 TFLOP/s on 8 x 197 x 12 heads of 64.
#include "attention.cuh"

namespace daf {

constexpr int kGenThreads = 256;
constexpr int kRowThreads = 256;
constexpr uint32_t kRowsPerCta = 128;            // what the workspace's rows are padded to
constexpr int kTile = 64;
constexpr int kScorePitch = kTile + 4;

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

// rows [first, first + 64) of one head into dst[row][DP + 4], zero beyond `limit` rows and D columns
template <int DP>
__device__ __forceinline__ void load_tile(float *dst, const AttnTensor &t, uint32_t b, uint32_t h, uint32_t first, uint32_t limit, uint32_t D)
{
    const float *base = reinterpret_cast<const float *>(t.p) + t.sb * b + t.sh * h;
#pragma unroll 8
    for (int i = threadIdx.x; i < kTile * (DP / 4); i += kGenThreads) {
        const uint32_t r = i / (DP / 4), c = (i % (DP / 4)) * 4;
        float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (first + r < limit && c < D) x = __ldg(reinterpret_cast<const float4 *>(base + t.ss * (first + r) + c));
        *reinterpret_cast<float4 *>(dst + r * (DP + 4) + c) = x;
    }
}

__device__ __forceinline__ float dot4(const float4 &a, const float4 &b, float c)
{
    return __fmaf_rn(a.w, b.w, __fmaf_rn(a.z, b.z, __fmaf_rn(a.y, b.y, __fmaf_rn(a.x, b.x, c))));
}

// acc[i][j] = A[4 ty + i] . B[tx + 16 j]
template <int DP> __device__ __forceinline__ void product_nt(const float *A, const float *B, int ty, int tx, float (&acc)[4][4])
{
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) acc[i][j] = 0.0f;
#pragma unroll 4
    for (int d = 0; d < DP; d += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; i++) {
            a[i] = *reinterpret_cast<const float4 *>(A + (4 * ty + i) * (DP + 4) + d);
            b[i] = *reinterpret_cast<const float4 *>(B + (tx + 16 * i) * (DP + 4) + d);
        }
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) acc[i][j] = dot4(a[i], b[j], acc[i][j]);
    }
}

// acc[i][4 jj + e] += sum over k of W[4 ty + i][k] * B[k][64 jj + 4 tx + e]
template <int DP> __device__ __forceinline__ void product_nn(const float *W, const float *B, int ty, int tx, float (&acc)[4][DP / 16])
{
#pragma unroll 2
    for (int k = 0; k < kTile; k += 4) {
        float4 w[4];
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = *reinterpret_cast<const float4 *>(W + (4 * ty + i) * kScorePitch + k);
#pragma unroll
        for (int kk = 0; kk < 4; kk++) {
#pragma unroll
            for (int jj = 0; jj < DP / 64; jj++) {
                const float4 b = *reinterpret_cast<const float4 *>(B + (k + kk) * (DP + 4) + 64 * jj + 4 * tx);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float x = kk == 0 ? w[i].x : kk == 1 ? w[i].y : kk == 2 ? w[i].z : w[i].w;
                    acc[i][4 * jj] = __fmaf_rn(x, b.x, acc[i][4 * jj]);
                    acc[i][4 * jj + 1] = __fmaf_rn(x, b.y, acc[i][4 * jj + 1]);
                    acc[i][4 * jj + 2] = __fmaf_rn(x, b.z, acc[i][4 * jj + 2]);
                    acc[i][4 * jj + 3] = __fmaf_rn(x, b.w, acc[i][4 * jj + 3]);
                }
            }
        }
    }
}

// 64 rows of a thread block's result, times by[i]
template <int DP>
__device__ __forceinline__ void store_tile(const AttnTensor &t, uint32_t b, uint32_t h, uint32_t first, uint32_t limit, uint32_t D, int ty, int tx,
                                           const float (&acc)[4][DP / 16], const float (&by)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t r = first + 4 * ty + i;
        if (r >= limit) continue;
        const uint64_t at = t.sb * b + t.sh * h + t.ss * r;
#pragma unroll
        for (int jj = 0; jj < DP / 64; jj++) {
            const uint32_t c = 64 * jj + 4 * tx;
            if (c < D)
                *reinterpret_cast<float4 *>(reinterpret_cast<float *>(t.p) + at + c) =
                    make_float4(acc[i][4 * jj] * by[i], acc[i][4 * jj + 1] * by[i], acc[i][4 * jj + 2] * by[i], acc[i][4 * jj + 3] * by[i]);
        }
    }
}

// What the backward kernels need of each row, D / 8 lanes (rounded up to a power of two) per row, 128 rows of a head per
// CTA: -lse in units of log2, -inf for rows that see nothing and for the padding (their probabilities then come out as
// exp2(-inf) = 0), and -delta = -sum(grad_out * out).
template <typename T> __global__ void __launch_bounds__(kRowThreads) attention_rows_kernel(const __grid_constant__ AttnArgs a, uint32_t lanes, WorkspaceHeader *header)
{
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) header->status = 0u;
    const uint32_t lane = threadIdx.x % lanes, per = kRowThreads / lanes, bh = blockIdx.y, b = bh / a.H, h = bh - b * a.H;
    const uint32_t first = blockIdx.x * kRowsPerCta;
    const bool reads = lane * 8u < a.D;
    const T *const o = reinterpret_cast<const T *>(a.out.p) + a.out.sb * b + a.out.sh * h + lane * 8u;
    const T *const g = reinterpret_cast<const T *>(a.grad_out.p) + a.grad_out.sb * b + a.grad_out.sh * h + lane * 8u;
#pragma unroll 4
    for (uint32_t r = threadIdx.x / lanes; r < kRowsPerCta; r += per) {        // whole warps leave together
        const uint32_t i = first + r;
        float nl2 = -INFINITY, delta = 0.0f;
        if (i < a.Sq) {
            const float l = a.lse[(uint64_t)bh * a.Sq + i];
            if (l != -INFINITY) nl2 = -l * 1.4426950408889634f;
            if (reads) {
                float x[8], y[8];
                load8_any<T>(o + a.out.ss * i, x);
                load8_any<T>(g + a.grad_out.ss * i, y);
#pragma unroll
                for (int e = 0; e < 8; e++) delta = __fmaf_rn(x[e], y[e], delta);
            }
        }
        for (uint32_t d = lanes >> 1; d; d >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, d);
        if (lane == 0) {
            a.row_nl2[(uint64_t)bh * a.rows_padded + i] = nl2;
            a.row_ndelta[(uint64_t)bh * a.rows_padded + i] = -delta;
        }
    }
}

template <int DP>
__global__ void __launch_bounds__(kGenThreads) attention_dq_f32_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(16) float smem[];
    constexpr int TW = kTile * (DP + 4);
    float *const Q = smem, *const G = Q + TW, *const K = G + TW, *const V = K + TW, *const S = V + TW;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const uint32_t m0 = blockIdx.x * kTile, h = blockIdx.y % a.H, b = blockIdx.y / a.H;
    const uint32_t n = attn_length(a, b);
    load_tile<DP>(Q, a.q, b, h, m0, a.Sq, a.D);
    load_tile<DP>(G, a.grad_out, b, h, m0, a.Sq, a.D);
    float nl2[4], nd[4], o[4][DP / 16] = {};
    int limit[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint64_t w = ((uint64_t)b * a.H + h) * a.rows_padded + m0 + 4 * ty + i;
        nl2[i] = a.row_nl2[w];
        nd[i] = a.row_ndelta[w];
        limit[i] = attn_limit(a, n, (int)m0 + 4 * ty + i);
    }
    const int end = attn_limit(a, n, (int)(m0 + kTile < a.Sq ? m0 + kTile : a.Sq) - 1);
    for (int n0 = 0; n0 < end; n0 += kTile) {
        __syncthreads();
        load_tile<DP>(K, a.k, b, h / a.group, n0, n, a.D);
        load_tile<DP>(V, a.v, b, h / a.group, n0, n, a.D);
        __syncthreads();
        float s[4][4], e[4][4];
        product_nt<DP>(Q, K, ty, tx, s);
        product_nt<DP>(G, V, ty, tx, e);
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const float p = exp2f(__fmaf_rn(s[i][j], a.scale_log2, nl2[i]));
                S[(4 * ty + i) * kScorePitch + tx + 16 * j] = n0 + tx + 16 * j < limit[i] ? p * (e[i][j] + nd[i]) : 0.0f;
            }
        __syncwarp();
        product_nn<DP>(S, K, ty, tx, o);
    }
    const float by[4] = {a.scale, a.scale, a.scale, a.scale};
    store_tile<DP>(a.dq, b, h, m0, a.Sq, a.D, ty, tx, o, by);
}

template <int DP>
__global__ void __launch_bounds__(kGenThreads) attention_dkv_f32_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(16) float smem[];
    constexpr int TW = kTile * (DP + 4), SW = kTile * kScorePitch;
    float *const K = smem, *const V = K + TW, *const Q = V + TW, *const G = Q + TW, *const P = G + TW, *const S = P + SW;
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const uint32_t n0 = blockIdx.x * kTile, kh = blockIdx.y % a.Hkv, b = blockIdx.y / a.Hkv;
    const uint32_t n = attn_length(a, b);
    load_tile<DP>(K, a.k, b, kh, n0, n, a.D);
    load_tile<DP>(V, a.v, b, kh, n0, n, a.D);
    float dk[4][DP / 16] = {}, dv[4][DP / 16] = {};
    // the first query that sees key n0
    const int64_t from = a.causal ? (int64_t)n0 + (int64_t)a.Sq - (int64_t)a.Sk : 0;
    const uint32_t start = from > 0 ? (uint32_t)(from / kTile * kTile) : 0u;
    for (uint32_t h = kh * a.group; n0 < n && h < (kh + 1) * a.group; h++)
        for (uint32_t m0 = start; m0 < a.Sq; m0 += kTile) {
            __syncthreads();
            load_tile<DP>(Q, a.q, b, h, m0, a.Sq, a.D);
            load_tile<DP>(G, a.grad_out, b, h, m0, a.Sq, a.D);
            __syncthreads();
            float s[4][4], e[4][4];
            product_nt<DP>(K, Q, ty, tx, s);
            product_nt<DP>(V, G, ty, tx, e);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint64_t w = ((uint64_t)b * a.H + h) * a.rows_padded + m0 + tx + 16 * j;
                const float nl2 = a.row_nl2[w], nd = a.row_ndelta[w];
                const int limit = attn_limit(a, n, (int)m0 + tx + 16 * j);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const bool see = (int)n0 + 4 * ty + i < limit;
                    const float p = see ? exp2f(__fmaf_rn(s[i][j], a.scale_log2, nl2)) : 0.0f;
                    P[(4 * ty + i) * kScorePitch + tx + 16 * j] = p;
                    S[(4 * ty + i) * kScorePitch + tx + 16 * j] = p * (e[i][j] + nd);
                }
            }
            __syncwarp();
            product_nn<DP>(P, G, ty, tx, dv);
            product_nn<DP>(S, Q, ty, tx, dk);
        }
    const float one[4] = {1.0f, 1.0f, 1.0f, 1.0f}, by[4] = {a.scale, a.scale, a.scale, a.scale};
    store_tile<DP>(a.dv, b, kh, n0, a.Sk, a.D, ty, tx, dv, one);
    store_tile<DP>(a.dk, b, kh, n0, a.Sk, a.D, ty, tx, dk, by);
}

template <typename K, typename... More>
static daf_status launch_f32(K kernel, uint32_t rows, uint32_t heads, uint32_t B, int smem, const AttnArgs &a, cudaStream_t s, More... more)
{
    int ctas = 0;                                                  // asked for the shared-memory limit it raises
    if (persistent_ctas(reinterpret_cast<const void *>(kernel), kGenThreads, smem, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    kernel<<<dim3((rows + kTile - 1) / kTile, heads * B), kGenThreads, smem, s>>>(a, more...);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

constexpr int tile_bytes(int DP, int tiles, int scores) { return (tiles * kTile * (DP + 4) + scores * kTile * kScorePitch) * 4; }

template <int DP> static daf_status backward(const AttnArgs &a, cudaStream_t s)
{
    const daf_status st = launch_f32(&attention_dq_f32_kernel<DP>, a.Sq, a.H, a.B, tile_bytes(DP, 4, 1), a, s);
    return st != DAF_OK ? st : launch_f32(&attention_dkv_f32_kernel<DP>, a.Sk, a.Hkv, a.B, tile_bytes(DP, 4, 2), a, s);
}

daf_status attn_backward_f32(const AttnArgs &a, cudaStream_t s) { return backward<128>(a, s); }

daf_status attn_rows(uint32_t dtype, const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s)
{
    uint32_t lanes = 1;
    while (lanes * 8u < a.D) lanes *= 2u;
    const dim3 grid(a.rows_padded / kRowsPerCta, a.B * a.H);
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
