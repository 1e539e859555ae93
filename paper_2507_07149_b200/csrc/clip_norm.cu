// Global gradient norm over a set of tensors, and clipping by it: the last step before an optimizer reads the gradients.
//
//   norm = sqrt(sum over all tensors and elements of g^2),   out = RNE_T(g * min(1, max_norm / (norm + eps)))
//
// Two launches.  clip_sum_kernel reads every gradient once; CTA c takes the chunks c, c + grid, ... of the set and leaves
// ONE binary32 partial sum of squares.  clip_scale_kernel adds up the partials (every CTA for itself, all in the same
// fixed order and in binary64, so no atomic, no counter and no order that changes from call to call), and writes the
// scaled tensors; where the factor is 1 and a tensor is clipped in place there is nothing to write.  Bound: HBM, one
// read for the norm, one read and one write for the scaling; sets below the L2's size are read from HBM only once.
//
// Tensors of different element types share a call: the type is a property of the table's entry.  Pointers need the
// alignment of their element only: a chunk is cut into a ragged head, 16-byte units and a ragged tail.
#include "common.cuh"

namespace daf {

constexpr int kClipThreads = 512;
constexpr int kClipTensors = 512;               // tensors per launch: 16 KiB of kernel arguments
constexpr uint32_t kClipChunk = 16384;          // elements of a chunk
constexpr uint32_t kClipCtas = 1024;            // partial sums per launch, at most

struct ClipTensor {
    const void *in;
    void *out;
    uint64_t numel;
    uint32_t first_chunk, dtype;
};
struct ClipTable {
    ClipTensor t[kClipTensors];
    uint32_t n, n_chunks;
};

template <typename T> struct ClipElem;
template <> struct ClipElem<float> {
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct ClipElem<__half> {
    static __device__ __forceinline__ float get(__half v) { return __half2float(v); }
    static __device__ __forceinline__ __half put(float v) { return __float2half_rn(v); }
};
template <> struct ClipElem<__nv_bfloat16> {
    static __device__ __forceinline__ float get(__nv_bfloat16 v) { return __bfloat162float(v); }
    static __device__ __forceinline__ __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
};

// Elements of a chunk ahead of the first 16-byte boundary.
template <typename T> __device__ __forceinline__ uint32_t head_elems(const void *p, uint32_t n)
{
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T);
    const uint32_t h = off ? 16u / sizeof(T) - off : 0u;
    return h < n ? h : n;
}

template <typename T> __device__ __forceinline__ float unit_sum_sq(const uint4 &u, float acc)
{
    float x[8];
    Elem<T>::widen8(u, x);
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); i++) acc = __fmaf_rn(x[i], x[i], acc);
    return acc;
}

template <typename T> __device__ float chunk_sum_sq(const T *p, uint32_t n)
{
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const uint32_t head = head_elems<T>(p, n), per = 16u / sizeof(T), units = (n - head) / per;
    const uint4 *v = reinterpret_cast<const uint4 *>(p + head);
    uint32_t u = threadIdx.x;
    for (; u + 3u * kClipThreads < units; u += 4u * kClipThreads) {
        uint4 x[4];
#pragma unroll
        for (int j = 0; j < 4; j++) x[j] = __ldg(v + u + j * kClipThreads);
#pragma unroll
        for (int j = 0; j < 4; j++) acc[j] = unit_sum_sq<T>(x[j], acc[j]);
    }
    for (; u < units; u += kClipThreads) acc[0] = unit_sum_sq<T>(__ldg(v + u), acc[0]);
    const uint32_t tail = head + units * per;
    if (threadIdx.x < head) {
        const float x = ClipElem<T>::get(p[threadIdx.x]);
        acc[1] = __fmaf_rn(x, x, acc[1]);
    }
    if (threadIdx.x < n - tail) {
        const float x = ClipElem<T>::get(p[tail + threadIdx.x]);
        acc[2] = __fmaf_rn(x, x, acc[2]);
    }
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

template <typename T> __device__ void chunk_scale(const T *p, T *q, uint32_t n, float by)
{
    constexpr uint32_t per = 16u / sizeof(T);
    // units need both sides at the same place within 16 bytes; otherwise element by element
    const bool same = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15u) == 0;
    const uint32_t head = same ? head_elems<T>(p, n) : n, units = (n - head) / per, tail = head + units * per;
    const uint4 *v = reinterpret_cast<const uint4 *>(p + head);
    uint4 *w = reinterpret_cast<uint4 *>(q + head);
    for (uint32_t u0 = threadIdx.x; u0 < units; u0 += 4u * kClipThreads) {
        uint4 x[4];
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (u0 + j * kClipThreads < units) x[j] = v[u0 + j * kClipThreads];
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (u0 + j * kClipThreads < units) {
                T e[per];
                *reinterpret_cast<uint4 *>(e) = x[j];
#pragma unroll
                for (uint32_t i = 0; i < per; i++) e[i] = ClipElem<T>::put(ClipElem<T>::get(e[i]) * by);
                w[u0 + j * kClipThreads] = *reinterpret_cast<uint4 *>(e);
            }
    }
    for (uint32_t i = threadIdx.x; i < head; i += kClipThreads) q[i] = ClipElem<T>::put(ClipElem<T>::get(p[i]) * by);
    if (threadIdx.x < n - tail) q[tail + threadIdx.x] = ClipElem<T>::put(ClipElem<T>::get(p[tail + threadIdx.x]) * by);
}

__device__ __forceinline__ double clip_block_sum(double v, double *s_part)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / 32; w++) v += s_part[w];
    return v;
}

__global__ void __launch_bounds__(kClipThreads) clip_sum_kernel(const __grid_constant__ ClipTable tab, float *partial)
{
    __shared__ double s_part[kClipThreads / 32];
    float acc = 0.0f;
    uint32_t t = 0;
    for (uint32_t c = blockIdx.x; c < tab.n_chunks; c += gridDim.x) {
        while (t + 1u < tab.n && c >= tab.t[t + 1u].first_chunk) t++;
        const uint64_t at = (uint64_t)(c - tab.t[t].first_chunk) * kClipChunk, left = tab.t[t].numel - at;
        const uint32_t n = left < kClipChunk ? (uint32_t)left : kClipChunk;
        if (tab.t[t].dtype == DAF_F32) acc += chunk_sum_sq(reinterpret_cast<const float *>(tab.t[t].in) + at, n);
        else if (tab.t[t].dtype == DAF_F16) acc += chunk_sum_sq(reinterpret_cast<const __half *>(tab.t[t].in) + at, n);
        else acc += chunk_sum_sq(reinterpret_cast<const __nv_bfloat16 *>(tab.t[t].in) + at, n);
    }
    const double sum = clip_block_sum((double)acc, s_part);
    if (threadIdx.x == 0) partial[blockIdx.x] = (float)sum;
}

// partial: all launches' partial sums, n_partial of them.  write: whether scaled tensors are wanted at all.
__global__ void __launch_bounds__(kClipThreads, 2)
clip_scale_kernel(const __grid_constant__ ClipTable tab, const float *partial, uint32_t n_partial, float max_norm, float eps,
                  float *norm_out, uint32_t write)
{
    __shared__ double s_part[kClipThreads / 32];
    double sum = 0.0;
    for (uint32_t i = threadIdx.x; i < n_partial; i += kClipThreads) sum += (double)partial[i];
    const float norm = (float)sqrt(clip_block_sum(sum, s_part));
    const float ratio = __fdiv_rn(max_norm, norm + eps);
    const float by = ratio > 1.0f ? 1.0f : ratio;                 // a norm that is not a number stays one
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = norm;
    if (!write) return;
    // last chunk first: what the norm's pass read last is still in L2
    uint32_t t = tab.n - 1u;
    for (uint32_t i = blockIdx.x; i < tab.n_chunks; i += gridDim.x) {
        const uint32_t c = tab.n_chunks - 1u - i;
        while (c < tab.t[t].first_chunk) t--;
        if (by == 1.0f && tab.t[t].in == tab.t[t].out) continue;
        const uint64_t at = (uint64_t)(c - tab.t[t].first_chunk) * kClipChunk, left = tab.t[t].numel - at;
        const uint32_t n = left < kClipChunk ? (uint32_t)left : kClipChunk;
        if (tab.t[t].dtype == DAF_F32)
            chunk_scale(reinterpret_cast<const float *>(tab.t[t].in) + at, reinterpret_cast<float *>(tab.t[t].out) + at, n, by);
        else if (tab.t[t].dtype == DAF_F16)
            chunk_scale(reinterpret_cast<const __half *>(tab.t[t].in) + at, reinterpret_cast<__half *>(tab.t[t].out) + at, n, by);
        else
            chunk_scale(reinterpret_cast<const __nv_bfloat16 *>(tab.t[t].in) + at,
                        reinterpret_cast<__nv_bfloat16 *>(tab.t[t].out) + at, n, by);
    }
}

// The next launch's table: tensors from *next on, as many as fit (empty ones are left out).
static daf_status fill_table(ClipTable *tab, uint32_t n, const uint32_t *dtypes, const void *const *d_in, void *const *d_out,
                             const uint64_t *numel, uint32_t *next)
{
    tab->n = 0;
    uint64_t chunks = 0;
    for (; *next < n && tab->n < (uint32_t)kClipTensors; ++*next) {
        const uint32_t i = *next;
        if (numel[i] == 0) continue;
        const uint64_t mine = (numel[i] + kClipChunk - 1u) / kClipChunk;
        if (chunks + mine > 0x7FFFFFFFull) {
            if (tab->n == 0) return DAF_ERR_SHAPE;                // more than 2^45 elements
            break;
        }
        tab->t[tab->n++] = {d_in[i], d_out ? d_out[i] : nullptr, numel[i], (uint32_t)chunks, dtypes[i]};
        chunks += mine;
    }
    tab->n_chunks = (uint32_t)chunks;
    return DAF_OK;
}

}  // namespace daf

using namespace daf;

extern "C" uint64_t daf_clip_norm_workspace(uint32_t n)
{
    // a launch takes kClipTensors tensors, or fewer where their chunks pass 2^31: then at least one
    return ((uint64_t)(n / kClipTensors) + 2u) * kClipCtas * sizeof(float);
}

extern "C" daf_status daf_clip_norm_batch(uint32_t n, const uint32_t *dtypes, const void *const *d_in, void *const *d_out,
                                          const uint64_t *numel, float max_norm, float eps, float *d_norm, void *d_workspace,
                                          uint64_t workspace_bytes, daf_stream stream)
{
    if ((n && (!dtypes || !d_in || !numel)) || !d_norm || !d_workspace || (reinterpret_cast<uintptr_t>(d_norm) & 3u) ||
        (reinterpret_cast<uintptr_t>(d_workspace) & 15u) || !(max_norm >= 0.0f) || !(eps >= 0.0f))
        return DAF_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < n; i++) {
        if (dtypes[i] > DAF_BF16) return DAF_ERR_INVALID_ARG;
        const uintptr_t mask = dtypes[i] == DAF_F32 ? 3u : 1u;
        if (numel[i] && (!d_in[i] || (reinterpret_cast<uintptr_t>(d_in[i]) & mask))) return DAF_ERR_INVALID_ARG;
        if (numel[i] && d_out && (!d_out[i] || (reinterpret_cast<uintptr_t>(d_out[i]) & mask))) return DAF_ERR_INVALID_ARG;
    }
    if (workspace_bytes < daf_clip_norm_workspace(n)) return DAF_ERR_CAPACITY;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    float *partial = reinterpret_cast<float *>(d_workspace);
    int sum_ctas = 0, scale_ctas = 0;
    if (persistent_ctas(reinterpret_cast<const void *>(&clip_sum_kernel), kClipThreads, 0, &sum_ctas) != cudaSuccess ||
        persistent_ctas(reinterpret_cast<const void *>(&clip_scale_kernel), kClipThreads, 0, &scale_ctas) != cudaSuccess)
        return DAF_ERR_CUDA;
    if (sum_ctas > (int)kClipCtas) sum_ctas = (int)kClipCtas;
    const uint64_t room = workspace_bytes / sizeof(float);
    ClipTable tab;
    uint32_t n_partial = 0;
    for (uint32_t next = 0; next < n;) {
        const daf_status st = fill_table(&tab, n, dtypes, d_in, d_out, numel, &next);
        if (st != DAF_OK) return st;
        if (tab.n == 0) break;
        const uint32_t grid = tab.n_chunks < (uint32_t)sum_ctas ? tab.n_chunks : (uint32_t)sum_ctas;
        if (n_partial + grid > room) return DAF_ERR_CAPACITY;
        clip_sum_kernel<<<grid, kClipThreads, 0, s>>>(tab, partial + n_partial);
        n_partial += grid;
    }
    uint32_t next = 0;
    bool first = true;
    do {                                                          // once at least: it also writes the norm
        const daf_status st = fill_table(&tab, n, dtypes, d_in, d_out, numel, &next);
        if (st != DAF_OK) return st;
        if (tab.n == 0 && !first) break;
        const uint32_t write = d_out && tab.n ? 1u : 0u;
        const uint32_t grid = !write ? 1u : tab.n_chunks < (uint32_t)scale_ctas ? tab.n_chunks : (uint32_t)scale_ctas;
        clip_scale_kernel<<<grid, kClipThreads, 0, s>>>(tab, partial, n_partial, max_norm, eps, first ? d_norm : nullptr, write);
        first = false;
    } while (d_out && next < n);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
