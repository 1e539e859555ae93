// The join between two blocks of a transformer: the block's output goes through its gate and residual scale into the
// residual stream, and the next block's norm is taken while the row is at hand.
//
//   u = norm(y) w1 + b1   (post norm; u = y without one)          norm(t) = (t - mean) r,  r = 1 / sqrt(var + eps)
//   z = x + a g u                                                 (kind "rms": mean counts as 0)
//   h = norm(z) w + b
//
// Backward, from z and y (the statistics are recomputed from the rows, nothing else is kept), G(t) standing for the
// gradient of a norm, r (t - avg t - that avg(t that)), the middle term only for layer norms:
//
//   dx = gz + G(gh w),  du = a dx,  dy = g du  or  G(g du w1),  dw = sum gh zhat,  db = sum gh,  dg = sum du u,
//   dw1 = sum g du yhat,  db1 = sum g du
//
// One thread owns eight columns of a row (one 16- or 32-byte access per tensor), ceil(C / 8) threads (rounded up to
// warps; 8 or 16 lanes for the narrowest rows) own a row, and a CTA holds as many rows ("slots") as fit its threads.
// Row sums: shuffles, then one meeting of the slot's warps per pair of sums.  The backward kernel keeps the column sums
// of its rows in registers and leaves one partial row per CTA; a second kernel adds the partials in a fixed order (no
// atomics: the same inputs give the same bits).  The next row's loads are issued before the current row's arithmetic.
// Bound: HBM, four tensors of the stream's size forward, six backward.
#include "common.cuh"
#include "pairs.cuh"

namespace daf {

constexpr int kJoinThreads = 512;            // threads of a CTA for rows of at most 4096 columns
constexpr int kJoinWide = 1024;              // for wider rows: one row per CTA
constexpr uint32_t kJoinMaxWidth = 8192;
constexpr uint32_t kJoinCtas = 296;          // CTAs of the backward kernel, at most: what the workspace is sized for
constexpr int kSums = 5;                     // column sums: weight, bias, post weight, post bias, gate

struct JoinArgs {
    const void *x, *y, *weight, *bias, *gate, *post_weight, *post_bias;   // backward: x is z
    const void *grad_z, *grad_h;
    void *out_a, *out_b;                                                  // z, h; backward: dx, dy
    float *partial, *gate_partial;                                        // [CTA][4][C] and [group * CTAs per group][C]
    void *grad_gate;                                                      // written directly with one CTA per group
    uint64_t rows, rows_per_gate;
    uint32_t C, tpr, slots, gates, per_group;
    float a, eps, inv_c;
    uint32_t layer, param_f32;
};

__device__ __forceinline__ void to_pairs(const float (&f)[8], uint64_t (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = pair(f[2 * i], f[2 * i + 1]);
}
template <typename T> __device__ __forceinline__ void store_pairs(void *p, const uint64_t (&x)[4])
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; i++) unpair(x[i], f[2 * i], f[2 * i + 1]);
    Elem<T>::store8(p, f);
}

// The next rows of a thread's eight columns of N tensors, DEPTH rows deep: each thread copies its own pieces into its own
// places of shared memory and reads them back itself, so no thread waits for another.  One row ahead in registers left
// the kernels waiting for memory (backward, 12608 x 768 bfloat16: 36 us; four rows ahead: see the kernel).
template <typename T, int N, int DEPTH, int THREADS> struct RowPipe {
    static constexpr int kDepth = DEPTH;
    static constexpr int kParts = Elem<T>::kBytes / 2;            // 16-byte pieces of eight elements
    static constexpr uint32_t kBytes = DEPTH * N * kParts * THREADS * 16u;
    uint4 *at;
    uint32_t stage;
    __device__ __forceinline__ void init(void *smem)
    {
        at = reinterpret_cast<uint4 *>(smem) + threadIdx.x;
        stage = 0;
    }
    __device__ __forceinline__ uint4 *place(int t, int part) const { return at + ((stage * N + t) * kParts + part) * THREADS; }
    // the pieces of the row that will be read DEPTH turns from now (nothing for a row that is not there)
    __device__ __forceinline__ void fetch(const char *const (&src)[N], uint64_t offset, bool there)
    {
        if (there) {
#pragma unroll
            for (int t = 0; t < N; t++)
                if (src[t]) {
#pragma unroll
                    for (int k = 0; k < kParts; k++)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(place(t, k))),
                                     "l"(src[t] + offset + 16 * k) : "memory");
                }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
    }
    __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory"); }
    __device__ __forceinline__ void get(int t, const char *const (&)[N], uint64_t, bool there, uint64_t (&x)[4]) const
    {
        x[0] = x[1] = x[2] = x[3] = 0ull;
        if (!there) return;
        float f[8];
        const uint4 u = *place(t, 0);
        Elem<T>::widen8(u, f);
        if (kParts == 2) {
            const uint4 v = *place(t, kParts - 1);
            f[4] = __uint_as_float(v.x); f[5] = __uint_as_float(v.y); f[6] = __uint_as_float(v.z); f[7] = __uint_as_float(v.w);
        }
        to_pairs(f, x);
    }
};
// No depth: rows are loaded when they are needed.
template <typename T, int N, int THREADS> struct RowPipe<T, N, 0, THREADS> {
    static constexpr int kDepth = 0;
    static constexpr uint32_t kBytes = 0;
    __device__ __forceinline__ void init(void *) {}
    __device__ __forceinline__ void fetch(const char *const (&)[N], uint64_t, bool) {}
    __device__ __forceinline__ void wait() const {}
    __device__ __forceinline__ void get(int t, const char *const (&src)[N], uint64_t offset, bool there, uint64_t (&x)[4]) const
    {
        x[0] = x[1] = x[2] = x[3] = 0ull;
        if (!there) return;
        float f[8];
        Elem<T>::load8(src[t] + offset, f);
        to_pairs(f, x);
    }
};
// Depths that fit shared memory: two CTAs per SM forward; one CTA backward, beside the wide kernel's 160 KiB of column sums
// (which leave no room for binary32 rows).
template <typename T, int THREADS> using ForwardPipe = RowPipe<T, 2, THREADS == kJoinThreads ? (Elem<T>::kBytes == 2 ? 4 : 3) : 2, THREADS>;
template <typename T, int THREADS> using BackwardPipe = RowPipe<T, 4, THREADS == kJoinThreads ? (Elem<T>::kBytes == 2 ? 4 : 3) : Elem<T>::kBytes == 2, THREADS>;

// Eight parameters of a vector (binary32 or the activations' type).
template <typename T> __device__ __forceinline__ void param8(const void *p, uint64_t at, uint32_t f32, uint64_t (&x)[4])
{
    if (f32) {
        const ulonglong2 *q = reinterpret_cast<const ulonglong2 *>(reinterpret_cast<const float *>(p) + at);
        const ulonglong2 u = __ldg(q), w = __ldg(q + 1);
        x[0] = u.x; x[1] = u.y; x[2] = w.x; x[3] = w.y;
    } else if (Elem<T>::kBytes == 2) {
        float f[8];
        Elem<T>::widen8(__ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) + at * Elem<T>::kBytes)), f);
        to_pairs(f, x);
    }
}

__device__ __forceinline__ void store_param(void *p, uint64_t at, uint32_t f32, uint32_t bf16, float v)
{
    if (f32) reinterpret_cast<float *>(p)[at] = v;
    else if (bf16) reinterpret_cast<__nv_bfloat16 *>(p)[at] = __float2bfloat16_rn(v);
    else reinterpret_cast<__half *>(p)[at] = __float2half_rn(v);
}

// Sums of two or four values over the threads of a slot.  Within a warp the first exchanges leave one of the sums in each
// half (quarter) of the warp, so that the remaining steps serve all; a slot of several warps meets once, and every warp
// adds up the warps' sums the same way.  Two buffers in turn: a warp that writes for sum k + 2 has met, at sum k + 1,
// every warp that still read sum k.
struct RowSums {
    float *buf;                                   // [2][4][32]
    uint32_t tpr, slot, parity;
    // v: sum number lane / span of the warp, complete within each span of lanes; afterwards that of the slot
    template <int SPAN> __device__ __forceinline__ void meet(float &v)
    {
        const uint32_t n = tpr >> 5, lane = threadIdx.x & 31u, i = lane % SPAN;
        float *const b = buf + parity * 128u + lane / SPAN * 32u + slot * n;
        if (i == 0) b[(threadIdx.x >> 5) - slot * n] = v;
        asm volatile("bar.sync %0, %1;" ::"r"(slot + 1u), "r"(tpr) : "memory");
        v = i < n ? b[i] : 0.0f;
#pragma unroll
        for (uint32_t k = SPAN; k < 32u; k += SPAN)
            if (n > k && i + k < n) v += b[i + k];
#pragma unroll
        for (int d = SPAN / 2; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        parity ^= 1u;
    }
    __device__ __forceinline__ void operator()(float &p, float &q)
    {
        if (tpr < 32u) {
            for (uint32_t d = tpr >> 1; d; d >>= 1) {
                p += __shfl_xor_sync(0xffffffffu, p, d);
                q += __shfl_xor_sync(0xffffffffu, q, d);
            }
            return;
        }
        const bool upper = threadIdx.x & 16u;
        float v = (upper ? q : p) + __shfl_xor_sync(0xffffffffu, upper ? p : q, 16);
#pragma unroll
        for (int d = 8; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (tpr > 32u) meet<16>(v);
        p = __shfl_sync(0xffffffffu, v, 0);
        q = __shfl_sync(0xffffffffu, v, 16);
    }
    __device__ __forceinline__ void operator()(float &p, float &q, float &r, float &s)
    {
        if (tpr < 32u) {
            (*this)(p, q);
            (*this)(r, s);
            return;
        }
        const bool upper = threadIdx.x & 16u, odd = threadIdx.x & 8u;
        const float v0 = (upper ? r : p) + __shfl_xor_sync(0xffffffffu, upper ? p : r, 16);
        const float v1 = (upper ? s : q) + __shfl_xor_sync(0xffffffffu, upper ? q : s, 16);
        float v = (odd ? v1 : v0) + __shfl_xor_sync(0xffffffffu, odd ? v0 : v1, 8);
#pragma unroll
        for (int d = 4; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
        if (tpr > 32u) meet<8>(v);
        p = __shfl_sync(0xffffffffu, v, 0);
        q = __shfl_sync(0xffffffffu, v, 8);
        r = __shfl_sync(0xffffffffu, v, 16);
        s = __shfl_sync(0xffffffffu, v, 24);
    }
};

__device__ __forceinline__ float sum8(const uint64_t (&x)[4])
{
    const uint64_t s = add2(add2(x[0], x[1]), add2(x[2], x[3]));
    return low(s) + high(s);
}
__device__ __forceinline__ float dot8(const uint64_t (&x)[4], const uint64_t (&y)[4])
{
    const uint64_t s = add2(fma2(x[1], y[1], mul2(x[0], y[0])), fma2(x[3], y[3], mul2(x[2], y[2])));
    return low(s) + high(s);
}
__device__ __forceinline__ void times(uint64_t (&x)[4], uint64_t by)
{
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = mul2(x[i], by);
}
__device__ __forceinline__ void times(uint64_t (&x)[4], const uint64_t (&by)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = mul2(x[i], by[i]);
}

// x <- x - mean (zero for kind "rms"), for two rows at once (the second only if TWO).
template <bool TWO> __device__ __forceinline__ void centre(RowSums &sums, const JoinArgs &p, uint64_t (&x)[4], uint64_t (&y)[4])
{
    if (!p.layer) return;
    float mx = sum8(x), my = TWO ? sum8(y) : 0.0f;
    sums(mx, my);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        x[i] = add2(x[i], both(-mx * p.inv_c));
        if (TWO) y[i] = add2(y[i], both(-my * p.inv_c));
    }
}
// x <- (x - mean) r; mine: the thread owns columns of the row.
__device__ __forceinline__ void normalize(RowSums &sums, const JoinArgs &p, bool mine, uint64_t (&x)[4])
{
    centre<false>(sums, p, x, x);
    float v = mine ? dot8(x, x) : 0.0f, none = 0.0f;
    sums(v, none);
    times(x, both(rsqrtf(__fmaf_rn(v, p.inv_c, p.eps))));
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kJoinThreads ? 2 : 1) join_kernel(const __grid_constant__ JoinArgs p)
{
    __shared__ float s_buf[256];
    const uint32_t slot = threadIdx.x / p.tpr, t = threadIdx.x - slot * p.tpr, col = t * 8u;
    RowSums sums{s_buf, p.tpr, slot, 0u};
    const bool owns = col < p.C;
    const uint64_t step = (uint64_t)gridDim.x * p.slots, n_turns = (p.rows + step - 1u) / step;
    uint64_t row = (uint64_t)blockIdx.x * p.slots + slot;
    extern __shared__ __align__(16) unsigned char s_pipe[];
    using Pipe = ForwardPipe<T, THREADS>;
    Pipe pipe;
    pipe.init(s_pipe);
    const char *const src[2] = {reinterpret_cast<const char *>(p.x), reinterpret_cast<const char *>(p.y)};
    const uint64_t ahead = Pipe::kDepth * step;
#pragma unroll
    for (int d = 0; d < Pipe::kDepth; d++) {
        const uint64_t r = row + d * step;
        pipe.fetch(src, (r * p.C + col) * Elem<T>::kBytes, owns && r < p.rows);
    }
    for (uint64_t turn = 0; turn < n_turns; turn++, row += step) {
        const bool mine = owns && row < p.rows;
        const uint64_t at = row * p.C + col;
        uint64_t x[4], u[4], v[4], w[4];
        pipe.wait();
        pipe.get(0, src, at * Elem<T>::kBytes, mine, x);
        pipe.get(1, src, at * Elem<T>::kBytes, mine, u);
        if (p.post_weight) {
            normalize(sums, p, mine, u);
            if (mine) {
                param8<T>(p.post_weight, col, p.param_f32, v);
                times(u, v);
                if (p.post_bias) {
                    param8<T>(p.post_bias, col, p.param_f32, w);
#pragma unroll
                    for (int i = 0; i < 4; i++) u[i] = add2(u[i], w[i]);
                }
            }
        }
        if (mine) {
            if (p.gate) {
                param8<T>(p.gate, p.gates > 1u ? row / p.rows_per_gate * p.C + col : col, p.param_f32, v);
                times(u, v);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) x[i] = fma2(both(p.a), u[i], x[i]);
            store_pairs<T>(reinterpret_cast<char *>(p.out_a) + at * Elem<T>::kBytes, x);
        }
        pipe.fetch(src, (at + ahead * p.C) * Elem<T>::kBytes, owns && row + ahead < p.rows);   // into the place just read
        normalize(sums, p, mine, x);
        if (mine) {
            param8<T>(p.weight, col, p.param_f32, v);
            w[0] = w[1] = w[2] = w[3] = 0ull;
            if (p.bias) param8<T>(p.bias, col, p.param_f32, w);
#pragma unroll
            for (int i = 0; i < 4; i++) x[i] = fma2(x[i], v[i], w[i]);
            store_pairs<T>(reinterpret_cast<char *>(p.out_b) + at * Elem<T>::kBytes, x);
        }
    }
}

// The column sums of one thread's eight columns: in registers, or for rows above 4096 columns (1024 threads, 64
// registers each) in shared memory, where a thread only ever touches its own columns.
template <bool SMEM> struct Columns {
    uint64_t v[kSums][4];
    __device__ __forceinline__ void init(float *, uint32_t, uint32_t)
    {
#pragma unroll
        for (int q = 0; q < kSums; q++)
#pragma unroll
            for (int i = 0; i < 4; i++) v[q][i] = 0ull;
    }
    __device__ __forceinline__ void add(int q, const uint64_t (&x)[4], const uint64_t (&y)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; i++) v[q][i] = fma2(x[i], y[i], v[q][i]);
    }
    __device__ __forceinline__ void add(int q, const uint64_t (&x)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; i++) v[q][i] = add2(x[i], v[q][i]);
    }
    __device__ __forceinline__ void take(int q, uint64_t (&x)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            x[i] = v[q][i];
            v[q][i] = 0ull;
        }
    }
};
template <> struct Columns<true> {
    ulonglong2 *base;
    uint32_t stride;                               // 16-byte units per sum
    __device__ __forceinline__ void init(float *smem, uint32_t C, uint32_t col)
    {
        base = reinterpret_cast<ulonglong2 *>(smem + col);
        stride = C >> 2;
        if (col < C)
            for (int q = 0; q < kSums; q++) base[q * stride] = base[q * stride + 1] = make_ulonglong2(0ull, 0ull);
    }
    __device__ __forceinline__ void add(int q, const uint64_t (&x)[4])
    {
        ulonglong2 *b = base + q * stride;
        const ulonglong2 u = b[0], w = b[1];
        b[0] = make_ulonglong2(add2(u.x, x[0]), add2(u.y, x[1]));
        b[1] = make_ulonglong2(add2(w.x, x[2]), add2(w.y, x[3]));
    }
    __device__ __forceinline__ void add(int q, const uint64_t (&x)[4], const uint64_t (&y)[4])
    {
        ulonglong2 *b = base + q * stride;
        const ulonglong2 u = b[0], w = b[1];
        b[0] = make_ulonglong2(fma2(x[0], y[0], u.x), fma2(x[1], y[1], u.y));
        b[1] = make_ulonglong2(fma2(x[2], y[2], w.x), fma2(x[3], y[3], w.y));
    }
    __device__ __forceinline__ void take(int q, uint64_t (&x)[4])
    {
        ulonglong2 *b = base + q * stride;
        const ulonglong2 u = b[0], w = b[1];
        x[0] = u.x; x[1] = u.y; x[2] = w.x; x[3] = w.y;
        b[0] = b[1] = make_ulonglong2(0ull, 0ull);
    }
};

// Adds one column sum over the CTA's slots (in slot order) and hands column c's total to out(c, total).
template <bool WIDE, typename Out>
__device__ __forceinline__ void over_slots(const JoinArgs &p, uint32_t slot, uint32_t col, const uint64_t (&pairs)[4], float *s_cols, Out out)
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; i++) unpair(pairs[i], x[2 * i], x[2 * i + 1]);
    if (WIDE || p.slots == 1u) {
        if (col < p.C)
            for (int i = 0; i < 8; i++) out(col + i, x[i]);
        return;
    }
    if (col < p.C) {
        float4 *d = reinterpret_cast<float4 *>(s_cols + (slot * p.C + col));
        d[0] = make_float4(x[0], x[1], x[2], x[3]);
        d[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < p.C; c += blockDim.x) {
        float v = 0.0f;
        for (uint32_t s = 0; s < p.slots; s++) v += s_cols[s * p.C + c];
        out(c, v);
    }
    __syncthreads();
}

template <typename T, bool POST, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) join_grad_kernel(const __grid_constant__ JoinArgs p)
{
    constexpr bool WIDE = THREADS == kJoinWide;
    __shared__ float s_buf[256];
    __shared__ __align__(16) float s_cols[WIDE ? 4 : kJoinThreads * 8];
    extern __shared__ __align__(16) float s_dyn[];
    const uint32_t slot = threadIdx.x / p.tpr, t = threadIdx.x - slot * p.tpr, col = t * 8u;
    RowSums sums{s_buf, p.tpr, slot, 0u};
    const bool owns = col < p.C;
    Columns<WIDE> cols;
    cols.init(s_dyn, p.C, col);
    using Pipe = BackwardPipe<T, THREADS>;
    Pipe pipe;
    pipe.init(s_dyn + (WIDE ? kSums * p.C : 0u));
    const char *const src[4] = {reinterpret_cast<const char *>(p.x), reinterpret_cast<const char *>(p.y),
                                reinterpret_cast<const char *>(p.grad_z), reinterpret_cast<const char *>(p.grad_h)};
    const uint64_t ahead = (uint64_t)Pipe::kDepth * p.slots;
    const uint32_t n_groups = p.gates > 1u ? p.gates : 1u;
    // CTA j of group g takes an equal run of the group's rows; with more groups than CTAs a CTA takes whole groups in turn
    for (uint32_t g = blockIdx.x / p.per_group, j = blockIdx.x % p.per_group; g < n_groups; g += gridDim.x / p.per_group) {
        const uint64_t lo = g * p.rows_per_gate + p.rows_per_gate * j / p.per_group;
        const uint64_t hi = g * p.rows_per_gate + p.rows_per_gate * (j + 1u) / p.per_group;
        uint64_t row = lo + slot;
#pragma unroll
        for (int d = 0; d < Pipe::kDepth; d++) {
            const uint64_t r = row + (uint64_t)d * p.slots;
            pipe.fetch(src, (r * p.C + col) * Elem<T>::kBytes, owns && r < hi);
        }
        for (uint64_t first = lo; first < hi; first += p.slots, row += p.slots) {
            const bool mine = owns && row < hi;
            const uint64_t at = row * p.C + col;
            uint64_t z[4], y[4], gz[4], gh[4], w[4];
            pipe.wait();
            pipe.get(0, src, at * Elem<T>::kBytes, mine, z);
            pipe.get(1, src, at * Elem<T>::kBytes, mine, y);
            pipe.get(2, src, at * Elem<T>::kBytes, mine && p.grad_z, gz);
            pipe.get(3, src, at * Elem<T>::kBytes, mine, gh);
            // all sums of the row at once: those of gh w and gh w (z - mean) need no r
            centre<POST>(sums, p, z, y);
            float vz = 0.0f, vy = 0.0f, st = 0.0f, sth = 0.0f;
            uint64_t t[4];
            if (mine) {
                vz = dot8(z, z);
                if (POST) vy = dot8(y, y);
                param8<T>(p.weight, col, p.param_f32, t);
                times(t, gh);
                st = p.layer ? sum8(t) : 0.0f;
                sth = dot8(t, z);
            }
            pipe.fetch(src, (at + ahead * p.C) * Elem<T>::kBytes, owns && row + ahead < hi);   // into the place just read
            sums(vz, sth, st, vy);
            const float rz = rsqrtf(__fmaf_rn(vz, p.inv_c, p.eps)), ry = POST ? rsqrtf(__fmaf_rn(vy, p.inv_c, p.eps)) : 0.0f;
            if (POST) times(y, both(ry));                          // the normalized y
            if (mine) {
                times(z, both(rz));                                // the normalized z
                cols.add(0, gh, z);
                cols.add(1, gh);
                const uint64_t m1 = both(-st * p.inv_c), m2 = both(-sth * rz * p.inv_c);
#pragma unroll
                for (int i = 0; i < 4; i++) gz[i] = fma2(both(rz), fma2(z[i], m2, add2(t[i], m1)), gz[i]);
                store_pairs<T>(reinterpret_cast<char *>(p.out_a) + at * Elem<T>::kBytes, gz);
                times(gz, both(p.a));                              // du
                if (p.gate) {
                    if (POST) {
                        param8<T>(p.post_weight, col, p.param_f32, gh);
                        w[0] = w[1] = w[2] = w[3] = 0ull;
                        if (p.post_bias) param8<T>(p.post_bias, col, p.param_f32, w);
#pragma unroll
                        for (int i = 0; i < 4; i++) w[i] = fma2(y[i], gh[i], w[i]);
                        cols.add(4, gz, w);
                    } else {
                        cols.add(4, gz, y);
                    }
                    param8<T>(p.gate, p.gates > 1u ? (uint64_t)g * p.C + col : col, p.param_f32, w);
                    times(gz, w);
                }
            }
            if (POST) {
                st = sth = 0.0f;
                if (mine) {
                    cols.add(2, gz, y);
                    cols.add(3, gz);
                    param8<T>(p.post_weight, col, p.param_f32, w);
                    times(gz, w);
                    st = p.layer ? sum8(gz) : 0.0f;
                    sth = dot8(gz, y);
                }
                sums(st, sth);
                const uint64_t m1 = both(-st * p.inv_c), m2 = both(-sth * p.inv_c);
#pragma unroll
                for (int i = 0; i < 4; i++) gz[i] = mul2(both(ry), fma2(y[i], m2, add2(gz[i], m1)));
            }
            if (mine) store_pairs<T>(reinterpret_cast<char *>(p.out_b) + at * Elem<T>::kBytes, gz);
        }
        if (p.gate && p.gates > 1u) {
            uint64_t x[4] = {0ull, 0ull, 0ull, 0ull};
            if (owns) cols.take(4, x);
            const uint64_t at = (uint64_t)(g * p.per_group + j) * p.C;
            over_slots<WIDE>(p, slot, col, x, s_cols, [&](uint32_t c, float v) {
                if (p.per_group > 1u) p.gate_partial[at + c] = v;
                else if (p.grad_gate) store_param(p.grad_gate, at + c, p.param_f32, sizeof(T) == 2 && __is_same(T, __nv_bfloat16), v);
            });
        }
    }
#pragma unroll
    for (int q = 0; q < kSums; q++) {
        if ((q == 2 || q == 3) && !POST) continue;
        if (q == 4 && p.gates != 1u) continue;
        uint64_t x[4] = {0ull, 0ull, 0ull, 0ull};
        if (owns) cols.take(q, x);
        float *const to = q == 4 ? p.gate_partial + (uint64_t)blockIdx.x * p.C : p.partial + ((uint64_t)blockIdx.x * 4u + q) * p.C;
        over_slots<WIDE>(p, slot, col, x, s_cols, [&](uint32_t c, float v) { to[c] = v; });
    }
}

struct JoinSums {
    const float *partial, *gate_partial;
    void *out[4], *grad_gate;
    uint32_t C, n_ctas, per_group, param_f32, bf16;
};
// blockIdx.y: 0-3 the parameter sums over all CTAs, 4 + g the gate sums of group g over its CTAs.  32 columns per CTA,
// 32 threads per column, each over every 32nd partial row in order, then in a fixed tree.  (Eight threads per column
// waited longer for their loads: 38.9 against 37.7 us for the whole backward call on 12608 x 768.)
__global__ void __launch_bounds__(1024) join_sums_kernel(const __grid_constant__ JoinSums p)
{
    __shared__ float s_part[32][33];
    const uint32_t lane = threadIdx.x & 31u, k = threadIdx.x >> 5, c = blockIdx.x * 32u + lane, q = blockIdx.y;
    void *const out = q < 4u ? p.out[q] : p.grad_gate;
    if (!out) return;
    const uint32_t n = q < 4u ? p.n_ctas : p.per_group;
    const uint64_t stride = q < 4u ? 4ull * p.C : p.C;
    const float *src = q < 4u ? p.partial + (uint64_t)q * p.C : p.gate_partial + (uint64_t)(q - 4u) * p.per_group * p.C;
    float v = 0.0f;
    if (c < p.C) {
#pragma unroll 8
        for (uint32_t i = k; i < n; i += 32u) v += src[i * stride + c];
    }
    s_part[k][lane] = v;
    __syncthreads();
    v = s_part[lane][k];                                           // warp k: column k of the CTA's
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    const uint32_t col = blockIdx.x * 32u + k;
    if (lane == 0 && col < p.C) store_param(out, (q < 4u ? 0ull : (uint64_t)(q - 4u) * p.C) + col, p.param_f32, p.bf16, v);
}

static bool join_aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1u)) == 0; }

static daf_status check_join(const daf_norm_params *p)
{
    if (!p || p->struct_size != sizeof(daf_norm_params) || p->dtype > DAF_BF16 || p->kind > DAF_NORM_RMS) return DAF_ERR_INVALID_ARG;
    if (p->param_dtype != DAF_F32 && p->param_dtype != p->dtype) return DAF_ERR_INVALID_ARG;
    if (!(p->eps >= 0.0f) || p->reserved != 0) return DAF_ERR_INVALID_ARG;
    if (p->width == 0 || p->width % 8u) return DAF_ERR_SHAPE;
    if (p->width > kJoinMaxWidth) return DAF_ERR_UNSUPPORTED;
    if (p->gates > 1u && p->rows % p->gates) return DAF_ERR_SHAPE;
    return DAF_OK;
}

// Threads of a row, rows of a CTA.
static void join_shape(const daf_norm_params *p, JoinArgs *a)
{
    const uint32_t chunks = p->width / 8u;
    a->tpr = chunks <= 8u ? 8u : chunks <= 16u ? 16u : (chunks + 31u) / 32u * 32u;
    a->slots = a->tpr > (uint32_t)kJoinThreads ? 1u : kJoinThreads / a->tpr;
    a->rows = p->rows;
    a->C = p->width;
    a->gates = p->gates;
    a->rows_per_gate = p->gates > 1u ? p->rows / p->gates : p->rows;
    a->a = p->residual_scale;
    a->eps = p->eps;
    a->inv_c = 1.0f / (float)p->width;
    a->layer = p->kind == DAF_NORM_LAYER;
    a->param_f32 = p->param_dtype == DAF_F32;
    a->per_group = 1;
}

// CTAs of the backward kernel and CTAs per gate group, with at most `most` CTAs.
static void join_grid(const JoinArgs &a, uint32_t most, uint32_t *grid, uint32_t *per_group)
{
    const uint32_t groups = a.gates > 1u ? a.gates : 1u;
    const uint64_t turns = (a.rows_per_gate + a.slots - 1u) / a.slots;       // turns of a CTA that has a group to itself
    uint64_t k = groups < most ? most / groups : 1u;
    if (k > turns) k = turns ? turns : 1u;
    *per_group = (uint32_t)k;
    *grid = groups < most ? groups * (uint32_t)k : most;
}

template <typename T, int THREADS> static daf_status launch_join(const JoinArgs &a, cudaStream_t s)
{
    int ctas = 0;
    const uint64_t turns = (a.rows + a.slots - 1u) / a.slots;
    const uint32_t smem = ForwardPipe<T, THREADS>::kBytes;
    if (persistent_ctas(reinterpret_cast<const void *>(&join_kernel<T, THREADS>), THREADS, (int)smem, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    join_kernel<T, THREADS><<<(uint32_t)(turns < (uint64_t)ctas ? turns : ctas), a.tpr * a.slots, smem, s>>>(a);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
template <typename T> static daf_status run_join(const JoinArgs &a, cudaStream_t s)
{
    return a.tpr > (uint32_t)kJoinThreads ? launch_join<T, kJoinWide>(a, s) : launch_join<T, kJoinThreads>(a, s);
}

template <typename T, bool POST, int THREADS> static daf_status launch_join_grad(JoinArgs &a, uint32_t *grid, cudaStream_t s)
{
    int ctas = 0;
    const auto kernel = &join_grad_kernel<T, POST, THREADS>;
    const uint32_t smem = (THREADS == kJoinWide ? kSums * a.C * 4u : 0u) + BackwardPipe<T, THREADS>::kBytes;
    if (persistent_ctas(reinterpret_cast<const void *>(kernel), THREADS, (int)smem, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    join_grid(a, ctas < (int)kJoinCtas ? (uint32_t)ctas : kJoinCtas, grid, &a.per_group);
    a.gate_partial = a.partial + (uint64_t)*grid * 4u * a.C;
    kernel<<<*grid, a.tpr * a.slots, smem, s>>>(a);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
template <typename T, bool POST> static daf_status run_join_grad(JoinArgs &a, uint32_t *grid, cudaStream_t s)
{
    return a.tpr > (uint32_t)kJoinThreads ? launch_join_grad<T, POST, kJoinWide>(a, grid, s) : launch_join_grad<T, POST, kJoinThreads>(a, grid, s);
}

}  // namespace daf

using namespace daf;

extern "C" daf_status daf_residual_norm(const daf_norm_params *params, const void *d_x, const void *d_y, const void *d_weight,
                                        const void *d_bias, const void *d_gate, const void *d_post_weight, const void *d_post_bias,
                                        void *d_z, void *d_h, daf_stream stream)
{
    const daf_status st = check_join(params);
    if (st != DAF_OK) return st;
    if ((d_gate != nullptr) != (params->gates > 0u) || (d_post_bias && !d_post_weight) || !d_weight) return DAF_ERR_INVALID_ARG;
    if (params->rows == 0) return DAF_OK;
    const uintptr_t al = params->dtype == DAF_F32 ? 32u : 16u;
    const void *const data[4] = {d_x, d_y, d_z, d_h};
    for (const void *q : data)
        if (!q || !join_aligned(q, al)) return DAF_ERR_INVALID_ARG;
    const void *const vec[5] = {d_weight, d_bias, d_gate, d_post_weight, d_post_bias};
    for (const void *q : vec)
        if (!join_aligned(q, 16u)) return DAF_ERR_INVALID_ARG;
    JoinArgs a = {};
    join_shape(params, &a);
    a.x = d_x; a.y = d_y; a.weight = d_weight; a.bias = d_bias; a.gate = d_gate; a.post_weight = d_post_weight; a.post_bias = d_post_bias;
    a.out_a = d_z; a.out_b = d_h;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return params->dtype == DAF_F32 ? run_join<float>(a, s) : params->dtype == DAF_F16 ? run_join<__half>(a, s) : run_join<__nv_bfloat16>(a, s);
}

extern "C" uint64_t daf_residual_norm_grad_workspace(const daf_norm_params *params)
{
    if (check_join(params) != DAF_OK) return 0;
    JoinArgs a = {};
    join_shape(params, &a);
    uint32_t grid = 0, per_group = 0;
    join_grid(a, kJoinCtas, &grid, &per_group);
    return (uint64_t)grid * kSums * a.C * 4u;
}

extern "C" daf_status daf_residual_norm_grad(const daf_norm_params *params, const void *d_z, const void *d_y, const void *d_weight,
                                             const void *d_gate, const void *d_post_weight, const void *d_post_bias,
                                             const void *d_grad_z, const void *d_grad_h, void *d_grad_x, void *d_grad_y,
                                             void *d_grad_weight, void *d_grad_bias, void *d_grad_gate, void *d_grad_post_weight,
                                             void *d_grad_post_bias, void *d_workspace, uint64_t workspace_bytes, daf_stream stream)
{
    daf_status st = check_join(params);
    if (st != DAF_OK) return st;
    if ((d_gate != nullptr) != (params->gates > 0u) || (d_post_bias && !d_post_weight) || !d_weight || (d_grad_gate && !d_gate) ||
        ((d_grad_post_weight || d_grad_post_bias) && !d_post_weight))
        return DAF_ERR_INVALID_ARG;
    const uint32_t pb = params->param_dtype == DAF_F32 ? 4u : 2u;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const void *const vec[9] = {d_weight, d_gate, d_post_weight, d_post_bias, d_grad_weight, d_grad_bias, d_grad_gate, d_grad_post_weight, d_grad_post_bias};
    for (const void *q : vec)
        if (!join_aligned(q, 16u)) return DAF_ERR_INVALID_ARG;
    if (params->rows == 0) {                                       // sums over nothing
        void *const sums[5] = {d_grad_weight, d_grad_bias, d_grad_post_weight, d_grad_post_bias, d_grad_gate};
        for (int q = 0; q < 5; q++)
            if (sums[q] && cudaMemsetAsync(sums[q], 0, (uint64_t)pb * params->width * (q == 4 ? params->gates : 1u), s) != cudaSuccess) return DAF_ERR_CUDA;
        return DAF_OK;
    }
    const uintptr_t al = params->dtype == DAF_F32 ? 32u : 16u;
    const void *const data[5] = {d_z, d_y, d_grad_h, d_grad_x, d_grad_y};
    for (const void *q : data)
        if (!q || !join_aligned(q, al)) return DAF_ERR_INVALID_ARG;
    if (!join_aligned(d_grad_z, al) || !d_workspace || !join_aligned(d_workspace, 16u)) return DAF_ERR_INVALID_ARG;
    if (workspace_bytes < daf_residual_norm_grad_workspace(params)) return DAF_ERR_CAPACITY;
    JoinArgs a = {};
    join_shape(params, &a);
    a.x = d_z; a.y = d_y; a.weight = d_weight; a.gate = d_gate; a.post_weight = d_post_weight; a.post_bias = d_post_bias;
    a.grad_z = d_grad_z; a.grad_h = d_grad_h; a.out_a = d_grad_x; a.out_b = d_grad_y;
    a.partial = reinterpret_cast<float *>(d_workspace);
    a.grad_gate = d_grad_gate;
    uint32_t grid = 0;
#define DAF_JOIN_GRAD(T) (d_post_weight ? run_join_grad<T, true>(a, &grid, s) : run_join_grad<T, false>(a, &grid, s))
    st = params->dtype == DAF_F32 ? DAF_JOIN_GRAD(float) : params->dtype == DAF_F16 ? DAF_JOIN_GRAD(__half) : DAF_JOIN_GRAD(__nv_bfloat16);
#undef DAF_JOIN_GRAD
    if (st != DAF_OK) return st;
    JoinSums f = {a.partial, a.gate_partial, {d_grad_weight, d_grad_bias, d_grad_post_weight, d_grad_post_bias}, d_grad_gate,
                  a.C, grid, a.gates > 1u ? a.per_group : grid, a.param_f32, params->dtype == DAF_BF16};
    // gates whose groups had one CTA each are written already
    const uint32_t gates = !d_grad_gate || (a.gates > 1u && a.per_group == 1u) ? 0u : a.gates;
    join_sums_kernel<<<dim3((a.C + 31u) / 32u, 4u + gates), 1024, 0, s>>>(f);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
