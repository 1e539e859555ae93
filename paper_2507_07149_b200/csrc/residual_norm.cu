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

// Eight elements as they lie in memory (widened only when they are used: half the registers for 16-bit types).
template <typename T> struct Raw8 {
    uint4 v;
    __device__ __forceinline__ void load(const void *p)
    {
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    }
    __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float (&x)[8]) const { Elem<T>::widen8(v, x); }
};
template <> struct Raw8<float> {
    float v[8];
    __device__ __forceinline__ void load(const void *p) { Elem<float>::load8(p, v); }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = 0.0f;
    }
    __device__ __forceinline__ void get(float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = v[i];
    }
};

// Eight parameters of a vector (binary32 or the activations' type); `fill` where the vector is absent.
template <typename T> __device__ __forceinline__ void param8(const void *p, uint64_t at, uint32_t f32, float fill, float (&x)[8])
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = fill;
    } else if (f32) {
        const float4 *q = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(p) + at);
        const float4 u = __ldg(q), w = __ldg(q + 1);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
        x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    } else {
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(p) + at * Elem<T>::kBytes));
        if (Elem<T>::kBytes == 2) Elem<T>::widen8(u, x);
    }
}

__device__ __forceinline__ void store_param(void *p, uint64_t at, uint32_t f32, uint32_t bf16, float v)
{
    if (f32) reinterpret_cast<float *>(p)[at] = v;
    else if (bf16) reinterpret_cast<__nv_bfloat16 *>(p)[at] = __float2bfloat16_rn(v);
    else reinterpret_cast<__half *>(p)[at] = __float2half_rn(v);
}

// Sums of two values over the threads of a slot.  Two buffers in turn: a warp that writes for sum k + 2 has met, at sum
// k + 1, every warp that still read sum k.
struct RowSums {
    float2 (*buf)[32];
    uint32_t tpr, slot, parity;
    __device__ __forceinline__ void operator()(float &p, float &q)
    {
        for (uint32_t d = (tpr < 32u ? tpr : 32u) >> 1; d; d >>= 1) {
            p += __shfl_xor_sync(0xffffffffu, p, d);
            q += __shfl_xor_sync(0xffffffffu, q, d);
        }
        if (tpr > 32u) {
            const uint32_t n = tpr >> 5, first = slot * n;
            if ((threadIdx.x & 31u) == 0) buf[parity][threadIdx.x >> 5] = make_float2(p, q);
            asm volatile("bar.sync %0, %1;" ::"r"(slot + 1u), "r"(tpr) : "memory");
            p = q = 0.0f;
            for (uint32_t w = 0; w < n; w++) {
                const float2 v = buf[parity][first + w];
                p += v.x;
                q += v.y;
            }
            parity ^= 1u;
        }
    }
};

__device__ __forceinline__ float sum8(const float (&x)[8])
{
    return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
}
__device__ __forceinline__ float dot8(const float (&x)[8], const float (&y)[8])
{
    float a = x[0] * y[0], b = x[1] * y[1];
#pragma unroll
    for (int i = 2; i < 8; i += 2) {
        a = __fmaf_rn(x[i], y[i], a);
        b = __fmaf_rn(x[i + 1], y[i + 1], b);
    }
    return a + b;
}

// 1 / sqrt(mean of squares + eps), correctly rounded steps (the row's 8192 elements share this one value).
__device__ __forceinline__ float inv_std(float sum_sq, float inv_c, float eps)
{
    return __fdiv_rn(1.0f, __fsqrt_rn(__fmaf_rn(sum_sq, inv_c, eps)));
}

// x <- (x - mean) r for two rows' worth at once (the second may be unused); mine: the thread owns columns of the row.
template <bool TWO>
__device__ __forceinline__ void normalize(RowSums &sums, const JoinArgs &p, bool mine, float (&x)[8], float (&y)[8], float &rx, float &ry)
{
    float mx = 0.0f, my = 0.0f;
    if (p.layer) {
        mx = sum8(x);
        my = TWO ? sum8(y) : 0.0f;
        sums(mx, my);
        mx *= p.inv_c;
        my *= p.inv_c;
    }
    float vx = 0.0f, vy = 0.0f;
    if (mine) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            x[i] -= mx;
            if (TWO) y[i] -= my;
        }
        vx = dot8(x, x);
        if (TWO) vy = dot8(y, y);
    }
    sums(vx, vy);
    rx = inv_std(vx, p.inv_c, p.eps);
    ry = TWO ? inv_std(vy, p.inv_c, p.eps) : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        x[i] *= rx;
        if (TWO) y[i] *= ry;
    }
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == kJoinThreads ? 2 : 1) join_kernel(const __grid_constant__ JoinArgs p)
{
    __shared__ float2 s_buf[2][32];
    const uint32_t slot = threadIdx.x / p.tpr, t = threadIdx.x - slot * p.tpr, col = t * 8u;
    RowSums sums{s_buf, p.tpr, slot, 0u};
    const bool owns = col < p.C;
    const uint64_t step = (uint64_t)gridDim.x * p.slots, n_turns = (p.rows + step - 1u) / step;
    uint64_t row = (uint64_t)blockIdx.x * p.slots + slot;
    const char *const xs = reinterpret_cast<const char *>(p.x), *const ys = reinterpret_cast<const char *>(p.y);
    Raw8<T> rx, ry;
    rx.zero();
    ry.zero();
    if (owns && row < p.rows) {
        rx.load(xs + (row * p.C + col) * Elem<T>::kBytes);
        ry.load(ys + (row * p.C + col) * Elem<T>::kBytes);
    }
    for (uint64_t turn = 0; turn < n_turns; turn++, row += step) {
        const bool mine = owns && row < p.rows;
        const uint64_t at = row * p.C + col;
        float x[8], u[8], v[8], r, unused;
        rx.get(x);
        ry.get(u);
        if (owns && row + step < p.rows) {
            rx.load(xs + (at + step * p.C) * Elem<T>::kBytes);
            ry.load(ys + (at + step * p.C) * Elem<T>::kBytes);
        }
        if (p.post_weight) {
            normalize<false>(sums, p, mine, u, u, r, unused);
            if (mine) {
                float b[8];
                param8<T>(p.post_weight, col, p.param_f32, 1.0f, v);
                param8<T>(p.post_bias, col, p.param_f32, 0.0f, b);
#pragma unroll
                for (int i = 0; i < 8; i++) u[i] = __fmaf_rn(u[i], v[i], b[i]);
            }
        }
        if (mine) {
            if (p.gate) {
                param8<T>(p.gate, p.gates > 1u ? row / p.rows_per_gate * p.C + col : col, p.param_f32, 1.0f, v);
#pragma unroll
                for (int i = 0; i < 8; i++) u[i] *= v[i];
            }
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = __fmaf_rn(p.a, u[i], x[i]);
            Elem<T>::store8(reinterpret_cast<char *>(p.out_a) + at * Elem<T>::kBytes, x);
        }
        normalize<false>(sums, p, mine, x, x, r, unused);
        if (mine) {
            param8<T>(p.weight, col, p.param_f32, 1.0f, v);
            param8<T>(p.bias, col, p.param_f32, 0.0f, u);
#pragma unroll
            for (int i = 0; i < 8; i++) x[i] = __fmaf_rn(x[i], v[i], u[i]);
            Elem<T>::store8(reinterpret_cast<char *>(p.out_b) + at * Elem<T>::kBytes, x);
        }
    }
}

// The column sums of one thread's eight columns: in registers, or for rows above 4096 columns (1024 threads, 64
// registers each) in shared memory, where a thread only ever touches its own columns.
template <bool SMEM> struct Columns {
    float v[kSums][8];
    __device__ __forceinline__ void init(float *, uint32_t, uint32_t)
    {
#pragma unroll
        for (int q = 0; q < kSums; q++)
#pragma unroll
            for (int i = 0; i < 8; i++) v[q][i] = 0.0f;
    }
    __device__ __forceinline__ void add(int q, const float (&x)[8], const float (&y)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; i++) v[q][i] = __fmaf_rn(x[i], y[i], v[q][i]);
    }
    __device__ __forceinline__ void add(int q, const float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; i++) v[q][i] += x[i];
    }
    __device__ __forceinline__ void take(int q, float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            x[i] = v[q][i];
            v[q][i] = 0.0f;
        }
    }
};
template <> struct Columns<true> {
    float4 *base;
    uint32_t stride;                               // float4 per sum
    __device__ __forceinline__ void init(float *smem, uint32_t C, uint32_t col)
    {
        base = reinterpret_cast<float4 *>(smem + col);
        stride = C >> 2;
        if (col < C)
            for (int q = 0; q < kSums; q++) base[q * stride] = base[q * stride + 1] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ __forceinline__ void add(int q, const float (&x)[8])
    {
        float4 *b = base + q * stride;
        const float4 u = b[0], w = b[1];
        b[0] = make_float4(u.x + x[0], u.y + x[1], u.z + x[2], u.w + x[3]);
        b[1] = make_float4(w.x + x[4], w.y + x[5], w.z + x[6], w.w + x[7]);
    }
    __device__ __forceinline__ void add(int q, const float (&x)[8], const float (&y)[8])
    {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = x[i] * y[i];
        add(q, t);
    }
    __device__ __forceinline__ void take(int q, float (&x)[8])
    {
        float4 *b = base + q * stride;
        const float4 u = b[0], w = b[1];
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
        x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
        b[0] = b[1] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
};

// Adds one column sum over the CTA's slots (in slot order) and hands column c's total to out(c, total).
template <bool WIDE, typename Out>
__device__ __forceinline__ void over_slots(const JoinArgs &p, uint32_t slot, uint32_t col, const float (&x)[8], float *s_cols, Out out)
{
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
    __shared__ float2 s_buf[2][32];
    __shared__ __align__(16) float s_cols[WIDE ? 4 : kJoinThreads * 8];
    extern __shared__ __align__(16) float s_dyn[];
    const uint32_t slot = threadIdx.x / p.tpr, t = threadIdx.x - slot * p.tpr, col = t * 8u;
    RowSums sums{s_buf, p.tpr, slot, 0u};
    const bool owns = col < p.C;
    Columns<WIDE> cols;
    cols.init(s_dyn, p.C, col);
    const char *const zs = reinterpret_cast<const char *>(p.x), *const ys = reinterpret_cast<const char *>(p.y);
    const char *const gzs = reinterpret_cast<const char *>(p.grad_z), *const ghs = reinterpret_cast<const char *>(p.grad_h);
    const uint32_t n_groups = p.gates > 1u ? p.gates : 1u;
    // CTA j of group g takes an equal run of the group's rows; with more groups than CTAs a CTA takes whole groups in turn
    for (uint32_t g = blockIdx.x / p.per_group, j = blockIdx.x % p.per_group; g < n_groups; g += gridDim.x / p.per_group) {
        const uint64_t lo = g * p.rows_per_gate + p.rows_per_gate * j / p.per_group;
        const uint64_t hi = g * p.rows_per_gate + p.rows_per_gate * (j + 1u) / p.per_group;
        Raw8<T> rz, ry, rgz, rgh;
        rz.zero();
        ry.zero();
        rgz.zero();
        rgh.zero();
        uint64_t row = lo + slot;
        if (owns && row < hi) {
            const uint64_t b = (row * p.C + col) * Elem<T>::kBytes;
            rz.load(zs + b);
            ry.load(ys + b);
            rgh.load(ghs + b);
            if (gzs) rgz.load(gzs + b);
        }
        for (uint64_t first = lo; first < hi; first += p.slots, row += p.slots) {
            const bool mine = owns && row < hi;
            const uint64_t at = row * p.C + col;
            float z[8], y[8], gz[8], gh[8], w[8], rz_, ry_;
            rz.get(z);
            ry.get(y);
            rgz.get(gz);
            rgh.get(gh);
            if (owns && row + p.slots < hi) {
                const uint64_t b = (at + (uint64_t)p.slots * p.C) * Elem<T>::kBytes;
                rz.load(zs + b);
                ry.load(ys + b);
                rgh.load(ghs + b);
                if (gzs) rgz.load(gzs + b);
            }
            normalize<POST>(sums, p, mine, z, y, rz_, ry_);      // z, and with a post norm y, are the normalized rows now
            float st = 0.0f, sth = 0.0f;
            if (mine) {
                cols.add(0, gh, z);
                cols.add(1, gh);
                param8<T>(p.weight, col, p.param_f32, 1.0f, w);
#pragma unroll
                for (int i = 0; i < 8; i++) gh[i] *= w[i];
                st = p.layer ? sum8(gh) : 0.0f;
                sth = dot8(gh, z);
            }
            sums(st, sth);
            st *= p.inv_c;
            sth *= p.inv_c;
            if (mine) {
#pragma unroll
                for (int i = 0; i < 8; i++) gz[i] = __fmaf_rn(rz_, __fmaf_rn(-z[i], sth, gh[i] - st), gz[i]);
                Elem<T>::store8(reinterpret_cast<char *>(p.out_a) + at * Elem<T>::kBytes, gz);
#pragma unroll
                for (int i = 0; i < 8; i++) gz[i] *= p.a;         // du
                if (p.gate) {
                    if (POST) {
                        float b1[8];
                        param8<T>(p.post_weight, col, p.param_f32, 1.0f, w);
                        param8<T>(p.post_bias, col, p.param_f32, 0.0f, b1);
#pragma unroll
                        for (int i = 0; i < 8; i++) w[i] = __fmaf_rn(y[i], w[i], b1[i]);
                        cols.add(4, gz, w);
                    } else {
                        cols.add(4, gz, y);
                    }
                    param8<T>(p.gate, p.gates > 1u ? (uint64_t)g * p.C + col : col, p.param_f32, 1.0f, w);
#pragma unroll
                    for (int i = 0; i < 8; i++) gz[i] *= w[i];
                }
            }
            if (POST) {
                st = sth = 0.0f;
                if (mine) {
                    cols.add(2, gz, y);
                    cols.add(3, gz);
                    param8<T>(p.post_weight, col, p.param_f32, 1.0f, w);
#pragma unroll
                    for (int i = 0; i < 8; i++) gz[i] *= w[i];
                    st = p.layer ? sum8(gz) : 0.0f;
                    sth = dot8(gz, y);
                }
                sums(st, sth);
                st *= p.inv_c;
                sth *= p.inv_c;
#pragma unroll
                for (int i = 0; i < 8; i++) gz[i] = ry_ * __fmaf_rn(-y[i], sth, gz[i] - st);
            }
            if (mine) Elem<T>::store8(reinterpret_cast<char *>(p.out_b) + at * Elem<T>::kBytes, gz);
        }
        if (p.gate && p.gates > 1u) {
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
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
        float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
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
// eight threads per column, each over every eighth partial row in order, then in a fixed tree.
__global__ void __launch_bounds__(256) join_sums_kernel(const __grid_constant__ JoinSums p)
{
    __shared__ float s_part[8][33];
    const uint32_t c = blockIdx.x * 32u + (threadIdx.x & 31u), k = threadIdx.x >> 5, q = blockIdx.y;
    void *const out = q < 4u ? p.out[q] : p.grad_gate;
    if (!out) return;
    const uint32_t n = q < 4u ? p.n_ctas : p.per_group;
    const uint64_t stride = q < 4u ? 4ull * p.C : p.C;
    const float *src = q < 4u ? p.partial + (uint64_t)q * p.C : p.gate_partial + (uint64_t)(q - 4u) * p.per_group * p.C;
    float v = 0.0f;
    if (c < p.C) {
#pragma unroll 4
        for (uint32_t i = k; i < n; i += 8u) v += src[i * stride + c];
    }
    s_part[k][threadIdx.x & 31u] = v;
    __syncthreads();
    if (k == 0 && c < p.C) {
        float r[8];
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] = s_part[i][threadIdx.x & 31u];
        store_param(out, (q < 4u ? 0ull : (uint64_t)(q - 4u) * p.C) + c, p.param_f32, p.bf16, sum8(r));
    }
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

template <typename T> static daf_status run_join(const JoinArgs &a, cudaStream_t s)
{
    int ctas = 0;
    const uint64_t turns = (a.rows + a.slots - 1u) / a.slots;
    if (a.tpr > (uint32_t)kJoinThreads) {
        if (persistent_ctas(reinterpret_cast<const void *>(&join_kernel<T, kJoinWide>), (int)a.tpr, 0, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
        join_kernel<T, kJoinWide><<<(uint32_t)(turns < (uint64_t)ctas ? turns : ctas), a.tpr, 0, s>>>(a);
    } else {
        if (persistent_ctas(reinterpret_cast<const void *>(&join_kernel<T, kJoinThreads>), kJoinThreads, 0, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
        join_kernel<T, kJoinThreads><<<(uint32_t)(turns < (uint64_t)ctas ? turns : ctas), a.tpr * a.slots, 0, s>>>(a);
    }
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

template <typename T, bool POST> static daf_status run_join_grad(JoinArgs &a, uint32_t *grid, cudaStream_t s)
{
    int ctas = 0;
    const bool wide = a.tpr > (uint32_t)kJoinThreads;
    const uint32_t smem = wide ? kSums * a.C * 4u : 0u;
    const void *k = wide ? reinterpret_cast<const void *>(&join_grad_kernel<T, POST, kJoinWide>)
                         : reinterpret_cast<const void *>(&join_grad_kernel<T, POST, kJoinThreads>);
    if (persistent_ctas(k, wide ? (int)a.tpr : kJoinThreads, (int)smem, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    join_grid(a, ctas < (int)kJoinCtas ? (uint32_t)ctas : kJoinCtas, grid, &a.per_group);
    a.gate_partial = a.partial + (uint64_t)*grid * 4u * a.C;
    if (wide) join_grad_kernel<T, POST, kJoinWide><<<*grid, a.tpr, smem, s>>>(a);
    else join_grad_kernel<T, POST, kJoinThreads><<<*grid, a.tpr * a.slots, 0, s>>>(a);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
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
    join_sums_kernel<<<dim3((a.C + 31u) / 32u, 4u + gates), 256, 0, s>>>(f);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
