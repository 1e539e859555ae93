// Norms of queries and keys, head by head, and the rotation by position in the same pass; and the gradient.
//
//   n = x / sqrt(mean(x^2) + eps) * weight over a head's D elements, then the first `rotary` of them in pairs (a, b) turned:
//   a' = a cos - b sin, b' = a sin + b cos by the angle position * frequency of the pair.
// Backward, for the gradient g of the output and xhat = x / sqrt(mean(x^2) + eps): g' = g turned back, weight gradient
// sum g' xhat over all rows, dx = (g' w - xhat mean(g' w xhat)) / sqrt(mean(x^2) + eps).
//
// Bound: HBM (each element read once, or x and g, and written once).  A row is held by a group of lanes, 2 V elements each:
// both halves of its V pairs, so nothing but the sums crosses lanes.  A group takes several heads of ONE token, because the
// angles are the token's: with cosines and sines of a lane's V pairs computed anew for each row the arithmetic would
// bound the kernel.  Angles: a pair's frequency is held as turns per position, a 64-bit fraction of a turn; position * frequency modulo
// 2^64 is then exact in integers, however far the position, and the top 32 bits give the angle within 2^-31 half turns.
//
// The weights' gradients are summed in registers over the rows of a group, over the groups of a CTA in shared memory and over
// the CTAs by a second launch, all in a fixed order.
#include "attention.cuh"

namespace daf {

constexpr uint32_t kRotaryThreads = 256, kRotaryMaxDim = 256, kRotaryRows = 4;  // rows of a group in flight
constexpr uint32_t kRotaryCtas = 148u * 4u;     // backward: CTAs at most, and so rows of partial sums

struct RotaryArgs {
    AttnTensor x[2], y[2], g[2];                // queries and keys: inputs; outputs, or gradients of the inputs; gradients of the outputs
    const void *weight[2];                      // null: ones
    const void *positions;
    float *partial;                             // [CTA][2][D]
    uint64_t turns[kRotaryMaxDim / 2];          // frequency of each pair in 2^-64 turns per position
    long long first;
    FastDiv tokens, runs[2];                    // tokens of a sequence; runs of heads of a token
    uint32_t heads[2], run[2], items[2];        // heads of a run
    uint32_t dim, rotary, lanes_log2, pairs_apart, position_bytes, shared_positions;
    float eps, inv_dim;
};

template <typename T, int V> struct Piece;      // V elements in one or two accesses
template <> struct Piece<float, 4> {
    static __device__ __forceinline__ void load(const float *p, float (&x)[4])
    {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    }
    static __device__ __forceinline__ void store(float *p, const float (&x)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Piece<float, 8> {            // rows start on 16 bytes, not on 32
    static __device__ __forceinline__ void load(const float *p, float (&x)[8])
    {
        const float4 u = *reinterpret_cast<const float4 *>(p), v = *reinterpret_cast<const float4 *>(p + 4);
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
    }
    static __device__ __forceinline__ void store(float *p, const float (&x)[8])
    {
        *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
    }
};
template <typename T> __device__ __forceinline__ float2 widen2(uint32_t v);
template <> __device__ __forceinline__ float2 widen2<__half>(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
template <> __device__ __forceinline__ float2 widen2<__nv_bfloat16>(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)); }
template <typename T> __device__ __forceinline__ uint32_t narrow2(float a, float b);
template <> __device__ __forceinline__ uint32_t narrow2<__half>(float a, float b)
{
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t narrow2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <typename T> struct Piece<T, 4> {
    static __device__ __forceinline__ void load(const T *p, float (&x)[4])
    {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        const float2 a = widen2<T>(v.x), b = widen2<T>(v.y);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[4])
    {
        *reinterpret_cast<uint2 *>(p) = make_uint2(narrow2<T>(x[0], x[1]), narrow2<T>(x[2], x[3]));
    }
};
template <typename T> struct Piece<T, 8> {
    static __device__ __forceinline__ void load(const T *p, float (&x)[8])
    {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const float2 a = widen2<T>(v.x), b = widen2<T>(v.y), c = widen2<T>(v.z), d = widen2<T>(v.w);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y; x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
    }
    static __device__ __forceinline__ void store(T *p, const float (&x)[8])
    {
        *reinterpret_cast<uint4 *>(p) = make_uint4(narrow2<T>(x[0], x[1]), narrow2<T>(x[2], x[3]), narrow2<T>(x[4], x[5]), narrow2<T>(x[6], x[7]));
    }
};

// Cosine and sine of a fraction of a turn given by its top 32 bits.  Binary32 results: the accurate functions; 16-bit ones: the
// fast ones, whose error on [-pi, pi] (2^-21) is far below the results' rounding.
template <typename T> __device__ __forceinline__ void turn_of(uint32_t top, float *c, float *s)
{
    const float half_turns = __int2float_rn((int)top) * 4.656612873077393e-10f;       // 2^-31
    if (sizeof(T) == 4) {
        sincospif(half_turns, s, c);
    } else {
        const float angle = half_turns * 3.14159265358979324f;
        *s = __sinf(angle);
        *c = __cosf(angle);
    }
}

__device__ __forceinline__ float group_sum(float v, uint32_t lanes)
{
    for (uint32_t d = lanes >> 1; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// What a lane holds of every row: two pieces of V elements, whether they turn, and as what.
struct LaneShare {
    uint32_t at0, at1, pair;                    // elements; the first pair's index
    bool here, turns;
};
template <int V> __device__ __forceinline__ LaneShare lane_share(const RotaryArgs &a, uint32_t lane)
{
    LaneShare l;
    const uint32_t turning = a.rotary / (2u * V);
    l.here = lane < a.dim / (2u * V);
    l.turns = lane < turning;
    l.pair = lane * V;
    const bool apart = l.turns && a.pairs_apart;
    l.at0 = apart ? lane * V : lane * 2u * V;
    l.at1 = apart ? a.rotary / 2u + lane * V : l.at0 + V;
    return l;
}

template <typename T, int V> struct TokenTurns {
    float c[V], s[V];
    __device__ __forceinline__ void of(const RotaryArgs &a, const LaneShare &l, uint32_t token, uint32_t in_sequence)
    {
        if (!l.turns) return;
        const uint32_t at = a.shared_positions ? in_sequence : token;
        long long p = a.first + (long long)in_sequence;
        if (a.position_bytes == 4u) p = __ldg(reinterpret_cast<const int *>(a.positions) + at);
        if (a.position_bytes == 8u) p = __ldg(reinterpret_cast<const long long *>(a.positions) + at);
#pragma unroll
        for (int i = 0; i < V; i++) turn_of<T>((uint32_t)(((uint64_t)p * a.turns[l.pair + i]) >> 32), &c[i], &s[i]);
    }
    // forward (by +angle) or back (by -angle)
    template <bool BACK> __device__ __forceinline__ void apply(const RotaryArgs &a, const LaneShare &l, float (&x0)[V], float (&x1)[V]) const
    {
        if (!l.turns) return;
        if (a.pairs_apart) {
#pragma unroll
            for (int i = 0; i < V; i++) turn<BACK>(x0[i], x1[i], c[i], s[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; i++) {
                turn<BACK>(x0[2 * i], x0[2 * i + 1], c[i], s[i]);
                turn<BACK>(x1[2 * i], x1[2 * i + 1], c[V / 2 + i], s[V / 2 + i]);
            }
        }
    }
    template <bool BACK> static __device__ __forceinline__ void turn(float &p, float &q, float c, float s)
    {
        const float u = BACK ? __fmaf_rn(p, c, q * s) : __fmaf_rn(p, c, -(q * s));
        q = BACK ? __fmaf_rn(q, c, -(p * s)) : __fmaf_rn(q, c, p * s);
        p = u;
    }
};

template <typename P, int V> __device__ __forceinline__ void load_weight(const void *w, const LaneShare &l, float (&w0)[V], float (&w1)[V])
{
    if (w && l.here) {
        Piece<P, V>::load(reinterpret_cast<const P *>(w) + l.at0, w0);
        Piece<P, V>::load(reinterpret_cast<const P *>(w) + l.at1, w1);
        return;
    }
#pragma unroll
    for (int i = 0; i < V; i++) w0[i] = w1[i] = 1.0f;
}

template <typename T> __device__ __forceinline__ T *row_at(const AttnTensor &t, uint32_t b, uint32_t s, uint32_t h)
{
    return reinterpret_cast<T *>(t.p) + (uint64_t)b * t.sb + (uint64_t)s * t.ss + (uint64_t)h * t.sh;
}

template <typename T, typename P, int V> __global__ void __launch_bounds__(kRotaryThreads) rotary_norm_kernel(const __grid_constant__ RotaryArgs a)
{
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1u), all = a.items[0] + a.items[1];
    const uint32_t item = blockIdx.x * (kRotaryThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    const bool busy = item < all;
    const LaneShare l = lane_share<V>(a, lane);
    const bool here = l.here && busy;
    const uint32_t which = busy && item >= a.items[0] ? 1u : 0u, mine = busy ? item - (which ? a.items[0] : 0u) : 0u;
    const uint32_t token = a.runs[which].div(mine), h0 = (mine - token * a.runs[which].d) * a.run[which];
    const uint32_t b = a.tokens.div(token), s = token - b * a.tokens.d;
    const uint32_t h1 = h0 + a.run[which] < a.heads[which] ? h0 + a.run[which] : a.heads[which];
    // a warp's groups take as many turns as the longest of them (their sums cross lanes together)
    uint32_t most = a.run[0] > a.run[1] ? a.run[0] : a.run[1];
    TokenTurns<T, V> turns;
    float w0[V], w1[V];
    load_weight<P, V>(a.weight[which], l, w0, w1);
    bool first = true;
    for (uint32_t k = 0; k < most; k += kRotaryRows) {
        float x0[kRotaryRows][V], x1[kRotaryRows][V];
#pragma unroll
        for (uint32_t u = 0; u < kRotaryRows; u++) {
            if (here && h0 + k + u < h1) {
                const T *row = row_at<T>(a.x[which], b, s, h0 + k + u);
                Piece<T, V>::load(row + l.at0, x0[u]);
                Piece<T, V>::load(row + l.at1, x1[u]);
            } else {
#pragma unroll
                for (int i = 0; i < V; i++) x0[u][i] = x1[u][i] = 0.0f;
            }
        }
        if (first && here) turns.of(a, l, token, s);
        first = false;
#pragma unroll
        for (uint32_t u = 0; u < kRotaryRows; u++) {
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < V; i++) ss = __fmaf_rn(x0[u][i], x0[u][i], __fmaf_rn(x1[u][i], x1[u][i], ss));
            const float r = rsqrtf(__fmaf_rn(group_sum(ss, lanes), a.inv_dim, a.eps));
#pragma unroll
            for (int i = 0; i < V; i++) {
                x0[u][i] = x0[u][i] * r * w0[i];
                x1[u][i] = x1[u][i] * r * w1[i];
            }
            if (here && h0 + k + u < h1) {
                turns.template apply<false>(a, l, x0[u], x1[u]);
                T *row = row_at<T>(a.y[which], b, s, h0 + k + u);
                Piece<T, V>::store(row + l.at0, x0[u]);
                Piece<T, V>::store(row + l.at1, x1[u]);
            }
        }
    }
}

template <typename T, typename P, int V> __global__ void __launch_bounds__(kRotaryThreads) rotary_norm_grad_kernel(const __grid_constant__ RotaryArgs a)
{
    __shared__ float s_sum[kRotaryThreads][2 * V + 1];
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1u), groups = kRotaryThreads >> a.lanes_log2;
    const LaneShare l = lane_share<V>(a, lane);
    constexpr uint32_t kRows = kRotaryRows / 2;
    for (uint32_t which = 0; which < 2; which++) {
        float w0[V], w1[V], sum0[V] = {}, sum1[V] = {};
        load_weight<P, V>(a.weight[which], l, w0, w1);
        // the whole CTA walks together: sums cross lanes, and a warp's groups must not part
        for (uint32_t first = blockIdx.x * groups; first < a.items[which]; first += gridDim.x * groups) {
            const uint32_t item = first + (threadIdx.x >> a.lanes_log2);
            const bool here = l.here && item < a.items[which];
            const uint32_t mine = here ? item : 0u, token = a.runs[which].div(mine), h0 = (mine - token * a.runs[which].d) * a.run[which];
            const uint32_t b = a.tokens.div(token), s = token - b * a.tokens.d;
            const uint32_t h1 = h0 + a.run[which] < a.heads[which] ? h0 + a.run[which] : a.heads[which];
            TokenTurns<T, V> turns;
            for (uint32_t k = 0; k < a.run[which]; k += kRows) {
                float x0[kRows][V], x1[kRows][V], g0[kRows][V], g1[kRows][V];
#pragma unroll
                for (uint32_t u = 0; u < kRows; u++) {
                    if (here && h0 + k + u < h1) {
                        const T *row = row_at<T>(a.x[which], b, s, h0 + k + u), *grad = row_at<T>(a.g[which], b, s, h0 + k + u);
                        Piece<T, V>::load(row + l.at0, x0[u]);
                        Piece<T, V>::load(row + l.at1, x1[u]);
                        Piece<T, V>::load(grad + l.at0, g0[u]);
                        Piece<T, V>::load(grad + l.at1, g1[u]);
                    } else {
#pragma unroll
                        for (int i = 0; i < V; i++) x0[u][i] = x1[u][i] = g0[u][i] = g1[u][i] = 0.0f;
                    }
                }
                if (k == 0 && here) turns.of(a, l, token, s);
#pragma unroll
                for (uint32_t u = 0; u < kRows; u++) {
                    const bool row_here = here && h0 + k + u < h1;
                    if (row_here) turns.template apply<true>(a, l, g0[u], g1[u]);
                    float ss = 0.0f, dot = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        ss = __fmaf_rn(x0[u][i], x0[u][i], __fmaf_rn(x1[u][i], x1[u][i], ss));
                        dot = __fmaf_rn(g0[u][i] * w0[i], x0[u][i], __fmaf_rn(g1[u][i] * w1[i], x1[u][i], dot));
                    }
                    const float r = rsqrtf(__fmaf_rn(group_sum(ss, lanes), a.inv_dim, a.eps));
                    const float mean = group_sum(dot, lanes) * r * a.inv_dim;          // of g' w xhat
                    if (!row_here) continue;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float h0_ = x0[u][i] * r, h1_ = x1[u][i] * r;
                        sum0[i] = __fmaf_rn(g0[u][i], h0_, sum0[i]);
                        sum1[i] = __fmaf_rn(g1[u][i], h1_, sum1[i]);
                        x0[u][i] = r * __fmaf_rn(-h0_, mean, g0[u][i] * w0[i]);
                        x1[u][i] = r * __fmaf_rn(-h1_, mean, g1[u][i] * w1[i]);
                    }
                    T *row = row_at<T>(a.y[which], b, s, h0 + k + u);
                    Piece<T, V>::store(row + l.at0, x0[u]);
                    Piece<T, V>::store(row + l.at1, x1[u]);
                }
            }
        }
        if (!a.weight[which]) continue;
#pragma unroll
        for (int i = 0; i < V; i++) {
            s_sum[threadIdx.x][i] = sum0[i];
            s_sum[threadIdx.x][V + i] = sum1[i];
        }
        __syncthreads();
        // element j of lane t % lanes, by the threads in turn
        for (uint32_t t = threadIdx.x; t < lanes * 2u * V; t += kRotaryThreads) {
            const uint32_t owner = t & (lanes - 1u), j = t >> a.lanes_log2;
            const LaneShare o = lane_share<V>(a, owner);
            if (!o.here) continue;
            float sum = 0.0f;
            for (uint32_t g = 0; g < groups; g++) sum += s_sum[(g << a.lanes_log2) + owner][j];
            a.partial[((uint64_t)blockIdx.x * 2u + which) * a.dim + (j < V ? o.at0 + j : o.at1 + j - V)] = sum;
        }
        __syncthreads();
    }
}

// Sums the CTAs' partial sums of one weight's gradient: 32 columns to a CTA, every 32nd row to a warp.
template <typename P> __global__ void __launch_bounds__(1024) rotary_weight_kernel(const float *partial, uint32_t rows, uint32_t dim, P *q_out, P *k_out)
{
    __shared__ float s_part[32][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, col = blockIdx.x * 32u + lane;
    P *const out = blockIdx.y ? k_out : q_out;
    if (!out) return;
    float sum = 0.0f;
    if (col < dim)
#pragma unroll 4
        for (uint32_t r = warp; r < rows; r += 32u) sum += partial[((uint64_t)r * 2u + blockIdx.y) * dim + col];
    s_part[warp][lane] = sum;
    __syncthreads();
    if (warp || col >= dim) return;
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < 32; w++) sum += s_part[w][lane];
    if (sizeof(P) == 4) reinterpret_cast<float *>(out)[col] = sum;
    else reinterpret_cast<uint16_t *>(out)[col] = (uint16_t)narrow2<P>(sum, 0.0f);
}
template <> __device__ __forceinline__ uint32_t narrow2<float>(float, float) { return 0u; }    // never called: the branch above

// --------------------------------------------------------------------------------------------- host
static daf_status check_rotary(const daf_rotary_params *p, const double *frequencies)
{
    if (!p || p->struct_size != sizeof(*p) || p->dtype > DAF_BF16 || (p->param_dtype != p->dtype && p->param_dtype != DAF_F32) ||
        p->style > DAF_ROTARY_PAIRS || (p->position_bytes != 0u && p->position_bytes != 4u && p->position_bytes != 8u) || p->shared_positions > 1u ||
        p->reserved[0] || p->reserved[1] || p->reserved[2] || !(p->eps >= 0.0f) || !(p->eps - p->eps == 0.0f) ||
        (!frequencies && p->rotary_dim && (!(p->base > 0.0) || !(p->base - p->base == 0.0))))
        return DAF_ERR_INVALID_ARG;
    if (p->head_dim == 0 || p->head_dim % 8u || p->rotary_dim % 8u || p->rotary_dim > p->head_dim || p->heads == 0) return DAF_ERR_SHAPE;
    if (p->head_dim > kRotaryMaxDim || p->tokens > (1u << 24) || p->heads > 65535u || p->kv_heads > 65535u ||
        (uint64_t)p->batch * p->tokens * (p->heads > p->kv_heads ? p->heads : p->kv_heads) > 0x3FFFFFFFull)
        return DAF_ERR_UNSUPPORTED;
    if (frequencies)
        for (uint32_t i = 0; i < p->rotary_dim / 2u; i++)
            if (!(frequencies[i] - frequencies[i] == 0.0)) return DAF_ERR_INVALID_ARG;
    return DAF_OK;
}

static bool rotary_tensor(AttnTensor *t, const void *d, const uint64_t (&stride)[3], const daf_rotary_params &p, uint32_t heads)
{
    const uint32_t extent[3] = {p.batch, p.tokens, heads}, unit = p.dtype == DAF_F32 ? 4u : 8u;
    *t = {const_cast<void *>(d), stride[0], stride[1], stride[2]};
    if (!d || (reinterpret_cast<uintptr_t>(d) & 15u)) return false;
    for (int i = 0; i < 3; i++)
        if (extent[i] > 1u && (stride[i] % unit || stride[i] < p.head_dim || stride[i] >= (1ull << 36))) return false;
    return true;
}

static bool rotary_vector(const void *d, bool needed)
{
    return d ? (reinterpret_cast<uintptr_t>(d) & 15u) == 0 : !needed;
}

// Turns per position in 2^-64: the fraction of frequency / (2 pi), from products and quotients of 64-bit mantissas.
static uint64_t fraction_of_turn(long double frequency)
{
    long double t = frequency / 6.283185307179586476925286766559005768L;
    t -= __builtin_floorl(t);
    t *= 18446744073709551616.0L;
    return t >= 18446744073709551615.0L ? 0u : (uint64_t)(t + 0.5L);
}

static int rotary_piece(const daf_rotary_params &p) { return p.head_dim % 16u == 0 && p.rotary_dim % 16u == 0 ? 8 : 4; }

static RotaryArgs rotary_args(const daf_rotary_params &p, const double *frequencies)
{
    RotaryArgs a = {};
    const uint32_t pairs = p.rotary_dim / 2u;
    if (frequencies) {
        for (uint32_t i = 0; i < pairs; i++) a.turns[i] = fraction_of_turn((long double)frequencies[i]);
    } else if (pairs) {
        const long double by = __builtin_powl((long double)p.base, -2.0L / p.rotary_dim);
        long double f = 1.0L;
        for (uint32_t i = 0; i < pairs; i++, f *= by) a.turns[i] = fraction_of_turn(f);
    }
    a.first = p.first_position;
    a.heads[0] = p.heads;
    a.heads[1] = p.kv_heads;
    a.dim = p.head_dim;
    a.rotary = p.rotary_dim;
    a.pairs_apart = p.style == DAF_ROTARY_HALVES;
    a.position_bytes = p.position_bytes;
    a.shared_positions = p.shared_positions;
    a.eps = p.eps;
    a.inv_dim = 1.0f / (float)p.head_dim;
    const uint32_t units = p.head_dim / (2u * (uint32_t)rotary_piece(p));
    while ((1u << a.lanes_log2) < units) a.lanes_log2++;
    a.tokens.set(p.tokens);
    // Heads of a run: eight share a token's angles; fewer where the call is small, so that its rows spread over the SMs.
    const uint64_t tokens = (uint64_t)p.batch * p.tokens, wanted = 148u * 1024u >> a.lanes_log2;
    uint32_t run = 8u;
    while (run > 1u && tokens * ((p.heads + run - 1u) / run) < wanted) run /= 2u;
    for (int i = 0; i < 2; i++) {
        const uint32_t heads = a.heads[i] ? a.heads[i] : 1u, runs = (heads + run - 1u) / run;
        a.run[i] = (heads + runs - 1u) / runs;
        a.runs[i].set(runs);
        a.items[i] = a.heads[i] ? (uint32_t)(tokens * runs) : 0u;
    }
    return a;
}

template <typename T, typename P, int V> static daf_status rotary_launch(const RotaryArgs &a, bool back, void *gqw, void *gkw, cudaStream_t s)
{
    const uint32_t groups = kRotaryThreads >> a.lanes_log2;
    if (!back) {
        rotary_norm_kernel<T, P, V><<<(a.items[0] + a.items[1] + groups - 1u) / groups, kRotaryThreads, 0, s>>>(a);
        return DAF_OK;
    }
    const uint32_t most = a.items[0] > a.items[1] ? a.items[0] : a.items[1];
    uint32_t ctas = (most + groups - 1u) / groups;
    if (ctas > kRotaryCtas) ctas = kRotaryCtas;
    rotary_norm_grad_kernel<T, P, V><<<ctas, kRotaryThreads, 0, s>>>(a);
    if (gqw || gkw) rotary_weight_kernel<P><<<dim3((a.dim + 31u) / 32u, 2), 1024, 0, s>>>(a.partial, ctas, a.dim, reinterpret_cast<P *>(gqw), reinterpret_cast<P *>(gkw));
    return DAF_OK;
}
static daf_status rotary_by_type(const daf_rotary_params &p, const RotaryArgs &a, bool back, void *gqw, void *gkw, cudaStream_t s)
{
    const bool wide = rotary_piece(p) == 8, f32 = p.param_dtype == DAF_F32;
#define DAF_ROTARY(T, P) (wide ? rotary_launch<T, P, 8>(a, back, gqw, gkw, s) : rotary_launch<T, P, 4>(a, back, gqw, gkw, s))
    if (p.dtype == DAF_F32) return DAF_ROTARY(float, float);
    if (p.dtype == DAF_F16) return f32 ? DAF_ROTARY(__half, float) : DAF_ROTARY(__half, __half);
    return f32 ? DAF_ROTARY(__nv_bfloat16, float) : DAF_ROTARY(__nv_bfloat16, __nv_bfloat16);
#undef DAF_ROTARY
}

}  // namespace daf

using namespace daf;

extern "C" daf_status daf_rotary_norm(const daf_rotary_params *params, const double *frequencies, const void *d_q, const void *d_k, const void *d_q_weight,
                                      const void *d_k_weight, const void *d_positions, void *d_q_out, void *d_k_out, daf_stream stream)
{
    const daf_status st = check_rotary(params, frequencies);
    if (st != DAF_OK) return st;
    const daf_rotary_params &p = *params;
    if (p.batch == 0 || p.tokens == 0) return DAF_OK;
    RotaryArgs a = rotary_args(p, frequencies);
    if (!rotary_tensor(&a.x[0], d_q, p.q_stride, p, p.heads) || !rotary_tensor(&a.y[0], d_q_out, p.q_out_stride, p, p.heads) ||
        (p.kv_heads && (!rotary_tensor(&a.x[1], d_k, p.k_stride, p, p.kv_heads) || !rotary_tensor(&a.y[1], d_k_out, p.k_out_stride, p, p.kv_heads))) ||
        !rotary_vector(d_q_weight, false) || !rotary_vector(d_k_weight, false) ||
        (p.position_bytes && (!d_positions || reinterpret_cast<uintptr_t>(d_positions) % p.position_bytes)))
        return DAF_ERR_INVALID_ARG;
    a.weight[0] = d_q_weight;
    a.weight[1] = d_k_weight;
    a.positions = d_positions;
    const daf_status ran = rotary_by_type(p, a, false, nullptr, nullptr, reinterpret_cast<cudaStream_t>(stream));
    return ran != DAF_OK ? ran : cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

extern "C" uint64_t daf_rotary_norm_grad_workspace(const daf_rotary_params *params)
{
    const double unit[kRotaryMaxDim / 2] = {};
    return check_rotary(params, unit) == DAF_OK ? (uint64_t)kRotaryCtas * 2u * params->head_dim * sizeof(float) : 0u;
}

extern "C" daf_status daf_rotary_norm_grad(const daf_rotary_params *params, const double *frequencies, const void *d_q, const void *d_k, const void *d_q_weight,
                                           const void *d_k_weight, const void *d_positions, const void *d_grad_q_out, const void *d_grad_k_out, void *d_grad_q,
                                           void *d_grad_k, void *d_grad_q_weight, void *d_grad_k_weight, void *d_workspace, uint64_t workspace_bytes,
                                           daf_stream stream)
{
    const daf_status st = check_rotary(params, frequencies);
    if (st != DAF_OK) return st;
    const daf_rotary_params &p = *params;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (!rotary_vector(d_q_weight, false) || !rotary_vector(d_k_weight, false) || (d_grad_q_weight && !d_q_weight) || (d_grad_k_weight && !d_k_weight) ||
        !rotary_vector(d_grad_q_weight, false) || !rotary_vector(d_grad_k_weight, false))
        return DAF_ERR_INVALID_ARG;
    if (p.batch == 0 || p.tokens == 0) {                            // no rows: the weights' gradients are zero
        const uint64_t bytes = (uint64_t)p.head_dim * (p.param_dtype == DAF_F32 ? 4u : 2u);
        for (void *const w : {d_grad_q_weight, d_grad_k_weight})
            if (w && cudaMemsetAsync(w, 0, bytes, s) != cudaSuccess) return DAF_ERR_CUDA;
        return DAF_OK;
    }
    RotaryArgs a = rotary_args(p, frequencies);
    if (!rotary_tensor(&a.x[0], d_q, p.q_stride, p, p.heads) || !rotary_tensor(&a.g[0], d_grad_q_out, p.q_out_stride, p, p.heads) ||
        !rotary_tensor(&a.y[0], d_grad_q, p.grad_q_stride, p, p.heads) ||
        (p.kv_heads && (!rotary_tensor(&a.x[1], d_k, p.k_stride, p, p.kv_heads) || !rotary_tensor(&a.g[1], d_grad_k_out, p.k_out_stride, p, p.kv_heads) ||
                        !rotary_tensor(&a.y[1], d_grad_k, p.grad_k_stride, p, p.kv_heads))) ||
        (p.position_bytes && (!d_positions || reinterpret_cast<uintptr_t>(d_positions) % p.position_bytes)) || !rotary_vector(d_workspace, true))
        return DAF_ERR_INVALID_ARG;
    if (workspace_bytes < daf_rotary_norm_grad_workspace(params)) return DAF_ERR_CAPACITY;
    a.weight[0] = d_q_weight;
    a.weight[1] = d_k_weight;
    a.positions = d_positions;
    a.partial = reinterpret_cast<float *>(d_workspace);
    const daf_status ran = rotary_by_type(p, a, true, d_grad_q_weight, d_grad_k_weight, s);
    return ran != DAF_OK ? ran : cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
