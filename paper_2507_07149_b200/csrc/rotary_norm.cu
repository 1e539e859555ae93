// Norms of queries and keys, head by head, and the rotation by position in the same pass; and the gradient.
//
//   n = x / sqrt(mean(x^2) + eps) * weight over a head's D elements, then the first `rotary` of them in pairs (a, b) turned:
//   a' = a cos - b sin, b' = a sin + b cos by the angle position * frequency of the pair.
// Backward, for the gradient g of the output and xhat = x / sqrt(mean(x^2) + eps): g' = g turned back, weight gradient
// sum g' xhat over all rows, dx = (g' w - xhat mean(g' w xhat)) / sqrt(mean(x^2) + eps).
//
// Bound: HBM (each element read once, or x and g, and written once) as far as the instructions per row allow, which is why all of
// it is done on pairs of binary32.  A row is held by a group of lanes, 2 V elements each: both sides of its V pairs, so nothing but the
// sums crosses lanes.  A group takes several heads of ONE token, because the angles are the token's: cosines and sines of a lane's V pairs
// cost as much as a row.  Angles: a pair's frequency is held as turns per position, a 64-bit fraction of a turn; its product with the position
// modulo 2^64 is exact in integers, so that only the frequency's own rounding (2^-64 turns) grows with the position, and the top 32 bits give
// the angle within 2^-31 half turns.
//
// The weights' gradients are summed in registers over the rows of a group, over the groups of a CTA in shared memory and over
// the CTAs by a second launch, all in a fixed order.
#include "attention.cuh"
#include "pairs.cuh"

namespace daf {

constexpr uint32_t kRotaryThreads = 256, kRotaryMaxDim = 256;
// Shared memory of a thread for rows on their way and in work, and CTAs of an SM.  Measured with 4 x 8192 tokens, 16 and 4 heads of
// 128 (forward) and 64 x 197 tokens, 12 and 12 of 64 (backward), bfloat16: 128 bytes and three CTAs 73.5, 256 and two 61.6 us;
// rows held in registers instead of shared memory 72 to 76; backward 256 and two 34.0, 512 and one 42.7, three CTAs (80 registers) 38.4.
constexpr uint32_t kRotaryBytes = 256, kRotaryCtasPerSm = 2;
constexpr uint32_t kRotaryCtas = 148u * kRotaryCtasPerSm;       // backward: CTAs at most, and so rows of partial sums

struct RotaryArgs {
    AttnTensor x[2], y[2], g[2];                // queries and keys: inputs; outputs, or gradients of the inputs; gradients of the outputs
    const void *weight[2];                      // null: ones
    const void *positions;
    float *partial;                             // [CTA][2][D]
    uint64_t turns[kRotaryMaxDim / 2];          // frequency of each pair in 2^-64 turns per position
    long long first;
    FastDiv tokens, runs[2];                    // tokens of a sequence; runs of heads of a token
    uint32_t heads[2], run[2], items[2];        // heads of a run
    uint32_t dim, rotary, lanes_log2, position_bytes, shared_positions;
    float eps, inv_dim;
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
template <> __device__ __forceinline__ uint32_t narrow2<float>(float, float) { return 0u; }    // for code that a binary32 call does not reach

// V elements of a row as they lie in memory (rows start on 16 bytes).  They come through shared memory: a thread copies its own
// pieces of the rows ahead into places of its own, so nobody but the thread has to wait for them, and rows on their way take no registers.
template <typename T, int V> struct Piece {
    static constexpr int kWords = V * (int)sizeof(T) / 4, kAccess = kWords == 2 ? 8 : 16, kAccesses = kWords * 4 / kAccess;
    uint32_t w[kWords];
    // place: of access 0; the next one of the thread lies kRotaryThreads accesses behind
    static __device__ __forceinline__ void fetch(uint32_t place, const T *p)
    {
#pragma unroll
        for (int i = 0; i < kAccesses; i++) {
            const char *const from = reinterpret_cast<const char *>(p) + i * kAccess;
            const uint32_t to = place + i * kRotaryThreads * kAccess;
            if constexpr (kAccess == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(from) : "memory");
        }
    }
    __device__ __forceinline__ void take(uint32_t place)
    {
        if constexpr (kAccess == 8) {
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(place) : "memory");
        } else {
#pragma unroll
            for (int i = 0; i < kAccesses; i++)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(w[4 * i]), "=r"(w[4 * i + 1]), "=r"(w[4 * i + 2]), "=r"(w[4 * i + 3]) : "r"(place + i * kRotaryThreads * kAccess) : "memory");
        }
    }
    __device__ __forceinline__ void load(const T *p)
    {
        if constexpr (kAccess == 8) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(p));
            w[0] = v.x; w[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4 v = __ldg(reinterpret_cast<const uint4 *>(p) + i / 4);
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ float2 two(int i) const             // elements 2 i and 2 i + 1
    {
        if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
        else return widen2<T>(w[i]);
    }
    __device__ __forceinline__ void put_two(int i, float a, float b)
    {
        if constexpr (sizeof(T) == 4) {
            w[2 * i] = __float_as_uint(a);
            w[2 * i + 1] = __float_as_uint(b);
        } else {
            w[i] = narrow2<T>(a, b);
        }
    }
    __device__ __forceinline__ void store(T *p) const
    {
        if constexpr (kWords == 2) {
            *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) *(reinterpret_cast<uint4 *>(p) + i / 4) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
        }
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

// Sums over the lanes of a group, of several values side by side.
template <int N> __device__ __forceinline__ void group_sum(float (&v)[N], uint32_t lanes)
{
    for (uint32_t d = lanes >> 1; d; d >>= 1)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
}

// What a lane holds of every row: two pieces of V elements, whether they turn, and as what.
struct LaneShare {
    uint32_t at0, at1, pair;                    // elements; the first pair's index
    bool here, turns;
};
template <int V, bool HALVES> __device__ __forceinline__ LaneShare lane_share(const RotaryArgs &a, uint32_t lane)
{
    LaneShare l;
    l.here = lane < a.dim / (2u * V);
    l.turns = lane < a.rotary / (2u * V);
    l.pair = lane * V;
    const bool apart = HALVES && l.turns;
    l.at0 = apart ? lane * V : lane * 2u * V;
    l.at1 = apart ? a.rotary / 2u + lane * V : l.at0 + V;
    return l;
}

// A lane's elements of a row, as the two sides of its V pairs, two values to a register pair: all arithmetic below takes two elements an
// instruction.  HALVES: the sides are the two pieces; else they alternate in memory.  In elements that do not turn the sides
// mean nothing.
template <int V> struct Sides {
    uint64_t p[V / 2], q[V / 2];
};
template <typename T, int V, bool HALVES> __device__ __forceinline__ Sides<V> sides_of(const Piece<T, V> &u, const Piece<T, V> &v)
{
    Sides<V> x;
#pragma unroll
    for (int i = 0; i < V / 2; i++) {
        const float2 a = HALVES ? u.two(i) : i < V / 4 ? u.two(2 * i) : v.two(2 * i - V / 2);
        const float2 b = HALVES ? v.two(i) : i < V / 4 ? u.two(2 * i + 1) : v.two(2 * i + 1 - V / 2);
        x.p[i] = HALVES ? pair(a.x, a.y) : pair(a.x, b.x);
        x.q[i] = HALVES ? pair(b.x, b.y) : pair(a.y, b.y);
    }
    return x;
}
template <typename T, int V, bool HALVES> __device__ __forceinline__ void pieces_of(const Sides<V> &x, Piece<T, V> &u, Piece<T, V> &v)
{
#pragma unroll
    for (int i = 0; i < V / 2; i++) {
        if (HALVES) {
            u.put_two(i, low(x.p[i]), high(x.p[i]));
            v.put_two(i, low(x.q[i]), high(x.q[i]));
        } else if (i < V / 4) {
            u.put_two(2 * i, low(x.p[i]), low(x.q[i]));
            u.put_two(2 * i + 1, high(x.p[i]), high(x.q[i]));
        } else {
            v.put_two(2 * i - V / 2, low(x.p[i]), low(x.q[i]));
            v.put_two(2 * i + 1 - V / 2, high(x.p[i]), high(x.q[i]));
        }
    }
}
// The element of the row that value j (0 .. V-1: side p, then q) of the lane is.
template <int V, bool HALVES> __device__ __forceinline__ uint32_t element_of(const LaneShare &l, uint32_t j)
{
    if (HALVES) return j < V ? l.at0 + j : l.at1 + j - V;
    return l.at0 + (j < V ? 2u * j : 2u * (j - V) + 1u);
}

template <typename T, int V> struct TokenTurns {
    uint64_t c[V / 2], s[V / 2];
    __device__ __forceinline__ void of(const RotaryArgs &a, const LaneShare &l, uint32_t token, uint32_t in_sequence)
    {
        if (!l.turns) return;
        const uint32_t at = a.shared_positions ? in_sequence : token;
        long long p = a.first + (long long)in_sequence;
        if (a.position_bytes == 4u) p = __ldg(reinterpret_cast<const int *>(a.positions) + at);
        if (a.position_bytes == 8u) p = __ldg(reinterpret_cast<const long long *>(a.positions) + at);
#pragma unroll
        for (int i = 0; i < V / 2; i++) {
            float c0, s0, c1, s1;
            turn_of<T>((uint32_t)(((uint64_t)p * a.turns[l.pair + 2 * i]) >> 32), &c0, &s0);
            turn_of<T>((uint32_t)(((uint64_t)p * a.turns[l.pair + 2 * i + 1]) >> 32), &c1, &s1);
            c[i] = pair(c0, c1);
            s[i] = pair(s0, s1);
        }
    }
    // back (by -angle)
    __device__ __forceinline__ void back(const LaneShare &l, Sides<V> &x) const
    {
        if (!l.turns) return;
#pragma unroll
        for (int i = 0; i < V / 2; i++) {
            const uint64_t p = fma2(x.q[i], s[i], mul2(x.p[i], c[i]));
            x.q[i] = fma2(x.q[i], c[i], mul2(x.p[i], s[i] ^ 0x8000000080000000ull));
            x.p[i] = p;
        }
    }
};

template <typename P, int V, bool HALVES> __device__ __forceinline__ Sides<V> load_weight(const void *w, const LaneShare &l)
{
    Sides<V> x;
    if (w && l.here) {
        Piece<P, V> u, v;
        u.load(reinterpret_cast<const P *>(w) + l.at0);
        v.load(reinterpret_cast<const P *>(w) + l.at1);
        return sides_of<P, V, HALVES>(u, v);
    }
#pragma unroll
    for (int i = 0; i < V / 2; i++) x.p[i] = x.q[i] = both(1.0f);
    return x;
}

// A group's way through its items of work, each some heads of one token, in units of UNIT of them.  All groups of a CTA
// take the same number of units.
template <int UNIT> struct Walk {
    uint32_t item, at, rows, which, token, b, s, h;                 // at: rows ahead of the unit; rows: of the item
    __device__ __forceinline__ void enter(const RotaryArgs &a, bool here)
    {
        const uint32_t all = a.items[0] + a.items[1];
        at = 0;
        rows = 0;
        if (item >= all) return;
        which = item >= a.items[0] ? 1u : 0u;
        const uint32_t mine = which ? item - a.items[0] : item;
        const uint32_t runs = which ? a.runs[1].d : a.runs[0].d, run = which ? a.run[1] : a.run[0], heads = which ? a.heads[1] : a.heads[0];
        token = which ? a.runs[1].div(mine) : a.runs[0].div(mine);
        h = (mine - token * runs) * run;
        b = a.tokens.div(token);
        s = token - b * a.tokens.d;
        rows = !here ? 0u : heads - h < run ? heads - h : run;
    }
    __device__ __forceinline__ void next(const RotaryArgs &a, uint32_t most, uint32_t stride, bool here)
    {
        at += UNIT;
        if (at < most) return;
        item += stride;
        enter(a, here);
    }
    template <typename T> __device__ __forceinline__ T *first_row(const AttnTensor (&t)[2]) const
    {
        const AttnTensor &x = t[which];
        return reinterpret_cast<T *>(x.p) + (uint64_t)b * x.sb + (uint64_t)s * x.ss + (uint64_t)(h + at) * x.sh;
    }
};
__device__ __forceinline__ void fetch_done() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void fetched() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Units of a CTA: as many rounds over the grid as its first group needs.
template <int UNIT> __device__ __forceinline__ uint32_t walk_units(const RotaryArgs &a, uint32_t groups, uint32_t most)
{
    const uint32_t all = a.items[0] + a.items[1], first = blockIdx.x * groups, stride = gridDim.x * groups;
    return first < all ? ((all - first + stride - 1u) / stride) * ((most + UNIT - 1u) / UNIT) : 0u;
}

// Two units of a thread's rows lie in shared memory, one worked on, the next on its way.
template <typename T, typename P, int V, bool HALVES> __global__ void __launch_bounds__(kRotaryThreads, kRotaryCtasPerSm) rotary_norm_kernel(const __grid_constant__ RotaryArgs a)
{
    using Part = Piece<T, V>;
    constexpr int kUnit = (int)(kRotaryBytes / (2u * 2u * Part::kWords * 4u));
    constexpr uint32_t kPlace = Part::kWords * 4 * kRotaryThreads, kRow = 2u * kPlace;
    extern __shared__ __align__(16) unsigned char s_rows[];
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_rows) + threadIdx.x * Part::kAccess;
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1u), groups = kRotaryThreads >> a.lanes_log2, stride = gridDim.x * groups;
    const uint32_t most = a.run[0] > a.run[1] ? a.run[0] : a.run[1], units = walk_units<kUnit>(a, groups, most);
    const LaneShare l = lane_share<V, HALVES>(a, lane);
    Walk<kUnit> now = {};
    now.item = blockIdx.x * groups + (threadIdx.x >> a.lanes_log2);
    now.enter(a, l.here);
    Walk<kUnit> then = now;
    const auto ahead = [&](uint32_t half) {
        if (then.at < then.rows) {
            const T *from = then.template first_row<const T>(a.x);
            const uint64_t apart = a.x[then.which].sh;
#pragma unroll
            for (int u = 0; u < kUnit; u++) {
                if (then.at + u < then.rows) {
                    Part::fetch(ring + (half * kUnit + u) * kRow, from + l.at0);
                    Part::fetch(ring + (half * kUnit + u) * kRow + kPlace, from + l.at1);
                }
                from += apart;
            }
        }
        fetch_done();
        then.next(a, most, stride, l.here);
    };
    ahead(0);
    // weights and turns of a token as one two by two matrix for each pair: (p, q) -> (pp p + qp q, pq p + qq q)
    uint64_t pp[V / 2], qp[V / 2], pq[V / 2], qq[V / 2];
    for (uint32_t i = 0, half = 0; i < units; i++, half ^= 1u) {
        ahead(half ^ 1u);
        if (now.at == 0 && now.rows) {
            const Sides<V> w = load_weight<P, V, HALVES>(a.weight[now.which], l);
            TokenTurns<T, V> turns;
            turns.of(a, l, now.token, now.s);
#pragma unroll
            for (int e = 0; e < V / 2; e++) {
                pp[e] = w.p[e];
                qq[e] = w.q[e];
                qp[e] = pq[e] = 0ull;
                if (l.turns) {
                    pp[e] = mul2(w.p[e], turns.c[e]);
                    pq[e] = mul2(w.p[e], turns.s[e]);
                    qp[e] = mul2(w.q[e], turns.s[e]) ^ 0x8000000080000000ull;
                    qq[e] = mul2(w.q[e], turns.c[e]);
                }
            }
        }
        fetched<1>();
        const uint32_t rows = now.at < now.rows ? now.rows - now.at : 0u, place = ring + half * kUnit * kRow;
        float ss[kUnit];
#pragma unroll
        for (int u = 0; u < kUnit; u++) {
            ss[u] = 0.0f;
            if ((uint32_t)u >= rows) continue;
            Part c, d;
            c.take(place + u * kRow);
            d.take(place + u * kRow + kPlace);
            const Sides<V> x = sides_of<T, V, HALVES>(c, d);
            uint64_t sum = 0ull;
#pragma unroll
            for (int e = 0; e < V / 2; e++) sum = fma2(x.q[e], x.q[e], fma2(x.p[e], x.p[e], sum));
            ss[u] = low(sum) + high(sum);
        }
        __syncwarp();
        group_sum(ss, lanes);
        if (rows) {
            T *to = now.template first_row<T>(a.y);
            const uint64_t apart = a.y[now.which].sh;
#pragma unroll
            for (int u = 0; u < kUnit; u++) {
                if ((uint32_t)u < rows) {
                    Part c, d;
                    c.take(place + u * kRow);
                    d.take(place + u * kRow + kPlace);
                    Sides<V> x = sides_of<T, V, HALVES>(c, d);
                    const uint64_t r = both(rsqrtf(__fmaf_rn(ss[u], a.inv_dim, a.eps)));
#pragma unroll
                    for (int e = 0; e < V / 2; e++) {
                        const uint64_t p = mul2(r, fma2(x.q[e], qp[e], mul2(x.p[e], pp[e])));
                        x.q[e] = mul2(r, fma2(x.q[e], qq[e], mul2(x.p[e], pq[e])));
                        x.p[e] = p;
                    }
                    pieces_of<T, V, HALVES>(x, c, d);
                    c.store(to + l.at0);
                    d.store(to + l.at1);
                }
                to += apart;
            }
        }
        now.next(a, most, stride, l.here);
    }
    fetched<0>();
}

template <typename T, typename P, int V, bool HALVES> __global__ void __launch_bounds__(kRotaryThreads, kRotaryCtasPerSm) rotary_norm_grad_kernel(const __grid_constant__ RotaryArgs a)
{
    next_may_start();
    using Part = Piece<T, V>;
    constexpr int kUnit = (int)(kRotaryBytes / (2u * 4u * Part::kWords * 4u));
    constexpr uint32_t kPlace = Part::kWords * 4 * kRotaryThreads, kRow = 4u * kPlace;
    extern __shared__ __align__(16) unsigned char s_rows[];
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(s_rows) + threadIdx.x * Part::kAccess;
    float *const s_sum = reinterpret_cast<float *>(s_rows + 2u * kUnit * kRow);       // [2][2 V][thread]
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1u), groups = kRotaryThreads >> a.lanes_log2, stride = gridDim.x * groups;
    const uint32_t most = a.run[0] > a.run[1] ? a.run[0] : a.run[1], units = walk_units<kUnit>(a, groups, most);
    const LaneShare l = lane_share<V, HALVES>(a, lane);
    Walk<kUnit> now = {};
    now.item = blockIdx.x * groups + (threadIdx.x >> a.lanes_log2);
    now.enter(a, l.here);
    Walk<kUnit> then = now;
    const auto ahead = [&](uint32_t half) {
        if (then.at < then.rows) {
            const T *from = then.template first_row<const T>(a.x), *up = then.template first_row<const T>(a.g);
            const uint64_t apart = a.x[then.which].sh, up_apart = a.g[then.which].sh;
#pragma unroll
            for (int u = 0; u < kUnit; u++) {
                if (then.at + u < then.rows) {
                    const uint32_t place = ring + (half * kUnit + u) * kRow;
                    Part::fetch(place, from + l.at0);
                    Part::fetch(place + kPlace, from + l.at1);
                    Part::fetch(place + 2u * kPlace, up + l.at0);
                    Part::fetch(place + 3u * kPlace, up + l.at1);
                }
                from += apart;
                up += up_apart;
            }
        }
        fetch_done();
        then.next(a, most, stride, l.here);
    };
    ahead(0);
    Sides<V> sum, w;
#pragma unroll
    for (int e = 0; e < V / 2; e++) sum.p[e] = sum.q[e] = w.p[e] = w.q[e] = 0ull;
    const auto keep_sum = [&](uint32_t which) {                     // to the thread's own places; the next sums begin at zero
#pragma unroll
        for (int e = 0; e < V / 2; e++) {
            float *const at = s_sum + which * 2u * V * kRotaryThreads + threadIdx.x;
            at[(2 * e) * kRotaryThreads] = low(sum.p[e]);
            at[(2 * e + 1) * kRotaryThreads] = high(sum.p[e]);
            at[(V + 2 * e) * kRotaryThreads] = low(sum.q[e]);
            at[(V + 2 * e + 1) * kRotaryThreads] = high(sum.q[e]);
            sum.p[e] = sum.q[e] = 0ull;
        }
    };
    TokenTurns<T, V> turns;
    uint32_t side = 0;                                              // queries first, then keys
    bool weighed = false;
    for (uint32_t i = 0, half = 0; i < units; i++, half ^= 1u) {
        ahead(half ^ 1u);
        if (now.at == 0 && now.rows) {
            turns.of(a, l, now.token, now.s);
            if (now.which != side) {
                keep_sum(0);
                side = 1;
                weighed = false;
            }
            if (!weighed) w = load_weight<P, V, HALVES>(a.weight[side], l);
            weighed = true;
        }
        fetched<1>();
        const uint32_t rows = now.at < now.rows ? now.rows - now.at : 0u;
        T *to = now.template first_row<T>(a.y);
#pragma unroll
        for (int u = 0; u < kUnit; u++) {
            const bool row = (uint32_t)u < rows;
            if (!__any_sync(0xffffffffu, row)) break;
            const uint32_t place = ring + (half * kUnit + u) * kRow;
            Part c, d;
            c.take(place + 2u * kPlace);
            d.take(place + 3u * kPlace);
            Sides<V> g = sides_of<T, V, HALVES>(c, d);
            if (row) turns.back(l, g);
            c.take(place);
            d.take(place + kPlace);
            Sides<V> x = sides_of<T, V, HALVES>(c, d);
            uint64_t ss = 0ull, dot = 0ull;
#pragma unroll
            for (int e = 0; e < V / 2; e++) {
                ss = fma2(x.q[e], x.q[e], fma2(x.p[e], x.p[e], ss));
                dot = fma2(mul2(g.q[e], w.q[e]), x.q[e], fma2(mul2(g.p[e], w.p[e]), x.p[e], dot));
            }
            float sums[2] = {row ? low(ss) + high(ss) : 0.0f, row ? low(dot) + high(dot) : 0.0f};
            __syncwarp();
            group_sum(sums, lanes);
            if (row) {
                const float r1 = rsqrtf(__fmaf_rn(sums[0], a.inv_dim, a.eps));
                const uint64_t r = both(r1), mean = both(-(sums[1] * r1 * a.inv_dim));      // -(mean of g' w xhat)
#pragma unroll
                for (int e = 0; e < V / 2; e++) {
                    const uint64_t hp = mul2(x.p[e], r), hq = mul2(x.q[e], r);
                    sum.p[e] = fma2(g.p[e], hp, sum.p[e]);
                    sum.q[e] = fma2(g.q[e], hq, sum.q[e]);
                    x.p[e] = mul2(r, fma2(hp, mean, mul2(g.p[e], w.p[e])));
                    x.q[e] = mul2(r, fma2(hq, mean, mul2(g.q[e], w.q[e])));
                }
                pieces_of<T, V, HALVES>(x, c, d);
                c.store(to + l.at0);
                d.store(to + l.at1);
            }
            to += a.y[now.which].sh;
        }
        now.next(a, most, stride, l.here);
    }
    fetched<0>();
    keep_sum(side);
    if (side == 0) keep_sum(1);                                     // no keys here: zeros
    __syncthreads();
    // value j of lane t % lanes, by the threads in turn
    for (uint32_t which = 0; which < 2u; which++)
        for (uint32_t t = threadIdx.x; a.weight[which] && t < lanes * 2u * V; t += kRotaryThreads) {
            const uint32_t owner = t & (lanes - 1u), j = t >> a.lanes_log2;
            const LaneShare o = lane_share<V, HALVES>(a, owner);
            if (!o.here) continue;
            float all = 0.0f;
            for (uint32_t g = 0; g < groups; g++) all += s_sum[(which * 2u * V + j) * kRotaryThreads + (g << a.lanes_log2) + owner];
            a.partial[((uint64_t)blockIdx.x * 2u + which) * a.dim + element_of<V, HALVES>(o, j)] = all;
        }
}

// Sums the CTAs' partial sums of one weight's gradient: 32 columns to a CTA, every 32nd row to a warp.
template <typename P> __global__ void __launch_bounds__(1024) rotary_weight_kernel(const float *partial, uint32_t rows, uint32_t dim, P *q_out, P *k_out)
{
    __shared__ float s_part[32][33];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, col = blockIdx.x * 32u + lane;
    P *const out = blockIdx.y ? k_out : q_out;
    wait_for_ahead();
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
        (uint64_t)p->batch * p->tokens > 0x3FFFFFFFull / (p->heads > p->kv_heads ? p->heads : p->kv_heads))       // heads > 0; the product may pass 2^64
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

// Turns per position in 2^-64, from turns as products of 64-bit mantissas.  Off by at most 2^-64 for frequencies of up to a turn: half of it
// by this rounding or that of the product below, the rest by 1 / (2 pi).  Powers of a base of 100 or more, one product after another, stay
// within that, too (computed for bases up to 10^8); a power function for each of 64 pairs would take 20 us of the host.
static uint64_t fraction_of_turn(long double turns)
{
    if (!(turns >= 0.0L && turns < 1.0L)) turns -= __builtin_floorl(turns);
    turns *= 18446744073709551616.0L;
    if (turns >= 9223372036854775808.0L) return turns >= 18446744073709551616.0L ? 0u : (uint64_t)turns;      // whole, and a half more would be rounded
    return (uint64_t)(turns + 0.5L);
}
constexpr long double kTurnsPerRadian = 0.159154943091895335768883763372514362L;

static int rotary_piece(const daf_rotary_params &p) { return p.head_dim % 16u == 0 && p.rotary_dim % 16u == 0 ? 8 : 4; }

static RotaryArgs rotary_args(const daf_rotary_params &p, const double *frequencies)
{
    RotaryArgs a = {};
    const uint32_t pairs = p.rotary_dim / 2u;
    if (frequencies) {
        for (uint32_t i = 0; i < pairs; i++) a.turns[i] = fraction_of_turn((long double)frequencies[i] * kTurnsPerRadian);
    } else if (pairs) {
        const long double by = __builtin_powl((long double)p.base, -2.0L / p.rotary_dim);
        long double f = kTurnsPerRadian;
        for (uint32_t i = 0; i < pairs; i++, f *= by) a.turns[i] = fraction_of_turn(f);
    }
    a.first = p.first_position;
    a.heads[0] = p.heads;
    a.heads[1] = p.kv_heads;
    a.dim = p.head_dim;
    a.rotary = p.rotary_dim;
    a.position_bytes = p.position_bytes;
    a.shared_positions = p.shared_positions;
    a.eps = p.eps;
    a.inv_dim = 1.0f / (float)p.head_dim;
    const uint32_t units = p.head_dim / (2u * (uint32_t)rotary_piece(p));
    while ((1u << a.lanes_log2) < units) a.lanes_log2++;
    a.tokens.set(p.tokens);
    // Heads of a run, up to eight: as many as take the least time, a round of runs counted as its rows and what the angles and the
    // weights cost (three rows' time, with the accurate functions four: 4 x 8192 tokens 61.6 us with runs of eight that this finds, 64.3 with four).
    const uint64_t tokens = (uint64_t)p.batch * p.tokens, places = 148u * kRotaryCtasPerSm * kRotaryThreads >> a.lanes_log2;
    const uint32_t angles = p.dtype == DAF_F32 ? 4u : 3u;
    uint64_t best = ~0ull;
    for (uint32_t run = 1; run <= 8u; run++) {
        uint32_t heads_of[2], runs_of[2];
        uint64_t items = 0;
        for (int i = 0; i < 2; i++) {
            const uint32_t heads = a.heads[i] ? a.heads[i] : 1u;
            runs_of[i] = (heads + run - 1u) / run;
            heads_of[i] = (heads + runs_of[i] - 1u) / runs_of[i];
            if (a.heads[i]) items += tokens * runs_of[i];
        }
        const uint64_t cost = (items + places - 1u) / places * ((heads_of[0] > heads_of[1] ? heads_of[0] : heads_of[1]) + angles);
        if (cost >= best) continue;
        best = cost;
        for (int i = 0; i < 2; i++) {
            a.run[i] = heads_of[i];
            a.runs[i].set(runs_of[i]);
            a.items[i] = a.heads[i] ? (uint32_t)(tokens * runs_of[i]) : 0u;
        }
    }
    return a;
}

template <typename T, typename P, int V, bool HALVES> static daf_status rotary_launch(const RotaryArgs &a, bool back, void *gqw, void *gkw, cudaStream_t s)
{
    const auto kernel = back ? &rotary_norm_grad_kernel<T, P, V, HALVES> : &rotary_norm_kernel<T, P, V, HALVES>;
    const uint32_t groups = kRotaryThreads >> a.lanes_log2, wanted = (a.items[0] + a.items[1] + groups - 1u) / groups;
    const uint32_t smem = (kRotaryBytes + (back ? 4u * V * (uint32_t)sizeof(float) : 0u)) * kRotaryThreads;
    int most = 0;
    if (persistent_ctas(reinterpret_cast<const void *>(kernel), (int)kRotaryThreads, (int)smem, &most) != cudaSuccess) return DAF_ERR_CUDA;
    if (back && most > (int)kRotaryCtas) most = (int)kRotaryCtas;
    const uint32_t ctas = wanted < (uint32_t)most ? wanted : (uint32_t)most;
    kernel<<<ctas, kRotaryThreads, smem, s>>>(a);
    if (!gqw && !gkw) return DAF_OK;
    return launch_behind(&rotary_weight_kernel<P>, dim3((a.dim + 31u) / 32u, 2), 1024, 0, s, static_cast<const float *>(a.partial), ctas, a.dim,
                         reinterpret_cast<P *>(gqw), reinterpret_cast<P *>(gkw)) == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
static daf_status rotary_by_type(const daf_rotary_params &p, const RotaryArgs &a, bool back, void *gqw, void *gkw, cudaStream_t s)
{
    const bool wide = rotary_piece(p) == 8, f32 = p.param_dtype == DAF_F32, halves = p.style == DAF_ROTARY_HALVES;
#define DAF_ROTARY_V(T, P, V) (halves ? rotary_launch<T, P, V, true>(a, back, gqw, gkw, s) : rotary_launch<T, P, V, false>(a, back, gqw, gkw, s))
#define DAF_ROTARY(T, P) (wide ? DAF_ROTARY_V(T, P, 8) : DAF_ROTARY_V(T, P, 4))
    if (p.dtype == DAF_F32) return DAF_ROTARY(float, float);
    if (p.dtype == DAF_F16) return f32 ? DAF_ROTARY(__half, float) : DAF_ROTARY(__half, __half);
    return f32 ? DAF_ROTARY(__nv_bfloat16, float) : DAF_ROTARY(__nv_bfloat16, __nv_bfloat16);
#undef DAF_ROTARY
#undef DAF_ROTARY_V
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
