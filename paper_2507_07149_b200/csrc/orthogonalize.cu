// Orthogonalised updates: x = g / (|g| + eps), then `steps` times x = a x + (b G + c G^2) x with G = x x^T (x^T x and products
// from the right for matrices with more rows than columns: neither is ever transposed in memory).
//
// Per step three products of each matrix, m its shorter and n its longer side:
//   gram    G = x x^T            m m n multiply-adds, half of them by symmetry
//   poly    P = b G + c G G      m m m, half of them by symmetry
//   update  x' = a x + P x       2 m m n
// Bound: the tensor cores.  What is held between the products is float16, not bfloat16: 11 bits instead of 8 at the same rate,
// and the values' range is known (singular values below two), so powers of two keep them away from both ends of the type:
// x is held K times its size, G and P 2^12 times; K = |g| 2^s in [2^12, 2^13), so that the first x is g itself times a power of
// two, exact for bfloat16 (two parts: 2^12, so that no rounded factor moves all singular values at once: five steps multiply that
// by a hundred).  Relative error of the result in binary64 arithmetic with only these roundings (768 x 2304, spectra from flat to
// strongly decaying): 1.3e-3 to 5.0e-3 with x rounded at the start, 0.9e-3 to 3.4e-3 so, and at most 1.4e-3 with the linear term
// a x of the steps behind the first two taken from two float16 parts (the small singular values live there: what rounds the large
// ones away by 2^-12 is large next to them); rounding the result to bfloat16 is 1.7e-3.  Other spectra give more: an eighth of the directions
// and next to nothing else, because the linear term of the last two steps is rounded; all alike, because what rounds the diagonals of G and P
// moves all singular values the same way.  bfloat16 results of 650 matrices of 33 to 4000 rows and columns were 1.8e-3 to 3.2e-3 off in the
// middle of each of eight kinds of spectra and 4.6e-3 at worst (47 x 629, all equal).  Two parts of G, P and x in the polynomial and the
// update would bring that below the rounding (computed: 1.5e-3 at most), at three products for one.
// float16 and binary32 matrices are held in two parts throughout (three products instead of one): 7e-7, and with the sums 1e-6 (some
// directions far stronger than others) to 4.2e-6 (all alike, 8192 x 48).
//
// One persistent kernel runs all products of all steps and matrices.  Pairs of CTAs take tiles of 256 x N by a ticket, in an order
// in which whatever a tile needs comes before it; a tile waits until its matrix's tiles of the earlier products are done
// (a counter), so a pair that waits only ever waits for tiles that running pairs hold, and the matrices of a call fill one
// another's gaps.  A pair, because one SM's shared memory cannot feed its tensor core: of a product of 256 x 256 each CTA holds half of
// either operand.  Roles: the first CTA's warp 2 takes tickets, waits and tells both; warp 0 of each copies its halves of the operands
// (TMA, a copy of 16 KB for each operand and 64 of the summed dimension, warp 3 those of the second operand: a copy takes some 200
// cycles to issue whatever its size, and copies of 8 KB took longer than the products, 0.45 against 0.31 us); the first CTA's warp 1
// issues the products (two accumulators in tensor memory); eight warps of each read its half of the result's rows, form the
// polynomial or the update and store them.  Matrices of few rows have a kernel of their own (orth_small_kernel).
#include "attention.cuh"
#include "tensor_core.cuh"

namespace daf {

constexpr uint32_t kOrthThreads = 384, kOrthStages = 6, kOrthBox = 8192, kOrthStage = 4u * kOrthBox, kOrthOut = 2048, kOrthRows = 256;
constexpr uint32_t kOrthGroups = 16, kOrthMatrices = 192, kOrthSlots = 2;
constexpr uint32_t kOrthBars = 1024, kOrthSmem = kOrthBars + kOrthStages * kOrthStage + 8u * kOrthOut;
constexpr uint64_t kOrthBatch = 1ull << 27;     // elements of a batch, rows taken up to their pitch: bounds the workspace (8 to 16 bytes each)
// Binary32: sums of 128 of the summed dimension are taken in tensor memory and added up in registers.  A tensor memory sum loses about two
// units of its 24th bit at every addition of 16 products, always downwards (measured: all seventeen are cut two bits below the last of the
// largest one's 24): 4096 columns of one row 2e-5 without, 5e-7 so; segments of 64 cost a fifth of the time (results cannot run as far
// ahead), of 256 are 2.5 times as far off.  float16 does without up to 8192 rows or columns, where the loss (3e-5 to 6e-5) is far below the
// result's rounding: 403 us against 444 for the set of 768 and 2304.
constexpr uint32_t kOrthSegment = 2;            // copies of 64
constexpr float kHeld = 4096.0f;                // G and P times this
constexpr uint32_t kPrepUnits = 64;             // pieces of 256 columns of a row to a CTA of the preparing kernels

struct OrthGroup {                              // matrices of one shape and type
    // operands of the products, for each of x's two places: the Gram matrix's (of x), the polynomial's (of G), the update's
    // (across: what of a symmetric matrix lies left of its stored half)
    CUtensorMap gram_a[2], gram_b[2], poly_a, poly_b, poly_a_across, poly_b_across, upd_x[2], upd_poly, upd_poly_across;
    __half *x_at[2], *gram_at, *poly_at;        // [matrix][plane][row][pitch]; x always has two planes; of the others only tiles that
                                                // reach the diagonal or lie right of it
    uint64_t x_plane, m_plane;                  // elements of a plane
    uint32_t r, c, m, x_pitch, m_pitch, tall, planes, count, first, dtype;
    uint32_t sym_tiles, sym_cols, sym_n, upd_tiles, upd_rows, upd_n;     // of one matrix; columns of a tile
    uint32_t sym_first, upd_first, prep_ctas, prep_first;
};
struct OrthArgs {
    OrthGroup g[kOrthGroups];
    const void *in[kOrthMatrices];
    void *out[kOrthMatrices];
    uint32_t groups, matrices, steps, sym_total, upd_total, prep_total, keep_status;
    float a, b, c, eps;
    double *partial;
    float *scale;                               // K of each matrix
    uint32_t *done;                             // finished sixteenths of tiles of each matrix
    WorkspaceHeader *header;
    unsigned int *device_status;
};
static_assert(sizeof(OrthArgs) <= 32000, "kernel arguments");

// --------------------------------------------------------------------------------------------- norms, first operands
// Eight columns of a row as they lie in memory, zeros behind its end.
template <typename T> struct OrthEight {
    static constexpr int kVectors = (int)sizeof(T) / 2;
    uint4 v[kVectors];
    __device__ __forceinline__ void load(const OrthGroup &g, const T *p, uint32_t row, uint32_t col, bool here, bool wide)
    {
        const uint64_t at = (uint64_t)row * g.c + col;
#pragma unroll
        for (int i = 0; i < kVectors; i++) v[i] = make_uint4(0, 0, 0, 0);
        if (!here || col >= g.c) return;
        if (wide) {
#pragma unroll
            for (int i = 0; i < kVectors; i++) v[i] = __ldg(reinterpret_cast<const uint4 *>(p + at) + i);
            return;
        }
        T e[8];
#pragma unroll
        for (uint32_t i = 0; i < 8u; i++) e[i] = col + i < g.c ? p[at + i] : T(0.0f);
#pragma unroll
        for (int i = 0; i < kVectors; i++) v[i] = *(reinterpret_cast<const uint4 *>(e) + i);
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const
    {
        if constexpr (sizeof(T) == 2) {
            Elem<T>::widen8(v[0], x);
        } else {
            x[0] = __uint_as_float(v[0].x); x[1] = __uint_as_float(v[0].y); x[2] = __uint_as_float(v[0].z); x[3] = __uint_as_float(v[0].w);
            x[4] = __uint_as_float(v[1].x); x[5] = __uint_as_float(v[1].y); x[6] = __uint_as_float(v[1].z); x[7] = __uint_as_float(v[1].w);
        }
    }
    static __device__ __forceinline__ bool wide(const OrthGroup &g, const void *p)
    {
        return g.c % 8u == 0 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0;
    }
};
// The CTA's matrix and its share of it: units, pieces of 256 columns of a row, of which a warp takes kPrepUnits / 8 at a time.
struct PrepShare {
    uint32_t group, matrix, cta, cols, units;   // cta: within the matrix; cols: units of a row
    __device__ __forceinline__ bool place(const OrthGroup &g, uint32_t j, uint32_t *row, uint32_t *col) const      // false: no such columns
    {
        const uint32_t unit = cta * kPrepUnits + (threadIdx.x >> 5) + 8u * j;
        *row = cols == 1u ? unit : unit / cols;
        *col = (unit - *row * cols) * 256u + (threadIdx.x & 31u) * 8u;
        return unit < units && *col < g.x_pitch;
    }
};
__device__ __forceinline__ PrepShare prep_share(const OrthArgs &a)
{
    PrepShare s = {};
    while (s.group + 1u < a.groups && blockIdx.x >= a.g[s.group + 1u].prep_first) s.group++;
    const OrthGroup &g = a.g[s.group];
    const uint32_t at = blockIdx.x - g.prep_first;
    s.matrix = at / g.prep_ctas;
    s.cta = at - s.matrix * g.prep_ctas;
    s.cols = (g.c + 255u) / 256u;
    s.units = g.r * s.cols;                                         // 2^24 at most
    return s;
}
__device__ __forceinline__ double cta_sum(double v, double *s_part)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31u) == 0) s_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.0;
#pragma unroll
    for (int w = 0; w < 8; w++) v += s_part[w];
    return v;
}

constexpr uint32_t kPrepFlight = 4;             // units of a warp on their way
template <typename T> __device__ __forceinline__ double sum_squares(const OrthGroup &g, const PrepShare &s, const void *in)
{
    const bool wide = OrthEight<T>::wide(g, in);
    double sum = 0.0;
#pragma unroll 1
    for (uint32_t j0 = 0; j0 < kPrepUnits / 8u; j0 += kPrepFlight) {
        OrthEight<T> v[kPrepFlight];
#pragma unroll
        for (uint32_t j = 0; j < kPrepFlight; j++) {
            uint32_t row, col;
            const bool here = s.place(g, j0 + j, &row, &col);
            v[j].load(g, static_cast<const T *>(in), row, col, here, wide);
        }
#pragma unroll
        for (uint32_t j = 0; j < kPrepFlight; j++) {
            float x[8];
            v[j].widen(x);
#pragma unroll
            for (int e = 0; e < 8; e++) sum = fma((double)x[e], (double)x[e], sum);
        }
    }
    return sum;
}

__global__ void __launch_bounds__(256, 5) orth_norm_kernel(const __grid_constant__ OrthArgs a)
{
    __shared__ double s_part[8];
    next_may_start();
    if (blockIdx.x == 0) {
        for (uint32_t i = threadIdx.x; i < a.matrices; i += 256u) a.done[i] = 0;
        if (threadIdx.x == 0) {
            a.header->ticket = 0;
            if (!a.keep_status) a.header->status = DAF_OK;
        }
    }
    const PrepShare s = prep_share(a);
    const OrthGroup &g = a.g[s.group];
    const void *in = a.in[g.first + s.matrix];
    double sum = g.dtype == DAF_F32 ? sum_squares<float>(g, s, in) : g.dtype == DAF_F16 ? sum_squares<__half>(g, s, in) : sum_squares<__nv_bfloat16>(g, s, in);
    sum = cta_sum(sum, s_part);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

template <typename T> __device__ __forceinline__ void first_operand(const OrthArgs &a, const OrthGroup &g, const PrepShare &s, double *s_part)
{
    const T *in = static_cast<const T *>(a.in[g.first + s.matrix]);
    const bool wide = OrthEight<T>::wide(g, in);
    const double *parts = a.partial + g.prep_first + s.matrix * g.prep_ctas;
    __half *hi = g.x_at[0] + (uint64_t)s.matrix * 2u * g.x_plane, *lo = hi + g.x_plane;
    float by = 0.0f, by2 = 0.0f;
    double factor = 0.0;
#pragma unroll 1
    for (uint32_t j0 = 0; j0 < kPrepUnits / 8u; j0 += kPrepFlight) {
        OrthEight<T> v[kPrepFlight];                                // on their way while the norm is summed up
#pragma unroll
        for (uint32_t j = 0; j < kPrepFlight; j++) {
            uint32_t row, col;
            const bool here = s.place(g, j0 + j, &row, &col);
            v[j].load(g, in, row, col, here, wide);
        }
        if (j0 == 0) {
            double sum = 0.0;
#pragma unroll 4
            for (uint32_t i = threadIdx.x; i < g.prep_ctas; i += 256u) sum += parts[i];
            const double norm = sqrt(cta_sum(sum, s_part)) + (double)a.eps;
            const bool finite = norm - norm == 0.0;
            const int up = finite ? 12 - ilogb(norm) : 0;
            if (s.cta == 0 && threadIdx.x == 0)
                a.scale[g.first + s.matrix] = !finite ? __int_as_float(0x7FC00000) : g.planes == 2u ? kHeld : (float)scalbn(norm, up);
            // one part: 2^up as two factors that binary32 holds; two: any factor
            by = finite ? scalbnf(1.0f, up / 2) : __int_as_float(0x7FC00000);
            by2 = scalbnf(1.0f, up - up / 2);
            factor = (double)kHeld / norm;
        }
#pragma unroll
        for (uint32_t j = 0; j < kPrepFlight; j++) {
            uint32_t row, col;
            if (!s.place(g, j0 + j, &row, &col)) continue;          // columns up to the pitch: products read the zeros behind the end
            float x[8], rest[8];
            v[j].widen(x);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = g.planes == 2u ? (float)((double)x[e] * factor) * (by == by ? 1.0f : by) : x[e] * by * by2;
                rest[e] = x[e] - __half2float(__float2half_rn(x[e]));
            }
            Elem<__half>::store8(hi + (uint64_t)row * g.x_pitch + col, x);
            if (g.planes == 2u) Elem<__half>::store8(lo + (uint64_t)row * g.x_pitch + col, rest);
        }
    }
}

__global__ void __launch_bounds__(256, 5) orth_start_kernel(const __grid_constant__ OrthArgs a)
{
    __shared__ double s_part[8];
    next_may_start();
    wait_for_ahead();
    const PrepShare s = prep_share(a);
    const OrthGroup &g = a.g[s.group];
    if (g.dtype == DAF_F32) first_operand<float>(a, g, s, s_part);
    else if (g.dtype == DAF_F16) first_operand<__half>(a, g, s, s_part);
    else first_operand<__nv_bfloat16>(a, g, s, s_part);
}

// --------------------------------------------------------------------------------------------- the products
enum : uint32_t { kGram = 0, kPoly = 1, kUpdate = 2, kNoTile = 3 };
struct OrthTile {
    uint32_t kind, step, group, matrix, row, col;
    __device__ __forceinline__ uint4 packed() const { return make_uint4(kind | step << 8 | group << 16, matrix, row, col); }
    __device__ __forceinline__ uint32_t width(const OrthGroup &g) const { return kind == kUpdate ? g.upd_n : g.sym_n; }
    static __device__ __forceinline__ OrthTile from(uint4 v) { return {v.x & 255u, v.x >> 8 & 255u, v.x >> 16, v.y, v.z, v.w}; }
};

// ---- a pair of CTAs
__device__ __forceinline__ uint32_t pair_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_meet() { asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// The address of the CTA `rank`'s copy of something in this CTA's shared memory.
__device__ __forceinline__ uint32_t in_cta(const void *mine, uint32_t rank)
{
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(mine)), "r"(rank));
    return at;
}
__device__ __forceinline__ void arrive_in(uint32_t bar) { asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool try_from_pair(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// bar_wait for a barrier at which the other CTA arrives, too.
__device__ __forceinline__ bool wait_from_pair(uint64_t *bar, uint32_t parity, volatile uint32_t *abort_flag)
{
    if (try_from_pair(bar, parity)) return true;
    const uint64_t start = now_ns();
    while (!try_from_pair(bar, parity)) {
        if (*abort_flag) return false;
        if (now_ns() - start > kWaitNanoseconds) {
            *abort_flag = 1u;
            return false;
        }
    }
    return true;
}
// A copy into this CTA's shared memory that is counted at a barrier of either CTA.
__device__ __forceinline__ void pair_load(uint32_t dst, const CUtensorMap *map, uint32_t bar, int elem, int row, int span, int matrix)
{
    asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(elem), "r"(row), "r"(span), "r"(matrix) : "memory");
}
template <bool ADD_ALWAYS = false>
__device__ __forceinline__ void pair_product(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add = true)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 q, %4, 0;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 da, {%1, %5};\n\t"
                 "mov.b64 db, {%2, %5};\n\t@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(one), "n"(kOperandHigh), "r"((uint32_t)(ADD_ALWAYS || add)) : "memory");
}
// The barrier of each CTA in `mask` is arrived at when every product issued so far by this lane is done.
__device__ __forceinline__ void pair_done(uint32_t one, uint64_t *bar, uint32_t mask)
{
    asm volatile("{\n\t.reg .pred q;\n\t.reg .b16 m;\n\tsetp.ne.b32 q, %1, 0;\n\tcvt.u16.u32 m, %2;\n\t"
                 "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], m;\n\t}"
                 ::"r"(smem_u32(bar)), "r"(one), "r"(mask) : "memory");
}

__device__ __forceinline__ OrthTile orth_tile(const OrthArgs &a, uint32_t ticket)
{
    OrthTile t = {};
    const uint32_t per_step = 2u * a.sym_total + a.upd_total;
    t.step = ticket / per_step;
    if (t.step >= a.steps) {
        t.kind = kNoTile;
        return t;
    }
    uint32_t i = ticket - t.step * per_step;
    if (i >= 2u * a.sym_total) {
        t.kind = kUpdate;
        i -= 2u * a.sym_total;
        while (t.group + 1u < a.groups && i >= a.g[t.group + 1u].upd_first) t.group++;
        const OrthGroup &g = a.g[t.group];
        i -= g.upd_first;
        t.matrix = i / g.upd_tiles;
        i -= t.matrix * g.upd_tiles;
        const uint32_t col = i / g.upd_rows;
        t.row = (i - col * g.upd_rows) * kOrthRows;
        t.col = col * g.upd_n;
        return t;
    }
    if (i >= a.sym_total) {
        t.kind = kPoly;
        i -= a.sym_total;
    }
    while (t.group + 1u < a.groups && i >= a.g[t.group + 1u].sym_first) t.group++;
    const OrthGroup &g = a.g[t.group];
    i -= g.sym_first;
    t.matrix = i / g.sym_tiles;
    i -= t.matrix * g.sym_tiles;
    // rows of tiles from the top; of each, the tiles that reach the diagonal or lie right of it
    for (uint32_t first = 0;;) {
        const uint32_t left = g.sym_cols - first;
        if (i < left) {
            t.col = (first + i) * g.sym_n;
            return t;
        }
        i -= left;
        t.row += kOrthRows;
        first = t.row / g.sym_n;
    }
}

// What of a tile's operands lies how: keys, the length of the summed dimension; from which of its elements on an operand is
// copied along its rows.  Ahead of that it is copied across them, rows summed over: all of x where it stands that way,
// and of a symmetric matrix the part left of the stored half, whose mirror image lies in the columns of the earlier rows.
struct OrthOperands {
    uint32_t keys, along_a, along_b;
    static __device__ __forceinline__ OrthOperands of(const OrthGroup &g, const OrthTile &t)
    {
        OrthOperands o = {g.m, 0u, 0u};
        if (t.kind == kGram) {
            o.keys = g.tall ? g.r : g.c;
            o.along_a = o.along_b = g.tall ? o.keys : 0u;
        } else {
            if (t.kind == kPoly || !g.tall) o.along_a = t.row;      // a multiple of 256
            if (t.kind == kPoly || g.tall) o.along_b = t.col & ~(kOrthRows - 1u);
            if (t.kind == kUpdate && !g.tall) o.along_b = o.keys;
        }
        return o;
    }
    __device__ __forceinline__ bool cross_a(uint32_t k) const { return k < along_a; }
    __device__ __forceinline__ bool cross_b(uint32_t k) const { return k < along_b; }
};

// Waits, with a limit, until `need` tiles of the matrix are done.
__device__ __forceinline__ bool wait_tiles(const uint32_t *done, uint32_t need, volatile uint32_t *stop)
{
    uint64_t start = 0;
    for (uint32_t polls = 1;; polls++) {
        uint32_t n;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(n) : "l"(done) : "memory");
        if (n >= need) return true;
        if (*stop) return false;
        if (polls & 15u) continue;
        const uint64_t now = now_ns();
        if (!start) start = now;
        if (now - start > kWaitNanoseconds) {
            *stop = 1u;
            return false;
        }
    }
}

// A 32 x 32 block of a float16 matrix between global memory (a quarter row of 64 bytes to four lanes) and one row to a lane,
// through 2 KiB of shared memory.
struct OrthBlock {
    uint4 v[4];
    __device__ __forceinline__ void load(const __half *at, uint32_t pitch, uint32_t row, uint32_t rows, uint32_t col, uint32_t lane)
    {
#pragma unroll
        for (uint32_t q = 0; q < 4u; q++) {
            const uint32_t r = row + (lane >> 2) + 8u * q, c = col + (lane & 3u) * 8u;
            v[q] = make_uint4(0, 0, 0, 0);
            if (r < rows && c < pitch) v[q] = __ldcg(reinterpret_cast<const uint4 *>(at + (uint64_t)r * pitch + c));
        }
    }
    // afterwards the lane's own row
    __device__ __forceinline__ void to_rows(unsigned char *stage, uint32_t lane)
    {
        __syncwarp();
#pragma unroll
        for (uint32_t q = 0; q < 4u; q++) stage_piece(stage, (lane >> 2) + 8u * q, lane & 3u, v[q]);
        __syncwarp();
#pragma unroll
        for (uint32_t p = 0; p < 4u; p++) v[p] = *reinterpret_cast<const uint4 *>(stage + lane * 64u + ((p ^ (lane >> 1 & 3u)) * 16u));
    }
    __device__ __forceinline__ void add(float (&x)[32], float by) const
    {
#pragma unroll
        for (uint32_t p = 0; p < 4u; p++) {
            const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
            for (uint32_t i = 0; i < 4u; i++) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                x[8u * p + 2u * i] = __fmaf_rn(by, f.x, x[8u * p + 2u * i]);
                x[8u * p + 2u * i + 1u] = __fmaf_rn(by, f.y, x[8u * p + 2u * i + 1u]);
            }
        }
    }
    // back: from rows to the quarters
    __device__ __forceinline__ void to_quarters(unsigned char *stage, uint32_t lane)
    {
        __syncwarp();
#pragma unroll
        for (uint32_t p = 0; p < 4u; p++) stage_piece(stage, lane, p, v[p]);
        __syncwarp();
#pragma unroll
        for (uint32_t q = 0; q < 4u; q++) {
            const uint32_t r = (lane >> 2) + 8u * q;
            v[q] = *reinterpret_cast<const uint4 *>(stage + r * 64u + (((lane & 3u) ^ (r >> 1 & 3u)) * 16u));
        }
    }
    __device__ __forceinline__ void store(void *at, uint64_t pitch, uint32_t row, uint32_t rows, uint32_t col, uint32_t cols, uint32_t lane) const
    {
#pragma unroll
        for (uint32_t q = 0; q < 4u; q++) {
            const uint32_t r = row + (lane >> 2) + 8u * q, c = col + (lane & 3u) * 8u;
            if (r < rows && c < cols) *reinterpret_cast<uint4 *>(reinterpret_cast<__half *>(at) + (uint64_t)r * pitch + c) = v[q];
        }
    }
};
template <typename T> __device__ __forceinline__ void round32(const float (&x)[32], uint4 (&v)[4])
{
#pragma unroll
    for (uint32_t p = 0; p < 4u; p++)
        v[p] = make_uint4(round2<T>(x[8u * p], x[8u * p + 1u]), round2<T>(x[8u * p + 2u], x[8u * p + 3u]), round2<T>(x[8u * p + 4u], x[8u * p + 5u]),
                          round2<T>(x[8u * p + 6u], x[8u * p + 7u]));
}
// What the rounding to float16 (the row in v) has left of x.
__device__ __forceinline__ void take_away(float (&x)[32], const uint4 (&v)[4])
{
#pragma unroll
    for (uint32_t p = 0; p < 4u; p++) {
        const uint32_t w[4] = {v[p].x, v[p].y, v[p].z, v[p].w};
#pragma unroll
        for (uint32_t i = 0; i < 4u; i++) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
            x[8u * p + 2u * i] -= f.x;
            x[8u * p + 2u * i + 1u] -= f.y;
        }
    }
}
// SEGMENTS: two parts throughout, sums added up in registers every kOrthSegment copies; else as many parts as the group has.
template <bool SEGMENTS> __global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kOrthThreads, 1) orthogonalize_kernel(const __grid_constant__ OrthArgs a)
{
    extern __shared__ __align__(1024) unsigned char s_raw[];
    struct Bars {
        // full, heard, acc_empty, seg_empty, drain: the first CTA's count for both
        uint64_t full[kOrthStages], empty[kOrthStages], told[kOrthSlots], heard[kOrthSlots], acc_full[2], acc_empty[2], seg_full[2], seg_empty[2], drain, pad;
        uint4 tile[kOrthSlots];
        uint32_t tmem, abort, late;
    };
    static_assert(sizeof(Bars) <= kOrthBars, "barriers fit their place");
    Bars &bars = *reinterpret_cast<Bars *>(s_raw);
    if (smem_u32(s_raw) & 1023u) {                                 // the same for every thread of both
        if (threadIdx.x == 0) record_error(a.header, a.device_status, DAF_ERR_UNSUPPORTED);
        return;
    }
    unsigned char *const stages = s_raw + kOrthBars;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u, rank = pair_rank();
    if (threadIdx.x == 0) {
        bars.abort = bars.late = 0u;
        for (uint32_t i = 0; i < kOrthStages; i++) {
            bar_init(&bars.full[i], 1);
            bar_init(&bars.empty[i], 1);
        }
        for (uint32_t i = 0; i < kOrthSlots; i++) {
            bar_init(&bars.told[i], 1);
            bar_init(&bars.heard[i], 21);                           // eight warps of each, the products, four copiers
        }
        bar_init(&bars.drain, 1);
        for (uint32_t i = 0; i < 2u; i++) {
            bar_init(&bars.acc_full[i], 1);
            bar_init(&bars.acc_empty[i], 16);
            bar_init(&bars.seg_full[i], 1);
            bar_init(&bars.seg_empty[i], 16);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tmem_before_sync();
    __syncthreads();
    pair_meet();
    tmem_after_sync();
    const uint32_t tmem = bars.tmem;
    volatile uint32_t *const stop = &bars.abort;
    next_may_start();
    wait_for_ahead();

    if (warp == 2 && rank == 0) {                                  // ---- tickets, one tile ahead of the copies
        if (lane == 0) {
            uint32_t ticket = atomicAdd(&a.header->ticket, 1u);
            for (uint32_t n = 0;; n++) {
                const uint32_t slot = n % kOrthSlots;
                const OrthTile t = orth_tile(a, ticket);
                if (n >= kOrthSlots && !wait_from_pair(&bars.heard[slot], (n / kOrthSlots - 1u) & 1u, stop)) break;
                if (t.kind != kNoTile) {
                    ticket = atomicAdd(&a.header->ticket, 1u);
                    const OrthGroup &g = a.g[t.group];
                    const uint32_t need = 16u * (t.step * (2u * g.sym_tiles + g.upd_tiles) + t.kind * g.sym_tiles);
                    if (need && !wait_tiles(a.done + g.first + t.matrix, need, stop)) break;
                }
                const uint4 v = t.packed();
                bars.tile[slot] = v;
                asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(in_cta(&bars.tile[slot], 1)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
                bar_arrive(&bars.told[slot]);
                arrive_in(in_cta(&bars.told[slot], 1));
                if (t.kind == kNoTile) break;
            }
        }
    } else if (warp == 0 || warp == 3) {                           // ---- copies: warp 0 the first operand's, warp 3 the second's
        if (lane == 0) {
            const bool second = warp == 3, counts = rank == 0 && !second;       // counts: says how many bytes come
            uint32_t st = 0, ph = 0, issued = 0;
            for (uint32_t n = 0;; n++) {
                const uint32_t slot = n % kOrthSlots;
                if (!wait_from_pair(&bars.told[slot], n / kOrthSlots & 1u, stop)) break;
                const OrthTile t = OrthTile::from(bars.tile[slot]);
                arrive_in(in_cta(&bars.heard[slot], 0));
                if (t.kind == kNoTile) break;
                const OrthGroup &g = a.g[t.group];
                asm volatile("fence.proxy.async.global;" ::: "memory");    // what other CTAs wrote by stores is now read by copies
                const uint32_t buf = t.step & 1u;
                const OrthOperands o = OrthOperands::of(g, t);
                const uint32_t width = t.width(g);
                const int lines = (int)(second ? t.col + width / 2u * rank : t.row + 128u * rank);
                // x, held in two planes, or a symmetric matrix, in as many as the group's products take
                const bool of_x = t.kind == kGram || (t.kind == kUpdate && second != (g.tall != 0u));
                const uint32_t planes = SEGMENTS ? 2u : g.planes;
                const int matrix = (int)(t.matrix * (of_x ? 2u : planes));
                const uint32_t to = smem_u32(stages) + (second ? 2u * kOrthBox : 0u), bytes = 2u * (2u * kOrthBox + width / 128u * kOrthBox);
                bool ok = true;
                const auto copy = [&](const CUtensorMap *map, bool across, int from, int end) {
                    for (int k = from; k < end; k += 64)
                        for (uint32_t part = 0; part < planes; part++) {
                            if (issued >= kOrthStages && !(ok = bar_wait(&bars.empty[st], ph ^ 1u, stop))) return;
                            if (counts) bar_expect(&bars.full[st], bytes);
                            pair_load(to + st * kOrthStage, map, in_cta(&bars.full[st], 0), across ? 0 : k, across ? k : lines, across ? lines / 64 : 0, matrix + (int)part);
                            issued++;
                            if (++st == kOrthStages) st = 0, ph ^= 1u;
                        }
                };
                const int along = (int)(second ? o.along_b : o.along_a);
                const CUtensorMap *map, *map_across;
                if (t.kind == kPoly) {
                    map = second ? &g.poly_b : &g.poly_a;
                    map_across = second ? &g.poly_b_across : &g.poly_a_across;
                } else if (t.kind == kGram) {
                    map = map_across = second ? &g.gram_b[buf] : &g.gram_a[buf];
                } else {
                    map = of_x ? &g.upd_x[buf] : &g.upd_poly;
                    map_across = of_x ? &g.upd_x[buf] : &g.upd_poly_across;
                }
                copy(map_across, true, 0, along);
                if (ok) copy(map, false, along, (int)o.keys);
                if (!ok) break;
            }
            // Nothing may be on its way into shared memory when the CTA ends.  Normally all has long arrived: the products took it.
            if (*stop)
                for (const uint64_t start = now_ns(); now_ns() - start < 1000000u;) {}
        }
    } else if (warp == 1 && rank == 0) {                           // ---- products
        const uint32_t one = elect_lane();
        uint32_t st = 0, ph = 0, segment = 0;                       // segment: of all tiles
        const auto step_on = [&]() {
            if (++st == kOrthStages) st = 0, ph ^= 1u;
        };
        // the large parts of one operand with the small ones of the other, which lie in the stage `st`
        const auto small_parts = [&](uint32_t la, uint32_t lb, uint32_t step_a, uint32_t step_b, uint32_t desc, uint32_t to, bool add) {
            const uint32_t at = smem_u32(stages + st * kOrthStage);
            const uint32_t sa = operand_low(at, kOrthBox), sb = operand_low(at + 2u * kOrthBox, kOrthBox);
            pair_product(one, to, la, sb, desc, add);
            pair_product<true>(one, to, sa, lb, desc);
#pragma unroll
            for (uint32_t s = 1; s < 4u; s++) {
                pair_product<true>(one, to, la + s * step_a, sb + s * step_b, desc);
                pair_product<true>(one, to, sa + s * step_a, lb + s * step_b, desc);
            }
        };
        for (uint32_t n = 0;; n++) {
            const uint32_t slot = n % kOrthSlots, buf = n & 1u;
            if (!bar_wait(&bars.told[slot], n / kOrthSlots & 1u, stop)) break;
            const OrthTile t = OrthTile::from(bars.tile[slot]);
            __syncwarp();
            if (lane == 0) bar_arrive(&bars.heard[slot]);
            if (t.kind == kNoTile) break;
            if (n >= 2u && !wait_from_pair(&bars.acc_empty[buf], (n / 2u - 1u) & 1u, stop)) break;
            tmem_after_sync();
            const OrthGroup &g = a.g[t.group];
            const OrthOperands o = OrthOperands::of(g, t);
            const uint32_t plain = product_desc(false, t.width(g), false) + ((256u - 128u) >> 4 << 24);   // M = 256, where product_desc says 128
            const uint32_t rounds = (o.keys + 63u) / 64u, d = tmem + buf * 256u;
            bool ok = true;
            for (uint32_t k = 0; k < rounds; k++) {
                if (!(ok = wait_from_pair(&bars.full[st], ph, stop))) break;
                tmem_after_sync();
                // 16 of the summed dimension, in 16-byte units, and which dimension is the contiguous one
                const bool ca = o.cross_a(k * 64u), cb = o.cross_b(k * 64u);
                const uint32_t step_a = ca ? 128u : 2u, step_b = cb ? 128u : 2u, desc = plain | (ca ? 1u << 15 : 0u) | (cb ? 1u << 16 : 0u);
                const uint32_t at = smem_u32(stages + st * kOrthStage);
                const uint32_t la = operand_low(at, kOrthBox), lb = operand_low(at + 2u * kOrthBox, kOrthBox);
                if constexpr (!SEGMENTS) {
                    pair_product(one, d, la, lb, desc, k > 0);
#pragma unroll
                    for (uint32_t s = 1; s < 4u; s++) pair_product<true>(one, d, la + s * step_a, lb + s * step_b, desc);
                    if (g.planes == 2u) {                           // the stage behind holds the small parts
                        uint64_t *const first = &bars.empty[st];
                        step_on();
                        if (!(ok = wait_from_pair(&bars.full[st], ph, stop))) break;
                        tmem_after_sync();
                        small_parts(la, lb, step_a, step_b, desc, d + 128u, k > 0);
                        pair_done(one, first, 3u);
                    }
                } else {
                    // The large parts' products, a segment at a time: the accumulator cuts every sum at its last place, so results add segments
                    // up in registers.  The stage behind holds the small parts; their products have an accumulator for the whole tile.
                    const uint32_t main = tmem + (segment & 1u) * 128u, cross = tmem + 256u + buf * 128u;
                    const bool begins = k % kOrthSegment == 0;
                    if (begins && segment >= 2u && !(ok = wait_from_pair(&bars.seg_empty[segment & 1u], (segment / 2u - 1u) & 1u, stop))) break;
                    if (begins) tmem_after_sync();
                    pair_product(one, main, la, lb, desc, !begins);
#pragma unroll
                    for (uint32_t s = 1; s < 4u; s++) pair_product<true>(one, main, la + s * step_a, lb + s * step_b, desc);
                    if (k % kOrthSegment == kOrthSegment - 1u || k + 1u == rounds) {
                        pair_done(one, &bars.seg_full[segment & 1u], 3u);
                        segment++;
                    }
                    uint64_t *const first = &bars.empty[st];
                    step_on();
                    if (!(ok = wait_from_pair(&bars.full[st], ph, stop))) break;
                    tmem_after_sync();
                    small_parts(la, lb, step_a, step_b, desc, cross, k > 0);
                    pair_done(one, first, 3u);
                }
                pair_done(one, &bars.empty[st], 3u);
                step_on();
            }
            pair_done(one, &bars.acc_full[buf], 3u);
            if (!ok) break;
        }
        pair_done(one, &bars.drain, 1u);
        bar_wait(&bars.drain, 0, &bars.late);
    } else if (warp >= 4) {                                        // ---- results
        const uint32_t quarter = warp & 3u, half = (warp - 4u) >> 2;
        unsigned char *const stage = stages + kOrthStages * kOrthStage + (warp - 4u) * kOrthOut;
        uint32_t segment = 0;
        for (uint32_t n = 0;; n++) {
            const uint32_t slot = n % kOrthSlots, buf = n & 1u;
            if (!wait_from_pair(&bars.told[slot], n / kOrthSlots & 1u, stop)) break;
            const OrthTile t = OrthTile::from(bars.tile[slot]);
            __syncwarp();
            if (lane == 0) arrive_in(in_cta(&bars.heard[slot], 0));
            if (t.kind == kNoTile) break;
            const OrthGroup &g = a.g[t.group];
            const bool update = t.kind == kUpdate, gram = t.kind == kGram, last = t.step + 1u == a.steps;
            const uint32_t planes = SEGMENTS ? 2u : g.planes, chunks = SEGMENTS ? 2u : t.width(g) / 64u, row = t.row + 128u * rank + quarter * 32u;
            const uint32_t rows = update ? g.r : g.m, pitch = update ? g.x_pitch : g.m_pitch, matrix = g.first + t.matrix;
            const float k = __ldcg(a.scale + matrix);
            // what is added to the product, and factors of both
            const __half *with = update ? g.x_at[t.step & 1u] + (uint64_t)t.matrix * 2u * g.x_plane : g.gram_at + (uint64_t)t.matrix * planes * g.m_plane;
            const uint64_t plane = update ? g.x_plane : g.m_plane;
            const bool two = planes == 2u || (update && (t.step == 1u || t.step == 2u));
            const float of_product = gram ? __fdiv_rn(kHeld, k * k) : t.kind == kPoly ? a.c / kHeld : 1.0f / kHeld;
            const float of_with = update ? a.a : a.b;
            __half *to = update ? g.x_at[(t.step + 1u) & 1u] + (uint64_t)t.matrix * 2u * g.x_plane
                                : (gram ? g.gram_at : g.poly_at) + (uint64_t)t.matrix * planes * g.m_plane;
            OrthBlock ahead, ahead2;                                // of the next 32 columns, on their way during the products
            const auto look_ahead = [&](uint32_t j) {
                if (gram) return;
                const uint32_t col = t.col + (half * chunks + j) * 32u;
                ahead.load(with, pitch, row, rows, j < chunks ? col : pitch, lane);
                if (two) ahead2.load(with + plane, pitch, row, rows, j < chunks ? col : pitch, lane);
            };
            look_ahead(0);
            // one 32 x 32 block of the result, given its product
            const auto block = [&](uint32_t j, float (&x)[32]) {
                const uint32_t col = t.col + (half * chunks + j) * 32u;
                if (row >= rows || col >= pitch) return;
                OrthBlock w, w2;
                if constexpr (!SEGMENTS) {
                    w = ahead;
                    w2 = ahead2;
                    look_ahead(j + 1u);
                }
#pragma unroll
                for (int i = 0; i < 32; i++) x[i] *= of_product;
                if (!gram) {
                    OrthBlock &high = !SEGMENTS ? w : ahead, &low = !SEGMENTS ? w2 : ahead2;
                    if (two) {
                        low.to_rows(stage, lane);
                        low.add(x, of_with);
                    }
                    high.to_rows(stage, lane);
                    high.add(x, of_with);
                }
                if constexpr (SEGMENTS) look_ahead(j + 1u);         // here: before it there are no registers to be had
                if (update && last) {
                    const float by = __fdiv_rn(1.0f, k);
#pragma unroll
                    for (int i = 0; i < 32; i++) x[i] *= by;
                    char *const out = reinterpret_cast<char *>(a.out[matrix]);
                    const uint32_t eb = g.dtype == DAF_F32 ? 4u : 2u;
                    const bool wide = g.c * eb % 16u == 0 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0;
                    if (g.dtype == DAF_F32) {
                        const uint32_t ends = row + lane < rows ? g.c : 0u;             // lanes without a row store nothing
                        float *const at = reinterpret_cast<float *>(out) + (uint64_t)(row + lane) * g.c + col;
#pragma unroll
                        for (uint32_t i = 0; i < 32u; i += 4u) {
                            if (wide && col + i < ends) {
                                *reinterpret_cast<float4 *>(at + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                            } else {
#pragma unroll
                                for (uint32_t e = 0; e < 4u; e++)
                                    if (col + i + e < ends) at[i + e] = x[i + e];
                            }
                        }
                        return;
                    }
                    if (g.dtype == DAF_F16) round32<__half>(x, w.v);
                    else round32<__nv_bfloat16>(x, w.v);
                    w.to_quarters(stage, lane);
                    if (wide) w.store(out, g.c, row, rows, col, g.c, lane);
                    else if (col + lane < g.c)
                        for (uint32_t r = 0; r < 32u && row + r < rows; r++)
                            reinterpret_cast<uint16_t *>(out)[(uint64_t)(row + r) * g.c + col + lane] =
                                *reinterpret_cast<const uint16_t *>(stage + r * 64u + (((lane >> 3) ^ (r >> 1 & 3u)) * 16u) + (lane & 7u) * 2u);
                    return;
                }
                const uint32_t kept = planes == 2u || (update && t.step < 2u) ? 2u : 1u;
                for (uint32_t p = 0; p < kept; p++) {
                    round32<__half>(x, w.v);
                    if (p + 1u < kept) take_away(x, w.v);
                    w.to_quarters(stage, lane);
                    w.store(to + p * plane, pitch, row, rows, col, pitch, lane);
                }
            };
            const uint32_t own = (half * chunks) * 32u + (quarter << 21);                      // the warp's first column, its lanes
            if constexpr (!SEGMENTS) {
                if (!bar_wait(&bars.acc_full[buf], n / 2u & 1u, stop)) break;
                tmem_after_sync();
                for (uint32_t j = 0; j < chunks; j++) {
                    float x[32];
                    __syncwarp();
                    tmem_load32(tmem + buf * 256u + own + j * 32u, x);
                    tmem_wait_loads();
                    if (planes == 2u) {                             // the small parts' products
                        float small[32];
                        tmem_load32(tmem + buf * 256u + 128u + own + j * 32u, small);
                        tmem_wait_loads();
#pragma unroll
                        for (int i = 0; i < 32; i++) x[i] += small[i];
                    }
                    block(j, x);
                }
            } else {
                float x[2][32] = {}, part[32];
                const auto add = [&](uint32_t at) {
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        tmem_load32(at + own + 32u * j, part);
                        tmem_wait_loads();
#pragma unroll
                        for (int i = 0; i < 32; i++) x[j][i] += part[i];
                    }
                };
                const uint32_t rounds = (OrthOperands::of(g, t).keys + 63u) / 64u, segments = (rounds + kOrthSegment - 1u) / kOrthSegment;
                bool ok = true;
                for (uint32_t i = 0; i < segments; i++, segment++) {
                    if (!(ok = bar_wait(&bars.seg_full[segment & 1u], segment / 2u & 1u, stop))) break;
                    tmem_after_sync();
                    __syncwarp();
                    add(tmem + (segment & 1u) * 128u);
                    tmem_before_sync();
                    __syncwarp();
                    if (lane == 0) arrive_in(in_cta(&bars.seg_empty[segment & 1u], 0));
                }
                if (!ok || !bar_wait(&bars.acc_full[buf], n / 2u & 1u, stop)) break;
                tmem_after_sync();
                __syncwarp();
                add(tmem + 256u + buf * 128u);
                block(0, x[0]);
                block(1, x[1]);
            }
            tmem_before_sync();
            __syncwarp();
            if (lane == 0) arrive_in(in_cta(&bars.acc_empty[buf], 0));
            if (update && last) continue;                          // nothing waits for the result
            asm volatile("fence.proxy.async.global;" ::: "memory");
            __syncwarp();
            // each warp for itself: no meeting that one could miss
            if (lane == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(a.done + matrix) : "memory");
        }
    }
    __syncwarp();
    tmem_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && (bars.abort || bars.late)) record_error(a.header, a.device_status, DAF_ERR_TIMEOUT);
    pair_meet();                                                   // neither reaches into the other behind this
    if (warp == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

// --------------------------------------------------------------------------------------------- small matrices
// A matrix of few rows (or columns: it is held turned, so that the shorter side m is the rows) in one CTA's shared memory, all
// steps in one launch: a tensor core has nothing to do there, and what a step takes elsewhere is the way from SM to SM, 15 times
// for five steps.  The smallest are held and computed in binary64: their roundings do not average out.
// Gram matrix: a thread has 4 x 4 elements, of those that reach the diagonal or lie right of it, and every `parts`th column; the parts
// are added up in order.  Update: a thread has four rows of a column.
// One binary32 matrix here and by orthogonalize_kernel: 2 x 5 10 and 75 us, 512 x 16 35 and 113, 1 x 4096 41 and 231, 32 x 510 94 and
// 124 (150 of these 184 and 312); errors 1.4e-7 and 8.7e-7, 6.3e-7 and 1.1e-6, 1.4e-7 and 4.8e-7, 9.0e-7 and 2.4e-6.  The Gram
// matrix's parts, the polynomial, which rounds what five steps multiply by a hundred, and few rows' updates are summed in binary64
// in any case (all in binary32: 2 x 5 2e-6, 1 x 4096 1.4e-6, and 4 us less for 32 x 510).
constexpr uint32_t kSmallRows = 32, kSmallExact = 8;
template <typename S> struct OrthSmall {
    static constexpr bool kWide = sizeof(S) == 8;
    static constexpr uint32_t kThreads = kWide ? 512 : 1024, kElems = kWide ? 4096 : 16384, kPartElems = kWide ? 8192 : 16384, kParts = 64;
    S x[2][kElems + kSmallRows];                // rows of n | 1
    S part[kPartElems];
    double g[kSmallRows][kSmallRows + 1], sum[kThreads / 32];
    alignas(16) double p[kSmallRows][kSmallRows + 4];
    alignas(16) float p_float[kSmallRows][kSmallRows + 4];
};
struct OrthSmallArgs {
    const void *in[kOrthMatrices];
    void *out[kOrthMatrices];
    uint32_t r[kOrthMatrices], c[kOrthMatrices], dtype[kOrthMatrices];
    uint32_t steps;
    float a, b, c_, eps;
};

template <typename T> __device__ __forceinline__ float small_load(const void *p, uint32_t i) { return (float)static_cast<const T *>(p)[i]; }
__device__ __forceinline__ float fma_of(float a, float b, float c) { return __fmaf_rn(a, b, c); }
__device__ __forceinline__ double fma_of(double a, double b, double c) { return __fma_rn(a, b, c); }

// x' = by x + p x, summed as P.
template <typename P, typename S> __device__ __forceinline__ void small_update(const P (&p)[kSmallRows][kSmallRows + 4], P by, const S *x, S *to, uint32_t pitch,
                                                                              uint32_t rows, uint32_t n)
{
    struct alignas(16) Four { P v[4]; };
    for (uint32_t unit = threadIdx.x; unit < rows / 4u * n; unit += OrthSmall<S>::kThreads) {
        const uint32_t row = unit / n * 4u, col = unit % n;
        P acc[4];
#pragma unroll
        for (uint32_t e = 0; e < 4u; e++) acc[e] = by * (P)x[(row + e) * pitch + col];
#pragma unroll 2
        for (uint32_t k = 0; k < rows; k += 4u) {
            P v[4];
#pragma unroll
            for (uint32_t e = 0; e < 4u; e++) v[e] = (P)x[(k + e) * pitch + col];
#pragma unroll
            for (uint32_t e = 0; e < 4u; e++) {
                const Four w = *reinterpret_cast<const Four *>(&p[row + e][k]);
#pragma unroll
                for (int i = 0; i < 4; i++) acc[e] = fma_of(w.v[i], v[i], acc[e]);
            }
        }
#pragma unroll
        for (uint32_t e = 0; e < 4u; e++) to[(row + e) * pitch + col] = (S)acc[e];
    }
}

template <typename S> __global__ void __launch_bounds__(OrthSmall<S>::kThreads, 1) orth_small_kernel(const __grid_constant__ OrthSmallArgs a)
{
    using Shared = OrthSmall<S>;
    constexpr uint32_t kThreads = Shared::kThreads;
    extern __shared__ __align__(16) unsigned char s_raw[];
    Shared &s = *reinterpret_cast<Shared *>(s_raw);
    const uint32_t tid = threadIdx.x, r = a.r[blockIdx.x], c = a.c[blockIdx.x], dtype = a.dtype[blockIdx.x];
    const bool tall = r > c;
    const uint32_t m = tall ? c : r, n = tall ? r : c, pitch = n | 1u, blocks = (m + 3u) / 4u, rows = 4u * blocks;
    const void *const in = a.in[blockIdx.x];
    const auto place = [&](uint32_t i) {                            // of element i in x
        const uint32_t row = i / c, col = i - row * c;
        return tall ? col * pitch + row : row * pitch + col;
    };
    double sum = 0.0;
    for (uint32_t i = tid; i < r * c; i += kThreads) {
        const float v = dtype == DAF_F32 ? small_load<float>(in, i) : dtype == DAF_F16 ? small_load<__half>(in, i) : small_load<__nv_bfloat16>(in, i);
        s.x[0][place(i)] = v;
        sum = fma((double)v, (double)v, sum);
    }
    for (uint32_t i = m * pitch + tid; i < rows * pitch; i += kThreads) s.x[0][i] = S(0);
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((tid & 31u) == 0) s.sum[tid >> 5] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < kThreads / 32u; w++) sum += s.sum[w];
    const double norm = sqrt(sum) + (double)a.eps, factor = norm - norm == 0.0 ? 1.0 / norm : norm - norm;      // not finite: NaN
    for (uint32_t i = tid; i < r * c; i += kThreads) s.x[0][place(i)] = (S)((double)s.x[0][place(i)] * factor);
    // this thread's share of the Gram matrix
    const uint32_t tiles = blocks * (blocks + 1u) / 2u, squares = rows * rows;
    const uint32_t apart = tiles <= 1u ? 1u : 1u << (32 - __clz(tiles - 1u));
    uint32_t parts = (n + 15u) / 16u < Shared::kParts ? (n + 15u) / 16u : Shared::kParts;       // 16 columns or more
    if (parts > kThreads / apart) parts = kThreads / apart;
    if (parts * squares > Shared::kPartElems) parts = Shared::kPartElems / squares;
    uint32_t bi = 0, bj = tid & (apart - 1u);
    const uint32_t part = bj < tiles ? tid / apart : parts;         // parts: none
    while (bi < blocks && bj >= blocks - bi) {
        bj -= blocks - bi;
        bi++;
    }
    bj += bi;
    for (uint32_t step = 0; step < a.steps; step++) {
        const S *const x = s.x[step & 1u];
        __syncthreads();
        if (part < parts) {
            S acc[4][4] = {};
            const S *const xi = x + 4u * bi * pitch, *const xj = x + 4u * bj * pitch;
#pragma unroll 2
            for (uint32_t k = part; k < n; k += parts) {
                S u[4], v[4];
#pragma unroll
                for (uint32_t i = 0; i < 4u; i++) u[i] = xi[i * pitch + k], v[i] = xj[i * pitch + k];
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int j = 0; j < 4; j++) acc[i][j] = fma_of(u[i], v[j], acc[i][j]);
            }
#pragma unroll
            for (uint32_t i = 0; i < 4u; i++)
#pragma unroll
                for (uint32_t j = 0; j < 4u; j++) s.part[part * squares + (4u * bi + i) * rows + 4u * bj + j] = acc[i][j];
        }
        __syncthreads();
        for (uint32_t e = tid; e < squares; e += kThreads) {
            const uint32_t i = e / rows, j = e - i * rows;
            if (j < i) continue;
            double v = 0.0;
#pragma unroll 8
            for (uint32_t q = 0; q < parts; q++) v += (double)s.part[q * squares + e];
            s.g[i][j] = v;
            s.g[j][i] = v;
        }
        __syncthreads();
        for (uint32_t e = tid; e < squares; e += kThreads) {
            const uint32_t i = e / rows, j = e - i * rows;
            double v = 0.0;
#pragma unroll 4
            for (uint32_t k = 0; k < rows; k++) v = fma_of(s.g[i][k], s.g[j][k], v);
            v = fma_of((double)a.c_, v, (double)a.b * s.g[i][j]);
            s.p[i][j] = v;
            s.p_float[i][j] = (float)v;
        }
        __syncthreads();
        S *const to = s.x[(step + 1u) & 1u];
        if (Shared::kWide || rows <= kSmallExact) small_update(s.p, (double)a.a, x, to, pitch, rows, n);
        else small_update(s.p_float, a.a, x, to, pitch, rows, n);
    }
    __syncthreads();
    const S *const x = s.x[a.steps & 1u];
    void *const out = a.out[blockIdx.x];
    for (uint32_t i = tid; i < r * c; i += kThreads) {
        const S v = x[place(i)];
        if (dtype == DAF_F32) static_cast<float *>(out)[i] = (float)v;
        else if (dtype == DAF_F16) static_cast<__half *>(out)[i] = Shared::kWide ? __double2half((double)v) : __float2half_rn((float)v);
        else static_cast<__nv_bfloat16 *>(out)[i] = Shared::kWide ? __double2bfloat16((double)v) : __float2bfloat16_rn((float)v);
    }
    // It may have run beside the products of larger matrices: whoever waits for this launch waits for those, too.
    wait_for_ahead();
}

// --------------------------------------------------------------------------------------------- host
static uint64_t up_to(uint64_t n, uint64_t by) { return (n + by - 1u) / by * by; }

static daf_status check_orth(const daf_orthogonalize_params *p, uint32_t n, const uint32_t *dtypes, const uint64_t *rows, const uint64_t *cols)
{
    if (!p || p->struct_size != sizeof(*p) || p->reserved[0] || p->reserved[1] || p->steps == 0 || !(p->eps > 0.0f) || !(p->eps - p->eps == 0.0f) ||
        (n && (!dtypes || !rows || !cols)))
        return DAF_ERR_INVALID_ARG;
    for (const float c : p->coefficients)
        if (!(c - c == 0.0f)) return DAF_ERR_INVALID_ARG;
    if (p->steps > 64u) return DAF_ERR_UNSUPPORTED;
    for (uint32_t i = 0; i < n; i++) {
        if (dtypes[i] > DAF_BF16) return DAF_ERR_INVALID_ARG;
        if (rows[i] > 65536u || cols[i] > 65536u) return DAF_ERR_UNSUPPORTED;
    }
    return DAF_OK;
}

// Tiles of a symmetric matrix: of each 256 rows, those that reach the diagonal or lie right of it.
static uint32_t orth_sym_tiles(uint32_t m, uint32_t width)
{
    const uint32_t cols = (m + width - 1u) / width;
    uint32_t tiles = 0;
    for (uint32_t row = 0; row < m; row += kOrthRows) tiles += cols - row / width;
    return tiles;
}

// Whether one CTA does it all, holding it as S.
template <typename S> static bool orth_small(uint64_t rows, uint64_t cols)
{
    const uint64_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    return m && m <= kSmallRows && (m + 3u) / 4u * 4u * (n | 1u) <= OrthSmall<S>::kElems + kSmallRows;
}
// Parts of a matrix's operands.  With few rows roundings do not average out: one row's polynomial is one number, and five steps with
// it in one part are up to 4e-3 off; so these take two, which costs them nothing to speak of.
static uint32_t orth_planes(uint32_t dtype, uint32_t rows, uint32_t cols) { return dtype == DAF_BF16 && rows > 32u && cols > 32u ? 1u : 2u; }
// Whether sums are taken in segments.
static bool orth_segments(uint32_t dtype, uint64_t rows, uint64_t cols) { return dtype == DAF_F32 || (dtype == DAF_F16 && (rows > 8192u || cols > 8192u)); }

// The next matrices, of those that take segments or of the others, that go together, from *next on: the table without pointers to
// the workspace, and the bytes it needs.
static void orth_batch(OrthArgs *a, const daf_orthogonalize_params *p, uint32_t n, const uint32_t *dtypes, const uint64_t *rows, const uint64_t *cols,
                       bool segments, uint32_t *next, uint32_t *index, uint64_t *workspace)
{
    struct Shape {
        uint32_t r, c, dtype, count, rank;
        bool ahead(const Shape &o) const { return (r > c ? r : c) > (o.r > o.c ? o.r : o.c); }
    } shape[kOrthGroups];
    uint32_t group_of[kOrthMatrices], taken[kOrthMatrices];
    uint64_t elems = 0;
    a->groups = a->matrices = 0;
    for (; *next < n && a->matrices < kOrthMatrices; ++*next) {
        const uint32_t i = *next, r = (uint32_t)rows[i], c = (uint32_t)cols[i];
        if (r == 0 || c == 0 || orth_small<float>(r, c) || orth_segments(dtypes[i], r, c) != segments) continue;
        const uint64_t held = r * up_to(c, 64u);
        if (elems && elems + held > kOrthBatch) break;
        uint32_t k = 0;
        while (k < a->groups && (shape[k].r != r || shape[k].c != c || shape[k].dtype != dtypes[i])) k++;
        if (k == kOrthGroups) break;
        if (k == a->groups) shape[a->groups++] = {r, c, dtypes[i], 0u, 0u};
        shape[k].count++;
        group_of[a->matrices] = k;
        taken[a->matrices++] = i;
        elems += held;
    }
    // Longest side first: the Gram matrix's tiles take as long as that is, and what waits for the last of them waits least so (two
    // blocks of width 2048: a tenth of the time).
    uint32_t first[kOrthGroups], at = 0;
    for (uint32_t k = 0; k < a->groups; k++)
        for (uint32_t j = 0; j < a->groups; j++) shape[k].rank += shape[j].ahead(shape[k]) || (j < k && !shape[k].ahead(shape[j]));
    for (uint32_t k = 0; k < a->groups; k++) {
        OrthGroup &g = a->g[shape[k].rank];
        g.r = shape[k].r;
        g.c = shape[k].c;
        g.dtype = shape[k].dtype;
        g.count = shape[k].count;
    }
    for (uint32_t k = 0; k < a->groups; k++) {
        a->g[k].first = first[k] = at;
        at += a->g[k].count;
    }
    for (uint32_t i = 0; i < a->matrices; i++) index[first[shape[group_of[i]].rank]++] = taken[i];
    a->steps = p->steps;
    a->a = p->coefficients[0];
    a->b = p->coefficients[1];
    a->c = p->coefficients[2];
    a->eps = p->eps;
    a->prep_total = 0;
    // Columns of a tile, 256 or 128, as what takes less by what was measured: a wave of tiles takes 0.31 or 0.29 us for 64 of the
    // longest summed dimension, or as long as its results where that is more (3.5 or 1.8 us of a symmetric matrix, 6.5 or 2.7 of an
    // update), and once the other.  Matrices in two parts take 128: the small parts' products and segments fill the rest of tensor memory
    // (and 256 with all products in one accumulator was slower, 426 us against 403 for the set of 768 and 2304 in float16).
    const auto width = [&](bool update) {
        double cost[2] = {0.0, 0.0};
        for (int i = 0; i < 2; i++) {
            const uint32_t w = i ? 128u : 256u;
            uint64_t tiles = 0;
            uint32_t keys = 0;
            for (uint32_t k = 0; k < a->groups; k++) {
                const uint32_t r = a->g[k].r, c = a->g[k].c, m = r < c ? r : c, n = r < c ? c : r;
                if (orth_planes(a->g[k].dtype, r, c) == 2u) continue;
                tiles += (uint64_t)a->g[k].count * (update ? (uint64_t)((r + kOrthRows - 1u) / kOrthRows) * ((c + w - 1u) / w) : orth_sym_tiles(m, w));
                keys = keys > (update ? m : n) ? keys : update ? m : n;
            }
            const double products = (double)keys / 64.0 * (i ? 0.29 : 0.31), results = update ? (i ? 2.7 : 6.5) : i ? 1.8 : 3.5;
            const double more = products > results ? products : results, waves = (double)((tiles + 73u) / 74u);
            cost[i] = waves * more + products + results - more;
        }
        return cost[1] < cost[0] ? 128u : 256u;
    };
    const uint32_t sym_n = width(false), upd_n = width(true);
    uint32_t sym = 0, upd = 0;
    uint64_t bytes = sizeof(WorkspaceHeader) + up_to(2ull * kOrthMatrices * sizeof(uint32_t), 256u);
    for (uint32_t k = 0; k < a->groups; k++) {
        OrthGroup &g = a->g[k];
        g.tall = g.r > g.c;
        g.m = g.tall ? g.c : g.r;
        g.planes = orth_planes(g.dtype, g.r, g.c);
        g.x_pitch = (uint32_t)up_to(g.c, 64u);
        g.m_pitch = (uint32_t)up_to(g.m, 64u);
        g.x_plane = (uint64_t)g.r * g.x_pitch;
        g.m_plane = (uint64_t)g.m * g.m_pitch;
        g.sym_n = g.planes == 2u ? 128u : sym_n;
        g.upd_n = g.planes == 2u ? 128u : upd_n;
        g.sym_cols = (g.m + g.sym_n - 1u) / g.sym_n;
        g.sym_tiles = orth_sym_tiles(g.m, g.sym_n);
        g.upd_rows = (g.r + kOrthRows - 1u) / kOrthRows;
        g.upd_tiles = g.upd_rows * ((g.c + g.upd_n - 1u) / g.upd_n);
        g.sym_first = sym;
        g.upd_first = upd;
        sym += g.count * g.sym_tiles;
        upd += g.count * g.upd_tiles;
        g.prep_ctas = (uint32_t)(((uint64_t)g.r * ((g.c + 255u) / 256u) + kPrepUnits - 1u) / kPrepUnits);
        g.prep_first = a->prep_total;
        a->prep_total += g.count * g.prep_ctas;
        bytes += 2u * (up_to(g.count * 2u * g.x_plane * sizeof(__half), 256u) + up_to(g.count * g.planes * g.m_plane * sizeof(__half), 256u));
    }
    a->sym_total = sym;
    a->upd_total = upd;
    *workspace = bytes + up_to(a->prep_total * sizeof(double), 256u);
}

// Maps of `matrices` float16 matrices for copies of a tile's share of an operand, 64 of the summed dimension at a time: along the rows
// (`lines` rows of 64 columns; what lies behind the last row or column comes as zeros) or, where rows are summed over, across
// them (64 rows of `lines` columns in spans of 64; the columns up to the pitch are zeros in memory).
static bool orth_map(CUtensorMap *map, __half *at, uint64_t plane, uint32_t matrices, uint32_t rows, uint32_t cols, uint32_t pitch, bool across, uint32_t lines)
{
    if (across)
        return tile_map(map, false, at, {64u, rows, pitch / 64u, matrices}, {2ull * pitch, 128u, 2ull * plane}, {64u, 64u, lines / 64u, 1u}, CU_TENSOR_MAP_SWIZZLE_128B);
    return tile_map(map, false, at, {cols, rows, 1u, matrices}, {2ull * pitch, 2ull * plane, 2ull * plane}, {64u, lines, 1u, 1u}, CU_TENSOR_MAP_SWIZZLE_128B);
}

// Where a batch's buffers lie, and their maps.
static bool orth_place(OrthArgs *a, char *at)
{
    a->header = reinterpret_cast<WorkspaceHeader *>(at);
    at += sizeof(WorkspaceHeader);
    a->done = reinterpret_cast<uint32_t *>(at);
    a->scale = reinterpret_cast<float *>(a->done + kOrthMatrices);
    at += up_to(2ull * kOrthMatrices * sizeof(uint32_t), 256u);
    a->partial = reinterpret_cast<double *>(at);
    at += up_to(a->prep_total * sizeof(double), 256u);
    const auto take = [&](uint64_t halves) {
        __half *const p = reinterpret_cast<__half *>(at);
        at += up_to(halves * sizeof(__half), 256u);
        return p;
    };
    for (uint32_t k = 0; k < a->groups; k++) {
        OrthGroup &g = a->g[k];
        const uint32_t half = g.sym_n / 2u, upd_half = g.upd_n / 2u, xs = g.count * 2u, ms = g.count * g.planes;      // columns of a tile in each CTA; planes in all
        for (int i = 0; i < 2; i++) g.x_at[i] = take(xs * g.x_plane);
        g.gram_at = take(ms * g.m_plane);
        g.poly_at = take(ms * g.m_plane);
        const auto square = [&](CUtensorMap *map, __half *p, bool across, uint32_t lines) { return orth_map(map, p, g.m_plane, ms, g.m, g.m, g.m_pitch, across, lines); };
        bool ok = square(&g.poly_a, g.gram_at, false, 128u) && square(&g.poly_a_across, g.gram_at, true, 128u) && square(&g.poly_b, g.gram_at, false, half) &&
                  square(&g.poly_b_across, g.gram_at, true, half) && square(&g.upd_poly, g.poly_at, false, g.tall ? upd_half : 128u) &&
                  square(&g.upd_poly_across, g.poly_at, true, g.tall ? upd_half : 128u);
        for (int i = 0; i < 2 && ok; i++)
            ok = orth_map(&g.gram_a[i], g.x_at[i], g.x_plane, xs, g.r, g.c, g.x_pitch, g.tall, 128u) &&
                 orth_map(&g.gram_b[i], g.x_at[i], g.x_plane, xs, g.r, g.c, g.x_pitch, g.tall, half) &&
                 orth_map(&g.upd_x[i], g.x_at[i], g.x_plane, xs, g.r, g.c, g.x_pitch, !g.tall, g.tall ? 128u : upd_half);
        if (!ok) return false;
    }
    return true;
}

template <typename S> static daf_status small_ones(const daf_orthogonalize_params *p, uint32_t n, const uint32_t *dtypes, const void *const *d_in,
                                                  void *const *d_out, const uint64_t *rows, const uint64_t *cols, bool *behind, cudaStream_t s)
{
    OrthSmallArgs a;
    a.steps = p->steps;
    a.a = p->coefficients[0];
    a.b = p->coefficients[1];
    a.c_ = p->coefficients[2];
    a.eps = p->eps;
    for (uint32_t i = 0, count = 0; i < n; i++) {
        if (orth_small<S>(rows[i], cols[i]) && (sizeof(S) == 8 || !orth_small<double>(rows[i], cols[i]))) {
            a.in[count] = d_in[i];
            a.out[count] = d_out[i];
            a.r[count] = (uint32_t)rows[i];
            a.c[count] = (uint32_t)cols[i];
            a.dtype[count++] = dtypes[i];
        }
        if (count == 0 || (count < kOrthMatrices && i + 1u < n)) continue;
        const auto kernel = &orth_small_kernel<S>;
        int ctas = 0;                                               // also raises the kernel's limit of shared memory
        if (persistent_ctas(reinterpret_cast<const void *>(kernel), (int)OrthSmall<S>::kThreads, (int)sizeof(OrthSmall<S>), &ctas) != cudaSuccess) return DAF_ERR_CUDA;
        if (!*behind) kernel<<<count, OrthSmall<S>::kThreads, sizeof(OrthSmall<S>), s>>>(a);
        else if (launch_behind(kernel, count, OrthSmall<S>::kThreads, sizeof(OrthSmall<S>), s, a) != cudaSuccess) return DAF_ERR_CUDA;
        *behind = false;
        count = 0;
    }
    return DAF_OK;
}

}  // namespace daf

using namespace daf;

extern "C" uint64_t daf_orthogonalize_workspace(const daf_orthogonalize_params *params, uint32_t n, const uint32_t *dtypes, const uint64_t *rows,
                                                const uint64_t *cols)
{
    if (check_orth(params, n, dtypes, rows, cols) != DAF_OK) return 0;
    uint64_t most = sizeof(WorkspaceHeader);
    uint32_t index[kOrthMatrices];
    OrthArgs a;
    for (const bool segments : {false, true})
        for (uint32_t next = 0; next < n;) {
            uint64_t bytes = 0;
            orth_batch(&a, params, n, dtypes, rows, cols, segments, &next, index, &bytes);
            if (bytes > most) most = bytes;
        }
    return most;
}

extern "C" daf_status daf_orthogonalize(const daf_orthogonalize_params *params, uint32_t n, const uint32_t *dtypes, const void *const *d_in,
                                        void *const *d_out, const uint64_t *rows, const uint64_t *cols, void *d_workspace, uint64_t workspace_bytes,
                                        daf_stream stream)
{
    const daf_status st = check_orth(params, n, dtypes, rows, cols);
    if (st != DAF_OK) return st;
    if ((n && (!d_in || !d_out)) || !d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255u)) return DAF_ERR_INVALID_ARG;
    for (uint32_t i = 0; i < n; i++) {
        const uintptr_t mask = dtypes[i] == DAF_F32 ? 3u : 1u;
        if (rows[i] && cols[i] && (!d_in[i] || !d_out[i] || ((reinterpret_cast<uintptr_t>(d_in[i]) | reinterpret_cast<uintptr_t>(d_out[i])) & mask)))
            return DAF_ERR_INVALID_ARG;
    }
    if (workspace_bytes < daf_orthogonalize_workspace(params, n, dtypes, rows, cols)) return DAF_ERR_CAPACITY;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    uint32_t index[kOrthMatrices];
    OrthArgs a;
    bool any = false;
    for (const bool segments : {false, true}) {
        const auto kernel = segments ? &orthogonalize_kernel<true> : &orthogonalize_kernel<false>;
        for (uint32_t next = 0; next < n;) {
            uint64_t bytes = 0;
            orth_batch(&a, params, n, dtypes, rows, cols, segments, &next, index, &bytes);
            if (a.matrices == 0) break;
            int ctas = 0;
            if (persistent_ctas(reinterpret_cast<const void *>(kernel), (int)kOrthThreads, (int)kOrthSmem, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
            if (!orth_place(&a, reinterpret_cast<char *>(d_workspace)) || !(a.device_status = device_status_word())) return DAF_ERR_CUDA;
            for (uint32_t i = 0; i < a.matrices; i++) {
                a.in[i] = d_in[index[i]];
                a.out[i] = d_out[index[i]];
            }
            a.keep_status = any;
            any = true;
            orth_norm_kernel<<<a.prep_total, 256, 0, s>>>(a);
            if (launch_behind(&orth_start_kernel, a.prep_total, 256, 0, s, a) != cudaSuccess) return DAF_ERR_CUDA;
            const uint32_t most = a.sym_total > a.upd_total ? a.sym_total : a.upd_total, pairs = (uint32_t)ctas / 2u;
            if (launch_behind(kernel, 2u * (most < pairs ? most : pairs), kOrthThreads, kOrthSmem, s, a) != cudaSuccess) return DAF_ERR_CUDA;
        }
    }
    bool behind = any;                                              // the first runs beside the last batch, where SMs are free
    for (const bool wide : {true, false}) {
        const daf_status ran = wide ? small_ones<double>(params, n, dtypes, d_in, d_out, rows, cols, &behind, s)
                                    : small_ones<float>(params, n, dtypes, d_in, d_out, rows, cols, &behind, s);
        if (ran != DAF_OK) return ran;
    }
    if (!any && cudaMemsetAsync(d_workspace, 0, sizeof(uint32_t), s) != cudaSuccess) return DAF_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
