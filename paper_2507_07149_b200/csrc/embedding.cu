// Token embedding and its gradient.
//
//   out[t] = RNE(scale * weight[token[t]]),      grad_weight[v] = RNE(scale * sum over t with token[t] == v of grad_out[t])
//
// Forward: a gather of rows; bound by HBM (the rows named, read once from there, and the output).
//
// Backward: the sum of a row's tokens runs in the order of the tokens, in binary32 and without atomics on floats, so the
// same inputs give the same bits.  Three launches:
//   embedding_sort_kernel  one cluster of sixteen CTAs sorts (token, position) by token, keeping the order of positions: a radix
//                          sort with digits of at most nine bits, whose histograms the CTAs read from one another's shared memory.
//                          The other clusters meanwhile write zeros to the first rows of the gradient, as many as that takes.
//   embedding_sum_kernel   the sorted list is cut into chunks of equal length; a run of equal tokens inside a chunk is summed and
//                          written, the part of one that crosses a chunk's border goes to the workspace.  Equal
//                          chunks keep the SMs evenly busy however often one token occurs.  CTAs among these write zeros to the
//                          other rows that no token names, so that reads and writes share the memory.
//   embedding_join_kernel  the parts of a run that crosses borders are added up, in order.
// Few tokens take one launch instead (embedding_few_kernel).
// Bound: HBM, grad_out read once and the table's gradient written once (named rows among the first: twice).
#include "common.cuh"

namespace daf {

constexpr uint32_t kSortCtas = 16, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kDigitBits = 9, kDigits = 1u << kDigitBits;
constexpr uint32_t kRowThreads = 256;
constexpr uint32_t kLaneCols = 8;               // columns of a lane

struct EmbeddingArgs {
    const void *tokens, *weight, *grad_out;
    void *out, *grad_weight;
    uint64_t n;
    uint32_t wide_tokens, vocabulary, width, lanes_log2, slabs;   // lanes of a row, slabs of 8 * lanes columns
    float scale;
    long long padding;
    // backward
    uint32_t *keys[2], *places[2], *n_jobs;
    uint4 *jobs;                                // runs that cross borders: the chunk in which one begins, how many it touches (0: more than two), its token
    float *part;                                // [2][chunks][pitch]: runs that a chunk begins with | ends with
    uint32_t chunk, n_chunks, pitch, digit_bits, passes;
    uint32_t early_rows, fill_rows, fill_ctas, sum_ctas;   // rows cleared beside the sort; rows of a clearing CTA beside the sums, and how many of each
    uint32_t across;                            // few tokens: slabs of a CTA
    WorkspaceHeader *header;
    unsigned int *device_status;                // forward: or the caller's own
};

__device__ __forceinline__ long long token_at(const EmbeddingArgs &a, uint64_t i)
{
    return a.wide_tokens ? __ldg(reinterpret_cast<const long long *>(a.tokens) + i) : (long long)__ldg(reinterpret_cast<const int *>(a.tokens) + i);
}
__device__ __forceinline__ float get1(float v) { return v; }
__device__ __forceinline__ float get1(__half v) { return __half2float(v); }
__device__ __forceinline__ float get1(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T put1(float v);
template <> __device__ __forceinline__ float put1<float>(float v) { return v; }
template <> __device__ __forceinline__ __half put1<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 put1<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The eight columns of a lane: consecutive ones in wide accesses where every row starts on their boundary (VEC), else
// `lanes` apart, one element per access (a row's accesses are contiguous all the same).
template <bool VEC> __device__ __forceinline__ uint32_t lane_column(uint32_t lane, uint32_t lanes, uint32_t e)
{
    return VEC ? lane * kLaneCols + e : lane + lanes * e;
}
template <typename T, bool VEC> __device__ __forceinline__ void load_columns(const T *row, uint32_t first, uint32_t lanes, uint32_t width, float (&x)[8])
{
    if constexpr (VEC) {
        Elem<T>::load8(row + first, x);
    } else {
#pragma unroll
        for (uint32_t e = 0; e < kLaneCols; e++) x[e] = first + lanes * e < width ? get1(row[first + lanes * e]) : 0.0f;
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void store_columns(T *row, uint32_t first, uint32_t lanes, uint32_t width, const float (&x)[8])
{
    if constexpr (VEC) {
        Elem<T>::store8(row + first, x);
    } else {
#pragma unroll
        for (uint32_t e = 0; e < kLaneCols; e++)
            if (first + lanes * e < width) row[first + lanes * e] = put1<T>(x[e]);
    }
}

// --------------------------------------------------------------------------------------------- forward
// Slabs of a row in flight, and CTAs of an SM (48 registers): 131072 rows of 2048 from binary32 153 us; without the bound (60 registers)
// 162, two slabs 174, eight 173, one 202.
constexpr uint32_t kForwardSlabs = 4, kForwardCtas = 5;

template <typename W, typename A, bool VEC> __global__ void __launch_bounds__(kRowThreads, kForwardCtas) embedding_kernel(const __grid_constant__ EmbeddingArgs a)
{
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1u);
    const uint32_t per_row = (a.slabs + kForwardSlabs - 1u) / kForwardSlabs;
    const uint64_t items = a.n * per_row, step = (uint64_t)gridDim.x * (kRowThreads >> a.lanes_log2);
    for (uint64_t i = (uint64_t)blockIdx.x * (kRowThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2); i < items; i += step) {
        const uint64_t t = items >> 32 ? i / per_row : (uint64_t)((uint32_t)i / per_row);
        const uint32_t slab = (uint32_t)(i - t * per_row) * kForwardSlabs;
        const long long token = token_at(a, t);
        const bool known = token >= 0 && token < (long long)a.vocabulary;
        if (!known && lane == 0 && slab == 0) atomicMax(a.device_status, (unsigned int)DAF_ERR_INVALID_ARG);
        const W *src = reinterpret_cast<const W *>(a.weight) + (uint64_t)(known ? token : 0) * a.width;
        A *dst = reinterpret_cast<A *>(a.out) + t * a.width;
        float x[kForwardSlabs][8];
#pragma unroll
        for (uint32_t j = 0; j < kForwardSlabs; j++) {
            const uint32_t col = (slab + j) * lanes * kLaneCols + lane_column<VEC>(lane, lanes, 0);
            if (col < a.width && known) load_columns<W, VEC>(src, col, lanes, a.width, x[j]);
            else
#pragma unroll
                for (int e = 0; e < 8; e++) x[j][e] = 0.0f;
        }
#pragma unroll
        for (uint32_t j = 0; j < kForwardSlabs; j++) {
            const uint32_t col = (slab + j) * lanes * kLaneCols + lane_column<VEC>(lane, lanes, 0);
            if (col >= a.width) continue;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; e++) y[e] = x[j][e] * a.scale;
            store_columns<A, VEC>(dst, col, lanes, a.width, y);
        }
    }
}

// --------------------------------------------------------------------------------------------- backward: the sort
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// All threads of the cluster; writes before it, to global memory too, are seen behind it.
__device__ __forceinline__ void cluster_meet()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t read_peer(const uint32_t *mine, uint32_t rank)
{
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

struct SortShared {
    uint32_t count[kSortWarps][kDigits];        // of each warp; then where its next item of a digit goes, from the digit's base on
    uint32_t total[kDigits], base[kDigits], warp_sum[kDigits / 32];
    uint32_t unknown;
};

// Zeros to `bytes` bytes, by CTA `cta` of `ctas`: copies of a zeroed piece of shared memory, which keep the memory busier than the
// threads' own stores, and those for what lies off the copies' boundaries.
constexpr uint32_t kFillPiece = 32768;
__device__ void fill_zeros(char *at, uint64_t bytes, unsigned char *zeros, uint32_t cta, uint32_t ctas)
{
    for (uint32_t i = threadIdx.x; i < kFillPiece / 16u; i += kSortThreads) reinterpret_cast<uint4 *>(zeros)[i] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    const uint64_t off = (16u - (reinterpret_cast<uintptr_t>(at) & 15u)) & 15u, head = off < bytes ? off : bytes;
    const uint64_t middle = (bytes - head) & ~15ull, tail = head + middle;
    if (cta == 0) {
        if (threadIdx.x < head / 2u) reinterpret_cast<uint16_t *>(at)[threadIdx.x] = 0;
        if (threadIdx.x < (bytes - tail) / 2u) reinterpret_cast<uint16_t *>(at + tail)[threadIdx.x] = 0;
    }
    if (threadIdx.x) return;
    for (uint64_t piece = (uint64_t)cta * kFillPiece; piece < middle; piece += (uint64_t)ctas * kFillPiece) {
        const uint32_t n = middle - piece < kFillPiece ? (uint32_t)(middle - piece) : kFillPiece;
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                     ::"l"(at + head + piece), "r"((uint32_t)__cvta_generic_to_shared(zeros)), "r"(n) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        asm volatile("cp.async.bulk.wait_group 4;" ::: "memory");
    }
    asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// The lanes with the same digit as this one, among those with an item, from a vote on each bit (one instruction that compares all
// lanes takes the distinct digits one after the other: 131072 tokens, eight CTAs, 76 us instead of 67).
__device__ __forceinline__ uint32_t same_digit(uint32_t digit, uint32_t bits, uint32_t items)
{
    uint32_t same = items;
#pragma unroll
    for (uint32_t b = 0; b < kDigitBits; b++) {
        if (b >= bits) break;
        const uint32_t set = __ballot_sync(0xffffffffu, digit >> b & 1u);
        same &= digit >> b & 1u ? set : ~set;
    }
    return same;
}
// One round of a warp: where each lane's item lies among those of the digit in this warp so far, and the count moved on.
__device__ __forceinline__ uint32_t place_in_warp(uint32_t *count, uint32_t digit, uint32_t bits, bool item, uint32_t lane)
{
    const uint32_t same = same_digit(digit, bits, __ballot_sync(0xffffffffu, item));
    const uint32_t below = __popc(same & ((1u << lane) - 1u)), before = item ? count[digit] : 0u;
    __syncwarp();
    if (item && below == 0u) count[digit] = before + __popc(same);
    __syncwarp();
    return before + below;
}

__global__ void __cluster_dims__(kSortCtas, 1, 1) __launch_bounds__(kSortThreads) embedding_sort_kernel(const __grid_constant__ EmbeddingArgs a, uint32_t table_bytes)
{
    extern __shared__ __align__(128) unsigned char raw[];
    SortShared &s = *reinterpret_cast<SortShared *>(raw);
    next_may_start();
    if (blockIdx.x >= kSortCtas) {
        fill_zeros(reinterpret_cast<char *>(a.grad_weight), (uint64_t)a.early_rows * a.width * table_bytes, raw, blockIdx.x - kSortCtas, gridDim.x - kSortCtas);
        return;
    }
    const uint32_t rank = cluster_rank(), lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, digits = 1u << a.digit_bits;
    // every warp has a run of the list, in the order of the warps
    const uint64_t per_warp = (a.n + kSortCtas * kSortThreads - 1u) / (kSortCtas * kSortThreads) * 32u;
    const uint64_t lo = (uint64_t)(rank * kSortWarps + warp) * per_warp, end = lo + per_warp < a.n ? lo + per_warp : a.n;
    if (threadIdx.x == 0) {
        s.unknown = 0;
        if (rank == 0) {
            *a.n_jobs = 0;
            a.header->status = DAF_OK;
        }
    }
    __syncthreads();
    for (uint32_t pass = 0; pass < a.passes; pass++) {
        const uint32_t shift = pass * a.digit_bits, from = (pass + 1u) & 1u, to = pass & 1u;
        const auto key_of = [&](uint64_t i) -> uint32_t {
            if (pass) return __ldcg(a.keys[from] + i);
            const long long t = token_at(a, i);
            return t < 0 || t >= (long long)a.vocabulary || t == a.padding ? a.vocabulary : (uint32_t)t;
        };
        for (uint32_t d = lane; d < digits; d += 32u) s.count[warp][d] = 0;
        __syncwarp();
        bool unknown = false;
        uint32_t key[4], rank_in_warp[4];                           // of the last four rounds
        for (uint64_t at = lo; at < end; at += 128u) {              // four rounds, their loads together
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const uint64_t i = at + j * 32u + lane;
                key[j] = i < end ? key_of(i) : 0u;
                if (pass == 0 && i < end && key[j] == a.vocabulary) {
                    const long long t = token_at(a, i);
                    unknown |= t < 0 || t >= (long long)a.vocabulary;
                }
            }
#pragma unroll
            for (uint32_t j = 0; j < 4; j++)
                if (at + j * 32u < end)
                    rank_in_warp[j] = place_in_warp(s.count[warp], key[j] >> shift & (digits - 1u), a.digit_bits, at + j * 32u + lane < end, lane);
        }
        if (unknown) s.unknown = 1;
        __syncthreads();
        uint32_t all = 0, before = 0;
        if (threadIdx.x < digits) {
            uint32_t sum = 0;
#pragma unroll 8
            for (uint32_t w = 0; w < kSortWarps; w++) {
                const uint32_t c = s.count[w][threadIdx.x];
                s.count[w][threadIdx.x] = sum;
                sum += c;
            }
            s.total[threadIdx.x] = sum;
        }
        cluster_meet();
        if (threadIdx.x < digits) {
#pragma unroll
            for (uint32_t r = 0; r < kSortCtas; r++) {
                const uint32_t c = read_peer(&s.total[threadIdx.x], r);
                before += r < rank ? c : 0u;
                all += c;
            }
        }
        uint32_t upto = all;                                        // sum over this and the lower digits
#pragma unroll
        for (uint32_t d = 1; d < 32u; d <<= 1) {
            const uint32_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31u && warp < kDigits / 32u) s.warp_sum[warp] = upto;
        __syncthreads();
        if (threadIdx.x < digits) {
            uint32_t lower = 0;
            for (uint32_t w = 0; w < warp; w++) lower += s.warp_sum[w];
            s.base[threadIdx.x] = lower + upto - all + before;
        }
        __syncthreads();
        const bool once = per_warp <= 128u;                         // what the first look found is still at hand
        for (uint64_t at = lo; at < end; at += 128u) {
            uint32_t place[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                const uint64_t i = at + j * 32u + lane;
                if (!once) key[j] = i < end ? key_of(i) : 0u;
                place[j] = i < end ? (pass ? __ldcg(a.places[from] + i) : (uint32_t)i) : 0u;
            }
#pragma unroll
            for (uint32_t j = 0; j < 4; j++) {
                if (at + j * 32u >= end) break;
                const bool item = at + j * 32u + lane < end;
                const uint32_t digit = key[j] >> shift & (digits - 1u);
                const uint32_t p = (once ? rank_in_warp[j] + s.count[warp][digit] : place_in_warp(s.count[warp], digit, a.digit_bits, item, lane)) + s.base[digit];
                if (item) {
                    a.keys[to][p] = key[j];
                    a.places[to][p] = place[j];
                }
            }
        }
        cluster_meet();
    }
    if (threadIdx.x == 0 && s.unknown) record_error(a.header, a.device_status, DAF_ERR_INVALID_ARG);
    // the lists end with tokens that are none, up to a whole number of chunks
    const uint32_t last = (a.passes + 1u) & 1u;
    for (uint64_t i = a.n + rank * kSortThreads + threadIdx.x; i < (uint64_t)a.n_chunks * a.chunk; i += kSortCtas * kSortThreads) {
        a.keys[last][i] = a.vocabulary;
        a.places[last][i] = 0;
    }
}

// --------------------------------------------------------------------------------------------- backward: the sums
// Rows of a chunk on their way, VEC: two blocks of them lie in shared memory, every thread's part in places of its own, so that
// rows on their way take no registers; else in registers, a block at a time.
constexpr uint32_t kSumBytes = 256;             // of a thread, for both blocks
template <typename A, bool VEC> struct RowBlock {
    static constexpr int kRows = VEC ? (int)(kSumBytes / 2u / (8u * sizeof(A))) : 8, kAccesses = (int)sizeof(A) / 2;
    uint32_t place;                             // of the thread's first 16 bytes
    A x[VEC ? 1 : kRows][8];
    __device__ __forceinline__ void fetch(int half, int j, const A *row, uint32_t first, uint32_t lanes, uint32_t width)
    {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < kAccesses; i++)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place + ((half * kRows + j) * kAccesses + i) * kRowThreads * 16u),
                             "l"(reinterpret_cast<const char *>(row + first) + 16 * i) : "memory");
        } else {
            // all of them together, whatever is behind the row's end or belongs to no token: nothing may wait for one of the loads
#pragma unroll
            for (uint32_t e = 0; e < kLaneCols; e++) x[j][e] = row[first + lanes * e < width ? first + lanes * e : width - 1u];
        }
    }
    __device__ __forceinline__ void take(int half, int j, float (&y)[8]) const
    {
        if constexpr (VEC) {
            uint4 v[kAccesses];
#pragma unroll
            for (int i = 0; i < kAccesses; i++)
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                             : "r"(place + ((half * kRows + j) * kAccesses + i) * kRowThreads * 16u) : "memory");
            if constexpr (sizeof(A) == 2) {
                Elem<A>::widen8(v[0], y);
            } else {
                y[0] = __uint_as_float(v[0].x); y[1] = __uint_as_float(v[0].y); y[2] = __uint_as_float(v[0].z); y[3] = __uint_as_float(v[0].w);
                y[4] = __uint_as_float(v[1].x); y[5] = __uint_as_float(v[1].y); y[6] = __uint_as_float(v[1].z); y[7] = __uint_as_float(v[1].w);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) y[e] = get1(x[j][e]);
        }
    }
};

// The sorted list, read behind wait_for_ahead(): the kernel that writes it may still run when these start, so the loads are neither the
// read-only kind, which holds for memory that nobody writes while the kernel runs, nor ones that the compiler may move.
__device__ __forceinline__ uint32_t listed(const uint32_t *p)
{
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint4 listed4(const uint32_t *p)
{
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

// The first place in keys[0, n) whose key is at least `key`, by a warp, thirty-two probes at a time.
__device__ __forceinline__ uint64_t warp_lower_bound(const uint32_t *keys, uint64_t n, uint32_t key, uint32_t lane)
{
    uint64_t lo = 0, hi = n;                                        // in [lo, hi]
    while (lo < hi) {
        const uint64_t step = (hi - lo + 31u) / 32u, at = lo + lane * step;
        const uint32_t less = __ballot_sync(0xffffffffu, at < hi && listed(keys + at) < key);       // a run from lane 0 on
        if (!less) return lo;
        const uint32_t most = 31u - __clz(less);
        lo += most * step + 1u;
        hi = most == 31u || lo + step - 1u > hi ? hi : lo + step - 1u;
    }
    return lo;
}
// Zeros to those of the rows from r0 on that are absent, by a CTA.
template <typename W> __device__ __forceinline__ void zero_rows(const EmbeddingArgs &a, uint32_t r0, uint32_t rows, const uint32_t *absent)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const float none[8] = {};
    for (uint32_t t = warp; t < rows; t += kRowThreads / 32u) {
        if (!absent[t]) continue;
        W *const row = reinterpret_cast<W *>(a.grad_weight) + (uint64_t)(r0 + t) * a.width;
        const uint32_t off = (uint32_t)((32u - (reinterpret_cast<uintptr_t>(row) & 31u)) & 31u) / (uint32_t)sizeof(W);
        const uint32_t head = off < a.width ? off : a.width, per = 32u / (uint32_t)sizeof(W), units = (a.width - head) / per, tail = head + units * per;
        for (uint32_t u = lane; u < units; u += 32u) Elem<float>::store8(row + head + u * per, none);
        if (lane < head) row[lane] = put1<W>(0.0f);
        if (lane < a.width - tail) row[tail + lane] = put1<W>(0.0f);
    }
}

// Zeros to the rows of a clearing CTA that no token names.
template <typename W> __device__ void clear_rows(const EmbeddingArgs &a, uint32_t cta, uint64_t *range, uint32_t *absent)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const uint32_t *keys = a.keys[(a.passes + 1u) & 1u];
    const uint32_t r0 = a.early_rows + cta * a.fill_rows, rows = a.vocabulary - r0 < a.fill_rows ? a.vocabulary - r0 : a.fill_rows;
    if (warp < 2u) {
        const uint64_t at = warp_lower_bound(keys, a.n, r0 + warp * rows, lane);
        if (lane == 0) range[warp] = at;
    }
    __syncthreads();
    for (uint32_t t = threadIdx.x; t < rows; t += kRowThreads) {
        uint64_t lo = range[0], hi = range[1];
        while (lo < hi) {
            const uint64_t mid = (lo + hi) / 2u;
            if (listed(keys + mid) < r0 + t) lo = mid + 1u;
            else hi = mid;
        }
        absent[t] = lo == range[1] || listed(keys + lo) != r0 + t;
    }
    __syncthreads();
    zero_rows<W>(a, r0, rows, absent);
}

constexpr uint32_t kFillRows = 256;             // of a clearing CTA at most

template <typename A, typename W, bool VEC> __global__ void __launch_bounds__(kRowThreads, VEC ? 3 : 2) embedding_sum_kernel(const __grid_constant__ EmbeddingArgs a)
{
    extern __shared__ __align__(128) unsigned char raw[];
    using Block = RowBlock<A, VEC>;
    constexpr int kRows = Block::kRows;
    next_may_start();
    wait_for_ahead();
    // clearing CTAs lie evenly among the others
    const uint64_t both = (uint64_t)a.sum_ctas + a.fill_ctas;
    const uint32_t fills = (uint32_t)((uint64_t)blockIdx.x * a.fill_ctas / both);
    if ((uint32_t)((blockIdx.x + 1ull) * a.fill_ctas / both) > fills) {
        __shared__ uint64_t range[2];
        __shared__ uint32_t absent[kFillRows];
        clear_rows<W>(a, fills, range, absent);
        return;
    }
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1u);
    const uint64_t item = (uint64_t)(blockIdx.x - fills) * (kRowThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    if (item >= (uint64_t)a.n_chunks * a.slabs) return;
    const uint32_t chunk = (uint32_t)(item / a.slabs), slab = (uint32_t)(item - (uint64_t)chunk * a.slabs);
    const uint32_t col = slab * lanes * kLaneCols + lane_column<VEC>(lane, lanes, 0);
    const bool mine = col < a.width;
    const uint32_t last = (a.passes + 1u) & 1u, none = a.vocabulary;
    const uint64_t first = (uint64_t)chunk * a.chunk;
    const uint32_t *keys = a.keys[last] + first, *places = a.places[last] + first;
    const uint32_t ahead = chunk ? listed(keys - 1) : none, behind = chunk + 1u < a.n_chunks ? listed(keys + a.chunk) : none;
    const A *grad = reinterpret_cast<const A *>(a.grad_out);
    const uint64_t part_col = (uint64_t)slab * lanes * kLaneCols + lane * kLaneCols;    // parts are always held in runs of eight
    float acc[8] = {};
    uint32_t run = listed(keys);
    bool open = run == ahead;                                       // the run began in an earlier chunk
    const auto finish = [&](bool goes_on) {
        if (run == none || !mine) return;
        if (open || goes_on) {
            Elem<float>::store8(a.part + ((uint64_t)(open ? 0u : a.n_chunks) + chunk) * a.pitch + part_col, acc);
            return;
        }
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = acc[e] * a.scale;
        store_columns<W, VEC>(reinterpret_cast<W *>(a.grad_weight) + (uint64_t)run * a.width, col, lanes, a.width, y);
    };
    Block block;
    block.place = (uint32_t)__cvta_generic_to_shared(raw) + threadIdx.x * 16u;
    uint32_t key[kRows], next[kRows], behind_next[kRows], place[kRows];     // the list comes a block ahead of the rows
    const auto list = [](const uint32_t *from, uint32_t (&to)[kRows]) {
#pragma unroll
        for (int h = 0; h < kRows; h += 4) *reinterpret_cast<uint4 *>(to + h) = listed4(from + h);
    };
    const auto fetch = [&](int half) {                              // the rows of next
#pragma unroll
        for (int j = 0; j < kRows; j++)
            if (!VEC || (mine && next[j] != none)) block.fetch(half, j, grad + (uint64_t)place[j] * a.width, col, lanes, a.width);
    };
    const auto look = [&](uint32_t i) {
        if (i >= a.chunk) return;
        list(keys + i, behind_next);
        list(places + i, place);
    };
    look(0);
    if (VEC) {
#pragma unroll
        for (int j = 0; j < kRows; j++) next[j] = behind_next[j];
        fetch(0);
        asm volatile("cp.async.commit_group;" ::: "memory");
        look(kRows);
    }
    int half = 0;
    for (uint32_t i = 0; i < a.chunk; i += kRows) {
#pragma unroll
        for (int j = 0; j < kRows; j++) {
            key[j] = VEC ? next[j] : behind_next[j];
            next[j] = behind_next[j];
        }
        if (key[0] == none) break;
        if (VEC) {
            if (i + kRows < a.chunk) fetch(half ^ 1);
            asm volatile("cp.async.commit_group;" ::: "memory");
            look(i + 2u * kRows);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            fetch(0);
            look(i + kRows);
        }
#pragma unroll
        for (int j = 0; j < kRows; j++) {
            if (key[j] != run) {
                finish(false);
                run = key[j];
                open = false;
#pragma unroll
                for (int e = 0; e < 8; e++) acc[e] = 0.0f;
            }
            if (mine && run != none) {
                float y[8];
                block.take(half, j, y);
#pragma unroll
                for (int e = 0; e < 8; e++) acc[e] += y[e];
            }
        }
        half ^= 1;
    }
    if (VEC) asm volatile("cp.async.wait_group 0;" ::: "memory");
    const bool goes_on = run != none && run == behind;
    finish(goes_on);
    if (goes_on && !open && slab == 0 && lane == 0) {
        // most such runs end in the next chunk; the others' ends are looked for by those who join them (0)
        const bool on = chunk + 2u < a.n_chunks && listed(keys + 2u * a.chunk) == run;
        a.jobs[atomicAdd(a.n_jobs, 1u)] = make_uint4(chunk, on ? 0u : 2u, run, 0u);
    }
}

// --------------------------------------------------------------------------------------------- backward: runs across chunks
template <typename W, bool VEC> __global__ void __launch_bounds__(kRowThreads) embedding_join_kernel(const __grid_constant__ EmbeddingArgs a)
{
    constexpr uint32_t kWarps = kRowThreads / 32;
    __shared__ float s_sum[kWarps][256];
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, blocks = (a.pitch + 255u) / 256u;
    wait_for_ahead();
    const uint64_t work = (uint64_t)*a.n_jobs * blocks;
    for (uint64_t i = blockIdx.x; i < work; i += gridDim.x) {
        const uint32_t job = (uint32_t)(i / blocks), block = (uint32_t)(i - (uint64_t)job * blocks);
        const uint4 run = a.jobs[job];
        const uint32_t begin = run.x, key = run.z;                  // the first part comes from the second half of the workspace
        uint32_t parts = run.y;
        if (parts == 0u) {                                          // the last chunk that begins with the key is in [lo, hi): 32 probes at a time
            const uint32_t *keys = a.keys[(a.passes + 1u) & 1u];
            uint32_t lo = begin + 2u, hi = a.n_chunks;
            while (hi - lo > 1u) {
                const uint32_t step = (hi - lo + 31u) / 32u;
                const uint64_t at = (uint64_t)lo + (uint64_t)lane * step;
                const uint32_t yes = __ballot_sync(0xffffffffu, at < hi && listed(keys + at * a.chunk) == key);
                const uint32_t next = lo + (31u - __clz(yes)) * step;       // lane 0 always says yes
                hi = hi - next < step ? hi : next + step;
                lo = next;
            }
            parts = lo - begin + 1u;
        }
        const uint32_t from = (uint32_t)((uint64_t)parts * warp / kWarps), to = (uint32_t)((uint64_t)parts * (warp + 1u) / kWarps);
        const uint32_t col = block * 256u + lane * 8u;
        float acc[8] = {};
        if (col < a.pitch) {
#pragma unroll 8
            for (uint32_t p = from; p < to; p++) {
                float x[8];
                Elem<float>::load8(a.part + ((uint64_t)(p ? 0u : a.n_chunks) + begin + p) * a.pitch + col, x);
#pragma unroll
                for (int e = 0; e < 8; e++) acc[e] += x[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; e++) s_sum[warp][e * 32u + lane] = acc[e];
        __syncthreads();
        float sum = 0.0f;                                           // thread: element threadIdx.x / 32 of lane threadIdx.x % 32
#pragma unroll
        for (uint32_t w = 0; w < kWarps; w++) sum += s_sum[w][threadIdx.x];
        // where that is in the row: parts are held lane by lane, as the lanes of embedding_sum_kernel own them
        const uint32_t lanes = 1u << a.lanes_log2, at = block * 256u + lane * 8u, e = warp;
        const uint32_t slab = at / (lanes * 8u), owner = at / 8u % lanes;
        const uint32_t c = slab * lanes * 8u + lane_column<VEC>(owner, lanes, 0) + (VEC ? e : lanes * e);
        if (at < a.pitch && c < a.width) reinterpret_cast<W *>(a.grad_weight)[(uint64_t)key * a.width + c] = put1<W>(sum * a.scale);
        __syncthreads();
    }
}

// --------------------------------------------------------------------------------------------- backward: few tokens
// Few of them are looked through instead of sorted, in one launch: an item, a token's place and `across` slabs of the row, ends if
// the token came earlier; else its other places are found and their rows summed, in pieces of that list that a CTA's groups of
// lanes take; clearing CTAs find which of their rows are named.  That grows with tokens times items and with the longest run, so it is
// for up to kFewTokens of up to kFewItems, above half of them for vocabularies that are no smaller.  Against the sorted way: 47
// tokens of 60000 x 344 from binary32 15 and 21 us, of 4000 x 2048 7.3 and 16.8, 512 of those 13 and 18, 1024 of 11327 x 135 9.4 and
// 19.9, 2048 14.7 and 20.2, of 15 x 158 25.6 and 14.3; the worst, 256 times the same token of 1000 x 4048, 16.8 and 13.4.
// kFewCtas, four an SM, take items in turn: 1024 of 60000 x 344 16.6 us, with two an SM 16.7, with a CTA for each 17.5.
constexpr uint32_t kFewTokens = 2048, kFewItems = 2048, kFewCtas = 148u * 4u;

template <typename A, typename W, bool VEC> __global__ void __launch_bounds__(kRowThreads, 4) embedding_few_kernel(const __grid_constant__ EmbeddingArgs a)
{
    __shared__ uint32_t key[kFewTokens], list[kFewTokens], warp_count[kRowThreads / 32];
    __shared__ float s_sum[kLaneCols][kRowThreads];
    const uint32_t n = (uint32_t)a.n, tid = threadIdx.x;
    bool unknown = false;
    for (uint32_t t = tid; t < n; t += kRowThreads) {
        const long long token = token_at(a, t);
        const bool known = token >= 0 && token < (long long)a.vocabulary;
        key[t] = known && token != a.padding ? (uint32_t)token : a.vocabulary;
        unknown |= !known;
    }
    const bool bad = __syncthreads_or(unknown);
    if (blockIdx.x == 0 && tid == 0) {
        a.header->status = DAF_OK;
        if (bad) record_error(a.header, a.device_status, DAF_ERR_INVALID_ARG);
    }
    if (blockIdx.x >= a.sum_ctas) {
        uint32_t *const absent = list;
        const uint32_t r0 = (blockIdx.x - a.sum_ctas) * a.fill_rows, rows = a.vocabulary - r0 < a.fill_rows ? a.vocabulary - r0 : a.fill_rows;
        if (tid < rows) absent[tid] = 1u;
        __syncthreads();
        for (uint32_t t = tid; t < n; t += kRowThreads)
            if (key[t] - r0 < rows) absent[key[t] - r0] = 0u;
        __syncthreads();
        zero_rows<W>(a, r0, rows, absent);
        return;
    }
    const uint32_t blocks = (a.slabs + a.across - 1u) / a.across, items = n * blocks;
    const uint32_t lanes = 1u << a.lanes_log2, lane = tid & (lanes - 1u), group = tid >> a.lanes_log2, most = (kRowThreads >> a.lanes_log2) / a.across;
    const uint32_t piece = group % most;
    for (uint32_t item = blockIdx.x; item < items; item += a.sum_ctas) {
        const uint32_t first = item / blocks, mine = key[first];
        if (mine == a.vocabulary) continue;
        bool earlier = false;
        for (uint32_t t = tid; t < first; t += kRowThreads) earlier |= key[t] == mine;
        if (__syncthreads_or(earlier)) continue;                    // behind it nobody reads what the item before left
        uint32_t m = 0;                                             // places of the token so far
        for (uint32_t base = first; base < n; base += kRowThreads) {
            const bool hit = base + tid < n && key[base + tid] == mine;
            const uint32_t hits = __ballot_sync(0xffffffffu, hit);
            if ((tid & 31u) == 0) warp_count[tid >> 5] = __popc(hits);
            __syncthreads();
            uint32_t before = m;
#pragma unroll
            for (uint32_t w = 0; w < kRowThreads / 32u; w++) {
                before += w < tid >> 5 ? warp_count[w] : 0u;
                m += warp_count[w];
            }
            if (hit) list[before + __popc(hits & ((1u << (tid & 31u)) - 1u))] = base + tid;
            __syncthreads();
        }
        const uint32_t pieces = m < most ? m : most, slab = (item - first * blocks) * a.across + group / most;
        const uint32_t col = slab * lanes * kLaneCols + lane_column<VEC>(lane, lanes, 0);
        const bool here = slab < a.slabs && col < a.width && piece < pieces;
        float acc[8] = {};
        if (here) {
            constexpr uint32_t kRows = 4;                           // together
            const A *const grad = reinterpret_cast<const A *>(a.grad_out);
            const uint32_t to = m * (piece + 1u) / pieces;
            for (uint32_t i = m * piece / pieces; i < to; i += kRows) {
                float x[kRows][8];
#pragma unroll
                for (uint32_t j = 0; j < kRows; j++)
                    load_columns<A, VEC>(grad + (uint64_t)list[i + j < to ? i + j : i] * a.width, col, lanes, a.width, x[j]);
#pragma unroll
                for (uint32_t j = 0; j < kRows; j++) {
                    if (i + j >= to) break;
#pragma unroll
                    for (int e = 0; e < 8; e++) acc[e] += x[j][e];
                }
            }
        }
        if (pieces > 1u) {
#pragma unroll
            for (int e = 0; e < 8; e++) s_sum[e][tid] = acc[e];
            __syncthreads();
        }
        if (!here || piece) continue;
        for (uint32_t p = 1; p < pieces; p++)
#pragma unroll
            for (int e = 0; e < 8; e++) acc[e] += s_sum[e][tid + p * lanes];
#pragma unroll
        for (int e = 0; e < 8; e++) acc[e] *= a.scale;
        store_columns<W, VEC>(reinterpret_cast<W *>(a.grad_weight) + (uint64_t)mine * a.width, col, lanes, a.width, acc);
    }
}

// --------------------------------------------------------------------------------------------- host
static uint32_t elem_bytes(uint32_t dtype) { return dtype == DAF_F32 ? 4u : 2u; }

static daf_status check_embedding(const daf_embedding_params *p)
{
    if (!p || p->struct_size != sizeof(*p) || p->dtype > DAF_BF16 || p->table_dtype > DAF_BF16 || p->reserved != 0 ||
        (p->table_dtype != p->dtype && p->table_dtype != DAF_F32) || (p->token_bytes != 4u && p->token_bytes != 8u) ||
        !(p->scale - p->scale == 0.0f))
        return DAF_ERR_INVALID_ARG;
    if (p->vocabulary == 0 || p->width == 0) return DAF_ERR_SHAPE;
    if (p->vocabulary > 0x7FFFFFFEull || p->tokens > 0x7FFFFF00ull || p->width > (1u << 24)) return DAF_ERR_UNSUPPORTED;
    if (p->padding >= (int64_t)p->vocabulary) return DAF_ERR_INVALID_ARG;
    return DAF_OK;
}

// Lanes of a row: as many as its units of eight columns, a power of two, 32 at most.  The sums of rows that cannot be read in wide
// accesses take a warp to a row: 37202 tokens of 28 columns 20 us on four lanes a row (few warps, many small accesses each).
static void row_shape(EmbeddingArgs *a, bool backward)
{
    const uint32_t units = (a->width + kLaneCols - 1u) / kLaneCols;
    a->lanes_log2 = backward && a->width % kLaneCols ? 5u : 0u;
    while (a->lanes_log2 < 5u && (1u << a->lanes_log2) < units) a->lanes_log2++;
    const uint32_t cols = kLaneCols << a->lanes_log2;
    a->slabs = (a->width + cols - 1u) / cols;
    a->pitch = a->slabs * cols;
}

// Chunks of the sorted list: 128 tokens, or as few (16 at least) as leave every SM 32 warps, each with eight rows on their way.
static void chunk_shape(EmbeddingArgs *a)
{
    constexpr uint64_t kWarpsWanted = 148u * 32u;
    const uint64_t warps_of_row = (uint64_t)a->slabs << a->lanes_log2;      // in lanes
    a->chunk = 128u;
    while (a->chunk > 16u && (a->n + a->chunk - 1u) / a->chunk * warps_of_row < kWarpsWanted * 32u) a->chunk /= 2u;
    a->n_chunks = (uint32_t)((a->n + a->chunk - 1u) / a->chunk);
}

static uint64_t up256(uint64_t n) { return (n + 255u) & ~255ull; }

static EmbeddingArgs embedding_args(const daf_embedding_params *p, bool backward)
{
    EmbeddingArgs a = {};
    a.n = p->tokens;
    a.wide_tokens = p->token_bytes == 8u;
    a.vocabulary = (uint32_t)p->vocabulary;
    a.width = p->width;
    a.scale = p->scale;
    a.padding = p->padding;
    row_shape(&a, backward);
    chunk_shape(&a);
    uint32_t bits = 32u - (uint32_t)__builtin_clz(a.vocabulary);
    a.passes = (bits + kDigitBits - 1u) / kDigitBits;
    a.digit_bits = (bits + a.passes - 1u) / a.passes;
    return a;
}

static uint64_t grad_workspace(const EmbeddingArgs &a)
{
    const uint64_t list = up256((uint64_t)a.n_chunks * a.chunk * sizeof(uint32_t));
    return sizeof(WorkspaceHeader) + 4u * list + 256u + up256(a.n_chunks * sizeof(uint4)) + 2ull * a.n_chunks * a.pitch * sizeof(float);
}

// Wide accesses: rows of both sides start on the boundaries of eight elements.
static bool wide(const EmbeddingArgs &a, const void *x, uint32_t dx, const void *y, uint32_t dy)
{
    return a.width % kLaneCols == 0 && reinterpret_cast<uintptr_t>(x) % (8u * elem_bytes(dx)) == 0 && reinterpret_cast<uintptr_t>(y) % (8u * elem_bytes(dy)) == 0;
}
static bool on_elements(const void *p, uint32_t bytes) { return p && reinterpret_cast<uintptr_t>(p) % bytes == 0; }

template <typename W, typename A, bool VEC> static daf_status forward(const EmbeddingArgs &a, cudaStream_t s)
{
    const uint64_t items = a.n * ((a.slabs + kForwardSlabs - 1u) / kForwardSlabs), per_cta = kRowThreads >> a.lanes_log2;
    const uint64_t ctas = (items + per_cta - 1u) / per_cta;
    embedding_kernel<W, A, VEC><<<(uint32_t)(ctas < (1u << 30) ? ctas : 1u << 30), kRowThreads, 0, s>>>(a);
    return DAF_OK;
}
template <typename W, typename A, bool VEC> static daf_status backward(const EmbeddingArgs &a, cudaStream_t s)
{
    if (a.across) {
        embedding_few_kernel<A, W, VEC><<<a.sum_ctas + a.fill_ctas, kRowThreads, 0, s>>>(a);
        return DAF_OK;
    }
    const auto sum = &embedding_sum_kernel<A, W, VEC>;
    const uint32_t smem = VEC ? kSumBytes * kRowThreads : 0u;
    int ctas = 0;                                                   // also raises the kernel's limit of shared memory
    if (persistent_ctas(reinterpret_cast<const void *>(sum), (int)kRowThreads, (int)smem, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    if (launch_behind(sum, a.sum_ctas + a.fill_ctas, kRowThreads, smem, s, a) != cudaSuccess) return DAF_ERR_CUDA;
    const uint64_t most = (uint64_t)a.n_chunks * ((a.pitch + 255u) / 256u);
    const auto join = &embedding_join_kernel<W, VEC>;
    return launch_behind(join, (uint32_t)(most < 148u * 8u ? most : 148u * 8u), kRowThreads, 0, s, a) == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
template <bool BACK, bool VEC> static daf_status by_type(uint32_t table, uint32_t act, const EmbeddingArgs &a, cudaStream_t s)
{
#define DAF_EMBEDDING(W, A) (BACK ? backward<W, A, VEC>(a, s) : forward<W, A, VEC>(a, s))
    if (table == DAF_F16) return DAF_EMBEDDING(__half, __half);
    if (table == DAF_BF16) return DAF_EMBEDDING(__nv_bfloat16, __nv_bfloat16);
    if (act == DAF_F16) return DAF_EMBEDDING(float, __half);
    if (act == DAF_BF16) return DAF_EMBEDDING(float, __nv_bfloat16);
    return DAF_EMBEDDING(float, float);
#undef DAF_EMBEDDING
}

}  // namespace daf

using namespace daf;

// Tokens that are none are recorded in *status; null: in the device's word.
static daf_status embedding_rows(const daf_embedding_params *params, const void *d_tokens, const void *d_weight, void *d_out, unsigned int *status, cudaStream_t s)
{
    EmbeddingArgs a = embedding_args(params, false);
    a.tokens = d_tokens;
    a.weight = d_weight;
    a.out = d_out;
    if (!(a.device_status = status ? status : device_status_word())) return DAF_ERR_CUDA;
    const daf_status ran = wide(a, d_weight, params->table_dtype, d_out, params->dtype) ? by_type<false, true>(params->table_dtype, params->dtype, a, s)
                                                                                       : by_type<false, false>(params->table_dtype, params->dtype, a, s);
    return ran != DAF_OK ? ran : cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

static daf_status check_embedding_rows(const daf_embedding_params *params, const void *d_tokens, const void *d_weight, const void *d_out)
{
    const daf_status st = check_embedding(params);
    if (st != DAF_OK || params->tokens == 0) return st;
    return on_elements(d_tokens, params->token_bytes) && on_elements(d_weight, elem_bytes(params->table_dtype)) && on_elements(d_out, elem_bytes(params->dtype))
               ? DAF_OK : DAF_ERR_INVALID_ARG;
}

extern "C" daf_status daf_embedding(const daf_embedding_params *params, const void *d_tokens, const void *d_weight, void *d_out, daf_stream stream)
{
    const daf_status st = check_embedding_rows(params, d_tokens, d_weight, d_out);
    if (st != DAF_OK || params->tokens == 0) return st;
    return embedding_rows(params, d_tokens, d_weight, d_out, nullptr, reinterpret_cast<cudaStream_t>(stream));
}

extern "C" uint64_t daf_embedding_workspace(const daf_embedding_params *params)
{
    return check_embedding(params) == DAF_OK ? sizeof(WorkspaceHeader) : 0;
}

extern "C" daf_status daf_embedding_checked(const daf_embedding_params *params, const void *d_tokens, const void *d_weight, void *d_out, void *d_workspace,
                                            uint64_t workspace_bytes, daf_stream stream)
{
    const daf_status st = check_embedding_rows(params, d_tokens, d_weight, d_out);
    if (st != DAF_OK) return st;
    if (!on_elements(d_workspace, 32u)) return DAF_ERR_INVALID_ARG;
    if (workspace_bytes < daf_embedding_workspace(params)) return DAF_ERR_CAPACITY;
    unsigned int *const status = &reinterpret_cast<WorkspaceHeader *>(d_workspace)->status;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (cudaMemsetAsync(status, 0, sizeof(*status), s) != cudaSuccess) return DAF_ERR_CUDA;
    return params->tokens ? embedding_rows(params, d_tokens, d_weight, d_out, status, s) : DAF_OK;
}

extern "C" uint64_t daf_embedding_grad_workspace(const daf_embedding_params *params)
{
    return check_embedding(params) == DAF_OK ? grad_workspace(embedding_args(params, true)) : 0;
}

extern "C" daf_status daf_embedding_grad(const daf_embedding_params *params, const void *d_tokens, const void *d_grad_out, void *d_grad_weight,
                                         void *d_workspace, uint64_t workspace_bytes, daf_stream stream)
{
    const daf_status st = check_embedding(params);
    if (st != DAF_OK) return st;
    const daf_embedding_params &p = *params;
    if (!on_elements(d_grad_weight, elem_bytes(p.table_dtype)) || !on_elements(d_workspace, 32u) ||
        (p.tokens && (!on_elements(d_tokens, p.token_bytes) || !on_elements(d_grad_out, elem_bytes(p.dtype)))))
        return DAF_ERR_INVALID_ARG;
    EmbeddingArgs a = embedding_args(params, true);
    if (workspace_bytes < grad_workspace(a)) return DAF_ERR_CAPACITY;
    a.tokens = d_tokens;
    a.grad_out = d_grad_out;
    a.grad_weight = d_grad_weight;
    char *at = reinterpret_cast<char *>(d_workspace);
    a.header = reinterpret_cast<WorkspaceHeader *>(at);
    at += sizeof(WorkspaceHeader);
    const uint64_t list = up256((uint64_t)a.n_chunks * a.chunk * sizeof(uint32_t));
    for (int i = 0; i < 2; i++, at += 2u * list) {
        a.keys[i] = reinterpret_cast<uint32_t *>(at);
        a.places[i] = reinterpret_cast<uint32_t *>(at + list);
    }
    a.n_jobs = reinterpret_cast<uint32_t *>(at);
    a.jobs = reinterpret_cast<uint4 *>(at + 256);
    a.part = reinterpret_cast<float *>(at + 256 + up256(a.n_chunks * sizeof(uint4)));
    if (!(a.device_status = device_status_word())) return DAF_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const uint32_t eb = elem_bytes(p.table_dtype);
    const uint64_t row_bytes = (uint64_t)a.width * eb;
    const uint32_t across = a.slabs > 1u ? 2u : 1u;                 // so that a warp sums a quarter of a token's rows
    const uint64_t items = a.n * ((a.slabs + across - 1u) / across);
    if (items <= kFewItems && (a.n <= kFewTokens / 2u || (a.n <= kFewTokens && a.vocabulary >= a.n))) {
        a.across = across;
        a.sum_ctas = items < kFewCtas ? (uint32_t)items : kFewCtas;
        const uint64_t share = a.vocabulary * row_bytes / (148u * 8u), piece = share < 4096u ? 4096u : share < 65536u ? share : 65536u;
        a.fill_rows = row_bytes >= piece ? 1u : piece / row_bytes > kFillRows ? kFillRows : (uint32_t)(piece / row_bytes);
        a.fill_ctas = (a.vocabulary + a.fill_rows - 1u) / a.fill_rows;
    } else {
        int ctas = 0;                                               // also raises the kernel's limits
        if (persistent_ctas(reinterpret_cast<const void *>(&embedding_sort_kernel), (int)kSortThreads, (int)sizeof(SortShared), &ctas) != cudaSuccess ||
            cudaFuncSetAttribute(embedding_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
            return DAF_ERR_CUDA;
        // Rows to clear beside the sort: about as much as its own time writes (measured 8 us and 0.3 ns a token; 4 GB a ms), all without
        // tokens; the rest beside the sums, 64 KiB to a CTA.
        const uint64_t early = (32000000ull + 1200ull * a.n) / row_bytes;
        a.early_rows = early > a.vocabulary ? a.vocabulary : (uint32_t)early;
        a.fill_rows = row_bytes >= 65536u ? 1u : 65536u / row_bytes > kFillRows ? kFillRows : (uint32_t)(65536u / row_bytes);
        a.fill_ctas = (a.vocabulary - a.early_rows + a.fill_rows - 1u) / a.fill_rows;
        const uint64_t per_cta = kRowThreads >> a.lanes_log2;
        a.sum_ctas = (uint32_t)(((uint64_t)a.n_chunks * a.slabs + per_cta - 1u) / per_cta);
        const uint64_t bytes = a.early_rows * row_bytes, clusters = (bytes + (1u << 20) - 1u) >> 20;      // 64 KiB to a CTA
        embedding_sort_kernel<<<kSortCtas * (uint32_t)(1u + (clusters < 8u ? clusters : 8u)), kSortThreads, sizeof(SortShared), s>>>(a, eb);
    }
    const daf_status ran = wide(a, d_grad_out, p.dtype, d_grad_weight, p.table_dtype) ? by_type<true, true>(p.table_dtype, p.dtype, a, s)
                                                                                     : by_type<true, false>(p.table_dtype, p.dtype, a, s);
    if (ran != DAF_OK) return ran;
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}
