// Attention forward for 16-bit inputs on the tensor cores.
//
//   S = q k^T,  P = exp2(c S - m),  O = sum over key blocks of P v,  out = O / l,  lse = (m + log2 l) ln 2,
// with c = scale log2(e), l = sum of P and m a reference of the row that follows its running maximum.
//
// A persistent CTA (one per SM) takes items of 256 queries of one head and walks the keys in blocks of 128:
//   warps 0-3, 4-7   softmax of the item's first / second 128 queries; a thread owns one row
//   warp 8           issues the products; warp 9 issues the copies (10 and 11 only complete their warpgroup)
// The warpgroups share out the CTA's 384 x 168 registers: 232 for a softmax thread, which holds a row of 128 scores, 40
// for the others.
// Tensor memory holds S and O of both halves (S: 2 x 128 columns, O: 2 x DP); P overwrites its S as 16-bit operands of
// P v, so scores and probabilities never leave the SM.  The halves alternate: while one is in softmax, the tensor cores
// work for the other.  Products of one thread execute in the order they are issued, which is what makes
// S(j + 1) over P(j) safe.
//
// m moves only when a block's maximum passes it by more than 8 (P <= 2^8 then, exact enough in every type): only then is
// O read, scaled and written back, by the warp whose rows need it.  P is rounded to the input type, which the second
// product needs; its sum l is taken before that rounding, so the rounding errors average out instead of adding up.
#pragma once
#include "attention.cuh"
#include "tensor_core.cuh"

namespace daf {

constexpr int kFwdThreads = 384;
constexpr int kFwdRows = 256, kBlock = 128;
constexpr float kLag = 8.0f;
constexpr float kNoMax = -1e30f;                 // reference of a row that has seen no key yet

struct AttnForwardArgs {
    CUtensorMap q, k, v, out;
    AttnArgs a;
    FastDiv heads, all_heads, tiles;             // H, B H, q_tiles
    uint32_t items, q_tiles;
    WorkspaceHeader *header;
};

template <int DP> struct FwdSmem {
    static constexpr int kStages = DP == 128 ? 4 : 8;
    static constexpr uint32_t kTile = 128u * DP * 2u;            // one tile of 128 rows
    static constexpr uint32_t kOut = 4096u;                       // two pieces of 32 x 32 outputs for each softmax warp
    static constexpr uint32_t kBytes = (2u + kStages) * kTile + 8u * kOut + 1024u;
};

// The item's head, batch entry and first query, and its number of key blocks per half.
struct FwdItem {
    uint32_t b, h, m0, n;
    int blocks[2], both;
    __device__ __forceinline__ FwdItem(const AttnForwardArgs &p, uint32_t item)
    {
        const AttnArgs &a = p.a;
        uint32_t bh, qt;
        if (a.causal) {                                            // longest rows first
            qt = p.all_heads.div(item);
            bh = item - qt * p.all_heads.d;
            qt = p.q_tiles - 1u - qt;
        } else {                                                   // neighbours share keys and values
            bh = p.tiles.div(item);
            qt = item - bh * p.q_tiles;
        }
        b = p.heads.div(bh);
        h = bh - b * a.H;
        m0 = qt * kFwdRows;
        n = attn_length(a, b);
        for (int w = 0; w < 2; w++) {
            const uint32_t first = m0 + 128u * w;
            blocks[w] = 0;
            if (first < a.Sq) {
                const int end = attn_limit(a, n, (int)(first + 128u < a.Sq ? first + 128u : a.Sq) - 1);
                blocks[w] = end > 0 ? (end + kBlock - 1) / kBlock : 0;
            }
        }
        both = blocks[0] > blocks[1] ? blocks[0] : blocks[1];
    }
};

// Zeroes rows [from, to) of a tile in shared memory (128-byte rows of each 64-element box, `box` bytes apart).
template <int DP> __device__ __forceinline__ void zero_rows(unsigned char *tile, uint32_t box, uint32_t from, uint32_t to, uint32_t lane)
{
    for (uint32_t i = lane; i < (to - from) * 8u * (DP / 64); i += 32u) {
        const uint32_t piece = i % 8u, r = from + i / 8u % (to - from), x = i / 8u / (to - from);
        *reinterpret_cast<uint4 *>(tile + x * box + r * 128u + piece * 16u) = make_uint4(0u, 0u, 0u, 0u);
    }
}

template <typename T, int DP>
__global__ void __launch_bounds__(kFwdThreads, 1) attention_kernel(const __grid_constant__ AttnForwardArgs p)
{
    using Smem = FwdSmem<DP>;
    constexpr bool BF16 = __is_same(T, __nv_bfloat16);
    constexpr int STAGES = Smem::kStages;
    extern __shared__ unsigned char s_raw[];
    __shared__ __align__(8) uint64_t q_full, q_empty, tail, drain, kv_full[STAGES], kv_empty[STAGES], s_full[2], p_ready[2], o_done[2];
    __shared__ uint32_t s_tmem, s_abort;
    unsigned char *const smem = s_raw + ((1024u - (smem_u32(s_raw) & 1023u)) & 1023u);
    const AttnArgs &a = p.a;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
    if (threadIdx.x == 0) {
        s_abort = 0u;
        bar_init(&q_full, 1);
        bar_init(&q_empty, 1);
        bar_init(&tail, 1);
        bar_init(&drain, 1);
        for (int i = 0; i < STAGES; i++) {
            bar_init(&kv_full[i], 1);
            bar_init(&kv_empty[i], 1);
        }
        for (int w = 0; w < 2; w++) {
            bar_init(&s_full[w], 1);
            bar_init(&p_ready[w], 4);
            bar_init(&o_done[w], 1);
        }
        fence_async();
        if (blockIdx.x == 0) p.header->status = 0u;
    }
    if (warp == 0) tmem_alloc(&s_tmem, 512);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = s_tmem;
    volatile uint32_t *const stop = &s_abort;

    if (warp < 8) {                                                // ---- softmax
        take_registers<232>();
        const uint32_t w = warp >> 2, quarter = (warp & 3u) << 21;  // lane 32 (warp % 4) in the address's upper half
        const uint32_t ts = tmem + w * 128u + quarter, to = tmem + 256u + w * DP + quarter;
        unsigned char *const s_out = smem + (2 + STAGES) * Smem::kTile + warp * Smem::kOut;
        uint32_t pieces = 0, s_ph = 0, pv = 0;                                  // pv: products into O that were handed over, ever
        const float c = a.scale_log2;
        for (uint32_t item = blockIdx.x; item < p.items; item += gridDim.x) {
            const FwdItem it(p, item);
            const uint32_t first = it.m0 + 128u * w, row = first + (warp & 3u) * 32u + lane;
            if (first >= a.Sq) continue;
            const int limit = row < a.Sq ? attn_limit(a, it.n, (int)row) : (int)it.n;
            const bool idle = first + (warp & 3u) * 32u >= a.Sq;   // none of the warp's rows exist
            float m = kNoMax, l = 0.0f;
            bool ok = true;
            for (int j = 0; j < it.blocks[w]; j++) {
                if (!(ok = bar_wait(&s_full[w], s_ph, stop))) break;
                s_ph ^= 1u;
                if (!idle) {
                    tmem_after_sync();
                    const int valid = (int)it.n - j * kBlock;       // columns that hold scores, at least
                    float x[128];
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        if (32 * i < valid) tmem_load32(ts + 32 * i, x + 32 * i);
                    tmem_wait_loads();
                    if (a.scale < 0.0f) {                           // c is its absolute value
#pragma unroll
                        for (int i = 0; i < 128; i++) x[i] = -x[i];
                    }
                    const int left = limit - j * kBlock;
                    if (__any_sync(0xffffffffu, left < kBlock)) {
#pragma unroll
                        for (int i = 0; i < 128; i++)
                            if (i >= left) x[i] = -INFINITY;
                    }
                    float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
                    for (int i = 4; i < 128; i += 8)
#pragma unroll
                        for (int k = 0; k < 4; k++)
                            top[k] = i + 4 + k < 128 ? fmax3(top[k], x[i + k], x[i + 4 + k]) : fmaxf(top[k], x[i + k]);
                    const float block_max = c * fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                    if (j == 0) {
                        m = fmaxf(block_max, kNoMax);
                    } else if (__any_sync(0xffffffffu, block_max > m + kLag)) {
                        const float next = fmaxf(m, block_max), fade = exp2_fast(m - next);
                        m = next;
                        l *= fade;
                        if (!(ok = bar_wait(&o_done[w], (pv - 1u) & 1u, stop))) break;
                        tmem_after_sync();
#pragma unroll
                        for (int i = 0; i < DP / 16; i++) {
                            float o[16];
                            tmem_load16(to + 16 * i, o);
                            tmem_wait_loads();
#pragma unroll
                            for (int k = 0; k < 16; k++) o[k] *= fade;
                            tmem_store16(to + 16 * i, reinterpret_cast<const uint32_t *>(o));
                        }
                    }
                    const uint64_t c2 = pair(c, c), m2 = pair(-m, -m);
                    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        if (32 * i < valid) {
                            uint32_t r[16];
#pragma unroll
                            for (int k = 0; k < 16; k++) {
                                float u, v;
                                unpair(fma2(pair(x[32 * i + 2 * k], x[32 * i + 2 * k + 1]), c2, m2), u, v);
                                u = exp2_fast(u);
                                v = exp2_fast(v);
                                sum[k & 1] = add2(sum[k & 1], pair(u, v));
                                r[k] = round2<T>(u, v);
                            }
                            tmem_store16(ts + 16 * i, r);
                        }
                    }
                    float u, v;
                    unpair(add2(sum[0], sum[1]), u, v);
                    l += u + v;
                    tmem_wait_stores();
                    tmem_before_sync();
                }
                __syncwarp();
                if (lane == 0) bar_arrive(&p_ready[w]);
                pv++;
            }
            if (!ok) break;
            float by = 0.0f;
            if (it.blocks[w] > 0) {
                if (!bar_wait(&o_done[w], (pv - 1u) & 1u, stop)) break;
                tmem_after_sync();
                by = l > 0.0f ? __fdiv_rn(1.0f, l) : 0.0f;
            }
            if (idle) continue;
            if (row < a.Sq) a.lse[((uint64_t)it.b * a.H + it.h) * a.Sq + row] = l > 0.0f ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
#pragma unroll
            for (int i = 0; i < DP / 32; i++) {
                if (32u * i >= a.D) continue;
                float o[32];
                if (it.blocks[w] > 0) {
                    tmem_load32(to + 32 * i, o);
                    tmem_wait_loads();
                }
                unsigned char *const piece = s_out + (pieces++ & 1u) * 2048;
                if (lane == 0) stores_read<1>();                   // the store before last is out of this half
                __syncwarp();
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (l > 0.0f) {
                        v.x = round2<T>(o[8 * k] * by, o[8 * k + 1] * by);
                        v.y = round2<T>(o[8 * k + 2] * by, o[8 * k + 3] * by);
                        v.z = round2<T>(o[8 * k + 4] * by, o[8 * k + 5] * by);
                        v.w = round2<T>(o[8 * k + 6] * by, o[8 * k + 7] * by);
                    }
                    stage_piece(piece, lane, k, v);
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tma_store(&p.out, piece, 32 * i, it.h, first + (warp & 3u) * 32u, it.b);
            }
            tmem_before_sync();
        }
        if (lane == 0) stores_done();
    } else {
        leave_registers<40>();
        if (warp == 9) {                                               // ---- copies
            uint32_t st = 0, ph = 1, q_ph = 1, tail_ph = 0;            // a fresh barrier's "previous" phase counts as complete
            for (uint32_t item = blockIdx.x; item < p.items; item += gridDim.x) {
                const FwdItem it(p, item);
                if (it.both == 0) continue;
                if (!bar_wait(&q_empty, q_ph, stop)) break;
                q_ph ^= 1u;
                if (lane == 0) {
                    bar_expect(&q_full, ((it.blocks[0] > 0) + (it.blocks[1] > 0)) * Smem::kTile);
                    for (int w = 0; w < 2; w++)
                        if (it.blocks[w] > 0)
                            for (int x = 0; x < DP / 64; x++)
                                tma_load(smem_u32(smem) + w * Smem::kTile + x * 16384, &p.q, &q_full, 64 * x, it.h, it.m0 + 128 * w, it.b);
                }
                for (int i = 0; i < 2 * it.both; i++) {                // K0 V0 K1 V1 ...
                    const int j = i >> 1;
                    const bool is_v = i & 1;
                    if (!bar_wait(&kv_empty[st], ph, stop)) break;
                    unsigned char *const dst = smem + (2 + st) * Smem::kTile;
                    // P is zero in a masked column, but 0 * NaN is not: rows of v behind the sequence's end that the
                    // last product's steps of 16 keys still touch are cleared
                    const uint32_t valid = it.n - (uint32_t)j * kBlock, end = (valid + 15u) & ~15u;
                    const bool clear = is_v && it.n < a.Sk && valid < (uint32_t)kBlock && valid != end;
                    uint64_t *const bar = clear ? &tail : &kv_full[st];
                    if (lane == 0) {
                        bar_expect(bar, Smem::kTile);
                        for (int x = 0; x < DP / 64; x++)
                            tma_load(smem_u32(dst) + x * 16384, is_v ? &p.v : &p.k, bar, 64 * x, it.h / a.group, j * kBlock, it.b);
                    }
                    if (clear) {
                        if (!bar_wait(&tail, tail_ph, stop)) break;
                        tail_ph ^= 1u;
                        zero_rows<DP>(dst, 16384u, valid, end, lane);
                        fence_async();
                        __syncwarp();
                        if (lane == 0) bar_arrive(&kv_full[st]);
                    }
                    if (++st == STAGES) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
                if (*stop) break;
            }
            if (*stop) {                                               // giving up: let the copies in flight land first
                const uint64_t until = now_ns() + 1000000000ull;
                while (now_ns() < until) __nanosleep(1000);
            }
        } else if (warp == 8) {                                        // ---- products
            const uint32_t one = elect_lane();
            uint32_t st = 0, ph = 0, q_ph = 0, p_ph[2] = {0, 0};
            const uint32_t q_smem = smem_u32(smem), kv_smem = q_smem + 2u * Smem::kTile;
            const uint32_t steps = (a.D + 15u) / 16u;              // of the first product
            const uint32_t pv_desc = product_desc(BF16, steps * 16u, true);
            for (uint32_t item = blockIdx.x; item < p.items; item += gridDim.x) {
                const FwdItem it(p, item);
                if (it.both == 0) continue;
                if (!bar_wait(&q_full, q_ph, stop)) break;
                q_ph ^= 1u;
                // S of half w for the key block in stage `at`
                auto scores = [&](int w, int j, uint32_t at) {
                    const uint32_t valid = it.n - (uint32_t)j * kBlock, cols = valid < (uint32_t)kBlock ? (valid + 15u) & ~15u : kBlock;
                    const uint32_t desc = product_desc(BF16, cols, false);
                    const uint32_t q = operand_low(q_smem + w * Smem::kTile, 16), k = operand_low(kv_smem + at * Smem::kTile, 16);
                    product_ss(one, tmem + w * 128u, q, k, desc, false);
#pragma unroll
                    for (uint32_t s = 1; s < DP / 16; s++) {
                        const uint32_t by = (s & 3u) * 2u + (s >> 2) * 1024u;         // 32 bytes along the row, 16 KiB per 64 elements
                        if (s < steps) product_ss<true>(one, tmem + w * 128u, q + by, k + by, desc);
                    }
                    products_done(one, &s_full[w]);
                };
                auto next = [&]() {
                    if (++st == STAGES) {
                        st = 0;
                        ph ^= 1u;
                    }
                };
                if (!bar_wait(&kv_full[st], ph, stop)) break;
                tmem_after_sync();
#pragma unroll
                for (int w = 0; w < 2; w++)
                    if (it.blocks[w] > 0) scores(w, 0, st);
                products_done(one, &kv_empty[st]);
                if (it.both == 1) products_done(one, &q_empty);
                next();
                for (int j = 0; j < it.both; j++) {
                    const uint32_t v_st = st;
                    if (!bar_wait(&kv_full[st], ph, stop)) break;
                    next();
                    const bool more = j + 1 < it.both;
                    if (more && !bar_wait(&kv_full[st], ph, stop)) break;
                    const uint32_t valid = it.n - (uint32_t)j * kBlock;
                    const uint32_t pv_steps = valid < (uint32_t)kBlock ? (valid + 15u) / 16u : kBlock / 16;
#pragma unroll
                    for (int w = 0; w < 2; w++) {
                        if (j >= it.blocks[w]) continue;
                        if (!bar_wait(&p_ready[w], p_ph[w], stop)) break;
                        p_ph[w] ^= 1u;
                        tmem_after_sync();
                        const uint32_t v = operand_low(kv_smem + v_st * Smem::kTile, 16384);
                        product_ts(one, tmem + 256u + w * DP, tmem + w * 128u, v, pv_desc, j > 0);
#pragma unroll
                        for (uint32_t s = 1; s < kBlock / 16; s++)                   // 16 keys: 2 KiB of v, 8 columns of P
                            if (s < pv_steps) product_ts<true>(one, tmem + 256u + w * DP, tmem + w * 128u + s * 8u, v + s * 128u, pv_desc);
                        products_done(one, &o_done[w]);
                        if (j + 1 < it.blocks[w]) scores(w, j + 1, st);
                    }
                    products_done(one, &kv_empty[v_st]);
                    if (more) {
                        products_done(one, &kv_empty[st]);
                        if (j + 2 == it.both) products_done(one, &q_empty);
                        next();
                    }
                }
                if (*stop) break;
            }
            products_done(one, &drain);
            bar_wait(&drain, 0, stop);
        }
    }
    tmem_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) p.header->status = DAF_ERR_TIMEOUT;
    if (warp == 0) tmem_free(tmem, 512);
}

template <typename T, int DP> static daf_status launch_forward(AttnForwardArgs &p, cudaStream_t s)
{
    int ctas = 0;
    const auto kernel = &attention_kernel<T, DP>;
    if (persistent_ctas(reinterpret_cast<const void *>(kernel), kFwdThreads, (int)FwdSmem<DP>::kBytes, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    kernel<<<p.items < (uint32_t)ctas ? p.items : (uint32_t)ctas, kFwdThreads, FwdSmem<DP>::kBytes, s>>>(p);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

template <typename T> daf_status attn_forward_tc(const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s)
{
    AttnForwardArgs p;
    p.a = a;
    p.a.scale_log2 = fmaxf(fabsf(a.scale_log2), 0x1p-100f);       // the sign is applied to S; never 0, which masks would turn into NaN
    p.q_tiles = (a.Sq + kFwdRows - 1u) / kFwdRows;
    p.items = p.q_tiles * a.B * a.H;
    p.header = header;
    const bool bf16 = __is_same(T, __nv_bfloat16);
    p.heads.set(a.H);
    p.all_heads.set(a.B * a.H);
    p.tiles.set(p.q_tiles);
    if (!attn_tensor_map(&p.q, bf16, a.q, a.B, a.Sq, a.H, a.D, 128) || !attn_store_map(&p.out, bf16, a.out, a.B, a.Sq, a.H, a.D)) return DAF_ERR_CUDA;
    if (a.Sk == 0) p.k = p.v = p.q;                                // never read
    else if (!attn_tensor_map(&p.k, bf16, a.k, a.B, a.Sk, a.Hkv, a.D, 128) || !attn_tensor_map(&p.v, bf16, a.v, a.B, a.Sk, a.Hkv, a.D, 128))
        return DAF_ERR_CUDA;
    return a.D <= 64u ? launch_forward<T, 64>(p, s) : launch_forward<T, 128>(p, s);
}

}  // namespace daf
