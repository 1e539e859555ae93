// Attention forward for 16-bit inputs on the tensor cores.
//
//   S = q k^T,  P = exp2(c S - m),  O = sum over key blocks of P v,  out = O / l,  lse = (m + log2 l) ln 2,
// with c = scale log2(e), l = sum of P and m a reference of the row that follows its running maximum.
//
// A persistent CTA (one per SM) takes items of 256 queries of one head and walks the keys in blocks of 128:
//   warps 0-7, 8-15  softmax of the item's first / second 128 queries; a thread owns 64 of the 128 columns of a row, and the
//                    two warps of a row exchange its maximum.  (A row to a thread, half the warps with twice the
//                    registers: 38.9 against 34.9 us for 64 x 197 tokens, 12 heads of 64.)
//   warp 16          issues the products; warp 17 issues the copies (18 and 19 only complete their warpgroup)
// The warpgroups share out the CTA's 640 x 96 registers: 104 for a softmax thread, 64 for the others.
// Tensor memory holds S and O of both halves (S: 2 x 128 columns, O: 2 x DP); P overwrites its S as 16-bit operands of
// P v, so scores and probabilities never leave the SM.  The halves alternate: while one is in softmax, the tensor cores
// work for the other.  Products of one thread execute in the order they are issued, which is what makes
// S(j + 1) over P(j) safe.
//
// m moves only when a block's maximum passes it by more than 8 (P <= 2^8 then, exact enough in every type): only then is
// O read, scaled and written back, by the warp whose rows need it.  P is rounded to the input type, which the second
// product needs; its sum l is taken before that rounding, so the rounding errors average out instead of adding up.
// c S - m is one fused operation against an m that is itself rounded: 2^-24 |m| off, the same for a whole row, which cancels
// in P v / l while P fits its type.  Beyond |c S| = 2^28 it need not, and the row becomes NaN.  (Scores taken relative to the
// unrounded maximum ahead of the product with c: in any of four forms 4 to 5 % of every call, 402 -> 420 us and more for
// 4 x 4096 x 16 heads of 64.)
#pragma once
#include "attention.cuh"
#include "tensor_core.cuh"

namespace daf {

constexpr int kFwdThreads = 640;
constexpr int kFwdRows = 256, kBlock = 128;
constexpr float kLag = 8.0f;
constexpr int kTurnPolls = 64;                   // about 2000 cycles
constexpr float kNoMax = -3.402823466e38f;       // reference of a row that has seen no key yet: no finite score is lower

struct AttnForwardArgs {
    CUtensorMap q, k, v, out;
    AttnArgs a;
    FastDiv heads, all_heads, tiles;             // H, B H, q_tiles
    FastDiv split_div;                           // splits
    uint32_t items, q_tiles, splits;             // splits: runs of key blocks of a row tile, each an item
    float *part_out, *part_lse2;                 // with splits: [split, B, H, Sq, D] and [split, B, H, Sq], see attn_splits
    WorkspaceHeader *header;
};

template <int DP> struct FwdSmem {
    static constexpr int kStages = DP == 128 ? 4 : 6, kQueries = DP == 128 ? 1 : 2;   // key / value tiles, items' queries
    static constexpr uint32_t kTile = 128u * DP * 2u;            // one tile of 128 rows
    static constexpr uint32_t kOut = 2048u;                       // a piece of 32 x 32 outputs for each softmax warp
    static constexpr uint32_t kBars = 1024u;                      // barriers and such, ahead of everything
    static constexpr uint32_t kKeys = 2u * kQueries * kTile;          // where they begin
    static constexpr uint32_t kBytes = kBars + kKeys + kStages * kTile + 16u * kOut + 16u * 32u * 4u;
};

// The item's head, batch entry and first query, and its number of key blocks per half.
struct FwdItem {
    uint32_t b, h, m0, n, split;
    int blocks[2], both, j0;                     // j0: the first key block
    __device__ __forceinline__ void set(const AttnForwardArgs &p, uint32_t item)
    {
        const AttnArgs &a = p.a;
        split = 0;
        if (p.splits > 1u) {
            const uint32_t whole = p.split_div.div(item);
            split = item - whole * p.splits;
            item = whole;
        }
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
        j0 = 0;
        if (p.splits > 1u) {                                       // the split's share of the blocks
            const int share = (both + (int)p.splits - 1) / (int)p.splits;
            j0 = (int)split * share;
            for (int w = 0; w < 2; w++) {
                const int left = blocks[w] - j0;
                blocks[w] = left < 0 ? 0 : left < share ? left : share;
            }
            both = blocks[0] > blocks[1] ? blocks[0] : blocks[1];
        }
    }
};

// The first item from `item` on (in this CTA's steps) that has key blocks.
__device__ __forceinline__ bool next_item(const AttnForwardArgs &p, uint32_t &item, FwdItem &it)
{
    for (; item < p.items; item += gridDim.x) {
        it.set(p, item);
        if (it.both) return true;
    }
    return false;
}

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
    // tiles need 1024-byte boundaries; with nothing declared statically the dynamic part starts on one
    extern __shared__ __align__(1024) unsigned char s_raw[];
    struct Bars {
        uint64_t kv_full[8], kv_empty[8], s_full[2], p_ready[2], o_done[2], q_full[2], q_empty[2], tail, drain;
        uint32_t tmem, abort, busy[16], left[16];
    };
    static_assert(sizeof(Bars) <= Smem::kBars && STAGES <= 8, "barriers fit their places");
    Bars &bars = *reinterpret_cast<Bars *>(s_raw);
    uint64_t *const kv_full = bars.kv_full, *const kv_empty = bars.kv_empty, *const s_full = bars.s_full, *const p_ready = bars.p_ready,
             *const o_done = bars.o_done, *const q_full = bars.q_full, *const q_empty = bars.q_empty;
    uint64_t &tail = bars.tail, &drain = bars.drain;
    uint32_t &s_tmem = bars.tmem, &s_abort = bars.abort;
    if (smem_u32(s_raw) & 1023u) {                                 // the same for every thread
        if (threadIdx.x == 0) record_error(p.header, p.a.device_status, DAF_ERR_UNSUPPORTED);
        return;
    }
    unsigned char *const smem = s_raw + Smem::kBars;
    // [warp][lane]: what the two warps of a row tell each other
    float (*const s_told)[32] = reinterpret_cast<float (*)[32]>(smem + Smem::kKeys + STAGES * Smem::kTile + 16u * Smem::kOut);
    const AttnArgs &a = p.a;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
    if (threadIdx.x < 16) bars.busy[threadIdx.x] = bars.left[threadIdx.x] = 0u;
    if (threadIdx.x == 0) {
        s_abort = 0u;
        bar_init(&tail, 1);
        bar_init(&drain, 1);
        for (int i = 0; i < STAGES; i++) {
            bar_init(&kv_full[i], 1);
            bar_init(&kv_empty[i], 1);
        }
        for (int w = 0; w < 2; w++) {
            bar_init(&q_full[w], 1);
            bar_init(&q_empty[w], 1);
            bar_init(&s_full[w], 1);
            bar_init(&p_ready[w], 8);
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

    if (warp < 16) {                                               // ---- softmax
        take_registers<104>();
        const uint32_t w = warp >> 3, part = warp >> 2 & 1u, quarter = (warp & 3u) << 21;   // lane 32 (warp % 4) in the address's upper half
        const uint32_t ts = tmem + w * 128u + part * 64u + quarter, to = tmem + 256u + w * DP + part * (DP / 2) + quarter;
        volatile uint32_t *const busy = bars.busy;
        WarpPair pair_of;                                           // the two warps that share 32 rows
        pair_of.init(bars.left, 1u + w * 4u + (warp & 3u), warp ^ 4u);
        unsigned char *const s_out = smem + Smem::kKeys + STAGES * Smem::kTile + warp * Smem::kOut;
        uint32_t s_ph = 0, pv = 0;                                  // pv: products into O that were handed over, ever
        const float c = a.scale_log2;
        uint32_t item = blockIdx.x;
        for (; item < p.items; item += gridDim.x) {
            FwdItem it;
            it.set(p, item);
            const uint32_t first = it.m0 + 128u * w, row = first + (warp & 3u) * 32u + lane;
            if (first >= a.Sq) continue;
            const int blocks = w ? it.blocks[1] : it.blocks[0];
            const int limit = row < a.Sq ? attn_limit(a, it.n, (int)row) : (int)it.n;
            const bool idle = first + (warp & 3u) * 32u >= a.Sq;   // none of the warp's rows exist
            float m = kNoMax, l = 0.0f;
            bool ok = true;
            for (int j = 0; j < blocks; j++) {
                if (!(ok = bar_wait(&s_full[w], s_ph, stop))) break;
                s_ph ^= 1u;
                if (!idle) {
                    tmem_after_sync();
                    const int valid = (int)it.n - (it.j0 + j) * kBlock - 64 * (int)part;   // columns that hold scores, at least
                    const int left = limit - (it.j0 + j) * kBlock - 64 * (int)part;
                    const bool masked = __any_sync(0xffffffffu, left < 64);
                    // 32 scores at a time, once for the maximum and once more for the exponentials: reading tensor memory
                    // twice costs less than 64 registers
                    const auto scores = [&](int i, float (&x)[32]) {
                        tmem_load32(ts + 32 * i, x);
                        tmem_wait_loads();
                        if (a.scale < 0.0f) {                       // c is its absolute value
#pragma unroll
                            for (int k = 0; k < 32; k++) x[k] = -x[k];
                        }
                        if (masked) {
#pragma unroll
                            for (int k = 0; k < 32; k++)
                                if (32 * i + k >= left) x[k] = -INFINITY;
                        }
                    };
                    float row_max = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        if (32 * i >= valid) continue;
                        float x[32];
                        scores(i, x);
                        float top[4] = {row_max, x[1], x[2], x[3]};
                        top[0] = fmaxf(top[0], x[0]);
#pragma unroll
                        for (int k = 4; k < 28; k += 8)
#pragma unroll
                            for (int e = 0; e < 4; e++) top[e] = fmax3(top[e], x[k + e], x[k + 4 + e]);
#pragma unroll
                        for (int e = 0; e < 4; e++) top[e] = fmaxf(top[e], x[28 + e]);
                        row_max = fmaxf(fmax3(top[0], top[1], top[2]), top[3]);
                    }
                    s_told[warp][lane] = row_max;
                    pair_of.meet_unseen();
                    const float others = s_told[warp ^ 4u][lane], block_max = c * fmaxf(row_max, others);   // a maximum is never NaN
                    if (j == 0) {
                        if (!(ok = !pair_of.gone(others))) break;
                        m = fmaxf(block_max, kNoMax);
                    } else if (__any_sync(0xffffffffu, block_max > m + kLag || others != others)) {   // the same in both warps
                        if (!(ok = !pair_of.gone(others))) break;
                        const float next = fmaxf(m, block_max);
                        const float fade = exp2_fast(m - next);
                        m = next;
                        l *= fade;
                        if (!(ok = bar_wait(&o_done[w], (pv - 1u) & 1u, stop))) break;
                        tmem_after_sync();
#pragma unroll
                        for (int i = 0; i < DP / 32; i++) {
                            float o[16];
                            tmem_load16(to + 16 * i, o);
                            tmem_wait_loads();
#pragma unroll
                            for (int k = 0; k < 16; k++) o[k] *= fade;
                            tmem_store16(to + 16 * i, reinterpret_cast<const uint32_t *>(o));
                        }
                    }
                    // The halves' exponentials take turns: side by side they would both end late and leave the tensor cores
                    // idle meanwhile.  Only an order that pays, so the wait for the other half's two warps on this
                    // scheduler is short and nothing depends on it.  Heads of up to 64 alone (4 x 4096 x 16 heads of 64:
                    // 441 -> 399 us): the products of wider ones take as long as the exponentials (8192 x 16 heads of
                    // 128: 514 us without, 524 with turns).
                    for (int i = 0; DP == 64 && i < kTurnPolls && (busy[warp ^ 8u] | busy[warp ^ 12u]); i++) {}
                    if (DP == 64 && lane == 0) busy[warp] = 1u;
                    const uint64_t c2 = pair(c, c), m2 = pair(-m, -m);
                    uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                        if (32 * i < valid) {
                            float x[32];
                            scores(i, x);
                            uint32_t r[16];
#pragma unroll
                            for (int k = 0; k < 16; k++) {
                                float u, v;
                                unpair(fma2(pair(x[2 * k], x[2 * k + 1]), c2, m2), u, v);
                                u = exp2_fast(u);
                                v = exp2_fast(v);
                                sum[k & 1] = add2(sum[k & 1], pair(u, v));
                                r[k] = round2<T>(u, v);
                            }
                            tmem_store16(ts + 16 * i, r);
                        }
                    }
                    if (DP == 64 && lane == 0) busy[warp] = 0u;
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
            if (!idle) {
                if (!pair_of.meet()) break;                         // both have read the last maximum
                s_told[warp][lane] = l;
                if (!pair_of.meet()) break;
                l += s_told[warp ^ 4u][lane];
                if (!pair_of.meet()) break;                         // and the sum, before the next item's maximum
            }
            // A row that sees none of these keys is told by the mask and not by its sum, so that a sum that is NaN (a score is, or
            // one is +inf) or zero (all scores are -inf) goes on to the results as NaN.
            const bool sees = row < a.Sq && limit > it.j0 * kBlock;
            const float by = __fdiv_rn(1.0f, l);
            if (blocks > 0) {
                if (!bar_wait(&o_done[w], (pv - 1u) & 1u, stop)) break;
                tmem_after_sync();
            }
            if (idle) continue;
            const uint64_t bh = (uint64_t)it.b * a.H + it.h, part_row = ((uint64_t)it.split * a.B * a.H + bh) * a.Sq + row;
            if (part == 0 && row < a.Sq) {
                const float lse2 = sees ? m + log2f(l) : -INFINITY;
                if (p.splits > 1u) p.part_lse2[part_row] = lse2;
                else a.lse[bh * a.Sq + row] = lse2 * 0.69314718055994531f;
            }
#pragma unroll
            for (int i = 0; i < DP / 64; i++) {
                const uint32_t from = part * (DP / 2) + 32u * i;
                if (from >= a.D) continue;
                float o[32];
                if (blocks > 0) {
                    tmem_load32(to + 32 * i, o);
                    tmem_wait_loads();
                }
                if (p.splits > 1u) {                                // for attention_join_kernel, in binary32
                    float4 *const to_part = reinterpret_cast<float4 *>(p.part_out + part_row * a.D + from);
#pragma unroll
                    for (int k = 0; k < 8; k++)
                        if (row < a.Sq && from + 4u * k < a.D)
                            to_part[k] = sees ? make_float4(o[4 * k] * by, o[4 * k + 1] * by, o[4 * k + 2] * by, o[4 * k + 3] * by)
                                                  : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    continue;
                }
                if (lane == 0) stores_read<0>();
                __syncwarp();
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (sees) {
                        v.x = round2<T>(o[8 * k] * by, o[8 * k + 1] * by);
                        v.y = round2<T>(o[8 * k + 2] * by, o[8 * k + 3] * by);
                        v.z = round2<T>(o[8 * k + 4] * by, o[8 * k + 5] * by);
                        v.w = round2<T>(o[8 * k + 6] * by, o[8 * k + 7] * by);
                    }
                    stage_piece(s_out, lane, k, v);
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tma_store(&p.out, s_out, from, it.h, first + (warp & 3u) * 32u, it.b);
            }
            tmem_before_sync();
        }
        if (item < p.items) pair_of.give_up(warp, lane, &s_told[warp][lane]);
        if (lane == 0) stores_done();
    } else {
        leave_registers<64>();
        if (warp == 17) {                                               // ---- copies
            uint32_t st = 0, ph = 1, q = 0, q_ph = 1, tail_ph = 0;   // a fresh barrier's "previous" phase counts as complete
            FwdItem it;
            for (uint32_t item = blockIdx.x; next_item(p, item, it); item += gridDim.x) {
                if (!bar_wait(&q_empty[q], q_ph, stop)) break;
                if (lane == 0) {
                    bar_expect(&q_full[q], ((it.blocks[0] > 0) + (it.blocks[1] > 0)) * Smem::kTile);
#pragma unroll
                    for (int w = 0; w < 2; w++)
                        if (it.blocks[w] > 0)
                            for (int x = 0; x < DP / 64; x++)
                                tma_load(smem_u32(smem) + (2u * q + w) * Smem::kTile + x * 16384, &p.q, &q_full[q], 64 * x, it.h, it.m0 + 128 * w, it.b);
                }
                if (++q == Smem::kQueries) {
                    q = 0;
                    q_ph ^= 1u;
                }
                for (int i = 0; i < 2 * it.both; i++) {                // K0 V0 K1 V1 ...
                    const int j = it.j0 + (i >> 1);
                    const bool is_v = i & 1;
                    if (!bar_wait(&kv_empty[st], ph, stop)) break;
                    unsigned char *const dst = smem + Smem::kKeys + st * Smem::kTile;
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
        } else if (warp == 16) {                                        // ---- products
            const uint32_t one = elect_lane();
            uint32_t st = 0, ph = 0, q_at = 0, q_ph = 0, p_ph[2] = {0, 0};
            const uint32_t q_smem = smem_u32(smem), kv_smem = q_smem + Smem::kKeys;
            const uint32_t steps = (a.D + 15u) / 16u;              // of the first product
            const uint32_t pv_desc = product_desc(BF16, steps * 16u, true);
            uint32_t item = blockIdx.x;
            FwdItem it, after;
            bool more_items = next_item(p, item, it);
            while (more_items) {
                const uint32_t qb = q_at;
                if (!bar_wait(&q_full[qb], q_ph, stop)) break;
                if (++q_at == Smem::kQueries) {
                    q_at = 0;
                    q_ph ^= 1u;
                }
                // S of half w for the key block in stage `at`
                auto scores = [&](int w, int j, uint32_t at) {
                    const uint32_t valid = it.n - (uint32_t)(it.j0 + j) * kBlock, cols = valid < (uint32_t)kBlock ? (valid + 15u) & ~15u : kBlock;
                    const uint32_t desc = product_desc(BF16, cols, false);
                    const uint32_t q = operand_low(q_smem + (2u * qb + w) * Smem::kTile, 16), k = operand_low(kv_smem + at * Smem::kTile, 16);
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
                if (it.both == 1) products_done(one, &q_empty[qb]);
                next();
                item += gridDim.x;                                 // decoded while softmax has the first block
                more_items = next_item(p, item, after);
                for (int j = 0; j < it.both; j++) {
                    const uint32_t v_st = st;
                    if (!bar_wait(&kv_full[st], ph, stop)) break;
                    next();
                    const bool more = j + 1 < it.both;
                    if (more && !bar_wait(&kv_full[st], ph, stop)) break;
                    const uint32_t valid = it.n - (uint32_t)(it.j0 + j) * kBlock;
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
                            if (s < pv_steps) product_ts<true>(one, tmem + 256u + w * DP, tmem + w * 128u + (s >> 2) * 64u + (s & 3u) * 8u, v + s * 128u, pv_desc);
                        products_done(one, &o_done[w]);
                        if (j + 1 < it.blocks[w]) scores(w, j + 1, st);
                    }
                    products_done(one, &kv_empty[v_st]);
                    if (more) {
                        products_done(one, &kv_empty[st]);
                        if (j + 2 == it.both) products_done(one, &q_empty[qb]);
                        next();
                    }
                }
                if (*stop) break;
                it = after;
            }
            products_done(one, &drain);
            bar_wait(&drain, 0, stop);
        }
    }
    tmem_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && s_abort) record_error(p.header, p.a.device_status, DAF_ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, 512);
}

// Joins the splits of each row, a warp per row, in the order of the keys: out = sum of 2^(lse2_s - lse2) out_s.
template <typename T> __global__ void __launch_bounds__(256) attention_join_kernel(const __grid_constant__ AttnForwardArgs p)
{
    const AttnArgs &a = p.a;
    const uint64_t rows = (uint64_t)a.B * a.H * a.Sq, r = (uint64_t)blockIdx.x * 8u + (threadIdx.x >> 5);
    const uint32_t lane = threadIdx.x & 31u;
    if (r >= rows) return;
    float top = -INFINITY;                                         // NaN if one of the splits' is
    for (uint32_t s = lane; s < p.splits; s += 32u) top = max_or_nan(top, p.part_lse2[s * rows + r]);
#pragma unroll
    for (int d = 16; d; d >>= 1) top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, d));
    const uint64_t bh = r / a.Sq;
    const uint32_t i = (uint32_t)(r - bh * a.Sq), b = (uint32_t)(bh / a.H), h = (uint32_t)(bh - (uint64_t)b * a.H);
    const bool some = attn_limit(a, attn_length(a, b), (int)i) > 0, mine = lane * 4u < a.D;   // the row sees a key
    float total = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t s = 0; some && s < p.splits; s++) {
        const float w = exp2_fast(p.part_lse2[s * rows + r] - top);
        total += w;
        if (!mine || w == 0.0f) continue;                          // nothing of a split that saw nothing, or only scores of -inf
        const float4 x = *reinterpret_cast<const float4 *>(p.part_out + (s * rows + r) * a.D + lane * 4u);
        o.x = __fmaf_rn(w, x.x, o.x);
        o.y = __fmaf_rn(w, x.y, o.y);
        o.z = __fmaf_rn(w, x.z, o.z);
        o.w = __fmaf_rn(w, x.w, o.w);
    }
    const float by = some ? __fdiv_rn(1.0f, total) : 0.0f;
    if (mine) {
        const uint2 v = make_uint2(round2<T>(o.x * by, o.y * by), round2<T>(o.z * by, o.w * by));
        *reinterpret_cast<uint2 *>(reinterpret_cast<char *>(a.out.p) + 2u * (a.out.sb * b + a.out.ss * i + a.out.sh * h + lane * 4u)) = v;
    }
    if (lane == 0) a.lse[r] = some && top != -INFINITY ? (top + log2f(total)) * 0.69314718055994531f : -INFINITY;
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
    AttnForwardArgs p = {};
    p.a = a;
    p.splits = attn_splits(a);
    p.split_div.set(p.splits);
    p.part_out = reinterpret_cast<float *>(header + 1);
    p.part_lse2 = p.part_out + (uint64_t)p.splits * a.B * a.H * a.Sq * a.D;
    p.a.scale_log2 = fmaxf(fabsf(a.scale_log2), 0x1p-100f);       // the sign is applied to S; never 0, which masks would turn into NaN
    p.q_tiles = (a.Sq + kFwdRows - 1u) / kFwdRows;
    p.items = p.q_tiles * a.B * a.H * p.splits;
    p.header = header;
    const bool bf16 = __is_same(T, __nv_bfloat16);
    p.heads.set(a.H);
    p.all_heads.set(a.B * a.H);
    p.tiles.set(p.q_tiles);
    if (!attn_tensor_map(&p.q, bf16, a.q, a.B, a.Sq, a.H, a.D, 128) || !attn_store_map(&p.out, bf16, a.out, a.B, a.Sq, a.H, a.D)) return DAF_ERR_CUDA;
    if (a.Sk == 0) p.k = p.v = p.q;                                // never read
    else if (!attn_tensor_map(&p.k, bf16, a.k, a.B, a.Sk, a.Hkv, a.D, 128) || !attn_tensor_map(&p.v, bf16, a.v, a.B, a.Sk, a.Hkv, a.D, 128))
        return DAF_ERR_CUDA;
    const daf_status st = a.D <= 64u ? launch_forward<T, 64>(p, s) : launch_forward<T, 128>(p, s);
    if (st != DAF_OK || p.splits == 1u) return st;
    attention_join_kernel<T><<<(uint32_t)(((uint64_t)a.B * a.H * a.Sq + 7u) / 8u), 256, 0, s>>>(p);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

}  // namespace daf
