// Attention backward for 16-bit inputs on the tensor cores: one kernel body, two instances.
//
//   dk / dv (DKV)  holds 128 keys,    walks the queries of every head that reads them:  T1 = k q^T,  T2 = v grad_out^T
//   dq             holds 128 queries, walks the keys:                                   T1 = q k^T,  T2 = grad_out v^T
//   P = exp2(c T1 - L),  dS = P (T2 - delta)      (L = lse log2(e); both operands of T1 and T2 come from shared memory)
//   dv += P grad_out,  dk += dS q                 /  dq += dS k        (P and dS, 16 bits, from tensor memory)
//
// No sum crosses CTAs: no atomics, the same bits every time, and no binary32 copies of the gradients.  The price is that
// S and dP are computed twice (7 products instead of 5); against it stands that every A operand of a second product is
// where softmax leaves it -- in tensor memory, row by row -- so that P and dS never pass through shared memory.
//
// A persistent CTA (one per SM): warps 0-7 and 8-15 take the walk's blocks of 64 in turn (a thread owns 32 columns of one
// of the 128 rows), warp 16 issues the products, up to three blocks of T ahead of the sums, warp 17 the copies.  Tensor
// memory: the sums (64 to 256 columns) and three blocks of T1, T2 (128 columns each; two where the sums take 256), P over
// T1 and dS over T2.  What bounds it is the way of a block -- product, tensor memory to registers, exponentials, back,
// second product, about 2500 cycles of latency --, so blocks in flight matter more than the wider products that blocks
// of 128 would give, and eight warps per block more than long rows in few threads.
// P and dS are rounded to the input type, which the second products need; everything else is binary32.  float16 reaches
// from 6e-5 (6e-8 with fewer bits) to 65504, and dS may lie anywhere -- a mean over many tokens, a loss on a few of them or a
// loss scale moves grad_out --, so there dS is multiplied by the power of two that brings its bound 2 |grad_out| max |v| to
// [2^14, 2^15) (max |v| taken as sqrt(D) times the largest element), and the sums by its inverse: |grad_out| is the row's in
// dq, whose sums belong to one row, and the largest row's of the head in dk.  P is held 2^8 times its size: probabilities down
// to 2^-22 keep their bits.
#pragma once
#include "attention.cuh"
#include "tensor_core.cuh"

namespace daf {

constexpr int kGradThreads = 640;                // 16 warps x 104 registers, 4 (two of them idle) x 64: what 640 x 96 gives
constexpr uint32_t kHeld = 128, kWalk = 64;

struct AttnGradArgs {
    CUtensorMap x1, x2, y1, y2;                  // held: k, v or q, grad_out; walked: q, grad_out or k, v; boxes of a walked tile's rows
    CUtensorMap out[2];                          // dv, dk or dq
    AttnArgs a;
    FastDiv heads, all_heads, tile_div;          // heads of the items, times B, tiles
    uint32_t items, tiles;
    WorkspaceHeader *header;
};

template <int DP, bool DKV> struct GradSmem {
    static constexpr int kHeldBuffers = DP == 128 ? 1 : 2, kStages = DP == 128 ? 4 : 6;
    static constexpr uint32_t kX = kHeld * DP * 2u, kY = kWalk * DP * 2u;
    static constexpr uint32_t kStats = 2u * kWalk * 4u;           // -L and -delta of a block's queries
    // blocks of T in tensor memory, behind the sums
    static constexpr uint32_t kAhead = (512u - (DKV ? 2u : 1u) * DP) / 128u < 3u ? 2u : 3u, kT = 512u - kAhead * 128u;
    static constexpr uint32_t kOut = 2048u;                       // a piece of 32 x 32 results for each of the 16 warps
    static constexpr uint32_t kBars = 1024u;                      // barriers and such, ahead of everything
    static constexpr uint32_t kBytes = kBars + kHeldBuffers * 2u * kX + kStages * (2u * kY + kStats) + 16u * kOut;
};

// That power of two, from the squared norms of grad_out and v (1 where one is zero or not finite).
__device__ __forceinline__ float score_grad_scale(float grad2, float value2)
{
    const int e = (int)(__float_as_uint(sqrtf(grad2) * sqrtf(value2)) >> 23) - 127;
    return e < -100 || e > 100 ? 1.0f : __uint_as_float((uint32_t)(127 + 13 - e) << 23);
}

// The i-th item of a CTA: there and back over the list, which starts with the longest items, so that who got a long
// one gets a short one next.
__device__ __forceinline__ uint32_t grad_item(uint32_t i)
{
    return i * gridDim.x + (i & 1u ? gridDim.x - 1u - blockIdx.x : blockIdx.x);
}

template <bool DKV, uint32_t WALK = kWalk> struct GradItem {
    uint32_t b, h, first, n;                     // h: key head (DKV) or query head
    uint32_t start, per_head, blocks;            // the walk: `per_head` blocks from `start` on, for each head
    __device__ __forceinline__ void set(const AttnGradArgs &p, uint32_t item)
    {
        const AttnArgs &a = p.a;
        uint32_t tile, bh;
        if (a.causal) {
            tile = p.all_heads.div(item);
            bh = item - tile * p.all_heads.d;
            if (!DKV) tile = p.tiles - 1u - tile;
        } else {
            bh = p.tile_div.div(item);
            tile = item - bh * p.tiles;
        }
        b = p.heads.div(bh);
        h = bh - b * p.heads.d;
        first = tile * kHeld;
        n = attn_length(a, b);
        start = 0;
        per_head = 0;
        if (DKV) {
            const int from = a.causal ? (int)(first + a.Sq) - (int)a.Sk : 0;   // the first query that sees a key of the tile
            if (from > 0) start = (uint32_t)from / WALK * WALK;
            if (first < n && start < a.Sq) per_head = (a.Sq - start + WALK - 1u) / WALK;
            blocks = per_head * a.group;
        } else {
            const uint32_t last = (first + kHeld < a.Sq ? first + kHeld : a.Sq) - 1u;
            const int end = attn_limit(a, n, (int)last);
            per_head = blocks = end > 0 ? ((uint32_t)end + WALK - 1u) / WALK : 0u;
        }
    }
};

// Walks the blocks of a CTA's items one after another: block `i` of the item, at row `row` of head `head`.
template <bool DKV, uint32_t WALK = kWalk> struct GradCursor {
    GradItem<DKV, WALK> it;
    uint32_t turn, i, in_head, row, head;
    bool more;
    __device__ __forceinline__ void open(const AttnGradArgs &p)
    {
        turn = 0;
        enter(p);
    }
    // to the first block of item number `turn`, or of the next one that has blocks
    __device__ __forceinline__ void enter(const AttnGradArgs &p)
    {
        for (;; turn++) {
            const uint32_t item = grad_item(turn);
            more = item < p.items;
            // the way back may pass the list's end before the way there of the same pair does
            if (!more && turn * gridDim.x >= p.items) return;
            if (!more) continue;
            it.set(p, item);
            if (it.blocks) break;
        }
        i = in_head = 0;
        row = it.start;
        head = DKV ? it.h * p.a.group : it.h / p.a.group;
    }
    __device__ __forceinline__ bool last() const { return i + 1u == it.blocks; }
    __device__ __forceinline__ uint32_t cols(const AttnGradArgs &p) const
    {
        const uint32_t left = (DKV ? p.a.Sq : it.n) - row;
        return left < WALK ? left : WALK;
    }
    __device__ __forceinline__ void step(const AttnGradArgs &p)
    {
        if (++i == it.blocks) {
            turn++;
            enter(p);
            return;
        }
        row += WALK;
        if (DKV && ++in_head == it.per_head) {
            in_head = 0;
            row = it.start;
            head++;
        }
    }
};

template <typename T, int DP, bool DKV>
__global__ void __launch_bounds__(kGradThreads, 1) attention_grad_kernel(const __grid_constant__ AttnGradArgs p)
{
    using Smem = GradSmem<DP, DKV>;
    constexpr bool BF16 = __is_same(T, __nv_bfloat16);
    constexpr int STAGES = Smem::kStages, HELD = Smem::kHeldBuffers;
    constexpr uint32_t AHEAD = Smem::kAhead;
    constexpr uint32_t XBOX = kHeld * 128u, YBOX = kWalk * 128u;  // bytes of a 64-element box
    // tiles need 1024-byte boundaries; with nothing declared statically the dynamic part starts on one
    extern __shared__ __align__(1024) unsigned char s_raw[];
    struct Bars {
        uint64_t x_full[2], x_empty[2], y_full[6], y_empty[6], t_full[3], ps_ready[3], acc_full, acc_empty, tail, drain;
        uint32_t tmem, abort;
    };
    static_assert(sizeof(Bars) <= Smem::kBars && HELD <= 2 && STAGES <= 6 && AHEAD <= 3, "barriers fit their places");
    Bars &bars = *reinterpret_cast<Bars *>(s_raw);
    uint64_t *const x_full = bars.x_full, *const x_empty = bars.x_empty, *const y_full = bars.y_full, *const y_empty = bars.y_empty,
             *const t_full = bars.t_full, *const ps_ready = bars.ps_ready;
    uint64_t &acc_full = bars.acc_full, &acc_empty = bars.acc_empty, &tail = bars.tail, &drain = bars.drain;
    uint32_t &s_tmem = bars.tmem, &s_abort = bars.abort;
    if (smem_u32(s_raw) & 1023u) {                                 // the same for every thread
        if (threadIdx.x == 0) record_error(p.header, p.a.device_status, DAF_ERR_UNSUPPORTED);
        return;
    }
    unsigned char *const smem = s_raw + Smem::kBars;
    unsigned char *const s_y = smem + HELD * 2u * Smem::kX;
    unsigned char *const s_out = s_y + STAGES * 2u * Smem::kY;
    float *const s_stats = reinterpret_cast<float *>(s_out + 16u * Smem::kOut);
    const AttnArgs &a = p.a;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
    if (threadIdx.x == 0) {
        s_abort = 0u;
        for (int i = 0; i < HELD; i++) {
            bar_init(&x_full[i], 1);
            bar_init(&x_empty[i], 1);
        }
        for (int i = 0; i < STAGES; i++) {
            bar_init(&y_full[i], 1);
            bar_init(&y_empty[i], 1);
        }
        for (uint32_t w = 0; w < AHEAD; w++) {
            bar_init(&t_full[w], 1);
            bar_init(&ps_ready[w], 8);
        }
        bar_init(&acc_full, 1);
        bar_init(&acc_empty, 16);
        bar_init(&tail, 1);
        bar_init(&drain, 1);
        fence_async();
    }
    if (warp == 0) tmem_alloc(&s_tmem, 512);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = s_tmem;
    volatile uint32_t *const stop = &s_abort;

    if (warp < 16) {                                               // ---- probabilities, score gradients, results
        take_registers<104>();
        const uint32_t turn_of = warp >> 3, part = (warp >> 2) & 1u, quarter = (warp & 3u) << 21, lane_row = (warp & 3u) * 32u + lane;
        uint32_t count = 0, buf = 0, t_ph = 0, acc_ph = 0, stage = 0, y_ph = 0;   // count: blocks passed, over all items
        const int off = (int)a.Sk - (int)a.Sq;
        const uint64_t c2 = pair(a.scale_log2, a.scale_log2);
        GradItem<DKV> it;
        float nl = 0.0f, nd = 0.0f, lift = 1.0f;                   // lift: what float16 multiplies its (lifted) P by for dS
        constexpr bool F16 = __is_same(T, __half);
        // item number `turn`, and for dq what its row brings along; false behind the last one
        auto enter = [&](uint32_t &turn) {
            for (; turn * gridDim.x < p.items; turn++) {
                const uint32_t item = grad_item(turn);
                if (item >= p.items) continue;
                it.set(p, item);
                if (F16) {
                    const uint32_t head = it.b * a.Hkv + (DKV ? it.h : it.h / a.group);
                    const float grad2 = DKV ? a.grad_max[head] : a.row_norm2[((uint64_t)it.b * a.H + it.h) * a.rows_padded + it.first + lane_row];
                    lift = score_grad_scale(grad2, a.value_max[head]) * exp2f(-kHalfLift);
                }
                if (!DKV && it.blocks) {
                    const uint64_t at = ((uint64_t)it.b * a.H + it.h) * a.rows_padded + it.first + lane_row;
                    nl = a.row_nl2[at];
                    nd = a.row_ndelta[at];
                }
                return true;
            }
            return false;
        };
        uint32_t turn = 0;
        bool ok = enter(turn);
        while (ok) {
            const uint32_t row = it.first + lane_row, rows = DKV ? a.Sk : a.Sq, live = DKV ? it.n : a.Sq;
            const bool idle = it.first + (warp & 3u) * 32u >= live; // no row of the warp takes part
            const int limit = DKV ? 0 : row < a.Sq ? attn_limit(a, it.n, (int)row) : (int)it.n;   // dq: keys the row sees
            uint32_t at = it.start, in_head = 0;
            for (uint32_t i = 0; i < it.blocks; i++) {
                if ((count & 1u) == turn_of) {
                    if (!(ok = bar_wait(&t_full[buf], t_ph, stop))) break;
                    if (DKV && !(ok = bar_wait(&y_full[stage], y_ph, stop))) break;   // the statistics came by copy
                    const int cols = (int)((DKV ? a.Sq : it.n) - at);
                    if (!idle && 32 * (int)part < cols) {
                        tmem_after_sync();
                        const uint32_t t = tmem + Smem::kT + buf * 128u + quarter;
                        float s[32], e[32];
                        tmem_load32(t + 32u * part, s);
                        tmem_load32(t + 64u + 32u * part, e);
                        // of these columns the row sees [lo, hi)
                        int lo = 0, hi = 32;
                        if (DKV) lo = row >= it.n ? 32 : a.causal ? (int)row - off - (int)at - 32 * (int)part : 0;
                        else hi = limit - (int)at - 32 * (int)part;
                        const bool masked = __any_sync(0xffffffffu, lo > 0 || hi < 32);
                        const float *const st = s_stats + stage * 2u * kWalk + 32u * part;
                        tmem_wait_loads();
                        uint32_t r1[16], r2[16];
#pragma unroll
                        for (int k = 0; k < 8; k++) {              // four columns
                            uint64_t l2[2], d2[2];
                            if (DKV) {
                                const float4 u = *reinterpret_cast<const float4 *>(st + 4 * k);
                                const float4 v = *reinterpret_cast<const float4 *>(st + kWalk + 4 * k);
                                l2[0] = pair(u.x, u.y); l2[1] = pair(u.z, u.w);
                                d2[0] = pair(v.x, v.y); d2[1] = pair(v.z, v.w);
                            } else {
                                l2[0] = l2[1] = pair(nl, nl);
                                d2[0] = d2[1] = pair(nd, nd);
                            }
#pragma unroll
                            for (int q = 0; q < 2; q++) {
                                const int c = 4 * k + 2 * q;
                                float u, v, x, y;
                                unpair(fma2(pair(s[c], s[c + 1]), c2, l2[q]), u, v);
                                u = exp2_fast(u);
                                v = exp2_fast(v);
                                const uint64_t pr = F16 ? mul2(pair(u, v), both(lift)) : pair(u, v);
                                unpair(mul2(pr, add2(pair(e[c], e[c + 1]), d2[q])), x, y);
                                r1[2 * k + q] = round2<T>(u, v);
                                r2[2 * k + q] = round2<T>(x, y);
                            }
                        }
                        if (masked) {                              // cleared, not multiplied: what is masked may be NaN
#pragma unroll
                            for (int k = 0; k < 16; k++) {
                                const uint32_t m = (2 * k >= lo && 2 * k < hi ? 0xFFFFu : 0u) | (2 * k + 1 >= lo && 2 * k + 1 < hi ? 0xFFFF0000u : 0u);
                                r1[k] &= m;
                                r2[k] &= m;
                            }
                        }
                        __syncwarp();
                        // P and dS go over the columns that this warp has read
                        if (DKV) tmem_store16(t + 32u * part, r1);
                        tmem_store16(t + 64u + 32u * part, r2);
                        tmem_wait_stores();
                        tmem_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) bar_arrive(&ps_ready[buf]);
                }
                count++;
                if (++buf == AHEAD) {
                    buf = 0;
                    t_ph ^= 1u;
                }
                if (++stage == STAGES) {
                    stage = 0;
                    y_ph ^= 1u;
                }
                at += kWalk;
                if (DKV && ++in_head == it.per_head) {
                    in_head = 0;
                    at = it.start;
                }
            }
            if (!ok) break;
            // DKV: warpgroups 0 and 2 store dv, 1 and 3 dk, half of the columns each; dq: 32 columns each, as far as they go
            const uint32_t group = warp >> 2;
            const CUtensorMap *const to = &p.out[DKV ? group & 1u : 0u];
            const float by = DKV && !(group & 1u) ? (F16 ? exp2f(-kHalfLift) : 1.0f) : F16 ? __fdiv_rn(a.scale * exp2f(-kHalfLift), lift) : a.scale;
            constexpr uint32_t WIDTH = DKV ? DP / 2 : 32;
            const uint32_t from = (DKV ? group >> 1 : group) * WIDTH;
            const uint32_t acc = tmem + (DKV ? (group & 1u) * DP : 0u) + from + quarter;
            const bool some = it.blocks > 0, any = some && !idle, keep = any && row < live && (DKV || limit > 0);
            const uint32_t out_h = it.h, out_b = it.b, out_row = it.first + (warp & 3u) * 32u;
            const bool exists = out_row < rows && from < a.D;
            turn++;
            const bool more = enter(turn);                          // its loads come back while this item's last products run
            if (some) {
                if (!(ok = bar_wait(&acc_full, acc_ph, stop))) break;
                acc_ph ^= 1u;
                tmem_after_sync();
            }
            unsigned char *const piece = s_out + warp * Smem::kOut;
#pragma unroll
            for (uint32_t ch = 0; ch < WIDTH / 32; ch++) {
                if (!exists || from + 32u * ch >= a.D) continue;
                float o[32];
                if (any) {
                    tmem_load32(acc + 32 * ch, o);
                    tmem_wait_loads();
                }
                if (lane == 0) stores_read<0>();
                __syncwarp();
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (keep) {
                        v.x = round2<T>(o[8 * k] * by, o[8 * k + 1] * by);
                        v.y = round2<T>(o[8 * k + 2] * by, o[8 * k + 3] * by);
                        v.z = round2<T>(o[8 * k + 4] * by, o[8 * k + 5] * by);
                        v.w = round2<T>(o[8 * k + 6] * by, o[8 * k + 7] * by);
                    }
                    stage_piece(piece, lane, k, v);
                }
                fence_async();
                __syncwarp();
                if (lane == 0) tma_store(to, piece, from + 32u * ch, out_h, out_row, out_b);
            }
            if (some) {
                tmem_before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&acc_empty);
            }
            ok = more;
        }
        if (lane == 0) stores_done();
    } else {
        leave_registers<64>();
        if (warp == 17) {                                          // ---- copies
            GradCursor<DKV> cur;
            uint32_t st = 0, ph = 1, x = 0, x_ph = 1, tail_ph = 0;
            for (cur.open(p); cur.more; cur.step(p)) {
                const bool one = lane == 0;
                if (cur.i == 0) {
                    if (!bar_wait(&x_empty[x], x_ph, stop)) break;
                    if (one) {
                        const uint32_t dst = smem_u32(smem) + x * 2u * Smem::kX;
                        bar_expect(&x_full[x], 2u * Smem::kX);
                        for (int e = 0; e < DP / 64; e++)
                            for (int r = 0; r < 2; r++) {          // a box has half of a held tile's rows
                                const int row = cur.it.first + kWalk * r;
                                tma_load(dst + e * XBOX + r * YBOX, &p.x1, &x_full[x], 64 * e, cur.it.h, row, cur.it.b);
                                tma_load(dst + Smem::kX + e * XBOX + r * YBOX, &p.x2, &x_full[x], 64 * e, cur.it.h, row, cur.it.b);
                            }
                    }
                    if (++x == HELD) {
                        x = 0;
                        x_ph ^= 1u;
                    }
                }
                if (!bar_wait(&y_empty[st], ph, stop)) break;
                const uint32_t cols = cur.cols(p), end = (cols + 15u) & ~15u;
                // P and dS are zero in a masked column, but 0 * NaN is not.  Cleared are rows of k behind the sequence's end that
                // the last product's steps of 16 keys still touch, and rows of q and grad_out that see no key at all.
                const int dead = DKV && a.causal ? (int)(a.Sq - cur.row) - (int)a.Sk : 0;
                const uint32_t clear_from = DKV ? 0u : cols;
                const uint32_t clear_to = !DKV ? (cur.it.n < a.Sk ? end : cols) : dead <= 0 ? 0u : dead < (int)kWalk ? (uint32_t)dead : kWalk;
                const bool clear = clear_from != clear_to;
                uint64_t *const bar = clear ? &tail : &y_full[st];
                unsigned char *const dst = s_y + st * 2u * Smem::kY;
                if (one) {
                    bar_expect(bar, 2u * Smem::kY + (DKV ? Smem::kStats : 0u));
                    for (int e = 0; e < DP / 64; e++) {
                        tma_load(smem_u32(dst) + e * YBOX, &p.y1, bar, 64 * e, cur.head, cur.row, cur.it.b);
                        tma_load(smem_u32(dst) + Smem::kY + e * YBOX, &p.y2, bar, 64 * e, cur.head, cur.row, cur.it.b);
                    }
                    if (DKV) {
                        const uint64_t at = ((uint64_t)cur.it.b * a.H + cur.head) * a.rows_padded + cur.row;
                        bulk_load(smem_u32(s_stats + st * 2u * kWalk), a.row_nl2 + at, kWalk * 4u, bar);
                        bulk_load(smem_u32(s_stats + st * 2u * kWalk + kWalk), a.row_ndelta + at, kWalk * 4u, bar);
                    }
                }
                if (clear) {
                    if (!bar_wait(&tail, tail_ph, stop)) break;
                    tail_ph ^= 1u;
                    const uint32_t pieces = 8u * (clear_to - clear_from);
                    for (uint32_t i = lane; i < pieces * (DP / 64) * (DKV ? 2u : 1u); i += 32u)    // boxes follow one another
                        *reinterpret_cast<uint4 *>(dst + i / pieces * YBOX + (clear_from * 8u + i % pieces) * 16u) = make_uint4(0u, 0u, 0u, 0u);
                    fence_async();
                    __syncwarp();
                    if (one) bar_arrive(&y_full[st]);
                }
                if (++st == STAGES) {
                    st = 0;
                    ph ^= 1u;
                }
            }
            if (*stop) {                                           // giving up: let the copies in flight land first
                const uint64_t until = now_ns() + 1000000000ull;
                while (now_ns() < until) __nanosleep(1000);
            }
        } else if (warp == 16) {                                   // ---- products
            const uint32_t one = elect_lane();
            const uint32_t steps = (a.D + 15u) / 16u;
            const uint32_t acc_desc = product_desc(BF16, steps * 16u, true);
            const uint32_t xs = smem_u32(smem), ys = smem_u32(s_y);
            GradCursor<DKV> ahead, cur;
            ahead.open(p);
            cur.open(p);
            uint32_t t_st = 0, t_phase = 0, t_buf = 0, x = 0, x_ph = 0, c_st = 0, c_buf = 0, acc_ph = 1, ps_ph = 0;
            bool ok = true;
            // T1 and T2 of the block `ahead` stands at
            auto scores = [&]() {
                if (!ahead.more) return;
                if (ahead.i == 0 && !(ok = bar_wait(&x_full[x], x_ph, stop))) return;
                if (!(ok = bar_wait(&y_full[t_st], t_phase, stop))) return;
                tmem_after_sync();
                const uint32_t t = tmem + Smem::kT + t_buf * 128u;
                const uint32_t desc = product_desc(BF16, (ahead.cols(p) + 15u) & ~15u, false);
#pragma unroll
                for (uint32_t k = 0; k < 2; k++) {
                    const uint32_t A = operand_low(xs + x * 2u * Smem::kX + k * Smem::kX, 16), B = operand_low(ys + t_st * 2u * Smem::kY + k * Smem::kY, 16);
                    product_ss(one, t + k * 64u, A, B, desc, false);
#pragma unroll
                    for (uint32_t s = 1; s < DP / 16; s++)
                        if (s < steps)
                            product_ss<true>(one, t + k * 64u, A + ((s & 3u) * 2u + (s >> 2) * (XBOX / 16u)), B + ((s & 3u) * 2u + (s >> 2) * (YBOX / 16u)), desc);
                }
                products_done(one, &t_full[t_buf]);
                if (++t_buf == AHEAD) t_buf = 0;
                if (ahead.last()) {
                    products_done(one, &x_empty[x]);
                    if (++x == HELD) {
                        x = 0;
                        x_ph ^= 1u;
                    }
                }
                if (++t_st == STAGES) {
                    t_st = 0;
                    t_phase ^= 1u;
                }
                ahead.step(p);
            };
            for (uint32_t i = 0; i < AHEAD && ok; i++) scores();
            for (; ok && cur.more; cur.step(p)) {
                const uint32_t t = tmem + Smem::kT + c_buf * 128u, n16 = (cur.cols(p) + 15u) / 16u;
                if (!bar_wait(&ps_ready[c_buf], ps_ph, stop)) break;
                if (++c_buf == AHEAD) {
                    c_buf = 0;
                    ps_ph ^= 1u;
                }
                if (cur.i == 0) {
                    if (!bar_wait(&acc_empty, acc_ph, stop)) break;
                    acc_ph ^= 1u;
                }
                tmem_after_sync();
                const uint32_t y1 = operand_low(ys + c_st * 2u * Smem::kY, YBOX), y2 = operand_low(ys + c_st * 2u * Smem::kY + Smem::kY, YBOX);
                const bool add = cur.i > 0;
                // 16 rows of the walk a step: 2 KiB of the tile, 8 columns of P or dS
                if (DKV) {
                    product_ts(one, tmem, t, y2, acc_desc, add);
#pragma unroll
                    for (uint32_t s = 1; s < kWalk / 16; s++)
                        if (s < n16) product_ts<true>(one, tmem, t + (s >> 1) * 32u + (s & 1u) * 8u, y2 + s * 128u, acc_desc);
                }
                product_ts(one, tmem + (DKV ? DP : 0), t + 64u, y1, acc_desc, add);
#pragma unroll
                for (uint32_t s = 1; s < kWalk / 16; s++)
                    if (s < n16) product_ts<true>(one, tmem + (DKV ? DP : 0), t + 64u + (s >> 1) * 32u + (s & 1u) * 8u, y1 + s * 128u, acc_desc);
                products_done(one, &y_empty[c_st]);
                if (cur.last()) products_done(one, &acc_full);
                if (++c_st == STAGES) c_st = 0;
                scores();
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

template <typename T, int DP, bool DKV> static daf_status launch_grad(const AttnGradArgs &p, cudaStream_t s)
{
    int ctas = 0;
    const auto kernel = &attention_grad_kernel<T, DP, DKV>;
    if (persistent_ctas(reinterpret_cast<const void *>(kernel), kGradThreads, (int)GradSmem<DP, DKV>::kBytes, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    kernel<<<p.items < (uint32_t)ctas ? p.items : (uint32_t)ctas, kGradThreads, GradSmem<DP, DKV>::kBytes, s>>>(p);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

// Keys and queries both exist (the entry point writes the gradients of the other cases).
template <typename T> daf_status attn_backward_tc(const AttnArgs &a, WorkspaceHeader *header, cudaStream_t s)
{
    const bool bf16 = __is_same(T, __nv_bfloat16);
    AttnGradArgs p;
    p.a = a;
    p.header = header;
    CUtensorMap q, k, v, g;
    if (!attn_tensor_map(&q, bf16, a.q, a.B, a.Sq, a.H, a.D, kWalk) || !attn_tensor_map(&g, bf16, a.grad_out, a.B, a.Sq, a.H, a.D, kWalk) ||
        !attn_tensor_map(&k, bf16, a.k, a.B, a.Sk, a.Hkv, a.D, kWalk) || !attn_tensor_map(&v, bf16, a.v, a.B, a.Sk, a.Hkv, a.D, kWalk) ||
        !attn_store_map(&p.out[0], bf16, a.dv, a.B, a.Sk, a.Hkv, a.D) || !attn_store_map(&p.out[1], bf16, a.dk, a.B, a.Sk, a.Hkv, a.D))
        return DAF_ERR_CUDA;
    const auto items = [&](uint32_t S, uint32_t H) {
        p.tiles = (S + kHeld - 1u) / kHeld;
        p.items = p.tiles * a.B * H;
        p.heads.set(H);
        p.all_heads.set(a.B * H);
        p.tile_div.set(p.tiles);
    };
    p.x1 = k; p.x2 = v; p.y1 = q; p.y2 = g;
    items(a.Sk, a.Hkv);
    daf_status st = a.D <= 64u ? launch_grad<T, 64, true>(p, s) : launch_grad<T, 128, true>(p, s);
    if (st != DAF_OK) return st;
    p.x1 = q; p.x2 = g; p.y1 = k; p.y2 = v;
    if (!attn_store_map(&p.out[0], bf16, a.dq, a.B, a.Sq, a.H, a.D)) return DAF_ERR_CUDA;
    items(a.Sq, a.H);
    st = a.D <= 64u ? launch_grad<T, 64, false>(p, s) : launch_grad<T, 128, false>(p, s);
    return st;
}

}  // namespace daf
