// Attention for binary32 inputs on the tensor cores, forward and backward.
//
// A binary32 number is the sum of three bfloat16 numbers, x = h + m + l (8 bits each, rounded to nearest one after the
// other: exact), and a product of two is h h' + (h m' + m h') + (m m' + h l' + l h') up to 2^-24: six bfloat16 products,
// whose binary32 accumulator takes the small ones first.  split_planes_kernel writes the planes of the inputs once; P and dS
// are split in registers on their way into tensor memory.  The accumulator of the tensor cores truncates, so it only ever
// holds one block of the walk: the running sums stay in registers, added there to nearest.
//
// Six products at the rate of bfloat16 leave a sixth of 1.6 PFLOP/s; a loop of binary32 multiply-adds, four by four scores
// to a thread, reached 25 TFLOP/s, and three TF32 products by mma.sync 30, with 22 bits of each factor.
//
//   FWD   holds 128 queries, walks 64 keys a block:     T1 = q k^T;                 sum += P v
//   DQ    holds 128 queries, walks 64 keys a block:     T1 = q k^T, T2 = g v^T;     sum += dS k
//   DKV   holds 128 keys, walks 32 queries a block:     T1 = k q^T, T2 = v g^T;     dv += P g, dk += dS q
// Backward, heads above 64 leave room for blocks of 16 only: the planes of the two held tiles take 192 KiB.
//
// A persistent CTA (one per SM): warps 0-7 softmax (two threads to a row), warp 8 the products, warp 9 the copies.  Tensor
// memory: two blocks of T, the planes of P and dS, one block's sums.
#include "attention_tc_grad.cuh"

namespace daf {

constexpr int kPlaneThreads = 384;               // 8 warps x 232 registers, 4 (two of them idle) x 40
enum { kFwd = 0, kDq = 1, kDkv = 2 };

template <int MODE, int DP> struct PlaneShape {
    static constexpr uint32_t WALK = MODE != kFwd && DP == 128 ? 16 : MODE == kDkv ? 32 : 64;
    static constexpr uint32_t kHeldTiles = MODE == kFwd ? 1 : 2;
    static constexpr uint32_t kX = 3u * kHeld * DP * 2u, kY = 3u * WALK * DP * 2u;   // a tensor's tile, three planes
    static constexpr uint32_t kSlots = DP == 128 ? 2 : MODE == kFwd ? 6 : MODE == kDq ? 4 : 8;
    static constexpr uint32_t kStats = MODE == kDkv ? 2u * WALK * 4u : 0u;           // for each pair of slots
    static constexpr uint32_t kT = WALK * kHeldTiles;              // tensor memory: columns of a block of T,
    static constexpr uint32_t kW = 3u * WALK / 2u * (MODE == kDkv ? 2 : 1);          // of the planes,
    static constexpr uint32_t kSum = MODE == kDkv ? 2u * DP : DP;                    // of the sums
    static constexpr uint32_t kAtW = 2u * kT, kAtSum = (kAtW + kW + 31u) & ~31u;
    static constexpr uint32_t kBars = 1024u;
    static constexpr uint32_t kBytes = kBars + kHeldTiles * kX + kSlots * kY + kSlots / 2u * kStats + 2u * 8u * 32u * 4u;
    static_assert(kAtSum + kSum <= 512u && kBytes <= 232448u, "fits the SM");
};

// x = h + m + l for two values at once, each plane's pair in one word
__device__ __forceinline__ void split3(float u, float v, uint32_t &h, uint32_t &m, uint32_t &l)
{
    h = round2<__nv_bfloat16>(u, v);
    u -= __uint_as_float(h << 16);
    v -= __uint_as_float(h & 0xFFFF0000u);
    m = round2<__nv_bfloat16>(u, v);
    u -= __uint_as_float(m << 16);
    v -= __uint_as_float(m & 0xFFFF0000u);
    l = round2<__nv_bfloat16>(u, v);
}

// The six products of planes (h 0, m 1, l 2), small ones first: m m, h l, l h, h m, m h, h h.
__device__ __forceinline__ uint32_t left_plane(uint32_t c) { return 0x010201u >> (4u * c) & 3u; }
__device__ __forceinline__ uint32_t right_plane(uint32_t c) { return 0x001021u >> (4u * c) & 3u; }

struct SplitTensor {
    AttnTensor from;
    __nv_bfloat16 *to;                           // [B, S, H, 3, D]
    uint32_t S, H, keys;                         // keys: a row is one of k or v, not of q or grad_out
    uint32_t rows;                               // B S H
};
struct SplitArgs {
    SplitTensor t[4];
    AttnArgs a;
    uint32_t pieces;                             // D / 8
    WorkspaceHeader *header;
};
__global__ void __launch_bounds__(256) split_planes_kernel(const __grid_constant__ SplitArgs p)
{
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && p.header) p.header->status = 0u;
    const SplitTensor &t = p.t[blockIdx.y];
    const uint32_t lanes = 256u / p.pieces, d = threadIdx.x % p.pieces, first = threadIdx.x / p.pieces;
    if (first >= lanes) return;
    for (uint32_t r = blockIdx.x * lanes + first; r < t.rows; r += gridDim.x * lanes) {
        const uint32_t bs = r / t.H, h = r - bs * t.H, b = bs / t.S, s = bs - b * t.S;
        uint4 out[3] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
        const uint32_t n = attn_length(p.a, b);
        if (t.keys ? s < n : attn_limit(p.a, n, (int)s) > 0) {      // what nobody sees, and what sees nothing, becomes zero
            const float4 *src = reinterpret_cast<const float4 *>(reinterpret_cast<const float *>(t.from.p) + t.from.sb * b + t.from.ss * s + t.from.sh * h + d * 8u);
            const float4 x = __ldg(src), y = __ldg(src + 1);
            split3(x.x, x.y, out[0].x, out[1].x, out[2].x);
            split3(x.z, x.w, out[0].y, out[1].y, out[2].y);
            split3(y.x, y.y, out[0].z, out[1].z, out[2].z);
            split3(y.z, y.w, out[0].w, out[1].w, out[2].w);
        }
        uint4 *const dst = reinterpret_cast<uint4 *>(t.to) + (uint64_t)r * 3u * p.pieces + d;
#pragma unroll
        for (int k = 0; k < 3; k++) dst[k * p.pieces] = out[k];
    }
}

template <int MODE, int DP>
__global__ void __launch_bounds__(kPlaneThreads, 1) attention_planes_kernel(const __grid_constant__ AttnGradArgs p)
{
    using Shape = PlaneShape<MODE, DP>;
    constexpr bool DKV = MODE == kDkv, FWD = MODE == kFwd;
    constexpr uint32_t WALK = Shape::WALK, SLOTS = Shape::kSlots, PLANE = WALK / 2u;   // columns of a plane
    constexpr uint32_t HALF = WALK == 16 ? 16 : WALK / 2u;         // columns of a thread (of 16, the first of a row's two has all)
    constexpr bool EARLY = FWD && SLOTS == 2u;
    constexpr uint32_t XBOX = kHeld * 128u, YBOX = WALK * 128u, XP = Shape::kX / 3u, YP = Shape::kY / 3u;
    extern __shared__ __align__(1024) unsigned char s_raw[];
    struct Bars {
        uint64_t y_full[8], y_empty[8], t_full[2], x_full, x_empty, w_ready, sum_full, drain;
        uint32_t tmem, abort, left[8];
    };
    static_assert(sizeof(Bars) <= Shape::kBars && SLOTS <= 8, "barriers fit their places");
    Bars &bars = *reinterpret_cast<Bars *>(s_raw);
    if (smem_u32(s_raw) & 1023u) {                                 // the same for every thread
        if (threadIdx.x == 0) record_error(p.header, p.a.device_status, DAF_ERR_UNSUPPORTED);
        return;
    }
    unsigned char *const s_x = s_raw + Shape::kBars, *const s_y = s_x + Shape::kHeldTiles * Shape::kX;
    float *const s_stats = reinterpret_cast<float *>(s_y + SLOTS * Shape::kY);
    float (*const s_told)[32] = reinterpret_cast<float (*)[32]>(s_y + SLOTS * Shape::kY + SLOTS / 2u * Shape::kStats);
    const AttnArgs &a = p.a;
    const uint32_t warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
    if (threadIdx.x < 8) bars.left[threadIdx.x] = 0u;
    if (threadIdx.x == 0) {
        bars.abort = 0u;
        for (uint32_t i = 0; i < SLOTS; i++) {
            bar_init(&bars.y_full[i], 1);
            bar_init(&bars.y_empty[i], 1);
        }
        bar_init(&bars.t_full[0], 1);
        bar_init(&bars.t_full[1], 1);
        bar_init(&bars.x_full, 1);
        bar_init(&bars.x_empty, 1);
        bar_init(&bars.w_ready, 8);
        bar_init(&bars.sum_full, 1);
        bar_init(&bars.drain, 1);
        fence_async();
    }
    if (warp == 0) tmem_alloc(&bars.tmem, 512);
    tmem_before_sync();
    __syncthreads();
    tmem_after_sync();
    const uint32_t tmem = bars.tmem;
    volatile uint32_t *const stop = &bars.abort;

    if (warp < 8) {                                                // ---- probabilities, score gradients, sums
        take_registers<232>();
        const uint32_t part = warp >> 2, quarter = (warp & 3u) << 21, lane_row = (warp & 3u) * 32u + lane;
        WarpPair pair_of;                                           // the two warps of a row (they only meet forward)
        pair_of.init(bars.left, 1u + (warp & 3u), warp ^ 4u);
        // What the other warp of the rows says to this one's value.  Two places in turn: T of the next block may be there before
        // the other warp has read, but who writes for exchange n + 2 has met, at n + 1, the warp that has read n.
        uint32_t told = 0;
        const auto exchange = [&](float value, float &others) {
            float (*const at)[32] = s_told + told;
            told ^= 8u;
            at[warp][lane] = value;
            if (!pair_of.meet()) return false;
            others = at[warp ^ 4u][lane];
            return true;
        };
        const int off = (int)a.Sk - (int)a.Sq;
        uint32_t buf = 0, t_ph = 0, sum_ph = 0, slot = 0, y_ph = 0;
        bool ok = true;
        GradItem<DKV, WALK> it;
        for (uint32_t turn = 0; ok && turn * gridDim.x < p.items; turn++) {
            const uint32_t item = grad_item(turn);
            if (item >= p.items) continue;
            it.set(p, item);
            const uint32_t row = it.first + lane_row, live = DKV ? it.n : a.Sq;
            const bool idle = it.first + (warp & 3u) * 32u >= live;
            const int limit = DKV ? 0 : row < a.Sq ? attn_limit(a, it.n, (int)row) : (int)it.n;
            float nl = 0.0f, nd = 0.0f, m = -INFINITY, l = 0.0f;
            if (MODE == kDq && it.blocks) {
                const uint64_t at = ((uint64_t)it.b * a.H + it.h) * a.rows_padded + row;
                nl = a.row_nl2[at];
                nd = a.row_ndelta[at];
            }
            constexpr int N = (int)Shape::kSum / 2;                // this thread's sums: DKV 32 of dv, 32 of dk, else half a row
            float sum[N];
#pragma unroll
            for (int i = 0; i < N; i++) sum[i] = 0.0f;
            // adds what the last block's products left in tensor memory, then fades the sums to a new maximum
            const auto fold = [&](float fade) {
                if (!bar_wait(&bars.sum_full, sum_ph, stop)) return false;
                sum_ph ^= 1u;
                if (idle) return true;
                tmem_after_sync();
#pragma unroll
                for (int c = 0; c < N / 32; c++) {
                    float x[32];
                    // dv in the first DP columns, dk in the next; half of each
                    constexpr int PER = DP / 64;                   // pieces of 32 of a tensor's half row
                    tmem_load32(tmem + Shape::kAtSum + quarter + (uint32_t)(c / PER) * DP + part * (DP / 2) + 32u * (c % PER), x);
                    tmem_wait_loads();
#pragma unroll
                    for (int k = 0; k < 32; k++) sum[32 * c + k] = FWD ? (sum[32 * c + k] + x[k]) * fade : sum[32 * c + k] + x[k];
                }
                return true;
            };
            uint32_t at = it.start, in_head = 0;
            for (uint32_t i = 0; i < it.blocks; i++) {
                if (!(ok = bar_wait(&bars.t_full[buf], t_ph, stop))) break;
                if (DKV && !(ok = bar_wait(&bars.y_full[slot + 1u], y_ph, stop))) break;   // the statistics came by copy
                // columns with values, at least
                const int cols = WALK == 16 && part ? 0 : (int)((DKV ? a.Sq : it.n) - at) - (int)(HALF * part);
                float s[HALF], e[HALF];
                float fade = 1.0f;
                if (!idle) {
                    tmem_after_sync();
                    const uint32_t t = tmem + buf * Shape::kT + part * HALF + quarter;
                    if (cols > 0) {
                        if (HALF == 32) {
                            tmem_load32(t, s);
                            if (!FWD) tmem_load32(t + WALK, e);
                        } else {
                            tmem_load16(t, s);
                            tmem_load16(t + WALK, e);
                        }
                        tmem_wait_loads();
                    }
                    // of these columns the row sees [lo, hi)
                    int lo = 0, hi = HALF;
                    if (DKV) lo = row >= it.n ? (int)HALF : a.causal ? (int)row - off - (int)at - (int)(HALF * part) : 0;
                    else hi = limit - (int)at - (int)(HALF * part);
                    const bool masked = __any_sync(0xffffffffu, lo > 0 || hi < (int)HALF);
                    if (FWD) {
                        float top = -INFINITY;
                        if (cols > 0) {
#pragma unroll
                            for (int k = 0; k < (int)HALF; k++) {
                                s[k] *= a.scale_log2;
                                if (masked && k >= hi) s[k] = -INFINITY;
                                top = fmaxf(top, s[k]);
                            }
                        }
                        float others = 0.0f;
                        if (!(ok = exchange(top, others))) break;
                        const float next = fmaxf(m, fmaxf(top, others)), base = next == -INFINITY ? 0.0f : next;
                        fade = exp2_fast(m - base);
                        m = next;
                        float total = 0.0f;
                        if (cols > 0) {
#pragma unroll
                            for (int k = 0; k < (int)HALF; k++) total += s[k] = exp2_fast(s[k] - base);
                        }
                        l = __fmaf_rn(l, fade, total);
                    } else if (cols > 0) {
                        const float *const st = s_stats + (slot >> 1) * 2u * WALK + HALF * part;
#pragma unroll
                        for (int k = 0; k < (int)HALF; k++) {
                            const float pr = exp2_fast(__fmaf_rn(s[k], a.scale_log2, DKV ? st[k] : nl)), ds = pr * (e[k] + (DKV ? st[WALK + k] : nd));
                            const bool see = !masked || (k >= lo && k < hi);         // selected: what is masked may be NaN
                            s[k] = see ? pr : 0.0f;
                            e[k] = see ? ds : 0.0f;
                        }
                    }
                }
                // the planes and the sums of the last block are the tensor cores' until its products are done
                if (i > 0 && !(ok = fold(fade))) break;
                if (!idle && cols > 0) {
#pragma unroll
                    for (int k = 0; k < (int)HALF / 16; k++) {
                        uint32_t h[8], mid[8], low_[8];
                        const uint32_t to = tmem + Shape::kAtW + quarter + part * (HALF / 2u) + 8u * k;
                        if (MODE != kDq) {
#pragma unroll
                            for (int c = 0; c < 8; c++) split3(s[16 * k + 2 * c], s[16 * k + 2 * c + 1], h[c], mid[c], low_[c]);
                            tmem_store8(to, h);
                            tmem_store8(to + PLANE, mid);
                            tmem_store8(to + 2u * PLANE, low_);
                        }
                        if (!FWD) {
#pragma unroll
                            for (int c = 0; c < 8; c++) split3(e[16 * k + 2 * c], e[16 * k + 2 * c + 1], h[c], mid[c], low_[c]);
                            const uint32_t ds = to + (DKV ? 3u * PLANE : 0u);
                            tmem_store8(ds, h);
                            tmem_store8(ds + PLANE, mid);
                            tmem_store8(ds + 2u * PLANE, low_);
                        }
                    }
                    tmem_wait_stores();
                }
                tmem_before_sync();
                __syncwarp();
                if (lane == 0) bar_arrive(&bars.w_ready);
                if ((buf ^= 1u) == 0) t_ph ^= 1u;
                if ((slot += 2u) == SLOTS) {
                    slot = 0;
                    y_ph ^= 1u;
                }
                at += WALK;
                if (DKV && ++in_head == it.per_head) {
                    in_head = 0;
                    at = it.start;
                }
            }
            if (!ok) break;
            if (it.blocks && !(ok = fold(1.0f))) break;
            tmem_before_sync();
            if (FWD && !idle) {
                float others = 0.0f;
                if (!(ok = exchange(l, others))) break;
                l += others;
                if (part == 0 && row < a.Sq)
                    a.lse[((uint64_t)it.b * a.H + it.h) * a.Sq + row] = limit > 0 ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
            }
            const uint32_t rows = DKV ? a.Sk : a.Sq;
            // what a row sees is told by the mask: forward, a sum that is NaN, or zero of scores that are all -inf, makes NaN
            const bool keep = it.blocks && row < live && (DKV || limit > 0);
            const float by = FWD ? __fdiv_rn(1.0f, l) : a.scale;
#pragma unroll
            for (int c = 0; c < N / 32; c++) {
                constexpr int PER = DP / 64;
                const AttnTensor &to = FWD ? a.out : !DKV ? a.dq : c / PER ? a.dk : a.dv;
                const float times = DKV && c / PER == 0 ? 1.0f : by;
                const uint32_t d0 = part * (DP / 2) + 32u * (c % PER);
                float *const dst = reinterpret_cast<float *>(to.p) + to.sb * it.b + to.sh * it.h + to.ss * row + d0;
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (row < rows && d0 + 4u * k < a.D)
                        reinterpret_cast<float4 *>(dst)[k] = keep ? make_float4(sum[32 * c + 4 * k] * times, sum[32 * c + 4 * k + 1] * times,
                                                                                sum[32 * c + 4 * k + 2] * times, sum[32 * c + 4 * k + 3] * times)
                                                                  : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            }
        }
        if (FWD && !ok) pair_of.give_up(warp, lane, &s_told[warp][lane]);
    } else {
        leave_registers<40>();
        if (warp == 9) {                                           // ---- copies
            GradCursor<DKV, WALK> cur;
            uint32_t slot = 0, ph = 1, x_ph = 1;
            const bool one = lane == 0;
            bool ok = true;
            for (cur.open(p); ok && cur.more; cur.step(p)) {
                if (cur.i == 0) {
                    if (!bar_wait(&bars.x_empty, x_ph, stop)) break;
                    x_ph ^= 1u;
                    if (one) {
                        bar_expect(&bars.x_full, Shape::kHeldTiles * Shape::kX);
                        for (uint32_t t = 0; t < Shape::kHeldTiles; t++)
                            for (uint32_t k = 0; k < 3; k++)
                                for (uint32_t e = 0; e < DP / 64; e++)
                                    tma_load(smem_u32(s_x) + t * Shape::kX + k * XP + e * XBOX, t ? &p.x2 : &p.x1, &bars.x_full, 64 * e, 3 * cur.it.h + k, cur.it.first, cur.it.b);
                    }
                }
                for (uint32_t t = 0; t < 2; t++) {
                    if (!(ok = bar_wait(&bars.y_empty[slot + t], ph, stop))) break;
                    if (one) {
                        uint64_t *const bar = &bars.y_full[slot + t];
                        bar_expect(bar, Shape::kY + (t ? Shape::kStats : 0u));
                        for (uint32_t k = 0; k < 3; k++)
                            for (uint32_t e = 0; e < DP / 64; e++)
                                tma_load(smem_u32(s_y) + (slot + t) * Shape::kY + k * YP + e * YBOX, t ? &p.y2 : &p.y1, bar, 64 * e, 3 * cur.head + k, cur.row, cur.it.b);
                        if (DKV && t) {
                            const uint64_t at = ((uint64_t)cur.it.b * a.H + cur.head) * a.rows_padded + cur.row;
                            const uint32_t dst = smem_u32(s_stats + (slot >> 1) * 2u * WALK);
                            bulk_load(dst, a.row_nl2 + at, WALK * 4u, bar);
                            bulk_load(dst + WALK * 4u, a.row_ndelta + at, WALK * 4u, bar);
                        }
                    }
                }
                if ((slot += 2u) == SLOTS) {
                    slot = 0;
                    ph ^= 1u;
                }
            }
            if (*stop) {                                           // giving up: let the copies in flight land first
                const uint64_t until = now_ns() + 1000000000ull;
                while (now_ns() < until) __nanosleep(1000);
            }
        } else if (warp == 8) {                                    // ---- products
            const uint32_t one = elect_lane();
            const uint32_t steps = (a.D + 15u) / 16u, sum_desc = product_desc(true, steps * 16u, true);
            const uint32_t xs = smem_u32(s_x), ys = smem_u32(s_y);
            GradCursor<DKV, WALK> ahead, cur;
            ahead.open(p);
            cur.open(p);
            uint32_t t_slot = 0, t_phase = 0, t_buf = 0, x_ph = 0, c_slot = 0, w_ph = 0;
            bool ok = true;
            // T1 and T2 of the block `ahead` stands at
            auto scores = [&]() {
                if (!ahead.more) return;
                if (ahead.i == 0 && !(ok = bar_wait(&bars.x_full, x_ph, stop))) return;
                const uint32_t desc = product_desc(true, (ahead.cols(p) + 15u) & ~15u, false);
#pragma unroll 1
                for (uint32_t k = 0; k < Shape::kHeldTiles; k++) {
                    if (!(ok = bar_wait(&bars.y_full[t_slot + k], t_phase, stop))) return;
                    tmem_after_sync();
#pragma unroll 1
                    for (uint32_t c = 0; c < 6; c++) {
                        const uint32_t A = operand_low(xs + k * Shape::kX + left_plane(c) * XP, 16);
                        const uint32_t B = operand_low(ys + (t_slot + k) * Shape::kY + right_plane(c) * YP, 16);
#pragma unroll
                        for (uint32_t s = 0; s < DP / 16; s++)
                            if (s < steps)
                                product_ss(one, tmem + t_buf * Shape::kT + k * WALK, A + ((s & 3u) * 2u + (s >> 2) * (XBOX / 16u)), B + ((s & 3u) * 2u + (s >> 2) * (YBOX / 16u)), desc, c > 0 || s > 0);
                    }
                }
                products_done(one, &bars.t_full[t_buf]);
                if (FWD) products_done(one, &bars.y_empty[t_slot]);            // the keys are done with
                t_buf ^= 1u;
                if (ahead.last()) {
                    products_done(one, &bars.x_empty);
                    x_ph ^= 1u;
                }
                if ((t_slot += 2u) == SLOTS) {
                    t_slot = 0;
                    t_phase ^= 1u;
                }
                ahead.step(p);
            };
            // one block's sum of the three planes at `w` and a walked tile
            auto sums = [&](uint32_t to, uint32_t w, uint32_t tile, uint32_t n16) {
#pragma unroll 1
                for (uint32_t c = 0; c < 6; c++) {
                    const uint32_t B = operand_low(tile + right_plane(c) * YP, YBOX);
#pragma unroll
                    for (uint32_t s = 0; s < WALK / 16; s++)
                        if (s < n16) product_ts(one, to, w + left_plane(c) * PLANE + s * 8u, B + s * 128u, sum_desc, c > 0 || s > 0);
                }
            };
            uint32_t c_phase = 0;
            scores();
            // with one pair of slots the next block's copies wait for this block's products: all of them, or, forward, T's
            if (ok && SLOTS > 2u) scores();
            for (; ok && cur.more; cur.step(p)) {
                const uint32_t n16 = (cur.cols(p) + 15u) / 16u, y1 = ys + c_slot * Shape::kY, y2 = y1 + Shape::kY, w = tmem + Shape::kAtW, to = tmem + Shape::kAtSum;
                if (EARLY) scores();
                if (!ok || !bar_wait(&bars.w_ready, w_ph, stop)) break;
                w_ph ^= 1u;
                if (FWD && !bar_wait(&bars.y_full[c_slot + 1u], c_phase, stop)) break;
                tmem_after_sync();
                if (MODE != kDq) sums(to, w, y2, n16);
                if (MODE != kFwd) sums(to + (DKV ? DP : 0), w + (DKV ? 3u * PLANE : 0u), y1, n16);
                products_done(one, &bars.sum_full);
                if (!FWD) products_done(one, &bars.y_empty[c_slot]);
                products_done(one, &bars.y_empty[c_slot + 1u]);
                if ((c_slot += 2u) == SLOTS) {
                    c_slot = 0;
                    c_phase ^= 1u;
                }
                if (!EARLY) scores();
            }
            products_done(one, &bars.drain);
            bar_wait(&bars.drain, 0, stop);
        }
    }
    tmem_before_sync();
    __syncthreads();
    if (threadIdx.x == 0 && bars.abort) record_error(p.header, p.a.device_status, DAF_ERR_TIMEOUT);
    if (warp == 0) tmem_free(tmem, 512);
}

template <int MODE, int DP> static daf_status launch_planes(const AttnGradArgs &p, cudaStream_t s)
{
    int ctas = 0;
    const auto kernel = &attention_planes_kernel<MODE, DP>;
    if (persistent_ctas(reinterpret_cast<const void *>(kernel), kPlaneThreads, (int)PlaneShape<MODE, DP>::kBytes, &ctas) != cudaSuccess) return DAF_ERR_CUDA;
    kernel<<<p.items < (uint32_t)ctas ? p.items : (uint32_t)ctas, kPlaneThreads, PlaneShape<MODE, DP>::kBytes, s>>>(p);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

// Bytes of the planes of B S H rows of D elements.
static uint64_t planes_bytes(uint64_t B, uint64_t S, uint64_t H, uint64_t D) { return (B * S * H * D * 6u + 255u) & ~255ull; }

// q, k, v and (backward) grad_out in three planes each, from `at` on; the planes as tensors of 3 H heads
static daf_status split_all(const AttnArgs &a, char *at, bool with_grad, WorkspaceHeader *header, AttnTensor (&planes)[4], cudaStream_t s)
{
    SplitArgs p = {};
    p.a = a;
    p.pieces = a.D / 8u;
    p.header = header;
    const AttnTensor from[4] = {a.q, a.k, a.v, a.grad_out};
    uint32_t most = 0;
    for (int i = 0; i < (with_grad ? 4 : 3); i++) {
        const bool keys = i == 1 || i == 2;
        const uint32_t S = keys ? a.Sk : a.Sq, H = keys ? a.Hkv : a.H;
        p.t[i] = {from[i], reinterpret_cast<__nv_bfloat16 *>(at), S, H, keys, a.B * S * H};
        planes[i] = {at, 3ull * S * H * a.D, 3ull * H * a.D, a.D};
        at += planes_bytes(a.B, S, H, a.D);
        most = p.t[i].rows > most ? p.t[i].rows : most;
    }
    const uint32_t lanes = 256u / p.pieces, grid = (most + lanes - 1u) / lanes;
    split_planes_kernel<<<dim3(grid < 8192u ? (grid ? grid : 1u) : 8192u, with_grad ? 4 : 3), 256, 0, s>>>(p);
    return cudaGetLastError() == cudaSuccess ? DAF_OK : DAF_ERR_CUDA;
}

static bool set_items(AttnGradArgs &p, const AttnTensor &x1, const AttnTensor &x2, uint32_t Sx, uint32_t Hx, const AttnTensor &y1, const AttnTensor &y2,
                      uint32_t Sy, uint32_t Hy, uint32_t walk)
{
    const AttnArgs &a = p.a;
    p.tiles = (Sx + kHeld - 1u) / kHeld;
    p.items = p.tiles * a.B * Hx;
    p.heads.set(Hx);
    p.all_heads.set(a.B * Hx);
    p.tile_div.set(p.tiles);
    return attn_tensor_map(&p.x1, true, x1, a.B, Sx, 3u * Hx, a.D, kHeld) && attn_tensor_map(&p.x2, true, x2, a.B, Sx, 3u * Hx, a.D, kHeld) &&
           attn_tensor_map(&p.y1, true, y1, a.B, Sy, 3u * Hy, a.D, walk) && attn_tensor_map(&p.y2, true, y2, a.B, Sy, 3u * Hy, a.D, walk);
}

uint64_t attn_planes_workspace(const AttnArgs &a, bool backward)
{
    return (backward ? 2u : 1u) * planes_bytes(a.B, a.Sq, a.H, a.D) + 2u * planes_bytes(a.B, a.Sk, a.Hkv, a.D);
}

// Queries exist; without keys the planes of k and v are empty and their maps stand on q's, never read.
daf_status attn_forward_planes(const AttnArgs &a, char *planes_at, WorkspaceHeader *header, cudaStream_t s)
{
    AttnTensor t[4];
    daf_status st = split_all(a, planes_at, false, header, t, s);
    if (st != DAF_OK) return st;
    AttnGradArgs p = {};
    p.a = a;
    p.header = header;
    const bool keys = a.Sk > 0;
    if (!set_items(p, t[0], t[0], a.Sq, a.H, keys ? t[1] : t[0], keys ? t[2] : t[0], keys ? a.Sk : a.Sq, keys ? a.Hkv : a.H, 64)) return DAF_ERR_CUDA;
    return a.D <= 64u ? launch_planes<kFwd, 64>(p, s) : launch_planes<kFwd, 128>(p, s);
}

template <int DP> static daf_status backward(AttnGradArgs &p, const AttnTensor (&t)[4], cudaStream_t s)
{
    const AttnArgs &a = p.a;
    if (!set_items(p, t[1], t[2], a.Sk, a.Hkv, t[0], t[3], a.Sq, a.H, PlaneShape<kDkv, DP>::WALK)) return DAF_ERR_CUDA;
    const daf_status st = launch_planes<kDkv, DP>(p, s);
    if (st != DAF_OK) return st;
    if (!set_items(p, t[0], t[3], a.Sq, a.H, t[1], t[2], a.Sk, a.Hkv, PlaneShape<kDq, DP>::WALK)) return DAF_ERR_CUDA;
    return launch_planes<kDq, DP>(p, s);
}

// Queries and keys exist.
daf_status attn_backward_planes(const AttnArgs &a, char *planes_at, WorkspaceHeader *header, cudaStream_t s)
{
    AttnTensor t[4];
    const daf_status st = split_all(a, planes_at, true, nullptr, t, s);
    if (st != DAF_OK) return st;
    AttnGradArgs p = {};
    p.a = a;
    p.header = header;
    return a.D <= 64u ? backward<64>(p, t, s) : backward<128>(p, t, s);
}

}  // namespace daf
