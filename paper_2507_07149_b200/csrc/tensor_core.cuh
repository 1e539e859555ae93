// The sm_100a instructions the tensor-core kernels are built from: tensor memory, tcgen05 products, tiled copies into
// shared memory, and barriers whose waits end.
#pragma once
#include <cuda.h>

#include "common.cuh"
#include "pairs.cuh"

namespace daf {

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---------------------------------------------------------------------------------------------
// Barriers.  Every wait ends: after two seconds (real time) the waiting thread raises the CTA's abort flag, which every
// other wait of the CTA looks at between polls; all roles then leave their loops.
// ---------------------------------------------------------------------------------------------
constexpr uint64_t kWaitNanoseconds = 2000000000ull;

__device__ __forceinline__ void bar_init(uint64_t *bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ bool bar_try(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// True when the phase of that parity is complete; false when the CTA gives up.
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, volatile uint32_t *abort_flag)
{
    if (bar_try(bar, parity)) return true;
    const uint64_t start = now_ns();
    while (!bar_try(bar, parity)) {
        if (*abort_flag) return false;
        if (now_ns() - start > kWaitNanoseconds) {
            *abort_flag = 1u;
            return false;
        }
    }
    return true;
}

// Two warps that share rows and meet to exchange a number per row.  Either may find in a wait of its own that the CTA gives
// up, while the other one comes to their next meeting; that must not wait for good.  So a warp that gives up (and only such a
// one: the other may not have looked behind the last meeting yet) says so and arrives once more without waiting, and a meeting
// that ended by such an arrival is the other warp's last.  left: a flag of each warp, cleared ahead of the first meeting.  A
// warp that gives up also puts NaN in the place of its numbers: where those are never NaN themselves, their reader needs no
// second look (8192 causal tokens, 16 heads of 128: the flag read behind every block's meeting costs 326 us against 315).
struct WarpPair {
    uint32_t barrier, other;
    volatile uint32_t *left;
    bool alone;
    __device__ __forceinline__ void init(volatile uint32_t *flags, uint32_t id, uint32_t other_warp)
    {
        left = flags;
        barrier = id;
        other = other_warp;
        alone = false;
    }
    // behind it, `gone` looks at the number that was read
    __device__ __forceinline__ void meet_unseen() const { asm volatile("bar.sync %0, 64;" ::"r"(barrier) : "memory"); }
    __device__ __forceinline__ bool gone(float read) { return alone = __any_sync(0xffffffffu, read != read); }
    // false: the other warp is gone, and what it last wrote is not what was asked for
    __device__ __forceinline__ bool meet()
    {
        meet_unseen();
        alone = left[other] != 0u;
        return !alone;
    }
    __device__ __forceinline__ void give_up(uint32_t warp, uint32_t lane, float *place)
    {
        if (alone) return;
        *place = __uint_as_float(0x7FC00000u);
        if (lane == 0) left[warp] = 1u;
        __syncwarp();
        asm volatile("bar.arrive %0, 64;" ::"r"(barrier) : "memory");
    }
};

// ---------------------------------------------------------------------------------------------
// Copies.  A tile is loaded as boxes of 64 16-bit elements (128 bytes, the swizzle's span) times some rows.
// Coordinates: element (a multiple of 64), head, row, batch.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int elem, int head, int row, int batch)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(elem), "r"(head), "r"(row), "r"(batch) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// The way out for a warp's 32 rows: 32 columns at a time through 2 KiB of shared memory and a tiled store, which clips rows
// and columns behind the tensor's ends.  (Stored by the threads, each its own row, a warp's store touches 32 lines for 512
// bytes: a third of the time of short sequences.)  The pieces of a row lie where a 64-byte swizzle wants them.
__device__ __forceinline__ void stage_piece(unsigned char *stage, uint32_t row, uint32_t piece, uint4 v)
{
    *reinterpret_cast<uint4 *>(stage + row * 64u + ((piece ^ (row >> 1 & 3u)) * 16u)) = v;
}
__device__ __forceinline__ void tma_store(const CUtensorMap *map, const unsigned char *stage, int elem, int head, int row, int batch)
{
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(map), "r"(smem_u32(stage)), "r"(elem), "r"(head), "r"(row), "r"(batch) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// At most N of this thread's stores still read shared memory.
template <int N> __device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Orders this thread's writes to shared memory ahead of later reads by copies and products.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---------------------------------------------------------------------------------------------
// Tensor memory and products
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t *slot, uint32_t columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 or 16 columns of the thread's lane (the warp's quarter of the 128 lanes is part of `at`: lane in bits 31-16).
__device__ __forceinline__ void tmem_load32(uint32_t at, float *x)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(x);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
                   "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_load16(uint32_t at, float *x)
{
    uint32_t *r = reinterpret_cast<uint32_t *>(x);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
                 "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at) : "memory");
}

// Operand descriptor of a tile in shared memory with 128-byte swizzle.  Low word: the address and the distance `lead`
// between 64-element spans of the contiguous dimension (used where that dimension is not the summed one); high word, the
// same for all: 1024 bytes between groups of eight rows.  Steps along a tile are added to the low word (16-byte units).
constexpr uint32_t kOperandHigh = 1024u >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t operand_low(uint32_t smem, uint32_t lead) { return (smem >> 4 & 0x3FFFu) | lead >> 4 << 16; }
// Instruction descriptor: 16-bit operands (both of one type), binary32 accumulator, M = 128.  across: operand B's contiguous
// dimension is N and not the summed one.
__device__ __forceinline__ uint32_t product_desc(bool bf16, uint32_t n, bool across)
{
    const uint32_t t = bf16 ? 1u : 0u;
    return 1u << 4 | t << 7 | t << 10 | (across ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(at) : "memory");
}

// One lane of the (whole, converged) warp.  The products are issued by that lane under a predicate while the warp computes
// their operands together: those then stay in uniform registers, which the instructions take; inside a branch of one lane
// every operand would be moved there for each product.
__device__ __forceinline__ uint32_t elect_lane()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r;
}
template <bool ADD_ALWAYS = false>
__device__ __forceinline__ void product_ss(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add = true)
{
    if (ADD_ALWAYS)
        asm volatile("{\n\t.reg .pred q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 q, %4, 0;\n\tmov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                     "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, 1;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(one), "n"(kOperandHigh) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 q, %4, 0;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 da, {%1, %5};\n\t"
                     "mov.b64 db, {%2, %5};\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(one), "n"(kOperandHigh), "r"((uint32_t)add) : "memory");
}
template <bool ADD_ALWAYS = false>
__device__ __forceinline__ void product_ts(uint32_t one, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add = true)
{
    if (ADD_ALWAYS)
        asm volatile("{\n\t.reg .pred q;\n\t.reg .b64 db;\n\tsetp.ne.b32 q, %4, 0;\n\tmov.b64 db, {%2, %5};\n\t"
                     "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, 1;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(one), "n"(kOperandHigh) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\tsetp.ne.b32 q, %4, 0;\n\tsetp.ne.b32 p, %6, 0;\n\tmov.b64 db, {%2, %5};\n\t"
                     "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(one), "n"(kOperandHigh), "r"((uint32_t)add) : "memory");
}
// The barrier is arrived at when every product issued so far by this lane is done.
__device__ __forceinline__ void products_done(uint32_t one, uint64_t *bar)
{
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(bar)), "r"(one) : "memory");
}

// A warpgroup's share of the registers the CTA was launched with (its shares must not add up to more).
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void leave_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ---------------------------------------------------------------------------------------------
// The exponential, and rounding to operands
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Two values rounded to nearest even into one word, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t round2(float a, float b);
template <> __device__ __forceinline__ uint32_t round2<__half>(float a, float b)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <> __device__ __forceinline__ uint32_t round2<__nv_bfloat16>(float a, float b)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

}  // namespace daf
