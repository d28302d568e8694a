// The sm_100a instructions behind the attention kernels: mbarriers, TMA tile loads, tensor memory and
// tcgen05.mma with one issuing thread.  16-bit operands, binary32 accumulators.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "fewbit_packed.cuh"

namespace fewbit {
namespace tc {

__device__ __forceinline__ uint32_t smem_address(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// ---- mbarriers ------------------------------------------------------------------------------------
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
__device__ __forceinline__ uint32_t now_ticks() {                     // of 2^17 ns
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return static_cast<uint32_t>(t >> 17);
}

// No wait is endless: after two seconds a wait gives up, the CTA's other waits follow, and the kernel winds up.  The timer runs
// on while the program is not on the device: a round of tries counts for a tenth of a second at most.
constexpr uint32_t kWaitLimit = 15259, kRoundLimit = 763;

// Waits of a whole warp (every lane gets the same answer).  false: given up; `stop` (shared memory) is set.
__device__ __forceinline__ bool barrier_wait_slow(uint32_t bar, uint32_t parity, volatile int *stop, unsigned int *timeouts) {
    uint32_t last = now_ticks(), spent = 0;
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (barrier_try(bar, parity)) return true;
        if (stop != nullptr && *stop != 0) return false;
        const uint32_t now = now_ticks();
        spent += min(now - last, kRoundLimit);
        last = now;
        if (spent > kWaitLimit) {
            if (stop != nullptr) *stop = 1;
            atomicAdd(timeouts, 1u);
            return false;
        }
    }
}
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile int *stop, unsigned int *timeouts) {
    const bool ok = barrier_try(bar, parity) || barrier_wait_slow(bar, parity, stop, timeouts);
    return __all_sync(0xffffffffu, ok);
}

// ---- TMA ------------------------------------------------------------------------------------------
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
}
// (x, row, head, batch) box of the map's size to shared memory; x is a multiple of 64 elements (128 bytes).
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, int x, int row, int head, int batch, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2,%3,%4,%5}], [%6];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(row), "r"(head), "r"(batch), "r"(bar) : "memory");
}

// Contiguous bytes (a multiple of 16, both ends 16-byte aligned) to shared memory.
__device__ __forceinline__ void load_bytes(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// ---- clusters -------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {                      // every thread of every CTA of the cluster
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the same in two halves
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float load_peer(uint32_t address, uint32_t rank) {
    float v;
    asm volatile("{\n.reg .b32 a;\nmapa.shared::cluster.u32 a, %1, %2;\nld.shared::cluster.f32 %0, [a];\n}" : "=f"(v) : "r"(address), "r"(rank) : "memory");
    return v;
}

// ---- registers: a warpgroup hands some to the others (the sums stay within what the CTA was launched with).  Code behind
// the roles' branches runs with the smaller number: it must be next to nothing.
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(N)); }
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(N)); }

// ---- tensor memory --------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t columns) {        // one whole warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The values that the loads before it were given may be used only behind it: they pass through it.
template <int N>
__device__ __forceinline__ void wait_ld(uint32_t (&r)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of this thread's lane
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t at, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                    "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
                    "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
                    "r"(r[30]), "r"(r[31])
                 : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                    "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

__device__ __forceinline__ void tmem_ld8(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(at) : "memory");
}
// 16 lanes x 32 columns of 32 bits: in group g of 8 columns a thread gets columns 8g + 2 (lane % 4) and the next one of
// lanes lane / 4 (r[4g], r[4g + 1]) and lane / 4 + 8 (r[4g + 2], r[4g + 3])
__device__ __forceinline__ void tmem_ld_16x32(uint32_t at, uint32_t *r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
// 16 lanes x 16 columns of 32 bits: in group g of 4 columns a thread gives column 4g + lane % 4 of lanes lane / 4 (r[2g]) and
// lane / 4 + 8 (r[2g + 1]): where pairs of the values above, rounded to 16 bits, belong
__device__ __forceinline__ void tmem_st_16x16(uint32_t at, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t *r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}

// 16 bytes of a tile: elements [8 chunk, 8 chunk + 8) of a row, where TMA's 128-byte swizzle put them
__device__ __forceinline__ uint4 tile_chunk(uint32_t tile, int row, int chunk) {
    uint4 v;
    const uint32_t at = tile + (chunk / 8) * (128 * 128) + row * 128 + (((chunk % 8) ^ (row & 7)) << 4);
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// ---- tcgen05.mma ----------------------------------------------------------------------------------
// Shared-memory tiles hold rows of 64 elements (128 bytes) in the 128-byte swizzle, 128 rows = 16 KB; a tile of
// 128 columns is two of them.  The same bytes serve as an operand whose contraction runs along the row (K-major)
// and as one whose contraction runs down the rows (MN-major).
constexpr uint32_t kHalfTile = 128 * 128;       // bytes of 128 rows x 64 elements
__device__ __forceinline__ uint64_t descriptor(uint32_t address, uint32_t leading, uint32_t stride) {
    return static_cast<uint64_t>((address >> 4) & 0x3fffu) | static_cast<uint64_t>(leading >> 4) << 16 |
           static_cast<uint64_t>(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
__device__ __forceinline__ uint64_t k_major(uint32_t address) { return descriptor(address, 16, 1024); }       // groups of 8 rows: 1 KB apart
__device__ __forceinline__ uint64_t mn_major(uint32_t address) { return descriptor(address, kHalfTile, 1024); } // 64-element blocks: one half tile apart

template <typename T> struct Format;
template <> struct Format<__half> { static constexpr uint32_t value = 0; };
template <> struct Format<__nv_bfloat16> { static constexpr uint32_t value = 1; };
// M = 128, N, binary32 accumulator; b_mn: B is MN-major
template <typename T>
__host__ __device__ constexpr uint32_t instruction(uint32_t n, bool b_mn) {
    return 1u << 4 | Format<T>::value << 7 | Format<T>::value << 10 | (b_mn ? 1u << 16 : 0u) | (n >> 3) << 17 | (128u >> 4) << 24;
}
// The issuing warp runs these with all its lanes and in step: operands then live in uniform registers, where the instruction
// takes them, and only `leader` (one lane's 1, chosen by elect) issues.  In a branch of one lane every operand is moved there
// first, and an MMA takes 110 clocks to issue in place of the 64 that it computes.
__device__ __forceinline__ uint32_t elect_leader() {
    uint32_t leader;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(leader));
    return leader;
}
template <typename V>
__device__ __forceinline__ V uniform(V x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %4, 0;\nsetp.ne.b32 q, %5, 0;\n@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(static_cast<uint32_t>(accumulate)), "r"(leader) : "memory");
}
// the barrier's phase ends when every MMA issued so far by the leader has finished
__device__ __forceinline__ void commit(uint32_t leader, uint32_t bar) {
    asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}"
                 :: "r"(bar), "r"(leader) : "memory");
}

// D (128 x 128) = A B^T over DIM: both tiles K-major
template <typename T, int DIM>
__device__ __forceinline__ void product_rows(uint32_t leader, uint32_t d, uint32_t a, uint32_t b) {
    constexpr uint32_t idesc = instruction<T>(128, false);
    const uint64_t da = k_major(a), db = k_major(b);
#pragma unroll
    for (int k = 0; k < DIM / 16; ++k) {
        const uint64_t off = ((k / 4) * kHalfTile + (k % 4) * 32) >> 4;
        mma_ss(leader, d, da + off, db + off, idesc, k > 0);
    }
}
// The same with A (16 bits) in tensor memory: a step of 16 takes 8 TMEM columns.  An MMA from tensor memory reads half the
// shared memory of one whose operands both lie there, which takes all of the 128 bytes that a clock has.
template <typename T, int DIM>
__device__ __forceinline__ void product_rows_tmem(uint32_t leader, uint32_t d, uint32_t a, uint32_t b) {
    constexpr uint32_t idesc = instruction<T>(128, false);
    const uint64_t db = k_major(b);
#pragma unroll
    for (int k = 0; k < DIM / 16; ++k) mma_ts(leader, d, a + 8 * k, db + (((k / 4) * kHalfTile + (k % 4) * 32) >> 4), idesc, k > 0);
}
// D (128 x DIM) (+)= A B: A (128 x 128, 16 bits) in tensor memory, B's rows are the contraction.  Its 8 steps of 16 take 8
// TMEM columns of A each, GROUP steps side by side and each group PITCH columns after the one before (the element-wise
// threads write where they have read).  STEPS: a bit for each step to do.
template <typename T, int DIM, int GROUP, int PITCH, int STEPS = 0xff>
__device__ __forceinline__ void product_columns(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, bool accumulate) {
    constexpr uint32_t idesc = instruction<T>(DIM, true);
    constexpr int kFirst = STEPS & 1 ? 0 : STEPS & 2 ? 1 : 2;
    const uint64_t db = mn_major(b);
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (STEPS >> k & 1) mma_ts(leader, d, a + (k / GROUP) * PITCH + (k % GROUP) * 8, db + k * (2048 >> 4), idesc, accumulate || k > kFirst);
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {   // NaN if one of them is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 2^x for two values on the FMA pipe, which has room where the exponential unit (16 results a clock) is the limit:
// x = n + f with n the nearest integer, f in [-1/2, 1/2] (as in Cody and Waite, Software Manual for the Elementary Functions,
// 1980); 2^f by the degree-4 polynomial of least relative error (2.6e-6,
// found by iteratively reweighted least squares), n added to the exponent.  Values below 2^-126 come out as 2^-126; a NaN or
// an infinity comes out as a value that is not finite in 16 bits but may be in 32: where such a value may be the only one of a
// sum, the caller has to see to it.
__device__ __forceinline__ void exp2_polynomial(float &d0, float &d1, float x0, float x1) {
    constexpr float kMagic = 12582912.0f;                             // 1.5 * 2^23: the sum's low bits are the integer
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(x0) : "f"(x0), "f"(-126.0f));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(x1) : "f"(x1), "f"(-126.0f));
    float t0, t1, n0, n1, f0, f1, p0, p1;
    add2(t0, t1, x0, x1, kMagic, kMagic);
    add2(n0, n1, t0, t1, -kMagic, -kMagic);
    fma2(f0, f1, n0, n1, -1.0f, -1.0f, x0, x1);
    fma2(p0, p1, f0, f1, 0.009570102207362652f, 0.009570102207362652f, 0.05591785907745361f, 0.05591785907745361f);
    fma2(p0, p1, p0, p1, f0, f1, 0.240247443318367f, 0.240247443318367f);
    fma2(p0, p1, p0, p1, f0, f1, 0.6931217908859253f, 0.6931217908859253f);
    fma2(p0, p1, p0, p1, f0, f1, 0.9999992847442627f, 0.9999992847442627f);
    d0 = __int_as_float(__float_as_int(p0) + (__float_as_int(t0) << 23));
    d1 = __int_as_float(__float_as_int(p1) + (__float_as_int(t1) << 23));
}
// (d0, d1) = 2^(x c + m); POLY: on the FMA pipe
template <bool POLY>
__device__ __forceinline__ void exp2_scaled(float &d0, float &d1, float x0, float x1, float c, float m0, float m1) {
    float y0, y1;
    fma2(y0, y1, x0, x1, c, c, m0, m1);
    if constexpr (POLY) {
        exp2_polynomial(d0, d1, y0, y1);
    } else {
        d0 = exp2_fast(y0);
        d1 = exp2_fast(y1);
    }
}

}  // namespace tc
}  // namespace fewbit
