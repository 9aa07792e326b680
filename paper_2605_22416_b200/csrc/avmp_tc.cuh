// Blackwell building blocks of the attention kernels: mbarriers with bounded waits, tiled bulk loads of page slices,
// tensor-core products with accumulators in tensor memory.
#pragma once

#include <cuda.h>

#include "avmp_dev.cuh"
#include "avmp_mma.cuh"

namespace avmp {

// Bounded waits of a CTA.  A wait that runs out makes all its later waits fail at once, so that every role stops issuing.  Once all
// roles have stopped, behind a barrier of the whole CTA, the kernel looks at over(): it counts one AVMP_DEV_TIMEOUT, and whoever has
// copies in flight lets them land (mbar_land) before the CTA's memory is given away.
struct Waits {
    volatile uint32_t *gave_up;   // in shared memory
    WaitLimit limit;
    __device__ bool over() const { return *gave_up != 0; }
};

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_fence_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)      // the same without staying
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Waits until the phase with this parity is complete.  False once the limit has passed, for this wait or an earlier one of the CTA:
// the caller then issues nothing more.
__device__ __forceinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, Waits w)
{
    const unsigned long long t0 = global_ns();
    while (!mbar_test(bar, parity)) {
        if (w.over()) return false;
        if (global_ns() - t0 >= w.limit.ns) {
            *w.gave_up = 1;
            return false;
        }
    }
    return true;
}
// For one thread on its own.
__device__ __forceinline__ bool mbar_wait_one(uint32_t bar, uint32_t parity, const Waits &w)
{
    bool ok = mbar_test(bar, parity);
#pragma unroll 1
    for (uint32_t i = 0; i < w.limit.tries && !ok; ++i) ok = mbar_try(bar, parity);
    return ok || mbar_wait_slow(bar, parity, w);
}
// For a whole warp; the same answer for all its lanes.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const Waits &w)
{
    return __all_sync(0xFFFFFFFFu, mbar_wait_one(bar, parity, w));
}
// A copy or product in flight is given two seconds to complete, whatever the limit is.
__device__ __forceinline__ void mbar_land(uint32_t bar, uint32_t parity)
{
    const unsigned long long t0 = global_ns();
    while (!mbar_test(bar, parity) && global_ns() - t0 < kWaitLimitNs) {}
}
// One thread of a converged warp (the form the compiler knows as a single issuing thread).
__device__ __forceinline__ bool elect_one()
{
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}

// One box of the page tensor: 64 elements of `rows` tokens of a run of heads, at (x, token, head, layer and part, slot).
__device__ __forceinline__ void tma_load_page(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int token, int head,
                                              int part, int slot)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(token), "r"(head), "r"(part), "r"(slot) : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
}
// Writes of ordinary stores to shared memory become visible to bulk copies and tensor-core operand reads.
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory and tensor-core products (one CTA per tile)
__device__ __forceinline__ void tmem_alloc512(uint32_t smem_dst)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_dst) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free512(uint32_t tmem)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The barrier gets one arrival when every product issued so far by this thread is complete.
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
// D[tmem] (+)= A[smem] B[smem], and with A in tensor memory.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, unsigned long long a, unsigned long long b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, unsigned long long b, uint32_t idesc, bool add)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// Shared-memory operand in rows of 128 bytes whose 16-byte units are permuted by the row index (128-byte swizzle):
// groups of 8 rows `group` bytes apart; `lead` is the distance between column blocks of 64 elements where the operand's
// long axis runs along the rows.
__device__ __forceinline__ unsigned long long tc_desc(uint32_t addr, uint32_t group, uint32_t lead)
{
    return (unsigned long long)((addr & 0x3FFFFu) >> 4) | ((unsigned long long)(lead >> 4) << 16) | ((unsigned long long)(group >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: 16-bit operands, 32-bit sums, M = 128.
constexpr uint32_t kNegateA = 1u << 13;
__device__ __forceinline__ constexpr uint32_t tc_idesc(bool f16, bool b_by_rows, uint32_t n)
{
    return (1u << 4) | ((f16 ? 0u : 1u) << 7) | ((f16 ? 0u : 1u) << 10) | ((b_by_rows ? 1u : 0u) << 16) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

#define AVMP_R8(r, o) "=r"((r)[(o)]), "=r"((r)[(o) + 1]), "=r"((r)[(o) + 2]), "=r"((r)[(o) + 3]), "=r"((r)[(o) + 4]), "=r"((r)[(o) + 5]), "=r"((r)[(o) + 6]), "=r"((r)[(o) + 7])
#define AVMP_W8(r, o) "r"((r)[(o)]), "r"((r)[(o) + 1]), "r"((r)[(o) + 2]), "r"((r)[(o) + 3]), "r"((r)[(o) + 4]), "r"((r)[(o) + 5]), "r"((r)[(o) + 6]), "r"((r)[(o) + 7])
// 32 columns of this thread's lane.
__device__ __forceinline__ void tmem_ld32(uint32_t *r, uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : AVMP_R8(r, 0), AVMP_R8(r, 8), AVMP_R8(r, 16), AVMP_R8(r, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
                 "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(addr), AVMP_W8(r, 0), AVMP_W8(r, 8), AVMP_W8(r, 16), AVMP_W8(r, 24) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t *r, uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : AVMP_R8(r, 0), AVMP_R8(r, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(addr), AVMP_W8(r, 0), AVMP_W8(r, 8) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- pairs of 32-bit floats in one instruction
__device__ __forceinline__ unsigned long long pack2(float lo, float hi)
{
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpack2(unsigned long long v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c)
{
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b)
{
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Largest of three; a NaN wins.
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// 2^x of a pair on the multiply-add pipe (the special-function unit gives 4 exponentials a cycle and scheduler).  x is split into an integer n, by adding and taking away 1.5 * 2^23, and |f| <= 1/2;
// 2^f is a polynomial of degree 4 fitted for least relative error (2.6e-6) on that interval, 2^n is put together from
// its exponent.  x <= 2^6; below -126.5 the result is 0 (a masked token's weight, which a large value would make visible otherwise).
__device__ __forceinline__ float2 exp2_poly2(unsigned long long x)
{
    float2 t = unpack2(x);
    t.x = fmaxf(t.x, -127.f); t.y = fmaxf(t.y, -127.f);
    const unsigned long long v = pack2(t.x, t.y);
    const unsigned long long n = add2(v, pack2(12582912.f, 12582912.f));
    const unsigned long long f = add2(v, fma2(n, pack2(-1.f, -1.f), pack2(12582912.f, 12582912.f)));
    unsigned long long y = fma2(f, pack2(9.570101754e-03f, 9.570101754e-03f), pack2(5.591786031e-02f, 5.591786031e-02f));
    y = fma2(y, f, pack2(2.402474483e-01f, 2.402474483e-01f));
    y = fma2(y, f, pack2(6.931218147e-01f, 6.931218147e-01f));
    y = fma2(y, f, pack2(9.999992614e-01f, 9.999992614e-01f));
    const float2 m = unpack2(n);      // an exponent field of 0 for n = -127
    return unpack2(mul2(y, pack2(__uint_as_float((__float_as_uint(m.x) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(m.y) << 23) + 0x3F800000u))));
}

// The pages as a five-dimensional tensor [slot][layer, K or V][head][token][dim] with boxes of box_tokens x box_heads rows of
// 64 elements; dimensions need not be in memory order, so a box arrives sorted by head.  (avmp_attn.cu)
bool page_map(CUtensorMap *map, const Geom &g, uint32_t kv_heads, uint32_t head_dim, uint32_t box_tokens, uint32_t box_heads);

// The rows of one head as [head row of the arena][8-token group][64 columns][token of the group][column]: a box of whole
// groups arrives as [group][column block][token], which is what the tensor cores read, in one copy.  The outermost
// coordinate counts rows of head_dim elements from the arena's start (pages and heads lie at multiples of them).
bool row_map(CUtensorMap *map, const Geom &g, uint32_t head_dim, uint32_t box_tokens);
// Query rows as [token][query head][dim], boxes of box_tokens x box_heads rows of 64 elements.
bool query_map(CUtensorMap *map, const void *q, uint32_t head_dim, uint32_t q_heads, uint32_t rows, unsigned long long stride,
               uint32_t box_tokens, uint32_t box_heads);
__device__ __forceinline__ void tma_load_query(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int head, int token)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(head), "r"(token) : "memory");
}
// Packed rows of 16-bit numbers, boxes of `rows` x `columns` (16, 32 or 64) with the swizzle of that width; rows behind the last are zeros.
bool rows_map(CUtensorMap *map, const void *p, uint32_t row_elems, uint32_t n_rows, unsigned long long stride, uint32_t columns, uint32_t rows);
__device__ __forceinline__ void tma_load_tile(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int row)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(row) : "memory");
}
__device__ __forceinline__ void tma_prefetch_rows(const CUtensorMap *map, int group, int row)
{
    asm volatile("cp.async.bulk.prefetch.tensor.5d.L2.global.tile [%0, {%3, %3, %3, %1, %2}];" :: "l"(map), "r"(group), "r"(row), "r"(0) : "memory");
}
__device__ __forceinline__ void tma_load_rows(uint32_t dst, const CUtensorMap *map, uint32_t bar, int group, int row)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%5, %5, %5, %3, %4}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(group), "r"(row), "r"(0) : "memory");
}

// Tokens that a slot's chain holds; 0 for a slot that is empty or out of range.  Both tables are read at once, and past the
// L1 cache (a kernel that starts without waiting has nothing else to tell it that its lines are new).
__device__ __forceinline__ uint32_t held_tokens(const Geom &g, uint32_t r)
{
    const uint32_t i = r < g.R ? r : 0u, state = __ldcg(g.r_state + i), len = __ldcg(g.r_len + i);
    return r < g.R && state != AVMP_REQ_EMPTY ? len : 0u;
}

// What the parts of an attention call leave for the joining pass: sums over part of the tokens, not yet divided.
struct Parts {
    float *o;        // [part][head][dim]
    float2 *ml;      // [part][head]: maximum (log2 units) that the sums are relative to, sum of exponentials (0: no sums written)
};

// The pass over the shared prefix of a batch of single tokens: fills *out with *parts parts of [n][q_heads].  (avmp_attn_prompt.cu)
cudaError_t launch_attn_prefix(const Geom &g, const AttnArgs &a, const Launch &l, Parts *out, uint32_t *parts);
size_t attn_tile_ws_bytes(const Geom &g, uint32_t n, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, int n_sms);

}  // namespace avmp
