// What the calls over request lists share: the state block behind a list entry, repeated slots, runs of rows of packed buffers.
#pragma once

#include "avmp_dev.cuh"
#include "avmp_mma.cuh"

namespace avmp {

// The block of a request's state layer, or null where the slot is out of range or not LIVE.
__device__ __forceinline__ float *state_block(const Geom &g, uint32_t layer, uint32_t r)
{
    uint32_t slot = kInvalid;
    if (r < g.R) {
        const uint32_t state = g.r_state[r], h = g.r_ssm[(unsigned long long)r * g.ns + layer];
        if (state == AVMP_REQ_LIVE && h != kInvalid) slot = g.VT[1][h & 0x7FFFFFFFu];
    }
    return slot == kInvalid ? nullptr : reinterpret_cast<float *>(unit_ptr(g, AVMP_POOL_SSM, slot));
}
// Whether an earlier entry of the list names the same slot (two entries would write one block at the same time).  Whole CTA.
__device__ __forceinline__ bool named_before(const uint32_t *reqs, uint32_t k, uint32_t r)
{
    bool dup = false;
    for (uint32_t j = threadIdx.x; j < k; j += blockDim.x) dup |= reqs[j] == r;
    return __syncthreads_or(dup);
}

// The same for entries k .. k + each - 1 (each <= 4; those behind the n-th are not looked at): a bit for each.  `flags` is a word of
// shared memory; a barrier has to stand between two calls.  Whole CTA.
__device__ __forceinline__ uint32_t named_before_each(const uint32_t *reqs, uint32_t k, uint32_t each, uint32_t n, uint32_t *flags)
{
    const uint32_t last = min(n, k + each);
    uint32_t r[4], bits = 0;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e) r[e] = k + e < last ? reqs[k + e] : 0u;
    if (threadIdx.x == 0) *flags = 0;
    __syncthreads();
    for (uint32_t j = threadIdx.x; j + 1 < last; j += blockDim.x) {
        const uint32_t x = reqs[j];
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) bits |= (uint32_t)(x == r[e] && j < k + e) << e;
    }
    bits = __reduce_or_sync(0xFFFFFFFFu, bits);
    if (bits && threadIdx.x % 32 == 0) atomicOr(flags, bits);
    __syncthreads();
    return *flags;
}

// The rows of all list entries, in runs of `rows` at most: an entry without rows, with offsets that do not fit the buffers, or with more rows
// than `most` has one too, so that somebody looks after it.  A CTA walks them in ascending order; the entries' offsets pass through shared
// memory as many at a time as the CTA has threads.  (Offsets that swing to and fro may name the buffers' rows many times over: runs are
// counted in 64 bits.)
struct Runs {
    const uint32_t *cu;
    uint32_t n, total, rows;
    unsigned long long most;
    unsigned long long *pre;     // shared, blockDim.x
    unsigned long long *tmp;     // shared, 32
    uint32_t k0, cnt;
    unsigned long long begin, end;

    __device__ Runs(const uint32_t *cu_, uint32_t n_, uint32_t total_, uint32_t rows_, unsigned long long most_, unsigned long long *pre_,
                    unsigned long long *tmp_)
        : cu(cu_), n(n_), total(total_), rows(rows_), most(most_), pre(pre_), tmp(tmp_), k0(0), cnt(0), begin(0), end(0) {}
    // Run i: its entry and its number there.  False behind the last one.  Whole CTA; i ascends from call to call.
    __device__ bool seek(unsigned long long i, uint32_t *k, uint32_t *run)
    {
        while (i >= end) {
            if (k0 + cnt >= n) return false;
            k0 += cnt;
            cnt = min(blockDim.x, n - k0);
            __syncthreads();                       // the offsets before have been read
            unsigned long long mine = 0, all;
            if (threadIdx.x < cnt) {
                const uint32_t c0 = cu[k0 + threadIdx.x], c1 = cu[k0 + threadIdx.x + 1];
                mine = c1 > c0 && c1 <= total && c1 - c0 <= most ? (c1 - c0 + rows - 1) / rows : 1u;
            }
            const unsigned long long incl = block_incl_scan(mine, tmp, &all);
            pre[threadIdx.x] = incl - mine;
            begin = end; end += all;
            __syncthreads();
        }
        uint32_t lo = 0, hi = cnt;                 // the last entry that begins at run i or before
        while (lo + 1 < hi) {
            const uint32_t mid = (lo + hi) >> 1;
            if (pre[mid] <= i - begin) lo = mid; else hi = mid;
        }
        *k = k0 + lo; *run = (uint32_t)(i - begin - pre[lo]);
        return true;
    }
};

// x / (1 + e^-x)
__device__ __forceinline__ float silu(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + exp2_approx(x * -1.4426950408889634f)));
    return x * r;
}

}  // namespace avmp
