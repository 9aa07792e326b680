// Attention of single tokens over paged KV chains, read where they lie (no counterpart in the paper).
//
//   attn_decode_kernel   every request's chain against its one query row per head;
//   attn_join_kernel     puts the parts of a request together that different CTAs (or the prefix pass) worked out.
//
// Bound by HBM: a token's K and V are read once for all query heads that share them.  The work of a launch is
// the list of all steps (16 tokens, or 16 per token share) of all requests in order; CTA i of P takes the i-th P-th of it,
// whatever the lengths, so a batch with one 64 k chain is as balanced as one of equal chains.  A request cut by a
// border leaves unnormalised sums, maximum and denominator in the workspace; the joining pass adds the parts in CTA
// order, so results do not depend on timing.  Weights are rounded to the 16 bits of V for the tensor cores (eps/2 each, averaged over the tokens: an
// output is 1.1 to 1.2 times as far from the formula as its own rounding alone); maxima, denominators and sums are held in 32 bits.
//
// Measured (32 query heads on 8 KV heads of 128, bf16): 1024 chains of 40 to 2400 tokens 408 to 420 us (93 to 96 % of the measured copy
// rate), 128 chains, a fifth of 16 to 64 thousand tokens, 608 to 624 us (101 to 104 %); 32 chains of 48 to 640 tokens 16 to 19 us, of which the
// kernel's own beginning (list, pages: four dependent reads) and the second launch are most.  Through a window only the steps are listed that
// have a token that is seen: 128 chains, a fifth of 16 to 64 thousand tokens, window 4096, 176 to 181 us (90 to 93 %).
#include "avmp_tc.cuh"

namespace avmp {

namespace {

template <int N>
bool encode(CUtensorMap *map, const void *base, const cuuint64_t (&dims)[N], const cuuint64_t (&strides)[N - 1], const cuuint32_t (&box)[N],
            CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    return fn && fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, N, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

bool page_map(CUtensorMap *map, const Geom &g, uint32_t kv_heads, uint32_t head_dim, uint32_t box_tokens, uint32_t box_heads)
{
    return encode<5>(map, g.arena, {head_dim, g.T, kv_heads, 2ull * g.na, g.V[0]},
                  {g.row_bytes, head_dim * 2ull, g.T * g.row_bytes, g.U[0]}, {64, box_tokens, box_heads, 1, 1});
}

bool row_map(CUtensorMap *map, const Geom &g, uint32_t head_dim, uint32_t box_tokens)
{
    const uint64_t row = head_dim * 2ull;
    return encode<5>(map, g.arena, {64, 8, head_dim / 64, g.T / 8, g.V[0] * (g.U[0] / row)}, {g.row_bytes, 128, 8 * g.row_bytes, row},
                  {64, 8, head_dim / 64, box_tokens / 8, 1});
}

bool rows_map(CUtensorMap *map, const void *p, uint32_t row_elems, uint32_t n_rows, unsigned long long stride, uint32_t columns, uint32_t rows)
{
    return encode<2>(map, p, {row_elems, n_rows}, {stride}, {columns, rows},
                     columns == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : columns == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B);
}

bool query_map(CUtensorMap *map, const void *q, uint32_t head_dim, uint32_t q_heads, uint32_t rows, unsigned long long stride,
               uint32_t box_tokens, uint32_t box_heads)
{
    return encode<3>(map, q, {head_dim, q_heads, rows}, {head_dim * 2ull, stride}, {64, box_heads, box_tokens});
}

namespace {

constexpr int kWarps = 8;                      // consumer warps; one more loads
constexpr int kThreads = (kWarps + 1) * 32;
constexpr uint32_t kRingBytes = 192 * 1024;
constexpr int kMaxStages = 8;

// How a CTA's eight warps share a step: `heads` KV heads x `mtiles` tiles of 16 query rows x `shares` runs of 16 tokens.
struct Split {
    uint32_t group;        // query heads per KV head
    uint32_t heads, mtiles, shares, head_groups;
    uint32_t box_tokens, stage_bytes, stages;
    uint32_t ctas;         // P, along the step list
};

struct Plan {
    uint32_t *cu, *req, *len;   // first step, slot and length of each list entry (cu: one more)
};

struct DecodeArgs {
    AttnArgs a;
    Split s;
    Plan ws;                   // in the workspace
    uint2 *jobs;               // [P] per border: the request that is cut there for the first time and its last CTA, or kInvalid
    Parts own;                 // [2 P] cut requests, then [n] whole ones (only with a prefix)
    Parts pre;                 // [pre_parts][n]
    uint32_t pre_parts;
};

// What the one row of a chain of `len` tokens sees through a window, in steps: `lead` steps with sinks, then, `skip` steps further on,
// those from the window's first token.  Every one of them has a token that is seen.
struct Sight {
    uint32_t low, lead, skip;      // low: the window's first token
    __device__ Sight(const AttnArgs &a, uint32_t len, uint32_t step)
    {
        low = len > a.window ? len - a.window : 0u;
        lead = (min(a.sinks, low) + step - 1) / step;
        skip = low / step > lead ? low / step - lead : 0u;
    }
    __device__ uint32_t at(uint32_t i) const { return i < lead ? i : i + skip; }
};
template <bool WINDOW>
__device__ __forceinline__ uint32_t steps_of(const AttnArgs &a, uint32_t len, uint32_t step)
{
    const uint32_t all = (len + step - 1) / step;
    return WINDOW ? all - Sight(a, len, step).skip : all;
}

// CTAs that have work: at least one step each, so that every part that is read has been written.
__device__ __forceinline__ uint32_t busy_ctas(const Split &s, unsigned long long total)
{
    return total < s.ctas ? (uint32_t)total : s.ctas;
}

// The step list, by the whole CTA.  Bad entries own no step.
template <bool WINDOW>
__device__ __forceinline__ void make_plan(const Geom &g, const DecodeArgs &d, const Plan &to, unsigned long long *tmp, bool lead)
{
    const uint32_t n = d.a.n, step = 16 * d.s.shares;
    const bool dead = d.a.prefix != kInvalid && held_tokens(g, d.a.prefix) == 0;
    const uint32_t per = (n + blockDim.x - 1) / blockDim.x, k0 = min(n, threadIdx.x * per), k1 = min(n, k0 + per);
    unsigned long long mine = 0, tot;
    for (uint32_t k = k0; k < k1; ++k) {
        const uint32_t r = __ldcg(d.a.reqs + k), own = held_tokens(g, r), len = dead ? 0u : own;
        if (lead && len == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
        to.req[k] = r; to.len[k] = len;
        mine += steps_of<WINDOW>(d.a, len, step);
    }
    unsigned long long run = block_incl_scan(mine, tmp, &tot) - mine;
    for (uint32_t k = k0; k < k1; ++k) {
        to.cu[k] = (uint32_t)run;
        run += steps_of<WINDOW>(d.a, to.len[k], step);
    }
    if (threadIdx.x == 0) to.cu[n] = (uint32_t)tot;
}

template <bool WINDOW>
__global__ void __launch_bounds__(kStepThreads) attn_plan_kernel(const Geom g, const DecodeArgs d)
{
    __shared__ unsigned long long tmp[32];
    pdl_prologue();
    make_plan<WINDOW>(g, d, d.ws, tmp, true);
}

template <class T, int D, bool WINDOW>
__global__ void __launch_bounds__(kThreads, 1)
attn_decode_kernel(const Geom g, const DecodeArgs d, const __grid_constant__ CUtensorMap map)
{
    constexpr int KS = D / 16, ND = D / 8;
    // Weights are relative to this much below the maximum: fp16 has subnormal numbers from 2^-14 down, and tens of thousands of weights of
    // 2^-25 would be rounded to nothing.
    constexpr float kBelow = T::kF16 ? 14.f : 0.f;
    extern __shared__ uint8_t smem_raw[];                  // ring (1024-byte rows groups of the swizzle), then the plan
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ unsigned long long bars[2 * kMaxStages], tmp[32];
    __shared__ uint32_t gave_up;
    __shared__ float red[kWarps][16][17], red_ml[kWarps][16][2];
    const Split &s = d.s;
    const uint32_t n = d.a.n;
    const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
    const bool lead = blockIdx.x == 0 && blockIdx.y == 0;
    const Waits waits{&gave_up, d.a.wait};
    uint32_t loads = 0;
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8 * kMaxStages, ring = smem_u32(smem);
    if (threadIdx.x == 0) {
        gave_up = 0;
        for (uint32_t i = 0; i < s.stages; ++i) { mbar_init(full0 + 8 * i, 1); mbar_init(empty0 + 8 * i, kWarps); }
        mbar_fence_init();
        tma_prefetch_map(&map);
    }
    // Behind a prefix pass: that pass lets this kernel start once everything in front of itself is complete, and the two
    // touch nothing in common, so there is nothing to wait for here (the joining pass needs both: see the end).
    const bool behind = d.a.prefix != kInvalid && n <= kLocalPlanMax;
    if (behind) asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); else pdl_prologue();
    Plan p = d.ws;
    if (n <= kLocalPlanMax) {
        p.cu = reinterpret_cast<uint32_t *>(smem + s.stages * s.stage_bytes);
        p.req = p.cu + n + 1; p.len = p.req + n;
        make_plan<WINDOW>(g, d, p, tmp, lead);
    }
    __syncthreads();
    if (n <= kLocalPlanMax && lead) {       // the joining pass reads it
        for (uint32_t k = threadIdx.x; k <= n; k += kThreads) {
            d.ws.cu[k] = p.cu[k];
            if (k < n) d.ws.len[k] = p.len[k];
        }
    }
    const unsigned long long total = p.cu[n];
    const uint32_t P = busy_ctas(s, total);
    const uint32_t first = blockIdx.x < P ? (uint32_t)(total * blockIdx.x / P) : 0u;
    const uint32_t last = blockIdx.x < P ? (uint32_t)(total * (blockIdx.x + 1) / P) : 0u;
    const uint32_t step_tokens = 16 * s.shares, share_bytes = s.heads * 16 * D * 2, half_bytes = s.heads * 16 * 128;
    const uint32_t box_bytes = s.heads * s.box_tokens * 128, boxes = 16 / s.box_tokens;
    uint32_t k = first < last ? find_owner(p.cu, 0, n, 0, first) : n;

    if (w == kWarps) {
        // ---- loads: the lanes look up the pages of the next 32 box rows ahead, lane 0 issues
        const uint32_t per_step = s.shares * boxes;         // box rows per step, <= 32
        uint32_t pk = k;
        for (uint32_t st0 = first; st0 < last;) {
            // as many whole steps as 32 lanes hold
            const uint32_t batch = min(last - st0, 32u / per_step);
            uint32_t slot = kInvalid, tok = 0;
            if (lane < batch * per_step) {
                const uint32_t st = st0 + lane / per_step;
                uint32_t kk = pk;
                while (p.cu[kk + 1] <= st) ++kk;
                uint32_t i = st - p.cu[kk];
                if (WINDOW) i = Sight(d.a, p.len[kk], step_tokens).at(i);
                const uint32_t t = i * step_tokens + (lane % per_step) * s.box_tokens;
                if (t < p.len[kk]) {
                    const uint32_t h = __ldcg(g.r_chain + ((unsigned long long)p.req[kk] * g.max_pages + t / g.T));
                    slot = __ldcg(g.VT[0] + (h & 0x7FFFFFFFu));
                    tok = t % g.T;
                }
            }
            for (uint32_t b = 0; b < batch; ++b, ++loads) {
                const uint32_t stage = loads % s.stages, round = loads / s.stages;
                if (round && !mbar_wait(empty0 + 8 * stage, (round - 1) & 1, waits)) goto stop;
                // (a warp that gave this stage's copy up has freed the stage too: nothing is copied on top of what is in flight)
                if (__any_sync(0xFFFFFFFFu, waits.over())) goto stop;
                const bool mine = lane / per_step == b && slot != kInvalid;
                const uint32_t live = __popc(__ballot_sync(0xFFFFFFFFu, mine));
                if (lane == 0) mbar_expect(full0 + 8 * stage, live * box_bytes * (D / 64) * 2);
                __syncwarp();
                if (mine) {
                    const uint32_t i = lane % per_step;
                    const uint32_t dst = ring + stage * s.stage_bytes + (i / boxes) * share_bytes + (i % boxes) * box_bytes;
#pragma unroll
                    for (int v = 0; v < 2; ++v)
#pragma unroll
                        for (int x = 0; x < D / 64; ++x)
                            tma_load_page(dst + v * (s.stage_bytes / 2) + x * half_bytes, &map, full0 + 8 * stage, x * 64, tok,
                                          blockIdx.y * s.heads, d.a.layer * 2 + v, slot);
                }
            }
            st0 += batch;
            if (st0 < last) while (p.cu[pk + 1] <= st0) ++pk;
        }
stop:
        if (behind) asm volatile("griddepcontrol.wait;" ::: "memory");
    }

    // ---- consumers: one (head, 16 query rows, 16 tokens of a step) each
    const uint32_t units = s.heads * s.mtiles, unit = w % units, share = w / units;
    const bool works = (uint32_t)w < units * s.shares;
    const uint32_t hh = unit / s.mtiles, mt = unit % s.mtiles, kv_head = blockIdx.y * s.heads + hh;
    const int lr = lane >> 2, lc = (lane & 3) * 2;
    const uint32_t g0 = mt * 16 + lr, g1 = g0 + 8;             // rows of the head's group
    const uint32_t qh0 = kv_head * s.group + g0, qh1 = kv_head * s.group + g1;
    const bool row0 = works && g0 < s.group, row1 = works && g1 < s.group;
    const float sl2 = d.a.scale * 1.4426950408889634f;
    auto token_off = [&](uint32_t t) { return (t / s.box_tokens) * box_bytes + hh * s.box_tokens * 128 + (t % s.box_tokens) * 128; };
    const uint32_t kt = (lane & 7) + ((lane >> 4) << 3), vt = lane & 15;
    const uint32_t k_off = share * share_bytes + token_off(kt), v_off = share * share_bytes + token_off(vt) + s.stage_bytes / 2;
    uint32_t it = 0;
    bool there = true;
    for (uint32_t st = w == kWarps ? last : first; st < last;) {
        while (p.cu[k + 1] <= st) ++k;
        const uint32_t begin = p.cu[k], end = p.cu[k + 1], seg_end = min(last, end), len = p.len[k];
        // query rows as the left operand, straight from global memory
        uint32_t q[KS][4];
        {
            const uint8_t *q0 = d.a.q + k * d.a.qs + (unsigned long long)qh0 * D * 2, *q1 = d.a.q + k * d.a.qs + (unsigned long long)qh1 * D * 2;
#pragma unroll
            for (int x = 0; x < KS; ++x) {
                q[x][0] = row0 ? __ldcg(reinterpret_cast<const uint32_t *>(q0 + (x * 16 + lc) * 2)) : 0u;
                q[x][1] = row1 ? __ldcg(reinterpret_cast<const uint32_t *>(q1 + (x * 16 + lc) * 2)) : 0u;
                q[x][2] = row0 ? __ldcg(reinterpret_cast<const uint32_t *>(q0 + (x * 16 + 8 + lc) * 2)) : 0u;
                q[x][3] = row1 ? __ldcg(reinterpret_cast<const uint32_t *>(q1 + (x * 16 + 8 + lc) * 2)) : 0u;
            }
        }
        float o[ND][4];
#pragma unroll
        for (int x = 0; x < ND; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[x][i] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        const Sight sight(d.a, WINDOW ? len : 0u, step_tokens);
        for (uint32_t c = st; c < seg_end; ++c, ++it) {
            const uint32_t stage = it % s.stages;
            // A copy that does not land in time is reported and none is waited for again: the warps of this CTA keep their
            // barriers with each other, and the results are not to be used.
            if (there) there = mbar_wait(full0 + 8 * stage, (it / s.stages) & 1, waits);
            const uint32_t base = ring + stage * s.stage_bytes;
            const uint32_t t0 = (WINDOW ? sight.at(c - begin) : c - begin) * step_tokens + share * 16;
            if (works && t0 < len) {
                const uint32_t valid = len - t0;
                // of these 16 tokens: the first that the window shows, and how many are sinks
                const uint32_t low = sight.low > t0 ? sight.low - t0 : 0u, sinks = d.a.sinks > t0 ? d.a.sinks - t0 : 0u;
                auto seen = [&](uint32_t t) { return t < valid && (!WINDOW || t >= low || t < sinks); };
                float x[2][4] = {};
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    const uint32_t ch = i * 2 + ((lane >> 3) & 1);
                    uint32_t b[4];
                    ldsm4(b, base + k_off + (ch >> 3) * half_bytes + (((ch & 7) ^ (kt & 7)) << 4));
                    T::mma(x[0], q[i], b[0], b[1]);
                    T::mma(x[1], q[i], b[2], b[3]);
                }
                // scores in log2 units; what lies behind the last token is other requests' leftovers
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[h][i] = seen(h * 8 + lc + (i & 1)) ? x[h][i] * sl2 : -INFINITY;
                float n0 = fmaxf(fmaxf(x[0][0], x[0][1]), fmaxf(x[1][0], x[1][1]));
                float n1 = fmaxf(fmaxf(x[0][2], x[0][3]), fmaxf(x[1][2], x[1][3]));
#pragma unroll
                for (int i = 1; i < 4; i <<= 1) {
                    n0 = fmaxf(n0, __shfl_xor_sync(0xFFFFFFFFu, n0, i));
                    n1 = fmaxf(n1, __shfl_xor_sync(0xFFFFFFFFu, n1, i));
                }
                n0 -= kBelow; n1 -= kBelow;
                if (__any_sync(0xFFFFFFFFu, n0 > m0 || n1 > m1)) {
                    n0 = fmaxf(n0, m0); n1 = fmaxf(n1, m1);
                    const float f0 = m0 == n0 ? 1.f : exp2_approx(m0 - n0), f1 = m1 == n1 ? 1.f : exp2_approx(m1 - n1);
                    m0 = n0; m1 = n1; l0 *= f0; l1 *= f1;
#pragma unroll
                    for (int i = 0; i < ND; ++i) { o[i][0] *= f0; o[i][1] *= f0; o[i][2] *= f1; o[i][3] *= f1; }
                }
                // a row that has seen nothing but scores of minus infinity so far: their weights are 0, not 2^(-inf + inf)
                const float s0 = m0 == -INFINITY ? 0.f : m0, s1 = m1 == -INFINITY ? 0.f : m1;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    x[h][0] = exp2_approx(x[h][0] - s0); x[h][1] = exp2_approx(x[h][1] - s0);
                    x[h][2] = exp2_approx(x[h][2] - s1); x[h][3] = exp2_approx(x[h][3] - s1);
                    l0 += x[h][0] + x[h][1]; l1 += x[h][2] + x[h][3];
                }
                const uint32_t pa[4] = {T::pack(x[0][0], x[0][1]), T::pack(x[0][2], x[0][3]), T::pack(x[1][0], x[1][1]), T::pack(x[1][2], x[1][3])};
                // a weight of zero does not silence a NaN: leftover rows of V count as zeros
                const uint32_t keep0 = (seen(lc) ? 0xFFFFu : 0u) | (seen(lc + 1) ? 0xFFFF0000u : 0u);
                const uint32_t keep1 = (seen(lc + 8) ? 0xFFFFu : 0u) | (seen(lc + 9) ? 0xFFFF0000u : 0u);
#pragma unroll
                for (int i = 0; i < ND / 2; ++i) {
                    const uint32_t ch = i * 2 + (lane >> 4);
                    uint32_t b[4];
                    ldsm4_t(b, base + v_off + (ch >> 3) * half_bytes + (((ch & 7) ^ (vt & 7)) << 4));
                    T::mma(o[2 * i], pa, b[0] & keep0, b[1] & keep1);
                    T::mma(o[2 * i + 1], pa, b[2] & keep0, b[3] & keep1);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty0 + 8 * stage);
        }
        // ---- this CTA's part of the request
#pragma unroll
        for (int i = 1; i < 4; i <<= 1) {
            l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, i);
            l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, i);
        }
        if (s.shares > 1) {
            // warps that saw different tokens for the same rows: a common maximum, then sums in the order of the shares
            if ((lane & 3) == 0) { red_ml[w][lr][0] = m0; red_ml[w][lr][1] = l0; red_ml[w][lr + 8][0] = m1; red_ml[w][lr + 8][1] = l1; }
            bar_sync(1, kWarps * 32);
            if (works) {
                float n0 = -INFINITY, n1 = -INFINITY, t0 = 0.f, t1 = 0.f;
                for (uint32_t j = 0; j < s.shares; ++j) { n0 = fmaxf(n0, red_ml[j * units + unit][lr][0]); n1 = fmaxf(n1, red_ml[j * units + unit][lr + 8][0]); }
                for (uint32_t j = 0; j < s.shares; ++j) {
                    const float *e0 = red_ml[j * units + unit][lr], *e1 = red_ml[j * units + unit][lr + 8];
                    t0 += e0[1] == 0.f ? 0.f : e0[1] * exp2_approx(e0[0] - n0);
                    t1 += e1[1] == 0.f ? 0.f : e1[1] * exp2_approx(e1[0] - n1);
                }
                const float f0 = m0 == -INFINITY ? 0.f : exp2_approx(m0 - n0), f1 = m1 == -INFINITY ? 0.f : exp2_approx(m1 - n1);
                m0 = n0; m1 = n1; l0 = t0; l1 = t1;
#pragma unroll
                for (int i = 0; i < ND; ++i) { o[i][0] *= f0; o[i][1] *= f0; o[i][2] *= f1; o[i][3] *= f1; }
            }
#pragma unroll
            for (int i = 0; i < ND / 2; ++i) {
                bar_sync(1, kWarps * 32);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    red[w][lr][h * 8 + lc] = o[2 * i + h][0]; red[w][lr][h * 8 + lc + 1] = o[2 * i + h][1];
                    red[w][lr + 8][h * 8 + lc] = o[2 * i + h][2]; red[w][lr + 8][h * 8 + lc + 1] = o[2 * i + h][3];
                }
                bar_sync(1, kWarps * 32);
                if (works && share == 0)
                    for (uint32_t j = 1; j < s.shares; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t x = j * units + unit;
                            o[2 * i + h][0] += red[x][lr][h * 8 + lc]; o[2 * i + h][1] += red[x][lr][h * 8 + lc + 1];
                            o[2 * i + h][2] += red[x][lr + 8][h * 8 + lc]; o[2 * i + h][3] += red[x][lr + 8][h * 8 + lc + 1];
                        }
            }
        }
        if (share == 0) {
            const bool cut_front = st > begin, cut_back = seg_end < end;
            if (!cut_front && !cut_back && d.a.prefix == kInvalid) {
                const float i0 = 1.f / l0, i1 = 1.f / l1;
                uint8_t *out = d.a.out + k * d.a.os;
#pragma unroll
                for (int i = 0; i < ND; i += 4)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        uint32_t v[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) v[x] = T::pack(o[i + x][2 * r] * (r ? i1 : i0), o[i + x][2 * r + 1] * (r ? i1 : i0));
                        quad_transpose(v);      // the lane then holds the eight columns of tile `lane & 3`: rows go out in 16-byte units
                        if (r ? row1 : row0)
                            *reinterpret_cast<uint4 *>(out + ((unsigned long long)(r ? qh1 : qh0) * D + (i + (lane & 3)) * 8) * 2) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                if (d.a.lse && (lane & 3) == 0) {
                    constexpr float kLn2 = 0.6931471805599453f;
                    if (row0) d.a.lse[(unsigned long long)k * d.a.q_heads + qh0] = m0 * kLn2 + logf(l0);
                    if (row1) d.a.lse[(unsigned long long)k * d.a.q_heads + qh1] = m1 * kLn2 + logf(l1);
                }
            } else {
                const uint32_t part = cut_front ? 2 * blockIdx.x : cut_back ? 2 * blockIdx.x + 1 : 2 * s.ctas + k;
                const unsigned long long at = (unsigned long long)part * d.a.q_heads;
#pragma unroll
                for (int i = 0; i < ND; i += 4)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        uint32_t v[4], z[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) { v[x] = __float_as_uint(o[i + x][2 * r]); z[x] = __float_as_uint(o[i + x][2 * r + 1]); }
                        quad_transpose(v);
                        quad_transpose(z);
                        if (r ? row1 : row0) {
                            uint4 *to = reinterpret_cast<uint4 *>(d.own.o + (at + (r ? qh1 : qh0)) * D + (i + (lane & 3)) * 8);
                            to[0] = make_uint4(v[0], z[0], v[1], z[1]);
                            to[1] = make_uint4(v[2], z[2], v[3], z[3]);
                        }
                    }
                if ((lane & 3) == 0) {
                    if (row0) d.own.ml[at + qh0] = make_float2(m0, l0);
                    if (row1) d.own.ml[at + qh1] = make_float2(m1, l1);
                }
            }
        }
        st = seg_end;
    }
    if (threadIdx.x == 0 && blockIdx.y == 0 && d.a.prefix == kInvalid && blockIdx.x < s.ctas) {
        // the border behind this CTA, for the joining pass
        uint2 job = make_uint2(kInvalid, 0);
        if (last > first && last < total) {
            const uint32_t c = find_owner(p.cu, 0, n, 0, last);
            if (p.cu[c] != last && p.cu[c] >= first) job = make_uint2(c, (uint32_t)(((unsigned long long)p.cu[c + 1] * P - 1) / total));
        }
        d.jobs[blockIdx.x] = job;
    }
    __syncthreads();
    if (threadIdx.x == 0 && waits.over()) record_error(g.st, AVMP_DEV_TIMEOUT);
    if (w == kWarps && waits.over())          // copies in flight land before this CTA's memory is given away
        for (uint32_t i = loads > s.stages ? loads - s.stages : 0; i < loads; ++i) mbar_land(full0 + 8 * (i % s.stages), (i / s.stages) & 1);
}

// Joins parts, a warp per (request, query head): weights of 32 parts a time, one per lane, sums of 16 parts in flight.
//   without a prefix: CTA (j, y) joins the request that the border behind decode CTA j cuts for the first time;
//   with one: CTA (k, y) joins the prefix parts and the own parts of request k.
// y counts groups of blockDim.x / 32 query heads.
template <class T, int D>
__global__ void __launch_bounds__(128) attn_join_kernel(const DecodeArgs d)
{
    pdl_prologue();
    const uint32_t n = d.a.n, w = threadIdx.x / 32, lane = threadIdx.x % 32, head = blockIdx.y * (blockDim.x / 32) + w;
    uint32_t k, i0, i1;
    if (d.a.prefix == kInvalid) {
        const uint2 job = d.jobs[blockIdx.x];
        if (job.x == kInvalid) return;
        k = job.x; i0 = blockIdx.x; i1 = job.y;
    } else {
        k = blockIdx.x;
        const uint32_t begin = d.ws.cu[k], end = d.ws.cu[k + 1];
        const unsigned long long total = d.ws.cu[n];
        if (begin == end) return;
        const uint32_t P = busy_ctas(d.s, total);
        i0 = (uint32_t)((((unsigned long long)begin + 1) * P - 1) / total);
        i1 = (uint32_t)(((unsigned long long)end * P - 1) / total);
    }
    const uint32_t own = i1 - i0 + 1, parts = own + d.pre_parts;
    if (head >= d.a.q_heads) return;
    auto place = [&](uint32_t i) -> unsigned long long {      // of part i, in units of query heads
        if (i < d.pre_parts) return ((unsigned long long)i * n + k) * d.a.q_heads + head;
        const uint32_t c = i0 + i - d.pre_parts;
        return (unsigned long long)(own == 1 ? 2 * d.s.ctas + k : c == i0 ? 2 * c + 1 : 2 * c) * d.a.q_heads + head;
    };
    auto sums = [&](uint32_t i) { return i < parts ? (i < d.pre_parts ? d.pre.ml : d.own.ml)[place(i)] : make_float2(0.f, 0.f); };
    constexpr uint32_t kFly = 16;
    float4 v[kFly], acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto fetch = [&](uint32_t b) {
#pragma unroll
        for (uint32_t i = 0; i < kFly; ++i)
            if (b + i < parts && lane < D / 4)
                v[i] = *reinterpret_cast<const float4 *>((b + i < d.pre_parts ? d.pre.o : d.own.o) + place(b + i) * D + lane * 4);
    };
    float2 e = sums(lane);
    fetch(0);
    float top = e.y == 0.f ? -INFINITY : e.x;
    for (uint32_t c = 32 + lane; c < parts; c += 32) { const float2 x = sums(c); if (x.y != 0.f) top = fmaxf(top, x.x); }
#pragma unroll
    for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
    float den = 0.f;
    for (uint32_t c = 0; c < parts; c += 32) {
        if (c) e = sums(c + lane);
        const float f = e.y == 0.f ? 0.f : exp2_approx(e.x - top);
        den += e.y * f;
#pragma unroll
        for (uint32_t b = 0; b < 32; b += kFly) {
            if (c + b >= parts) break;
            if (c + b) fetch(c + b);
#pragma unroll
            for (uint32_t i = 0; i < kFly; ++i) {
                const float fi = __shfl_sync(0xFFFFFFFFu, f, b + i);
                if (fi != 0.f) { acc.x += v[i].x * fi; acc.y += v[i].y * fi; acc.z += v[i].z * fi; acc.w += v[i].w * fi; }   // an empty part wrote no sums
            }
        }
    }
#pragma unroll
    for (int x = 16; x; x >>= 1) den += __shfl_xor_sync(0xFFFFFFFFu, den, x);
    const float inv = 1.f / den;
    if (lane < D / 4)
        *reinterpret_cast<uint2 *>(d.a.out + k * d.a.os + ((unsigned long long)head * D + lane * 4) * 2) =
            make_uint2(T::pack(acc.x * inv, acc.y * inv), T::pack(acc.z * inv, acc.w * inv));
    if (d.a.lse && lane == 0) d.a.lse[(unsigned long long)k * d.a.q_heads + head] = top * 0.6931471805599453f + logf(den);
}

Split make_split(const Geom &g, const AttnArgs &a, int n_sms)
{
    Split s = {};
    s.group = a.q_heads / a.kv_heads;
    s.mtiles = (s.group + 15) / 16;
    for (s.heads = kWarps / s.mtiles; a.kv_heads % s.heads; --s.heads) {}
    s.shares = kWarps / (s.heads * s.mtiles);
    s.head_groups = a.kv_heads / s.heads;
    s.box_tokens = g.T % 16 == 0 ? 16 : 8;
    s.stage_bytes = 2 * s.shares * s.heads * 16 * a.head_dim * 2;
    s.stages = min(kRingBytes / s.stage_bytes, (uint32_t)kMaxStages);
    s.ctas = max(1u, (uint32_t)n_sms / s.head_groups);
    return s;
}

template <class T, int D, bool WINDOW>
cudaError_t decode_launch(const Geom &g, const DecodeArgs &d, const CUtensorMap &map, const Launch &l, uint32_t *launched)
{
    cudaError_t e;
    if (d.a.n > kLocalPlanMax) {
        e = launch_pdl(attn_plan_kernel<WINDOW>, dim3(1), dim3(kStepThreads), 0, l.stream, g, d);
        if (e != cudaSuccess) return e;
        *launched += 1;
    }
    const size_t smem = 1024 + d.s.stages * d.s.stage_bytes + (d.a.n <= kLocalPlanMax ? 3 * ((size_t)d.a.n + 1) * 4 : 0);
    e = allow_smem<attn_decode_kernel<T, D, WINDOW>>(l.device, 1024 + kRingBytes + 3 * (kLocalPlanMax + 1) * 4);
    if (e != cudaSuccess) return e;
    e = launch_pdl(attn_decode_kernel<T, D, WINDOW>, dim3(d.s.ctas, d.s.head_groups), dim3(kThreads), smem, l.stream, g, d, map);
    if (e != cudaSuccess) return e;
    *launched += 1;
    const uint32_t jobs = d.a.prefix == kInvalid ? d.s.ctas - 1 : d.a.n;
    if (jobs == 0) return cudaSuccess;
    *launched += 1;
    return launch_pdl(attn_join_kernel<T, D>, dim3(jobs, (d.a.q_heads + 3) / 4), dim3(128), 0, l.stream, d);
}

template <bool WINDOW>
cudaError_t decode_type(const Geom &g, const DecodeArgs &d, const CUtensorMap &map, const Launch &l, uint32_t *launched)
{
    if (d.a.head_dim == 128) return d.a.f16 ? decode_launch<F16, 128, WINDOW>(g, d, map, l, launched) : decode_launch<Bf16, 128, WINDOW>(g, d, map, l, launched);
    return d.a.f16 ? decode_launch<F16, 64, WINDOW>(g, d, map, l, launched) : decode_launch<Bf16, 64, WINDOW>(g, d, map, l, launched);
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

cudaError_t launch_attn_decode(const Geom &g, const AttnArgs &a, const Launch &l, uint32_t *launched)
{
    DecodeArgs d = {};
    d.a = a;
    d.s = make_split(g, a, l.n_sms);
    uint8_t *w = a.ws;
    d.ws.cu = reinterpret_cast<uint32_t *>(w);
    d.ws.req = d.ws.cu + a.n + 1;
    d.ws.len = d.ws.req + a.n;
    w += up256(3 * ((size_t)a.n + 1) * 4);
    d.jobs = reinterpret_cast<uint2 *>(w); w += up256((size_t)d.s.ctas * 8);
    const size_t own = (2 * (size_t)d.s.ctas + a.n) * a.q_heads;
    d.own.ml = reinterpret_cast<float2 *>(w); w += up256(own * 8);
    d.own.o = reinterpret_cast<float *>(w); w += up256(own * a.head_dim * 4);
    CUtensorMap map;
    if (!page_map(&map, g, a.kv_heads, a.head_dim, d.s.box_tokens, d.s.heads)) return cudaErrorNotSupported;
    if (a.prefix != kInvalid) {
        AttnArgs pre = a;
        pre.ws = w;
        const cudaError_t e = launch_attn_prefix(g, pre, l, &d.pre, &d.pre_parts);
        if (e != cudaSuccess) return e;
        *launched += 1;
    }
    return a.window ? decode_type<true>(g, d, map, l, launched) : decode_type<false>(g, d, map, l, launched);
}

size_t attn_ws_bytes(const Geom &g, uint32_t n, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, int n_sms)
{
    const size_t row = (size_t)head_dim * 4 + 8;
    const size_t decode = up256(3 * ((size_t)n + 1) * 4) + up256((size_t)n_sms * 8) + (2 * (size_t)n_sms + n) * q_heads * row + 1024;
    return decode + attn_tile_ws_bytes(g, n, q_heads, kv_heads, head_dim, n_sms);
}

}  // namespace avmp
