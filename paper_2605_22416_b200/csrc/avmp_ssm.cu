// Linear attention with a decay for each head, on the state elements of the SSM blocks in place:
//     S_t = exp(g_t) S_{t-1} + v_t k_t^T,   o_t = S_t q_t        (S: [dv][dk], fp32, one per request and head)
//
// ssm_step_kernel     one token per request: every state element is read once and written once, bound by HBM (1 GB of state:
//                     362 to 382 us, 89 to 94 % of the measured copy rate).
// ssm_prompt_kernel   whole prompts by pieces of 64 tokens: inside a piece the recurrence is two triangular
//                     products, between pieces only the state is carried.  65 521 tokens of 128 heads, dv 64, dk 16: 850 us, 2.7 TB/s
//                     of rows and state; two thirds of the issue slots and shared memory's cycles are taken, and four warps per scheduler
//                     leave the rest to latency: not bound by HBM.  65 536 tokens of 64 heads, dv 64, dk 128 (64 CTAs of two
//                     teams, which wait for each piece's rows): 2 650 us, 15 times what its bytes take.
#include "avmp_tc.cuh"

#include <type_traits>

namespace avmp {

namespace {

// The block of d_reqs[k]'s layer, or null where the slot is dead.
__device__ __forceinline__ float *ssm_block(const Geom &g, const SsmArgs &a, uint32_t r)
{
    uint32_t slot = kInvalid;
    if (r < g.R) {
        const uint32_t state = g.r_state[r], h = g.r_ssm[(unsigned long long)r * g.ns + a.layer];
        if (state == AVMP_REQ_LIVE && h != kInvalid) slot = g.VT[1][h & 0x7FFFFFFFu];
    }
    return slot == kInvalid ? nullptr : reinterpret_cast<float *>(unit_ptr(g, AVMP_POOL_SSM, slot));
}
// Whether an earlier entry of the list names the same slot (two entries would update one state at the same time).  Whole CTA.
__device__ __forceinline__ bool ssm_repeated(const SsmArgs &a, uint32_t k, uint32_t r)
{
    bool dup = false;
    for (uint32_t j = threadIdx.x; j < k; j += blockDim.x) dup |= a.reqs[j] == r;
    return __syncthreads_or(dup);
}
// Both; `report` tells which CTA of an item counts the error.
__device__ __forceinline__ float *ssm_item(const Geom &g, const SsmArgs &a, uint32_t k, bool report)
{
    const uint32_t r = a.reqs[k];
    float *S = ssm_block(g, a, r);
    if (ssm_repeated(a, k, r)) S = nullptr;
    if (!S && report && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
    return S;
}

// ---------------------------------------------------------------- one token
// Division by a number known at launch: a multiply and two shifts (round-up method of Granlund and Montgomery, exact for 32 bits).
struct Divider {
    uint32_t mul, shift, one;      // one: the divisor is 1
    static Divider of(uint32_t d)
    {
        uint32_t l = 0;
        while (l < 32 && (1ull << l) < d) ++l;
        return Divider{(uint32_t)((((1ull << l) - d) << 32) / d + 1), l ? l - 1 : 0, d == 1};
    }
    __device__ uint32_t operator()(uint32_t n) const
    {
        const uint32_t t = __umulhi(mul, n);
        return one ? n : (t + ((n - t) >> 1)) >> shift;
    }
};

constexpr int kStepCta = 128;                     // (256 threads: 391 us, 512: 423)
constexpr uint32_t kStepTile = kStepCta * 4;      // state elements a CTA touches per round (a float4 per thread)
constexpr int kStepRounds = 2;                    // rounds whose loads are in flight together (1 GB of state: 380 us with 1, 372 with 2, 456 with 4)

template <class T, int DK>
__global__ void __launch_bounds__(kStepCta)
ssm_step_kernel(const Geom g, const SsmArgs a, uint32_t parts, uint32_t part_elems, const Divider by_dv, const Divider by_rep)
{
    constexpr int LANES = DK / 4;                 // lanes that share a state row
    pdl_prologue();
    const uint32_t k = blockIdx.x / parts, part = blockIdx.x % parts;
    const uint32_t r = a.reqs[k];
    float *S = ssm_block(g, a, r);
    const uint32_t elems = a.heads * a.dv * DK;
    const uint32_t end = min(elems, (part + 1) * part_elems), own = threadIdx.x * 4;
    const uint8_t *qrow = a.q + k * a.qs, *krow = a.k + k * a.ks;
    const uint16_t *vrow = reinterpret_cast<const uint16_t *>(a.v + k * a.vs);
    const float *grow = reinterpret_cast<const float *>(a.g + k * a.gs);
    uint16_t *orow = reinterpret_cast<uint16_t *>(a.out + k * a.os);
    const uint32_t col = own % DK;
    bool checked = false;
    for (uint32_t e0 = part * part_elems; e0 < end; e0 += kStepTile * kStepRounds) {
        float4 s[kStepRounds];
#pragma unroll
        for (int u = 0; u < kStepRounds; ++u) {
            const uint32_t e = e0 + own + u * kStepTile;
            if (S && e < end) s[u] = *reinterpret_cast<const float4 *>(S + e);
        }
        if (!checked) {      // while the first loads are on their way
            if (ssm_repeated(a, k, r) || !S) {
                if (part == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
                return;
            }
            checked = true;
        }
#pragma unroll
        for (int u = 0; u < kStepRounds; ++u) {
            const uint32_t e = e0 + own + u * kStepTile;
            float acc = 0.f;
            uint32_t row = 0;
            if (e < end) {
                row = e / DK;
                const uint32_t head = by_dv(row), grp = by_rep(head);
                const uint2 kk = *reinterpret_cast<const uint2 *>(krow + (grp * DK + col) * 2);
                const uint2 qq = *reinterpret_cast<const uint2 *>(qrow + (grp * DK + col) * 2);
                const float2 k0 = T::unpack(kk.x), k1 = T::unpack(kk.y), q0 = T::unpack(qq.x), q1 = T::unpack(qq.y);
                const float v = T::unpack(vrow[row]).x, w = exp2_approx(grow[head] * 1.4426950408889634f);
                // w == 0 clears the state, whatever it held
                s[u].x = w == 0.f ? v * k0.x : fmaf(w, s[u].x, v * k0.x);
                s[u].y = w == 0.f ? v * k0.y : fmaf(w, s[u].y, v * k0.y);
                s[u].z = w == 0.f ? v * k1.x : fmaf(w, s[u].z, v * k1.x);
                s[u].w = w == 0.f ? v * k1.y : fmaf(w, s[u].w, v * k1.y);
                *reinterpret_cast<float4 *>(S + e) = s[u];
                acc = s[u].x * q0.x + s[u].y * q0.y + s[u].z * q1.x + s[u].w * q1.y;
            }
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
            if (e < end && col == 0) orow[row] = (uint16_t)T::pack(acc, 0.f);
        }
    }
}

// ---------------------------------------------------------------- whole prompts
// One CTA per (request, head, 64 or 32 columns of dv).  Inside a piece of 64 tokens with running decays c_i,
//     O = ((Q K^T) o D) V + diag(e^c) Q S^T,  D_ij = e^(c_i - c_j) for j <= i,
//     S <- e^(c_64) S + sum_j e^(c_64 - c_j) v_j k_j^T.
// Only the last line is sequential, and of it only the scaled sum: NT teams of four warps take the pieces in turn,
// each works out its own products and waits for its predecessor's state alone, so that the loads, products and
// exponentials of NT pieces overlap.  A named barrier per team carries the hand-over; there is no spinning.
// What is rounded to 16 bits: the scores after their decay and the state as an operand of Q S^T (both enter an output
// that is rounded to 16 bits itself).  The state's own update keeps 32 bits: e^(..) v_j is split into
// 16-bit parts, two for fp16 and three for bf16 (k_j has 16 bits to begin with), 2^-23 relative, and summed in 32 bits.
// Where requests, heads and columns leave SMs idle, each prompt is cut into `shares` runs of pieces. A first pass works out
// each run's final state from zero (the first run's from the state in the block) and its whole decay, a second one starts
// every run from the states of those before it.
// fp16 has little range: its scores (per row) and states and updates (per 16 rows of S) carry a power of two each.
// A product takes in rows that count for nothing with a weight of zero, and 0 x NaN and 0 x inf are NaN; the parts of an infinite
// e^(..) v are inf - inf.  Every row of V and K enters some warp's update, so an update that is not finite shows a piece with such a
// row: its update and its output rows are then worked out again token by token, as the recurrence is written (walk_state, walk_rows).
// The look at the updates costs 3 to 8 % (the two prompts above: 826 and 2 520 us without).
constexpr int kC = 64;                            // tokens per piece

template <int DK, int DVT, int NT>
struct PromptSmem {
    // A stage holds the rows as tiled copies leave them, their 16-byte units permuted against bank conflicts (see `unit`);
    // everything else has rows of an odd number of 16-byte units.
    static constexpr int kRowK = DK < 64 ? DK * 2 : 128, kBlocksK = DK == 128 ? 2 : 1;   // 128 columns: two blocks of 64
    static constexpr int kRowV = DVT * 2;
    static constexpr int kStageV = 0, kStageQ = kC * kRowV, kStageK = kStageQ + kC * DK * 2, kStageG = kStageK + kC * DK * 2;
    static constexpr int kStage = (kStageG + kC * 4 + 1023) / 1024 * 1024;
    static constexpr int kQ = DK * 2 + 16, kV = DVT * 2 + 16;
    static constexpr int kBufs = DK == 128 ? 1 : 2;          // loads run a team's next piece ahead where the memory allows it
    static constexpr int kRing = NT + 2;          // copies of the state in 16 bits: see the hand-over
    static constexpr int kS = DVT * kQ;
    static constexpr int kO = kC * kV;            // output staging
    static constexpr int kF = DVT * DK * 4;       // the state in 32 bits, thread-private places
    static constexpr int kW = kC * 2 * 4;         // running decays and tail weights, of this piece and the team's next
    static constexpr int oStage = 0;
    static constexpr int oS = oStage + NT * kBufs * kStage;
    static constexpr int oO = oS + kRing * kS;
    static constexpr int oF = oO + NT * kO;
    static constexpr int oW = oF + kF;
    static constexpr int oScale = oW + NT * 2 * kW;
    static constexpr int oBars = oScale + kRing * 4 * 4;
    static constexpr int kTotal = oBars + NT * kBufs * 8 + 1024;
};

// Place of 16-byte unit c of row r where rows of ROW bytes were copied with the swizzle of that width.
template <int ROW>
__device__ __forceinline__ uint32_t unit(uint32_t r, uint32_t c)
{
    const uint32_t x = ROW == 128 ? r & 7 : ROW == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
    return r * ROW + ((c ^ x) << 4);
}

// A power of two that brings `m` (>= 0) to about 2^13; 1 for zero.
__device__ __forceinline__ float pow2_to_2_13(float m)
{
    int e = (int)(__float_as_uint(m) >> 23) - 127;
    if (m == 0.f) e = 13;
    e = max(-60, min(60, 13 - e));
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

template <int DK>
__device__ __forceinline__ uint32_t place_k(uint32_t r, uint32_t c)        // 16-byte unit c of a row of Q or K in a stage
{
    constexpr int kRowK = DK < 64 ? DK * 2 : 128;
    return DK == 128 ? (c >> 3) * (kC * 128) + unit<128>(r, c & 7) : unit<kRowK>(r, c);
}

// A piece's update token by token, for 16 rows of the state from `d` on: F (this thread's places in it, `pitch` apart) from the
// state in front to the one behind.  Returns the decay over the piece.  Whole warp; not inlined, so that its registers cost nothing elsewhere.
template <class T, class L, int DK, int DVT>
__device__ __noinline__ float walk_state(const uint8_t *st, uint32_t tokens, uint32_t d, float *F, uint32_t pitch)
{
    const uint32_t lane = threadIdx.x % 32, lc = (lane & 3) * 2;
    const float *g = reinterpret_cast<const float *>(st + L::kStageG);
    float over = 1.f;
    d += lane >> 2;
    for (uint32_t t = 0; t < tokens; ++t) {
        const float w = exp2_approx(g[t] * 1.4426950408889634f);
        const uint8_t *row = st + L::kStageV + (d & 7) * 2;
        const float v0 = T::unpack(*reinterpret_cast<const uint16_t *>(row + unit<L::kRowV>(t, d >> 3))).x;
        const float v1 = T::unpack(*reinterpret_cast<const uint16_t *>(row + unit<L::kRowV>(t, (d >> 3) + 1))).x;
#pragma unroll 1
        for (uint32_t n = 0; n < DK / 8; ++n) {
            const float2 k = T::unpack(*reinterpret_cast<const uint32_t *>(st + L::kStageK + place_k<DK>(t, n) + lc * 2));
            const float add[4] = {v0 * k.x, v0 * k.y, v1 * k.x, v1 * k.y};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                float *f = F + (n * 4 + i) * pitch;
                *f = w == 0.f ? add[i] : fmaf(w, *f, add[i]);
            }
        }
        over = w == 0.f ? 0.f : over * w;
    }
    return over;
}

// Output rows row0 .. row1 of a piece, each from the last token it sees backwards to a reset or to the state in front of the
// piece (its 16-bit copy sb, with the factors sc); into `so`.  Whole warp.
template <class T, class L, int DK, int DVT>
__device__ __noinline__ void walk_rows(const uint8_t *st, const uint8_t *sb, const float *sc, uint32_t row0, uint32_t row1, uint8_t *so)
{
    const uint32_t lane = threadIdx.x % 32;
    const float *g = reinterpret_cast<const float *>(st + L::kStageG);
    auto number = [](const uint8_t *unit_at, uint32_t c) { return T::unpack(*reinterpret_cast<const uint16_t *>(unit_at + (c & 7) * 2)).x; };
    for (uint32_t r = row0; r < row1; ++r, so += L::kV) {
        float acc[DVT / 32] = {}, weight = 1.f;
        for (int j = (int)r; j >= 0 && weight != 0.f; --j) {
            float s = 0.f;
            for (uint32_t c = lane; c < DK; c += 32)
                s += number(st + L::kStageQ + place_k<DK>(r, c >> 3), c) * number(st + L::kStageK + place_k<DK>(j, c >> 3), c);
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
#pragma unroll
            for (uint32_t x = 0; x < DVT / 32; ++x)
                acc[x] += s * weight * number(st + L::kStageV + unit<L::kRowV>(j, (lane + x * 32) >> 3), lane);
            const float w = exp2_approx(g[j] * 1.4426950408889634f);
            weight = w == 0.f ? 0.f : weight * w;
        }
#pragma unroll
        for (uint32_t x = 0; x < DVT / 32; ++x) {
            const uint32_t d = lane + x * 32;
            if (weight != 0.f) {
                float s = 0.f;
                for (uint32_t c = 0; c < DK; ++c) s += number(st + L::kStageQ + place_k<DK>(r, c >> 3), c) * number(sb + d * L::kQ + (c >> 3) * 16, c);
                acc[x] += weight * s * (T::kF16 ? sc[d >> 4] : 1.f);
            }
            *reinterpret_cast<uint16_t *>(so + d * 2) = (uint16_t)T::pack(acc[x], 0.f);
        }
    }
}

template <class T, int DK, int DVT, int NT>
__global__ void __launch_bounds__(NT * 128, NT == 2 && DK == 16 ? 2 : 1)
ssm_prompt_kernel(const Geom g, const SsmArgs a, uint32_t tiles, uint32_t shares, bool locals, const __grid_constant__ CUtensorMap q_map,
                  const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    using L = PromptSmem<DK, DVT, NT>;
    constexpr int KS = DK / 16;                   // k-steps of a product over dk
    constexpr int NV = DVT / 8;                   // 8-column tiles of the output
    constexpr int ND = DK / 8;                    // 8-column tiles of the state
    constexpr int WM = DVT / 16;                  // warps of a team that own 16 rows of the state each
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint32_t gave_up;
    __shared__ float decayed;
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    if (threadIdx.x == 0) {
        gave_up = 0;
        decayed = 1.f;
        for (int i = 0; i < NT * L::kBufs; ++i) mbar_init(smem_u32(smem + L::oBars) + 8 * i, 1);
        mbar_fence_init();
    }
    pdl_prologue();
    const uint32_t per_req = a.heads * tiles;
    // the first pass needs no last run
    const uint32_t runs = locals ? shares - 1 : shares, run = blockIdx.x % runs, item = blockIdx.x / runs;
    const uint32_t k = item / per_req, head = (item % per_req) / tiles, tile = item % tiles;
    const bool lead = item % per_req == 0 && run == 0 && !locals;
    float *S = ssm_item(g, a, k, lead);
    if (!S) return;
    uint32_t row0 = a.cu[k];
    const uint32_t row1 = a.cu[k + 1];
    if (row1 < row0 || row1 > a.total) {
        if (lead && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
        return;
    }
    uint32_t len = row1 - row0, pieces = (len + kC - 1) / kC;
    const bool last = run + 1 == shares;
    if (shares > 1) {
        const uint32_t p0 = (uint32_t)((unsigned long long)pieces * run / shares), p1 = (uint32_t)((unsigned long long)pieces * (run + 1) / shares);
        row0 += p0 * kC;
        len = min(len - p0 * kC, (p1 - p0) * kC);
        pieces = p1 - p0;
    }
    const bool resume = a.resume && a.resume[k];
    const uint32_t grp = head / (a.heads / a.groups);
    const int team = threadIdx.x / 128, tid = threadIdx.x % 128, w = tid / 32, lane = tid % 32;
    const int lr = lane >> 2, lc = (lane & 3) * 2;
    const Waits waits{&gave_up, a.wait};
    uint32_t loads = 0;                                    // pieces of this team whose rows have been asked for (first thread)
    uint8_t *stage0 = smem + L::oStage + team * L::kBufs * L::kStage;
    float *F = reinterpret_cast<float *>(smem + L::oF);
    float *decays = reinterpret_cast<float *>(smem + L::oW + team * 2 * L::kW);
    float *sscale = reinterpret_cast<float *>(smem + L::oScale);
    S += ((unsigned long long)head * a.dv + tile * DVT) * DK;
    // workspace: [item][share] states, then decays.  The last share's place keeps the state that the first run starts from (the
    // last run of the second pass may replace the block's before the first one reads it).
    float *place = a.ws + (unsigned long long)item * shares * DVT * DK;
    float *decays_out = a.ws + (unsigned long long)(gridDim.x / runs) * shares * DVT * DK + (unsigned long long)item * shares;
    float *to = locals ? place + run * DVT * DK : last ? S : nullptr;

    constexpr int CV = DVT / 8;                            // 16-byte units per row of the output
    const unsigned long long own_row = row0 + (unsigned long long)team * kC;
    const uint8_t *gg = a.g + (own_row + 2 * lane) * a.gs + head * 4;       // two decays a lane of the first warp
    uint8_t *og = a.out + (own_row + w * 16 + lane / CV) * a.os + ((unsigned long long)head * a.dv + tile * DVT) * 2 + lane % CV * 16;
    const unsigned long long g_next = (unsigned long long)NT * kC * a.gs;
    const uint32_t bars = smem_u32(smem + L::oBars) + 8 * team * L::kBufs;

    // Piece p of this team (called for p = team, team + NT, ... in turn): rows by tiled copies, decays by small ones.  Rows behind
    // the request's last are the next request's, or zeros behind the last of all: see the last piece.
    auto load = [&](uint32_t p, int buf) {
        if (p < pieces) {
            const uint32_t base = smem_u32(stage0 + buf * L::kStage), left = len - p * kC, row = row0 + p * kC;
            if (tid == 0 && !waits.over()) {               // (nothing is copied on top of what may still be in flight)
                loads += 1;
                mbar_expect(bars + 8 * buf, kC * (DVT + 2 * DK) * 2);
                tma_load_tile(base + L::kStageV, &v_map, bars + 8 * buf, head * a.dv + tile * DVT, row);
#pragma unroll
                for (int x = 0; x < L::kBlocksK; ++x) {
                    tma_load_tile(base + L::kStageQ + x * kC * 128, &q_map, bars + 8 * buf, grp * DK + x * 64, row);
                    tma_load_tile(base + L::kStageK + x * kC * 128, &k_map, bars + 8 * buf, grp * DK + x * 64, row);
                }
            }
            if (w == 0)
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i) {
                    const bool ok = 2 * lane + i < left;
                    cp_async4(base + L::kStageG + (2 * lane + i) * 4, ok ? gg + i * a.gs : a.g, ok);
                }
            gg += g_next;
        }
        cp_async_commit();
    };

    // First warp: running sums in units of log2, from the front for the decays, from the back for the tail weights (the weights
    // of the state keep their relative precision that way).
    auto scan = [&](const float *gs, float *cs) {
        float *wt = cs + kC;
        constexpr float kLog2e = 1.4426950408889634f;
        float g0 = gs[2 * lane] * kLog2e, g1 = gs[2 * lane + 1] * kLog2e;
        // 2^-300 is 0 in 32 bits; -inf itself would make differences of sums undefined
        g0 = g0 < -300.f ? -300.f : g0; g1 = g1 < -300.f ? -300.f : g1;
        float f = g0 + g1, b = f;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const float x = __shfl_up_sync(0xFFFFFFFFu, f, o), y = __shfl_down_sync(0xFFFFFFFFu, b, o);
            if (lane >= o) f += x;
            if (lane + o < 32) b += y;
        }
        float b_next = __shfl_down_sync(0xFFFFFFFFu, b, 1);
        if (lane == 31) b_next = 0.f;
        float f_prev = __shfl_up_sync(0xFFFFFFFFu, f, 1);
        if (lane == 0) f_prev = 0.f;
        cs[2 * lane] = f_prev + g0; cs[2 * lane + 1] = f;
        wt[2 * lane] = exp2_approx(b_next + g1); wt[2 * lane + 1] = exp2_approx(b_next);
    };
    // Publishes a state fragment as the 16-bit operand of piece p.
    auto publish = [&](const float (&f)[ND][4], uint32_t p) {
        const uint32_t slot = p % L::kRing;
        uint8_t *sb = smem + L::oS + slot * L::kS;
        float sc = 1.f;
        if (T::kF16) {
            float m = 0.f;
#pragma unroll
            for (int n = 0; n < ND; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) m = fmaxf(m, fabsf(f[n][i]));
            m = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m)));
            if (m == INFINITY) {            // it would scale the numbers beside it to nothing
                m = 0.f;
#pragma unroll
                for (int n = 0; n < ND; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) m = fmaxf(m, fabsf(f[n][i]) < INFINITY ? fabsf(f[n][i]) : 0.f);
                m = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m)));
            }
            sc = pow2_to_2_13(m);
            if (lane == 0) sscale[slot * 4 + w] = 1.f / sc;
        }
#pragma unroll
        for (int n = 0; n < ND; ++n) {
            *reinterpret_cast<uint32_t *>(sb + (w * 16 + lr) * L::kQ + (n * 8 + lc) * 2) = T::pack(f[n][0] * sc, f[n][1] * sc);
            *reinterpret_cast<uint32_t *>(sb + (w * 16 + lr + 8) * L::kQ + (n * 8 + lc) * 2) = T::pack(f[n][2] * sc, f[n][3] * sc);
        }
    };
    // This warp's rows of piece p, whole 16-byte units.
    auto rows_out = [&](uint32_t p, const uint8_t *so) {
#pragma unroll
        for (int i = 0; i < 16 * CV / 32; ++i) {
            const uint32_t t = lane / CV + i * (32 / CV);
            if (p * kC + w * 16 + t < len)
                *reinterpret_cast<uint4 *>(og + i * (32 / CV) * a.os) = *reinterpret_cast<const uint4 *>(so + t * L::kV + lane % CV * 16);
        }
    };
    auto put = [&](float *to, const float (&f)[ND][4]) {
#pragma unroll
        for (int n = 0; n < ND; ++n) {
            *reinterpret_cast<float2 *>(to + (w * 16 + lr) * DK + n * 8 + lc) = make_float2(f[n][0], f[n][1]);
            *reinterpret_cast<float2 *>(to + (w * 16 + lr + 8) * DK + n * 8 + lc) = make_float2(f[n][2], f[n][3]);
        }
    };
    auto get = [&](const float *from, float (&f)[ND][4]) {
#pragma unroll
        for (int n = 0; n < ND; ++n) {
            const float2 x = *reinterpret_cast<const float2 *>(from + (w * 16 + lr) * DK + n * 8 + lc);
            const float2 y = *reinterpret_cast<const float2 *>(from + (w * 16 + lr + 8) * DK + n * 8 + lc);
            f[n][0] = x.x; f[n][1] = x.y; f[n][2] = y.x; f[n][3] = y.y;
        }
    };
    auto store_state = [&](const float (&f)[ND][4]) {
        if (to) put(to, f);
        if (locals && w == 0 && lane == 0) decays_out[run] = decayed;
    };

    __syncthreads();
    for (int i = 0; i < (L::kBufs > 1 ? L::kBufs - 1 : 1); ++i) load(team + i * NT, i);
    if (team == 0 && w < WM) {
        float f[ND][4];
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[n][i] = 0.f;
        if (shares == 1 || locals) {
            if (resume && run == 0) get(S, f);
            if (locals && run == 0) put(place + (shares - 1) * DVT * DK, f);
        } else {
            get(place + (run ? 0 : shares - 1) * DVT * DK, f);
            for (uint32_t j = 1; j < run; ++j) {
                float x[ND][4];
                get(place + j * DVT * DK, x);
                const float d = decays_out[j];
#pragma unroll
                for (int n = 0; n < ND; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) f[n][i] = d == 0.f ? x[n][i] : fmaf(d, f[n][i], x[n][i]);
            }
        }
#pragma unroll
        for (int n = 0; n < ND; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) F[(n * 4 + i) * (WM * 32) + tid] = f[n][i];
        publish(f, 0);
        if (pieces == 0) store_state(f);
    }
    if (L::kBufs > 1 && w == 0) {          // the first piece's decays; later ones are worked out a piece ahead
        cp_async_wait<0>();
        __syncwarp();
        scan(reinterpret_cast<const float *>(stage0 + L::kStageG), decays);
    }
    __syncthreads();

    static_assert(NT >= 2, "the hand-over goes from one team to another");
    constexpr int kTeamBar = 1 + NT;
    int buf = 0;
    uint32_t round = 0;
    bool there = true;
    for (uint32_t p = team; p < pieces; p += NT, ++round) {
        if (L::kBufs > 1) load(p + (L::kBufs - 1) * NT, (buf + L::kBufs - 1) % L::kBufs);
        uint8_t *st = stage0 + buf * L::kStage;
        const uint32_t sq = smem_u32(st + L::kStageQ), sk = smem_u32(st + L::kStageK), sv = smem_u32(st + L::kStageV);
        // a copy that does not land in time is reported and none is waited for again; the barriers between the teams are still kept
        if (there) there = mbar_wait(bars + 8 * buf, round / L::kBufs & 1, waits);
        if (len - p * kC < kC) {
            // behind the request's last row: zeros, as a weight of zero does not silence a NaN
            constexpr int C = (L::kRowV + 2 * DK * 2) / 16;
            const uint32_t gone = kC - (len - p * kC);
            for (uint32_t i = tid; i < gone * C; i += 128) {
                const uint32_t r = len - p * kC + i / C, c = i % C;
                // (whole rows are cleared, so the order of their units does not matter)
                uint8_t *to = c < L::kRowV / 16 ? st + L::kStageV + r * L::kRowV + c * 16
                                                : st + L::kStageQ + (c - L::kRowV / 16) / (L::kRowK / 16) * (kC * L::kRowK) + r * L::kRowK + (c - L::kRowV / 16) % (L::kRowK / 16) * 16;
                *reinterpret_cast<uint4 *>(to) = make_uint4(0, 0, 0, 0);
            }
        }
        float *cs = decays + (L::kBufs > 1 ? (round & 1) * 2 * kC : 0), *wt = cs + kC;
        if (L::kBufs == 1 && w == 0) {
            cp_async_wait<0>();
            __syncwarp();
            scan(reinterpret_cast<const float *>(st + L::kStageG), cs);
        }
        if (L::kBufs == 1 || len - p * kC < kC) bar_sync(kTeamBar + team, 128);

        // ---- scores of this warp's 16 rows.  Against earlier blocks of 16 tokens the decay is a row factor, from the block's
        // front c_ref on, times a column factor up to it (both at most 1); inside the own block it is one per pair.
        uint32_t aq[KS][4];
#pragma unroll
        for (int s = 0; s < KS; ++s) ldsm4(aq[s], sq + place_k<DK>(w * 16 + (lane & 15), s * 2 + (lane >> 4)));
        const float c0 = cs[w * 16 + lr], c1 = cs[w * 16 + lr + 8], cref = w ? cs[w * 16 - 1] : 0.f;
        auto score = [&](int j, float (&x)[2][4]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[0][i] = x[1][i] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                uint32_t b[4];
                ldsm4(b, sk + place_k<DK>(j * 16 + (lane & 7) + ((lane >> 4) << 3), s * 2 + ((lane >> 3) & 1)));
                T::mma(x[0], aq[s], b[0], b[1]);
                T::mma(x[1], aq[s], b[2], b[3]);
            }
        };
        auto weigh = [&](const uint32_t (&pa)[4], int j, float (&o)[NV][4]) {
#pragma unroll
            for (int n = 0; n < NV / 2; ++n) {
                uint32_t b[4];
                ldsm4_t(b, sv + unit<L::kRowV>(j * 16 + (lane & 15), n * 2 + (lane >> 4)));
                T::mma(o[2 * n], pa, b[0], b[1]);
                T::mma(o[2 * n + 1], pa, b[2], b[3]);
            }
        };
        auto row_scale = [&](float m0, float m1, float &s0, float &s1) {      // fp16: scores of a row brought to 2^13
#pragma unroll
            for (int x = 1; x < 4; x <<= 1) {
                m0 = fmaxf(m0, __shfl_xor_sync(0xFFFFFFFFu, m0, x));
                m1 = fmaxf(m1, __shfl_xor_sync(0xFFFFFFFFu, m1, x));
            }
            s0 = pow2_to_2_13(m0); s1 = pow2_to_2_13(m1);
        };
        float o[NV][4];
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
        uint32_t own[4];                               // weights of the own block
        float so0 = 1.f, so1 = 1.f, sd0 = 1.f, sd1 = 1.f;
        // (compiled for each warp of the team on its own: as a loop up to w its blocks ran one after the other)
        auto scores = [&](auto which) {
            constexpr int W = decltype(which)::value;
            float x[W + 1][2][4], m0 = 0.f, m1 = 0.f, d0 = 0.f, d1 = 0.f;
#pragma unroll
            for (int j = 0; j <= W; ++j) score(j, x[j]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = h * 8 + lc;
                float *y = x[W][h];
                const float2 ct = *reinterpret_cast<const float2 *>(cs + W * 16 + t);
                y[0] = t <= lr ? y[0] * exp2_approx(c0 - ct.x) : 0.f;
                y[1] = t + 1 <= lr ? y[1] * exp2_approx(c0 - ct.y) : 0.f;
                y[2] = t <= lr + 8 ? y[2] * exp2_approx(c1 - ct.x) : 0.f;
                y[3] = t + 1 <= lr + 8 ? y[3] * exp2_approx(c1 - ct.y) : 0.f;
                if (T::kF16) { d0 = fmaxf(d0, fmaxf(fabsf(y[0]), fabsf(y[1]))); d1 = fmaxf(d1, fmaxf(fabsf(y[2]), fabsf(y[3]))); }
            }
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float2 ct = *reinterpret_cast<const float2 *>(cs + j * 16 + h * 8 + lc);
                    const float f0 = exp2_approx(cref - ct.x), f1 = exp2_approx(cref - ct.y);
                    float *y = x[j][h];
                    y[0] *= f0; y[1] *= f1; y[2] *= f0; y[3] *= f1;
                    if (T::kF16) { m0 = fmaxf(m0, fmaxf(fabsf(y[0]), fabsf(y[1]))); m1 = fmaxf(m1, fmaxf(fabsf(y[2]), fabsf(y[3]))); }
                }
            if (T::kF16) { row_scale(d0, d1, sd0, sd1); if (W) row_scale(m0, m1, so0, so1); }
#pragma unroll
            for (int h = 0; h < 2; ++h) { own[2 * h] = T::pack(x[W][h][0] * sd0, x[W][h][1] * sd0); own[2 * h + 1] = T::pack(x[W][h][2] * sd1, x[W][h][3] * sd1); }
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const uint32_t pa[4] = {T::pack(x[j][0][0] * so0, x[j][0][1] * so0), T::pack(x[j][0][2] * so1, x[j][0][3] * so1),
                                        T::pack(x[j][1][0] * so0, x[j][1][1] * so0), T::pack(x[j][1][2] * so1, x[j][1][3] * so1)};
                weigh(pa, j, o);
            }
        };
        if (locals) {}                             // states alone are wanted
        else if (w == 0) scores(std::integral_constant<int, 0>{});
        else if (w == 1) scores(std::integral_constant<int, 1>{});
        else if (w == 2) scores(std::integral_constant<int, 2>{});
        else scores(std::integral_constant<int, 3>{});

        // ---- this piece's own contribution to the state (16 rows of dv per owning warp)
        float ds[ND][4];
        float dinv = 1.f;
        if (w < WM) {
            float xs = 1.f;
            if (T::kF16) {
                float m = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t v[4];
                    ldsm4_t(v, sv + unit<L::kRowV>(j * 16 + (lane & 7) + ((lane >> 4) << 3), w * 2 + ((lane >> 3) & 1)));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 x = T::unpack(v[i]), y = *reinterpret_cast<const float2 *>(wt + j * 16 + (i >> 1) * 8 + lc);
                        m = fmaxf(m, fmaxf(fabsf(x.x * y.x), fabsf(x.y * y.y)));
                    }
                }
                m = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(m)));
                xs = pow2_to_2_13(m);
                dinv = 1.f / xs;
            }
            // the parts' products are summed apart (short dependent chains) where registers allow it
            constexpr int kSums = ND <= 4 ? (T::kF16 ? 2 : 3) : 1;
            float part[kSums][ND][4];
#pragma unroll
            for (int y = 0; y < kSums; ++y)
#pragma unroll
                for (int n = 0; n < ND; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[y][n][i] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t v[4], x3[3][4];
                ldsm4_t(v, sv + unit<L::kRowV>(j * 16 + (lane & 7) + ((lane >> 4) << 3), w * 2 + ((lane >> 3) & 1)));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 x = T::unpack(v[i]);
                    const float2 y = *reinterpret_cast<const float2 *>(wt + j * 16 + (i >> 1) * 8 + lc);
                    x.x *= y.x * xs; x.y *= y.y * xs;
                    x3[0][i] = T::pack(x.x, x.y);
                    const float2 h = T::unpack(x3[0][i]);
                    x.x -= h.x; x.y -= h.y;
                    x3[1][i] = T::pack(x.x, x.y);
                    const float2 m = T::unpack(x3[1][i]);
                    x3[2][i] = T::pack(x.x - m.x, x.y - m.y);
                }
#pragma unroll
                for (int n = 0; n < ND / 2; ++n) {
                    uint32_t b[4];
                    ldsm4_t(b, sk + place_k<DK>(j * 16 + (lane & 15), n * 2 + (lane >> 4)));
#pragma unroll
                    for (int y = 0; y < (T::kF16 ? 2 : 3); ++y) {
                        T::mma(part[y % kSums][2 * n], x3[y], b[0], b[1]);
                        T::mma(part[y % kSums][2 * n + 1], x3[y], b[2], b[3]);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < ND; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    ds[n][i] = part[kSums - 1][n][i];
#pragma unroll
                    for (int y = kSums - 2; y >= 0; --y) ds[n][i] += part[y][n][i];
                }
        }

        if (L::kBufs > 1 && w == 0 && p + NT < pieces) {      // the team's next piece, while the other warps have more rows to see
            cp_async_wait<0>();
            __syncwarp();
            scan(reinterpret_cast<const float *>(stage0 + (buf ^ 1) * L::kStage + L::kStageG), decays + ((round + 1) & 1) * 2 * kC);
        }

        // ---- hand-over: wait for the state in front of this piece, pass the one behind it on at once
        if (p > 0) bar_sync(1 + team, 256);
        bool odd = false;                              // the update is not finite
        if (w < WM) {
            float dec = exp2_approx(cs[kC - 1]), mark = cs[kC - 1] * 0.f;        // 0, or NaN once a number is not finite
#pragma unroll
            for (int n = 0; n < ND; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) mark = fmaf(ds[n][i], 0.f, mark);
            odd = __any_sync(0xFFFFFFFFu, mark != 0.f);
#pragma unroll
            for (int n = 0; n < ND; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float *f = F + (n * 4 + i) * (WM * 32) + tid;
                    const float add = T::kF16 ? ds[n][i] * dinv : ds[n][i];
                    ds[n][i] = dec == 0.f ? add : fmaf(dec, *f, add);
                    if (!odd) *f = ds[n][i];
                }
            if (odd) {
                dec = walk_state<T, L, DK, DVT>(st, min((uint32_t)kC, len - p * kC), w * 16, F + tid, WM * 32);
#pragma unroll
                for (int n = 0; n < ND; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) ds[n][i] = F[(n * 4 + i) * (WM * 32) + tid];
            }
            if (locals && w == 0 && lane == 0) decayed = dec == 0.f ? 0.f : decayed * dec;
            if (p + 1 < pieces) publish(ds, p + 1); else store_state(ds);
        }
        if (p + 1 < pieces) bar_arrive(1 + (team + 1) % NT, 256);

        if (!locals) {
            // ---- what the earlier pieces add to the outputs
            // r * (earlier blocks + e^c_ref Q S^T), then the own block on top
            const float r0 = exp2_approx(c0 - cref), r1 = exp2_approx(c1 - cref), er = exp2_approx(cref);
            const float z0 = r0 * sd0 / so0, z1 = r1 * sd1 / so1, y0 = r0 * sd0 * er, y1 = r1 * sd1 * er;
            const uint32_t sb = smem_u32(smem + L::oS + (p % L::kRing) * L::kS);
#pragma unroll
            for (int n = 0; n < NV / 2; ++n) {
                float x[2][4] = {};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    uint32_t b[4];
                    ldsm4(b, sb + (n * 16 + (lane & 7) + ((lane >> 4) << 3)) * L::kQ + s * 32 + ((lane >> 3) & 1) * 16);
                    T::mma(x[0], aq[s], b[0], b[1]);
                    T::mma(x[1], aq[s], b[2], b[3]);
                }
                const float sc = T::kF16 ? sscale[(p % L::kRing) * 4 + n] : 1.f;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // a cleared state adds nothing, whatever it held
                    float *y = o[2 * n + h];
                    y[0] = fmaf(y[0], z0, y0 == 0.f ? 0.f : x[h][0] * (y0 * sc)); y[1] = fmaf(y[1], z0, y0 == 0.f ? 0.f : x[h][1] * (y0 * sc));
                    y[2] = fmaf(y[2], z1, y1 == 0.f ? 0.f : x[h][2] * (y1 * sc)); y[3] = fmaf(y[3], z1, y1 == 0.f ? 0.f : x[h][3] * (y1 * sc));
                }
            }
            weigh(own, w, o);
            if (T::kF16) {
                const float i0 = 1.f / sd0, i1 = 1.f / sd1;
#pragma unroll
                for (int n = 0; n < NV; ++n) { o[n][0] *= i0; o[n][1] *= i0; o[n][2] *= i1; o[n][3] *= i1; }
            }
            // ---- rows out
            uint8_t *so = smem + L::oO + team * L::kO + w * 16 * L::kV;
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                *reinterpret_cast<uint32_t *>(so + lr * L::kV + (n * 8 + lc) * 2) = T::pack(o[n][0], o[n][1]);
                *reinterpret_cast<uint32_t *>(so + (lr + 8) * L::kV + (n * 8 + lc) * 2) = T::pack(o[n][2], o[n][3]);
            }
            __syncwarp();
            rows_out(p, so);
        }
        if (bar_or(kTeamBar + team, 128, odd) && !locals) {
            uint8_t *so = smem + L::oO + team * L::kO + w * 16 * L::kV;
            walk_rows<T, L, DK, DVT>(st, smem + L::oS + (p % L::kRing) * L::kS, sscale + (p % L::kRing) * 4, w * 16,
                                     min((uint32_t)w * 16 + 16, len - p * kC), so);
            __syncwarp();
            rows_out(p, so);
            bar_sync(kTeamBar + team, 128);
        }
        // the stage may be filled again, the next decays are there
        og += (unsigned long long)NT * kC * a.os;
        buf = (buf + 1) % L::kBufs;
        if (L::kBufs == 1) load(p + NT, 0);
    }
    cp_async_wait<0>();
    __syncthreads();
    if (threadIdx.x == 0 && waits.over()) record_error(g.st, AVMP_DEV_TIMEOUT);
    if (tid == 0 && waits.over())          // copies in flight land before this CTA's memory is given away
        for (uint32_t i = loads > (uint32_t)L::kBufs ? loads - L::kBufs : 0; i < loads; ++i) mbar_land(bars + 8 * (i % L::kBufs), i / L::kBufs & 1);
}

template <class T, int DK>
cudaError_t step_dk(const Geom &g, const SsmArgs &a, const Launch &l)
{
    // Parts of 16 rounds (64 KB) amortise the look-ups of a CTA; smaller ones where that leaves SMs idle.
    const uint32_t elems = a.heads * a.dv * DK;
    uint32_t part = kStepTile * 16;
    while (part > kStepTile && (unsigned long long)a.n * ((elems + part - 1) / part) < 8ull * l.n_sms) part >>= 1;
    const uint32_t parts = (elems + part - 1) / part;
    return launch_pdl(ssm_step_kernel<T, DK>, dim3(a.n * parts), dim3(kStepCta), 0, l.stream, g, a, parts, part, Divider::of(a.dv),
                      Divider::of(a.heads / a.groups));
}

template <class T, int DK, int DVT, int NT>
cudaError_t prompt_launch(const Geom &g, const SsmArgs &a, const Launch &l, uint32_t *launched)
{
    using L = PromptSmem<DK, DVT, NT>;
    static_assert(L::kTotal <= 227 * 1024, "shared memory of one CTA");
    const cudaError_t e = allow_smem<ssm_prompt_kernel<T, DK, DVT, NT>>(l.device, L::kTotal);
    if (e != cudaSuccess) return e;
    const uint32_t tiles = a.dv / DVT;
    CUtensorMap q = {}, k = {}, v = {};
    if (a.total && !(rows_map(&q, a.q, a.groups * DK, a.total, a.qs, DK < 64 ? DK : 64, kC) &&
                     rows_map(&k, a.k, a.groups * DK, a.total, a.ks, DK < 64 ? DK : 64, kC) &&
                     rows_map(&v, a.v, a.heads * a.dv, a.total, a.vs, DVT, kC)))
        return cudaErrorNotSupported;
    const uint32_t shares = ssm_shares(a.n, a.heads, a.dv, a.total, l.n_sms), items = a.n * a.heads * tiles;
    if (shares > 1) {
        const cudaError_t f = launch_pdl(ssm_prompt_kernel<T, DK, DVT, NT>, dim3(items * (shares - 1)), dim3(NT * 128), L::kTotal, l.stream, g, a,
                                         tiles, shares, true, q, k, v);
        if (f != cudaSuccess) return f;
        *launched += 1;
    }
    *launched += 1;
    return launch_pdl(ssm_prompt_kernel<T, DK, DVT, NT>, dim3(items * shares), dim3(NT * 128), L::kTotal, l.stream, g, a, tiles, shares, false, q, k, v);
}
template <class T, int DVT>
cudaError_t prompt_dv(const Geom &g, const SsmArgs &a, const Launch &l, uint32_t *launched)
{
    // Short keys: two CTAs of two teams on an SM overlap their beginnings and ends, one of four teams walks a long prompt faster.
    // us with two and with four, 32 heads: 32 prompts of 272 tokens 45 and 64, of 512 62 and 84, 16 of 1 024 62 and 74, of 2 048 116
    // and 128, of 8 192 433 and 440, 12 of 8 192 348 and 331; 63 of 100 beside one of 50 000 851 and 666.  Only the mean length is known
    // here, and a long prompt may hide behind a short mean: from 1 024 on four teams, which gives away up to a sixth where all
    // are alike; below two, which gives away a fifth where one is long.
    const bool small = a.total / a.n < 1024u && (unsigned long long)a.n * a.heads * (a.dv / DVT) >= 2ull * l.n_sms;
    switch (a.dk) {
    case 16: return small ? prompt_launch<T, 16, DVT, 2>(g, a, l, launched) : prompt_launch<T, 16, DVT, 4>(g, a, l, launched);
    case 32: return prompt_launch<T, 32, DVT, 3>(g, a, l, launched);
    case 64: return prompt_launch<T, 64, DVT, 2>(g, a, l, launched);
    default: return prompt_launch<T, 128, DVT, 2>(g, a, l, launched);
    }
}
template <class T>
cudaError_t step_type(const Geom &g, const SsmArgs &a, const Launch &l)
{
    switch (a.dk) {
    case 16: return step_dk<T, 16>(g, a, l);
    case 32: return step_dk<T, 32>(g, a, l);
    case 64: return step_dk<T, 64>(g, a, l);
    default: return step_dk<T, 128>(g, a, l);
    }
}

}  // namespace

cudaError_t launch_ssm_step(const Geom &g, const SsmArgs &a, const Launch &l)
{
    return a.f16 ? step_type<F16>(g, a, l) : step_type<Bf16>(g, a, l);
}
cudaError_t launch_ssm_prompt(const Geom &g, const SsmArgs &a, const Launch &l, uint32_t *launched)
{
    if (a.dv % 64 == 0) return a.f16 ? prompt_dv<F16, 64>(g, a, l, launched) : prompt_dv<Bf16, 64>(g, a, l, launched);
    return a.f16 ? prompt_dv<F16, 32>(g, a, l, launched) : prompt_dv<Bf16, 32>(g, a, l, launched);
}
// Runs that each prompt is cut into: as many as leave no SM without one, of 8 pieces or more on the mean; 1 where the first pass
// would cost more than it gives (it reads keys and values once more).  65 536 tokens of 1 head 61 us, of 8 heads 97, of 48 495, each
// about 800 in one run; 16 384 tokens of 32 heads of 64 keys 183 against 390.
uint32_t ssm_shares(uint32_t n, uint32_t heads, uint32_t dv, uint32_t total, int n_sms)
{
    const unsigned long long items = (unsigned long long)n * heads * (dv % 64 ? dv / 32 : dv / 64);
    unsigned long long s = (unsigned long long)n_sms / items;
    if (s > total / n / (8 * kC)) s = total / n / (8 * kC);
    return s < 3 ? 1u : (uint32_t)(s < 32 ? s : 32);
}

}  // namespace avmp
