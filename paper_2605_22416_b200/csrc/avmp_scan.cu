// Selective scan: the recurrence of a state layer with a decay for every channel and state element, on the blocks in place:
//     D_t = softplus(d_t + bias),   h <- exp(D_t A) h + D_t u_t B_t,   y_t = <C_t, h> + D u_t,   out_t = y_t z_t / (1 + e^-z_t)
// (h, A: [channels][states]; u, d, z, out: a row per token and channel; B, C: a row per token and group of channels).
//
// scan_prompt_kernel   whole prompts.  Bound by the exponentials: one per token, channel and state, of which the special-function unit gives
//                      16 a cycle and SM, and three more per token and channel; the rows are 8 bytes a channel.  Measured (16 states): 32 prompts of
//                      1000 tokens, 8192 channels, 1 414 us (that unit is busy 76 % of the time, 61 % of the issue slots are taken; bytes alone
//                      322); one of 4096 tokens 258 (61 %: 256 CTAs on 148 SMs, two warps of the scan to a scheduler); 32 of 32 to 512
//                      tokens, 2048 channels, 84.  An eighth of the exponentials as polynomials on the multiply-add pipe 3 % slower, a quarter 8 %:
//                      the issue slots are short too.
// scan_step_kernel     one token per request: bound by HBM, every state element is read and written once.  1 GB of state 395 to 415 us (84 to 88 % of
//                      the measured copy rate); 32 requests of 128 KB 4.6 (latency).
#include "avmp_lists.cuh"
#include "avmp_tc.cuh"

namespace avmp {

namespace {

uint32_t scan_tiles(uint32_t channels, uint32_t groups, uint32_t cb) { return groups * ((channels / groups + cb - 1) / cb); }

// How a call is cut up.  A lane with 16 states (all 8 of 8) costs the fewest instructions, one with 4 walks a prompt fastest.
struct ScanPlan {
    bool wide;
    uint32_t shares;      // runs that each prompt is cut into
};
ScanPlan scan_plan(uint32_t n, uint32_t channels, uint32_t groups, uint32_t states, uint32_t total, int n_sms)
{
    const uint32_t lanes = states > 16 ? states / 16 : 1;
    const unsigned long long wide = (unsigned long long)n * scan_tiles(channels, groups, 128 / lanes);       // CTAs, two on an SM
    const unsigned long long narrow = (unsigned long long)n * scan_tiles(channels, groups, 128 * 4 / states);
    if (wide >= 3ull * n_sms) return {true, 1};
    // Several prompts are seldom alike, and only their mean is known here: the longest holds an uncut call up, and is better cut finely.
    if (4 * narrow >= (n == 1 ? 3ull : 6ull) * n_sms) return {false, 1};
    // As many runs as fill the SMs, of 128 tokens or more on the mean: what the first pass costs is two thirds of the second one.
    unsigned long long s = total / n / 128;
    if (s > 64) s = 64;
    if (narrow * s <= 2ull * n_sms) return {false, s < 3 ? 1u : (uint32_t)s};
    const unsigned long long most = (n == 1 ? 2ull : 4ull) * n_sms / wide;
    if (s > most) s = most;
    return s < 3 ? ScanPlan{false, 1} : ScanPlan{true, (uint32_t)s};
}

constexpr int kCta = 128;
constexpr float kLog2e = 1.4426950408889634f;
// The approximate exponential is too small on the mean, by 4e-9 to 9e-9 of its value for arguments of -2^-8 and above, by 1e-8 to 3e-8 from there to -1
// (measured at 2^18 points a quarter of an octave), and a state adds that up over the tokens that it remembers.  So decays' arguments are raised a
// little: nothing to pay, as products and sums are one instruction, and 2^kMean is 1 exactly, so that a step of 0 leaves a state as it was.
constexpr float kMean = 1.2e-8f;

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x| (its argument's rounding is made up for; 0 from -100 on, infinities included).
// log(1 + e) / e on [0, 1] is a polynomial of degree 9 fitted for least relative error (5e-9; 1.4e-7 with its roundings).
__device__ __forceinline__ constexpr float log_poly(int i)
{
    constexpr float c[10] = {1.f, -4.9999901652e-01f, 3.3329963684e-01f, -2.4954134226e-01f, 1.9675938785e-01f,
                             -1.5305592120e-01f, 1.0603653640e-01f, -5.6959517300e-02f, 1.9851453602e-02f, -3.2440233e-03f};
    return c[i];
}
constexpr float kLn2 = 0.6931471806f, kLog2eLow = 1.925963033e-8f;      // log2(e) - kLog2e
__device__ __forceinline__ float ramp(float x) { return max3_nan(x, 0.f, 0.f); }
__device__ __forceinline__ float softplus(float x)
{
    const float a = fmaxf(-fabsf(x), -100.f), t = a * kLog2e, rest = fmaf(a, kLog2eLow, fmaf(a, kLog2e, -t));
    float e = exp2_approx(t);
    e = fmaf(e * kLn2, rest, e);
    float y = log_poly(9);
#pragma unroll
    for (int i = 8; i >= 0; --i) y = fmaf(y, e, log_poly(i));
    return fmaf(y, e, ramp(x));
}
__device__ __forceinline__ unsigned long long both(float x) { return pack2(x, x); }
// The same of a pair.
__device__ __forceinline__ float2 softplus2(float2 x)
{
    const unsigned long long a2 = pack2(fmaxf(-fabsf(x.x), -100.f), fmaxf(-fabsf(x.y), -100.f)), t2 = mul2(a2, both(kLog2e));
    const float2 t = unpack2(t2);
    const unsigned long long rest = fma2(a2, both(kLog2eLow), fma2(a2, both(kLog2e), pack2(-t.x, -t.y)));
    unsigned long long e = pack2(exp2_approx(t.x), exp2_approx(t.y));
    e = fma2(mul2(e, both(kLn2)), rest, e);
    unsigned long long y = both(log_poly(9));
#pragma unroll
    for (int i = 8; i >= 0; --i) y = fma2(y, e, both(log_poly(i)));
    return unpack2(fma2(y, e, pack2(ramp(x.x), ramp(x.y))));
}

// 2^x h + s of a pair, 2^x being the decay of a whole run.  By itself that may pass the range of 32 bits where the product does not, and would make NaN
// of a zero or an infinity then.  So it is taken as two factors, the second being 1 up to 2^+-125 (both within the range: together up to
// 2^+-250, from where on all but zeros, infinities and numbers below 2^-122 have left it).
__device__ __forceinline__ unsigned long long over_run(unsigned long long h, float2 x, unsigned long long s)
{
    x = make_float2(fminf(fmaxf(x.x, -250.f), 250.f), fminf(fmaxf(x.y, -250.f), 250.f));
    const float2 near = make_float2(fminf(fmaxf(x.x, -125.f), 125.f), fminf(fmaxf(x.y, -125.f), 125.f));
    const unsigned long long far = pack2(exp2_approx(x.x - near.x), exp2_approx(x.y - near.y));
    return fma2(pack2(exp2_approx(near.x), exp2_approx(near.y)), mul2(far, h), s);
}

// ---------------------------------------------------------------- whole prompts
// One CTA per (request, CB channels of a group, run of tokens), of eight warps.  Four scan: a lane has S states of a channel, Q = states / S lanes
// share a channel (lane q * 32 / Q + c has part q of channel c), and a warp works token by token; sums over the states are put together
// across lanes four tokens at a time.  The other four work for them, a tile of kTok tokens ahead and one behind: they copy the rows in, work
// out step sizes once per token and channel, widen B and C, and finish and store the outputs.  One barrier a tile.
// Where requests and channels leave SMs idle, every prompt is cut into `shares` runs: a first pass leaves, for every run but the last,
// the state that it makes from nothing, and the sum of its steps (whose product with A is the run's whole decay); a second pass
// starts every run from those in front of it.
constexpr int kStages = 4;            // a tile's rows are copied two tiles ahead and needed until its outputs are out
constexpr int kBoth = 2 * kCta;

template <int N, int S>
struct Tile {
    static constexpr int Q = N / S, P = S / 2;
    static constexpr int J = P > 4 ? 1 : P > 2 ? 2 : 4;              // tokens that are worked out ahead of the state
    static constexpr int W = 32 / Q, CB = kCta / 32 * W;             // channels of a warp and of a CTA
    static constexpr int kTok = Q == 1 ? 8 : 32;                     // tokens of a tile (a lane with all states: 1 400 us with 8, 1 459 with 16, 32 prompts of 1000; else 266 with 32, 281 with 16, one of 4096, before kApart)
    static constexpr uint32_t kRow = CB * 2, kRows = kTok * kRow, kBc = kTok * N * 2;
    static constexpr uint32_t kStage = 3 * kRows + 2 * kBc;          // u, d, z, B, C
    static constexpr uint32_t kSteps = kTok * CB * 8;                // (D, D u), [token][channel]
    static constexpr uint32_t kWide = 2 * kTok * N * 4;              // B and C in 32 bits, [B or C][token][state]
    // sums over the states, [token][channel]; where four lanes share a channel, of each of them: the warps around the scan add them up
    // (one of 4096 tokens 258 us, 266 with the sums put together across lanes by the warps that scan)
    static constexpr bool kApart = Q == 4 && S == 4;                 // (with more states there is no room for two CTAs on an SM then)
    static constexpr uint32_t kParts = kApart ? 4 : 1, kPart = kTok * CB * 4 + (kApart ? 32 : 0), kOut = kParts * kPart;
    static constexpr uint32_t oSteps = kStages * kStage, oWide = oSteps + 2 * kSteps, oOut = oWide + 2 * kWide, kTotal = oOut + 2 * kOut;
};

template <class T, int N, int S>
__global__ void __launch_bounds__(kBoth, 2) scan_prompt_kernel(const Geom g, const ScanArgs a, uint32_t tiles, uint32_t shares, bool locals)
{
    using L = Tile<N, S>;
    constexpr int CB = L::CB, Q = L::Q, P = L::P, J = L::J, kTok = L::kTok;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ uint32_t order[kCta];
    pdl_prologue();
    const uint32_t runs = locals ? shares - 1 : shares, per = tiles * runs;
    uint32_t k = blockIdx.x / per;
    const uint32_t tile = blockIdx.x % per / runs, run = blockIdx.x % runs;
    if (a.n > 1 && a.n <= kCta) {
        // the longest first, so that no long one begins when the others are about to end
        uint32_t len = 0;
        if (threadIdx.x < a.n) {
            const uint32_t c0 = a.cu[threadIdx.x], c1 = a.cu[threadIdx.x + 1];
            order[threadIdx.x] = len = c1 > c0 ? c1 - c0 : 0u;
        }
        __syncthreads();
        uint32_t rank = 0;
        if (threadIdx.x < a.n)
            for (uint32_t j = 0; j < a.n; ++j) rank += order[j] > len || (order[j] == len && j < threadIdx.x);
        __syncthreads();
        if (threadIdx.x < a.n) order[rank] = threadIdx.x;
        __syncthreads();
        k = order[k];
    }
    const uint32_t r = a.reqs[k], c0 = a.cu[k], c1 = a.cu[k + 1];
    float *block = state_block(g, a.layer, r);
    if (named_before(a.reqs, k, r) || !block || c1 < c0 || c1 > a.total) {
        if (threadIdx.x == 0 && tile == 0 && run == 0 && !locals) record_error(g.st, AVMP_DEV_BAD_REQUEST);
        return;
    }
    const uint32_t per_group = a.channels / a.groups, tiles_group = tiles / a.groups, grp = tile / tiles_group;
    const uint32_t ch0 = grp * per_group + tile % tiles_group * CB;          // first channel of the CTA
    const uint32_t chs = min((uint32_t)CB, (grp + 1) * per_group - ch0);
    // tokens of the run: whole tiles, so that all runs but the last are alike
    const uint32_t len = c1 - c0, step = (len + shares * kTok - 1) / (shares * kTok) * kTok;
    const uint32_t t0 = min(len, run * step), t1 = min(len, t0 + step), n_tiles = (t1 - t0 + kTok - 1) / kTok;
    // In the workspace: [entry][run][channel][state], slot 0 what the request starts from, slot j what run j - 1 makes; the sums of steps behind.
    const unsigned long long slot = (unsigned long long)a.channels * N, sums = (unsigned long long)a.n * shares * slot;
    auto ws_state = [&](uint32_t j) { return a.ws + ((unsigned long long)k * shares + j) * slot; };
    auto ws_sum = [&](uint32_t j) { return a.ws + sums + ((unsigned long long)k * shares + j) * a.channels + ch0; };

    if (threadIdx.x >= kCta) {
        // ---------------- the warps around the scan
        const uint32_t tid = threadIdx.x - kCta, base = smem_u32(smem);
        constexpr int kQuads = CB / 4, kPass = kCta / kQuads;                // a thread has four channels, of every kPass-th token
        const uint32_t mych = tid % kQuads * 4, myrow = tid / kQuads;
        const bool mine = mych < chs;
        float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), skip = bias, sum = bias;
        auto four = [&](const float *p) { return make_float4(p[0], p[1], p[2], p[3]); };
        if (mine && a.bias) bias = four(a.bias + ch0 + mych);
        if (mine && a.skip) skip = four(a.skip + ch0 + mych);
        const unsigned long long row0 = c0 + t0;
        const uint8_t *urow = a.u + row0 * a.us + ch0 * 2, *drow = a.d + row0 * a.ds + ch0 * 2, *zrow = a.z ? a.z + row0 * a.zs + ch0 * 2 : nullptr;
        const uint8_t *brow = a.b + row0 * a.bs + grp * N * 2, *crow = a.c + row0 * a.cs + grp * N * 2;
        uint8_t *orow = a.out + row0 * a.os + (ch0 + mych) * 2;
        // 16-byte units of rows, zeros behind the last row and channel
        auto load = [&](uint32_t i) {
            if (i < n_tiles) {
                const uint32_t at = base + i % kStages * L::kStage, rows = t1 - t0 - i * kTok;
                for (uint32_t y = tid; y < kTok * CB / 8; y += kCta) {
                    const uint32_t t = y / (CB / 8), e = y % (CB / 8);
                    const bool there = t < rows && e * 8 < chs;
                    const uint32_t dst = at + y * 16;
                    const unsigned long long tok = i * kTok + t;
                    cp_async16(dst, there ? urow + tok * a.us + e * 16 : a.u, there);
                    cp_async16(dst + L::kRows, there ? drow + tok * a.ds + e * 16 : a.u, there);
                    if (zrow && !locals) cp_async16(dst + 2 * L::kRows, there ? zrow + tok * a.zs + e * 16 : a.u, there);
                }
                for (uint32_t y = tid; y < kTok * N / 8; y += kCta) {
                    const uint32_t t = y / (N / 8), e = y % (N / 8), dst = at + 3 * L::kRows + y * 16;
                    const bool there = t < rows;
                    const unsigned long long tok = i * kTok + t;
                    cp_async16(dst, there ? brow + tok * a.bs + e * 16 : a.u, there);
                    if (!locals) cp_async16(dst + L::kBc, there ? crow + tok * a.cs + e * 16 : a.u, there);
                }
            }
            cp_async_commit();
        };
        auto unpack4 = [](uint2 v) {
            const float2 lo = T::unpack(v.x), hi = T::unpack(v.y);
            return make_float4(lo.x, lo.y, hi.x, hi.y);
        };
        auto before = [&](uint32_t i) {
            const uint8_t *at = smem + i % kStages * L::kStage;
            const uint32_t rows = t1 - t0 - i * kTok;
            float4 *to = reinterpret_cast<float4 *>(smem + L::oSteps + (i & 1) * L::kSteps);
#pragma unroll
            for (uint32_t t = myrow; t < kTok; t += kPass) {
                const uint32_t e = (t * CB + mych) * 2;
                const float4 u = unpack4(*reinterpret_cast<const uint2 *>(at + e)), d = unpack4(*reinterpret_cast<const uint2 *>(at + L::kRows + e));
                float2 lo = make_float2(d.x + bias.x, d.y + bias.y), hi = make_float2(d.z + bias.z, d.w + bias.w);
                if (a.softplus) { lo = softplus2(lo); hi = softplus2(hi); }
                if (t >= rows) lo = hi = make_float2(0.f, 0.f);
                if (locals) { sum.x += lo.x; sum.y += lo.y; sum.z += hi.x; sum.w += hi.y; }
                float4 *p = to + (t * CB + mych) / 2;
                p[0] = make_float4(lo.x, lo.x * u.x, lo.y, lo.y * u.y);
                p[1] = make_float4(hi.x, hi.x * u.z, hi.y, hi.y * u.w);
            }
            for (uint32_t y = tid; y < (locals ? 1u : 2u) * kTok * N / 4; y += kCta) {
                *reinterpret_cast<float4 *>(smem + L::oWide + (i & 1) * L::kWide + y * 16) = unpack4(*reinterpret_cast<const uint2 *>(at + 3 * L::kRows + y * 8));
            }
        };
        auto behind = [&](uint32_t i) {
            const uint8_t *at = smem + i % kStages * L::kStage;
            const uint32_t rows = t1 - t0 - i * kTok;
            const float4 *from = reinterpret_cast<const float4 *>(smem + L::oOut + (i & 1) * L::kOut);
#pragma unroll
            for (uint32_t t = myrow; t < kTok; t += kPass) {
                const uint32_t e = (t * CB + mych) * 2;
                float4 o = from[e / 8];
#pragma unroll
                for (uint32_t x = 1; x < L::kParts; ++x) {
                    const float4 v = from[x * (L::kPart / 16) + e / 8];
                    o = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
                }
                if (a.skip) {
                    const float4 u = unpack4(*reinterpret_cast<const uint2 *>(at + e));
                    o = make_float4(fmaf(skip.x, u.x, o.x), fmaf(skip.y, u.y, o.y), fmaf(skip.z, u.z, o.z), fmaf(skip.w, u.w, o.w));
                }
                if (zrow) {
                    const float4 z = unpack4(*reinterpret_cast<const uint2 *>(at + 2 * L::kRows + e));
                    o = make_float4(o.x * silu(z.x), o.y * silu(z.y), o.z * silu(z.z), o.w * silu(z.w));
                }
                if (mine && t < rows) *reinterpret_cast<uint2 *>(orow + (i * kTok + t) * a.os) = make_uint2(T::pack(o.x, o.y), T::pack(o.z, o.w));
            }
        };
        load(0);
        load(1);
        cp_async_wait<1>();
        bar_sync(1, kCta);
        if (n_tiles) before(0);
        cp_async_wait<0>();
        __syncthreads();
        for (uint32_t i = 0; i < n_tiles; ++i) {
            load(i + 2);
            if (i + 1 < n_tiles) before(i + 1);
            if (i && !locals) behind(i - 1);
            cp_async_wait<0>();
            __syncthreads();
        }
        if (n_tiles && !locals) behind(n_tiles - 1);
        if (locals) {      // a thread has summed every kPass-th token's steps
            float4 *part = reinterpret_cast<float4 *>(smem);
            part[tid] = sum;
            bar_sync(1, kCta);
            if (myrow == 0 && mine) {
                for (uint32_t j = 1; j < kPass; ++j) {
                    const float4 v = part[tid + j * kQuads];
                    sum = make_float4(sum.x + v.x, sum.y + v.y, sum.z + v.z, sum.w + v.w);
                }
                float *to = ws_sum(run + 1) + mych;
                to[0] = sum.x; to[1] = sum.y; to[2] = sum.z; to[3] = sum.w;
            }
        }
        return;
    }

    // ---------------- the scan.  Two states go through the multiply-add pipe at a time.
    const int w = threadIdx.x / 32, lane = threadIdx.x % 32, q = lane / L::W, c = lane % L::W;
    const uint32_t mych = w * L::W + c;
    const bool mine = mych < chs;
    const unsigned long long first = (unsigned long long)(ch0 + mych) * N + q * S;
    auto pairs = [&](float *from) { return reinterpret_cast<unsigned long long *>(from + first); };      // this lane's part of a [channels][states] array
    unsigned long long A[P], h[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        A[p] = mine ? mul2(reinterpret_cast<const unsigned long long *>(a.a + first)[p], both(kLog2e)) : 0ull;
        h[p] = 0ull;
    }
    if (shares == 1 || locals) {
        const bool kept = a.resume && a.resume[k];
        if (run == 0 && mine) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const unsigned long long v = kept ? pairs(block)[p] : 0ull;
                if (locals) pairs(ws_state(0))[p] = v; else h[p] = v;
            }
        }
    } else if (mine) {
#pragma unroll
        for (int p = 0; p < P; ++p) h[p] = pairs(ws_state(0))[p];
        for (uint32_t j = 1; j <= run; ++j) {
            const unsigned long long d2 = both(ws_sum(j)[mych]);
#pragma unroll
            for (int p = 0; p < P; ++p) h[p] = over_run(h[p], unpack2(mul2(A[p], d2)), pairs(ws_state(j))[p]);
        }
    }
    __syncthreads();
    for (uint32_t i = 0; i < n_tiles; ++i) {
        const uint8_t *st = smem + L::oSteps + (i & 1) * L::kSteps + mych * 8;
        const unsigned long long *bq = reinterpret_cast<const unsigned long long *>(smem + L::oWide + (i & 1) * L::kWide) + q * P, *cq = bq + kTok * N / 2;
        float *to = reinterpret_cast<float *>(smem + L::oOut + (i & 1) * L::kOut + (L::kApart ? q * L::kPart : 0u)) + mych;
        // Some tokens' decays, additions and C, worked out while those before go through the state: a warp may be alone on its scheduler, and
        // nothing but the state itself then waits for what is in front of it.
        struct Ahead {
            unsigned long long e[J][P], g[J][P], c[J][P];
        };
        auto fetch = [&](Ahead &f, int t) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                const float2 v = *reinterpret_cast<const float2 *>(st + (t + j) * CB * 8);
                const unsigned long long d2 = both(v.x), u2 = both(v.y);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float2 e = unpack2(fma2(d2, A[p], both(kMean)));
                    f.e[j][p] = pack2(exp2_approx(e.x), exp2_approx(e.y));
                    f.g[j][p] = mul2(u2, bq[(t + j) * (N / 2) + p]);
                    f.c[j][p] = cq[(t + j) * (N / 2) + p];
                }
            }
        };
        auto take = [&](const Ahead &f, float *y) {
#pragma unroll
            for (int j = 0; j < J; ++j) {
                unsigned long long acc = 0;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    h[p] = fma2(f.e[j][p], h[p], f.g[j][p]);
                    acc = p ? fma2(h[p], f.c[j][p], acc) : mul2(h[p], f.c[j][p]);
                }
                const float2 z = unpack2(acc);
                y[j] = z.x + z.y;
            }
        };
        // sums of four tokens over the lanes of a channel; where there are four or more, four of them keep one each
        auto put = [&](float (&y)[4], int t) {
            if (locals) return;
            if (Q == 1 || L::kApart) {
#pragma unroll
                for (int j = 0; j < 4; ++j) to[(t + j) * CB] = y[j];
                return;
            }
#pragma unroll
            for (int o = L::W; o < 16 / (Q > 2 ? 2 : 1); o <<= 1)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] += __shfl_xor_sync(0xFFFFFFFFu, y[j], o);
            const bool hi = lane & 16, odd = lane & 8;
            const float s0 = __shfl_xor_sync(0xFFFFFFFFu, hi ? y[0] : y[2], 16), s1 = __shfl_xor_sync(0xFFFFFFFFu, hi ? y[1] : y[3], 16);
            const float a0 = (hi ? y[2] : y[0]) + s0, a1 = (hi ? y[3] : y[1]) + s1;
            if (Q == 2) {
                to[(t + (hi ? 2 : 0)) * CB] = a0;
                to[(t + (hi ? 3 : 1)) * CB] = a1;
                return;
            }
            const float o = (odd ? a1 : a0) + __shfl_xor_sync(0xFFFFFFFFu, odd ? a0 : a1, 8);
            if (Q == 4 || lane % 8 < L::W) to[(t + (lane >> 3)) * CB] = o;
        };
        Ahead f[2];
        float y[4];
        fetch(f[0], 0);
        constexpr int kBody = J == 4 ? 8 : 4;          // an even number of fetches
#pragma unroll 1
        for (int t = 0; t < kTok - kBody; t += kBody)
#pragma unroll
            for (int x = 0; x < kBody; x += J) {
                fetch(f[(x / J + 1) & 1], t + x + J);
                take(f[x / J & 1], y + x % 4);
                if (x % 4 == 4 - J) put(y, t + x / 4 * 4);
            }
#pragma unroll
        for (int x = 0; x < kBody; x += J) {
            if (x + J < kBody) fetch(f[(x / J + 1) & 1], kTok - kBody + x + J);
            take(f[x / J & 1], y + x % 4);
            if (x % 4 == 4 - J) put(y, kTok - kBody + x / 4 * 4);
        }
        __syncthreads();
    }
    if (!mine) return;
    float *to = locals ? ws_state(run + 1) : run == shares - 1 ? block : nullptr;
    if (to)
#pragma unroll
        for (int p = 0; p < P; ++p) pairs(to)[p] = h[p];
}

// ---------------------------------------------------------------- one token
// The work is the list of all (tile, entry) pairs, a tile being 16 KB of states (4096 / N channels of a group); each CTA has a share of it, so that
// a tile's decays stay in registers over many entries.  A thread has four float4 of a tile, one in each quarter: accesses cover whole
// lines, and steps, gates and outputs are worked out by a lane each, the lanes of a channel sharing out the four.  States and rows come
// through a ring in shared memory, so that their number in flight costs no registers.  (1 GB of state, loads into registers: 448 us with
// 40 warps on an SM, 463 with the next round's ahead, 555 with four entries at a time.)
constexpr int kStep = 256;
constexpr uint32_t kBatch = 256;      // entries whose blocks are looked up at a time

template <int N>
struct StepTile {
    static constexpr uint32_t LANES = N / 4, CH = 4096 / N, kQuarter = CH / 4;       // lanes of a channel; channels of a tile and of a quarter
    static constexpr uint32_t kStages = 4;                                           // entries: one is worked on, the others are on their way
    static constexpr uint32_t kRow = CH * 2, oRows = 16384, oBc = oRows + 3 * kRow, kStage = oBc + 4 * N;      // states, u, d, z, B, C
    static constexpr uint32_t kTotal = kStages * kStage;
};

template <class T, int N>
__global__ void __launch_bounds__(kStep, 3) scan_step_kernel(const Geom g, const ScanArgs a, uint32_t tiles_group)
{
    using L = StepTile<N>;
    constexpr uint32_t LANES = L::LANES, OWN = LANES < 4 ? 2 : 1;                    // quarters that a lane finishes
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float *blocks[kBatch];
    pdl_prologue();
    const uint32_t tid = threadIdx.x, w = tid / 32, lane = tid % 32, q = tid % LANES, base = smem_u32(smem);
    const uint32_t per_group = a.channels / a.groups;
    const unsigned long long pairs = (unsigned long long)a.groups * tiles_group * a.n, last = pairs * (blockIdx.x + 1) / gridDim.x;
    auto channel = [&](uint32_t j) { return j * L::kQuarter + tid / LANES; };        // of the tile: this thread's in quarter j
    // quarters that this lane finishes: j0, and j0 + 1 where a channel has two lanes
    const uint32_t j0 = LANES < 4 ? 2 * q : q % 4;
    const bool finishes = q < 4;
    uint32_t count;
    for (unsigned long long at = pairs * blockIdx.x / gridDim.x; at < last; at += count) {
        const uint32_t tile = (uint32_t)(at / a.n), from = (uint32_t)(at % a.n), grp = tile / tiles_group;
        count = (uint32_t)min((unsigned long long)min(kBatch, a.n - from), last - at);
        const uint32_t ch0 = grp * per_group + tile % tiles_group * L::CH, chs = min(L::CH, (grp + 1) * per_group - ch0);
        __syncthreads();                           // the blocks before have been used
        if (tid < count) blocks[tid] = state_block(g, a.layer, a.reqs[from + tid]);
        unsigned long long A[4][2];
        float bias[OWN], skip[OWN];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (channel(j) < chs) v = *reinterpret_cast<const float4 *>(a.a + (unsigned long long)(ch0 + channel(j)) * N + q * 4);
            A[j][0] = pack2(v.x * kLog2e, v.y * kLog2e);
            A[j][1] = pack2(v.z * kLog2e, v.w * kLog2e);
        }
#pragma unroll
        for (uint32_t o = 0; o < OWN; ++o) {
            const uint32_t ch = channel(j0 + o);
            bias[o] = a.bias && ch < chs ? a.bias[ch0 + ch] : 0.f;
            skip[o] = a.skip && ch < chs ? a.skip[ch0 + ch] : 0.f;
        }
        __syncthreads();
        uint32_t next = 0, in = 0;
        auto load = [&] {
            if (next < count) {
                float *block = blocks[next];
                const unsigned long long k = from + next;
                const uint32_t to = base + in * L::kStage;
                if (block) {
                    const float *src = block + (unsigned long long)ch0 * N + tid * 4;
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j)
                        if (channel(j) < chs) cp_async16(to + j * 4096 + tid * 16, src + j * 1024, true);
                    constexpr uint32_t kUnits = L::kRow / 16;
                    for (uint32_t x = tid; x < 3 * kUnits + N / 4; x += kStep) {
                        const uint32_t part = x / kUnits, unit = x % kUnits;
                        if (x >= 3 * kUnits) {             // B, then C
                            const uint32_t y = x - 3 * kUnits, e = y % (N / 8);
                            cp_async16(to + L::oBc + y * 16, (y < N / 8 ? a.b + k * a.bs : a.c + k * a.cs) + grp * N * 2 + e * 16, true);
                        } else if (unit * 8 < chs && (part < 2 || a.z)) {
                            const uint8_t *row = part == 0 ? a.u + k * a.us : part == 1 ? a.d + k * a.ds : a.z + k * a.zs;
                            cp_async16(to + L::oRows + x * 16, row + (ch0 + unit * 8) * 2, true);
                        }
                    }
                }
            }
            cp_async_commit();
            ++next;
            in = in + 1 == L::kStages ? 0 : in + 1;
        };
#pragma unroll
        for (uint32_t x = 0; x < L::kStages - 1; ++x) load();
        // Repeated slots, a warp an entry, while the first copies are on their way.  (What is copied for one is not looked at.)
        for (uint32_t i = w; i < count; i += kStep / 32) {
            const uint32_t k = from + i, r = a.reqs[k];
            bool dup = false;
            for (uint32_t j = lane; j < k; j += 32) dup |= a.reqs[j] == r;
            dup = __any_sync(0xFFFFFFFFu, dup);
            if (lane == 0) {
                if ((dup || !blocks[i]) && tile == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
                if (dup) blocks[i] = nullptr;
            }
        }
        uint32_t out = 0;
        for (uint32_t i = 0; i < count; ++i) {
            cp_async_wait<L::kStages - 2>();
            __syncthreads();                       // this stage is there, and the one before has been read
            load();
            const uint8_t *st = smem + out * L::kStage;
            out = out + 1 == L::kStages ? 0 : out + 1;
            float *block = blocks[i];
            if (!block) continue;
            const unsigned long long k = from + i;
            auto row = [&](uint32_t part, uint32_t ch) { return T::unpack(*reinterpret_cast<const uint16_t *>(st + L::oRows + part * L::kRow + ch * 2)).x; };
            float u[OWN], d[OWN], du[OWN];
#pragma unroll
            for (uint32_t o = 0; o < OWN; ++o) {
                u[o] = row(0, channel(j0 + o));
                d[o] = row(1, channel(j0 + o)) + bias[o];
                if (a.softplus) d[o] = softplus(d[o]);
                du[o] = d[o] * u[o];
            }
            const uint2 bb = *reinterpret_cast<const uint2 *>(st + L::oBc + q * 8), cc = *reinterpret_cast<const uint2 *>(st + L::oBc + N * 2 + q * 8);
            auto pair = [](uint32_t v) { const float2 x = T::unpack(v); return pack2(x.x, x.y); };
            const unsigned long long B[2] = {pair(bb.x), pair(bb.y)}, C[2] = {pair(cc.x), pair(cc.y)};
            float *to = block + (unsigned long long)ch0 * N + tid * 4;
            float y[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                const uint32_t owner = lane - q + (LANES < 4 ? j / 2 : j);
                const float step = __shfl_sync(0xFFFFFFFFu, d[LANES < 4 ? j % 2 : 0], owner), add = __shfl_sync(0xFFFFFFFFu, du[LANES < 4 ? j % 2 : 0], owner);
                const ulonglong2 h0 = *reinterpret_cast<const ulonglong2 *>(st + j * 4096 + tid * 16);
                const float2 e0 = unpack2(fma2(A[j][0], both(step), both(kMean))), e1 = unpack2(fma2(A[j][1], both(step), both(kMean)));
                ulonglong2 h;
                h.x = fma2(pack2(exp2_approx(e0.x), exp2_approx(e0.y)), h0.x, mul2(both(add), B[0]));
                h.y = fma2(pack2(exp2_approx(e1.x), exp2_approx(e1.y)), h0.y, mul2(both(add), B[1]));
                if (channel(j) < chs) *reinterpret_cast<ulonglong2 *>(to + j * 1024) = h;
                const float2 z = unpack2(fma2(h.x, C[0], mul2(h.y, C[1])));
                y[j] = z.x + z.y;
            }
            // sums over the lanes of a channel: each keeps its own quarters
#pragma unroll
            for (uint32_t o = LANES / 2; o >= 4; o >>= 1)
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j) y[j] += __shfl_xor_sync(0xFFFFFFFFu, y[j], o);
            const bool hi = LANES < 4 ? q & 1 : q & 2, odd = q & 1;
            constexpr uint32_t kFar = LANES < 4 ? 1 : 2;
            const float s0 = __shfl_xor_sync(0xFFFFFFFFu, hi ? y[0] : y[2], kFar), s1 = __shfl_xor_sync(0xFFFFFFFFu, hi ? y[1] : y[3], kFar);
            float v[2] = {(hi ? y[2] : y[0]) + s0, (hi ? y[3] : y[1]) + s1};
            if (LANES >= 4) {
                const float x = __shfl_xor_sync(0xFFFFFFFFu, odd ? v[0] : v[1], 1);
                v[0] = (odd ? v[1] : v[0]) + x;
            }
#pragma unroll
            for (uint32_t o = 0; o < OWN; ++o) {
                const uint32_t ch = channel(j0 + o);
                float x = a.skip ? fmaf(skip[o], u[o], v[o]) : v[o];
                if (a.z) x *= silu(row(2, ch));
                if (finishes && ch < chs) *reinterpret_cast<uint16_t *>(a.out + k * a.os + (ch0 + ch) * 2) = (uint16_t)T::pack(x, 0.f);
            }
        }
        cp_async_wait<0>();
    }
}

template <class T, int N, int S>
cudaError_t prompt_launch(const Geom &g, const ScanArgs &a, const Launch &l, uint32_t *launched)
{
    using L = Tile<N, S>;
    static_assert(L::kTotal <= 227 * 1024, "shared memory of one CTA");
    cudaError_t e = allow_smem<scan_prompt_kernel<T, N, S>>(l.device, L::kTotal);
    if (e != cudaSuccess) return e;
    const uint32_t tiles = scan_tiles(a.channels, a.groups, L::CB), shares = a.shares;
    if (shares > 1) {
        e = launch_pdl(scan_prompt_kernel<T, N, S>, dim3(a.n * tiles * (shares - 1)), dim3(kBoth), L::kTotal, l.stream, g, a, tiles, shares, true);
        if (e != cudaSuccess) return e;
        *launched += 1;
    }
    *launched += 1;
    return launch_pdl(scan_prompt_kernel<T, N, S>, dim3(a.n * tiles * shares), dim3(kBoth), L::kTotal, l.stream, g, a, tiles, shares, false);
}
template <class T, int N>
cudaError_t prompt_width(const Geom &g, const ScanArgs &a, const Launch &l, uint32_t *launched)
{
    return scan_plan(a.n, a.channels, a.groups, a.states, a.total, l.n_sms).wide ? prompt_launch<T, N, N < 16 ? N : 16>(g, a, l, launched)
                                                                                  : prompt_launch<T, N, 4>(g, a, l, launched);
}
template <class T>
cudaError_t prompt_type(const Geom &g, const ScanArgs &a, const Launch &l, uint32_t *launched)
{
    switch (a.states) {
    case 8: return prompt_width<T, 8>(g, a, l, launched);
    case 16: return prompt_width<T, 16>(g, a, l, launched);
    case 32: return prompt_width<T, 32>(g, a, l, launched);
    default: return prompt_width<T, 64>(g, a, l, launched);
    }
}
template <class T, int N>
cudaError_t step_launch(const Geom &g, const ScanArgs &a, const Launch &l)
{
    using L = StepTile<N>;
    const cudaError_t e = allow_smem<scan_step_kernel<T, N>>(l.device, L::kTotal);
    if (e != cudaSuccess) return e;
    const uint32_t tiles_group = (a.channels / a.groups + L::CH - 1) / L::CH;
    const unsigned long long pairs = (unsigned long long)a.groups * tiles_group * a.n, ctas = (unsigned long long)l.n_sms * (L::kTotal > 72 * 1024 ? 2 : 3);
    return launch_pdl(scan_step_kernel<T, N>, dim3((uint32_t)min(pairs, ctas)), dim3(kStep), L::kTotal, l.stream, g, a, tiles_group);
}
template <class T>
cudaError_t step_type(const Geom &g, const ScanArgs &a, const Launch &l)
{
    switch (a.states) {
    case 8: return step_launch<T, 8>(g, a, l);
    case 16: return step_launch<T, 16>(g, a, l);
    case 32: return step_launch<T, 32>(g, a, l);
    default: return step_launch<T, 64>(g, a, l);
    }
}

}  // namespace

uint32_t scan_shares(uint32_t n, uint32_t channels, uint32_t groups, uint32_t states, uint32_t total, int n_sms)
{
    return scan_plan(n, channels, groups, states, total, n_sms).shares;
}
cudaError_t launch_scan_prompt(const Geom &g, const ScanArgs &a, const Launch &l, uint32_t *launched)
{
    return a.f16 ? prompt_type<F16>(g, a, l, launched) : prompt_type<Bf16>(g, a, l, launched);
}
cudaError_t launch_scan_step(const Geom &g, const ScanArgs &a, const Launch &l)
{
    return a.f16 ? step_type<F16>(g, a, l) : step_type<Bf16>(g, a, l);
}

}  // namespace avmp
