// Selective scan: the recurrence of a state layer with a decay for every channel and state element, on the blocks in place:
//     D_t = softplus(d_t + bias),   h <- exp(D_t A) h + D_t u_t B_t,   y_t = <C_t, h> + D u_t,   out_t = y_t z_t / (1 + e^-z_t)
// (h, A: [channels][states]; u, d, z, out: a row per token and channel; B, C: a row per token and group of channels).
//
// scan_prompt_kernel   whole prompts.  Bound by the exponentials: one per token, channel and state, of which the special-function unit gives
//                      16 a cycle and SM; the rows are 8 bytes a channel.
// scan_step_kernel     one token per request: bound by HBM, every state element is read and written once.
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
    if (4 * narrow >= 3ull * n_sms) return {false, 1};
    // As many runs as fill the SMs, of 128 tokens or more on the mean: what the first pass costs is two thirds of the second one.
    unsigned long long s = total / n / 128;
    if (s > 64) s = 64;
    if (narrow * s <= 2ull * n_sms) return {false, s < 3 ? 1u : (uint32_t)s};
    if (s > 2ull * n_sms / wide) s = 2ull * n_sms / wide;
    return s < 3 ? ScanPlan{false, 1} : ScanPlan{true, (uint32_t)s};
}

constexpr int kCta = 128;
constexpr float kLog2e = 1.4426950408889634f;

// log(1 + e^x) = max(x, 0) + log(1 + e), e = e^-|x| (its argument's rounding is made up for).  log(1 + e) / e on [0, 1] is a polynomial of
// degree 9 fitted for least relative error (5e-9; 1.4e-7 with its roundings).
__device__ __forceinline__ constexpr float log_poly(int i)
{
    constexpr float c[10] = {1.f, -4.9999901652e-01f, 3.3329963684e-01f, -2.4954134226e-01f, 1.9675938785e-01f,
                             -1.5305592120e-01f, 1.0603653640e-01f, -5.6959517300e-02f, 1.9851453602e-02f, -3.2440233e-03f};
    return c[i];
}
constexpr float kLn2 = 0.6931471806f, kLog2eLow = 1.925963033e-8f;      // log2(e) - kLog2e
__device__ __forceinline__ float softplus(float x)
{
    const float a = -fabsf(x), t = a * kLog2e, rest = fmaf(a, kLog2eLow, fmaf(a, kLog2e, -t));
    float e = exp2_approx(t);
    e = fmaf(e * kLn2, rest, e);
    float y = log_poly(9);
#pragma unroll
    for (int i = 8; i >= 0; --i) y = fmaf(y, e, log_poly(i));
    return fmaf(y, e, fmaxf(x, 0.f));
}
__device__ __forceinline__ unsigned long long both(float x) { return pack2(x, x); }
// The same of a pair.
__device__ __forceinline__ float2 softplus2(float2 x)
{
    const float2 a = make_float2(-fabsf(x.x), -fabsf(x.y));
    const unsigned long long a2 = pack2(a.x, a.y), t2 = mul2(a2, both(kLog2e));
    const float2 t = unpack2(t2);
    const unsigned long long rest = fma2(a2, both(kLog2eLow), fma2(a2, both(kLog2e), pack2(-t.x, -t.y)));
    unsigned long long e = pack2(exp2_approx(t.x), exp2_approx(t.y));
    e = fma2(mul2(e, both(kLn2)), rest, e);
    unsigned long long y = both(log_poly(9));
#pragma unroll
    for (int i = 8; i >= 0; --i) y = fma2(y, e, both(log_poly(i)));
    return unpack2(fma2(y, e, pack2(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f))));
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
    static constexpr int kTok = Q == 1 ? 16 : 32;                    // tokens of a tile
    static constexpr uint32_t kRow = CB * 2, kRows = kTok * kRow, kBc = kTok * N * 2;
    static constexpr uint32_t kStage = 3 * kRows + 2 * kBc;          // u, d, z, B, C
    static constexpr uint32_t kSteps = kTok * CB * 8;                // (D, D u), [token][channel]
    static constexpr uint32_t kWide = 2 * kTok * N * 4;              // B and C in 32 bits, [B or C][token][state]
    static constexpr uint32_t kOut = kTok * CB * 4;                  // sums over the states, [token][channel]
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
            for (int p = 0; p < P; ++p) {
                const float2 e = unpack2(mul2(A[p], d2));
                h[p] = fma2(pack2(exp2_approx(e.x), exp2_approx(e.y)), h[p], pairs(ws_state(j))[p]);
            }
        }
    }
    __syncthreads();
    for (uint32_t i = 0; i < n_tiles; ++i) {
        const uint8_t *st = smem + L::oSteps + (i & 1) * L::kSteps + mych * 8;
        const unsigned long long *bq = reinterpret_cast<const unsigned long long *>(smem + L::oWide + (i & 1) * L::kWide) + q * P, *cq = bq + kTok * N / 2;
        float *to = reinterpret_cast<float *>(smem + L::oOut + (i & 1) * L::kOut) + mych;
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
                    const float2 e = unpack2(mul2(d2, A[p]));
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
        // sums of four tokens over the lanes of a channel; where there are four, each keeps one
        auto put = [&](float (&y)[4], int t) {
            if (locals) return;
            if (Q == 1) {
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
// CTA (i, j): kEntries entries, the j-th run of `rounds` times kCta * 8 / N channels.  A thread has eight states of a channel, for all entries of
// the CTA, so that decays and B and C are read once for several states; the next round's loads are on their way while one is worked on.
constexpr int kEntries = 2;

template <class T, int N>
__global__ void __launch_bounds__(kCta) scan_step_kernel(const Geom g, const ScanArgs a, uint32_t rounds)
{
    constexpr int LANES = N / 8;
    constexpr uint32_t CB = kCta / LANES;
    pdl_prologue();
    const uint32_t k0 = blockIdx.x * kEntries, s = threadIdx.x % LANES * 8, end = min(a.channels, (blockIdx.y + 1) * rounds * CB);
    float *block[kEntries];
#pragma unroll
    for (int e = 0; e < kEntries; ++e) block[e] = k0 + e < a.n ? state_block(g, a.layer, a.reqs[k0 + e]) : nullptr;
    const uint32_t per_group = a.channels / a.groups;
    struct Round {
        float4 h[kEntries][2], A[2];
        uint16_t u[kEntries], d[kEntries], z[kEntries];
        float bias, skip;
    };
    auto fetch = [&](Round &r, uint32_t ch) {
        if (ch >= end) return;
        const unsigned long long at = (unsigned long long)ch * N + s;
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            if (!block[e]) continue;
            const uint32_t k = k0 + e;
            r.h[e][0] = *reinterpret_cast<const float4 *>(block[e] + at);
            r.h[e][1] = *reinterpret_cast<const float4 *>(block[e] + at + 4);
            r.u[e] = *reinterpret_cast<const uint16_t *>(a.u + k * a.us + ch * 2);
            r.d[e] = *reinterpret_cast<const uint16_t *>(a.d + k * a.ds + ch * 2);
            if (a.z) r.z[e] = *reinterpret_cast<const uint16_t *>(a.z + k * a.zs + ch * 2);
        }
        r.A[0] = *reinterpret_cast<const float4 *>(a.a + at);
        r.A[1] = *reinterpret_cast<const float4 *>(a.a + at + 4);
        r.bias = a.bias ? a.bias[ch] : 0.f;
        r.skip = a.skip ? a.skip[ch] : 0.f;
    };
    uint4 b[kEntries], c[kEntries];
    uint32_t grp = kInvalid;
    auto work = [&](Round &r, uint32_t ch) {
        const bool mine = ch < end;
        if (mine && ch / per_group != grp) {
            grp = ch / per_group;
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                if (!block[e]) continue;
                b[e] = *reinterpret_cast<const uint4 *>(a.b + (k0 + e) * a.bs + (grp * N + s) * 2);
                c[e] = *reinterpret_cast<const uint4 *>(a.c + (k0 + e) * a.cs + (grp * N + s) * 2);
            }
        }
        const float A[8] = {r.A[0].x, r.A[0].y, r.A[0].z, r.A[0].w, r.A[1].x, r.A[1].y, r.A[1].z, r.A[1].w};
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            const bool there = mine && block[e];
            float y = 0.f, u = 0.f;
            if (there) {
                u = T::unpack(r.u[e]).x;
                float d = T::unpack(r.d[e]).x + r.bias;
                if (a.softplus) d = softplus(d);
                const float du = d * u, x = d * kLog2e;
                const uint32_t bb[4] = {b[e].x, b[e].y, b[e].z, b[e].w}, cc[4] = {c[e].x, c[e].y, c[e].z, c[e].w};
                float h[8] = {r.h[e][0].x, r.h[e][0].y, r.h[e][0].z, r.h[e][0].w, r.h[e][1].x, r.h[e][1].y, r.h[e][1].z, r.h[e][1].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 B = T::unpack(bb[i]), C = T::unpack(cc[i]);
                    h[2 * i] = fmaf(exp2_approx(x * A[2 * i]), h[2 * i], du * B.x);
                    h[2 * i + 1] = fmaf(exp2_approx(x * A[2 * i + 1]), h[2 * i + 1], du * B.y);
                    y = fmaf(h[2 * i], C.x, fmaf(h[2 * i + 1], C.y, y));
                }
                float *to = block[e] + (unsigned long long)ch * N + s;
                *reinterpret_cast<float4 *>(to) = make_float4(h[0], h[1], h[2], h[3]);
                *reinterpret_cast<float4 *>(to + 4) = make_float4(h[4], h[5], h[6], h[7]);
            }
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
            if (there && s == 0) {
                y = fmaf(r.skip, u, y);
                if (a.z) y *= silu(T::unpack(r.z[e]).x);
                *reinterpret_cast<uint16_t *>(a.out + (k0 + e) * a.os + ch * 2) = (uint16_t)T::pack(y, 0.f);
            }
        }
    };
    const uint32_t ch0 = blockIdx.y * rounds * CB + threadIdx.x / LANES;
    Round r[2];
    fetch(r[0], ch0);
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {      // while the first loads are on their way
        if (k0 + e >= a.n) continue;
        if (named_before(a.reqs, k0 + e, a.reqs[k0 + e])) block[e] = nullptr;
        if (!block[e] && blockIdx.y == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
    }
    for (uint32_t i = 0; i < rounds; i += 2) {
        fetch(r[1], ch0 + (i + 1) * CB);
        work(r[0], ch0 + i * CB);
        fetch(r[0], ch0 + (i + 2) * CB);
        work(r[1], ch0 + (i + 1) * CB);
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
    const uint32_t cb = kCta / (N / 8), parts = (a.channels + cb - 1) / cb, groups = (a.n + kEntries - 1) / kEntries;
    // 8 rounds amortise a CTA's look-ups; fewer where that leaves SMs idle
    uint32_t rounds = 8;
    while (rounds > 2 && (unsigned long long)groups * ((parts + rounds - 1) / rounds) < 8ull * l.n_sms) rounds >>= 1;
    return launch_pdl(scan_step_kernel<T, N>, dim3(groups, (parts + rounds - 1) / rounds), dim3(kCta), 0, l.stream, g, a, rounds);
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
