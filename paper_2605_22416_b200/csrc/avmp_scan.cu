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

// log(1 + e^x)
__device__ __forceinline__ float softplus(float x) { return x > 20.f ? x : log1pf(expf(x)); }

constexpr int kCta = 128;
constexpr float kLog2e = 1.4426950408889634f;

// ---------------------------------------------------------------- whole prompts
// One CTA per (request, CB channels of a group, run of tokens).  A warp holds 8 K channels: lane 8 q + c has quarter q of the states of K
// channels, and works for them token by token; in four tokens the quarters' products with C are summed across lanes such that lane
// 8 q + c ends up with token q, which it finishes.  The rows come in by asynchronous copies, kTok tokens at a time, two such tiles
// ahead; step sizes are worked out once per token and channel, a tile ahead of their use.
// Where requests and channels leave SMs idle, every prompt is cut into `shares` runs: a first pass leaves, for every run but the last,
// the state that it makes from nothing, and the sum of its steps (whose product with A is the run's whole decay); a second pass
// starts every run from those in front of it.
constexpr int kTok = 32;
constexpr int kStages = 3;

template <int N, int K>
struct Tile {
    static constexpr int CB = kCta / 32 * 8 * K;                     // channels of a CTA
    static constexpr int P = N / 8;                                  // pairs of states of a lane
    static constexpr uint32_t kRow = CB * 2 + (K == 2 ? 32 : 0);     // bytes between staged rows (four tokens side by side: no bank twice)
    static constexpr uint32_t kRows = kTok * kRow, kBc = kTok * N * 2;
    static constexpr uint32_t kStage = 3 * kRows + 2 * kBc;          // u, d, z (then out), B, C
    static constexpr uint32_t oSteps = kStages * kStage;             // (D, D u) of a tile, [token][channel]
    static constexpr uint32_t oBc = oSteps + kTok * CB * 8;          // B and C of a tile in 32 bits, [B or C][token][state]
    static constexpr uint32_t kTotal = oBc + 2 * kTok * N * 4;
};

template <class T, int N, int K>
__global__ void __launch_bounds__(kCta) scan_prompt_kernel(const Geom g, const ScanArgs a, uint32_t tiles, uint32_t shares, bool locals)
{
    using L = Tile<N, K>;
    constexpr int CB = L::CB, P = L::P;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ uint32_t order[kCta];
    pdl_prologue();
    const uint32_t base = smem_u32(smem);
    const int w = threadIdx.x / 32, lane = threadIdx.x % 32, q = lane >> 3, c = lane & 7;
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
    const uint32_t mych = (w * 8 + c) * K;                                   // this lane's first channel of the CTA
    const bool mine = mych < chs;

    // ---- what comes in: 16-byte units of rows, zeros behind the last row and channel
    const uint8_t *urow = a.u + (unsigned long long)(c0 + t0) * a.us + ch0 * 2, *drow = a.d + (unsigned long long)(c0 + t0) * a.ds + ch0 * 2;
    const uint8_t *zrow = a.z ? a.z + (unsigned long long)(c0 + t0) * a.zs + ch0 * 2 : nullptr;
    const uint8_t *brow = a.b + (unsigned long long)(c0 + t0) * a.bs + grp * N * 2, *crow = a.c + (unsigned long long)(c0 + t0) * a.cs + grp * N * 2;
    auto load = [&](uint32_t i) {
        if (i < n_tiles) {
            const uint32_t at = base + i % kStages * L::kStage, rows = t1 - t0 - i * kTok;
#pragma unroll
            for (int x = 0; x < kTok * CB / 8 / kCta; ++x) {
                const uint32_t y = threadIdx.x + x * kCta, t = y / (CB / 8), e = y % (CB / 8);
                const bool there = t < rows && e * 8 < chs;
                const uint32_t dst = at + t * L::kRow + e * 16;
                const unsigned long long tok = i * kTok + t;
                cp_async16(dst, there ? urow + tok * a.us + e * 16 : a.u, there);
                cp_async16(dst + L::kRows, there ? drow + tok * a.ds + e * 16 : a.u, there);
                if (zrow && !locals) cp_async16(dst + 2 * L::kRows, there ? zrow + tok * a.zs + e * 16 : a.u, there);
            }
            for (uint32_t y = threadIdx.x; y < kTok * N / 8; y += kCta) {
                const uint32_t t = y / (N / 8), e = y % (N / 8), dst = at + 3 * L::kRows + y * 16;
                const bool there = t < rows;
                cp_async16(dst, there ? brow + (i * kTok + t) * a.bs + e * 16 : a.u, there);
                if (!locals) cp_async16(dst + L::kBc, there ? crow + (i * kTok + t) * a.cs + e * 16 : a.u, there);
            }
        }
        cp_async_commit();
    };
    load(0);
    load(1);

    // ---- this lane's part of the state, and what belongs to its channels
    unsigned long long A[K][P], h[K][P];
    float bias[K], skip[K], sum[K];
    const uint32_t states = q * (N / 4);
#pragma unroll
    for (int x = 0; x < K; ++x) {
        const uint32_t ch = ch0 + mych + x;
        bias[x] = skip[x] = sum[x] = 0.f;
        if (mine && a.bias) bias[x] = a.bias[ch];
        if (mine && a.skip) skip[x] = a.skip[ch];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float2 v = make_float2(0.f, 0.f);
            if (mine) v = *reinterpret_cast<const float2 *>(a.a + (unsigned long long)ch * N + states + 2 * p);
            A[x][p] = pack2(v.x * kLog2e, v.y * kLog2e);
            h[x][p] = pack2(0.f, 0.f);
        }
    }
    // In the workspace: [entry][run][channel][state], slot 0 what the request starts from, slot j what run j - 1 makes; the sums of steps behind.
    const unsigned long long slot = (unsigned long long)a.channels * N, sums = (unsigned long long)a.n * shares * slot;
    auto ws_state = [&](uint32_t j, int x, int p) {
        return reinterpret_cast<float2 *>(a.ws + ((unsigned long long)k * shares + j) * slot + (unsigned long long)(ch0 + mych + x) * N + states + 2 * p);
    };
    auto ws_sum = [&](uint32_t j, int x) { return a.ws + sums + ((unsigned long long)k * shares + j) * a.channels + ch0 + mych + x; };
    if (shares == 1 || locals) {
        const bool kept = a.resume && a.resume[k];
        if (run == 0 && mine) {
#pragma unroll
            for (int x = 0; x < K; ++x)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    float2 v = make_float2(0.f, 0.f);
                    if (kept) v = *reinterpret_cast<const float2 *>(block + (unsigned long long)(ch0 + mych + x) * N + states + 2 * p);
                    if (locals) *ws_state(0, x, p) = v; else h[x][p] = pack2(v.x, v.y);
                }
        }
    } else if (mine) {
        for (uint32_t j = 0; j <= run; ++j)
#pragma unroll
            for (int x = 0; x < K; ++x) {
                const float s = j ? *ws_sum(j, x) : 0.f;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float2 v = *ws_state(j, x, p), d = unpack2(mul2(A[x][p], pack2(s, s)));
                    h[x][p] = j ? fma2(pack2(exp2_approx(d.x), exp2_approx(d.y)), h[x][p], pack2(v.x, v.y)) : pack2(v.x, v.y);
                }
            }
    }

    float2 *steps = reinterpret_cast<float2 *>(smem + L::oSteps);
    float *bc = reinterpret_cast<float *>(smem + L::oBc);
    auto put_out = [&](uint32_t i) {
        const uint8_t *from = smem + i % kStages * L::kStage + 2 * L::kRows;
        const uint32_t rows = t1 - t0 - i * kTok;
#pragma unroll
        for (int x = 0; x < kTok * CB / 8 / kCta; ++x) {
            const uint32_t y = threadIdx.x + x * kCta, t = y / (CB / 8), e = y % (CB / 8);
            if (t < rows && e * 8 < chs)
                *reinterpret_cast<uint4 *>(a.out + (unsigned long long)(c0 + t0 + i * kTok + t) * a.os + (ch0 + e * 8) * 2) =
                    *reinterpret_cast<const uint4 *>(from + t * L::kRow + e * 16);
        }
    };
    for (uint32_t i = 0; i < n_tiles; ++i) {
        uint8_t *at = smem + i % kStages * L::kStage;
        const uint32_t rows = t1 - t0 - i * kTok;
        cp_async_wait<1>();
        __syncthreads();
        if (i && !locals) put_out(i - 1);
        // step sizes of this warp's channels
#pragma unroll
        for (int y = 0; y < kTok / 4; ++y) {
            const uint32_t t = y * 4 + q;
            uint32_t du[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint8_t *p = at + x * L::kRows + t * L::kRow + mych * 2;
                du[x] = K == 2 ? *reinterpret_cast<const uint32_t *>(p) : *reinterpret_cast<const uint16_t *>(p);
            }
            const float2 u = T::unpack(du[0]), d = T::unpack(du[1]);
#pragma unroll
            for (int x = 0; x < K; ++x) {
                float v = (x ? d.y : d.x) + bias[x];
                if (a.softplus) v = softplus(v);
                if (t >= rows) v = 0.f;
                steps[t * CB + mych + x] = make_float2(v, t < rows ? v * (x ? u.y : u.x) : 0.f);
                if (locals) sum[x] += v;
            }
        }
        for (uint32_t y = threadIdx.x; y < (locals ? 1u : 2u) * kTok * N / 4; y += kCta) {
            const uint2 v = *reinterpret_cast<const uint2 *>(at + 3 * L::kRows + y * 8);
            const float2 lo = T::unpack(v.x), hi = T::unpack(v.y);
            *reinterpret_cast<float4 *>(bc + y * 4) = make_float4(lo.x, lo.y, hi.x, hi.y);
        }
        __syncthreads();
        load(i + 2);
        const float2 *st = steps + mych;
        const float *bq = bc + states, *cq = bq + kTok * N;
        for (int t = 0; t < kTok; t += 4) {
            float y[K][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned long long B[P], C[P];
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    B[p] = *reinterpret_cast<const unsigned long long *>(bq + (t + j) * N + 2 * p);
                    C[p] = locals ? 0ull : *reinterpret_cast<const unsigned long long *>(cq + (t + j) * N + 2 * p);
                }
#pragma unroll
                for (int x = 0; x < K; ++x) {
                    const float2 s = st[(t + j) * CB + x];
                    const unsigned long long d2 = pack2(s.x, s.x), u2 = pack2(s.y, s.y);
                    unsigned long long acc = 0;
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const float2 e = unpack2(mul2(d2, A[x][p]));
                        h[x][p] = fma2(pack2(exp2_approx(e.x), exp2_approx(e.y)), h[x][p], mul2(u2, B[p]));
                        acc = p ? fma2(h[x][p], C[p], acc) : mul2(h[x][p], C[p]);
                    }
                    const float2 z = unpack2(acc);
                    y[x][j] = z.x + z.y;
                }
            }
            if (locals) continue;
            float o[K];
#pragma unroll
            for (int x = 0; x < K; ++x) {
                const bool hi = q & 2, odd = q & 1;
                const float s0 = __shfl_xor_sync(0xFFFFFFFFu, hi ? y[x][0] : y[x][2], 16), s1 = __shfl_xor_sync(0xFFFFFFFFu, hi ? y[x][1] : y[x][3], 16);
                const float a0 = (hi ? y[x][2] : y[x][0]) + s0, a1 = (hi ? y[x][3] : y[x][1]) + s1;
                o[x] = (odd ? a1 : a0) + __shfl_xor_sync(0xFFFFFFFFu, odd ? a0 : a1, 8);
            }
            uint8_t *p = at + (t + q) * L::kRow + mych * 2;
            const uint32_t uu = K == 2 ? *reinterpret_cast<const uint32_t *>(p) : *reinterpret_cast<const uint16_t *>(p);
            const float2 u = T::unpack(uu);
            o[0] = fmaf(skip[0], u.x, o[0]);
            if (K == 2) o[K - 1] = fmaf(skip[K - 1], u.y, o[K - 1]);
            p += 2 * L::kRows;
            if (zrow) {
                const uint32_t zz = K == 2 ? *reinterpret_cast<const uint32_t *>(p) : *reinterpret_cast<const uint16_t *>(p);
                const float2 z = T::unpack(zz);
                o[0] *= silu(z.x);
                if (K == 2) o[K - 1] *= silu(z.y);
            }
            if (K == 2) *reinterpret_cast<uint32_t *>(p) = T::pack(o[0], o[K - 1]);
            else *reinterpret_cast<uint16_t *>(p) = (uint16_t)T::pack(o[0], 0.f);
        }
    }
    cp_async_wait<0>();
    if (locals) {
#pragma unroll
        for (int x = 0; x < K; ++x) {
            // a lane has summed every fourth token's steps
            sum[x] += __shfl_xor_sync(0xFFFFFFFFu, sum[x], 8);
            sum[x] += __shfl_xor_sync(0xFFFFFFFFu, sum[x], 16);
            if (!mine) continue;
            if (q == 0) *ws_sum(run + 1, x) = sum[x];
#pragma unroll
            for (int p = 0; p < P; ++p) *ws_state(run + 1, x, p) = unpack2(h[x][p]);
        }
        return;
    }
    __syncthreads();
    if (n_tiles) put_out(n_tiles - 1);
    if (run == shares - 1 && mine)
#pragma unroll
        for (int x = 0; x < K; ++x)
#pragma unroll
            for (int p = 0; p < P; ++p)
                *reinterpret_cast<float2 *>(block + (unsigned long long)(ch0 + mych + x) * N + states + 2 * p) = unpack2(h[x][p]);
}

// ---------------------------------------------------------------- one token
// CTA (i, j): kEntries entries, every gridDim.y-th run of kCta * 4 / N channels.  A thread has four states of a channel, for all entries of the CTA:
// their decays stay in registers.
constexpr int kEntries = 2;

template <class T, int N>
__global__ void __launch_bounds__(kCta) scan_step_kernel(const Geom g, const ScanArgs a)
{
    constexpr int LANES = N / 4;
    constexpr uint32_t CB = kCta / LANES;
    pdl_prologue();
    const uint32_t k0 = blockIdx.x * kEntries, s = threadIdx.x % LANES * 4;
    float *block[kEntries];
#pragma unroll
    for (int e = 0; e < kEntries; ++e) block[e] = k0 + e < a.n ? state_block(g, a.layer, a.reqs[k0 + e]) : nullptr;
    bool checked = false;
    const uint32_t per_group = a.channels / a.groups;
    for (uint32_t ch = blockIdx.y * CB + threadIdx.x / LANES; ch - threadIdx.x / LANES < a.channels; ch += gridDim.y * CB) {
        const bool mine = ch < a.channels;
        const unsigned long long at = (unsigned long long)ch * N + s;
        float4 h[kEntries], A = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int e = 0; e < kEntries; ++e)
            if (mine && block[e]) h[e] = *reinterpret_cast<const float4 *>(block[e] + at);
        if (mine) A = *reinterpret_cast<const float4 *>(a.a + at);
        if (!checked) {          // while the first loads are on their way
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                if (k0 + e >= a.n) continue;
                if (named_before(a.reqs, k0 + e, a.reqs[k0 + e])) block[e] = nullptr;
                if (!block[e] && blockIdx.y == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            }
            checked = true;
        }
        const uint32_t grp = mine ? ch / per_group : 0u;
        const float bias = mine && a.bias ? a.bias[ch] : 0.f, skip = mine && a.skip ? a.skip[ch] : 0.f;
#pragma unroll
        for (int e = 0; e < kEntries; ++e) {
            const uint32_t k = k0 + e;
            float y = 0.f, u = 0.f;
            if (mine && block[e]) {
                u = T::unpack(*reinterpret_cast<const uint16_t *>(a.u + k * a.us + ch * 2)).x;
                float d = T::unpack(*reinterpret_cast<const uint16_t *>(a.d + k * a.ds + ch * 2)).x + bias;
                if (a.softplus) d = softplus(d);
                const uint2 bb = *reinterpret_cast<const uint2 *>(a.b + k * a.bs + (grp * N + s) * 2);
                const uint2 cc = *reinterpret_cast<const uint2 *>(a.c + k * a.cs + (grp * N + s) * 2);
                const float2 b0 = T::unpack(bb.x), b1 = T::unpack(bb.y), c0 = T::unpack(cc.x), c1 = T::unpack(cc.y);
                const float du = d * u, x = d * kLog2e;
                h[e].x = fmaf(exp2_approx(x * A.x), h[e].x, du * b0.x);
                h[e].y = fmaf(exp2_approx(x * A.y), h[e].y, du * b0.y);
                h[e].z = fmaf(exp2_approx(x * A.z), h[e].z, du * b1.x);
                h[e].w = fmaf(exp2_approx(x * A.w), h[e].w, du * b1.y);
                *reinterpret_cast<float4 *>(block[e] + at) = h[e];
                y = h[e].x * c0.x + h[e].y * c0.y + h[e].z * c1.x + h[e].w * c1.y;
            }
#pragma unroll
            for (int o = LANES / 2; o; o >>= 1) y += __shfl_xor_sync(0xFFFFFFFFu, y, o);
            if (mine && block[e] && s == 0) {
                y = fmaf(skip, u, y);
                if (a.z) y *= silu(T::unpack(*reinterpret_cast<const uint16_t *>(a.z + k * a.zs + ch * 2)).x);
                *reinterpret_cast<uint16_t *>(a.out + k * a.os + ch * 2) = (uint16_t)T::pack(y, 0.f);
            }
        }
    }
}

template <int N, int K>
uint32_t tiles_of(const ScanArgs &a)
{
    const uint32_t per_group = a.channels / a.groups;
    return a.groups * ((per_group + Tile<N, K>::CB - 1) / Tile<N, K>::CB);
}

template <class T, int N, int K>
cudaError_t prompt_launch(const Geom &g, const ScanArgs &a, const Launch &l, uint32_t *launched)
{
    using L = Tile<N, K>;
    static_assert(L::kTotal <= 227 * 1024, "shared memory of one CTA");
    cudaError_t e = allow_smem<scan_prompt_kernel<T, N, K>>(l.device, L::kTotal);
    if (e != cudaSuccess) return e;
    const uint32_t tiles = tiles_of<N, K>(a), shares = a.shares;
    if (shares > 1) {
        e = launch_pdl(scan_prompt_kernel<T, N, K>, dim3(a.n * tiles * (shares - 1)), dim3(kCta), L::kTotal, l.stream, g, a, tiles, shares, true);
        if (e != cudaSuccess) return e;
        *launched += 1;
    }
    *launched += 1;
    return launch_pdl(scan_prompt_kernel<T, N, K>, dim3(a.n * tiles * shares), dim3(kCta), L::kTotal, l.stream, g, a, tiles, shares, false);
}
template <class T, int N>
cudaError_t prompt_width(const Geom &g, const ScanArgs &a, const Launch &l, uint32_t *launched)
{
    if (N <= 16 && (unsigned long long)a.n * tiles_of<N, 2>(a) >= 8ull * l.n_sms) return prompt_launch<T, N, N <= 16 ? 2 : 1>(g, a, l, launched);
    return prompt_launch<T, N, 1>(g, a, l, launched);
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
    const uint32_t cb = kCta / (N / 4), parts = (a.channels + cb - 1) / cb, groups = (a.n + kEntries - 1) / kEntries;
    // 8 rounds amortise a CTA's look-ups; fewer where that leaves SMs idle
    uint32_t rounds = 8;
    while (rounds > 1 && (unsigned long long)groups * ((parts + rounds - 1) / rounds) < 16ull * l.n_sms) rounds >>= 1;
    return launch_pdl(scan_step_kernel<T, N>, dim3(groups, (parts + rounds - 1) / rounds), dim3(kCta), 0, l.stream, g, a);
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

// Runs that each prompt is cut into; 1 where the first pass would cost more than it gives.
uint32_t scan_shares(uint32_t n, uint32_t channels, uint32_t groups, uint32_t total, int n_sms)
{
    const unsigned long long items = (unsigned long long)n * groups * ((channels / groups + 31) / 32);
    unsigned long long s = 4ull * n_sms / items;
    if (s > total / n / (8 * kTok)) s = total / n / (8 * kTok);
    return s < 3 ? 1u : (uint32_t)(s < 32 ? s : 32);
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
