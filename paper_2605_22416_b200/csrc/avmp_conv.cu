// Short causal convolution over the rows of a state layer, with the window that its block keeps:
//     y_t = act(b + sum_j w_j x_(t - W + 1 + j)),   act(y) = y or y / (1 + e^-y),   window <- the last W - 1 rows.
//
// Bound by HBM: a prompt's element is read and written once (2 bytes each), a single token's window besides (W - 1 floats each way).
// A thread owns 4 channels (8 bytes of a row) and walks down the rows with the last W - 1 in registers.  The rows come through a ring in shared
// memory by asynchronous copies, each thread's for itself, so that their number in flight costs no registers (loads into registers: 607 us
// with 4 channels a thread, 668 with 8, for what takes 358 so).
//
// Measured (width 4, bf16): 66 000 rows of 8192 channels 355 to 359 us (a copy of as many bytes: 338 to 343; 392 in turn on three sets of buffers),
// 32 prompts of 32 to 512 rows, 2048 channels, 16 (floor 7.6); one token for 1023 requests of 16 384 channels 78 us (92 % of the
// measured copy rate), for 32 of 2048 channels 2.6 (latency).
#include "avmp_lists.cuh"

namespace avmp {

namespace {

constexpr int kCta = 128;
constexpr int kCh = 4;                // channels of a thread
constexpr int kFly = 4;               // rows of a stage
constexpr int kStages = 5;            // stages of the ring: one is worked on, the others are on their way

template <class T>
__device__ __forceinline__ void unpack4(const uint2 &v, float (&x)[kCh])
{
    const float2 p = T::unpack(v.x), q = T::unpack(v.y);
    x[0] = p.x; x[1] = p.y; x[2] = q.x; x[3] = q.y;
}
__device__ __forceinline__ void load4(const float *p, float (&x)[kCh])
{
    const float4 a = *reinterpret_cast<const float4 *>(p);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
}
__device__ __forceinline__ void store4(float *p, const float (&x)[kCh]) { *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]); }

// Taps of a thread's channels.
template <int W>
struct Taps {
    float w[kCh][W], b[kCh];
    __device__ void load(const ConvArgs &a, uint32_t ch)
    {
        float *to = &w[0][0];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float4 v = *reinterpret_cast<const float4 *>(a.weight + (unsigned long long)ch * W + i * 4);
            to[4 * i] = v.x; to[4 * i + 1] = v.y; to[4 * i + 2] = v.z; to[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < kCh; ++i) b[i] = 0.f;
        if (a.bias) load4(a.bias + ch, b);
    }
    // One row: old[0] is the oldest.  Moves the rows up.
    template <class T, bool ACT>
    __device__ uint2 row(float (&old)[W - 1][kCh], const float (&x)[kCh]) const
    {
        float y[kCh];
#pragma unroll
        for (int i = 0; i < kCh; ++i) {
            y[i] = b[i];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) y[i] = fmaf(w[i][j], old[j][i], y[i]);
            y[i] = fmaf(w[i][W - 1], x[i], y[i]);
            if (ACT) y[i] = silu(y[i]);
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) old[j][i] = old[j + 1][i];
            old[W - 2][i] = x[i];
        }
        return make_uint2(T::pack(y[0], y[1]), T::pack(y[2], y[3]));
    }
};

// CTA (c, i): channels c * 512 and on, runs i, i + gridDim.y, .. of all entries; CTAs that run together work on the same
// rows.  The CTA of an entry's first run reads the old window
// and, behind that, writes the new one: nobody else touches it.
template <class T, int W, bool ACT>
__global__ void __launch_bounds__(kCta) conv_prompt_kernel(const Geom g, const ConvArgs a, uint32_t rows)
{
    __shared__ unsigned long long pre[kCta], tmp[32];
    __shared__ uint2 ring[kStages * kFly][kCta];
    pdl_prologue();
    const uint32_t ch = (blockIdx.x * kCta + threadIdx.x) * kCh, slot0 = smem_u32(&ring[0][threadIdx.x]);
    const bool mine = ch < a.channels;
    Taps<W> taps;
    if (mine) taps.load(a, ch);
    Runs runs(a.cu, a.n, a.total, rows, a.total, pre, tmp);
    uint32_t k, run;
    for (unsigned long long i = blockIdx.y; runs.seek(i, &k, &run); i += gridDim.y) {
        const uint32_t r = a.reqs[k], c0 = a.cu[k], c1 = a.cu[k + 1];
        const bool rows_ok = c1 >= c0 && c1 <= a.total;
        const uint32_t len = rows_ok ? c1 - c0 : 0u, t0 = run * rows, t1 = min(len, t0 + rows);
        const uint8_t *x = a.x + (unsigned long long)c0 * a.xs + ch * 2;
        uint32_t next = t0, stage_in = 0;                    // first row of the next stage, and its place in the ring
        auto load = [&] {
            const uint8_t *from = x + (unsigned long long)next * a.xs;
            const uint32_t to = slot0 + stage_in * (kFly * kCta * 8);
#pragma unroll
            for (int e = 0; e < kFly; ++e, from += a.xs)
                if (mine && next + e < t1) cp_async8(to + e * kCta * 8, from);
            cp_async_commit();
            next += kFly;
            stage_in = stage_in + 1 == kStages ? 0 : stage_in + 1;
        };
#pragma unroll
        for (int e = 0; e < kStages - 1; ++e) load();
        float *block = state_block(g, a.layer, r);
        if (named_before(a.reqs, k, r) || !block || !rows_ok) {
            if (run == 0 && blockIdx.x == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            cp_async_wait<0>();
            continue;
        }
        if (!mine) continue;
        uint8_t *out = a.out + (unsigned long long)(c0 + t0) * a.os + ch * 2;
        float *window = block + a.state_elems + ch;
        const bool kept = a.resume && a.resume[k];
        float old[W - 1][kCh];
        // row p of the request, from its inputs, the window in front of them, or nothing
        auto before = [&](int p, float (&v)[kCh]) {
#pragma unroll
            for (int e = 0; e < kCh; ++e) v[e] = 0.f;
            if (p >= 0) unpack4<T>(*reinterpret_cast<const uint2 *>(x + (unsigned long long)p * a.xs), v);
            else if (kept) load4(window + (unsigned long long)(p + W - 1) * a.channels, v);
        };
#pragma unroll
        for (int j = 0; j < W - 1; ++j) before((int)t0 - (W - 1) + j, old[j]);
        if (run == 0) {
            float last[W - 1][kCh];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) before((int)len - (W - 1) + j, last[j]);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) store4(window + (unsigned long long)j * a.channels, last[j]);
        }
        uint32_t stage = 0;
        for (uint32_t t = t0; t < t1; t += kFly) {
            load();
            cp_async_wait<kStages - 1>();
            const uint2 *from = &ring[stage * kFly][threadIdx.x];
            stage = stage + 1 == kStages ? 0 : stage + 1;
            float y[kCh];
            if (t + kFly <= t1) {
#pragma unroll
                for (int e = 0; e < kFly; ++e, out += a.os) {
                    unpack4<T>(from[e * kCta], y);
                    *reinterpret_cast<uint2 *>(out) = taps.template row<T, ACT>(old, y);
                }
            } else {
                for (uint32_t e = 0; e < t1 - t; ++e, out += a.os) {
                    unpack4<T>(from[e * kCta], y);
                    *reinterpret_cast<uint2 *>(out) = taps.template row<T, ACT>(old, y);
                }
            }
        }
        cp_async_wait<0>();
    }
}

// CTA (c, i): entries i * each and on.
template <class T, int W, bool ACT>
__global__ void __launch_bounds__(kCta) conv_step_kernel(const Geom g, const ConvArgs a, uint32_t each)
{
    pdl_prologue();
    const uint32_t ch = (blockIdx.x * kCta + threadIdx.x) * kCh;
    const bool mine = ch < a.channels;
    Taps<W> taps;
    if (mine) taps.load(a, ch);
    for (uint32_t k = blockIdx.y * each; k < min(a.n, (blockIdx.y + 1) * each); ++k) {
        const uint32_t r = a.reqs[k];
        float *block = state_block(g, a.layer, r), *window = block + a.state_elems + ch;
        float old[W - 1][kCh], x[kCh];
        if (mine && block) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) load4(window + (unsigned long long)j * a.channels, old[j]);
            unpack4<T>(*reinterpret_cast<const uint2 *>(a.x + k * a.xs + ch * 2), x);
        }
        if (named_before(a.reqs, k, r) || !block) {
            if (blockIdx.x == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            continue;
        }
        if (!mine) continue;
        *reinterpret_cast<uint2 *>(a.out + k * a.os + ch * 2) = taps.template row<T, ACT>(old, x);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) store4(window + (unsigned long long)j * a.channels, old[j]);
    }
}

template <class T, int W, bool ACT>
cudaError_t prompt_launch(const Geom &g, const ConvArgs &a, const Launch &l)
{
    const uint32_t parts = (a.channels + kCh * kCta - 1) / (kCh * kCta);
    // Runs of 128 rows read 2 % of them twice; shorter ones where that leaves SMs idle.
    uint32_t rows = 128;
    while (rows > 8 && (unsigned long long)(a.total / rows) * parts < 4ull * l.n_sms) rows >>= 1;
    const unsigned long long runs = (unsigned long long)a.total / rows + a.n;
    return launch_pdl(conv_prompt_kernel<T, W, ACT>, dim3(parts, (uint32_t)min(runs, 65535ull)), dim3(kCta), 0, l.stream, g, a, rows);
}
template <class T, int W, bool ACT>
cudaError_t step_launch(const Geom &g, const ConvArgs &a, const Launch &l)
{
    const uint32_t parts = (a.channels + kCh * kCta - 1) / (kCh * kCta);
    uint32_t each = 4;
    while (each > 1 && (unsigned long long)(a.n / each) * parts < 8ull * l.n_sms) each >>= 1;
    while ((a.n + each - 1) / each > 65535u) each <<= 1;
    return launch_pdl(conv_step_kernel<T, W, ACT>, dim3(parts, (a.n + each - 1) / each), dim3(kCta), 0, l.stream, g, a, each);
}
template <class T, bool ACT>
cudaError_t launch_width(const Geom &g, const ConvArgs &a, const Launch &l)
{
    switch (a.width) {
    case 2: return a.cu ? prompt_launch<T, 2, ACT>(g, a, l) : step_launch<T, 2, ACT>(g, a, l);
    case 3: return a.cu ? prompt_launch<T, 3, ACT>(g, a, l) : step_launch<T, 3, ACT>(g, a, l);
    default: return a.cu ? prompt_launch<T, 4, ACT>(g, a, l) : step_launch<T, 4, ACT>(g, a, l);
    }
}
template <class T>
cudaError_t launch(const Geom &g, const ConvArgs &a, const Launch &l) { return a.act ? launch_width<T, true>(g, a, l) : launch_width<T, false>(g, a, l); }

}  // namespace

cudaError_t launch_conv(const Geom &g, const ConvArgs &a, const Launch &l) { return a.f16 ? launch<F16>(g, a, l) : launch<Bf16>(g, a, l); }

}  // namespace avmp
