// Short causal convolution over the rows of a state layer, with the window that its block keeps:
//     y_t = act(b + sum_j w_j x_(t - W + 1 + j)),   act(y) = y or y / (1 + e^-y),   window <- the last W - 1 rows.
//
// Bound by HBM: a prompt's element is read and written once (2 bytes each), a single token's window besides (W - 1 floats each way).
// A thread owns 8 channels (16 bytes of a row) and walks down the rows with the last W - 1 in registers.
#include "avmp_lists.cuh"

namespace avmp {

namespace {

constexpr int kCta = 128;
constexpr int kFly = 8;               // rows whose loads are in flight together

template <class T>
__device__ __forceinline__ void unpack8(const uint4 &v, float (&x)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = T::unpack(w[i]);
        x[2 * i] = p.x; x[2 * i + 1] = p.y;
    }
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8])
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// Taps of 8 channels.
template <int W>
struct Taps {
    float w[8][W], b[8];
    __device__ void load(const ConvArgs &a, uint32_t ch)
    {
        float *to = &w[0][0];
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) {
            const float4 v = *reinterpret_cast<const float4 *>(a.weight + (unsigned long long)ch * W + i * 4);
            to[4 * i] = v.x; to[4 * i + 1] = v.y; to[4 * i + 2] = v.z; to[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = 0.f;
        if (a.bias) load8(a.bias + ch, b);
    }
    // One row: old[0] is the oldest.  Moves the rows up.
    template <class T>
    __device__ uint4 row(float (&old)[W - 1][8], const float (&x)[8], bool act) const
    {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = b[i];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) y[i] = fmaf(w[i][j], old[j][i], y[i]);
            y[i] = fmaf(w[i][W - 1], x[i], y[i]);
            if (act) y[i] = silu(y[i]);
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) old[j][i] = old[j + 1][i];
            old[W - 2][i] = x[i];
        }
        return make_uint4(T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7]));
    }
};

// CTA (i, c): runs i, i + gridDim.x, .. of all entries, channels c * 1024 and on.  The CTA of an entry's first run reads the old window
// and, behind that, writes the new one: nobody else touches it.
template <class T, int W>
__global__ void __launch_bounds__(kCta) conv_prompt_kernel(const Geom g, const ConvArgs a, uint32_t rows)
{
    __shared__ uint32_t pre[kCta + 1];
    __shared__ unsigned long long tmp[32];
    pdl_prologue();
    const uint32_t ch = (blockIdx.y * kCta + threadIdx.x) * 8;
    const bool mine = ch < a.channels;
    Taps<W> taps;
    if (mine) taps.load(a, ch);
    Runs runs(a.cu, a.n, a.total, rows, pre, tmp);
    uint32_t k, run;
    for (unsigned long long i = blockIdx.x; runs.seek(i, &k, &run); i += gridDim.x) {
        const uint32_t r = a.reqs[k], c0 = a.cu[k], c1 = a.cu[k + 1];
        float *block = state_block(g, a.layer, r);
        if (named_before(a.reqs, k, r) || !block || c1 < c0 || c1 > a.total) {
            if (run == 0 && blockIdx.y == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            continue;
        }
        if (!mine) continue;
        const uint32_t len = c1 - c0, t0 = run * rows, t1 = min(len, t0 + rows);
        const uint8_t *x = a.x + (unsigned long long)c0 * a.xs + ch * 2;
        uint8_t *out = a.out + (unsigned long long)c0 * a.os + ch * 2;
        float *window = block + a.state_elems + ch;
        const bool kept = a.resume && a.resume[k];
        float old[W - 1][8];
        // row p of the request, from its inputs, the window in front of them, or nothing
        auto before = [&](int p, float (&v)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
            if (p >= 0) unpack8<T>(*reinterpret_cast<const uint4 *>(x + (unsigned long long)p * a.xs), v);
            else if (kept) load8(window + (unsigned long long)(p + W - 1) * a.channels, v);
        };
#pragma unroll
        for (int j = 0; j < W - 1; ++j) before((int)t0 - (W - 1) + j, old[j]);
        if (run == 0) {
            float last[W - 1][8];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) before((int)len - (W - 1) + j, last[j]);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) store8(window + (unsigned long long)j * a.channels, last[j]);
        }
        for (uint32_t t = t0; t < t1; t += kFly) {
            uint4 v[kFly];
#pragma unroll
            for (int e = 0; e < kFly; ++e)
                if (t + e < t1) v[e] = *reinterpret_cast<const uint4 *>(x + (unsigned long long)(t + e) * a.xs);
#pragma unroll
            for (int e = 0; e < kFly; ++e) {
                if (t + e >= t1) break;
                float y[8];
                unpack8<T>(v[e], y);
                *reinterpret_cast<uint4 *>(out + (unsigned long long)(t + e) * a.os) = taps.template row<T>(old, y, a.act);
            }
        }
    }
}

// CTA (i, c): entries i * each and on.
template <class T, int W>
__global__ void __launch_bounds__(kCta) conv_step_kernel(const Geom g, const ConvArgs a, uint32_t each)
{
    pdl_prologue();
    const uint32_t ch = (blockIdx.y * kCta + threadIdx.x) * 8;
    const bool mine = ch < a.channels;
    Taps<W> taps;
    if (mine) taps.load(a, ch);
    for (uint32_t k = blockIdx.x * each; k < min(a.n, (blockIdx.x + 1) * each); ++k) {
        const uint32_t r = a.reqs[k];
        float *block = state_block(g, a.layer, r), *window = block + a.state_elems + ch;
        float old[W - 1][8], x[8];
        if (mine && block) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) load8(window + (unsigned long long)j * a.channels, old[j]);
            unpack8<T>(*reinterpret_cast<const uint4 *>(a.x + k * a.xs + ch * 2), x);
        }
        if (named_before(a.reqs, k, r) || !block) {
            if (blockIdx.y == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            continue;
        }
        if (!mine) continue;
        *reinterpret_cast<uint4 *>(a.out + k * a.os + ch * 2) = taps.template row<T>(old, x, a.act);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) store8(window + (unsigned long long)j * a.channels, old[j]);
    }
}

template <class T, int W>
cudaError_t prompt_launch(const Geom &g, const ConvArgs &a, const Launch &l)
{
    const uint32_t parts = (a.channels + 8 * kCta - 1) / (8 * kCta);
    // Runs of 64 rows read 5 % of them twice; shorter ones where that leaves SMs idle.
    uint32_t rows = 64;
    while (rows > 8 && (unsigned long long)(a.total / rows) * parts < 8ull * l.n_sms) rows >>= 1;
    const unsigned long long runs = (unsigned long long)a.total / rows + a.n;
    return launch_pdl(conv_prompt_kernel<T, W>, dim3((uint32_t)min(runs, 1ull << 20), parts), dim3(kCta), 0, l.stream, g, a, rows);
}
template <class T, int W>
cudaError_t step_launch(const Geom &g, const ConvArgs &a, const Launch &l)
{
    const uint32_t parts = (a.channels + 8 * kCta - 1) / (8 * kCta);
    uint32_t each = 4;
    while (each > 1 && (unsigned long long)(a.n / each) * parts < 8ull * l.n_sms) each >>= 1;
    return launch_pdl(conv_step_kernel<T, W>, dim3((a.n + each - 1) / each, parts), dim3(kCta), 0, l.stream, g, a, each);
}
template <class T>
cudaError_t launch(const Geom &g, const ConvArgs &a, const Launch &l)
{
    switch (a.width) {
    case 2: return a.cu ? prompt_launch<T, 2>(g, a, l) : step_launch<T, 2>(g, a, l);
    case 3: return a.cu ? prompt_launch<T, 3>(g, a, l) : step_launch<T, 3>(g, a, l);
    default: return a.cu ? prompt_launch<T, 4>(g, a, l) : step_launch<T, 4>(g, a, l);
    }
}

}  // namespace

cudaError_t launch_conv(const Geom &g, const ConvArgs &a, const Launch &l) { return a.f16 ? launch<F16>(g, a, l) : launch<Bf16>(g, a, l); }

}  // namespace avmp
