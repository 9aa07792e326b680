// Between a projection and attention: every query and key head of the new tokens is normalised,
//     y = x / sqrt(mean(x^2) + eps) * weight,
// its leading columns are rotated by the token's position (pairs of columns as complex numbers, times e^(i position freq)), keys and
// values are written to their pages and queries to a buffer; all in one pass.
//
// Bound by HBM: every element is read once and written once, 2 bytes each way.  A lane has 8 columns of a head such that both columns of
// every pair are its own; sines and cosines are worked out once for all heads of a token.  Angles are taken in 64 bits: 2^-24 of a far
// position's angle would be thousandths of a turn.
#include "avmp_lists.cuh"
#include "avmp_tc.cuh"

namespace avmp {

namespace {

constexpr int kCta = 128;
constexpr int kMostRows = 4;          // tokens of a run
constexpr int kFly = 4;               // heads of a lane whose loads are in flight together

// NEIGHBOURS: pairs are columns (2 i, 2 i + 1), else (i, i + rotary / 2).
template <class T, int D, bool NEIGHBOURS>
__global__ void __launch_bounds__(kCta) rows_kernel(const Geom g, const RowsArgs a, uint32_t rows)
{
    constexpr uint32_t LANES = D / 8, HEADS = 32 / LANES;      // lanes of a head; heads a warp has at a time
    __shared__ uint32_t pre[kCta + 1];
    __shared__ unsigned long long tmp[32];
    __shared__ __align__(16) float cosine[kMostRows][D / 2], sine[kMostRows][D / 2], weight[2][D];
    __shared__ uint8_t *page[kMostRows];
    pdl_prologue();
    const uint32_t half = a.rotary / 2, w = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % LANES;
    for (uint32_t i = threadIdx.x; i < 2 * D; i += kCta) {
        const float *from = i < D ? a.wq : a.wk;
        weight[i / D][i % D] = from ? from[i % D] : 1.f;
    }
    // this lane's columns: f .. f + 3 and s .. s + 3
    const bool turns = 8 * l < a.rotary;
    const uint32_t f = NEIGHBOURS || !turns ? 8 * l : 4 * l, s = NEIGHBOURS || !turns ? 8 * l + 4 : half + 4 * l;
    const uint32_t heads = a.q_heads + 2 * a.kv_heads, chunks = (heads + HEADS - 1) / HEADS;
    Runs runs(a.cu, a.n, a.total, rows, pre, tmp);
    uint32_t k, run;
    for (unsigned long long i = blockIdx.x; runs.seek(i, &k, &run); i += gridDim.x) {
        const uint32_t r = a.reqs[k], c0 = a.cu ? a.cu[k] : k, c1 = a.cu ? a.cu[k + 1] : k + 1, held = held_tokens(g, r);
        if (named_before(a.reqs, k, r) || held == 0 || c1 < c0 || c1 > a.total || c1 - c0 > held) {
            if (run == 0 && threadIdx.x == 0) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            continue;
        }
        const uint32_t first = c0 + run * rows, count = min(rows, c1 - first), place = held - (c1 - first);      // place of the run's first token in the chain
        uint32_t t = 0, chunk = w;
        auto settle = [&] { while (chunk >= chunks) { chunk -= chunks; ++t; } };
        uint4 x[kFly];
        uint32_t head[kFly], tok[kFly];
        auto fetch = [&] {
#pragma unroll
            for (int e = 0; e < kFly; ++e) {
                head[e] = t < count ? chunk * HEADS + lane / LANES : heads;
                tok[e] = t;
                chunk += kCta / 32;
                settle();
                if (head[e] >= heads) continue;
                const unsigned long long row = first + tok[e];
                const uint8_t *from = head[e] < a.q_heads ? a.q + row * a.qs + head[e] * D * 2
                    : head[e] < a.q_heads + a.kv_heads ? a.k + row * a.ks + (head[e] - a.q_heads) * D * 2
                                                       : a.v + row * a.vs + (head[e] - a.q_heads - a.kv_heads) * D * 2;
                if (NEIGHBOURS) {
                    x[e] = *reinterpret_cast<const uint4 *>(from + f * 2);
                } else {
                    const uint2 lo = *reinterpret_cast<const uint2 *>(from + f * 2), hi = *reinterpret_cast<const uint2 *>(from + s * 2);
                    x[e] = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
        };
        settle();
        fetch();                      // while the pages are looked up
        if (threadIdx.x < count) {
            const uint32_t p = place + threadIdx.x, h = __ldcg(g.r_chain + ((unsigned long long)r * g.max_pages + p / g.T));
            page[threadIdx.x] = unit_ptr(g, AVMP_POOL_KV, __ldcg(g.VT[0] + (h & 0x7FFFFFFFu))) + a.layer * g.kv_layer_bytes + p % g.T * g.row_bytes;
        }
        for (uint32_t x = threadIdx.x; x < count * half; x += kCta) {
            const uint32_t t = x / half, j = x % half;
            const double turn = (double)(a.pos ? a.pos[first + t] : place + t) * (double)a.freq[j] * 0.15915494309189533577;
            float sn, cs;
            sincospif((float)(2.0 * (turn - rint(turn))), &sn, &cs);
            cosine[t][j] = cs; sine[t][j] = sn;
        }
        __syncthreads();
        for (;;) {
#pragma unroll
            for (int e = 0; e < kFly; ++e) {
                const bool there = head[e] < heads, is_q = head[e] < a.q_heads, is_v = head[e] >= a.q_heads + a.kv_heads;
                const uint32_t in[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
                float y[8], sq = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 v = there ? T::unpack(in[j]) : make_float2(0.f, 0.f);
                    y[2 * j] = v.x; y[2 * j + 1] = v.y;
                    sq = fmaf(v.x, v.x, fmaf(v.y, v.y, sq));
                }
#pragma unroll
                for (uint32_t o = LANES / 2; o; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
                if (!there) continue;
                uint4 to = x[e];
                if (!is_v) {
                    if (is_q ? a.wq != nullptr : a.wk != nullptr) {
                        const float by = rsqrtf(sq * (1.f / D) + a.eps);
                        const float4 w0 = *reinterpret_cast<const float4 *>(&weight[is_q ? 0 : 1][f]), w1 = *reinterpret_cast<const float4 *>(&weight[is_q ? 0 : 1][s]);
                        y[0] *= by * w0.x; y[1] *= by * w0.y; y[2] *= by * w0.z; y[3] *= by * w0.w;
                        y[4] *= by * w1.x; y[5] *= by * w1.y; y[6] *= by * w1.z; y[7] *= by * w1.w;
                    }
                    if (turns) {
                        const float4 c4 = *reinterpret_cast<const float4 *>(&cosine[tok[e]][4 * l]), s4 = *reinterpret_cast<const float4 *>(&sine[tok[e]][4 * l]);
                        const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float &p = y[NEIGHBOURS ? 2 * j : j], &o = y[NEIGHBOURS ? 2 * j + 1 : j + 4];
                            const float re = p * cs[j] - o * sn[j], im = o * cs[j] + p * sn[j];
                            p = re; o = im;
                        }
                    }
                    to = make_uint4(T::pack(y[0], y[1]), T::pack(y[2], y[3]), T::pack(y[4], y[5]), T::pack(y[6], y[7]));
                }
                uint8_t *dst = is_q ? a.out + (unsigned long long)(first + tok[e]) * a.os + head[e] * D * 2
                             : page[tok[e]] + (is_v ? g.T * g.row_bytes + (head[e] - a.q_heads - a.kv_heads) * D * 2 : (unsigned long long)(head[e] - a.q_heads) * D * 2);
                if (NEIGHBOURS) {
                    *reinterpret_cast<uint4 *>(dst + f * 2) = to;
                } else {
                    *reinterpret_cast<uint2 *>(dst + f * 2) = make_uint2(to.x, to.y);
                    *reinterpret_cast<uint2 *>(dst + s * 2) = make_uint2(to.z, to.w);
                }
            }
            if (t >= count) break;
            fetch();
        }
        __syncthreads();
    }
}

template <class T, int D>
cudaError_t launch(const Geom &g, const RowsArgs &a, const Launch &l)
{
    uint32_t rows = a.cu ? kMostRows : 1;
    while (rows > 1 && a.total / rows < 16u * l.n_sms) rows >>= 1;
    const unsigned long long runs = a.cu ? (unsigned long long)a.total / rows + a.n : a.n;
    const dim3 grid((uint32_t)min(runs, 1ull << 20));
    return a.neighbours ? launch_pdl(rows_kernel<T, D, true>, grid, dim3(kCta), 0, l.stream, g, a, rows)
                        : launch_pdl(rows_kernel<T, D, false>, grid, dim3(kCta), 0, l.stream, g, a, rows);
}

}  // namespace

cudaError_t launch_attn_rows(const Geom &g, const RowsArgs &a, const Launch &l)
{
    if (a.head_dim == 128) return a.f16 ? launch<F16, 128>(g, a, l) : launch<Bf16, 128>(g, a, l);
    return a.f16 ? launch<F16, 64>(g, a, l) : launch<Bf16, 64>(g, a, l);
}

}  // namespace avmp
