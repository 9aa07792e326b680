// Between a projection and attention: every query and key head of the new tokens is normalised,
//     y = x / sqrt(mean(x^2) + eps) * weight,
// its leading columns are rotated by the token's position (pairs of columns as complex numbers, times e^(i position freq)), keys and
// values are written to their pages and queries to a buffer; all in one pass.
//
// Bound by HBM: every element is read once and written once, 2 bytes each way.  A warp has one token, and of it two heads of 128 columns or four of 64 at a time;
// a lane has 8 columns of a head such that both columns of every pair are its own, so that a rotation needs no exchange, and
// weights, sines and cosines, multiplied once, serve all heads of the token from registers.  Angles are taken in 64 bits: 2^-24 of a far
// position's angle would be thousandths of a turn.  Heads come through a ring in shared memory by asynchronous copies, a lane's own columns for
// itself: with loads into registers too little is on its way (112 us for what took 82 so).
//
// Measured (heads of 128, 8 KV heads): 12 turns of 256 to 2048 tokens, 64 query heads, 78 us (83 % of the measured copy rate; 61 % of the issue slots
// are taken, 29 % of the warps' places: a token's look-ups take 2 to 3 us before its first head goes out); one token for 1024 requests,
// 32 query heads, 11 (floor 3.8), for 32 requests 5.
#include "avmp_lists.cuh"
#include "avmp_tc.cuh"

namespace avmp {

namespace {

constexpr int kCta = 128;
constexpr uint32_t kWarps = kCta / 32;
constexpr int kSteps = 2;             // a stage: so many heads (or pairs, or fours) of a warp
constexpr int kStages = 8;            // stages of the ring: one is worked on, the others are on their way

// NEIGHBOURS: pairs are columns (2 i, 2 i + 1), else (i, i + rotary / 2).
template <class T, int D, bool NEIGHBOURS>
__global__ void __launch_bounds__(kCta) rows_kernel(const Geom g, const RowsArgs a, uint32_t rows)
{
    constexpr uint32_t LANES = D / 8, HEADS = 32 / LANES;      // lanes of a head; heads a warp has at a time
    __shared__ unsigned long long pre[kCta], tmp[32];
    __shared__ uint4 ring[kStages * kSteps][kCta];
    __shared__ uint32_t flags;
    pdl_prologue();
    const uint32_t half = a.rotary / 2, w = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % LANES;
    // this lane's columns: f .. f + 3 and s .. s + 3; its pairs are 4 l .. 4 l + 3
    const bool turns = 8 * l < a.rotary;
    const uint32_t f = NEIGHBOURS || !turns ? 8 * l : 4 * l, s = NEIGHBOURS || !turns ? 8 * l + 4 : half + 4 * l;
    const uint32_t h0 = w / rows * HEADS + lane / LANES, h_step = kWarps / rows * HEADS;
    auto write = [&](uint8_t *p, const uint4 &v) {
        if (NEIGHBOURS) {
            *reinterpret_cast<uint4 *>(p + f * 2) = v;
        } else {
            *reinterpret_cast<uint2 *>(p + f * 2) = make_uint2(v.x, v.y);
            *reinterpret_cast<uint2 *>(p + s * 2) = make_uint2(v.z, v.w);
        }
    };
    Runs runs(a.cu, a.n, a.total, rows, (unsigned long long)g.max_pages * g.T, pre, tmp);
    uint32_t k, run;
    for (unsigned long long i = blockIdx.x;; i += gridDim.x) {
        // this warp's token: of a run of one entry, or of as many entries with one token each
        if (a.cu) {
            if (!runs.seek(i, &k, &run)) break;
        } else {
            if (i * rows >= a.n) break;
            if (i != blockIdx.x) __syncthreads();      // `flags` of the entries before have been read
            k = (uint32_t)i * rows + w % rows; run = 0;
        }
        const bool listed = k < a.n;
        const uint32_t r = listed ? a.reqs[k] : kInvalid, c0 = a.cu ? a.cu[k] : k, c1 = a.cu ? a.cu[k + 1] : k + 1;
        const bool rows_ok = listed && c1 >= c0 && c1 <= a.total;
        const uint32_t row = a.cu ? c0 + run * rows + w % rows : k;
        const bool mine = rows_ok && row < c1;
        const uint8_t *q = a.q + (unsigned long long)row * a.qs, *kk = a.k + (unsigned long long)row * a.ks, *v = a.v + (unsigned long long)row * a.vs;
        // the warp's stages: those of the query heads, then of the keys, then of the values
        const uint32_t q_stages = (a.q_heads + kSteps * h_step - 1) / (kSteps * h_step), kv_stages = (a.kv_heads + kSteps * h_step - 1) / (kSteps * h_step);
        uint32_t next = 0, place_in = 0;
        auto load = [&] {
            const bool is_q = next < q_stages, is_k = next < q_stages + kv_stages;
            const uint8_t *from = is_q ? q : is_k ? kk : v;
            const uint32_t heads = is_q ? a.q_heads : next < q_stages + 2 * kv_stages ? a.kv_heads : 0u;
            const uint32_t h = h0 + (next - (is_q ? 0u : is_k ? q_stages : q_stages + kv_stages)) * (kSteps * h_step);
#pragma unroll
            for (int e = 0; e < kSteps; ++e) {
                if (!mine || h + e * h_step >= heads) continue;
                const uint8_t *p = from + (h + e * h_step) * (D * 2);
                const uint32_t to = smem_u32(&ring[place_in * kSteps + e][threadIdx.x]);
                if (NEIGHBOURS) {
                    cp_async16(to, p + f * 2, true);
                } else {
                    cp_async8(to, p + f * 2);
                    cp_async8(to + 8, p + s * 2);
                }
            }
            cp_async_commit();
            next += 1;
            place_in = place_in + 1 == kStages ? 0 : place_in + 1;
        };
#pragma unroll
        for (int e = 0; e < kStages - 1; ++e) load();               // while the slot and the page are looked up
        const uint32_t held = held_tokens(g, r);
        const bool again = a.cu ? named_before(a.reqs, k, r) : (named_before_each(a.reqs, (uint32_t)i * rows, rows, a.n, &flags) >> (w % rows) & 1) != 0;
        if (again || held == 0 || !rows_ok || c1 - c0 > held) {
            if (listed && run == 0 && lane == 0 && w < (a.cu ? 1u : rows)) record_error(g.st, AVMP_DEV_BAD_REQUEST);
            cp_async_wait<0>();
            continue;
        }
        if (!mine) continue;
        const uint32_t place = held - (c1 - row), page = __ldcg(g.r_chain + ((unsigned long long)r * g.max_pages + place / g.T));
        uint8_t *to_k = unit_ptr(g, AVMP_POOL_KV, __ldcg(g.VT[0] + (page & 0x7FFFFFFFu))) + a.layer * g.kv_layer_bytes + place % g.T * g.row_bytes;
        uint8_t *to_v = to_k + g.T * g.row_bytes, *to_q = a.out + (unsigned long long)row * a.os;
        // sines and cosines: the lanes that have the same columns of different heads work out a share of them each
        float cs[4], sn[4];
        {
            constexpr uint32_t EACH = 4 / HEADS;
            float c[EACH], d[EACH];
#pragma unroll
            for (uint32_t j = 0; j < EACH; ++j) {
                c[j] = 1.f; d[j] = 0.f;
                if (turns) {
                    const double turn = (double)(a.pos ? a.pos[row] : place) * (double)a.freq[4 * l + lane / LANES * EACH + j] * 0.15915494309189533577;
                    sincospif((float)(2.0 * (turn - rint(turn))), &d[j], &c[j]);
                }
            }
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                cs[j] = __shfl_sync(0xFFFFFFFFu, c[j % EACH], l + j / EACH * LANES);
                sn[j] = __shfl_sync(0xFFFFFFFFu, d[j % EACH], l + j / EACH * LANES);
            }
        }
        uint32_t place_out = 0;
        auto heads_of = [&](uint8_t *to, uint32_t heads, uint32_t stages, const float *weight) {
            // A pair (p, o) becomes by * (p pc - o os, o oc + p ps).  Two numbers go through the multiply-add pipe at a time: two pairs' p or o
            // where they lie so (halves), else one pair.
            unsigned long long straight[4], cross[4];
            {
                float pc[4], os[4], oc[4], ps[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float wp = weight ? weight[NEIGHBOURS ? f + 2 * j : f + j] : 1.f, wo = weight ? weight[NEIGHBOURS ? f + 2 * j + 1 : s + j] : 1.f;
                    pc[j] = wp * cs[j]; os[j] = -wo * sn[j]; oc[j] = wo * cs[j]; ps[j] = wp * sn[j];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int x = 2 * (j % 2);
                    straight[j] = NEIGHBOURS ? pack2(pc[j], oc[j]) : j < 2 ? pack2(pc[x], pc[x + 1]) : pack2(oc[x], oc[x + 1]);
                    cross[j] = NEIGHBOURS ? pack2(os[j], ps[j]) : j < 2 ? pack2(os[x], os[x + 1]) : pack2(ps[x], ps[x + 1]);
                }
            }
            uint32_t h = h0;
            for (uint32_t x = 0; x < stages; ++x) {
                load();
                cp_async_wait<kStages - 1>();
#pragma unroll
                for (int e = 0; e < kSteps; ++e, h += h_step) {
                    const uint4 in4 = ring[place_out * kSteps + e][threadIdx.x];
                    const uint32_t in[4] = {in4.x, in4.y, in4.z, in4.w};
                    unsigned long long y[4], sum = 0;          // columns f, f + 1; f + 2, f + 3; s, s + 1; s + 2, s + 3
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 z = T::unpack(in[j]);
                        y[j] = pack2(z.x, z.y);
                        sum = j ? fma2(y[j], y[j], sum) : mul2(y[j], y[j]);
                    }
                    float by = 1.f;
                    if (weight) {
                        const float2 z = unpack2(sum);
                        float sq = z.x + z.y;
#pragma unroll
                        for (uint32_t o = LANES / 2; o; o >>= 1) sq += __shfl_xor_sync(0xFFFFFFFFu, sq, o);
                        by = rsqrtf(sq * (1.f / D) + a.eps);
                    }
                    uint32_t out[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 z = unpack2(y[j]);
                        const unsigned long long other = NEIGHBOURS ? pack2(z.y, z.x) : y[(j + 2) % 4];
                        unsigned long long v = mul2(y[j], straight[j]);
                        if (turns) v = fma2(other, cross[j], v);       // (columns that are not rotated have no partner to take an infinity from)
                        const float2 r = unpack2(mul2(v, pack2(by, by)));
                        out[j] = T::pack(r.x, r.y);
                    }
                    if (h < heads) write(to + h * (D * 2), make_uint4(out[0], out[1], out[2], out[3]));
                }
                place_out = place_out + 1 == kStages ? 0 : place_out + 1;
            }
        };
        heads_of(to_q, a.q_heads, q_stages, a.wq);
        heads_of(to_k, a.kv_heads, kv_stages, a.wk);
        uint32_t h = h0;
        for (uint32_t x = 0; x < kv_stages; ++x) {
            load();
            cp_async_wait<kStages - 1>();
#pragma unroll
            for (int e = 0; e < kSteps; ++e, h += h_step)
                if (h < a.kv_heads) write(to_v + h * (D * 2), ring[place_out * kSteps + e][threadIdx.x]);
            place_out = place_out + 1 == kStages ? 0 : place_out + 1;
        }
        cp_async_wait<0>();
    }
}

template <class T, int D>
cudaError_t launch(const Geom &g, const RowsArgs &a, const Launch &l)
{
    // A token for each warp; where that leaves SMs idle, one or two for all four.
    uint32_t rows = a.cu ? kWarps : 1;
    while (a.cu && rows > 1 && a.total / rows < 4u * l.n_sms) rows >>= 1;
    while (!a.cu && rows < kWarps && a.n / rows > 5u * l.n_sms) rows <<= 1;      // five CTAs fit on an SM: one wave
    const unsigned long long runs = a.cu ? (unsigned long long)a.total / rows + a.n : (a.n + rows - 1) / rows;
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
