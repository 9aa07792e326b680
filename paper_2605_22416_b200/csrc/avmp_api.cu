// Host side of the C ABI: argument checks, the Section 3.1 layout arithmetic, workspace
// carving, launch sequencing.  No device memory is allocated here; the context is a small
// host struct over the caller's arena and workspace.
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <new>
#include <vector>

#include "avmp_dev.cuh"

using namespace avmp;


namespace {

constexpr size_t kAlign = 256;
inline size_t up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct Carve {
    size_t off = 0;
    size_t take(size_t bytes) { size_t o = off; off += up(bytes ? bytes : 1); return o; }
};

// Offsets of every table inside the workspace, in one place so that size and carving agree.
struct WsLayout {
    size_t state, S[2], W[2], VT[2], OW[2], r_state, r_len, r_npages, r_chain, r_ssm;
    size_t reloc_src, reloc_dst, g_cu_items, g_cu_rows, stage_ops, stage_status, total;
};

WsLayout ws_layout(const avmp_layout &lay, const avmp_model_spec &spec, const avmp_options &opt)
{
    WsLayout w;
    Carve c;
    w.state = c.take(sizeof(DevState));
    for (int p = 0; p < 2; ++p) {
        const size_t v = (size_t)lay.vid_space[p] * 4;
        w.S[p] = c.take(v); w.W[p] = c.take(v); w.VT[p] = c.take(v); w.OW[p] = c.take(v);
    }
    const size_t R = opt.max_requests;
    w.r_state = c.take(R * 4); w.r_len = c.take(R * 4); w.r_npages = c.take(R * 4);
    w.r_chain = c.take(R * (size_t)opt.max_pages_per_request * 4);
    w.r_ssm = c.take(R * (size_t)spec.n_ssm_layers * 4);
    const size_t maxv = (size_t)(lay.vid_space[0] > lay.vid_space[1] ? lay.vid_space[0] : lay.vid_space[1]);
    w.reloc_src = c.take(maxv * 4); w.reloc_dst = c.take(maxv * 4);
    w.g_cu_items = c.take((R + 1) * 4); w.g_cu_rows = c.take((R + 1) * 4);
    w.stage_ops = c.take((size_t)kHostStepMaxOps * sizeof(avmp_op));
    w.stage_status = c.take((size_t)kHostStepMaxOps * 4);
    w.total = c.off;
    return w;
}

bool options_ok(const avmp_options &o)
{
    return o.threshold_low_ppm < o.threshold_high_ppm && o.threshold_high_ppm <= 1000000u &&
           o.min_rebalance_interval_ops >= 1 && o.max_requests >= 1 && o.max_pages_per_request >= 1 &&
           (uint64_t)o.max_requests * o.max_pages_per_request < (1ull << 32);
}

inline cudaStream_t S(void *s) { return reinterpret_cast<cudaStream_t>(s); }
inline Launch L(const avmp_ctx *c, void *s) { return Launch{S(s), c->n_sms, c->device}; }
inline int cu(cudaError_t e) { return e == cudaSuccess ? AVMP_OK : AVMP_ECUDA; }

void fill_stats(const avmp_ctx *c, const DevState &d, avmp_stats *o)
{
    o->op_counter = d.op_counter; o->last_rebalance_op = d.last_rebalance_op; o->n_oom = d.n_oom;
    o->n_capacity_error = d.n_capacity_error; o->n_rebalance = d.n_rebalance;
    o->migrated_bytes = d.migrated_bytes; o->wasted_bytes = d.wasted_bytes;
    o->relocated_blocks = d.relocated_blocks; o->relocated_bytes = d.relocated_bytes;
    o->gap_bytes = d.gap_bytes;
    for (int p = 0; p < 2; ++p) {
        o->cap[p] = d.cap[p]; o->free_units[p] = d.n_free[p];
        o->unit_bytes[p] = c->lay.unit_bytes[p]; o->vid_space[p] = c->lay.vid_space[p];
    }
    o->fsm_state = d.fsm; o->n_invalid = d.n_invalid;
    o->pool_bytes_aligned = c->lay.pool_bytes_aligned;
    o->error_code = d.error_code; o->error_count = d.error_count;
    const uint64_t last = (d.reloc_t1 > d.reloc_t0 && d.reloc_t0 != kNone64) ? d.reloc_t1 - d.reloc_t0 : 0;
    o->relocation_ns_last = last;
    o->relocation_ns_total = d.reloc_ns_total + (d.reloc_pending ? last : 0);
    const double ns_per_cycle = c->sm_khz > 0 ? 1e6 / (double)c->sm_khz : 0.0;
    o->step_ns_total = (uint64_t)(d.cyc_total * ns_per_cycle);
    o->step_ns_oom_retry = (uint64_t)(d.cyc_oom * ns_per_cycle);
    o->step_ns_migration_plan = (uint64_t)(d.cyc_mig * ns_per_cycle);
}

// The compute calls check that the context's device is the current one (the stream and the launch belong to it).
inline bool device_ok(const avmp_ctx *c)
{
    int dev = -1;
    return cudaGetDevice(&dev) == cudaSuccess && dev == c->device;
}

bool attn_desc_ok(const avmp_ctx *c, const avmp_attn_desc *d)
{
    if (!d || d->type > AVMP_TYPE_F16 || d->rsvd || !std::isfinite(d->scale)) return false;
    const avmp_model_spec &m = c->spec;
    if (m.n_attn_layers == 0 || m.kv_elem_bytes != 2 || (m.head_dim != 64 && m.head_dim != 128) || m.page_tokens % 8) return false;
    if (m.kv_heads == 0 || d->q_heads == 0 || d->q_heads > 65535u || d->q_heads % m.kv_heads || d->q_heads / m.kv_heads > 64) return false;
    const uint64_t row = (uint64_t)d->q_heads * m.head_dim * 2;
    auto stride_ok = [&](uint64_t s) { return s == 0 || (s >= row && s % 16 == 0 && s < (1ull << 40)); };
    return stride_ok(d->q_stride_bytes) && stride_ok(d->out_stride_bytes);
}

AttnArgs attn_args(const avmp_ctx *c, const avmp_attn_desc *d, uint32_t layer, const uint32_t *reqs, uint32_t n, const void *q,
                   void *out, float *lse, void *ws)
{
    AttnArgs a = {};
    a.layer = layer; a.n = n; a.q_heads = d->q_heads; a.kv_heads = c->spec.kv_heads; a.head_dim = c->spec.head_dim;
    a.prefix = kInvalid; a.f16 = d->type == AVMP_TYPE_F16; a.scale = d->scale;
    a.reqs = reqs; a.q = static_cast<const uint8_t *>(q); a.out = static_cast<uint8_t *>(out); a.lse = lse;
    const uint64_t row = (uint64_t)d->q_heads * c->spec.head_dim * 2;
    a.qs = d->q_stride_bytes ? d->q_stride_bytes : row; a.os = d->out_stride_bytes ? d->out_stride_bytes : row;
    a.ws = static_cast<uint8_t *>(ws);
    a.wait = c->wait;
    return a;
}

inline bool ssm_desc_ok(const avmp_ctx *c, const avmp_ssm_desc *d)
{
    if (!d || d->type > AVMP_TYPE_F16 || d->rsvd || c->spec.ssm_elem_bytes != 4 || c->spec.n_ssm_layers == 0) return false;
    if (d->dk != 16 && d->dk != 32 && d->dk != 64 && d->dk != 128) return false;
    if (d->dv == 0 || d->dv % 32 || d->heads == 0 || d->groups == 0 || d->heads % d->groups) return false;
    if ((unsigned __int128)d->heads * d->dv * d->dk != c->spec.ssm_state_elems) return false;
    if (c->spec.ssm_state_elems > 1u << 31) return false;      // the kernels count a block's elements, and a round beyond the last, in 32 bits
    const uint64_t qk = (uint64_t)d->groups * d->dk * 2, v = (uint64_t)d->heads * d->dv * 2;
    auto stride_ok = [](uint64_t s, uint64_t row, uint64_t unit) { return s == 0 || (s >= row && s % unit == 0 && s < (1ull << 40)); };
    return stride_ok(d->q_stride_bytes, qk, 16) && stride_ok(d->k_stride_bytes, qk, 16) && stride_ok(d->v_stride_bytes, v, 16) &&
           stride_ok(d->out_stride_bytes, v, 16) && stride_ok(d->decay_stride_bytes, (uint64_t)d->heads * 4, 4);
}

SsmArgs ssm_args(const avmp_ssm_desc *d, uint32_t layer, const uint32_t *reqs, uint32_t n, const void *q, const void *k,
                 const void *v, const float *decay, void *out)
{
    SsmArgs a = {};
    a.layer = layer; a.n = n; a.heads = d->heads; a.groups = d->groups; a.dk = d->dk; a.dv = d->dv;
    a.f16 = d->type == AVMP_TYPE_F16;
    a.reqs = reqs;
    a.q = static_cast<const uint8_t *>(q); a.k = static_cast<const uint8_t *>(k); a.v = static_cast<const uint8_t *>(v);
    a.g = reinterpret_cast<const uint8_t *>(decay); a.out = static_cast<uint8_t *>(out);
    const uint64_t qk = (uint64_t)d->groups * d->dk * 2, vr = (uint64_t)d->heads * d->dv * 2;
    a.qs = d->q_stride_bytes ? d->q_stride_bytes : qk; a.ks = d->k_stride_bytes ? d->k_stride_bytes : qk;
    a.vs = d->v_stride_bytes ? d->v_stride_bytes : vr; a.os = d->out_stride_bytes ? d->out_stride_bytes : vr;
    a.gs = d->decay_stride_bytes ? d->decay_stride_bytes : (uint64_t)d->heads * 4;
    return a;
}

bool ssm_rows_ok(const void *q, const void *k, const void *v, const float *decay, const void *out)
{
    return q && k && v && decay && out && !(((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 15) && !((uintptr_t)decay & 3);
}

inline bool stride_ok(uint64_t s, uint64_t row) { return s == 0 || (s >= row && s % 16 == 0 && s < (1ull << 40)); }
inline bool off16(const void *p) { return ((uintptr_t)p & 15) != 0; }
inline bool off4(const void *p) { return ((uintptr_t)p & 3) != 0; }

bool conv_desc_ok(const avmp_ctx *c, const avmp_conv_desc *d)
{
    const avmp_model_spec &m = c->spec;
    if (!d || d->type > AVMP_TYPE_F16 || d->silu > 1 || m.ssm_elem_bytes != 4 || m.n_ssm_layers == 0 || m.ssm_state_elems % 4) return false;
    if (d->width < 2 || d->width > 4 || d->channels == 0 || d->channels % 8 || d->channels > 1u << 24) return false;
    if ((uint64_t)d->channels * (d->width - 1) != m.ssm_conv_elems) return false;
    return stride_ok(d->x_stride_bytes, (uint64_t)d->channels * 2) && stride_ok(d->out_stride_bytes, (uint64_t)d->channels * 2);
}

int conv_call(avmp_ctx *c, uint32_t layer, const avmp_conv_desc *desc, const uint32_t *d_reqs, uint32_t n, const uint32_t *d_cu,
              uint32_t total, const uint32_t *d_resume, const void *d_x, const float *d_weight, const float *d_bias, void *d_out, void *stream)
{
    if (!d_weight || off16(d_weight) || off16(d_bias)) return AVMP_EINVAL;
    if (total && (!d_x || !d_out || off16(d_x) || off16(d_out))) return AVMP_EINVAL;
    ConvArgs a = {};
    a.layer = layer; a.n = n; a.channels = desc->channels; a.width = desc->width; a.total = total; a.state_elems = c->spec.ssm_state_elems;
    a.f16 = desc->type == AVMP_TYPE_F16; a.act = desc->silu != 0;
    a.reqs = d_reqs; a.cu = d_cu; a.resume = d_resume;
    a.x = static_cast<const uint8_t *>(d_x); a.weight = d_weight; a.bias = d_bias; a.out = static_cast<uint8_t *>(d_out);
    const uint64_t row = (uint64_t)desc->channels * 2;
    a.xs = desc->x_stride_bytes ? desc->x_stride_bytes : row; a.os = desc->out_stride_bytes ? desc->out_stride_bytes : row;
    c->launches += 1;
    return cu(launch_conv(c->g, a, L(c, stream)));
}

bool scan_desc_ok(const avmp_ctx *c, const avmp_scan_desc *d)
{
    const avmp_model_spec &m = c->spec;
    if (!d || d->type > AVMP_TYPE_F16 || d->softplus > 1 || d->rsvd || m.ssm_elem_bytes != 4 || m.n_ssm_layers == 0) return false;
    if (d->states != 8 && d->states != 16 && d->states != 32 && d->states != 64) return false;
    if (d->channels == 0 || d->channels > 1u << 24 || d->groups == 0 || d->channels % d->groups || d->channels / d->groups % 8) return false;
    if ((uint64_t)d->channels * d->states != m.ssm_state_elems) return false;
    const uint64_t row = (uint64_t)d->channels * 2, bc = (uint64_t)d->groups * d->states * 2;
    return stride_ok(d->u_stride_bytes, row) && stride_ok(d->delta_stride_bytes, row) && stride_ok(d->z_stride_bytes, row) &&
           stride_ok(d->out_stride_bytes, row) && stride_ok(d->b_stride_bytes, bc) && stride_ok(d->c_stride_bytes, bc);
}

// (rows: whether the call has any)
bool scan_rows_ok(bool rows, const void *u, const void *delta, const void *b, const void *c, const void *z, const float *a, const float *d,
                  const float *bias, const void *out)
{
    if (!a || off16(a) || off4(d) || off4(bias) || off16(z)) return false;
    return !rows || (u && delta && b && c && out && !(off16(u) || off16(delta) || off16(b) || off16(c) || off16(out)));
}

ScanArgs scan_args(const avmp_scan_desc *d, uint32_t layer, const uint32_t *reqs, uint32_t n, const void *u, const void *delta, const void *b,
                   const void *c, const void *z, const float *da, const float *dd, const float *bias, void *out)
{
    ScanArgs a = {};
    a.layer = layer; a.n = n; a.channels = d->channels; a.groups = d->groups; a.states = d->states; a.shares = 1;
    a.f16 = d->type == AVMP_TYPE_F16; a.softplus = d->softplus != 0;
    a.reqs = reqs;
    a.u = static_cast<const uint8_t *>(u); a.d = static_cast<const uint8_t *>(delta); a.b = static_cast<const uint8_t *>(b);
    a.c = static_cast<const uint8_t *>(c); a.z = static_cast<const uint8_t *>(z);
    a.a = da; a.skip = dd; a.bias = bias; a.out = static_cast<uint8_t *>(out);
    const uint64_t row = (uint64_t)d->channels * 2, bc = (uint64_t)d->groups * d->states * 2;
    a.us = d->u_stride_bytes ? d->u_stride_bytes : row; a.ds = d->delta_stride_bytes ? d->delta_stride_bytes : row;
    a.zs = d->z_stride_bytes ? d->z_stride_bytes : row; a.os = d->out_stride_bytes ? d->out_stride_bytes : row;
    a.bs = d->b_stride_bytes ? d->b_stride_bytes : bc; a.cs = d->c_stride_bytes ? d->c_stride_bytes : bc;
    return a;
}

// Scratch of one scan over prompts: a state and a sum of steps for each run of each (request, channel).
size_t scan_ws_bytes(const avmp_ctx *c, const avmp_scan_desc *d, uint32_t n, uint32_t total)
{
    const uint32_t shares = scan_shares(n, d->channels, d->groups, d->states, total, c->n_sms);
    return shares < 2 ? 0 : (size_t)n * shares * d->channels * (d->states + 1) * 4;
}

bool rows_desc_ok(const avmp_ctx *c, const avmp_rows_desc *d)
{
    const avmp_model_spec &m = c->spec;
    if (!d || d->type > AVMP_TYPE_F16 || d->pairing > AVMP_ROTATE_NEIGHBOURS || d->rsvd || !(d->eps >= 0.f) || !std::isfinite(d->eps)) return false;
    if (m.n_attn_layers == 0 || m.kv_elem_bytes != 2 || (m.head_dim != 64 && m.head_dim != 128) || m.kv_heads == 0 || m.kv_heads > 65535u) return false;
    if (d->q_heads == 0 || d->q_heads > 65535u || d->rotary_dim > m.head_dim || d->rotary_dim % 8) return false;
    const uint64_t q = (uint64_t)d->q_heads * m.head_dim * 2, kv = (uint64_t)m.kv_heads * m.head_dim * 2;
    return stride_ok(d->q_stride_bytes, q) && stride_ok(d->out_stride_bytes, q) && stride_ok(d->k_stride_bytes, kv) && stride_ok(d->v_stride_bytes, kv);
}

int rows_call(avmp_ctx *c, uint32_t layer, const avmp_rows_desc *desc, const uint32_t *d_reqs, uint32_t n, const uint32_t *d_cu,
              uint32_t total, const uint32_t *d_pos, const void *d_q, const void *d_k, const void *d_v, const float *d_q_weight,
              const float *d_k_weight, const float *d_freq, void *d_out, void *stream)
{
    if (off4(d_pos) || off4(d_q_weight) || off4(d_k_weight) || off4(d_freq) || (desc->rotary_dim && !d_freq)) return AVMP_EINVAL;
    if (total && (!d_q || !d_k || !d_v || !d_out || off16(d_q) || off16(d_k) || off16(d_v) || off16(d_out))) return AVMP_EINVAL;
    const avmp_model_spec &m = c->spec;
    RowsArgs a = {};
    a.layer = layer; a.n = n; a.q_heads = desc->q_heads; a.kv_heads = m.kv_heads; a.head_dim = m.head_dim; a.rotary = desc->rotary_dim; a.total = total;
    a.f16 = desc->type == AVMP_TYPE_F16; a.neighbours = desc->pairing == AVMP_ROTATE_NEIGHBOURS; a.eps = desc->eps;
    a.reqs = d_reqs; a.cu = d_cu; a.pos = d_pos;
    a.q = static_cast<const uint8_t *>(d_q); a.k = static_cast<const uint8_t *>(d_k); a.v = static_cast<const uint8_t *>(d_v);
    a.wq = d_q_weight; a.wk = d_k_weight; a.freq = d_freq; a.out = static_cast<uint8_t *>(d_out);
    const uint64_t q = (uint64_t)desc->q_heads * m.head_dim * 2, kv = (uint64_t)m.kv_heads * m.head_dim * 2;
    a.qs = desc->q_stride_bytes ? desc->q_stride_bytes : q; a.os = desc->out_stride_bytes ? desc->out_stride_bytes : q;
    a.ks = desc->k_stride_bytes ? desc->k_stride_bytes : kv; a.vs = desc->v_stride_bytes ? desc->v_stride_bytes : kv;
    c->launches += 1;
    return cu(launch_attn_rows(c->g, a, L(c, stream)));
}

// Scratch of one call of the recurrence over prompts: a state and a decay for each run of each (request, head, columns).
size_t ssm_ws_bytes(const avmp_ctx *c, const avmp_ssm_desc *d, uint32_t n, uint32_t total)
{
    const uint32_t shares = ssm_shares(n, d->heads, d->dv, total, c->n_sms);
    return shares < 2 ? 0 : (size_t)n * shares * ((size_t)d->heads * d->dv * d->dk + (size_t)d->heads * (d->dv / 32)) * 4;
}

// Attention calls with and without (window 0) a window.
int attn_prompt_call(avmp_ctx *c, uint32_t layer, const avmp_attn_desc *desc, uint32_t window, uint32_t sinks, const uint32_t *d_reqs, uint32_t n,
                     const uint32_t *d_cu_q, uint32_t total_q, const void *d_q, void *d_out, float *d_lse, void *d_workspace,
                     size_t workspace_bytes, void *stream)
{
    if (!c || layer >= c->spec.n_attn_layers || n > c->opt.max_requests || !attn_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_cu_q || (((uintptr_t)d_reqs | (uintptr_t)d_cu_q | (uintptr_t)d_lse) & 3)) return AVMP_EINVAL;
    if (total_q && (!d_q || !d_out || (((uintptr_t)d_q | (uintptr_t)d_out) & 15))) return AVMP_EINVAL;
    if ((uint64_t)total_q * desc->q_heads >= (1ull << 31)) return AVMP_EINVAL;
    if (!d_workspace || ((uintptr_t)d_workspace & 15)) return AVMP_EINVAL;
    if (workspace_bytes < avmp_attn_workspace_bytes(c, desc, n)) return AVMP_ENOSPC;
    AttnArgs a = attn_args(c, desc, layer, d_reqs, n, d_q, d_out, d_lse, d_workspace);
    a.window = window; a.sinks = sinks; a.cu = d_cu_q; a.total_q = total_q;
    uint32_t launched = 0;
    const cudaError_t e = launch_attn_prompt(c->g, a, L(c, stream), &launched);
    c->launches += launched;
    return cu(e);
}

int attn_decode_call(avmp_ctx *c, uint32_t layer, const avmp_attn_desc *desc, uint32_t window, uint32_t sinks, const uint32_t *d_reqs, uint32_t n,
                     uint32_t prefix_req, const void *d_q, void *d_out, float *d_lse, void *d_workspace, size_t workspace_bytes,
                     void *stream)
{
    if (!c || layer >= c->spec.n_attn_layers || n > c->opt.max_requests || !attn_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || (((uintptr_t)d_reqs | (uintptr_t)d_lse) & 3)) return AVMP_EINVAL;
    if (!d_q || !d_out || (((uintptr_t)d_q | (uintptr_t)d_out) & 15)) return AVMP_EINVAL;
    if ((uint64_t)n * desc->q_heads >= (1ull << 31)) return AVMP_EINVAL;
    if (!d_workspace || ((uintptr_t)d_workspace & 15)) return AVMP_EINVAL;
    if (workspace_bytes < avmp_attn_workspace_bytes(c, desc, n)) return AVMP_ENOSPC;
    AttnArgs a = attn_args(c, desc, layer, d_reqs, n, d_q, d_out, d_lse, d_workspace);
    a.window = window; a.sinks = sinks; a.prefix = prefix_req;
    uint32_t launched = 0;
    const cudaError_t e = launch_attn_decode(c->g, a, L(c, stream), &launched);
    c->launches += launched;
    return cu(e);
}

// A snapshot is accepted only if the kernels could have produced it: they index the tables
// without bounds checks, so a table that does not hang together must never reach the device.
bool tables_consistent(const avmp_ctx *c, const avmp_tables *t)
{
    const Geom &g = c->g;
    const avmp_stats &st = t->stats;
    if (st.fsm_state > AVMP_FSM_REBALANCING) return false;
    if (st.last_rebalance_op != kNone64 && st.last_rebalance_op > st.op_counter) return false;
    unsigned __int128 bytes = st.gap_bytes;
    for (int p = 0; p < 2; ++p) {
        if (st.cap[p] > g.V[p]) return false;
        bytes += (unsigned __int128)st.cap[p] * g.U[p];
    }
    if (bytes != g.P_al) return false;                         // pool bytes are conserved
    uint64_t live[2] = {0, 0};
    std::vector<uint8_t> mark;
    for (int p = 0; p < 2; ++p) {
        const uint32_t V = g.V[p], cap = (uint32_t)st.cap[p], nf = t->n_slot_stack[p], nv = t->n_vid_stack[p];
        const uint32_t *S = t->slot_stack[p], *W = t->vid_stack[p], *VT = t->vt[p], *OW = t->ow[p];
        if (nf > cap || nv > V) return false;
        mark.assign(V, 0);
        for (uint32_t i = 0; i < nf; ++i) {                    // free slots: inside the store, distinct
            if (S[i] >= cap || mark[S[i]]) return false;
            mark[S[i]] = 1;
        }
        for (uint32_t s = 0; s < V; ++s) {                     // owned slots: not free, mapped back by their id
            const uint32_t v = OW[s];
            if (v == kInvalid) continue;
            if (s >= cap || mark[s] || v >= V || VT[v] != s) return false;
            live[p] += 1;
        }
        if (live[p] != (uint64_t)cap - nf) return false;
        mark.assign(V, 0);
        for (uint32_t i = 0; i < nv; ++i) {                    // free ids: distinct, unmapped
            if (W[i] >= V || mark[W[i]] || VT[W[i]] != kInvalid) return false;
            mark[W[i]] = 1;
        }
        uint64_t mapped = 0;
        for (uint32_t v = 0; v < V; ++v) {
            if (VT[v] == kInvalid) continue;
            if (VT[v] >= cap || OW[VT[v]] != v) return false;
            mapped += 1;
        }
        if (mapped != live[p] || (uint64_t)nv != (uint64_t)V - live[p]) return false;
    }
    // every live unit belongs to exactly one request
    std::vector<uint8_t> ref[2];
    ref[0].assign(g.V[0], 0); ref[1].assign(g.V[1], 0);
    uint64_t held[2] = {0, 0};
    for (uint32_t r = 0; r < g.R; ++r) {
        const uint32_t state = t->req_state[r], np = t->req_npages[r], len = t->req_len[r];
        if (state == AVMP_REQ_EMPTY) { if (np || len) return false; continue; }
        if (state != AVMP_REQ_LIVE && state != AVMP_REQ_KV_ONLY) return false;
        // a held request has at least one token (ADMIT and EXTEND reject zero tokens)
        if (len == 0 || np > g.max_pages || ((uint64_t)len + g.T - 1) / g.T != np) return false;
        for (uint32_t j = 0; j < np; ++j) {
            const uint32_t h = t->req_chain[(size_t)r * g.max_pages + j], v = h & 0x7FFFFFFFu;
            if ((h >> 31) != AVMP_POOL_KV || v >= g.V[0] || t->vt[0][v] == kInvalid || ref[0][v]) return false;
            ref[0][v] = 1; held[0] += 1;
        }
        if (state == AVMP_REQ_LIVE)
            for (uint32_t l = 0; l < g.ns; ++l) {
                const uint32_t h = t->req_ssm[(size_t)r * g.ns + l], v = h & 0x7FFFFFFFu;
                if ((h >> 31) != AVMP_POOL_SSM || v >= g.V[1] || t->vt[1][v] == kInvalid || ref[1][v]) return false;
                ref[1][v] = 1; held[1] += 1;
            }
    }
    return held[0] == live[0] && held[1] == live[1];
}

}  // namespace

extern "C" {

void avmp_default_options(avmp_options *o)
{
    if (!o) return;
    o->threshold_low_ppm = 50000; o->threshold_high_ppm = 300000;
    o->min_rebalance_interval_ops = 1000; o->migration_enabled = 1;
    o->max_requests = 1024; o->max_pages_per_request = 4096; o->reclaim_gap = 0;
}

int avmp_derive_layout(const avmp_model_spec *m, uint64_t pool_bytes, double split, avmp_layout *out)
{
    if (!m || !out) return AVMP_EINVAL;
    if (!(split >= 0.0 && split <= 1.0) || m->page_tokens == 0) return AVMP_EINVAL;
    avmp_layout l;
    l.kv_row_bytes = (uint64_t)m->kv_heads * m->head_dim * m->kv_elem_bytes;
    l.kv_layer_bytes = 2ull * m->page_tokens * l.kv_row_bytes;
    l.ssm_state_bytes = (uint64_t)m->ssm_state_elems * m->ssm_elem_bytes;
    l.ssm_conv_bytes = (uint64_t)m->ssm_conv_elems * m->ssm_elem_bytes;
    l.unit_bytes[0] = ((uint64_t)m->n_attn_layers * l.kv_layer_bytes + 15u) & ~15ull;
    l.unit_bytes[1] = (l.ssm_state_bytes + l.ssm_conv_bytes + 15u) & ~15ull;
    if (l.unit_bytes[0] == 0 || l.unit_bytes[1] == 0) return AVMP_EINVAL;
    l.pool_bytes_aligned = pool_bytes & ~127ull;
    const uint64_t ppm = (uint64_t)llround(split * 1e6);
    const uint64_t ssm_bytes = (uint64_t)(((unsigned __int128)l.pool_bytes_aligned * ppm) / 1000000u) & ~127ull;
    l.cap0[0] = (l.pool_bytes_aligned - ssm_bytes) / l.unit_bytes[0];
    l.cap0[1] = ssm_bytes / l.unit_bytes[1];
    l.gap0 = l.pool_bytes_aligned - l.cap0[0] * l.unit_bytes[0] - l.cap0[1] * l.unit_bytes[1];
    for (int p = 0; p < 2; ++p) {
        l.vid_space[p] = l.pool_bytes_aligned / l.unit_bytes[p];
        if (l.vid_space[p] >= 0x7FFFFFFFull) return AVMP_EINVAL;
    }
    if (l.cap0[0] == 0 && l.cap0[1] == 0) return AVMP_EINVAL;
    *out = l;
    return AVMP_OK;
}

size_t avmp_workspace_bytes(const avmp_model_spec *spec, uint64_t pool_bytes, const avmp_options *opt)
{
    avmp_options o;
    if (opt) o = *opt; else avmp_default_options(&o);
    avmp_layout lay;
    if (!spec || !options_ok(o) || avmp_derive_layout(spec, pool_bytes, 0.5, &lay) != AVMP_OK) return 0;
    return ws_layout(lay, *spec, o).total;
}

int avmp_create(avmp_ctx **out, const avmp_model_spec *spec, void *d_arena, uint64_t pool_bytes,
                double initial_split, uint32_t migration_batch_size, const avmp_options *opt,
                void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!out || !spec || !d_arena || !d_workspace) return AVMP_EINVAL;
    if (((uintptr_t)d_arena | (uintptr_t)d_workspace) & (kAlign - 1)) return AVMP_EINVAL;
    avmp_options o;
    if (opt) o = *opt; else avmp_default_options(&o);
    if (!options_ok(o)) return AVMP_EINVAL;                       // Section 4.6: low >= high is invalid
    avmp_layout lay;
    if (avmp_derive_layout(spec, pool_bytes, initial_split, &lay) != AVMP_OK) return AVMP_EINVAL;
    const WsLayout w = ws_layout(lay, *spec, o);
    if (workspace_bytes < w.total) return AVMP_ENOSPC;

    avmp_ctx *c = new (std::nothrow) avmp_ctx();
    if (!c) return AVMP_EINVAL;
    c->spec = *spec; c->opt = o; c->lay = lay; c->B = migration_batch_size; c->launches = 0;
    (void)avmp_set_wait_limit(c, kWaitLimitNs);
    c->d_workspace = d_workspace; c->workspace_bytes = workspace_bytes;
    int &dev = c->device;
    dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&c->n_sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&c->sm_khz, cudaDevAttrClockRate, dev) != cudaSuccess) {
        delete c;
        return AVMP_ECUDA;
    }
    uint8_t *base = static_cast<uint8_t *>(d_workspace);
    Geom &g = c->g;
    g.P_al = lay.pool_bytes_aligned; g.U[0] = lay.unit_bytes[0]; g.U[1] = lay.unit_bytes[1];
    g.kv_layer_bytes = lay.kv_layer_bytes; g.row_bytes = lay.kv_row_bytes;
    g.state_bytes = lay.ssm_state_bytes; g.conv_bytes = lay.ssm_conv_bytes;
    g.min_interval = o.min_rebalance_interval_ops;
    g.V[0] = (uint32_t)lay.vid_space[0]; g.V[1] = (uint32_t)lay.vid_space[1];
    g.T = spec->page_tokens; g.na = spec->n_attn_layers; g.ns = spec->n_ssm_layers;
    g.R = o.max_requests; g.max_pages = o.max_pages_per_request; g.B = migration_batch_size;
    g.th_low = o.threshold_low_ppm; g.th_high = o.threshold_high_ppm; g.migration_enabled = o.migration_enabled;
    g.reclaim_gap = o.reclaim_gap ? 1u : 0u;
    g.arena = static_cast<uint8_t *>(d_arena);
    g.st = reinterpret_cast<DevState *>(base + w.state);
    for (int p = 0; p < 2; ++p) {
        g.S[p] = reinterpret_cast<uint32_t *>(base + w.S[p]); g.W[p] = reinterpret_cast<uint32_t *>(base + w.W[p]);
        g.VT[p] = reinterpret_cast<uint32_t *>(base + w.VT[p]); g.OW[p] = reinterpret_cast<uint32_t *>(base + w.OW[p]);
    }
    g.r_state = reinterpret_cast<uint32_t *>(base + w.r_state); g.r_len = reinterpret_cast<uint32_t *>(base + w.r_len);
    g.r_npages = reinterpret_cast<uint32_t *>(base + w.r_npages); g.r_chain = reinterpret_cast<uint32_t *>(base + w.r_chain);
    g.r_ssm = reinterpret_cast<uint32_t *>(base + w.r_ssm);
    g.reloc_src = reinterpret_cast<uint32_t *>(base + w.reloc_src); g.reloc_dst = reinterpret_cast<uint32_t *>(base + w.reloc_dst);
    g.g_cu_items = reinterpret_cast<uint32_t *>(base + w.g_cu_items); g.g_cu_rows = reinterpret_cast<uint32_t *>(base + w.g_cu_rows);
    c->d_stage_ops = reinterpret_cast<avmp_op *>(base + w.stage_ops);
    c->d_stage_status = reinterpret_cast<uint32_t *>(base + w.stage_status);

    DevState init;
    memset(&init, 0, sizeof(init));
    init.last_rebalance_op = kNone64;
    init.gap_bytes = lay.gap0;
    for (int p = 0; p < 2; ++p) {
        init.cap[p] = init.n_free[p] = (uint32_t)lay.cap0[p];
        init.n_vfree[p] = (uint32_t)lay.vid_space[p];
    }
    init.fsm = AVMP_FSM_BALANCED;
    // The row and piece prefix sums of a KV gather are 32-bit, like cu_seqlens: no request list of
    // up to max_requests entries (repeats allowed) may total 2^32 rows or copy pieces.
    {
        const uint64_t subs = kv_pieces_per_page(lay, spec->page_tokens);
        const uint64_t per_req = (uint64_t)o.max_pages_per_request * (spec->page_tokens > subs ? spec->page_tokens : subs);
        if ((unsigned __int128)o.max_requests * per_req >= ((unsigned __int128)1 << 32)) { delete c; return AVMP_EINVAL; }
    }
    if (launch_init(g, init, S(stream)) != cudaSuccess) { delete c; return AVMP_ECUDA; }
    // Bring avmp_gather_kv_static's in-library scratch onto this device now, while the caller still
    // has memory to spare (a failure here only shows up if that entry point is ever called).
    (void)static_gather_setup(dev);
    (void)cudaGetLastError();
    c->launches += 1;
    *out = c;
    return AVMP_OK;
}

int avmp_destroy(avmp_ctx *c)
{
    delete c;
    return AVMP_OK;
}

// A handle list to translate against the tables the step leaves (may be empty).
struct TranslateArgs {
    const uint32_t *h = nullptr;
    uint32_t n = 0;
    uint32_t *pool = nullptr;
    unsigned long long *off = nullptr, *aoff = nullptr;
};

static int step_rounds(avmp_ctx *c, const avmp_op *d_ops, uint32_t n_ops, const uint32_t *d_n_ops,
                       uint32_t *d_status, void *stream, const TranslateArgs &tr = TranslateArgs())
{
    // Section 3.2 throttle: migrations are >= min_interval logical ops apart, so a batch of n ops
    // holds at most (n - 1) / min_interval + 1 of them; one launch performs at most one.
    uint32_t rounds = 1;
    if (c->opt.migration_enabled)
        rounds = (uint32_t)((n_ops - 1) / c->opt.min_rebalance_interval_ops) + 1;
    // The copy grid is narrow (one 64-thread CTA per SM): a short handle list rides on it for free, a long one
    // (tens of thousands of handles; measured cross-over near 50 000) is faster in the wide translate kernel.
    const bool ride = c->opt.migration_enabled && tr.n && tr.n <= 32768u;
    for (uint32_t r = 0; r < rounds; ++r) {
        if (launch_step(c->g, d_ops, n_ops, d_n_ops, d_status, r == 0, S(stream)) != cudaSuccess) return AVMP_ECUDA;
        c->launches += 1;
        if (c->opt.migration_enabled) {
            // the last round's copy launch also carries the translation: two launches per step, not three
            const cudaError_t e = (ride && r + 1 == rounds)
                                      ? launch_relocate_translate(c->g, tr.h, tr.n, tr.pool, tr.off, tr.aoff, L(c, stream))
                                      : launch_relocate(c->g, L(c, stream));
            if (e != cudaSuccess) return AVMP_ECUDA;
            c->launches += 1;
        }
    }
    if (tr.n && !ride) {
        if (launch_translate(c->g, tr.h, tr.n, tr.pool, tr.off, tr.aoff, L(c, stream)) != cudaSuccess) return AVMP_ECUDA;
        c->launches += 1;
    }
    return AVMP_OK;
}

int avmp_step(avmp_ctx *c, const avmp_op *d_ops, uint32_t n_ops, uint32_t *d_status, void *stream)
{
    if (!c) return AVMP_EINVAL;
    if (n_ops == 0) return AVMP_OK;
    if (!d_ops || !d_status || ((uintptr_t)d_ops & 3) || ((uintptr_t)d_status & 3)) return AVMP_EINVAL;
    return step_rounds(c, d_ops, n_ops, nullptr, d_status, stream);
}

int avmp_step_translate(avmp_ctx *c, const avmp_op *d_ops, uint32_t n_ops, uint32_t *d_status, const uint32_t *d_handles,
                        uint32_t n_handles, uint32_t *d_pool, uint64_t *d_offset, uint64_t *d_arena_offset, void *stream)
{
    if (!c) return AVMP_EINVAL;
    if (n_handles && (!d_handles || !d_pool || !d_offset)) return AVMP_EINVAL;
    if (n_ops == 0) return avmp_translate(c, d_handles, n_handles, d_pool, d_offset, d_arena_offset, stream);
    if (!d_ops || !d_status || ((uintptr_t)d_ops & 3) || ((uintptr_t)d_status & 3)) return AVMP_EINVAL;
    TranslateArgs tr;
    tr.h = d_handles; tr.n = n_handles; tr.pool = d_pool;
    tr.off = (unsigned long long *)d_offset; tr.aoff = (unsigned long long *)d_arena_offset;
    return step_rounds(c, d_ops, n_ops, nullptr, d_status, stream, tr);
}

int avmp_step_indirect(avmp_ctx *c, const avmp_op *d_ops, const uint32_t *d_n_ops, uint32_t max_ops,
                       uint32_t *d_status, void *stream)
{
    if (!c || max_ops == 0) return AVMP_EINVAL;
    if (!d_ops || !d_n_ops || !d_status || ((uintptr_t)d_ops & 3) || ((uintptr_t)d_status & 3) || ((uintptr_t)d_n_ops & 3))
        return AVMP_EINVAL;
    return step_rounds(c, d_ops, max_ops, d_n_ops, d_status, stream);
}

int avmp_step_host(avmp_ctx *c, const avmp_op *h_ops, uint32_t n_ops, uint32_t *h_status, void *stream)
{
    if (!c) return AVMP_EINVAL;
    if (n_ops == 0) return AVMP_OK;
    if (!h_ops || !h_status || n_ops > kHostStepMaxOps) return AVMP_EINVAL;
    if (cudaMemcpyAsync(c->d_stage_ops, h_ops, (size_t)n_ops * sizeof(avmp_op), cudaMemcpyHostToDevice, S(stream)) != cudaSuccess)
        return AVMP_ECUDA;
    int rc = avmp_step(c, c->d_stage_ops, n_ops, c->d_stage_status, stream);
    if (rc != AVMP_OK) return rc;
    if (cudaMemcpyAsync(h_status, c->d_stage_status, (size_t)n_ops * 4, cudaMemcpyDeviceToHost, S(stream)) != cudaSuccess)
        return AVMP_ECUDA;
    return cu(cudaStreamSynchronize(S(stream)));
}

int avmp_translate(avmp_ctx *c, const uint32_t *d_handles, uint32_t n, uint32_t *d_pool,
                   uint64_t *d_offset, uint64_t *d_arena_offset, void *stream)
{
    if (!c) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_handles || !d_pool || !d_offset) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_translate(c->g, d_handles, n, d_pool, (unsigned long long *)d_offset,
                               (unsigned long long *)d_arena_offset, L(c, stream)));
}

int avmp_gather_kv(avmp_ctx *c, uint32_t layer, const uint32_t *d_reqs, uint32_t n, void *d_out_k,
                   void *d_out_v, uint64_t cap_tokens, uint32_t *d_cu, void *stream)
{
    if (!c || layer >= c->spec.n_attn_layers || n > c->opt.max_requests || !d_cu) return AVMP_EINVAL;
    if (n && (!d_reqs || !d_out_k || !d_out_v)) return AVMP_EINVAL;
    if (((uintptr_t)d_out_k | (uintptr_t)d_out_v) & 15) return AVMP_EINVAL;
    c->launches += n > kLocalPlanMax ? 2 : 1;      // a separate plan launch only for long lists
    return cu(launch_kv(c->g, false, layer, 1, d_reqs, nullptr, n, d_out_k, d_out_v, 0, cap_tokens, d_cu, L(c, stream)));
}

int avmp_scatter_kv(avmp_ctx *c, uint32_t layer, const uint32_t *d_reqs, const uint32_t *d_tok_start,
                    uint32_t n, const void *d_in_k, const void *d_in_v, void *stream)
{
    if (!c || layer >= c->spec.n_attn_layers || n > c->opt.max_requests) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_in_k || !d_in_v || (((uintptr_t)d_in_k | (uintptr_t)d_in_v) & 15)) return AVMP_EINVAL;
    c->launches += n > kLocalPlanMax ? 2 : 1;      // a separate plan launch only for long lists
    return cu(launch_kv(c->g, true, layer, 1, d_reqs, d_tok_start, n, const_cast<void *>(d_in_k),
                        const_cast<void *>(d_in_v), 0, ~0ull, nullptr, L(c, stream)));
}

int avmp_gather_ssm(avmp_ctx *c, uint32_t layer, const uint32_t *d_reqs, uint32_t n, void *d_out_state,
                    void *d_out_conv, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_out_state || !d_out_conv || (((uintptr_t)d_out_state | (uintptr_t)d_out_conv) & 15)) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_ssm(c->g, false, layer, 1, d_reqs, n, d_out_state, 0, d_out_conv, 0, L(c, stream)));
}

int avmp_scatter_ssm(avmp_ctx *c, uint32_t layer, const uint32_t *d_reqs, uint32_t n, const void *d_in_state,
                     const void *d_in_conv, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_in_state || !d_in_conv || (((uintptr_t)d_in_state | (uintptr_t)d_in_conv) & 15)) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_ssm(c->g, true, layer, 1, d_reqs, n, const_cast<void *>(d_in_state), 0,
                         const_cast<void *>(d_in_conv), 0, L(c, stream)));
}

int avmp_gather_kv_layers(avmp_ctx *c, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs, uint32_t n,
                          void *d_out_k, void *d_out_v, uint64_t layer_stride_bytes, uint64_t cap_tokens,
                          uint32_t *d_cu, void *stream)
{
    if (!c || n_layers == 0 || (uint64_t)first_layer + n_layers > c->spec.n_attn_layers) return AVMP_EINVAL;
    if (n > c->opt.max_requests || !d_cu) return AVMP_EINVAL;
    if (n && (!d_reqs || !d_out_k || !d_out_v)) return AVMP_EINVAL;
    if (((uintptr_t)d_out_k | (uintptr_t)d_out_v | layer_stride_bytes) & 15) return AVMP_EINVAL;
    if (n_layers > 1 && layer_stride_bytes < cap_tokens * c->lay.kv_row_bytes) return AVMP_EINVAL;
    c->launches += n > kLocalPlanMax ? 2 : 1;      // a separate plan launch only for long lists
    return cu(launch_kv(c->g, false, first_layer, n_layers, d_reqs, nullptr, n, d_out_k, d_out_v, layer_stride_bytes,
                        cap_tokens, d_cu, L(c, stream)));
}

int avmp_gather_ssm_layers(avmp_ctx *c, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs, uint32_t n,
                           void *d_out_state, uint64_t state_layer_stride_bytes, void *d_out_conv,
                           uint64_t conv_layer_stride_bytes, void *stream)
{
    if (!c || n_layers == 0 || (uint64_t)first_layer + n_layers > c->spec.n_ssm_layers) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_out_state || !d_out_conv) return AVMP_EINVAL;
    if (((uintptr_t)d_out_state | (uintptr_t)d_out_conv | state_layer_stride_bytes | conv_layer_stride_bytes) & 15) return AVMP_EINVAL;
    if (n_layers > 1 && (state_layer_stride_bytes < (uint64_t)n * c->lay.ssm_state_bytes ||
                         conv_layer_stride_bytes < (uint64_t)n * c->lay.ssm_conv_bytes)) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_ssm(c->g, false, first_layer, n_layers, d_reqs, n, d_out_state, state_layer_stride_bytes,
                         d_out_conv, conv_layer_stride_bytes, L(c, stream)));
}

int avmp_gather_step(avmp_ctx *c, const uint32_t *d_reqs, uint32_t n, uint32_t first_attn_layer, uint32_t n_attn_layers,
                     void *d_out_k, void *d_out_v, uint64_t kv_layer_stride_bytes, uint64_t cap_tokens, uint32_t *d_cu,
                     uint32_t first_ssm_layer, uint32_t n_ssm_layers, void *d_out_state, uint64_t state_layer_stride_bytes,
                     void *d_out_conv, uint64_t conv_layer_stride_bytes, void *stream)
{
    if (!c || n_attn_layers == 0 || (uint64_t)first_attn_layer + n_attn_layers > c->spec.n_attn_layers) return AVMP_EINVAL;
    if (n_ssm_layers == 0 || (uint64_t)first_ssm_layer + n_ssm_layers > c->spec.n_ssm_layers) return AVMP_EINVAL;
    if (n > c->opt.max_requests || !d_cu) return AVMP_EINVAL;
    if (n && (!d_reqs || !d_out_k || !d_out_v || !d_out_state || !d_out_conv)) return AVMP_EINVAL;
    if (((uintptr_t)d_out_k | (uintptr_t)d_out_v | kv_layer_stride_bytes | (uintptr_t)d_out_state | (uintptr_t)d_out_conv |
         state_layer_stride_bytes | conv_layer_stride_bytes) & 15) return AVMP_EINVAL;
    if (n_attn_layers > 1 && kv_layer_stride_bytes < cap_tokens * c->lay.kv_row_bytes) return AVMP_EINVAL;
    if (n_ssm_layers > 1 && (state_layer_stride_bytes < (uint64_t)n * c->lay.ssm_state_bytes ||
                             conv_layer_stride_bytes < (uint64_t)n * c->lay.ssm_conv_bytes)) return AVMP_EINVAL;
    c->launches += n > kLocalPlanMax ? 2 : 1;
    return cu(launch_step_gather(c->g, d_reqs, n, first_attn_layer, n_attn_layers, d_out_k, d_out_v, kv_layer_stride_bytes,
                                 cap_tokens, d_cu, first_ssm_layer, n_ssm_layers, d_out_state, state_layer_stride_bytes,
                                 d_out_conv, conv_layer_stride_bytes, L(c, stream)));
}

int avmp_scatter_kv_layers(avmp_ctx *c, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs,
                           const uint32_t *d_tok_start, uint32_t n, const void *d_in_k, const void *d_in_v,
                           uint64_t layer_stride_bytes, void *stream)
{
    if (!c || n_layers == 0 || (uint64_t)first_layer + n_layers > c->spec.n_attn_layers || n > c->opt.max_requests) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_in_k || !d_in_v || (((uintptr_t)d_in_k | (uintptr_t)d_in_v | layer_stride_bytes) & 15)) return AVMP_EINVAL;
    c->launches += n > kLocalPlanMax ? 2 : 1;      // a separate plan launch only for long lists
    return cu(launch_kv(c->g, true, first_layer, n_layers, d_reqs, d_tok_start, n, const_cast<void *>(d_in_k),
                        const_cast<void *>(d_in_v), layer_stride_bytes, ~0ull, nullptr, L(c, stream)));
}

int avmp_scatter_ssm_layers(avmp_ctx *c, uint32_t first_layer, uint32_t n_layers, const uint32_t *d_reqs, uint32_t n,
                            const void *d_in_state, uint64_t state_layer_stride_bytes, const void *d_in_conv,
                            uint64_t conv_layer_stride_bytes, void *stream)
{
    if (!c || n_layers == 0 || (uint64_t)first_layer + n_layers > c->spec.n_ssm_layers) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_in_state || !d_in_conv) return AVMP_EINVAL;
    if (((uintptr_t)d_in_state | (uintptr_t)d_in_conv | state_layer_stride_bytes | conv_layer_stride_bytes) & 15) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_ssm(c->g, true, first_layer, n_layers, d_reqs, n, const_cast<void *>(d_in_state),
                         state_layer_stride_bytes, const_cast<void *>(d_in_conv), conv_layer_stride_bytes, L(c, stream)));
}

size_t avmp_attn_workspace_bytes(const avmp_ctx *c, const avmp_attn_desc *desc, uint32_t n)
{
    if (!c || !attn_desc_ok(c, desc) || n > c->opt.max_requests) return 0;
    return attn_ws_bytes(c->g, n ? n : 1, desc->q_heads, c->spec.kv_heads, c->spec.head_dim, c->n_sms);
}

int avmp_attn_prompt(avmp_ctx *c, uint32_t layer, const avmp_attn_desc *desc, const uint32_t *d_reqs, uint32_t n,
                     const uint32_t *d_cu_q, uint32_t total_q, const void *d_q, void *d_out, float *d_lse, void *d_workspace,
                     size_t workspace_bytes, void *stream)
{
    return attn_prompt_call(c, layer, desc, 0, 0, d_reqs, n, d_cu_q, total_q, d_q, d_out, d_lse, d_workspace, workspace_bytes, stream);
}

int avmp_attn_window_prompt(avmp_ctx *c, uint32_t layer, const avmp_attn_desc *desc, uint32_t window, uint32_t sinks, const uint32_t *d_reqs,
                            uint32_t n, const uint32_t *d_cu_q, uint32_t total_q, const void *d_q, void *d_out, float *d_lse,
                            void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (window == 0) return AVMP_EINVAL;
    return attn_prompt_call(c, layer, desc, window, sinks, d_reqs, n, d_cu_q, total_q, d_q, d_out, d_lse, d_workspace, workspace_bytes, stream);
}

int avmp_attn_decode(avmp_ctx *c, uint32_t layer, const avmp_attn_desc *desc, const uint32_t *d_reqs, uint32_t n,
                     uint32_t prefix_req, const void *d_q, void *d_out, float *d_lse, void *d_workspace, size_t workspace_bytes,
                     void *stream)
{
    return attn_decode_call(c, layer, desc, 0, 0, d_reqs, n, prefix_req, d_q, d_out, d_lse, d_workspace, workspace_bytes, stream);
}

int avmp_attn_window_decode(avmp_ctx *c, uint32_t layer, const avmp_attn_desc *desc, uint32_t window, uint32_t sinks, const uint32_t *d_reqs,
                            uint32_t n, const void *d_q, void *d_out, float *d_lse, void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (window == 0) return AVMP_EINVAL;
    return attn_decode_call(c, layer, desc, window, sinks, d_reqs, n, AVMP_INVALID, d_q, d_out, d_lse, d_workspace, workspace_bytes, stream);
}

size_t avmp_ssm_workspace_bytes(const avmp_ctx *c, const avmp_ssm_desc *desc, uint32_t n, uint32_t total_tokens)
{
    if (!c || !ssm_desc_ok(c, desc)) return 0;
    // Fewer requests are cut into more runs; from n_sms / (3 heads) requests up none is (see ssm_shares).
    size_t most = 0;
    for (uint32_t k = 1; k <= n && k <= (uint32_t)c->n_sms; ++k) {
        const size_t b = ssm_ws_bytes(c, desc, k, total_tokens);
        if (b > most) most = b;
    }
    return most;
}

int avmp_ssm_prompt(avmp_ctx *c, uint32_t layer, const avmp_ssm_desc *desc, const uint32_t *d_reqs, uint32_t n,
                    const uint32_t *d_cu, uint32_t total_tokens, const uint32_t *d_resume, const void *d_q, const void *d_k,
                    const void *d_v, const float *d_log_decay, void *d_out, void *d_workspace, size_t workspace_bytes, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers || n > c->opt.max_requests || !ssm_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_cu || (((uintptr_t)d_reqs | (uintptr_t)d_cu | (uintptr_t)d_resume) & 3)) return AVMP_EINVAL;
    if (total_tokens && !ssm_rows_ok(d_q, d_k, d_v, d_log_decay, d_out)) return AVMP_EINVAL;
    if (total_tokens >= (1u << 31) || (uint64_t)n * desc->heads * (desc->dv / 32) >= (1ull << 31)) return AVMP_EINVAL;
    SsmArgs a = ssm_args(desc, layer, d_reqs, n, d_q, d_k, d_v, d_log_decay, d_out);
    a.cu = d_cu; a.resume = d_resume; a.total = total_tokens; a.wait = c->wait;
    if (ssm_ws_bytes(c, desc, n, total_tokens)) {
        if (!d_workspace || ((uintptr_t)d_workspace & 15)) return AVMP_EINVAL;
        if (workspace_bytes < avmp_ssm_workspace_bytes(c, desc, n, total_tokens)) return AVMP_ENOSPC;
        a.ws = static_cast<float *>(d_workspace);
    }
    uint32_t launched = 0;
    const cudaError_t e = launch_ssm_prompt(c->g, a, L(c, stream), &launched);
    c->launches += launched;
    return cu(e);
}

int avmp_ssm_step(avmp_ctx *c, uint32_t layer, const avmp_ssm_desc *desc, const uint32_t *d_reqs, uint32_t n, const void *d_q,
                  const void *d_k, const void *d_v, const float *d_log_decay, void *d_out, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers || n > c->opt.max_requests || !ssm_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || ((uintptr_t)d_reqs & 3) || !ssm_rows_ok(d_q, d_k, d_v, d_log_decay, d_out)) return AVMP_EINVAL;
    if ((uint64_t)n * ((c->spec.ssm_state_elems + 1023u) / 1024u) >= (1ull << 31)) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_ssm_step(c->g, ssm_args(desc, layer, d_reqs, n, d_q, d_k, d_v, d_log_decay, d_out), L(c, stream)));
}

int avmp_conv_prompt(avmp_ctx *c, uint32_t layer, const avmp_conv_desc *desc, const uint32_t *d_reqs, uint32_t n, const uint32_t *d_cu,
                     uint32_t total_tokens, const uint32_t *d_resume, const void *d_x, const float *d_weight, const float *d_bias,
                     void *d_out, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers || n > c->opt.max_requests || !conv_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_cu || off4(d_reqs) || off4(d_cu) || off4(d_resume) || total_tokens >= (1u << 31)) return AVMP_EINVAL;
    return conv_call(c, layer, desc, d_reqs, n, d_cu, total_tokens, d_resume, d_x, d_weight, d_bias, d_out, stream);
}

int avmp_conv_step(avmp_ctx *c, uint32_t layer, const avmp_conv_desc *desc, const uint32_t *d_reqs, uint32_t n, const void *d_x,
                   const float *d_weight, const float *d_bias, void *d_out, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers || n > c->opt.max_requests || !conv_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || off4(d_reqs)) return AVMP_EINVAL;
    return conv_call(c, layer, desc, d_reqs, n, nullptr, n, nullptr, d_x, d_weight, d_bias, d_out, stream);
}

size_t avmp_scan_workspace_bytes(const avmp_ctx *c, const avmp_scan_desc *desc, uint32_t n, uint32_t total_tokens)
{
    if (!c || !scan_desc_ok(c, desc)) return 0;
    // Fewer requests are cut into more runs; with more than 4 n_sms / 3 none is cut (see scan_plan: three runs each would pass 4 n_sms).
    size_t most = 0;
    for (uint32_t k = 1; k <= n && k <= 4 * (uint32_t)c->n_sms / 3; ++k) {
        const size_t b = scan_ws_bytes(c, desc, k, total_tokens);
        if (b > most) most = b;
    }
    return most;
}

int avmp_scan_prompt(avmp_ctx *c, uint32_t layer, const avmp_scan_desc *desc, const uint32_t *d_reqs, uint32_t n, const uint32_t *d_cu,
                     uint32_t total_tokens, const uint32_t *d_resume, const void *d_u, const void *d_delta, const void *d_b, const void *d_c,
                     const void *d_z, const float *d_a, const float *d_d, const float *d_delta_bias, void *d_out, void *d_workspace,
                     size_t workspace_bytes, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers || n > c->opt.max_requests || !scan_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_cu || off4(d_reqs) || off4(d_cu) || off4(d_resume) || total_tokens >= (1u << 31)) return AVMP_EINVAL;
    if (!scan_rows_ok(total_tokens != 0, d_u, d_delta, d_b, d_c, d_z, d_a, d_d, d_delta_bias, d_out)) return AVMP_EINVAL;
    if ((uint64_t)n * (desc->channels / 8) >= (1ull << 31)) return AVMP_EINVAL;
    ScanArgs a = scan_args(desc, layer, d_reqs, n, d_u, d_delta, d_b, d_c, d_z, d_a, d_d, d_delta_bias, d_out);
    a.cu = d_cu; a.resume = d_resume; a.total = total_tokens;
    if (scan_ws_bytes(c, desc, n, total_tokens)) {
        if (!d_workspace || off16(d_workspace)) return AVMP_EINVAL;
        if (workspace_bytes < avmp_scan_workspace_bytes(c, desc, n, total_tokens)) return AVMP_ENOSPC;
        a.ws = static_cast<float *>(d_workspace);
        a.shares = scan_shares(n, desc->channels, desc->groups, desc->states, total_tokens, c->n_sms);
    }
    uint32_t launched = 0;
    const cudaError_t e = launch_scan_prompt(c->g, a, L(c, stream), &launched);
    c->launches += launched;
    return cu(e);
}

int avmp_scan_step(avmp_ctx *c, uint32_t layer, const avmp_scan_desc *desc, const uint32_t *d_reqs, uint32_t n, const void *d_u,
                   const void *d_delta, const void *d_b, const void *d_c, const void *d_z, const float *d_a, const float *d_d,
                   const float *d_delta_bias, void *d_out, void *stream)
{
    if (!c || layer >= c->spec.n_ssm_layers || n > c->opt.max_requests || !scan_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || off4(d_reqs) || !scan_rows_ok(true, d_u, d_delta, d_b, d_c, d_z, d_a, d_d, d_delta_bias, d_out)) return AVMP_EINVAL;
    c->launches += 1;
    return cu(launch_scan_step(c->g, scan_args(desc, layer, d_reqs, n, d_u, d_delta, d_b, d_c, d_z, d_a, d_d, d_delta_bias, d_out), L(c, stream)));
}

int avmp_attn_rows_prompt(avmp_ctx *c, uint32_t layer, const avmp_rows_desc *desc, const uint32_t *d_reqs, uint32_t n, const uint32_t *d_cu,
                          uint32_t total_tokens, const uint32_t *d_pos, const void *d_q, const void *d_k, const void *d_v,
                          const float *d_q_weight, const float *d_k_weight, const float *d_freq, void *d_out, void *stream)
{
    if (!c || layer >= c->spec.n_attn_layers || n > c->opt.max_requests || !rows_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || !d_cu || off4(d_reqs) || off4(d_cu) || total_tokens >= (1u << 31)) return AVMP_EINVAL;
    return rows_call(c, layer, desc, d_reqs, n, d_cu, total_tokens, d_pos, d_q, d_k, d_v, d_q_weight, d_k_weight, d_freq, d_out, stream);
}

int avmp_attn_rows_step(avmp_ctx *c, uint32_t layer, const avmp_rows_desc *desc, const uint32_t *d_reqs, uint32_t n, const uint32_t *d_pos,
                        const void *d_q, const void *d_k, const void *d_v, const float *d_q_weight, const float *d_k_weight,
                        const float *d_freq, void *d_out, void *stream)
{
    if (!c || layer >= c->spec.n_attn_layers || n > c->opt.max_requests || !rows_desc_ok(c, desc) || !device_ok(c)) return AVMP_EINVAL;
    if (n == 0) return AVMP_OK;
    if (!d_reqs || off4(d_reqs)) return AVMP_EINVAL;
    return rows_call(c, layer, desc, d_reqs, n, nullptr, n, d_pos, d_q, d_k, d_v, d_q_weight, d_k_weight, d_freq, d_out, stream);
}

int avmp_get_stats(avmp_ctx *c, avmp_stats *h_out, void *stream)
{
    if (!c || !h_out) return AVMP_EINVAL;
    DevState d;
    if (cudaMemcpyAsync(&d, c->g.st, sizeof(d), cudaMemcpyDeviceToHost, S(stream)) != cudaSuccess) return AVMP_ECUDA;
    if (cudaStreamSynchronize(S(stream)) != cudaSuccess) return AVMP_ECUDA;
    fill_stats(c, d, h_out);
    return AVMP_OK;
}

int avmp_clear_error(avmp_ctx *c, void *stream)
{
    if (!c) return AVMP_EINVAL;
    return cu(cudaMemsetAsync(&c->g.st->error_code, 0, 16, S(stream)));
}

int avmp_export_tables(avmp_ctx *c, avmp_tables *t, void *stream)
{
    if (!c || !t) return AVMP_EINVAL;
    const Geom &g = c->g;
    cudaStream_t s = S(stream);
    DevState d;
    bool ok = cudaMemcpyAsync(&d, g.st, sizeof(d), cudaMemcpyDeviceToHost, s) == cudaSuccess;
    auto pull = [&](uint32_t *dst, const uint32_t *src, size_t n) {
        if (dst && n) ok = ok && cudaMemcpyAsync(dst, src, n * 4, cudaMemcpyDeviceToHost, s) == cudaSuccess;
    };
    for (int p = 0; p < 2; ++p) {
        pull(t->slot_stack[p], g.S[p], g.V[p]); pull(t->vid_stack[p], g.W[p], g.V[p]);
        pull(t->vt[p], g.VT[p], g.V[p]); pull(t->ow[p], g.OW[p], g.V[p]);
    }
    pull(t->req_state, g.r_state, g.R); pull(t->req_len, g.r_len, g.R); pull(t->req_npages, g.r_npages, g.R);
    pull(t->req_chain, g.r_chain, (size_t)g.R * g.max_pages); pull(t->req_ssm, g.r_ssm, (size_t)g.R * g.ns);
    if (!ok || cudaStreamSynchronize(s) != cudaSuccess) return AVMP_ECUDA;
    for (int p = 0; p < 2; ++p) { t->n_slot_stack[p] = d.n_free[p]; t->n_vid_stack[p] = d.n_vfree[p]; }
    fill_stats(c, d, &t->stats);
    return AVMP_OK;
}

int avmp_import_tables(avmp_ctx *c, const avmp_tables *t, void *stream)
{
    if (!c || !t) return AVMP_EINVAL;
    const Geom &g = c->g;
    cudaStream_t s = S(stream);
    for (int p = 0; p < 2; ++p) {
        if (!t->slot_stack[p] || !t->vid_stack[p] || !t->vt[p] || !t->ow[p]) return AVMP_EINVAL;
        if (t->n_slot_stack[p] > g.V[p] || t->n_vid_stack[p] > g.V[p] || t->stats.cap[p] > g.V[p]) return AVMP_EINVAL;
    }
    if (!t->req_state || !t->req_len || !t->req_npages || !t->req_chain || (g.ns && !t->req_ssm)) return AVMP_EINVAL;
    if (!tables_consistent(c, t)) return AVMP_EINVAL;          // nothing has been copied yet
    bool ok = true;
    auto push = [&](uint32_t *dst, const uint32_t *src, size_t n) {
        if (n) ok = ok && cudaMemcpyAsync(dst, src, n * 4, cudaMemcpyHostToDevice, s) == cudaSuccess;
    };
    for (int p = 0; p < 2; ++p) {
        push(g.S[p], t->slot_stack[p], g.V[p]); push(g.W[p], t->vid_stack[p], g.V[p]);
        push(g.VT[p], t->vt[p], g.V[p]); push(g.OW[p], t->ow[p], g.V[p]);
    }
    push(g.r_state, t->req_state, g.R); push(g.r_len, t->req_len, g.R); push(g.r_npages, t->req_npages, g.R);
    push(g.r_chain, t->req_chain, (size_t)g.R * g.max_pages); push(g.r_ssm, t->req_ssm, (size_t)g.R * g.ns);
    DevState d;
    memset(&d, 0, sizeof(d));
    const avmp_stats &st = t->stats;
    d.op_counter = st.op_counter; d.last_rebalance_op = st.last_rebalance_op; d.n_oom = st.n_oom;
    d.n_capacity_error = st.n_capacity_error; d.n_rebalance = st.n_rebalance;
    d.migrated_bytes = st.migrated_bytes; d.wasted_bytes = st.wasted_bytes;
    d.relocated_blocks = st.relocated_blocks; d.relocated_bytes = st.relocated_bytes;
    d.gap_bytes = st.gap_bytes; d.n_invalid = st.n_invalid;
    for (int p = 0; p < 2; ++p) {
        d.cap[p] = (uint32_t)st.cap[p]; d.n_free[p] = t->n_slot_stack[p]; d.n_vfree[p] = t->n_vid_stack[p];
    }
    d.fsm = (uint32_t)st.fsm_state;
    ok = ok && cudaMemcpyAsync(g.st, &d, sizeof(d), cudaMemcpyHostToDevice, s) == cudaSuccess;
    // the host arrays (and `d`) must outlive the copies
    if (!ok || cudaStreamSynchronize(s) != cudaSuccess) return AVMP_ECUDA;
    return AVMP_OK;
}

int avmp_set_wait_limit(avmp_ctx *c, uint64_t ns)
{
    if (!c) return AVMP_EINVAL;
    c->wait = WaitLimit{ns < kWaitLimitNs ? ns : kWaitLimitNs, ns < 1000000u ? 0u : 64u};
    return AVMP_OK;
}

uint64_t avmp_launch_count(const avmp_ctx *c) { return c ? c->launches : 0; }

const char *avmp_error_string(int code)
{
    switch (code) {
    case AVMP_OK: return "ok";
    case AVMP_EINVAL: return "invalid argument";
    case AVMP_ENOSPC: return "workspace too small";
    case AVMP_ECUDA: return "CUDA runtime error";
    case AVMP_ETOOBIG: return "request list longer than the fixed in-library scratch allows (AVMP_STATIC_GATHER_MAX_REQS)";
    default: return "unknown error";
    }
}

}  // extern "C"
