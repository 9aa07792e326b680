// Attention of many query rows over paged KV chains on the tensor cores: whole prompts (causal, packed requests of
// different lengths, grouped heads), and a batch of single tokens over a prefix that all of them share.
//
// A tile is 256 query rows of one KV head: the (token, query head) pairs that share that head, tokens first, so grouped
// heads fill the rows of the tensor-core tiles whatever the group is, and every K and V row is loaded once for all of them.
// Over it run the KV tokens, 128 at a time:
//     S = Q K^T  (tcgen05, sums in tensor memory),  P = 2^(S - m),  O += P V  (P as an operand in tensor memory).
// One CTA per SM, 12 warps: two warpgroups own 128 rows each (a thread is a row: the softmax needs no exchange), a warp each
// loads K and V slices of pages by tiled copies (the latter the query rows too), one issues the products, one hands out
// tiles.  While one warpgroup exponentiates, the tensor cores work for the other.  The running maximum m is only moved when
// it grows by more than 2^8 (sums are 32-bit), so the accumulator is rarely rescaled.  Weights are taken times a power of two that
// puts them where their type has room: bf16 to at most 1 (a weight of 2^8 times a value of 2^120 would pass 32 bits), fp16 to at most
// 2^15 (its subnormal numbers begin at 2^-14; tens of thousands of weights of 2^-25 would be rounded to nothing).
//
// Measured (32 query heads on 8 KV heads of 128, bf16): a prompt of 32 749 tokens 7.0 ms alone (1 250 TFLOP/s), 8.0 to 8.1 ms in a
// loop, where the card's power limit holds the clock near 1.58 GHz (1 090 TFLOP/s, 81 % of what cuBLAS sustains there).  Long
// tiles are bound by that; short ones (32 prompts of 32 to 512 tokens: 51 us) by the chain load, S, P, O, store.
// P is rounded to the 16 bits of V (eps/2 per weight, averaged over the tokens: an output is 1.2 to 1.4 times as far from the formula as its own
// rounding alone); denominators are summed before that.
// A weight of zero does not silence a NaN or an infinity in V, so one in a token that some rows of a tile do not see spoils those rows.
// It shows when they are written out: such tiles are noted and done once more behind the others, with zeros in the place of what is not finite
// in tokens that some row does not see, and with these values added, from the cache, to the rows that do see them.  (32 short
// prompts: 48.1 us without, 50.6 so; 55 to 58 with V looked over in every tile beforehand.)
// With a window (and the first tokens as sinks) a tile's rounds run over what any of its rows sees: the sinks, in whole boxes, then from the
// first token in its first row's window on, without the gap between, so that both may lie in one round; what a row does not see of
// a round is masked by bits.  Measured with a window of 1024 and 4 sinks: 12 turns of 256 to 2048 tokens behind up to 8192, 32 heads, fp16,
// 213 us (309 with sinks and window in rounds of their own), window 4096, 32 749 tokens 1 750 alone, 2 020 in a loop (power).  A tile costs
// about 7 us beside its rounds (first copies and products, last products and rows out), 1.9 each: small windows are bound by that.
#include "avmp_tc.cuh"

namespace avmp {

namespace {

constexpr int kRows = 256;                    // query rows per tile
constexpr int kKv = 128;                      // KV tokens per round
constexpr int kCta = 384;
constexpr int kAnnounce = 64;                 // the first 64 tokens' weights are announced behind the weights from here
constexpr uint32_t kAhead = 2;                // rounds ahead that the prefix pass calls rows into L2
constexpr int kPoly = 0x08;                   // which of 8 pairs of exponentials go to the multiply-add pipe (long prompt: none 8.40 ms, 1 8.33, 2 8.38, 3 8.85)

struct Tile { uint32_t k, b; };                          // list entry, row block
struct Item { uint32_t req, len, q0, nq; };              // slot, held tokens, first row, rows

struct PromptArgs {
    AttnArgs a;
    uint32_t group, splits, box_tokens;
    bool q_boxes;                 // query rows come in by tiled copies (groups of 1, 2, 4 .. 64)
    uint32_t cap;                 // entries of `tiles`
    uint32_t prefix_blocks;       // row blocks of the prefix pass
    uint32_t *n_tiles;
    Tile *tiles;
    Item *items;
    Parts parts;                  // [split][total rows][q_heads], where splits > 1 or for a prefix
};

// ---------------------------------------------------------------- plan
// One CTA: checks every list entry and writes the row blocks of the good ones, longest reach first within a request.
__global__ void __launch_bounds__(kStepThreads) prompt_plan_kernel(const Geom g, const PromptArgs p)
{
    __shared__ unsigned long long tmp[32];
    __shared__ uint32_t pre[kStepThreads + 1];
    pdl_prologue();
    uint32_t base = 0;
    for (uint32_t w = 0; w < p.a.n; w += kStepThreads) {
        const uint32_t k = w + threadIdx.x, cnt = min((uint32_t)kStepThreads, p.a.n - w);
        unsigned long long blocks = 0, tot;
        Item it = {};
        if (k < p.a.n) {
            const uint32_t r = p.a.reqs[k], c0 = p.a.cu[k], c1 = p.a.cu[k + 1];
            const uint32_t len = held_tokens(g, r);
            it = Item{r, len, c0, c1 - c0};
            if (len && c1 >= c0 && c1 <= p.a.total_q && it.nq <= len) blocks = ((unsigned long long)it.nq * p.group + kRows - 1) / kRows;
            else record_error(g.st, AVMP_DEV_BAD_REQUEST);
        }
        const unsigned long long incl = block_incl_scan(blocks, tmp, &tot);
        // offsets that run backwards can own more blocks than there are rows: what passes the list's end is skipped
        if (k < p.a.n && base + incl > p.cap && blocks) record_error(g.st, AVMP_DEV_BAD_REQUEST);
        pre[threadIdx.x] = (uint32_t)min((unsigned long long)p.cap, base + incl - blocks);
        if (threadIdx.x == 0) pre[cnt] = (uint32_t)min((unsigned long long)p.cap, base + tot);
        if (k < p.a.n) p.items[k] = it;
        __syncthreads();
        for (uint32_t i = base + threadIdx.x; i < pre[cnt]; i += kStepThreads) {
            const uint32_t e = find_owner(pre, 0, cnt, 0, i);
            const uint32_t n_blocks = (uint32_t)(((unsigned long long)(p.a.cu[w + e + 1] - p.a.cu[w + e]) * p.group + kRows - 1) / kRows);
            p.tiles[i] = Tile{w + e, n_blocks - 1 - (i - pre[e])};
        }
        base = pre[cnt];
        __syncthreads();
    }
    if (threadIdx.x == 0) *p.n_tiles = base;
}

// Adds what is not finite among 16 columns of V, tokens t0 .. t1 of a chain, to a row's sums.  (For the few rows that have such values.)
template <class T>
__device__ __forceinline__ void add_not_finite(const Geom &g, const uint32_t *chain, uint32_t t0, uint32_t t1, unsigned long long in_page, uint32_t (&o)[16])
{
    for (uint32_t t = t0; t < t1; ++t) {
        const uint8_t *row = unit_ptr(g, AVMP_POOL_KV, g.VT[0][chain[t / g.T] & 0x7FFFFFFFu]) + in_page + t % g.T * g.row_bytes;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const uint4 x = *reinterpret_cast<const uint4 *>(row + u * 16);
            const uint32_t v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (!T::marked(T::mark(v[i], 0))) continue;
                const float2 y = T::unpack(v[i]);
                uint32_t *to = o + u * 8 + i * 2;
                if (!(fabsf(y.x) < INFINITY)) to[0] = __float_as_uint(__uint_as_float(to[0]) + y.x);
                if (!(fabsf(y.y) < INFINITY)) to[1] = __float_as_uint(__uint_as_float(to[1]) + y.y);
            }
        }
    }
}

// ---------------------------------------------------------------- the tiles
struct Work {
    uint32_t k, head, split, req;
    uint32_t rows, row0;          // rows of this tile, its first row (token * group + head in group)
    uint32_t q0;                  // first row of the request in the packed buffers
    uint32_t past;                // tokens in front of the request's first query row
    uint32_t held;                // tokens of the chain
    uint32_t len;                 // tokens that the tile's last row sees
    uint32_t j0, j1;              // KV rounds
    uint32_t lead, shift;         // with a window, `past`, `held` and `len` leave the `shift` tokens out that no row sees: they lie behind the first `lead`
    uint32_t tok0, rem0;          // token and head in group of the tile's first row
    bool end;                     // with no rows: nothing follows
};

// The i-th tile of CTA c: the list runs from long tiles to short ones, every other pass over the CTAs backwards.
__device__ __forceinline__ uint32_t nth_tile(uint32_t i) { return i * gridDim.x + (i & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x); }

template <bool WINDOW>
__device__ __forceinline__ Work make_work(const PromptArgs &p, uint32_t k, uint32_t req, uint32_t held, uint32_t past, uint32_t q0,
                                          uint32_t all_rows, uint32_t block, uint32_t head, uint32_t split, bool causal)
{
    Work w;
    w.k = k; w.req = req; w.held = held; w.past = past; w.q0 = q0; w.head = head; w.split = split;
    w.row0 = block * kRows;
    w.rows = min((uint32_t)kRows, all_rows - w.row0);
    w.tok0 = w.row0 / p.group; w.rem0 = w.row0 - w.tok0 * p.group;
    w.len = causal ? past + (w.row0 + w.rows - 1) / p.group + 1 : held;
    w.lead = w.shift = 0;
    if (WINDOW) {
        // What the tile's rows see: the sinks, then everything from the first token in the first row's window, in whole boxes.  Rounds
        // run over these tokens without the gap between.
        const uint32_t at = past + w.tok0, low = at >= p.a.window ? (at - p.a.window + 1) / p.box_tokens * p.box_tokens : 0u;
        w.lead = p.a.sinks < low ? (p.a.sinks + p.box_tokens - 1) / p.box_tokens * p.box_tokens : low;
        w.shift = low - w.lead;
        w.past -= w.shift; w.held -= w.shift; w.len -= w.shift;
    }
    const uint32_t rounds = (w.len + kKv - 1) / kKv;
    w.j0 = 0; w.j1 = rounds;
    if (p.splits > 1) {      // shares of whole rounds: the first `rest` get one more
        const uint32_t each = rounds / p.splits, rest = rounds - each * p.splits;
        w.j0 = split * each + min(split, rest);
        w.j1 = w.j0 + each + (split < rest ? 1u : 0u);
    }
    return w;
}

// One warp hands the CTA's tiles out, a few ahead of the others, through a ring in shared memory.  `give(work)` returns
// false when the CTA stops; `wanted(n)` tells whether the CTA's n-th tile is to be given; `report`: bad entries are recorded (the first time).
//   prefix: row blocks of the whole batch.
//   up to 32 list entries: a lane per entry; tiles in descending order of their KV rounds over all entries, so that the
//     long ones start first.  How many row blocks have R rounds or more has a closed form per entry, so the i-th of
//     that order is found by bisection over R and a sum over the lanes, without a list.
//   more: the list that prompt_plan_kernel wrote.
template <bool PREFIX, bool WINDOW, class Wanted, class Give>
__device__ __forceinline__ void hand_out(const Geom &g, const PromptArgs &p, bool report, Wanted wanted, Give give)
{
    const uint32_t lane = threadIdx.x % 32, per = p.a.kv_heads * p.splits;
    if (PREFIX) {
        const uint32_t r = p.a.prefix, held = held_tokens(g, r);
        for (uint32_t n = 0, i; (i = nth_tile(n)) < p.prefix_blocks * per; ++n)
            if (wanted(n) && !give(make_work<WINDOW>(p, 0, r, held, 0, 0, p.a.n * p.group, i / per, i % per / p.splits, i % p.splits, false))) return;
    } else if (p.tiles) {
        const uint32_t n_tiles = *(volatile uint32_t *)p.n_tiles;
        for (uint32_t n = 0, i; (i = nth_tile(n)) < n_tiles * per; ++n) {
            if (!wanted(n)) continue;
            const Tile t = p.tiles[i / per];
            const Item it = p.items[t.k];
            if (!give(make_work<WINDOW>(p, t.k, it.req, it.len, it.len - it.nq, it.q0, it.nq * p.group, t.b, i % per / p.splits, i % p.splits, true))) return;
        }
    } else {
        uint32_t req = 0, held = 0, q0 = 0, nq = 0, blocks = 0, top = 0;
        if (lane < p.a.n) {
            req = p.a.reqs[lane]; q0 = p.a.cu[lane];
            const uint32_t q1 = p.a.cu[lane + 1];
            held = held_tokens(g, req);
            if (held && q1 >= q0 && q1 <= p.a.total_q && q1 - q0 <= held) {
                nq = q1 - q0;
                blocks = (nq * p.group + kRows - 1) / kRows;      // total_q * q_heads < 2^31
                if (nq) top = (held + kKv - 1) / kKv;
            } else if (report && blockIdx.x == 0) {
                record_error(g.st, AVMP_DEV_BAD_REQUEST);
            }
        }
        const uint32_t past = held - nq, all = __reduce_add_sync(0xFFFFFFFFu, blocks), most = __reduce_max_sync(0xFFFFFFFFu, top);
        // first row block of this lane's entry with at least R rounds (R >= 1)
        auto first = [&](uint32_t R) {
            const uint32_t x = (R - 1) * kKv;            // its last token stands at position x or later
            if (x <= past) return 0u;
            return x - past >= nq ? blocks : min(blocks, (x - past) * p.group / kRows);
        };
        for (uint32_t n = 0, i; (i = nth_tile(n)) < all * p.a.kv_heads; ++n) {
            if (!wanted(n)) continue;
            const uint32_t e = i / p.a.kv_heads;
            uint32_t lo = 1, hi = most + 1;              // count(lo) > e >= count(hi)
            while (lo + 1 < hi) {
                const uint32_t mid = (lo + hi) >> 1;
                if (__reduce_add_sync(0xFFFFFFFFu, blocks - first(mid)) > e) lo = mid; else hi = mid;
            }
            const uint32_t f0 = first(lo), f1 = first(lo + 1), mine = f1 - f0;      // blocks with exactly lo rounds
            uint32_t incl = mine;
#pragma unroll
            for (int x = 1; x < 32; x <<= 1) {
                const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, incl, x);
                if (lane >= x) incl += y;
            }
            const uint32_t at = e - __reduce_add_sync(0xFFFFFFFFu, blocks - f1);
            const uint32_t owner = __ffs(__ballot_sync(0xFFFFFFFFu, incl > at)) - 1;
            const uint32_t block = __shfl_sync(0xFFFFFFFFu, f0 + at - (incl - mine), owner);
            if (!give(make_work<WINDOW>(p, owner, __shfl_sync(0xFFFFFFFFu, req, owner), __shfl_sync(0xFFFFFFFFu, held, owner),
                                __shfl_sync(0xFFFFFFFFu, past, owner), __shfl_sync(0xFFFFFFFFu, q0, owner),
                                __shfl_sync(0xFFFFFFFFu, nq, owner) * p.group, block, i - e * p.a.kv_heads, 0, true))) return;
        }
    }
}

template <int D>
struct Smem {
    static constexpr uint32_t kQ = 128 * D * 2;             // one warpgroup's query rows
    static constexpr uint32_t kTile = kKv * D * 2;          // K or V of a round
    static constexpr uint32_t kSlots = D == 128 ? 5 : 10;
    static constexpr uint32_t oRing = 2 * kQ;
    static constexpr uint32_t kTotal = oRing + kSlots * kTile + 1024;
};

enum { B_FULL = 0, B_EMPTY = 10, B_Q = 20, B_S = 22, B_P = 24, B_O = 28, B_DONE = 30, B_WORK = 31, B_TAKEN = 35, B_QFREE = 39, B_COUNT = 41 };
constexpr int kRowsBar = 1, kRowsBarThreads = 288;       // the rows' warps and the one that hands tiles out: all rows are out
constexpr uint32_t kWorks = 4;                // ring of work items
constexpr uint32_t kMarks = 8;                // marks of tiles, by their count (the warpgroups are less than kWorks tiles apart)
constexpr uint32_t kRedo = 2048;              // bits for tiles to be done again (tiles that share a bit are done again together)

template <class T> constexpr float kLift = T::kF16 ? 7.f : -8.f;         // weights are 2^(score - m + kLift), score - m at most 8

template <class T, int D, bool PREFIX, bool WINDOW>
__global__ void __launch_bounds__(kCta, 1)
attn_tile_kernel(const Geom g, const PromptArgs p, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map)
{
    using M = Smem<D>;
    constexpr uint32_t kHalf = kKv * 128;                    // 64 columns of a Q tile
    constexpr uint32_t kGroup = 8 * D * 2;                   // 8 tokens of a K or V tile: its column blocks one behind the other
    constexpr uint32_t kS = 0, kO = 256;                     // tensor memory columns: S0 S1 (P in their first half) O0 O1
    extern __shared__ uint8_t smem_raw[];
    __shared__ unsigned long long bars_s[B_COUNT];
    __shared__ Work works[kWorks];
    __shared__ uint32_t tmem_s, gave_up, marks[kMarks], redo[kRedo / 32], any_redo, loads[2];
    uint8_t *smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const uint32_t base = smem_u32(smem), bars = smem_u32(bars_s);
    const int w = threadIdx.x / 32, lane = threadIdx.x % 32;
    const Waits waits{&gave_up, p.a.wait};
    uint32_t q_loads[2] = {0, 0};                            // query copies issued (by the warp that loads V)
    auto bar = [&](uint32_t i) { return bars + 8 * i; };
    if (threadIdx.x == 0) {
        gave_up = any_redo = 0;
        for (uint32_t i = 0; i < kMarks; ++i) marks[i] = 0;
        for (uint32_t i = 0; i < M::kSlots; ++i) { mbar_init(bar(B_FULL + i), 1); mbar_init(bar(B_EMPTY + i), 1); }
        for (uint32_t t = 0; t < 2; ++t) {
            mbar_init(bar(B_Q + t), p.q_boxes ? 1 : 128); mbar_init(bar(B_QFREE + t), 1); mbar_init(bar(B_S + t), 1); mbar_init(bar(B_O + t), 1);
            mbar_init(bar(B_P + 2 * t), 128); mbar_init(bar(B_P + 2 * t + 1), 128);
        }
        for (uint32_t i = 0; i < kWorks; ++i) { mbar_init(bar(B_WORK + i), 1); mbar_init(bar(B_TAKEN + i), 11); }
        mbar_init(bar(B_DONE), 1);
        mbar_fence_init();
        tma_prefetch_map(&map);
        if (p.q_boxes) tma_prefetch_map(&q_map);
    }
    if (w == 9) tmem_alloc512(smem_u32(&tmem_s));
    if (w == 10) for (uint32_t i = lane; i < kRedo / 32; i += 32) redo[i] = 0;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_s;
    if (PREFIX) {
        // the decode kernel that follows starts without waiting for this one: let it only once all in front is complete
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    } else {
        pdl_prologue();
    }

    if (w >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (w == 8 || w == 10) {
            // ---------------- loads: K by one warp, V by another.  The lanes look the pages up a round ahead; one thread issues.
            const uint32_t v = w == 8 ? 0 : 1, page_rows = (uint32_t)(g.U[0] / (D * 2));
            uint32_t it = v;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                ok = mbar_wait(bar(B_WORK + n % kWorks), n / kWorks & 1, waits);
                if (!ok) break;
                const Work t = works[n % kWorks];
                const uint32_t rows = t.rows, j0 = t.j0, j1 = t.j1, head = t.head, token = t.q0 + t.tok0;
                const bool t_end = t.end;
                const uint32_t need = min((t.len + 15u) & ~15u, t.held);     // products run over whole steps of 16 tokens
                const uint32_t *chain = g.r_chain + (unsigned long long)t.req * g.max_pages;
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_TAKEN + n % kWorks));
                if (rows == 0) {
                    if (t_end) break;
                    continue;
                }
                const uint32_t part_row = (p.a.layer * 2 + v) * g.T * p.a.kv_heads + head;
                auto in_chain = [&](uint32_t tok) { return WINDOW && tok >= t.lead ? tok + t.shift : tok; };
                auto look = [&](uint32_t j) -> uint32_t {      // lane b: slot of the page that holds box b of round j
                    const uint32_t tok = j * kKv + lane * p.box_tokens;
                    if (j >= j1 || lane * p.box_tokens >= kKv || tok >= need) return kInvalid;
                    return g.VT[0][chain[in_chain(tok) / g.T] & 0x7FFFFFFFu];
                };
                uint32_t next = look(j0);
                if (v == 1 && p.q_boxes && j0 < j1) {
                    // query rows, as soon as the products of the tile before have read theirs
#pragma unroll
                    for (uint32_t m = 0; m < 2; ++m) {
                        if (m * 128 >= rows || !ok) continue;
                        if (q_loads[m]) ok = mbar_wait(bar(B_QFREE + m), (q_loads[m] - 1) & 1, waits);
                        if (!ok) continue;
                        q_loads[m] += 1;
                        if (elect_one()) {
                            mbar_expect(bar(B_Q + m), M::kQ);
#pragma unroll
                            for (int x = 0; x < D / 64; ++x)
                                tma_load_query(base + m * M::kQ + x * kHalf, &q_map, bar(B_Q + m), x * 64, head * p.group, token + m * 128 / p.group);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
                for (uint32_t j = j0; j < j1; ++j, it += 2) {
                    const uint32_t slot = next;
                    const uint32_t boxes = __popc(__ballot_sync(0xFFFFFFFFu, slot != kInvalid));
                    uint32_t tok = (j * kKv) % g.T;
                    const uint32_t off = WINDOW ? in_chain(j * kKv + lane * p.box_tokens) % g.T : 0u;      // lane b: of box b in its page
                    const uint32_t s = it % M::kSlots, round = it / M::kSlots, full = bar(B_FULL + s);
                    ok = !round || mbar_wait(bar(B_EMPTY + s), (round - 1) & 1, waits);
                    if (!ok) break;
                    uint32_t dst = base + M::oRing + s * M::kTile;
                    if (elect_one()) mbar_expect(full, boxes * p.box_tokens * D * 2);
                    for (uint32_t b = 0; b < boxes; ++b) {
                        const uint32_t page = __shfl_sync(0xFFFFFFFFu, slot, b);
                        if (WINDOW) tok = __shfl_sync(0xFFFFFFFFu, off, b);
                        if (elect_one()) tma_load_rows(dst, &map, full, tok / 8, page * page_rows + part_row);
                        dst += p.box_tokens * D * 2;
                        tok += p.box_tokens;
                        if (tok >= g.T) tok = 0;
                    }
                    next = look(j + 1);
                    if (PREFIX) {
                        // every row of the prefix is read once and comes from HBM: the round behind the ring is called into L2 now
                        const uint32_t far = look(j + kAhead), n_far = __popc(__ballot_sync(0xFFFFFFFFu, far != kInvalid));
                        uint32_t tok_far = ((j + kAhead) * kKv) % g.T;
                        for (uint32_t b = 0; b < n_far; ++b) {
                            const uint32_t page = __shfl_sync(0xFFFFFFFFu, far, b);
                            if (elect_one()) tma_prefetch_rows(&map, tok_far / 8, page * page_rows + part_row);
                            tok_far += p.box_tokens;
                            if (tok_far >= g.T) tok_far = 0;
                        }
                    }
                }
            }
            if (lane == 0) loads[v] = it;
        } else if (w == 9) {
            // ---------------- products, all by one thread and for the two warpgroups in turn: that keeps them apart, so that one
            // exponentiates while the tensor cores work for the other.  (With a thread for each they fall into step and
            // contend for everything: 10.4 against 8.2 ms for the long prompt.)
            if (elect_one()) {
                const uint32_t id_s = tc_idesc(T::kF16, false, kKv) | (p.a.scale < 0.f ? kNegateA : 0u);    // a negative scale is one of -q
                constexpr uint32_t id_o = tc_idesc(T::kF16, true, D);
                uint32_t it = 0, tiles0 = 0, tiles1 = 0, rounds0 = 0, rounds1 = 0;
                bool ok = true;
                const unsigned long long q_desc = tc_desc(base, 1024, 16), k_desc = tc_desc(base + M::oRing, kGroup, 16), v_desc = tc_desc(base + M::oRing, kGroup, 1024);
                auto issue_s = [&](uint32_t m, uint32_t slot) {
                    const unsigned long long a = q_desc + ((m * M::kQ) >> 4), b = k_desc + ((slot * M::kTile) >> 4);
#pragma unroll
                    for (int x = 0; x < D / 16; ++x) {
                        tc_mma_ss(tmem + kS + m * 128, a + (((x >> 2) * kHalf + (x & 3) * 32) >> 4), b + (((x >> 2) * 1024 + (x & 3) * 32) >> 4), id_s, x > 0);
                    }
                    tc_commit(bar(B_S + m));
                };
                auto full = [&](uint32_t n) { return mbar_wait_one(bar(B_FULL + n % M::kSlots), (n / M::kSlots) & 1, waits); };
                for (uint32_t n = 0; ok; ++n) {
                    ok = mbar_wait_one(bar(B_WORK + n % kWorks), n / kWorks & 1, waits);
                    if (!ok) break;
                    const Work t = works[n % kWorks];
                    const uint32_t rows = t.rows, j0 = t.j0, j1 = t.j1, len = t.len;
                    const bool t_end = t.end;
                    mbar_arrive(bar(B_TAKEN + n % kWorks));
                    if (rows == 0 && t_end) break;
                    if (rows == 0 || j0 == j1) continue;
                    const bool two = rows > 128;
                    // K of round j is load it + 2 (j - j0), V the one behind it
                    ok = full(it) && mbar_wait_one(bar(B_Q), tiles0++ & 1, waits);
                    if (!ok) break;
                    tc_fence_after();
                    issue_s(0, it % M::kSlots);
                    if (j0 + 1 == j1) tc_commit(bar(B_QFREE));
                    if (two) {
                        ok = mbar_wait_one(bar(B_Q + 1), tiles1++ & 1, waits);
                        if (!ok) break;
                        tc_fence_after();
                        issue_s(1, it % M::kSlots);
                        if (j0 + 1 == j1) tc_commit(bar(B_QFREE + 1));
                    }
                    tc_commit(bar(B_EMPTY + it % M::kSlots));
                    ok = full(it + 1) && (j0 + 1 == j1 || full(it + 2));
                    for (uint32_t j = j0; j < j1 && ok; ++j, it += 2) {
                        const uint32_t sv = (it + 1) % M::kSlots, sk = (it + 2) % M::kSlots;
                        const bool more = j + 1 < j1;
                        const uint32_t steps = min((uint32_t)kKv / 16, (len - j * kKv + 15) / 16);
                        const unsigned long long b = v_desc + ((sv * M::kTile) >> 4);
                        auto weigh = [&](uint32_t m, uint32_t r) {
                            // first the half of the tokens whose weights are written first
#pragma unroll
                            for (uint32_t h = 0; h < 2; ++h) {
                                if (!mbar_wait_one(bar(B_P + 2 * m + h), r & 1, waits)) return false;
                                tc_fence_after();
#pragma unroll
                                for (uint32_t x = h * 4; x < h * 4 + 4; ++x)
                                    if (x < steps) tc_mma_ts(tmem + kO + m * D, tmem + kS + m * 128 + x * 8, b + ((x * 2 * kGroup) >> 4), id_o, j > j0 || x > 0);
                            }
                            if (more) issue_s(m, sk);
                            else tc_commit(bar(B_O + m));
                            if (j + 2 == j1) tc_commit(bar(B_QFREE + m));       // the last products with these query rows
                            return true;
                        };
                        ok = weigh(0, rounds0++);
                        // the next round's V and K: looked at here, where the tensor cores have work in hand (an mbarrier
                        // costs this thread 100 to 250 cycles, and behind the last product they would be idle ones)
                        if (more) ok = ok && full(it + 3) && (j + 2 == j1 || full(it + 4));
                        ok = ok && (!two || weigh(1, rounds1++));
                        if (!ok) break;
                        tc_commit(bar(B_EMPTY + sv));
                        if (more) tc_commit(bar(B_EMPTY + sk));
                    }
                }
                // every product is complete before tensor memory is given back
                tc_commit(bar(B_DONE));
                mbar_land(bar(B_DONE), 0);
            }
            __syncwarp();
        } else {
            // ---------------- tiles, then those that are done once more
            uint32_t n = 0;
            auto give = [&](const Work &t) {
                if (n >= kWorks && !mbar_wait(bar(B_TAKEN + n % kWorks), (n / kWorks - 1) & 1, waits)) return false;
                if (lane == 0) { works[n % kWorks] = t; mbar_arrive(bar(B_WORK + n % kWorks)); }
                __syncwarp();
                n += 1;
                return true;
            };
            Work none = {};
            hand_out<PREFIX, WINDOW>(g, p, true, [](uint32_t) { return true; }, give);
            if (!PREFIX) {
                give(none);
                bar_sync(kRowsBar, kRowsBarThreads);
                if (*(volatile uint32_t *)&any_redo) hand_out<PREFIX, WINDOW>(g, p, false, [&](uint32_t i) { return (redo[i % kRedo / 32] >> (i % 32) & 1) != 0; }, give);
            }
            none.end = true;
            give(none);
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        // ---------------- softmax: warpgroup m, one row per thread
        const uint32_t m = w >> 2, tid = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)(w & 3) << 21;                 // this warp's quarter of the lanes
        const uint32_t ts = tmem + kS + m * 128 + lanes, to = tmem + kO + m * D + lanes;
        // 1e-30: with a scale of 0 masked scores still become 2^-inf
        const float sl2 = fmaxf(fabsf(p.a.scale) * 1.4426950408889634f, 1e-30f);
        const unsigned long long sl22 = pack2(sl2, sl2);
        const uint32_t magic = (0xFFFFFFFFu / p.group) + 1u;            // x / group for x < 2^26
        auto per_group = [&](uint32_t x) { return p.group == 1 ? x : __umulhi(x, magic); };
        // rows of Q in 128-byte swizzle, zeros behind the last
        auto load_q = [&](const Work &t) {
            constexpr uint32_t C = D / 8, R = 128 / C;                 // 16-byte units per row; rows per pass
            const uint32_t c = tid % C;
#pragma unroll
            for (uint32_t x = 0; x < C; ++x) {
                const uint32_t r = tid / C + x * R, y = t.rem0 + m * 128 + r, tok = per_group(y);
                const bool there = m * 128 + r < t.rows;
                const uint8_t *src = p.a.q + (unsigned long long)(t.q0 + t.tok0 + tok) * p.a.qs + ((t.head * p.group + y - tok * p.group) * D + c * 8) * 2;
                cp_async16(base + m * M::kQ + (c >> 3) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4), there ? src : p.a.q, there);
            }
            cp_async_commit();
        };
        auto q_there = [&] {
            cp_async_wait<0>();
            fence_async_smem();
            mbar_arrive(bar(B_Q + m));
        };
        uint32_t rounds = 0, tiles = 0, it = 0;                         // it: loads of the tiles before
        bool ok = true;
        uint32_t n = 0;
        Work t = {};
        // the next tile that has rows for this warpgroup (a short one has none for the second)
        auto advance = [&] {
            for (;; ++n) {
                ok = ok && mbar_wait(bar(B_WORK + n % kWorks), n / kWorks & 1, waits);
                if (!ok) return false;
                t = works[n % kWorks];
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_TAKEN + n % kWorks));
                if (t.rows == 0) { n += 1; return false; }
                if (m * 128 < t.rows) { n += 1; return true; }
                it += 2 * (t.j1 - t.j0);
            }
        };
        bool again = false;
        for (;;) {
            bool have = advance();
            if (have && t.j0 < t.j1 && !p.q_boxes) { load_q(t); q_there(); }
            while (have && ok) {
                const uint32_t y = t.rem0 + m * 128 + tid, tok = per_group(y), token = t.tok0 + tok;
                const bool mine = m * 128 + tid < t.rows;
                const uint32_t qh = t.head * p.group + y - tok * p.group;
                float top = -INFINITY, sum = 0.f;
                // columns of a round up to this one are seen by the row
                const uint32_t sees = PREFIX ? t.len - 1 : t.past + token;
                const uint32_t least = t.past + t.tok0 + per_group(t.rem0 + m * 128);      // what the warpgroup's first row sees
                const uint32_t low = WINDOW && sees >= p.a.window ? sees - p.a.window + 1 : 0u;     // the first token in the row's window
                for (uint32_t j = t.j0; j < t.j1; ++j, ++rounds) {
                    ok = mbar_wait(bar(B_S + m), rounds & 1, waits);
                    if (!ok) break;
                    tc_fence_after();
                    uint32_t u[128];
#pragma unroll
                    for (int c = 0; c < 128; c += 32) tmem_ld32(u + c, ts + c);
                    tmem_wait_ld();
                    float *s = reinterpret_cast<float *>(u);
                    if (!WINDOW && __any_sync(0xFFFFFFFFu, sees < j * kKv + kKv - 1)) {
                        const int lim = sees >= j * kKv ? (int)min(sees - j * kKv, 127u) : -1;
#pragma unroll
                        for (int c = 0; c < 128; ++c) s[c] = c <= lim ? s[c] : -INFINITY;
                    }
                    if (WINDOW && __any_sync(0xFFFFFFFFu, sees < j * kKv + kKv - 1 || (low > j * kKv && low > p.a.sinks))) {
                        // columns up to the row's own, and of them those in its window or among the sinks: a bit each, 32 at a time
                        auto count = [&](uint32_t x) { return x > j * kKv ? (int)min(x - j * kKv, (uint32_t)kKv) : 0; };
                        auto below = [](int x) { return x <= 0 ? 0u : 0xFFFFFFFFu >> (32 - min(x, 32)); };
                        const int seen = count(sees + 1), from = count(low), sinks = count(p.a.sinks);
#pragma unroll
                        for (int c = 0; c < 128; c += 32) {
                            const uint32_t bits = below(seen - c) & (~below(from - c) | below(sinks - c));
#pragma unroll
                            for (int e = 0; e < 32; ++e) s[c + e] = bits >> e & 1 ? s[c + e] : -INFINITY;
                        }
                    }
                    float x0 = s[0], x1 = s[1], x2 = s[2], x3 = s[3];
#pragma unroll
                    for (int c = 4; c < 124; c += 8) {
                        x0 = max3_nan(x0, s[c], s[c + 1]); x1 = max3_nan(x1, s[c + 2], s[c + 3]);
                        x2 = max3_nan(x2, s[c + 4], s[c + 5]); x3 = max3_nan(x3, s[c + 6], s[c + 7]);
                    }
                    x0 = max3_nan(x0, s[124], s[125]); x1 = max3_nan(x1, s[126], s[127]);
                    const float now = max3_nan(max3_nan(x0, x1, x2), x3, x3) * sl2;
                    const bool grow = now > top + 8.f || (top == -INFINITY && now > -INFINITY);
                    if (__any_sync(0xFFFFFFFFu, grow)) {
                        const float f = grow ? exp2_approx(top - now) : 1.f;
                        if (grow) { top = now; sum *= f; }
                        if (j > t.j0) {
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                tmem_ld16(o, to + c);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                tmem_st16(to + c, o);
                            }
                        }
                    }
                    // Tokens of this round that the products run over; of them those of the chain; of them, once more, those that every row here sees.
                    const uint32_t rows = min((uint32_t)kKv, (t.len - j * kKv + 15) / 16 * 16), valid = min(t.held - j * kKv, rows);
                    const uint32_t clear = !again ? valid : WINDOW ? 0u : min(valid, least >= j * kKv ? least - j * kKv + 1 : 0u);
                    if (clear < rows) {
                        // Before this round's weights are announced: V behind the last token of the chain (leftovers of other requests) becomes
                        // zeros, and the second time so does what is not finite in tokens that some rows do not see.
                        const uint32_t x = it + 2 * (j - t.j0) + 1;
                        ok = mbar_wait(bar(B_FULL + x % M::kSlots), (x / M::kSlots) & 1, waits);
                        if (!ok) break;
                        uint8_t *v = smem + M::oRing + (x % M::kSlots) * M::kTile;
                        for (uint32_t y = tid; y < (rows - clear) * (D / 8); y += 128) {
                            const uint32_t c = y % (D / 8), r = clear + y / (D / 8);
                            uint4 *at = reinterpret_cast<uint4 *>(v + (r >> 3) * kGroup + (c >> 3) * 1024 + (r & 7) * 128 + (c & 7) * 16);
                            if (r >= valid) { *at = make_uint4(0, 0, 0, 0); continue; }
                            const uint4 z = *at;
                            if (!T::marked(T::mark(z.x, T::mark(z.y, T::mark(z.z, T::mark(z.w, 0)))))) continue;
                            // The other warpgroup may see this token: it learns from the mark, set before the zero is, that there was something.
                            *(volatile uint32_t *)&marks[n % kMarks] = n;
                            __threadfence_block();
                            *at = make_uint4(T::finite(z.x), T::finite(z.y), T::finite(z.z), T::finite(z.w));
                        }
                        fence_async_smem();
                    }
                    // a NaN among the scores makes the weights NaN (but for those on the multiply-add pipe) and with them the whole row
                    const float sub = now != now ? now : top == -INFINITY ? 0.f : kLift<T> - top;
                    const unsigned long long sub2 = pack2(sub, sub);
                    unsigned long long sum0 = 0, sum1 = 0;
                    // weights of 16 tokens at a time, rounded, to the first registers that are free again
#pragma unroll
                    for (int c = 0; c < 128; c += 16) {
                        float2 e[8];
#pragma unroll
                        for (int y = 0; y < 8; ++y) {
                            const unsigned long long v = fma2(pack2(s[c + 2 * y], s[c + 2 * y + 1]), sl22, sub2);
                            if (kPoly >> y & 1) e[y] = exp2_poly2(v);
                            else { const float2 z = unpack2(v); e[y] = make_float2(exp2_approx(z.x), exp2_approx(z.y)); }
                        }
#pragma unroll
                        for (int y = 0; y < 8; ++y) u[c / 2 + y] = T::pack(e[y].x, e[y].y);
#pragma unroll
                        for (int y = 0; y < 8; y += 4) {
                            sum0 = add2(sum0, add2(pack2(e[y].x, e[y].y), pack2(e[y + 1].x, e[y + 1].y)));
                            sum1 = add2(sum1, add2(pack2(e[y + 2].x, e[y + 2].y), pack2(e[y + 3].x, e[y + 3].y)));
                        }
                        if (c == 48) tmem_st32(ts, u);
                        if (c == kAnnounce) {                    // the store has landed meanwhile
                            tmem_wait_st();
                            tc_fence_before();
                            mbar_arrive(bar(B_P + 2 * m));
                        }
                    }
                    tmem_st32(ts + 32, u + 32);
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(B_P + 2 * m + 1));
                    const float2 z = unpack2(add2(sum0, sum1));
                    sum += z.x + z.y;
                }
                if (!ok) break;
                // ---------------- rows out, while the tensor cores start on the next tile
                const Work d = t;
                const uint32_t count = n;
                it += 2 * (d.j1 - d.j0);
                have = advance();
                if (have && t.j0 < t.j1 && !p.q_boxes) { load_q(t); q_there(); }
                const unsigned long long at = (PREFIX || p.splits > 1)
                    ? ((unsigned long long)d.split * (PREFIX ? p.a.n : p.a.total_q) + d.q0 + token) * p.a.q_heads + qh : 0ull;
                if (d.j0 < d.j1) {
                    ok = mbar_wait(bar(B_O + m), tiles & 1, waits);
                    if (!ok) break;
                    tiles += 1;
                    tc_fence_after();
                }
                if ((PREFIX || p.splits > 1) && mine) p.parts.ml[at] = make_float2(top - kLift<T>, sum);
                if (d.j0 < d.j1) {
                    const float inv = 1.f / sum;
                    uint32_t odd = 0;
                    if (again && *(volatile uint32_t *)&marks[count % kMarks] == count) {
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(o, to + c);
                            tmem_wait_ld();
                            const uint32_t *chain = g.r_chain + (unsigned long long)d.req * g.max_pages;
                            const unsigned long long in_page = (unsigned long long)(p.a.layer * 2 + 1) * g.T * g.row_bytes + ((unsigned long long)d.head * D + c) * 2;
                            if (mine && !WINDOW)        // tokens behind the tile's first row, of this tile's rounds
                                add_not_finite<T>(g, chain, max(d.past + d.tok0 + 1, d.j0 * kKv), min(sees + 1, d.j1 * kKv), in_page, o);
                            if (mine && WINDOW) {       // all that the row sees of this tile's rounds: sinks, and what is in its window
                                const uint32_t from = d.j0 * kKv, end = min(sees + 1, d.j1 * kKv);
                                add_not_finite<T>(g, chain, from, min(end, p.a.sinks), in_page, o);
                                add_not_finite<T>(g, chain, max(from, max(low, p.a.sinks)) + d.shift, end + d.shift, in_page, o);
                            }
                            __syncwarp();
                            tmem_st16(to + c, o);
                        }
                        tmem_wait_st();
                    }
                    // A thread holds a row, and a store of 32 rows costs a cycle each (4000 a tile).  Quads of lanes swap 16-byte units
                    // first: a store then covers 64 bytes of 8 rows.
                    const bool whole = !PREFIX && p.splits == 1;
                    const unsigned long long mine_at = !mine ? 0ull : whole
                        ? reinterpret_cast<unsigned long long>(p.a.out + (unsigned long long)(d.q0 + token) * p.a.os + (unsigned long long)qh * D * 2)
                        : reinterpret_cast<unsigned long long>(p.parts.o + at * D);
                    uint8_t *rows[4];                      // of the quad's four lanes, at this lane's unit; null: no such row
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const unsigned long long x = __shfl_sync(0xFFFFFFFFu, mine_at, (lane & ~3) + r);
                        rows[r] = x ? reinterpret_cast<uint8_t *>(x) + (lane & 3) * 16 : nullptr;
                    }
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o, to + c);
                        tmem_wait_ld();
                        if (whole) {
#pragma unroll
                            for (int e = 0; e < 32; e += 2) {
                                o[e / 2] = T::pack(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv);
                                odd = T::mark(o[e / 2], odd);
                            }
                        } else if (!PREFIX) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) odd |= __float_as_uint(__uint_as_float(o[e]) * 0.f);
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (whole && h) break;
                            uint32_t v[4][4];              // [word][row]
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
#pragma unroll
                                for (int x = 0; x < 4; ++x) v[k][x] = o[h * 16 + x * 4 + k];
                                quad_transpose(v[k]);
                            }
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                if (rows[r]) *reinterpret_cast<uint4 *>(rows[r] + (whole ? c * 2 : (c + h * 16) * 4)) = make_uint4(v[0][r], v[1][r], v[2][r], v[3][r]);
                        }
                        __syncwarp();
                    }
                    if (!PREFIX && !again && mine && T::marked(odd)) {
                        atomicOr(&redo[(count - 1) % kRedo / 32], 1u << ((count - 1) % 32));
                        any_redo = 1;
                    }
                    if (!PREFIX && p.splits == 1 && mine && p.a.lse)
                        p.a.lse[(unsigned long long)(d.q0 + token) * p.a.q_heads + qh] = (top - kLift<T>) * 0.6931471805599453f + logf(sum);
                    tc_fence_before();     // the accumulator has been read: the next weights let products overwrite it
                }
            }
            if (PREFIX || again) break;
            bar_sync(kRowsBar, kRowsBarThreads);
            if (!*(volatile uint32_t *)&any_redo) break;
            again = true;
        }
        cp_async_wait<0>();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (w == 9) tmem_free512(tmem);
    if (threadIdx.x == 0 && waits.over()) record_error(g.st, AVMP_DEV_TIMEOUT);
    if ((w == 8 || w == 10) && waits.over()) {
        // Copies in flight land before this CTA's memory is given away.  K and V have even and odd numbers; a slot that has been filled
        // again had got its earlier copy.
        const uint32_t v = w == 8 ? 0 : 1;
        for (uint32_t x = loads[v] > 2 * M::kSlots + v ? loads[v] - 2 * M::kSlots : v; x < loads[v]; x += 2)
            if (x + M::kSlots >= loads[(x + M::kSlots) & 1]) mbar_land(bar(B_FULL + x % M::kSlots), (x / M::kSlots) & 1);
        for (uint32_t m = 0; m < 2; ++m)
            if (q_loads[m]) mbar_land(bar(B_Q + m), (q_loads[m] - 1) & 1);
    }
}

// Rows of a prompt call whose tokens were split: a warp per (row, query head), eight rows of a tile per CTA.  Maxima and denominators of 32
// parts come by one load, a lane each, and the sums of eight parts are on their way together.  (With a CTA per tile and one
// part at a time 100 rows of 32 heads took 79 us.)
template <class T, int D>
__global__ void __launch_bounds__(256) prompt_join_kernel(const PromptArgs p)
{
    pdl_prologue();
    constexpr uint32_t kGroups = kRows / 8, kFly = 8;
    const uint32_t n = *p.n_tiles * p.a.kv_heads * kGroups, lane = threadIdx.x % 32;
    constexpr int E = D / 32;
    for (uint32_t i = blockIdx.x; i < n; i += gridDim.x) {
        const uint32_t y = i / kGroups, row_in = i % kGroups * 8 + threadIdx.x / 32;
        const Tile t = p.tiles[y / p.a.kv_heads];
        const Item it = p.items[t.k];
        const uint32_t head = y % p.a.kv_heads, rows = min((uint32_t)kRows, it.nq * p.group - t.b * kRows);
        if (row_in >= rows) continue;
        const uint32_t row = t.b * kRows + row_in, qh = head * p.group + row % p.group;
        const unsigned long long at = (unsigned long long)(it.q0 + row / p.group) * p.a.q_heads + qh;
        const unsigned long long step = (unsigned long long)p.a.total_q * p.a.q_heads;
        auto sums = [&](uint32_t s) { return s < p.splits ? p.parts.ml[at + s * step] : make_float2(0.f, 0.f); };
        float2 e = sums(lane);
        float top = e.y != 0.f ? e.x : -INFINITY, den = 0.f, acc[E] = {};
        for (uint32_t s = 32 + lane; s < p.splits; s += 32) { const float2 x = sums(s); if (x.y != 0.f) top = fmaxf(top, x.x); }
#pragma unroll
        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
        for (uint32_t s0 = 0; s0 < p.splits; s0 += 32) {
            if (s0) e = sums(s0 + lane);
            const float f = e.y == 0.f ? 0.f : exp2_approx(e.x - top);
            for (uint32_t b = 0; b < min(32u, p.splits - s0); b += kFly) {
                float v[kFly][E];
#pragma unroll
                for (uint32_t x = 0; x < kFly; ++x) {
                    if (s0 + b + x >= p.splits) continue;
                    const float *from = p.parts.o + (at + (s0 + b + x) * step) * D + lane * E;
                    if (E == 4) { const float4 z = *reinterpret_cast<const float4 *>(from); v[x][0] = z.x; v[x][1] = z.y; v[x][E - 2] = z.z; v[x][E - 1] = z.w; }
                    else { const float2 z = *reinterpret_cast<const float2 *>(from); v[x][0] = z.x; v[x][1] = z.y; }
                }
#pragma unroll
                for (uint32_t x = 0; x < kFly; ++x) {
                    const float ey = __shfl_sync(0xFFFFFFFFu, e.y, b + x), fx = __shfl_sync(0xFFFFFFFFu, f, b + x);
                    if (ey == 0.f) continue;          // an empty part wrote no sums
                    den += ey * fx;
#pragma unroll
                    for (int c = 0; c < E; ++c) acc[c] += fx * v[x][c];
                }
            }
        }
        const float inv = 1.f / den;
        uint8_t *out = p.a.out + (unsigned long long)(it.q0 + row / p.group) * p.a.os + ((unsigned long long)qh * D + lane * E) * 2;
#pragma unroll
        for (int x = 0; x < E; x += 2) *reinterpret_cast<uint32_t *>(out + x * 2) = T::pack(acc[x] * inv, acc[x + 1] * inv);
        if (p.a.lse && lane == 0) p.a.lse[at] = top * 0.6931471805599453f + logf(den);
    }
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

uint32_t box_of(uint32_t T, uint32_t most)
{
    uint32_t b = 8;
    while (b < most && T % (2 * b) == 0) b *= 2;
    return b;
}

// Rows of partial sums that a call may leave.  Splits x row blocks x KV heads never pass the SMs, and a row block has 256 rows.
size_t part_rows(size_t rows, int n_sms) { const size_t full = (size_t)n_sms * kRows; return rows > full ? rows : full; }

template <class T, int D, bool PREFIX, bool WINDOW>
cudaError_t tile_launch(const Geom &g, const PromptArgs &p, uint32_t grid, const Launch &l)
{
    CUtensorMap map;
    if (!row_map(&map, g, p.a.head_dim, p.box_tokens)) return cudaErrorNotSupported;
    const cudaError_t e = allow_smem<attn_tile_kernel<T, D, PREFIX, WINDOW>>(l.device, Smem<D>::kTotal);
    if (e != cudaSuccess) return e;
    CUtensorMap q_map = {};
    PromptArgs a = p;
    const uint32_t rows = PREFIX ? p.a.n : p.a.total_q;
    a.q_boxes = (p.group & (p.group - 1)) == 0 && rows &&
                query_map(&q_map, p.a.q, p.a.head_dim, p.a.q_heads, rows, p.a.qs, 128 / p.group, p.group);
    return launch_pdl(attn_tile_kernel<T, D, PREFIX, WINDOW>, dim3(grid), dim3(kCta), Smem<D>::kTotal, l.stream, g, a, map, q_map);
}
template <bool PREFIX, bool WINDOW = false>
cudaError_t tile_type(const Geom &g, const PromptArgs &p, uint32_t grid, const Launch &l)
{
    if (p.a.head_dim == 128) return p.a.f16 ? tile_launch<F16, 128, PREFIX, WINDOW>(g, p, grid, l) : tile_launch<Bf16, 128, PREFIX, WINDOW>(g, p, grid, l);
    return p.a.f16 ? tile_launch<F16, 64, PREFIX, WINDOW>(g, p, grid, l) : tile_launch<Bf16, 64, PREFIX, WINDOW>(g, p, grid, l);
}
template <class T>
cudaError_t join_type(const PromptArgs &p, uint32_t grid, const Launch &l)
{
    return p.a.head_dim == 128 ? launch_pdl(prompt_join_kernel<T, 128>, dim3(grid), dim3(256), 0, l.stream, p)
                               : launch_pdl(prompt_join_kernel<T, 64>, dim3(grid), dim3(256), 0, l.stream, p);
}

// As many shares of the KV tokens as leave every SM a tile.
uint32_t split_of(unsigned long long tiles, int n_sms)
{
    return tiles >= (unsigned long long)n_sms ? 1u : (uint32_t)(n_sms / (tiles ? tiles : 1));
}

}  // namespace

cudaError_t launch_attn_prefix(const Geom &g, const AttnArgs &a, const Launch &l, Parts *out, uint32_t *parts)
{
    PromptArgs p = {};
    p.a = a;
    p.group = a.q_heads / a.kv_heads;
    p.prefix_blocks = (uint32_t)(((unsigned long long)a.n * p.group + kRows - 1) / kRows);
    const unsigned long long tiles = (unsigned long long)p.prefix_blocks * a.kv_heads;
    p.splits = split_of(tiles, l.n_sms);
    p.box_tokens = box_of(g.T, kKv);
    const size_t rows = (size_t)p.splits * a.n * a.q_heads;
    p.parts.ml = reinterpret_cast<float2 *>(a.ws);
    p.parts.o = reinterpret_cast<float *>(a.ws + up256(rows * 8));
    *out = p.parts;
    *parts = p.splits;
    return tile_type<true>(g, p, (uint32_t)min(tiles * p.splits, (unsigned long long)l.n_sms), l);
}

size_t attn_tile_ws_bytes(const Geom &g, uint32_t n, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim, int n_sms)
{
    // tiles: no request has more query rows than it can hold tokens
    const size_t cap = (size_t)n * (((size_t)g.max_pages * g.T * (q_heads / kv_heads) + kRows - 1) / kRows);
    return 256 + up256(cap * sizeof(Tile)) + up256((size_t)n * sizeof(Item)) + part_rows((size_t)n * q_heads, n_sms) * ((size_t)head_dim * 4 + 8) + 512;
}

cudaError_t launch_attn_prompt(const Geom &g, const AttnArgs &a, const Launch &l, uint32_t *launched)
{
    PromptArgs p = {};
    p.a = a;
    p.group = a.q_heads / a.kv_heads;
    p.box_tokens = box_of(g.T, a.window ? 32 : kKv);        // (with a window: what is read beside it is less than a box)
    const unsigned long long full = (unsigned long long)a.n * (((unsigned long long)g.max_pages * g.T * p.group + kRows - 1) / kRows);
    const unsigned long long most = (unsigned long long)a.total_q * p.group / kRows + a.n;      // row blocks of the buffers' rows
    p.cap = (uint32_t)min(full, most);
    p.splits = split_of(most * a.kv_heads, l.n_sms);           // (parts lie by row of the buffers: see part_rows)
    if (a.window) {      // no more than a tile has rounds: those of its rows' windows and of the sinks, each with two ends that need not be at a round's
        const unsigned long long rounds = ((unsigned long long)a.window + kRows) / kKv + a.sinks / kKv + 4;
        if (p.splits > rounds) p.splits = (uint32_t)rounds;
    }
    uint8_t *w = a.ws;
    p.n_tiles = reinterpret_cast<uint32_t *>(w); w += 256;
    p.tiles = reinterpret_cast<Tile *>(w); w += up256((size_t)full * sizeof(Tile));
    p.items = reinterpret_cast<Item *>(w); w += up256((size_t)a.n * sizeof(Item));
    const size_t rows = (size_t)p.splits * a.total_q * a.q_heads;
    p.parts.ml = reinterpret_cast<float2 *>(w);
    p.parts.o = reinterpret_cast<float *>(w + up256(rows * 8));
    cudaError_t e = cudaSuccess;
    if (a.n <= 32 && p.splits == 1) {
        p.tiles = nullptr;                 // the tile kernel plans for itself
    } else {
        e = launch_pdl(prompt_plan_kernel, dim3(1), dim3(kStepThreads), 0, l.stream, g, p);
        if (e != cudaSuccess) return e;
        *launched += 1;
    }
    const unsigned long long tiles = (unsigned long long)p.cap * a.kv_heads * p.splits;
    const uint32_t grid = (uint32_t)min(tiles, (unsigned long long)l.n_sms);
    e = a.window ? tile_type<false, true>(g, p, grid, l) : tile_type<false>(g, p, grid, l);
    if (e != cudaSuccess) return e;
    *launched += 1;
    if (p.splits > 1) {
        const uint32_t joins = (uint32_t)min((unsigned long long)p.cap * a.kv_heads * (kRows / 8), 8ull * l.n_sms);
        e = a.f16 ? join_type<F16>(p, joins, l) : join_type<Bf16>(p, joins, l);
        *launched += 1;
    }
    return e;
}

}  // namespace avmp
