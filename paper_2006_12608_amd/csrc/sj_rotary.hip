// sj_rotary.hip -- rotary positions (sj_rotary) and rows appended to a cache
// (sj_cache_append): pair i of a head turned by pos * f_i, with f_i in turns of
// 2^-64 so that the phase of any position is one 64-bit product.
#include "sj_cache.h"
#include "sj_turn.h"

namespace sjc {

namespace {

constexpr uint32_t RO_PAIRS = 256;   // sines kept per workgroup at most (tokens x pairs)
constexpr uint32_t RO_TOKENS = 8;    // tokens of a workgroup at most
constexpr uint64_t RO_GRID = 1u << 22;   // workgroups of a launch at most (one holds fewer
                                         // than 2^32 threads)

struct RotaryArgs {
    Rotary r;
    uint32_t tokens;          // of one workgroup
    uint64_t first, n;        // first token of the launch; batch * t
    uint32_t turned;          // 16-byte pair chunks of a head: ceil(pairs / 8)
    uint32_t q_rest, k_rest;  // 16-element chunks of a head past the pairs, copied
    uint32_t q_items, k_items, items;  // (head, chunk) items of a token: queries, keys, all
    PageDiv by_items, by_q, by_k, by_v, by_t, by_pairs;
};

// One 8-pair chunk: lo and hi hold its 16 elements, (a_0 .. a_7) and (b_0 .. b_7) in the
// half layout, (a_0, b_0, a_1, ..) in the interleaved one.
template <int DT, bool HALF>
__device__ __forceinline__ void turn8(i32x4 &lo, i32x4 &hi, const float2 *cs)
{
#pragma unroll
    for (int p = 0; p < 8; ++p) {
        const float c = cs[p].x, s = cs[p].y;
        if constexpr (HALF) {
            const int w = p >> 1, sh = 16 * (p & 1);
            const float a = to_float(DT, ((uint32_t)lo[w] >> sh) & 0xffffu);
            const float b = to_float(DT, ((uint32_t)hi[w] >> sh) & 0xffffu);
            const uint32_t x = to_bits(DT, turn_a(a, b, c, s)), y = to_bits(DT, turn_b(a, b, c, s));
            lo[w] = (int)(((uint32_t)lo[w] & ~(0xffffu << sh)) | (x << sh));
            hi[w] = (int)(((uint32_t)hi[w] & ~(0xffffu << sh)) | (y << sh));
        } else {
            i32x4 &v = p < 4 ? lo : hi;
            const uint32_t w = (uint32_t)v[p & 3];
            const float a = to_float(DT, w & 0xffffu), b = to_float(DT, w >> 16);
            v[p & 3] = (int)(to_bits(DT, turn_a(a, b, c, s)) | (to_bits(DT, turn_b(a, b, c, s)) << 16));
        }
    }
}

// Two times eight elements of a head on their way: a chunk of eight pairs, or 16 elements
// that pass unturned.
struct Item {
    i32x4 lo, hi;
};

// A workgroup takes `tokens` tokens: it computes their sines and their rows' places in the
// cache once for all heads (LDS), then its threads run over the tokens' (head, 16 elements)
// items, the next item's loads issued before the present one is stored and the first ones
// before the sines.  EXACT: no item has a partial chunk; a last one that would be partial is
// moved back onto its neighbour, and both write the same (16384 x 32 heads of 128, 100 of them
// turned: 66 -> 45 us; not where the rows are turned in place).
// Bound by HBM (each element read and written once): 268 MB of bf16 in 41 us, 403 MB of prompt
// tokens with their queries in 82 (101 when each item looked its place up and loaded after
// the sines; a large copy moves 4.9 TB/s).
template <int DT, bool HALF, bool EXACT>
__global__ void __launch_bounds__(256) rotary_rows(const RotaryArgs g)
{
    __shared__ float2 table[RO_PAIRS + 8];
    __shared__ Place place[RO_TOKENS];
    const Rotary &r = g.r;
    const uint32_t pairs = r.turn.pairs, stride = 8 * g.turned, d = r.d, rot = 2 * pairs;
    const uint64_t tok0 = g.first + (uint64_t)blockIdx.x * g.tokens;
    const uint32_t mine = g.n - tok0 < g.tokens ? (uint32_t)(g.n - tok0) : g.tokens;
    const uint32_t n_items = mine * g.items;

    // item i: its token of the workgroup, tensor (0 queries, 1 keys, 2 values), head and chunk
    struct Which {
        uint32_t u, b, w, kind, head, chunk;
    };
    auto which = [&](uint32_t i) -> Which {
        Which k;
        k.u = g.by_items.quot(i);
        uint32_t x = i - k.u * g.items;
        const uint32_t tok = (uint32_t)tok0 + k.u;
        k.b = g.by_t.quot(tok);
        k.w = tok - k.b * r.t;
        if (x < g.q_items) {
            k.kind = 0;
            k.head = g.by_q.quot(x);
            k.chunk = x - k.head * (g.turned + g.q_rest);
        } else if ((x -= g.q_items) < g.k_items) {
            k.kind = 1;
            k.head = g.by_k.quot(x);
            k.chunk = x - k.head * (g.turned + g.k_rest);
        } else {
            x -= g.k_items;
            k.kind = 2;
            k.head = g.by_v.quot(x);
            k.chunk = x - k.head * g.by_v.page;
        }
        return k;
    };
    // first elements of an item's two chunks and how many of each exist
    struct Span {
        uint32_t lo, hi, p0;    // (and the first of the pairs)
        int n_lo, n_hi;
    };
    auto turns = [&](const Which &k) { return k.kind < 2 && k.chunk < g.turned; };
    auto span = [&](const Which &k) -> Span {
        Span e;
        if (turns(k)) {
            uint32_t p0 = 8 * k.chunk;
            if (EXACT && p0 + 8 > pairs)
                p0 = pairs - 8;
            const int np = (int)(pairs - p0 < 8 ? pairs - p0 : 8);
            e.lo = HALF ? p0 : 2 * p0;
            e.hi = HALF ? pairs + p0 : 2 * p0 + 8;
            e.p0 = p0;
            e.n_lo = HALF ? np : 2 * np;
            e.n_hi = HALF ? np : 2 * np - 8;
        } else {
            e.lo = k.kind == 2 ? 16 * k.chunk : rot + 16 * (k.chunk - g.turned);
            if (EXACT && e.lo + 16 > d)
                e.lo = d - 16;
            e.p0 = 0;
            e.hi = e.lo + 8;
            e.n_lo = (int)(d - e.lo);
            e.n_hi = e.n_lo - 8;
        }
        if (EXACT)
            e.n_lo = e.n_hi = 8;
        return e;
    };
    auto load = [&](uint32_t i) -> Item {
        const Which k = which(i);
        const Span e = span(k);
        const Strided &t = k.kind == 0 ? r.x : (k.kind == 1 ? r.key : r.value);
        const uint16_t *in = t.in + (int64_t)k.b * t.in_seq + (int64_t)k.w * t.in_tok +
                             (int64_t)k.head * t.in_head;
        return {load8(in + e.lo, e.n_lo), load8(in + e.hi, e.n_hi)};
    };
    auto finish = [&](uint32_t i, Item v) {
        const Which k = which(i);
        const Span e = span(k);
        uint16_t *out;
        if (k.kind == 0) {
            out = r.x.out + (int64_t)k.b * r.x.out_seq + (int64_t)k.w * r.x.out_tok +
                  (int64_t)k.head * r.x.out_head;
        } else {
            const Place p = place[k.u];
            if (p.page < 0)
                return;
            out = k.kind == 1 ? const_cast<uint16_t *>(r.c.k) + (int64_t)p.page * r.c.k_page +
                                    (int64_t)p.slot * r.c.k_row + (int64_t)k.head * r.c.k_head
                              : const_cast<uint16_t *>(r.c.v) + (int64_t)p.page * r.c.v_page +
                                    (int64_t)p.slot * r.c.v_row + (int64_t)k.head * r.c.v_head;
        }
        if (turns(k))
            turn8<DT, HALF>(v.lo, v.hi, table + k.u * stride + e.p0);
        store8(out + e.lo, v.lo, e.n_lo);
        store8(out + e.hi, v.hi, e.n_hi);
    };

    uint32_t i = threadIdx.x;
    Item cur = load(i < n_items ? i : 0);
    const uint32_t last = 255 - threadIdx.x;    // (the first waves have the sines)
    if (g.k_items && last < mine) {
        const uint32_t tok = (uint32_t)tok0 + last;
        const uint32_t b = g.by_t.quot(tok), w = tok - b * r.t;
        const uint32_t count = r.count ? clamp_rows(r.count[b], r.t) : r.t;
        const uint64_t n = (uint64_t)clamp_rows(r.len[b], r.c.room) + w;
        Place p = {-1, 0u};
        if (w < count && n < r.c.room)
            p = place_of(r.c, b, (uint32_t)n);
        place[last] = p;
    }
    for (uint32_t y = threadIdx.x; y < mine * stride; y += 256) {
        const uint32_t u = g.by_pairs.quot(y), p = y - u * stride;
        if (p < pairs) {
            table[y] = sine_of(r.turn, (uint64_t)(int64_t)r.turn.pos[tok0 + u], p);
        }
    }
    __syncthreads();
    if (i >= n_items)
        return;
    for (; i + 256 < n_items; i += 256) {
        const Item nxt = load(i + 256);
        finish(i, cur);
        cur = nxt;
    }
    finish(i, cur);
}

template <int DT>
void launch_rows(const RotaryArgs &g, dim3 grid, bool half, bool exact, hipStream_t s)
{
    if (half)
        (exact ? rotary_rows<DT, true, true> : rotary_rows<DT, true, false>)<<<grid, 256, 0, s>>>(g);
    else
        (exact ? rotary_rows<DT, false, true> : rotary_rows<DT, false, false>)<<<grid, 256, 0, s>>>(g);
}

}  // namespace

hipError_t launch_rotary(const Rotary &r, hipStream_t s)
{
    RotaryArgs g{};
    g.r = r;
    g.n = (uint64_t)r.batch * r.t;
    const uint32_t pairs = r.turn.pairs, d = r.d, rest = (d - 2 * pairs + 15) / 16;
    g.turned = (pairs + 7) / 8;
    const bool in_place = r.x.heads && r.x.in == r.x.out;
    g.q_rest = in_place ? 0 : rest;
    g.k_rest = rest;
    const uint32_t q_chunks = g.turned + g.q_rest, k_chunks = g.turned + g.k_rest;
    g.q_items = r.x.heads * q_chunks;
    g.k_items = r.c.batch ? r.c.heads * k_chunks : 0;
    const uint32_t v_chunks = (d + 15) / 16;
    g.items = g.q_items + g.k_items + (r.c.batch ? r.c.heads * v_chunks : 0);
    if (g.n == 0 || g.items == 0)
        return hipSuccess;
    auto by = [](uint32_t x) { return PageDiv::of(x ? x : 1); };
    g.by_items = by(g.items);
    g.by_q = by(q_chunks);
    g.by_k = by(k_chunks);
    g.by_v = by(v_chunks);
    g.by_t = by(r.t);
    g.by_pairs = by(8 * g.turned);
    // Tokens of a workgroup: the fewest whose items fill its rounds of 256 threads to 90%, as
    // far as 1024 workgroups remain and the sines fit (5000 tokens of 72 items: 10.0 us with
    // one token, 7.0 with three; 8 x 2048 of 384: 82 with one or two).
    g.tokens = 1;
    uint32_t best = 0;
    for (uint32_t t = 1; t <= RO_TOKENS && (t == 1 || (g.n / t >= 1024 && t * 8 * g.turned <= RO_PAIRS)); ++t) {
        const uint32_t full = t * g.items * 100 / ((t * g.items + 255) / 256 * 256);
        if (full > best) {
            best = full;
            g.tokens = t;
        }
        if (full >= 90)
            break;
    }
    const uint32_t passed = d - 2 * pairs;
    const bool exact = (pairs % 8 == 0 || (pairs > 8 && !in_place)) &&
                       (passed % 16 == 0 || passed > 16) && (d % 16 == 0 || d > 16);
    hipError_t e = hipSuccess;
    for (; g.first < g.n && e == hipSuccess; g.first += RO_GRID * g.tokens) {
        const uint64_t groups = (g.n - g.first + g.tokens - 1) / g.tokens;
        const dim3 grid((uint32_t)(groups < RO_GRID ? groups : RO_GRID));
        if (r.dtype == sjk::DT_F16)
            launch_rows<sjk::DT_F16>(g, grid, r.turn.layout == 0, exact, s);
        else
            launch_rows<sjk::DT_BF16>(g, grid, r.turn.layout == 0, exact, s);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sjc
