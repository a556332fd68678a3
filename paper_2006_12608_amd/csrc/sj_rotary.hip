// sj_rotary.hip -- rotary positions (sj_rotary) and rows appended to a cache
// (sj_cache_append): pair i of a head turned by pos * f_i, with f_i in turns of
// 2^-64 so that the phase of any position is one 64-bit product.
#include "sj_cache.h"

namespace sjc {

namespace {

constexpr uint32_t RO_PAIRS = 256;   // sines kept per workgroup at most (tokens x pairs)

struct RotaryArgs {
    Rotary r;
    uint32_t tokens;          // of one workgroup
    uint64_t n;               // batch * t
    uint32_t turned;          // 16-byte pair chunks of a head: ceil(pairs / 8)
    uint32_t q_rest, k_rest;  // 8-element chunks of a head past the pairs, copied
    uint32_t q_items, k_items, items;  // (head, chunk) items of a token: queries, keys, all
    PageDiv by_items, by_q, by_k, by_v, by_t, by_pairs;
};

__device__ __forceinline__ float to_float(int dt, uint32_t x)
{
    return dt == sjk::DT_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)x)
                             : __uint_as_float(x << 16);
}

__device__ __forceinline__ uint32_t to_bits(int dt, float x)
{
    return dt == sjk::DT_F16 ? (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x)
                             : (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x);
}

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
            const uint32_t x = to_bits(DT, a * c - b * s), y = to_bits(DT, b * c + a * s);
            lo[w] = (int)(((uint32_t)lo[w] & ~(0xffffu << sh)) | (x << sh));
            hi[w] = (int)(((uint32_t)hi[w] & ~(0xffffu << sh)) | (y << sh));
        } else {
            i32x4 &v = p < 4 ? lo : hi;
            const uint32_t w = (uint32_t)v[p & 3];
            const float a = to_float(DT, w & 0xffffu), b = to_float(DT, w >> 16);
            v[p & 3] = (int)(to_bits(DT, a * c - b * s) | (to_bits(DT, b * c + a * s) << 16));
        }
    }
}

// A workgroup takes `tokens` tokens: it computes their sines once for all heads (LDS),
// then its threads run over the tokens' (head, chunk of 16 elements) items.
// Bound by HBM (each element read and written once).
template <int DT, bool HALF>
__global__ void __launch_bounds__(256) rotary_rows(const RotaryArgs g)
{
    __shared__ float2 table[RO_PAIRS + 8];
    const Rotary &r = g.r;
    const uint32_t pairs = r.turn.pairs, stride = 8 * g.turned;
    const uint64_t tok0 = (uint64_t)blockIdx.x * g.tokens;
    const uint32_t mine = g.n - tok0 < g.tokens ? (uint32_t)(g.n - tok0) : g.tokens;
    for (uint32_t i = threadIdx.x; i < mine * stride; i += 256) {
        const uint32_t u = g.by_pairs.quot(i), p = i - u * stride;
        if (p < pairs) {
            const uint64_t phase =
                (uint64_t)(int64_t)r.turn.pos[tok0 + u] * (uint64_t)r.turn.turns[p];
            // signed fraction of a turn; 2^-31 half turns a unit
            const float half = (float)(int32_t)(phase >> 32) * 4.656612873077393e-10f;
            float s, c;
            sincospif(half, &s, &c);
            table[i] = float2{c * r.turn.factor, (r.turn.inverse ? -s : s) * r.turn.factor};
        }
    }
    __syncthreads();
    const uint32_t d = r.d, rot = 2 * pairs;
    for (uint32_t i = threadIdx.x; i < mine * g.items; i += 256) {
        const uint32_t u = g.by_items.quot(i);
        uint32_t x = i - u * g.items;
        const uint64_t tok = tok0 + u;
        const uint32_t b = g.by_t.quot((uint32_t)tok), w = (uint32_t)tok - b * r.t;
        const uint16_t *in;
        uint16_t *out;
        uint32_t chunk;
        bool copy = false;      // values pass unturned
        if (x < g.q_items) {
            const uint32_t head = g.by_q.quot(x);
            chunk = x - head * (g.turned + g.q_rest);
            in = r.x.in + (int64_t)b * r.x.in_seq + (int64_t)w * r.x.in_tok + (int64_t)head * r.x.in_head;
            out = r.x.out + (int64_t)b * r.x.out_seq + (int64_t)w * r.x.out_tok +
                  (int64_t)head * r.x.out_head;
        } else {
            x -= g.q_items;
            const uint32_t count = r.count ? clamp_rows(r.count[b], r.t) : r.t;
            const uint64_t n = (uint64_t)clamp_rows(r.len[b], r.c.room) + w;
            if (w >= count || n >= r.c.room)
                continue;
            const Place p = place_of(r.c, b, (uint32_t)n);
            if (p.page < 0)
                continue;
            if (x < g.k_items) {
                const uint32_t head = g.by_k.quot(x);
                chunk = x - head * (g.turned + g.k_rest);
                in = r.key.in + (int64_t)b * r.key.in_seq + (int64_t)w * r.key.in_tok +
                     (int64_t)head * r.key.in_head;
                out = const_cast<uint16_t *>(r.c.k) + (int64_t)p.page * r.c.k_page +
                      (int64_t)p.slot * r.c.k_row + (int64_t)head * r.c.k_head;
            } else {
                x -= g.k_items;
                const uint32_t head = g.by_v.quot(x);
                chunk = x - head * g.by_v.page;
                copy = true;
                in = r.value.in + (int64_t)b * r.value.in_seq + (int64_t)w * r.value.in_tok +
                     (int64_t)head * r.value.in_head;
                out = const_cast<uint16_t *>(r.c.v) + (int64_t)p.page * r.c.v_page +
                      (int64_t)p.slot * r.c.v_row + (int64_t)head * r.c.v_head;
            }
        }
        if (copy || chunk >= g.turned) {
            const uint32_t at = copy ? 8 * chunk : rot + 8 * (chunk - g.turned);
            store8(out + at, load8(in + at, (int)(d - at)), (int)(d - at));
            continue;
        }
        const uint32_t p0 = 8 * chunk;
        const int np = (int)(pairs - p0 < 8 ? pairs - p0 : 8);
        const uint32_t at_lo = HALF ? p0 : 2 * p0, at_hi = HALF ? pairs + p0 : 2 * p0 + 8;
        const int n_lo = HALF ? np : 2 * np, n_hi = HALF ? np : 2 * np - 8;
        i32x4 lo = load8(in + at_lo, n_lo), hi = load8(in + at_hi, n_hi);
        turn8<DT, HALF>(lo, hi, table + u * stride + p0);
        store8(out + at_lo, lo, n_lo);
        store8(out + at_hi, hi, n_hi);
    }
}

}  // namespace

hipError_t launch_rotary(const Rotary &r, hipStream_t s)
{
    RotaryArgs g{};
    g.r = r;
    g.n = (uint64_t)r.batch * r.t;
    const uint32_t pairs = r.turn.pairs, d = r.d, rest = (d - 2 * pairs + 7) / 8;
    g.turned = (pairs + 7) / 8;
    const bool in_place = r.x.in == r.x.out;
    g.q_rest = in_place ? 0 : rest;
    g.k_rest = rest;
    const uint32_t q_chunks = g.turned + g.q_rest, k_chunks = g.turned + g.k_rest;
    g.q_items = r.x.heads * q_chunks;
    g.k_items = r.c.batch ? r.c.heads * k_chunks : 0;
    const uint32_t v_chunks = (d + 7) / 8;
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
    // far as 1024 workgroups remain and the sines fit (8 x 2048 tokens of 608 items:
    // 105 us with one token, 101 with two; 5000 of 96: 9.2 us with one, 7.4 with five).
    g.tokens = 1;
    uint32_t best = 0;
    for (uint32_t t = 1; t <= 8 && (t == 1 || (g.n / t >= 1024 && t * 8 * g.turned <= RO_PAIRS)); ++t) {
        const uint32_t full = t * g.items * 100 / ((t * g.items + 255) / 256 * 256);
        if (full > best) {
            best = full;
            g.tokens = t;
        }
        if (full >= 90)
            break;
    }
    const dim3 grid((uint32_t)((g.n + g.tokens - 1) / g.tokens));
    const bool half = r.turn.layout == 0;
    if (r.dtype == sjk::DT_F16) {
        if (half)
            rotary_rows<sjk::DT_F16, true><<<grid, 256, 0, s>>>(g);
        else
            rotary_rows<sjk::DT_F16, false><<<grid, 256, 0, s>>>(g);
    } else {
        if (half)
            rotary_rows<sjk::DT_BF16, true><<<grid, 256, 0, s>>>(g);
        else
            rotary_rows<sjk::DT_BF16, false><<<grid, 256, 0, s>>>(g);
    }
    return hipGetLastError();
}

}  // namespace sjc
