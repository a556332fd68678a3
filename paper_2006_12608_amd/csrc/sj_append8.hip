// sj_append8.hip -- rows appended to a cache in 8 bits (sj_cache8_append): keys turned, and keys
// and values rounded to e4m3 at a power of two for each block of rows and head.
#include "sj_cache.h"
#include "sj_turn.h"

namespace sjc {

namespace {

constexpr uint32_t A8_GRID = 1u << 22;  // workgroups of a launch at most
// 16-byte chunks of a block that a lane holds (fewer where it turns them: with 8 the kernel needs all
// registers, and 8 x 2048 tokens of 8 heads of 128 take 97 us)
constexpr int held_chunks(bool turn) { return turn ? 4 : 8; }

struct Append8Args {
    Append8 r;
    uint64_t first;             // of the launch's workgroups
    PageDiv by_lanes;           // lanes of a row: d / 8
    uint32_t step1, step4;      // rows that a wave, and four, have lanes for
    uint32_t units, groups;     // heads x {k, v}; workgroups for them
    uint32_t each;              // of a wave, one after the other
    PageDiv by_blocks, by_groups, by_pairs;
};

template <int DT>
struct Type8;
template <>
struct Type8<sjk::DT_F16> {
    static constexpr uint32_t INF = 0x7c00u;
    static constexpr int LEAST = -15, MOST = 7;
};
template <>
struct Type8<sjk::DT_BF16> {
    static constexpr uint32_t INF = 0x7f80u;
    static constexpr int LEAST = -117, MOST = 119;
};

// The least e with x <= 448 2^e = 1.75 2^(e + 8), for a value of the 16-bit type, in its range.
template <int DT>
__device__ __forceinline__ int exponent_of(float x)
{
    const uint32_t u = __float_as_uint(x);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < Type8<DT>::LEAST ? Type8<DT>::LEAST : (e > Type8<DT>::MOST ? Type8<DT>::MOST : e);
}

// 2^e, -126 <= e <= 127.
__device__ __forceinline__ float power(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// 2^-e, -127 <= e <= 127 (2^-127 is subnormal).
__device__ __forceinline__ float power_less(int e) { return e < 127 ? power(-e) : 0x1p-127f; }

// x between e4m3's least and largest values, -448 and 448, or NaN where it is not finite.
__device__ __forceinline__ float bound(float x, bool finite)
{
    return finite ? fminf(fmaxf(x, -448.f), 448.f) : __uint_as_float(0x7fc00000u);
}

// Four values rounded to e4m3, ties to even, in the bytes of a word.
__device__ __forceinline__ uint32_t four(float a, float b, float c, float d)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Eight elements of a key row from element c on, turned and rounded to the 16-bit type.  The partner of
// an element is `pairs`, a multiple of 8, elements on or back (HALF), or beside it; x cos -+ partner sin
// is turn_a and turn_b, as they round.
template <int DT, bool HALF>
__device__ __forceinline__ i32x4 turned8(uint32_t pairs, const uint16_t *row, i32x4 v, uint32_t c,
                                         const float2 *sines)
{
    const uint32_t rot = 2 * pairs;
    if (c >= rot)
        return v;
    i32x4 w = v;
    if (HALF)
        w = load8(c < pairs ? row + c + pairs : row + c - pairs, 8);
#pragma unroll
    for (uint32_t e = 0; e < 8; ++e) {
        const uint32_t i = c + e, sh = 16 * (e & 1), sw = HALF ? sh : 16 - sh;
        const bool first = HALF ? c < pairs : (e & 1) == 0;
        const uint32_t at = HALF ? (first ? i : i - pairs) : i >> 1;
        const float2 cs = sines[HALF || at < pairs ? at : 0];
        const float x = to_float(DT, ((uint32_t)v[e >> 1] >> sh) & 0xffffu);
        const float y = to_float(DT, ((uint32_t)(HALF ? w : v)[e >> 1] >> sw) & 0xffffu) * cs.y;
        const uint32_t z = to_bits(DT, __builtin_fmaf(x, cs.x, first ? -y : y));
        // (w at e has been read: it takes the result)
        const uint32_t r = HALF || i < rot ? z : ((uint32_t)v[e >> 1] >> sh) & 0xffffu;
        w[e >> 1] = (int)(((uint32_t)w[e >> 1] & ~(0xffffu << sh)) | (r << sh));
    }
    return w;
}

// A wave (or all four of a workgroup, where a block has more chunks than its lanes hold: 2 x 1184 tokens
// in blocks of 64 rows of 256, 17 -> 6 us) takes one block of a sequence's rows, one head, keys or
// values: the largest magnitude of the new rows in it (a maximum of 16-bit integers), from that
// the exponent, the rows before len[b] rounded to it where it grows, and the new rows' e4m3
// values.  Sines are computed once for the workgroup's heads, into LDS.  Bound by HBM (2 bytes in, 1
// out: 8 x 2048 tokens of 8 heads of 128, 101 MB, in 23 us), for a token or two by the chain
// lengths, page, exponent, rows.
// TURN: keys are turned in halves (1) or adjacent pairs (2).
template <int DT, int TURN, uint32_t WAVES>
__global__ void __launch_bounds__(256, 4) append8_blocks(const Append8Args g)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    constexpr int HELD = held_chunks(TURN != 0);
    __shared__ float2 sines[TURN != 0 ? A8_SINES : 1];
    const Append8 &r = g.r;
    const uint32_t tid = threadIdx.x & (64 * WAVES - 1);    // of the unit's threads
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t id = (uint32_t)(g.first + blockIdx.x);
    const uint32_t bj = g.by_groups.quot(id), first_unit = (id - bj * g.groups) * g.each * (4 / WAVES);
    const uint32_t b = g.by_blocks.quot(bj), j = bj - b * r.blocks;
    const uint32_t d = r.c.d, size = r.c.by_block.page, pairs = r.turn.pairs;
    const uint32_t len = clamp_rows(r.len[b], r.c.room);
    const uint32_t count = r.count ? clamp_rows(r.count[b], r.t) : r.t;
    const uint64_t all = (uint64_t)len + count;
    const uint32_t end = all < r.c.room ? (uint32_t)all : r.c.room;
    // (blocks do not cross pages, so a sequence's blocks are those of its rows)
    const uint64_t row0 = ((uint64_t)r.c.by_block.quot(len) + j) * size;
    // (a sequence that appends nothing writes nothing: its page may be another one's by now)
    if (row0 >= end || len >= end)
        return;
    const Place p = place_of(r.c, b, (uint32_t)row0);
    if (p.page < 0)
        return;
    const uint32_t from = len > row0 ? len - (uint32_t)row0 : 0;    // slots of the block
    const uint32_t to = end - (uint32_t)row0 < size ? end - (uint32_t)row0 : size;
    // (as many rows side by side as fit in the threads; those left over do nothing)
    const uint32_t sub = g.by_lanes.quot(tid), c = 8 * (tid - sub * g.by_lanes.page);
    const uint32_t step = WAVES == 1 ? g.step1 : g.step4;
    const int left = sub < step ? (int)d - (int)c : 0;
    if constexpr (TURN != 0) {      // (a block's rows x pairs fit)
        for (uint32_t y = threadIdx.x; y < (to - from) * pairs; y += 256) {
            const uint32_t s = g.by_pairs.quot(y);
            const uint32_t u = (uint32_t)row0 + from + s - len;
            sines[y] = sine_of(r.turn, (uint64_t)(int64_t)r.turn.pos[(uint64_t)b * r.t + u], y - s * pairs);
        }
        __syncthreads();
    }
#pragma unroll 1
    for (uint32_t z = 0; z < (TURN != 0 ? g.each : 1); ++z) {
        const uint32_t unit = first_unit + z * (4 / WAVES) + wave / WAVES;
        if (unit >= g.units)
            return;
        const uint32_t h = unit >> 1, kv = unit & 1;
        const Strided &x = kv ? r.value : r.key;
        const int64_t page_s = kv ? r.c.v_page : r.c.k_page, row_s = kv ? r.c.v_row : r.c.k_row;
        uint8_t *out = (uint8_t *)(kv ? r.c.v : r.c.k) + (int64_t)p.page * page_s +
                       (int64_t)p.slot * row_s + (int64_t)h * (kv ? r.c.v_head : r.c.k_head);
        const uint16_t *in = x.in + (int64_t)b * x.in_seq + (int64_t)h * x.in_head;
        int8_t *at = (int8_t *)r.c.ex +
                     2 * (((int64_t)p.page * r.c.blocks + r.c.by_block.quot(p.slot)) * r.c.heads + h) + kv;
        const int was = *at;

        auto get = [&](uint32_t s) -> i32x4 {       // eight elements of slot s, from < = s < to
            const uint32_t u = (uint32_t)row0 + s - len;
            const uint16_t *row = in + (int64_t)u * x.in_tok;
            i32x4 v = load8(row + c, left);
            if (TURN != 0 && kv == 0)
                v = turned8<DT, TURN == 1>(pairs, row, v, c, sines + (s - from) * pairs);
            return v;
        };
        u16x2 most = {0, 0};
        auto look = [&](i32x4 v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                u16x2 m = __builtin_bit_cast(u16x2, (uint32_t)v[e] & 0x7fff7fffu);
                m.x = m.x >= Type8<DT>::INF ? 0 : m.x;
                m.y = m.y >= Type8<DT>::INF ? 0 : m.y;
                most = __builtin_elementwise_max(most, m);
            }
        };
        // (the first HELD chunks of a lane stay, others are loaded again)
        i32x4 held[HELD];
        const uint32_t round = HELD * step;
        auto load = [&](i32x4 *v, uint32_t s0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const uint32_t s = s0 + i * step + sub;
                v[i] = s < to && left > 0 ? get(s) : i32x4{0, 0, 0, 0};
            }
        };
        auto look_all = [&](const i32x4 *v) {
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                look(v[i]);
        };
        load(held, from);
        look_all(held);
        for (uint32_t s0 = from + round; s0 < to; s0 += round) {
            i32x4 more[HELD];
            load(more, s0);
            look_all(more);
        }
        uint32_t top = most.x > most.y ? most.x : most.y;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t y = (uint32_t)__shfl_xor((int)top, o);
            top = top > y ? top : y;
        }
        if constexpr (WAVES == 4) {
            __shared__ uint32_t tops[4];
            __syncthreads();
            if ((threadIdx.x & 63) == 0)
                tops[wave] = top;
            __syncthreads();
            top = tops[0];
#pragma unroll
            for (int w = 1; w < 4; ++w)
                top = top > tops[w] ? top : tops[w];
        }
        int e = exponent_of<DT>(to_float(DT, top));
        if (from > 0) {
            const int old = was < -126 ? -126 : was;
            e = e > old ? e : old;
            if (e > old) {      // the rows that are there
                const float f = power(old - e < -126 ? -126 : old - e);
                for (uint32_t s = sub; s < from; s += step) {
                    if (left <= 0)
                        continue;
                    uint32_t w[2];
                    uint8_t *q = out + (int64_t)s * row_s + c;
                    __builtin_memcpy(w, q, 8);
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false);
                        const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
                        w[k] = four(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
                    }
                    __builtin_memcpy(q, w, 8);
                }
            }
        }
        const float f = power_less(e);
        auto put = [&](uint32_t s, i32x4 v) {
            uint32_t w[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float y[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const uint32_t bits = ((uint32_t)v[2 * k + (z >> 1)] >> (16 * (z & 1))) & 0xffffu;
                    y[z] = bound(to_float(DT, bits) * f, (bits & 0x7fffu) < Type8<DT>::INF);
                }
                w[k] = four(y[0], y[1], y[2], y[3]);
            }
            __builtin_memcpy(out + (int64_t)s * row_s + c, w, 8);
        };
        auto put_all = [&](const i32x4 *v, uint32_t s0) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const uint32_t s = s0 + i * step + sub;
                if (s < to && left > 0)
                    put(s, v[i]);
            }
        };
        put_all(held, from);
        for (uint32_t s0 = from + round; s0 < to; s0 += round) {
            i32x4 more[HELD];
            load(more, s0);
            put_all(more, s0);
        }
        if (tid == 0)
            *at = (int8_t)e;
    }
}

template <int DT, int TURN>
void (*append8_of(bool all))(const Append8Args)
{
    return all ? append8_blocks<DT, TURN, 4> : append8_blocks<DT, TURN, 1>;
}

template <int DT>
void (*append8_kernel(const Turn &t, bool all))(const Append8Args)
{
    if (t.pairs == 0)
        return append8_of<DT, 0>(all);
    return t.layout == 0 ? append8_of<DT, 1>(all) : append8_of<DT, 2>(all);
}

}  // namespace

hipError_t launch_append8(const Append8 &r, hipStream_t s)
{
    Append8Args g{};
    g.r = r;
    const uint32_t lanes = r.c.d / 8;
    g.by_lanes = PageDiv::of(lanes);
    g.step1 = 64 / lanes;
    g.step4 = 256 / lanes;
    g.units = 2 * r.c.heads;
    const bool all = r.c.by_block.page > g.step1 * held_chunks(r.turn.pairs != 0);
    // A workgroup goes on with the next heads while 1024 workgroups remain and it has sines to share
    // (8 x 2048 tokens of 8 heads of 128, turned: 98 us with sines for each head, 31 so).
    const uint32_t once = all ? 1 : 4;
    const uint64_t sets = (uint64_t)r.c.batch * r.blocks;
    g.each = 1;
    while (r.turn.pairs && g.each * once < g.units &&
           sets * ((g.units + 2 * g.each * once - 1) / (2 * g.each * once)) >= 1024)
        g.each *= 2;
    g.groups = (g.units + g.each * once - 1) / (g.each * once);
    g.by_pairs = PageDiv::of(r.turn.pairs ? r.turn.pairs : 1);
    g.by_blocks = PageDiv::of(r.blocks);
    g.by_groups = PageDiv::of(g.groups);
    const uint64_t total = sets * g.groups;
    hipError_t e = hipSuccess;
    for (; g.first < total && e == hipSuccess; g.first += A8_GRID) {
        const uint64_t left = total - g.first;
        const dim3 grid((uint32_t)(left < A8_GRID ? left : A8_GRID));
        if (r.dtype == sjk::DT_F16)
            append8_kernel<sjk::DT_F16>(r.turn, all)<<<grid, 256, 0, s>>>(g);
        else
            append8_kernel<sjk::DT_BF16>(r.turn, all)<<<grid, 256, 0, s>>>(g);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sjc
