// sj_attend_kernels.h -- attention of a few tokens of every sequence over its rows in
// the cache (sj_attend), for one element type per translation unit.
//
// For a query row q and the rows n it sees, with s_n = scale <q, k_n>:
//   m = max s_n, l = sum exp(s_n - m), out = sum exp(s_n - m) v_n / l, lse = m + log l.
// One pass over the rows keeps (m, l, sum) and rescales them when m grows;
// results over disjoint sets of rows join by the same rule.  The exponentials enter the
// product with v rounded to 16 bits, as the matrix cores take them: each costs up to half a
// unit of its last place, which rows of equal scores share, beside the rounding of out itself.
// Binary16 ends at 2^-14 (2^-24 with fewer bits): its exponentials are scaled by 2^LIFT, so that
// the largest ones lie at the type's upper end and rows keep all their bits down to 2^-25 of
// the largest, or 2^-28 (with the largest at 1, 32768 rows of weight e^-17.4 beside one of
// weight 1 came out as 0).  Statistics, sums and weights stay in 32 bits.
#pragma once

#include <type_traits>

#include "sj_cache.h"

namespace sjc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int64_t i64x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

template <int DT>
struct Elem;
template <>
struct Elem<sjk::DT_F16> {
    typedef _Float16 one;
    typedef f16x8 eight;
    static constexpr uint32_t EXP = 0x7c00u;   // exponent bits: all set = not finite
    // the exponentials' scale where the maximum is followed at once and where it is
    // followed late, once a score is 2^LATE times the weight of m's: 2^15 at most
    static constexpr int LIFT = 14, LATE = 4, LATE_LIFT = 11;
    static __device__ __forceinline__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mma(i32x4 a, i32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
template <>
struct Elem<sjk::DT_BF16> {
    typedef __bf16 one;
    typedef bf16x8 eight;
    static constexpr uint32_t EXP = 0x7f80u;
    static constexpr int LIFT = 0, LATE = 8, LATE_LIFT = 0;     // (the exponents of fp32)
    static __device__ __forceinline__ f32x4 mma(i32x4 a, i32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mma(i32x4 a, i32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

__device__ __forceinline__ float bits_to_float(uint16_t x, int dt)
{
    return dt == sjk::DT_F16 ? (float)__builtin_bit_cast(_Float16, x)
                             : __uint_as_float((uint32_t)x << 16);
}

// The eight elements with zeros in the place of infinities and NaN if the row is one of the
// call's own tokens (all tokens see the others); returns whether there were any.
template <int DT>
__device__ __forceinline__ uint32_t drop_odd8(i32x4 &v, bool own)
{
    constexpr uint32_t EXP = Elem<DT>::EXP;
    const uint32_t mask = own ? ~0u : 0u;
    uint32_t odd = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t x = (uint32_t)v[e];
        const uint32_t lo = (x & EXP) == EXP ? mask & 0xffffu : 0u;
        const uint32_t hi = ((x >> 16) & EXP) == EXP ? mask & 0xffff0000u : 0u;
        v[e] = (int)(x & ~(lo | hi));
        odd |= lo | hi;
    }
    return odd;
}

// Eight 16-bit values down a column of LDS rows: each group of 16 lanes reads 4 rows x 16
// columns at lo and 4 more at hi (lane l passes the address of columns 4 (l % 4) .. + 3 of row
// (l / 4) % 4) and lane l receives column l % 16 of both.
__device__ __forceinline__ i32x4 column8(const uint8_t *lo, const uint8_t *hi)
{
    typedef __attribute__((address_space(3))) s16x4 lds4;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)lo);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)hi);
    return __builtin_bit_cast(i32x4, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Waits for the loads so far.  Before a loop: registers loaded ahead of it would
// otherwise be waited for at their first use in every round, and with them the
// round's own loads.
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// LDS written by the wave's lanes is there for its other lanes.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 2^x, 2^-inf = 0.
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ int64_t shfl64(int64_t v, int lane)
{
    const uint32_t lo = (uint32_t)__shfl((int)(uint32_t)v, lane);
    const uint32_t hi = (uint32_t)__shfl((int)(uint32_t)((uint64_t)v >> 32), lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// How the heads' d elements fill the kernels' 32 DC: all of them, whole 16-byte chunks of them, or
// any number (its own variant, since the last chunk's element-wise loads are waited for where
// they are made: 64 query rows on 8 sequences of 1000 to 7000 rows, d = 192: 117 us, 102 with chunks).
enum Fit { FIT_ANY = 0, FIT_CHUNKS = 1, FIT_WHOLE = 2 };

template <int FIT>
__device__ __forceinline__ i32x4 load_fit(const uint16_t *p, int left)
{
    if constexpr (FIT == FIT_ANY)
        return load8(p, left);
    i32x4 v = {0, 0, 0, 0};
    if (FIT == FIT_WHOLE || left > 0)
        __builtin_memcpy(&v, p, 16);
    return v;
}

// Eight elements of a query, negated for a negative scale: the scores' order is then
// that of the products, and the maximum can be taken before the scale.
template <int FIT>
__device__ __forceinline__ i32x4 load_q8(const Attend &a, const uint16_t *p, int left)
{
    i32x4 v = load_fit<FIT>(p, left);
    const int flip = a.negate ? (int)0x80008000 : 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] ^= flip;
    return v;
}

// Rows of sequence b: those before the call's tokens, the tokens there are, and the
// end of the tokens' rows.
struct Rows {
    uint32_t len, count, end;
};

__device__ __forceinline__ Rows rows_of(const Attend &a, uint32_t b)
{
    Rows r;
    r.len = clamp_rows(a.len[b], a.c.room);
    r.count = a.count ? clamp_rows(a.count[b], a.t) : a.t;
    r.end = r.len + r.count < a.c.room ? r.len + r.count : a.c.room;
    return r;
}

// Whether token u sees row n of its sequence (n < r.end).
__device__ __forceinline__ bool sees(const Attend &a, uint32_t b, const Rows &r, uint32_t u,
                                     uint32_t n)
{
    if (n < r.len)
        return true;
    const uint32_t w = n - r.len;
    if (!a.tree)
        return w <= u;
    return (a.tree[(int64_t)b * a.tree_seq + (int64_t)u * a.tree_tok + (w >> 6)] >> (w & 63)) & 1;
}

// Which of the 64 rows from row0 on token u sees, bit by bit, among rows that exist.
__device__ __forceinline__ uint64_t seen64(const Attend &a, uint32_t b, const Rows &r, uint32_t u,
                                           uint32_t row0)
{
    const int64_t o = (int64_t)row0 - r.len;     // of the tokens' own rows
    const uint64_t before = o >= 0 ? 0 : (o <= -64 ? ~(uint64_t)0 : ((uint64_t)1 << -o) - 1);
    if (!a.tree) {
        const int64_t n = (int64_t)u + 1 - o;    // a chain: the rows below this one
        return n <= 0 ? 0 : (n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1);
    }
    if (o <= -64)
        return before;
    const uint64_t *t = a.tree + (int64_t)b * a.tree_seq + (int64_t)u * a.tree_tok;
    if (o < 0)
        return before | t[0] << -o;
    const uint32_t words = (a.t + 63) / 64, w = (uint32_t)(o >> 6), sh = (uint32_t)(o & 63);
    uint64_t v = w < words ? t[w] >> sh : 0;
    if (sh && w + 1 < words)
        v |= t[w + 1] << (64 - sh);
    return v;
}

// Calls f(row of values) for the tokens' own rows in [from, to) that token u sees.  The
// products leave out what is not finite in these rows, since 0 x inf and 0 x NaN would
// reach the queries that do not see them; added up afterwards, what a query does
// see of them decides its output whatever the weights are.
template <class F>
__device__ __forceinline__ void own_rows(const Attend &a, uint32_t b, uint32_t h, const Rows &r,
                                         uint32_t u, uint32_t from, uint32_t to, F f)
{
#pragma unroll 1
    for (uint32_t n = from > r.len ? from : r.len; n < to; ++n) {
        const Place p = place_of(a.c, b, n);
        if (p.page >= 0 && sees(a, b, r, u, n))
            f(a.c.v + (int64_t)p.page * a.c.v_page + (int64_t)p.slot * a.c.v_row +
              (int64_t)h * a.c.v_head);
    }
}

// x where it is infinite or NaN, else 0.
template <int DT>
__device__ __forceinline__ float odd_part(uint16_t x)
{
    return (x & Elem<DT>::EXP) == Elem<DT>::EXP ? bits_to_float(x, DT) : 0.f;
}

// For each of the query rows r0 .. r0 + n - 1 of q_rows, which of the 64 rows from row0 on it
// sees, among those in `there`: to `vis`, a row a lane.
__device__ __forceinline__ void seen_rows(const Attend &a, uint32_t b, const Rows &r, uint32_t r0,
                                          uint32_t n, uint32_t q_rows, uint32_t row0, uint64_t there,
                                          uint64_t *vis)
{
    wave_sync();        // (the last rows have been read)
    for (uint32_t i = threadIdx.x & 63; i < n; i += 64)
        vis[i] = r0 + i < q_rows ? there & seen64(a, b, r, a.by_group.quot(r0 + i), row0) : 0;
    wave_sync();
}

// Weights of key row n (of 64) from the scores and lse (z, base 2) of the query rows
// v[8 (e / 4) + e % 4]: of those that see it (lse may be NaN in the others).
template <class S>
__device__ __forceinline__ float weigh_seen(const S &s, const f32x4 *z, float scale2,
                                            const uint64_t *v, uint32_t n)
{
    float w = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const uint32_t bits = ((const uint32_t *)(v + 8 * (e >> 2) + (e & 3)))[n >> 5];
        const float p = exp2_(__builtin_fmaf(s[e], scale2, -z[e >> 2][e & 3]));
        w += (bits >> (n & 31)) & 1 ? p : 0.f;
    }
    return w;
}

// The share of the work that a workgroup takes: blocks [first, last) of
// AT_ROWS rows of sequence b, number `share` of its `shares`.
struct Share {
    uint32_t b, share, shares, first, last;
    Rows rows;
};

// Finds share number `slot` of the batch.  Each sequence's blocks are cut into whole shares
// of at most `size` blocks, one at least.  `size` is the smallest with which the
// shares of all sequences come to no more than `want`, per head and tile
// the workgroups that the GPU holds at once, since one more would run after all
// others.  (For more than 64 sequences, where the search takes several passes, a
// size that is large enough; with want sequences or more there is one share each.)
// Every workgroup computes the cut from the lengths on the device, so the grid
// does not depend on them.  Returns false when there are fewer shares.  Called
// by whole waves.
__device__ __forceinline__ bool find_share(const Attend &a, uint32_t slot, Share *out)
{
    const uint32_t lane = threadIdx.x & 63, B = a.c.batch;
    const uint32_t want = a.want;
    auto blocks_of = [&](uint32_t b) -> uint32_t {
        return b < B ? (rows_of(a, b).end + AT_ROWS - 1) / AT_ROWS : 0;
    };
    uint32_t blocks = 0, size;
    if (B <= 64) {
        blocks = blocks_of(lane);
        const uint32_t total = sum_all(blocks);     // (64 x 2^26 blocks at most)
        size = total / want + (total % want != 0);
        size = size < AT_WAVES ? AT_WAVES : size;   // (a block per wave at least)
        uint32_t most = B < want ? total / (want - B) + 1 : total + 1;
        if (B > 1)
            while (size < most) {
                const uint32_t mid = size + (most - size) / 2;
                const uint32_t n = lane < B ? (blocks + mid - 1) / mid : 0;
                if (sum_all(lane < B && n == 0 ? 1 : n) <= want)
                    most = mid;
                else
                    size = mid + 1;
            }
    } else {
        unsigned long long total = 0;
        for (uint32_t b0 = 0; b0 < B; b0 += 64)
            total += blocks_of(b0 + lane);
        for (int o = 1; o < 64; o <<= 1)
            total += __shfl_xor(total, o);
        total = B < want ? total / (want - B) + 1 : total;
        size = total < AT_WAVES ? AT_WAVES : (total < 1u << 30 ? (uint32_t)total : 1u << 30);
    }
    uint32_t base = 0;
    for (uint32_t b0 = 0; b0 < B; b0 += 64) {
        if (B > 64)
            blocks = blocks_of(b0 + lane);
        uint32_t shares = (blocks + size - 1) / size;
        shares = b0 + lane >= B ? 0 : (shares ? shares : 1);
        const uint32_t incl = sum_upto(shares);
        const uint32_t sum = (uint32_t)__builtin_amdgcn_readlane((int)incl, 63);
        if (slot < base + sum) {
            const int who = __builtin_amdgcn_readfirstlane(
                __ffsll((unsigned long long)__ballot(slot < base + incl)) - 1);
            const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)shares, who);
            const uint32_t nb = (uint32_t)__builtin_amdgcn_readlane((int)blocks, who);
            out->b = b0 + who;
            out->shares = mine;
            out->share = slot - (base + (uint32_t)__builtin_amdgcn_readlane((int)incl, who) - mine);
            out->first = (uint32_t)((unsigned long long)nb * out->share / mine);
            out->last = (uint32_t)((unsigned long long)nb * (out->share + 1) / mine);
            out->rows = rows_of(a, out->b);
            return true;
        }
        base += sum;
    }
    return false;
}

__device__ __forceinline__ float max_all(float x)
{
#pragma unroll
    for (int o = 1; o < 64; o <<= 1)
        x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

// Place of query row r of head h among the results of share s.
__device__ __forceinline__ uint64_t part_of(const Attend &a, uint32_t s, uint32_t h, uint32_t r,
                                            uint32_t QT)
{
    return ((uint64_t)s * a.c.heads * a.tiles + h * a.tiles + r / QT) * QT + r % QT;
}

// The last workgroup of a sequence, head and tile to arrive joins their shares, in the shares'
// order whichever it is.  The shares' results travel as relaxed atomic stores and loads of the
// device's scope, which pass by the XCDs' own caches: a fence would write back and
// drop a whole cache instead.  Each wave waits for its stores before the
// workgroup is counted; the counter is 0 again for the next call.
__device__ __forceinline__ void put2(float *p, float x, float y)
{
    const uint64_t v = (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32;
    __hip_atomic_store((uint64_t *)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ f32x2 get2(const float *p)
{
    const uint64_t v =
        __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return f32x2{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
}

template <int DT, uint32_t QT, uint32_t D>
__device__ __forceinline__ void join_last(const Attend &a, uint32_t b, uint32_t h, uint32_t unit,
                                          uint32_t slot, uint32_t shares, uint32_t count)
{
    typedef Elem<DT> E;
    __shared__ uint32_t arrived;
    wait_loads();       // (stores count as loads do)
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t *n = a.arrivals + (uint64_t)b * a.c.heads * a.tiles + unit;
        arrived = __hip_atomic_fetch_add(n, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (arrived == shares - 1)
            __hip_atomic_store(n, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (arrived != shares - 1)
        return;
    const uint64_t first = (uint64_t)slot * a.c.heads * a.tiles + unit;
    const uint64_t step = (uint64_t)a.c.heads * a.tiles;
    // 16 threads a query row, columns 4 (threadIdx.x % 16) + 64 k
    for (uint32_t q0 = 0; q0 < QT; q0 += 16) {
        const uint32_t qi = q0 + (threadIdx.x >> 4), x = threadIdx.x & 15;
        const uint32_t r = unit % a.tiles * QT + qi, u = a.by_group.quot(r);
        auto at = [&](uint32_t s) { return (first + s * step) * QT + qi; };
        if (r >= a.t * a.group)
            continue;
        float top = -INFINITY;
        for (uint32_t s = x; s < shares; s += 16)
            top = fmaxf(top, get2(a.part_ml + 2 * at(s))[0]);
#pragma unroll
        for (int o = 1; o < 16; o <<= 1)
            top = fmaxf(top, __shfl_xor(top, o));
        const float base = top == -INFINITY ? 0.f : top;
        f32x4 o[D / 64] = {};
        float l = 0.f;
#pragma unroll 4
        for (uint32_t s = 0; s < shares; ++s) {
            const uint64_t p = at(s);
            const f32x2 ml = get2(a.part_ml + 2 * p);
            const float f = exp2_(ml[0] - base);
            l += ml[1] * f;
#pragma unroll
            for (uint32_t k = 0; k < D / 64; ++k) {
                const float *y = a.part_o + p * D + 64 * k + 4 * x;
                const f32x2 lo = get2(y), hi = get2(y + 2);
                o[k] += f32x4{lo[0], lo[1], hi[0], hi[1]} * f;
            }
        }
        const bool live = u < count && l != 0.f;
        const float inv = live ? 1.f / l : 0.f;
        const uint64_t row = ((uint64_t)b * a.t + u) * a.q_heads + h * a.group + r - u * a.group;
#pragma unroll
        for (uint32_t k = 0; k < D / 64; ++k)
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
                const uint32_t c = 64 * k + 4 * x + e;
                if (c < a.c.d)
                    a.out[row * a.c.d + c] =
                        __builtin_bit_cast(uint16_t, (typename E::one)(live ? o[k][e] * inv : 0.f));
            }
        if (x == 0)
            a.lse[row] = live ? (top + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : -INFINITY;
    }
}

// ------------------------------------------------------------- the split kernel
//
// A workgroup takes one share of a sequence's rows for one cache head and its up to
// QT = 16 NQ query rows (row r = token r / group, query head r % group: all
// that read this cache head, so that a cache row is loaded once for all of them).
// Its four waves take blocks of 32 rows in turn, each with running statistics
// of its own; they join at the end through LDS.
//
// A block on a wave: S^T = K Q^T as 16 x 16 x 32 tiles with K's rows from global
// memory straight in operand layout (lane l: row l % 16, elements 8 (l / 16) ..
// + 7 of each 32), so that lane l holds the scores of query l % 16 with rows
// 4 (l / 16) .. + 3 of both 16-row halves: the statistics of a query need two
// exchanges, and the exponentials are, without moving, the operand of
// O^T = V^T P^T in the order of rows {4g .. 4g + 3, 16 + 4g .. 16 + 4g + 3} of lane group g.
// V goes through the wave's own LDS and comes back transposed (ds_read_b64_tr_b16:
// each 16-lane group reads 4 rows x 16 columns, lane l receives column l) in
// the same order of rows.  LDS rows are padded by 32 bytes: the 4 rows x 32 bytes that a
// lane group reads then lie in different banks.
// The next block's K and V are loaded while this one is worked on.
// Bound by HBM: up to 16 query rows need 4 d operations a byte pair, far below what the matrix
// cores could do.  1.09 GB of cache rows (2 sequences of 131072 x 8 heads of 128) in 200 us,
// 5.4 TB/s, or 231 with the scores kept (33 MB); 32 sequences of 200 to 8192 rows, 550 MB, in
// 116 (4.7 TB/s).  One sequence of 2048 rows: 10 us, of which most is the latency of the chain
// lengths, page numbers, rows, join.
template <int DT, int DC, int NQ, int FIT>
__global__ void __launch_bounds__(256) attend_split(const Attend a)
{
    typedef Elem<DT> E;
    constexpr int QT = AT_Q * NQ, D = 32 * DC;
    constexpr int RS = 2 * D + 32;              // bytes of a V row in LDS
    constexpr int OS = D + 4;                   // floats of a query's sums in LDS
    constexpr int NV = 2 * DC;                  // 16-byte loads of V per lane and block
    constexpr int VR = 16 / DC;                 // rows of V per load
    constexpr int WAVE_LDS = AT_ROWS * RS;
    static_assert(AT_Q * OS * 4 <= WAVE_LDS, "the sums of a query tile fit in the wave's V");
    __shared__ __align__(16) uint8_t lds[AT_WAVES * WAVE_LDS];
    __shared__ float stat[AT_WAVES][QT][2];
    __shared__ uint32_t odd_any;      // infinities or NaN among the tokens' own values

    const uint32_t lane = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t units = a.c.heads * a.tiles;
    const uint32_t unit = blockIdx.x % units, slot = blockIdx.x / units;
    const uint32_t h = unit / a.tiles, tile = unit % a.tiles;
    Share sh;
    if (slot >= a.slots || !find_share(a, slot, &sh))
        return;
    const uint32_t b = __builtin_amdgcn_readfirstlane(sh.b);
    const uint32_t first = __builtin_amdgcn_readfirstlane(sh.first);
    const uint32_t last = __builtin_amdgcn_readfirstlane(sh.last);
    const uint32_t shares = __builtin_amdgcn_readfirstlane(sh.shares);
    const Rows rows = {(uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.len),
                       (uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.count),
                       (uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.end)};
    if (unit == 0 && sh.share == 0 && threadIdx.x == 0) {
        a.plan[2 * b] = slot;
        a.plan[2 * b + 1] = shares;
    }

    const uint32_t to = last * AT_ROWS < rows.end ? last * AT_ROWS : rows.end;
    const uint32_t q16 = lane & 15, g4 = lane >> 4;
    const uint32_t d = a.c.d;
    const uint32_t q_rows = a.t * a.group;

    // the first blocks' page numbers, on their way with the queries
    auto entry = [&](uint32_t blk) {
        return entry_of(a.c, a.len, b, blk * AT_ROWS + (lane & 31));
    };
    Entry first_at = {0, 0u}, ahead = {0, 0u};
    if (first + wave < last) {
        first_at = entry(first + wave);
        ahead = entry(first + wave + AT_WAVES);
    }

    // queries: lane l holds query l % 16 of each tile in operand layout
    i32x4 Q[NQ][DC];
    uint32_t tok[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        const uint32_t r = tile * QT + AT_Q * j + q16;
        const bool there = r < q_rows && r / a.group < rows.count;
        tok[j] = there ? r / a.group : 0;
        const uint16_t *p = a.q + (int64_t)b * a.q_seq + (int64_t)tok[j] * a.q_tok +
                            (int64_t)(h * a.group + (there ? r % a.group : 0)) * a.q_head + 8 * g4;
#pragma unroll
        for (int c = 0; c < DC; ++c)
            Q[j][c] = there ? load_q8<FIT>(a, p + 32 * c, (int)d - (int)(32 * c + 8 * g4))
                            : i32x4{0, 0, 0, 0};
    }

    wait_loads();
    f32x4 O[NQ][NV];
    float m[NQ], l[NQ];
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        m[j] = -INFINITY;
        l[j] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            O[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const uint16_t *kb = a.c.k + (int64_t)h * a.c.k_head, *vb = a.c.v + (int64_t)h * a.c.v_head;
    uint8_t *const my = lds + wave * WAVE_LDS;

    // place of row lane % 32 of a block: absent rows read page 0, row 0 (their
    // scores and values are replaced below)
    auto place = [&](const Entry &e) { return place_of(a.c, b, e, to); };
    i32x4 K[2][DC], V[NV];
    auto load_k = [&](const Place &p) {
        const int64_t off = p.page < 0 ? 0
                                       : (int64_t)p.page * a.c.k_page + (int64_t)p.slot * a.c.k_row;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint16_t *r = kb + shfl64(off, (int)q16 + 16 * t) + 8 * g4;
#pragma unroll
            for (int c = 0; c < DC; ++c)
                K[t][c] = load_fit<FIT>(r + 32 * c, (int)d - (int)(32 * c + 8 * g4));
        }
    };
    const uint32_t v_row = lane / (4 * DC), v_col = 8 * (lane % (4 * DC));
    auto load_v = [&](const Place &p) {
        const int64_t off = p.page < 0 ? 0
                                       : (int64_t)p.page * a.c.v_page + (int64_t)p.slot * a.c.v_row;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint16_t *r = vb + shfl64(off, VR * i + (int)v_row) + v_col;
            V[i] = load_fit<FIT>(r, (int)d - (int)v_col);
        }
    };

    if (threadIdx.x == 0)
        odd_any = 0;
    __syncthreads();
    uint32_t blk = first + wave;
    Place cur = {-1, 0u}, nxt = {-1, 0u};
    if (blk < last) {
        cur = place(first_at);
        load_k(cur);
        load_v(cur);
    }
    for (; blk < last; blk += AT_WAVES) {
        nxt = place(ahead);
        // bit r: row r of the block exists
        const uint32_t there = (uint32_t)__ballot(cur.page >= 0);
        const bool tail = blk * AT_ROWS + AT_ROWS > rows.len;

        f32x4 s[NQ][2];
#pragma unroll
        for (int j = 0; j < NQ; ++j)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                s[j][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DC; ++c)
                    s[j][t] = E::mma(K[t][c], Q[j][c], s[j][t]);
            }
        ahead = entry(blk + 2 * AT_WAVES);
        load_k(nxt);        // (past the end: page 0, row 0; a branch would cost full waits)

        // V to LDS; rows that do not exist as zeros (0 x NaN would reach every query)
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (tail || there != 0xffffffffu) {
                if (!((there >> (VR * i + v_row)) & 1))
                    V[i] = i32x4{0, 0, 0, 0};
                odd |= drop_odd8<DT>(V[i], blk * AT_ROWS + VR * i + v_row >= rows.len);
                asm volatile("");       // (a branch, not selects in every round)
            }
            *(i32x4 *)(my + (VR * i + v_row) * RS + 2 * v_col) = V[i];
        }
        load_v(nxt);

        // scores to exponentials
        i32x4 P[NQ];
        float pf[NQ][8];
        uint32_t seen[NQ];
#pragma unroll
        for (int j = 0; j < NQ; ++j) {
            seen[j] = there & (tail ? (uint32_t)seen64(a, b, rows, tok[j], blk * AT_ROWS) : ~0u);
            if (tail || there != 0xffffffffu) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    s[j][e >> 2][e & 3] = (seen[j] >> (16 * (e >> 2) + 4 * g4 + (e & 3))) & 1
                                              ? s[j][e >> 2][e & 3]
                                              : -INFINITY;
                asm volatile("");       // (a branch, not selects in every round)
            }
            if (NQ == 1 && a.scores && q16 < q_rows && blk * AT_ROWS < a.s_cols) {
                float *to_s = a.scores + ((uint64_t)(b * a.c.heads + h) * q_rows + q16) * a.s_cols +
                              blk * AT_ROWS + 4 * g4;
                *(f32x4 *)to_s = s[j][0] * a.scale2;
                *(f32x4 *)(to_s + 16) = s[j][1] * a.scale2;
            }
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                top = fmaxf(top, s[j][e >> 2][e & 3]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m[j], top);
            // nothing seen yet: any finite maximum will do
            const float high = m_new == -INFINITY ? 0.f : m_new * a.scale2;
            const float shrink = exp2_(m[j] * a.scale2 - high), base = high - E::LIFT;
            m[j] = m_new;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pf[j][e] = exp2_(__builtin_fmaf(s[j][e >> 2][e & 3], a.scale2, -base));
                sum += pf[j][e];
            }
            l[j] = l[j] * shrink + sum;     // this lane's rows only; joined at the end
            typename E::eight p8;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                p8[e] = (typename E::one)pf[j][e];
            P[j] = __builtin_bit_cast(i32x4, p8);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                O[j][i] *= shrink;
        }

        if (odd)
            odd_any = 1;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint8_t *at = my + (4 * g4 + (q16 >> 2)) * RS + 32 * i + 8 * (q16 & 3);
            const i32x4 vt = column8(at, at + 16 * RS);
#pragma unroll
            for (int j = 0; j < NQ; ++j)
                O[j][i] = E::mma(vt, P[j], O[j][i]);
        }
        cur = nxt;
    }

    // join the lanes of a query, then the waves; the scale 2^LIFT ends here
    constexpr float DOWN = 1.f / (1 << E::LIFT);
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        l[j] *= DOWN;
        l[j] += __shfl_xor(l[j], 16);
        l[j] += __shfl_xor(l[j], 32);
        m[j] *= a.scale2;
        if (g4 == 0) {
            stat[wave][AT_Q * j + q16][0] = m[j];
            stat[wave][AT_Q * j + q16][1] = l[j];
        }
    }
    __syncthreads();
    const uint64_t part = (uint64_t)slot * units + unit;
#pragma unroll
    for (int j = 0; j < NQ; ++j) {
        float top = -INFINITY;
#pragma unroll
        for (uint32_t w = 0; w < AT_WAVES; ++w)
            top = fmaxf(top, stat[w][AT_Q * j + q16][0]);
        const float f = exp2_(m[j] - (top == -INFINITY ? 0.f : top)) * DOWN;
        if (j)
            __syncthreads();
        float *mine = (float *)my + q16 * OS;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            *(f32x4 *)(mine + 16 * i + 4 * g4) = O[j][i] * f;
        __syncthreads();
        // 256 threads: query threadIdx.x / 16, columns 4 (threadIdx.x % 16) + 64 k
        const uint32_t qi = threadIdx.x >> 4, c0 = 4 * (threadIdx.x & 15);
        float tot = -INFINITY, sum = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < AT_WAVES; ++w)
            tot = fmaxf(tot, stat[w][AT_Q * j + qi][0]);
        const float base = tot == -INFINITY ? 0.f : tot;
#pragma unroll
        for (uint32_t w = 0; w < AT_WAVES; ++w)
            sum += stat[w][AT_Q * j + qi][1] * exp2_(stat[w][AT_Q * j + qi][0] - base);
        const uint32_t r = tile * QT + AT_Q * j + qi;
        const uint32_t u = r / a.group;
        if (r < q_rows) {
            const bool live = u < rows.count;
            const uint64_t row = ((uint64_t)b * a.t + u) * a.q_heads + h * a.group + r % a.group;
#pragma unroll
            for (uint32_t c = c0; c < (uint32_t)D; c += 64) {
                f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (uint32_t w = 0; w < AT_WAVES; ++w)
                    o += *(const f32x4 *)((const float *)(lds + w * WAVE_LDS) + qi * OS + c);
                if (odd_any && live)
                    own_rows(a, b, h, rows, u, first * AT_ROWS, to, [&](const uint16_t *v) {
#pragma unroll
                        for (uint32_t e = 0; e < 4; ++e)
                            if (c + e < d)
                                o[e] += odd_part<DT>(v[c + e]);
                    });
                if (shares > 1) {
                    float *p = a.part_o + (part * QT + AT_Q * j + qi) * D + c;
                    if (a.arrivals) {
                        put2(p, o[0], o[1]);
                        put2(p + 2, o[2], o[3]);
                    } else {
                        *(f32x4 *)p = o;
                    }
                } else {
                    const float inv = live && sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e)
                        if (FIT == FIT_WHOLE || c + e < d)
                            a.out[row * d + c + e] = __builtin_bit_cast(
                                uint16_t, (typename E::one)(live && sum != 0.f ? o[e] * inv : 0.f));
                }
            }
            if (c0 == 0) {
                if (shares > 1) {
                    put2(a.part_ml + (part * QT + AT_Q * j + qi) * 2, tot, sum);
                } else {
                    a.lse[row] = live && sum != 0.f
                                     ? (tot + __builtin_amdgcn_logf(sum)) * 0.69314718055994531f
                                     : -INFINITY;
                }
            }
        }
    }
    if (shares > 1 && a.arrivals)
        join_last<DT, QT, D>(a, b, h, unit, slot - sh.share, shares, rows.count);
}

// ------------------------------------------------------------- the tiled kernel
//
// For more query rows than 32: QW groups of 32 query rows share tiles of BN cache rows
// in LDS (32 x 32 x 16 products).  With QW = 4 and 8 every wave takes 32 queries and all rows of a
// tile, with QW = 2 two waves share 32 queries and take half of its rows each.  Eight waves
// halve the loads and LDS writes for a query (256 query rows over 4 x 32768 rows: 180 us in
// two tiles of four waves, 157 in one of eight).  As above
// S^T = K Q^T leaves query l % 32 in lane l with rows 8 (r / 4) + 4 (l / 32) + r % 4 in
// register r, which is, register by register, the operand of O^T = V^T P^T for steps of 16
// rows in the order {4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3} of lane half h.
// Two buffers; the next tile's loads go to registers while a tile is worked on
// and to LDS at the start of the next, one barrier a tile.  The 16-byte
// chunks of a row are permuted by the row (swz) so that neither the K reads (16
// rows, one chunk) nor the transposed V reads (4 rows, 4 chunks) meet in a bank.
// Bound by HBM up to 64 query rows (16 sequences of 1024 to 6000 rows, 8 heads of 128: 242 MB in 51
// us, 4.7 TB/s); with 256 rows (4 x 30000 to 32768) 132 GFLOP in 199 us in a row of calls (164
// in the first, before the clock falls to 2 GHz), 660 TFLOP/s: matrix cores 38% busy, the
// exponentials of the waves of a SIMD mostly beside each other's and not beside products.
// Every query tile runs over all rows of its sequence: of a long chain's own rows half are
// multiplied and masked.
template <int DC>
__device__ __forceinline__ uint32_t swz(uint32_t row, uint32_t chunk)
{
    if constexpr (DC == 2)
        return chunk ^ ((((row >> 1) & 1) << 2) | ((row >> 2) & 3));
    else
        return chunk ^ (((row & 3) << 2) | ((row >> 2) & 3));
}

template <int DT, int DC, int QW, int FIT>
__global__ void __launch_bounds__(QW == 8 ? 512 : 256, DC == 8 ? 1 : 2) attend_tiles(const Attend a)
{
    typedef Elem<DT> E;
    constexpr uint32_t NT = QW == 8 ? 512 : 256, D = 32 * DC, QT = 32 * QW, RW = QW == 8 ? 1 : 4 / QW;
    constexpr uint32_t BN = DC == 8 ? 32 : 64;      // rows of a tile
    constexpr uint32_t WR = BN / RW;                // of these, one wave's
    constexpr int SR = WR / 32;                     // 32-row products of a wave
    constexpr uint32_t CPR = 4 * DC;                // 16-byte chunks of a row
    constexpr int NL = BN * CPR / NT;              // loads per thread of K, of V
    constexpr uint32_t RPL = NT / CPR;             // rows per load of the workgroup
    constexpr uint32_t TILE = BN * D * 2;           // bytes
    static_assert(WR % 32 == 0, "whole products");
    __shared__ __align__(16) uint8_t lds[4 * TILE]; // K, V of two tiles
    __shared__ float stat[4][32][2];
    __shared__ uint32_t odd_any;
    __shared__ i64x2 where[8][BN];
    __shared__ uint64_t exist[8];

    const uint32_t lane = threadIdx.x & 63, tid = threadIdx.x;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t qw = wave % QW, rw = wave / QW;
    const uint32_t units = a.c.heads * a.tiles;
    // neighbours in (share, head, tile) on one XCD: the tiles of a head read the same rows
    const uint32_t per = gridDim.x / 8, id = (blockIdx.x % 8) * per + blockIdx.x / 8;
    const uint32_t unit = id % units, slot = id / units;
    const uint32_t h = unit / a.tiles, tile = unit % a.tiles;
    Share sh;
    if (slot >= a.slots || !find_share(a, slot, &sh))
        return;
    const uint32_t b = __builtin_amdgcn_readfirstlane(sh.b);
    const uint32_t shares = __builtin_amdgcn_readfirstlane(sh.shares);
    const Rows rows = {(uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.len),
                       (uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.count),
                       (uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.end)};
    const uint32_t from = __builtin_amdgcn_readfirstlane(sh.first) * AT_ROWS;
    const uint32_t last = __builtin_amdgcn_readfirstlane(sh.last) * AT_ROWS;
    const uint32_t to = last < rows.end ? last : rows.end;      // rows [from, to)
    if (unit == 0 && sh.share == 0 && tid == 0) {
        a.plan[2 * b] = slot;
        a.plan[2 * b + 1] = shares;
    }

    const uint32_t q32 = lane & 31, half = lane >> 5, g = lane >> 4, l16 = lane & 15;
    const uint32_t d = a.c.d, q_rows = a.t * a.group;
    const uint32_t r_mine = tile * QT + 32 * qw + q32;
    const bool live = r_mine < q_rows && a.by_group.quot(r_mine) < rows.count;
    const uint32_t tok = live ? a.by_group.quot(r_mine) : 0;
    const bool idle = tile * QT + 32 * qw >= q_rows;    // the wave has no query rows: it only loads
    i32x4 Q[2 * DC];
    {
        const uint16_t *p = a.q + (int64_t)b * a.q_seq + (int64_t)tok * a.q_tok +
                            (int64_t)(h * a.group + (live ? (r_mine - a.by_group.quot(r_mine) * a.group) : 0)) * a.q_head +
                            8 * half;
#pragma unroll
        for (int k = 0; k < 2 * DC; ++k)
            Q[k] = live ? load_q8<FIT>(a, p + 16 * k, (int)d - (int)(16 * k + 8 * half))
                        : i32x4{0, 0, 0, 0};
    }
    wait_loads();
    f32x16 O[DC];
#pragma unroll
    for (int i = 0; i < DC; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            O[i][r] = 0.f;
    float m = -INFINITY, l = 0.f;

    const uint16_t *kb = a.c.k + (int64_t)h * a.c.k_head, *vb = a.c.v + (int64_t)h * a.c.v_head;
    // places in a tile: chunk 2 k + half of row q32 of K (the same for every 32 rows), and of V
    // columns 32 z + 16 (g % 2) + 4 (l16 % 4) .. of rows 4 half + l16 / 4 and 8 further (the same
    // for every 16 rows)
    uint32_t k_at[2 * DC], v_at[DC][2];
#pragma unroll
    for (uint32_t k = 0; k < 2 * DC; ++k)
        k_at[k] = (rw * WR + q32) * (2 * D) + 16 * swz<DC>(q32, 2 * k + half);
#pragma unroll
    for (uint32_t z = 0; z < DC; ++z)
#pragma unroll
        for (uint32_t x = 0; x < 2; ++x) {
            const uint32_t r = 4 * half + (l16 >> 2) + 8 * x;
            v_at[z][x] = TILE + (rw * WR + r) * (2 * D) +
                         16 * swz<DC>(r, 4 * z + 2 * (g & 1) + ((l16 & 3) >> 1)) + 8 * (l16 & 1);
        }
    const uint32_t n_tiles = from < to ? (to - from + BN - 1) / BN : 0;
    const uint32_t row_at = tid / CPR, chunk = tid % CPR;
    auto entry = [&](uint32_t i) {
        return entry_of(a.c, a.len, b, from + i * BN + (lane & (BN - 1)));
    };
    // Offsets of tile i's rows, for the threads that load them, and which rows exist; absent
    // rows read page 0, row 0.  Waves 0 .. 3 (and 4 .. 7, alike)
    // do one tile of four each.
    auto post = [&](uint32_t i, const Entry &e) {
        const Place p = place_of(a.c, b, e, to);
        const uint64_t there = __ballot(p.page >= 0);
        if (lane < BN) {
            i64x2 o = {0, 0};
            if (p.page >= 0)
                o = i64x2{(int64_t)p.page * a.c.k_page + (int64_t)p.slot * a.c.k_row,
                          (int64_t)p.page * a.c.v_page + (int64_t)p.slot * a.c.v_row};
            where[i & 7][lane] = o;
        }
        if (lane == 0)
            exist[i & 7] = there;
    };
    auto exists = [&](uint32_t i) -> uint64_t {
        const uint64_t x = exist[i & 7];
        return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x) |
               (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32;
    };
    i32x4 kr[NL], vr[NL];
    auto fetch = [&](uint32_t i) {
        const int left = (int)d - (int)(8 * chunk);
        i64x2 o[NL];
#pragma unroll
        for (int x = 0; x < NL; ++x)
            o[x] = where[i & 7][RPL * x + row_at];
#pragma unroll
        for (int x = 0; x < NL; ++x) {
            kr[x] = load_fit<FIT>(kb + o[x][0] + 8 * chunk, left);
            vr[x] = load_fit<FIT>(vb + o[x][1] + 8 * chunk, left);
        }
    };
    // (the swizzle repeats every 16 rows, and RPL is a multiple of 8: one place, or two)
    uint32_t to_at[2];
#pragma unroll
    for (uint32_t x = 0; x < 2; ++x)
        to_at[x] = (RPL * x + row_at) * (2 * D) + 16 * swz<DC>(RPL * x + row_at, chunk);
    auto stash = [&](uint32_t i, uint32_t buf, uint64_t there) {
        uint8_t *kt = lds + buf * 2 * TILE, *vt = kt + TILE;
        if (from + i * BN + BN > rows.len || there != ~(uint64_t)0) {
            uint32_t odd = 0;
#pragma unroll
            for (int x = 0; x < NL; ++x) {
                if (!((there >> (RPL * x + row_at)) & 1))
                    vr[x] = i32x4{0, 0, 0, 0};  // (0 x NaN would reach every query)
                odd |= drop_odd8<DT>(vr[x], from + i * BN + RPL * x + row_at >= rows.len);
            }
            if (odd)
                odd_any = 1;
            asm volatile("");       // (a branch, not selects in every round)
        }
#pragma unroll
        for (int x = 0; x < NL; ++x) {
            const uint32_t at = to_at[x & 1] + (x >> 1) * 2 * RPL * (2 * D);
            *(i32x4 *)(kt + at) = kr[x];
            *(i32x4 *)(vt + at) = vr[x];
        }
    };

    if (tid == 0)
        odd_any = 0;
    // ahead of tile i: tile i + 1 on its way to LDS, i + 2 from memory, the offsets of the
    // next four tiles, the page numbers of the four after
    uint64_t there = 0;
    Entry ahead = {0, 0u};
    if (n_tiles > 0) {
        post(wave & 3, entry(wave & 3));
        ahead = entry(4 + (wave & 3));
        __syncthreads();
        there = exists(0);
        fetch(0);
        stash(0, 0, there);
        fetch(1);
    }
    __syncthreads();
    auto round = [&](uint32_t i, auto buf_) {
        constexpr uint32_t buf = decltype(buf_)::value;     // i % 2
        if ((i & 3) == 0) {
            post(i + 4 + (wave & 3), ahead);
            ahead = entry(i + 8 + (wave & 3));
        }
        const uint64_t there1 = exists(i + 1);
        stash(i + 1, 1 - buf, there1);
        fetch(i + 2);       // (past the end: page 0, row 0; a branch would cost full waits)
        if (idle) {
            there = there1;
            __syncthreads();
            return;
        }
        uint8_t *const kt = lds + buf * 2 * TILE;
        const uint32_t row0 = from + i * BN;
        const bool tail = row0 + BN > rows.len;
        const bool masked = tail || there != ~(uint64_t)0;

        f32x16 s[SR];
#pragma unroll
        for (int x = 0; x < SR; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                s[x][e] = 0.f;
        // four K fragments are read while four are multiplied
        constexpr int KS = 2 * DC * SR / 4;
        i32x4 f[2][4];
        auto read_k = [&](int y) {
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                const int n = 4 * y + z;
                f[y & 1][z] = *(const i32x4 *)(kt + k_at[n / SR] + 32 * (n % SR) * 2 * D);
            }
        };
        read_k(0);
#pragma unroll
        for (int y = 0; y < KS; ++y) {
            if (y + 1 < KS)
                read_k(y + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                const int n = 4 * y + z;
                s[n % SR] = E::mma(f[y & 1][z], Q[n / SR], s[n % SR]);
            }
        }
        if (masked) {
            // bit 8 (r / 4) + r % 4 of a word: this lane's row in register r
            const uint64_t v = (there & (tail ? seen64(a, b, rows, tok, row0) : ~(uint64_t)0)) >>
                               (rw * WR + 4 * half);
#pragma unroll
            for (int x = 0; x < SR; ++x) {
                const uint32_t seen = (uint32_t)(v >> (32 * x));
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[x][e] = seen & (1u << (8 * (e >> 2) + (e & 3))) ? s[x][e] : -INFINITY;
            }
            asm volatile("");           // (a branch, not selects in every round)
        }
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < SR; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                top = fmaxf(top, s[x][e]);
        // m follows the maximum only once a score is 2^LATE times the weight of m's: the
        // exponentials then stay below 2^LATE (times 2^LATE_LIFT), inside the 16-bit types, and
        // the sums are rescaled in few rounds instead of most (32 queries are in a wave)
        if (__any(top * a.scale2 > m * a.scale2 + E::LATE)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m_new = fmaxf(m, top);
            const float shrink =
                exp2_(m * a.scale2 - (m_new == -INFINITY ? 0.f : m_new * a.scale2));
            m = m_new;
            l *= shrink;
#pragma unroll
            for (int y = 0; y < DC; ++y)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    O[y][e] *= shrink;
        }
        const float base = (m == -INFINITY ? 0.f : m * a.scale2) - E::LATE_LIFT;
        i32x4 P[SR][2];
#pragma unroll
        for (int x = 0; x < SR; ++x) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[x][e] = exp2_(__builtin_fmaf(s[x][e], a.scale2, -base));
                l += s[x][e];
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                typename E::eight p8;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    p8[e] = (typename E::one)s[x][8 * y + e];
                P[x][y] = __builtin_bit_cast(i32x4, p8);
            }
        }
        // as above with V: the fragments of 128 columns (16 rows) at a time
        constexpr int VS = 2 * SR * DC / 4 > 0 ? 2 * SR * DC / 4 : 1, VG = 2 * SR * DC / VS;
        auto read_v = [&](int y) {
#pragma unroll
            for (int z = 0; z < VG; ++z) {
                const int n = VG * y + z;
                const uint8_t *at = kt + 16 * (n / DC) * 2 * D;
                f[y & 1][z] = column8(at + v_at[n % DC][0], at + v_at[n % DC][1]);
            }
        };
        read_v(0);
#pragma unroll
        for (int y = 0; y < VS; ++y) {
            if (y + 1 < VS)
                read_v(y + 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int z = 0; z < VG; ++z) {
                const int n = VG * y + z;
                O[n % DC] = E::mma(f[y & 1][z], P[n / DC / 2][n / DC % 2], O[n % DC]);
            }
        }
        there = there1;
        __syncthreads();
    };
    for (uint32_t i = 0; i < n_tiles; i += 2) {
        round(i, std::integral_constant<uint32_t, 0>());
        if (i + 1 >= n_tiles)
            break;
        round(i + 1, std::integral_constant<uint32_t, 1>());
    }

    // join the halves of a query, then (QW = 2) the two waves of its rows; the scale
    // 2^LATE_LIFT ends here
    m *= a.scale2;
    l += __shfl_xor(l, 32);
    if constexpr (E::LATE_LIFT != 0) {
        constexpr float DOWN = 1.f / (1 << E::LATE_LIFT);
        l *= DOWN;
#pragma unroll
        for (int z = 0; z < DC; ++z)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                O[z][e] *= DOWN;
    }
    if constexpr (RW == 2) {
        if (half == 0) {
            stat[wave][q32][0] = m;
            stat[wave][q32][1] = l;
        }
        float *sums = (float *)lds + qw * (16 * DC * 64);
        __syncthreads();
        const float m2 = stat[wave ^ QW][q32][0], l2 = stat[wave ^ QW][q32][1];
        const float all = fmaxf(m, m2), base = all == -INFINITY ? 0.f : all;
        const float f = exp2_(m - base);
        l = l * f + l2 * exp2_(m2 - base);
        m = all;
#pragma unroll
        for (int z = 0; z < DC; ++z)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                O[z][e] *= f;
                if (rw == 1)
                    sums[(16 * z + e) * 64 + lane] = O[z][e];
            }
        __syncthreads();
        if (rw == 1)
            return;
#pragma unroll
        for (int z = 0; z < DC; ++z)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                O[z][e] += sums[(16 * z + e) * 64 + lane];
    }
    if (r_mine >= q_rows)
        return;
    const uint32_t u = a.by_group.quot(r_mine);
    const uint64_t row = ((uint64_t)b * a.t + u) * a.q_heads + h * a.group + (r_mine - a.by_group.quot(r_mine) * a.group);
    const uint64_t part = ((uint64_t)slot * units + unit) * QT + 32 * qw + q32;
    if (odd_any && live)
        own_rows(a, b, h, rows, tok, from, to, [&](const uint16_t *v) {
#pragma unroll
            for (int z = 0; z < DC; ++z)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const uint32_t c = 32 * z + 8 * (e >> 2) + 4 * half + (e & 3);
                    if (FIT == FIT_WHOLE || c < d)
                        O[z][e] += odd_part<DT>(v[c]);
                }
        });
    const bool some = live && l != 0.f;
    const float inv = some ? 1.f / l : 0.f;
#pragma unroll
    for (int z = 0; z < DC; ++z)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t c = 32 * z + 8 * x + 4 * half;
            const f32x4 o = {O[z][4 * x], O[z][4 * x + 1], O[z][4 * x + 2], O[z][4 * x + 3]};
            if (shares > 1) {
                *(f32x4 *)(a.part_o + part * D + c) = o;
            } else {
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
                    if (FIT == FIT_WHOLE || c + e < d)
                        a.out[row * d + c + e] = __builtin_bit_cast(
                            uint16_t, (typename E::one)(some ? o[e] * inv : 0.f));
            }
        }
    if (half == 0) {
        if (shares > 1) {
            a.part_ml[part * 2] = m;
            a.part_ml[part * 2 + 1] = l;
        } else {
            a.lse[row] = some ? (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : -INFINITY;
        }
    }
}

// Joins the shares of query row `row` of the batch, if it has more than one, by T = 64 or 256
// threads.  Groups of D / 4 of them take every 4 T / D-th share, four elements a thread; the
// groups' sums join through LDS.  A wave a row where there are many rows (8192 rows of
// 8 shares: 15 -> 9 us), a workgroup where there are few (64 rows of 33 shares: 15 -> 5).
template <int DT, uint32_t T>
__device__ __forceinline__ void join_row(const Attend &a, uint32_t QT, uint32_t D, uint64_t row)
{
    typedef Elem<DT> E;
    __shared__ f32x4 sums[256];
    __shared__ float ls[4][16];
    const uint32_t lane = threadIdx.x & 63, tid = threadIdx.x % T, mine = threadIdx.x / T;
    const uint32_t head = (uint32_t)(row % a.q_heads);
    const uint32_t u = (uint32_t)(row / a.q_heads % a.t), b = (uint32_t)(row / a.q_heads / a.t);
    const uint32_t slot = a.plan[2 * b], shares = a.plan[2 * b + 1];
    if (shares <= 1)
        return;
    const uint32_t h = head / a.group, r = u * a.group + head % a.group;
    float top = -INFINITY;
    for (uint32_t s = lane; s < shares; s += 64)
        top = fmaxf(top, a.part_ml[2 * part_of(a, slot + s, h, r, QT)]);
    top = max_all(top);
    const float base = top == -INFINITY ? 0.f : top;
    const uint32_t per = D / 4, c = 4 * (tid % per), groups = T / per;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll 4
    for (uint32_t s = tid / per; s < shares; s += groups) {
        const uint64_t p = part_of(a, slot + s, h, r, QT);
        const f32x2 ml = *(const f32x2 *)(a.part_ml + 2 * p);
        const float f = exp2_(ml[0] - base);
        o += *(const f32x4 *)(a.part_o + p * D + c) * f;
        l += ml[1] * f;
    }
    if (tid % per == 0)
        ls[mine][tid / per] = l;
    sums[threadIdx.x] = o;
    if (T == 256)
        __syncthreads();
    else
        wave_sync();
    if (tid >= per)
        return;
    l = 0.f;
    o = f32x4{0.f, 0.f, 0.f, 0.f};
    for (uint32_t g = 0; g < groups; ++g) {
        o += sums[mine * T + g * per + tid];
        l += ls[mine][g];
    }
    const bool live = u < rows_of(a, b).count && l != 0.f;
    const float inv = live ? 1.f / l : 0.f;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e)
        if (c + e < a.c.d)
            a.out[row * a.c.d + c + e] =
                __builtin_bit_cast(uint16_t, (typename E::one)(live ? o[e] * inv : 0.f));
    if (tid == 0)
        a.lse[row] = live ? (top + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : -INFINITY;
}

// Weights of 1024 columns from the scores that the split kernel left (16 query rows at
// most): w_out = w_in + sum over the rows of 2^(score - lse).  The rows' lse comes from
// the shares, as in join_row, which may not have run yet.
__device__ __forceinline__ void weigh_scores(const Attend &a, uint32_t QT, uint32_t part)
{
    __shared__ float lse2[AT_Q];
    const uint32_t strips = (uint32_t)((a.w_cols + 1023) / 1024);
    const uint32_t bh = part / strips, n0 = part % strips * 1024 + 4 * threadIdx.x;
    const uint32_t h = bh % a.c.heads, b = bh / a.c.heads, q_rows = a.t * a.group;
    const Rows rows = rows_of(a, b);
    const uint32_t slot = a.plan[2 * b], shares = a.plan[2 * b + 1];
    const bool any = part % strips * 1024 < rows.end;
    if (any) {
        // 16 threads a row
        const uint32_t r = threadIdx.x >> 4, x = threadIdx.x & 15;
        float y = INFINITY;     // weighs nothing
        if (r < q_rows && r / a.group < rows.count) {
            if (shares > 1) {
                float top = -INFINITY, l = 0.f;
                for (uint32_t s = x; s < shares; s += 16)
                    top = fmaxf(top, a.part_ml[2 * part_of(a, slot + s, h, r, QT)]);
#pragma unroll
                for (int o = 1; o < 16; o <<= 1)
                    top = fmaxf(top, __shfl_xor(top, o));
                for (uint32_t s = x; s < shares; s += 16) {
                    const f32x2 ml = *(const f32x2 *)(a.part_ml + 2 * part_of(a, slot + s, h, r, QT));
                    l += ml[1] * exp2_(ml[0] - (top == -INFINITY ? 0.f : top));
                }
#pragma unroll
                for (int o = 1; o < 16; o <<= 1)
                    l += __shfl_xor(l, o);
                y = l == 0.f ? INFINITY : top + __builtin_amdgcn_logf(l);
            } else {
                y = a.lse[((uint64_t)b * a.t + r / a.group) * a.q_heads + h * a.group + r % a.group] *
                    1.4426950408889634f;
                y = y == -INFINITY ? INFINITY : y;
            }
        }
        if (x == 0)
            lse2[r] = y;
    }
    __syncthreads();
    if (n0 >= a.w_cols)
        return;
    f32x4 w = {0.f, 0.f, 0.f, 0.f};
    if (n0 < rows.end) {
        const float *s = a.scores + (uint64_t)bh * q_rows * a.s_cols + n0;
#pragma unroll 4
        for (uint32_t r = 0; r < q_rows; ++r) {
            const float y = lse2[r];
            const f32x4 x = *(const f32x4 *)(s + (uint64_t)r * a.s_cols);
            if (y != INFINITY)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] += x[e] == -INFINITY ? 0.f : exp2_(x[e] - y);
        }
    }
    const uint64_t at = (uint64_t)bh * a.w_cols + n0;
#pragma unroll
    for (uint32_t e = 0; e < 4; ++e)
        if (n0 + e < a.w_cols)
            a.w_out[at + e] = (a.w_in ? a.w_in[at + e] : 0.f) + (n0 + e < rows.end ? w[e] : 0.f);
}

// What is left once the shares are there: the first `joins` workgroups join query rows (one each,
// or four), the others weigh columns from the scores, strips `first` on.
template <int DT>
__global__ void __launch_bounds__(256) attend_join(const Attend a, uint32_t QT, uint32_t D,
                                                   uint32_t joins, uint32_t first, bool four)
{
    if (blockIdx.x >= joins) {
        weigh_scores(a, QT, first + (blockIdx.x - joins));
    } else if (!four) {
        join_row<DT, 256>(a, QT, D, blockIdx.x);
    } else {
        const uint64_t row = (uint64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (row < (uint64_t)a.c.batch * a.t * a.q_heads)
            join_row<DT, 64>(a, QT, D, row);
    }
}

// Weights: w_out[b, h, n] = w_in[b, h, n] + sum over the query rows r that read head h of
// exp(s_rn - lse_r).  A wave holds 32 WT key rows in operand layout and runs
// through the query rows, 64 of them in LDS at a time: S = Q K^T leaves key row l % 32 in
// lane l with query rows 8 (r / 4) + 4 (l / 32) + r % 4 in register r, so the sum stays in
// the lane until the end.  Two buffers of query rows, the next one's on their way
// while one is worked on.
template <int DT, int DC, int FIT>
__global__ void __launch_bounds__(256) attend_weights(const Attend a)
{
    typedef Elem<DT> E;
    constexpr uint32_t D = 32 * DC, CPR = 4 * DC, QS = DC == 8 ? 32 : 64, WT = DC == 8 ? 1 : 2;
    constexpr uint32_t WROWS = 32 * WT, QB = QS * D * 2, RPL = 256 / CPR;
    constexpr int NL = QS * CPR / 256;
    __shared__ __align__(16) uint8_t qs[2 * QB];
    __shared__ __align__(16) float lse2[2][QS];
    __shared__ uint64_t vis[4][QS];
    const uint32_t lane = threadIdx.x & 63, tid = threadIdx.x;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t l32 = lane & 31, half = lane >> 5, d = a.c.d;
    const uint32_t h = blockIdx.y % a.c.heads, b = blockIdx.y / a.c.heads;
    const uint32_t block0 = blockIdx.x * 4 * WROWS, row0 = block0 + wave * WROWS;
    const Rows rows = rows_of(a, b);
    const uint32_t q_rows = rows.count * a.group;
    float w[WT] = {};
    if (block0 < rows.end && q_rows > 0) {
        const uint32_t n = row0 + (lane & (WROWS - 1));
        const Place p = n < rows.end ? place_of(a.c, b, n) : Place{-1, 0u};
        const uint64_t there = __ballot(p.page >= 0);
        const bool masked = row0 + WROWS > rows.len || there != ~(uint64_t)0;
        const int64_t off =
            p.page < 0 ? 0 : (int64_t)p.page * a.c.k_page + (int64_t)p.slot * a.c.k_row;
        i32x4 K[WT][2 * DC];
#pragma unroll
        for (int t = 0; t < (int)WT; ++t) {
            const uint16_t *r =
                a.c.k + (int64_t)h * a.c.k_head + shfl64(off, (int)l32 + 32 * t) + 8 * half;
#pragma unroll
            for (int k = 0; k < 2 * DC; ++k)
                K[t][k] = load_fit<FIT>(r + 16 * k, (int)d - (int)(16 * k + 8 * half));
        }
        uint32_t q_at[2 * DC];      // chunk 2 k + half of query row l32 (the same for every 32)
#pragma unroll
        for (uint32_t k = 0; k < 2 * DC; ++k)
            q_at[k] = l32 * (2 * D) + 16 * swz<DC>(l32, 2 * k + half);
        // query rows r0 .. r0 + QS - 1 to registers, then to LDS; rows past the end repeat the
        // last one and weigh nothing
        const uint32_t row_at = tid / CPR, chunk = tid % CPR;
        i32x4 qr[NL];
        float lr = 0.f;
        bool lr_there = false;
        auto fetch = [&](uint32_t r0) {
#pragma unroll
            for (int x = 0; x < NL; ++x) {
                uint32_t r = r0 + RPL * x + row_at;
                r = r < q_rows ? r : q_rows - 1;
                const uint32_t u = a.by_group.quot(r);
                qr[x] = load_fit<FIT>(a.q + (int64_t)b * a.q_seq + (int64_t)u * a.q_tok +
                                  (int64_t)(h * a.group + r - u * a.group) * a.q_head + 8 * chunk,
                              (int)d - (int)(8 * chunk));
            }
            uint32_t r = r0 + (tid & (QS - 1));
            lr_there = r < q_rows;
            r = lr_there ? r : q_rows - 1;
            const uint32_t u = a.by_group.quot(r);
            lr = a.lse[((uint64_t)b * a.t + u) * a.q_heads + h * a.group + r - u * a.group];
        };
        auto stash = [&](uint32_t buf) {
            const int flip = a.negate ? (int)0x80008000 : 0;    // (as load_q8)
#pragma unroll
            for (int x = 0; x < NL; ++x) {
                const uint32_t r = RPL * x + row_at;
                *(i32x4 *)(qs + buf * QB + r * (2 * D) + 16 * swz<DC>(r, chunk)) = qr[x] ^ flip;
            }
            if (tid < QS)
                lse2[buf][tid] = lr_there && lr != -INFINITY ? lr * 1.4426950408889634f : INFINITY;
        };
        wait_loads();
        fetch(0);
        stash(0);
        __syncthreads();
        uint32_t buf = 0;
        for (uint32_t r0 = 0; r0 < q_rows; r0 += QS, buf ^= 1) {
            fetch(r0 + QS);
            if (masked)
                seen_rows(a, b, rows, r0, QS, q_rows, row0, there, vis[wave]);
            const uint8_t *qt = qs + buf * QB;
#pragma unroll 1
            for (uint32_t q0 = 0; q0 < QS; q0 += 32) {
                if (r0 + q0 >= q_rows)
                    break;
                f32x16 s[WT];
#pragma unroll
                for (int t = 0; t < (int)WT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        s[t][e] = 0.f;
                i32x4 qf[2 * DC];
#pragma unroll
                for (uint32_t k = 0; k < 2 * DC; ++k)
                    qf[k] = *(const i32x4 *)(qt + q0 * (2 * D) + q_at[k]);
                f32x4 z[4];
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    z[x] = *(const f32x4 *)(lse2[buf] + q0 + 8 * x + 4 * half);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (uint32_t k = 0; k < 2 * DC; ++k)
#pragma unroll
                    for (int t = 0; t < (int)WT; ++t)
                        s[t] = E::mma(qf[k], K[t][k], s[t]);
                if (masked) {
#pragma unroll
                    for (int t = 0; t < (int)WT; ++t)
                        w[t] += weigh_seen(s[t], z, a.scale2, vis[wave] + q0 + 4 * half, 32 * t + l32);
                } else {
#pragma unroll
                    for (int t = 0; t < (int)WT; ++t)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            w[t] += exp2_(__builtin_fmaf(s[t][e], a.scale2, -z[e >> 2][e & 3]));
                }
            }
            stash(buf ^ 1);
            __syncthreads();
        }
    }
#pragma unroll
    for (int t = 0; t < (int)WT; ++t) {
        w[t] += __shfl_xor(w[t], 32);
        const uint64_t n = (uint64_t)row0 + 32 * t + l32;
        if (half == 0 && n < a.w_cols) {
            const uint64_t at = ((uint64_t)b * a.c.heads + h) * a.w_cols + n;
            a.w_out[at] = (a.w_in ? a.w_in[at] : 0.f) + w[t];
        }
    }
}

// The same with all query rows in LDS (64 KiB at most: 256 rows of 128 elements), so that a
// workgroup can stay: it takes a share of a sequence's rows for one head, as the attention
// kernels do, its waves 32 WT rows at a time in turn, the next rows' keys on their way to
// registers while these are multiplied.  (With a workgroup for every 256 rows the
// keys were waited for at each start: 131072 rows of 8 heads x 256 query rows, 185 us; 64
// rows at a time, 121 us, need twice the registers; 32, 96 us (118 in a long row of calls): matrix
// cores 31% busy beside an exponential, a product and a sum per score.  64 query rows on 58000 rows
// of 8 heads: 25 us, 4.8 TB/s, bound by HBM.)
template <int DC>
constexpr uint32_t kWeighRows = DC == 8 ? 128 : 256;

template <int DT, int DC, int FIT>
__global__ void __launch_bounds__(256, 2) attend_weights_held(const Attend a)
{
    typedef Elem<DT> E;
    constexpr uint32_t D = 32 * DC, CPR = 4 * DC, QM = kWeighRows<DC>, WT = 1;
    constexpr uint32_t WROWS = 32 * WT;
    __shared__ __align__(16) uint8_t qs[QM * D * 2];
    __shared__ __align__(16) float lse2[QM];
    __shared__ uint64_t vis[4][QM];
    const uint32_t lane = threadIdx.x & 63, tid = threadIdx.x;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t l32 = lane & 31, half = lane >> 5, d = a.c.d;
    const uint32_t h = blockIdx.x % a.c.heads, slot = blockIdx.x / a.c.heads;
    Share sh;
    if (slot >= a.slots || !find_share(a, slot, &sh))
        return;
    const uint32_t b = __builtin_amdgcn_readfirstlane(sh.b);
    const Rows rows = {(uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.len),
                       (uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.count),
                       (uint32_t)__builtin_amdgcn_readfirstlane(sh.rows.end)};
    const uint32_t q_rows = rows.count * a.group;
    const uint32_t end = rows.end < a.w_cols ? rows.end : (uint32_t)a.w_cols;
    const uint32_t from = __builtin_amdgcn_readfirstlane(sh.first) * AT_ROWS;
    const uint32_t last = __builtin_amdgcn_readfirstlane(sh.last) * AT_ROWS;
    const uint32_t to = q_rows == 0 ? from : (last < end ? last : end);
    const uint64_t at0 = ((uint64_t)b * a.c.heads + h) * a.w_cols;

    // columns that no row of this call weighs, evenly over the sequence's shares
    const uint32_t rest = q_rows == 0 ? 0 : end;
    const uint64_t n_rest = a.w_cols - rest;
    for (uint64_t n = rest + n_rest * sh.share / sh.shares + tid;
         n < rest + n_rest * (sh.share + 1) / sh.shares; n += 256)
        if (!a.w_in)
            a.w_out[at0 + n] = 0.f;
        else if (a.w_in != a.w_out)
            a.w_out[at0 + n] = a.w_in[at0 + n];
    if (from >= to)
        return;

    // query rows and their lse; rows past the end repeat the last one (zeros times an infinite
    // key would be NaN, which no lse takes back to 0) and weigh nothing
    const uint32_t n_q = (q_rows + 31) / 32;
    const int flip = a.negate ? (int)0x80008000 : 0;    // (as load_q8)
    for (uint32_t i0 = tid; i0 < n_q * 32 * CPR; i0 += 4 * 256) {
        i32x4 v[4];
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) {      // (four loads at once)
            uint32_t r = (i0 + 256 * x) / CPR;
            const uint32_t c = (i0 + 256 * x) % CPR;
            r = r < q_rows ? r : q_rows - 1;
            const uint32_t u = a.by_group.quot(r);
            v[x] = load_fit<FIT>(a.q + (int64_t)b * a.q_seq + (int64_t)u * a.q_tok +
                             (int64_t)(h * a.group + r - u * a.group) * a.q_head + 8 * c,
                         (int)d - (int)(8 * c));
        }
#pragma unroll
        for (uint32_t x = 0; x < 4; ++x) {
            const uint32_t r = (i0 + 256 * x) / CPR, c = (i0 + 256 * x) % CPR;
            if (r < n_q * 32)
                *(i32x4 *)(qs + r * (2 * D) + 16 * swz<DC>(r, c)) = v[x] ^ flip;
        }
    }
    for (uint32_t r = tid; r < n_q * 32; r += 256) {
        float x = INFINITY;
        if (r < q_rows) {
            const uint32_t u = a.by_group.quot(r);
            x = a.lse[((uint64_t)b * a.t + u) * a.q_heads + h * a.group + r - u * a.group];
            x = x == -INFINITY ? INFINITY : x * 1.4426950408889634f;
        }
        lse2[r] = x;
    }
    uint32_t q_at[2 * DC];      // chunk 2 k + half of query row l32 (the same for every 32)
#pragma unroll
    for (uint32_t k = 0; k < 2 * DC; ++k)
        q_at[k] = l32 * (2 * D) + 16 * swz<DC>(l32, 2 * k + half);

    const uint16_t *kb = a.c.k + (int64_t)h * a.c.k_head + 8 * half;
    const uint32_t n_blk = (to - from + WROWS - 1) / WROWS;
    auto entry = [&](uint32_t i) {
        return entry_of(a.c, a.len, b, from + i * WROWS + (lane & (WROWS - 1)));
    };
    i32x4 K[2][WT][2 * DC];
    auto load_k = [&](const Place &p, auto set_) {      // absent rows read page 0, row 0
        constexpr int set = decltype(set_)::value;
        const int64_t off =
            p.page < 0 ? 0 : (int64_t)p.page * a.c.k_page + (int64_t)p.slot * a.c.k_row;
#pragma unroll
        for (int t = 0; t < (int)WT; ++t) {
            const uint16_t *r = kb + shfl64(off, (int)l32 + 32 * t);
#pragma unroll
            for (int k = 0; k < 2 * DC; ++k)
                K[set][t][k] = load_fit<FIT>(r + 16 * k, (int)d - (int)(16 * k + 8 * half));
        }
    };
    auto add = [&](uint32_t n) -> float {               // (a load whether it is needed or not)
        n = n < to ? n : to - 1;
        return a.w_in ? a.w_in[at0 + n] : 0.f;
    };
    Place cur = place_of(a.c, b, entry(wave), to);
    Entry ahead = entry(wave + 4);
    load_k(cur, std::integral_constant<int, 0>());
    __syncthreads();
    auto round = [&](uint32_t i, auto set_) {
        constexpr int set = decltype(set_)::value;
        const Place nxt = place_of(a.c, b, ahead, to);
        ahead = entry(i + 8);
        const uint32_t row0 = from + i * WROWS;
        const uint64_t there = __ballot(cur.page >= 0);
        const bool masked = row0 + WROWS > rows.len || there != ~(uint64_t)0;
        float w[WT], w0[WT];
#pragma unroll
        for (int t = 0; t < (int)WT; ++t) {
            w[t] = 0.f;
            w0[t] = add(row0 + 32 * t + l32);
        }
        load_k(nxt, std::integral_constant<int, 1 - set>());
        if (masked)
            seen_rows(a, b, rows, 0, n_q * 32, q_rows, row0, there, vis[wave]);
        i32x4 qf[2 * DC];
        auto read_q = [&](uint32_t q0) {
#pragma unroll
            for (uint32_t k = 0; k < 2 * DC; ++k)
                qf[k] = *(const i32x4 *)(qs + q0 * (2 * D) + q_at[k]);
        };
        read_q(0);
#pragma unroll 1
        for (uint32_t q = 0; q < n_q; ++q) {
            const uint32_t q0 = 32 * q;
            f32x16 s[WT];
#pragma unroll
            for (int t = 0; t < (int)WT; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    s[t][e] = 0.f;
#pragma unroll
            for (uint32_t k = 0; k < 2 * DC; ++k)
#pragma unroll
                for (int t = 0; t < (int)WT; ++t)
                    s[t] = E::mma(qf[k], K[set][t][k], s[t]);
            __builtin_amdgcn_sched_barrier(0);
            read_q(q + 1 < n_q ? q0 + 32 : 0);
            f32x4 z[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                z[x] = *(const f32x4 *)(lse2 + q0 + 8 * x + 4 * half);
            if (masked) {
#pragma unroll
                for (int t = 0; t < (int)WT; ++t)
                    w[t] += weigh_seen(s[t], z, a.scale2, vis[wave] + q0 + 4 * half, 32 * t + l32);
            } else {
#pragma unroll
                for (int t = 0; t < (int)WT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        w[t] += exp2_(__builtin_fmaf(s[t][e], a.scale2, -z[e >> 2][e & 3]));
            }
        }
#pragma unroll
        for (int t = 0; t < (int)WT; ++t) {
            w[t] += __shfl_xor(w[t], 32);
            const uint32_t n = row0 + 32 * t + l32;
            if (half == 0 && n < to)
                a.w_out[at0 + n] = w0[t] + w[t];
        }
        cur = nxt;
    };
    for (uint32_t i = wave; i < n_blk; i += 8) {
        round(i, std::integral_constant<int, 0>());
        if (i + 4 >= n_blk)
            break;
        round(i + 4, std::integral_constant<int, 1>());
    }
}

constexpr uint32_t kStrips = 1u << 20;     // of columns that one launch weighs at most

// The kernel for tiles of qt query rows.
template <int DT, int DC, int FIT>
void (*attend_kernel(uint32_t qt))(const Attend)
{
    if (qt == 16)
        return attend_split<DT, DC, 1, FIT>;
    if (qt == 32)
        return attend_split<DT, DC, 2, FIT>;
    if (qt == 64 && DC != 8)
        return attend_tiles<DT, DC, DC != 8 ? 2 : 4, FIT>;
    if (qt == 256 && DC != 8)
        return attend_tiles<DT, DC, DC != 8 ? 8 : 4, FIT>;
    return attend_tiles<DT, DC, 4, FIT>;
}

template <int DT, int DC, int FIT>
hipError_t launch_attend_dc(const Attend &a, hipStream_t s)
{
    const uint32_t qt = attend_tile_rows(a.t * a.group, a.c.d);
    const uint64_t rows = (uint64_t)a.c.batch * a.t * a.q_heads;
    hipError_t e;
    if (rows) {
        // (a multiple of 8 workgroups: the tiled kernel deals them out by XCD)
        const dim3 grid((a.slots * a.c.heads * a.tiles + 7) / 8 * 8);
        attend_kernel<DT, DC, FIT>(qt)<<<grid, qt == 256 ? 512 : 256, 0, s>>>(a);
        if ((e = hipGetLastError()) != hipSuccess)
            return e;
        if (a.scores || !(a.arrivals || a.whole)) {
            const uint32_t strips =
                a.scores ? (uint32_t)((a.w_cols + 1023) / 1024) * a.c.batch * a.c.heads : 0;
            const bool four = rows > 1024;
            uint32_t joins = a.whole ? 0 : (uint32_t)(four ? (rows + 3) / 4 : rows), first = 0;
            do {        // (a launch holds fewer than 2^32 threads)
                const uint32_t left = strips - first, now = left < kStrips ? left : kStrips;
                attend_join<DT><<<dim3(joins + now), 256, 0, s>>>(a, qt, 32 * DC, joins, first, four);
                if ((e = hipGetLastError()) != hipSuccess)
                    return e;
                first += now;
                joins = 0;
            } while (first < strips);
            if (a.scores)
                return e;
        }
    }
    if (!a.w_out || !a.w_cols)
        return hipSuccess;
    if (a.t * a.group <= kWeighRows<DC>) {
        Attend w = a;       // (its own cut of the rows: a workgroup a share and head)
        w.want = a.w_want;
        w.slots = a.w_want > a.c.batch ? a.w_want : a.c.batch;
        attend_weights_held<DT, DC, FIT><<<dim3(w.slots * a.c.heads), 256, 0, s>>>(w);
        return hipGetLastError();
    }
    const uint32_t w_rows = DC == 8 ? 128 : 256;
    const dim3 wg((uint32_t)((a.w_cols + w_rows - 1) / w_rows), a.c.batch * a.c.heads);
    attend_weights<DT, DC, FIT><<<wg, 256, 0, s>>>(a);
    return hipGetLastError();
}

template <int DT, int DC>
hipError_t launch_attend_fit(const Attend &a, hipStream_t s)
{
    if (a.c.d == 32 * DC)
        return launch_attend_dc<DT, DC, FIT_WHOLE>(a, s);
    return a.c.d % 8 == 0 ? launch_attend_dc<DT, DC, FIT_CHUNKS>(a, s)
                          : launch_attend_dc<DT, DC, FIT_ANY>(a, s);
}

template <int DT>
hipError_t launch_attend(const Attend &a, hipStream_t s)
{
    const uint32_t d = a.c.d;
    return d <= 64 ? launch_attend_fit<DT, 2>(a, s)
                   : (d <= 128 ? launch_attend_fit<DT, 4>(a, s) : launch_attend_fit<DT, 8>(a, s));
}

// Workgroups of the kernel for d and qt that one CU holds at once.
template <int DT>
int attend_occupancy(uint32_t d, uint32_t qt)
{
    static int known[3][5];
    int &n = known[d <= 64 ? 0 : (d <= 128 ? 1 : 2)][qt == 16 ? 0 : (qt == 32 ? 1 : (qt == 64 ? 2 : (qt == 128 ? 3 : 4)))];
    if (n == 0) {
        const void *k = d <= 64 ? (const void *)attend_kernel<DT, 2, FIT_ANY>(qt)
                                : (d <= 128 ? (const void *)attend_kernel<DT, 4, FIT_ANY>(qt)
                                            : (const void *)attend_kernel<DT, 8, FIT_ANY>(qt));
        int x = 0;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&x, k, qt == 256 ? 512 : 256, 0) != hipSuccess)
            (void)hipGetLastError();
        n = x > 0 ? x : 1;
    }
    return n;
}

}  // namespace sjc
