// sj_evict.hip -- eviction from a cache by accumulated weight (sj_cache_evict): which
// rows stay, then their copies.
#include "sj_cache.h"

namespace sjc {

namespace {

// Unsigned key in the order of the weights: NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float w)
{
    if (w != w)
        w = -INFINITY;
    const uint32_t u = __float_as_uint(w + 0.f);   // (-0 + 0 = 0)
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr uint32_t EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64, EV_BINS = 2048;

__device__ __forceinline__ float weight_at(const Evict &e, const float *w, uint32_t n)
{
    return n < e.w_cols ? w[n] : 0.f;
}

// Writes kept row number j of a set.
__device__ __forceinline__ void keep_row(const Evict &e, uint64_t set, const float *w, uint32_t j,
                                         uint32_t n)
{
    e.index[set * e.keep + j] = (int32_t)n;
    if (e.w_out && j < e.w_out_cols)
        e.w_out[set * e.w_out_cols + j] = weight_at(e, w, n);
}

// The kept rows of one set (a sequence and a head, or a sequence), in order: a
// workgroup a set.  Radix selection of the last weight that stays: three
// histograms of 11, 11 and 10 key bits, each over the rows whose higher bits are
// those of the key sought; then every wave counts the kept rows and the ties of its
// own stretch of rows, and writes its rows at the sum of the waves before it.
__global__ void __launch_bounds__(EV_THREADS) evict_select(const Evict e)
{
    __shared__ uint32_t hist[EV_BINS];
    __shared__ uint32_t above[EV_WAVES], ties[EV_WAVES], found[2];
    const uint64_t set = blockIdx.x;
    const uint32_t b = (uint32_t)(set / e.sets);
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t n = clamp_rows(e.len[b], e.src.room);
    const uint32_t m = n < e.keep ? n : e.keep;
    const float *w = e.weight + set * e.w_cols;
    if (threadIdx.x == 0 && set % e.sets == 0)
        e.new_len[b] = (int32_t)m;
    for (uint32_t j = m + threadIdx.x; j < e.keep; j += EV_THREADS)
        e.index[set * e.keep + j] = -1;
    if (e.w_out)
        for (uint64_t j = m + threadIdx.x; j < e.w_out_cols; j += EV_THREADS)
            e.w_out[set * e.w_out_cols + j] = 0.f;
    if (n <= e.keep) {
        for (uint32_t j = threadIdx.x; j < m; j += EV_THREADS)
            keep_row(e, set, w, j, j);
        return;
    }
    const uint32_t lo = e.sink, hi = n - e.recent;   // rows between compete
    uint32_t need = e.keep - e.sink - e.recent;      // of these stay (< hi - lo)
    uint32_t prefix = 0, known = 0;                  // the sought key's known top bits
    if (need > 0) {
        for (int step = 0; step < 3; ++step) {
            const uint32_t bits = step == 2 ? 10 : 11, shift = 32 - known - bits;
            const uint32_t bins = 1u << bits;
            for (uint32_t i = threadIdx.x; i < EV_BINS; i += EV_THREADS)
                hist[i] = 0;
            __syncthreads();
            for (uint32_t i = lo + threadIdx.x; i < hi; i += EV_THREADS) {
                const uint32_t key = order_key(weight_at(e, w, i));
                if (known == 0 || key >> (32 - known) == prefix)
                    atomicAdd(&hist[(key >> shift) & (bins - 1)], 1u);
            }
            __syncthreads();
            // the bin, from the top, in which the need-th key lies: one wave, 32 bins a lane
            if (wave == 0) {
                uint32_t sum = 0;
                const uint32_t per = bins / 64, top = bins - 1 - lane * per;
                for (uint32_t i = 0; i < per; ++i)
                    sum += hist[top - i];
                uint32_t incl = sum;
                for (int o = 1; o < 64; o <<= 1) {
                    const uint32_t y = __shfl_up(incl, o);
                    incl += (int)lane >= o ? y : 0;
                }
                if (need > incl - sum && need <= incl) {
                    uint32_t before = incl - sum;
                    for (uint32_t i = 0; i < per; ++i) {
                        const uint32_t c = hist[top - i];
                        if (need <= before + c) {
                            found[0] = top - i;
                            found[1] = need - before;
                            break;
                        }
                        before += c;
                    }
                }
            }
            __syncthreads();
            prefix = (prefix << bits) | found[0];
            need = found[1];
            known += bits;
            __syncthreads();
        }
    }
    // prefix is the last key that stays, need the number of its rows that do (the
    // lowest ones); with nothing to choose none does
    const bool none = known == 0;
    const uint32_t per = ((n + EV_WAVES - 1) / EV_WAVES + 63) & ~63u;
    const uint32_t from = wave * per < n ? wave * per : n, to = from + per < n ? from + per : n;
    uint32_t n_above = 0, n_ties = 0;
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
        const uint32_t i = i0 + lane;
        const bool mid = i >= lo && i < hi && i < to;
        const uint32_t key = mid && !none ? order_key(weight_at(e, w, i)) : 0;
        n_above += __popcll(__ballot(i < to && (!mid || (!none && key > prefix))));
        n_ties += __popcll(__ballot(mid && !none && key == prefix));
    }
    if (lane == 0) {
        above[wave] = n_above;
        ties[wave] = n_ties;
    }
    __syncthreads();
    uint32_t out = 0, tied = 0;      // kept rows and ties before this wave's
    for (uint32_t i = 0; i < wave; ++i) {
        out += above[i];
        tied += ties[i];
    }
    out += tied < need ? tied : need;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (uint32_t i0 = from; i0 < to; i0 += 64) {
        const uint32_t i = i0 + lane;
        const bool mid = i >= lo && i < hi && i < to;
        const uint32_t key = mid && !none ? order_key(weight_at(e, w, i)) : 0;
        const bool tie = mid && !none && key == prefix;
        const uint64_t tie_mask = __ballot(tie);
        const bool kept = i < to && (!mid || (!none && key > prefix) ||
                                     (tie && tied + __popcll(tie_mask & below) < need));
        const uint64_t kept_mask = __ballot(kept);
        if (kept)
            keep_row(e, set, w, out + __popcll(kept_mask & below), i);
        out += __popcll(kept_mask);
        tied += __popcll(tie_mask);
    }
}

// Copies the kept rows of one (sequence, head): each thread 16 bytes of a row of k and
// of v.  Bound by HBM.
__global__ void __launch_bounds__(256) evict_copy(const Evict e, uint32_t chunks, PageDiv by_chunks,
                                                  uint32_t rows_per)
{
    const uint32_t h = blockIdx.y % e.src.heads, b = blockIdx.y / e.src.heads;
    const uint32_t n = clamp_rows(e.len[b], e.src.room);
    const uint32_t m = n < e.keep ? n : e.keep;
    const uint32_t j0 = blockIdx.x * rows_per;
    const uint32_t rows = j0 >= m ? 0 : (m - j0 < rows_per ? m - j0 : rows_per);
    const int32_t *index =
        e.index + ((uint64_t)b * e.sets + (e.sets == 1 ? 0 : h)) * e.keep + j0;
    for (uint32_t i = threadIdx.x; i < rows * chunks; i += 256) {
        const uint32_t j = by_chunks.quot(i), c = 8 * (i - j * chunks);
        const Place to = place_of(e.dst, b, j0 + j);
        if (to.page < 0)
            continue;
        const Place from = place_of(e.src, b, (uint32_t)index[j]);
        const int left = (int)(e.src.d - c);
        i32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
        if (from.page >= 0) {
            k = load8(e.src.k + (int64_t)from.page * e.src.k_page + (int64_t)from.slot * e.src.k_row +
                          (int64_t)h * e.src.k_head + c,
                      left);
            v = load8(e.src.v + (int64_t)from.page * e.src.v_page + (int64_t)from.slot * e.src.v_row +
                          (int64_t)h * e.src.v_head + c,
                      left);
        }
        store8(const_cast<uint16_t *>(e.dst.k) + (int64_t)to.page * e.dst.k_page +
                   (int64_t)to.slot * e.dst.k_row + (int64_t)h * e.dst.k_head + c,
               k, left);
        store8(const_cast<uint16_t *>(e.dst.v) + (int64_t)to.page * e.dst.v_page +
                   (int64_t)to.slot * e.dst.v_row + (int64_t)h * e.dst.v_head + c,
               v, left);
    }
}

}  // namespace

hipError_t launch_evict(const Evict &e, int num_cus, hipStream_t s)
{
    (void)num_cus;
    evict_select<<<dim3(e.src.batch * e.sets), EV_THREADS, 0, s>>>(e);
    hipError_t err = hipGetLastError();
    const uint32_t most = e.keep < e.src.room ? e.keep : e.src.room;
    if (err != hipSuccess || most == 0)
        return err;
    const uint32_t chunks = (e.src.d + 7) / 8, rows_per = 64;
    evict_copy<<<dim3((most + rows_per - 1) / rows_per, e.src.batch * e.src.heads), 256, 0, s>>>(
        e, chunks, PageDiv::of(chunks), rows_per);
    return hipGetLastError();
}

}  // namespace sjc
