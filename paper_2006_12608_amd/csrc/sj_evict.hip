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

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
constexpr uint32_t EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64;
constexpr int EV_STEPS = 3;
// key bits of the three steps, from the top
__device__ __forceinline__ uint32_t step_bits(int step) { return step == 2 ? 10 : 11; }
__device__ __forceinline__ uint32_t bits_before(int step) { return 11 * step; }

// What one set (a sequence and a head, or a sequence) keeps of its n rows: all m = n, or the
// rows outside [lo, hi) and `need` of those inside.
struct Task {
    uint32_t n, m, lo, hi, need;
    uint64_t set;
    const float *w;
};

__device__ __forceinline__ Task task_of(const Evict &e, uint64_t set)
{
    Task t;
    t.set = set;
    t.w = e.weight + set * e.w_cols;
    t.n = clamp_rows(e.len[set / e.sets], e.src.room);
    t.m = t.n < e.keep ? t.n : e.keep;
    const bool all = t.n <= e.keep;
    t.lo = all ? t.n : e.sink;
    t.hi = all ? t.n : t.n - e.recent;
    t.need = all ? 0 : e.keep - e.sink - e.recent;
    return t;
}

// Weights of the rows from + 64 k + lane, k < PER, of a wave, loaded once and all
// at once (loads under conditions of their own wait for each other).
template <int PER>
struct Rows {
    float w[PER];
    __device__ __forceinline__ void load(const Evict &e, const Task &t, uint32_t from)
    {
        const uint32_t lane = threadIdx.x & 63, cols = (uint32_t)e.w_cols;
        const float *p = cols ? t.w : (const float *)e.len;     // (anything readable)
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t i = from + 64 * k + lane;
            w[k] = p[i < cols ? i : (cols ? cols - 1 : 0)];
        }
#pragma unroll
        for (int k = 0; k < PER; ++k)
            w[k] = from + 64 * k + lane < cols ? w[k] : 0.f;
    }
    // key of row i in w[k]; 0 outside [lo, hi) (below every key: -inf is 0x007fffff)
    __device__ __forceinline__ uint32_t key(const Task &t, int k, uint32_t i) const
    {
        return i >= t.lo && i < t.hi ? order_key(w[k]) : 0;
    }
    // adds the digit of `step` of every key whose higher bits are `prefix` to hist
    __device__ __forceinline__ void count(const Task &t, uint32_t *hist, uint32_t from, int step,
                                          uint32_t prefix) const
    {
        const uint32_t bits = step_bits(step), known = bits_before(step), shift = 32 - known - bits;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t x = key(t, k, from + 64 * k + (threadIdx.x & 63));
            if (x && (known == 0 || x >> (32 - known) == prefix))
                atomicAdd(&hist[(x >> shift) & ((1u << bits) - 1)], 1u);
        }
    }
};

// The bin, from the top, in which the need-th of all counted keys lies, and how many keys of
// that bin are still needed; thread t passes the counts of bins 2047 - 2 t and
// 2046 - 2 t.  Called by the whole workgroup.
__device__ __forceinline__ void find_bin(uint32_t c0, uint32_t c1, uint32_t need, uint32_t *bin,
                                         uint32_t *left)
{
    __shared__ uint32_t waves[EV_WAVES], found[2];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t incl = sum_upto(c0 + c1);
    if (lane == 63)
        waves[wave] = incl;
    __syncthreads();
    uint32_t before = incl - c0 - c1;
#pragma unroll
    for (uint32_t w = 0; w < EV_WAVES; ++w)
        before += w < wave ? waves[w] : 0;
    if (need > before && need <= before + c0 + c1) {
        const bool first = need <= before + c0;
        found[0] = EV_BINS - 1 - 2 * threadIdx.x - (first ? 0 : 1);
        found[1] = need - before - (first ? 0 : c0);
    }
    __syncthreads();
    *bin = found[0];
    *left = found[1];
    __syncthreads();
}

// Writes what the wave's rows keep: all outside [lo, hi) and, inside, the keys above `last` and
// of those equal to it the first `need` (over all waves).  Rows and ties before the
// workgroup's come in out0 and ties0.  Called by the whole workgroup.
template <int PER>
__device__ __forceinline__ void emit(const Evict &e, const Task &t, const Rows<PER> &rows,
                                     uint32_t from, uint32_t last, uint32_t need,
                                     uint32_t out0, uint32_t ties0)
{
    __shared__ uint32_t above[EV_WAVES], ties[EV_WAVES];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    uint32_t n_above = 0, n_ties = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const uint32_t i = from + 64 * k + lane;
        const bool mid = i >= t.lo && i < t.hi;
        const uint32_t x = rows.key(t, k, i);
        n_above += __popcll(__ballot(i < t.n && (!mid || (need && x > last))));
        n_ties += __popcll(__ballot(mid && need && x == last));
    }
    if (lane == 0) {
        above[wave] = n_above;
        ties[wave] = n_ties;
    }
    __syncthreads();
    uint32_t out = out0, tied = ties0;
    for (uint32_t w = 0; w < wave; ++w) {
        out += above[w];
        tied += ties[w];
    }
    out += tied < need ? tied : need;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const uint32_t i = from + 64 * k + lane;
        const bool mid = i >= t.lo && i < t.hi;
        const uint32_t x = rows.key(t, k, i);
        const bool tie = mid && need && x == last;
        const uint64_t tie_mask = __ballot(tie);
        const bool kept = i < t.n && (!mid || (need && x > last) ||
                                      (tie && tied + __popcll(tie_mask & below) < need));
        const uint64_t kept_mask = __ballot(kept);
        if (kept) {
            const uint32_t j = out + __popcll(kept_mask & below);
            e.index[t.set * e.keep + j] = (int32_t)i;
            if (e.w_out && j < e.w_out_cols)
                e.w_out[t.set * e.w_out_cols + j] = rows.w[k];
        }
        out += __popcll(kept_mask);
        tied += __popcll(tie_mask);
    }
}

// -1 and 0 past the kept rows, by `share` of `shares` workgroups; the new length.
__device__ __forceinline__ void pad(const Evict &e, const Task &t, uint32_t share, uint32_t shares)
{
    const uint32_t at = share * EV_THREADS + threadIdx.x, all = shares * EV_THREADS;
    if (at == 0 && t.set % e.sets == 0)
        e.new_len[t.set / e.sets] = (int32_t)t.m;
    for (uint64_t j = (uint64_t)t.m + at; j < e.keep; j += all)
        e.index[t.set * e.keep + j] = -1;
    if (e.w_out)
        for (uint64_t j = (uint64_t)t.m + at; j < e.w_out_cols; j += all)
            e.w_out[t.set * e.w_out_cols + j] = 0.f;
}

// The kept rows of one set, in order: a workgroup a set of up to EV_ONE rows, each wave a
// stretch of them, the weights in registers.  Radix selection of the last key that stays: three
// histograms of 11, 11 and 10 key bits, each over the keys whose higher bits are
// those of the key sought.  The weights are read once and all at once; what is left is the
// latency of the steps' barriers: 128 sets of 2500 to 16000 rows, 19 us (4 MB), 2 of 3000, 6.5.
template <int PER>
__global__ void __launch_bounds__(EV_THREADS) evict_select(const Evict e)
{
    __shared__ uint32_t hist[EV_BINS];
    const Task t = task_of(e, blockIdx.x);
    pad(e, t, 0, 1);
    const uint32_t from = (threadIdx.x >> 6) * 64 * PER;
    Rows<PER> rows;
    rows.load(e, t, from);
    uint32_t prefix = 0, need = t.need;
    if (need > 0)
        for (int step = 0; step < EV_STEPS; ++step) {
            hist[threadIdx.x] = 0;
            hist[threadIdx.x + EV_THREADS] = 0;
            __syncthreads();
            rows.count(t, hist, from, step, prefix);
            __syncthreads();
            uint32_t bin;
            find_bin(hist[EV_BINS - 1 - 2 * threadIdx.x], hist[EV_BINS - 2 - 2 * threadIdx.x], need,
                     &bin, &need);
            prefix = prefix << step_bits(step) | bin;
        }
    emit(e, t, rows, from, prefix, need, 0, 0);
}

// The same for more rows, a workgroup a chunk of EV_CHUNK: step s = 0, 1, 2 leaves the chunk's
// histogram, after finding the bin of step s - 1 from all chunks' (every workgroup by itself);
// step 3 writes the rows.  Two sets of 131072 rows: 28 us for the four launches against 209 with
// a workgroup a set; of 30000, one workgroup's 30 us are no more than the launches'.
template <int STEP>
__global__ void __launch_bounds__(EV_THREADS) evict_step(const Evict e)
{
    constexpr int PER = EV_CHUNK / EV_THREADS;
    __shared__ uint32_t hist[EV_BINS], sums[2];
    const Task t = task_of(e, blockIdx.y);
    const uint32_t chunk = blockIdx.x;
    if (STEP == 3)
        pad(e, t, chunk, e.chunks);
    if (chunk * EV_CHUNK >= t.n && STEP == 3)
        return;
    const uint32_t from = chunk * EV_CHUNK + (threadIdx.x >> 6) * 64 * PER;
    Rows<PER> rows;
    rows.load(e, t, from);
    uint32_t *const mine = e.state + (t.set * e.chunks + chunk) * 8;
    auto hist_of = [&](int step, uint32_t c) {
        return e.hist + ((t.set * EV_STEPS + step) * e.chunks + c) * EV_BINS;
    };
    uint32_t prefix = 0, need = t.need, out0 = 0, ties0 = 0;
    if (STEP > 0 && t.need > 0) {
        // the previous step's bin, and this chunk's keys above it
        if (STEP > 1) {
            prefix = mine[2 * (STEP - 2)];
            need = mine[2 * (STEP - 2) + 1];
        }
        const uint32_t b0 = EV_BINS - 1 - 2 * threadIdx.x;
        uint32_t c0 = 0, c1 = 0, before0 = 0, before1 = 0;
        for (uint32_t c8 = 0; c8 < e.chunks; c8 += 8) {
            u32x2 h[8];     // (eight loads at once)
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x)
                h[x] = *(const u32x2 *)(hist_of(STEP - 1, c8 + x < e.chunks ? c8 + x : 0) + b0 - 1);
#pragma unroll
            for (uint32_t x = 0; x < 8; ++x) {
                const bool in = c8 + x < e.chunks, early = c8 + x < chunk;
                c0 += in ? h[x][1] : 0;
                c1 += in ? h[x][0] : 0;
                before0 += early ? h[x][1] : 0;
                before1 += early ? h[x][0] : 0;
            }
        }
        uint32_t bin;
        find_bin(c0, c1, need, &bin, &need);
        prefix = prefix << step_bits(STEP - 1) | bin;
        if (threadIdx.x < 2)
            sums[threadIdx.x] = 0;
        __syncthreads();
        if (STEP == 3) {
            // rows of earlier chunks: keys above (this step's; the others' from their
            // workgroups) and ties
            uint32_t x = (b0 > bin ? before0 : 0) + (b0 - 1 > bin && b0 > 0 ? before1 : 0);
            for (uint32_t c = threadIdx.x; c < chunk; c += EV_THREADS) {
                const uint32_t *s = e.state + (t.set * e.chunks + c) * 8;
                x += s[4] + s[5];
            }
            x = sum_all(x);
            if ((threadIdx.x & 63) == 0 && x)
                atomicAdd(&sums[0], x);
            if (b0 == bin)
                sums[1] = before0;
            if (b0 - 1 == bin)
                sums[1] = before1;
            __syncthreads();
            out0 = sums[0];
            ties0 = sums[1];
        } else {
            const uint32_t *h = hist_of(STEP - 1, chunk);
            const uint32_t x = sum_all((b0 > bin ? h[b0] : 0) + (b0 - 1 > bin ? h[b0 - 1] : 0));
            if ((threadIdx.x & 63) == 0 && x)
                atomicAdd(&sums[0], x);
            __syncthreads();
            if (threadIdx.x == 0) {
                mine[2 * (STEP - 1)] = prefix;
                mine[2 * (STEP - 1) + 1] = need;
                mine[3 + STEP] = sums[0];
            }
        }
    }
    if constexpr (STEP == 3) {
        // rows of earlier chunks outside [lo, hi)
        const uint32_t row0 = chunk * EV_CHUNK;
        out0 += row0 < t.lo ? row0 : t.lo;
        out0 += row0 > t.hi ? row0 - t.hi : 0;
        emit(e, t, rows, from, prefix, need, out0, ties0);
    } else {
        hist[threadIdx.x] = 0;
        hist[threadIdx.x + EV_THREADS] = 0;
        __syncthreads();
        if (t.need > 0)
            rows.count(t, hist, from, STEP, prefix);
        __syncthreads();
        uint32_t *h = hist_of(STEP, chunk);
        h[threadIdx.x] = hist[threadIdx.x];
        h[threadIdx.x + EV_THREADS] = hist[threadIdx.x + EV_THREADS];
    }
}

// Copies the kept rows of one (sequence, head): each thread 16 bytes of a row of k and
// of v.  Bound by HBM: 525 MB (read and written) in 109 us, 4.8 TB/s, as a large copy.
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

hipError_t launch_evict(const Evict &e, hipStream_t s)
{
    const uint32_t sets = e.src.batch * e.sets;
    if (e.chunks == 0) {
        // (registers, and code, for no more rows than there can be)
        if (e.src.room <= EV_ONE / 8)
            evict_select<EV_ONE / 8 / EV_THREADS><<<dim3(sets), EV_THREADS, 0, s>>>(e);
        else if (e.src.room <= EV_ONE / 2)
            evict_select<EV_ONE / 2 / EV_THREADS><<<dim3(sets), EV_THREADS, 0, s>>>(e);
        else
            evict_select<EV_ONE / EV_THREADS><<<dim3(sets), EV_THREADS, 0, s>>>(e);
    } else {
        const dim3 grid(e.chunks, sets);
        evict_step<0><<<grid, EV_THREADS, 0, s>>>(e);
        evict_step<1><<<grid, EV_THREADS, 0, s>>>(e);
        evict_step<2><<<grid, EV_THREADS, 0, s>>>(e);
        evict_step<3><<<grid, EV_THREADS, 0, s>>>(e);
    }
    hipError_t err = hipGetLastError();
    const uint32_t most = e.keep < e.src.room ? e.keep : e.src.room;
    if (err != hipSuccess || most == 0)
        return err;
    // 64 rows a workgroup, more where a launch would reach 2^32 threads
    const uint32_t chunks = (e.src.d + 7) / 8, rows_per = most <= 1u << 29 ? 64 : 128;
    evict_copy<<<dim3((most + rows_per - 1) / rows_per, e.src.batch * e.src.heads), 256, 0, s>>>(
        e, chunks, PageDiv::of(chunks), rows_per);
    return hipGetLastError();
}

}  // namespace sjc
