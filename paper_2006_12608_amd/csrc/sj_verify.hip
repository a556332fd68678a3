// sj_verify.hip -- verification of drafted tokens against the target's probabilities
// (sj_verify).
#include "sj_cache.h"

namespace sjc {

namespace {

struct VerifyArgs {
    Verify v;
    uint64_t first;         // workgroup of the launch: sequence x chunks + chunk
    PageDiv by_chunks;
};

// A probability; what is no positive finite number is 0.
__device__ __forceinline__ float clean(float x) { return x > 0.f && x < INFINITY ? x : 0.f; }

template <int DT>
struct Prob;
template <>
struct Prob<5> {
    typedef float one;
    static __device__ __forceinline__ float of(float x) { return x; }
};
template <>
struct Prob<sjk::DT_F16> {
    typedef uint16_t one;
    static __device__ __forceinline__ float of(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
};
template <>
struct Prob<sjk::DT_BF16> {
    typedef uint16_t one;
    static __device__ __forceinline__ float of(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
};

constexpr uint32_t VE_EACH = VE_CHUNK / 256;    // tokens of a thread, side by side

// Where a sequence's walk ended.
struct Walk {
    uint32_t node, nodes;   // the last accepted one; nodes of the sequence
    bool refused;           // a drafted token was refused there, with draft
    uint32_t gone;          // tokens refused there, without draft
};

struct Shared {
    double p[VE_MOST];      // of a node's token after its parent
    int64_t token[VE_MOST];
    float u[VE_MOST], q[VE_MOST];
    int32_t parent[VE_MOST], path[VE_MOST];
    int64_t gone[VE_MOST];
    uint32_t found;
};

// The sequence's walk, by every workgroup for itself: the probabilities of the drafted tokens are
// gathered at once, a thread a node; a wave then goes from node to node with ballots over 64 of
// them at a time.
template <int DT>
__device__ __forceinline__ Walk walk(const Verify &v, uint32_t b, Shared &sh)
{
    typedef typename Prob<DT>::one one;
    __shared__ Walk out;
    const uint32_t T = v.count ? clamp_rows(v.count[b], v.t) : v.t;
    for (uint32_t n = threadIdx.x; n < T; n += 256) {
        const int32_t from = v.parent ? v.parent[(int64_t)b * v.parent_seq + n] : (int32_t)n - 1;
        const bool real = n > 0 && (uint32_t)from < n;
        const int64_t x = v.tokens[(uint64_t)b * v.t + n];
        const bool known = real && (uint64_t)x < v.vocab;
        const one *p = (const one *)v.target + (int64_t)b * v.p_seq;
        sh.p[n] = known ? clean(Prob<DT>::of(p[(int64_t)from * v.p_row + x])) : 0.f;
        if (v.draft) {
            const one *q = (const one *)v.draft + (int64_t)b * v.q_seq;
            sh.q[n] = known ? clean(Prob<DT>::of(q[(int64_t)from * v.q_row + x])) : 0.f;
        }
        const float u = v.uniform[(uint64_t)b * v.t + n];
        sh.u[n] = u > 0.f ? (u < 1.f ? u : 0x1.fffffep-1f) : 0.f;
        sh.parent[n] = real ? from : -1;
        sh.token[n] = x;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint32_t lane = threadIdx.x;
        Walk w = {0, T, false, 0};
        uint32_t found = T ? 1 : 0;
        double left = 1.0;
        if (lane == 0)
            sh.path[0] = 0;
        for (uint32_t n0 = 0; n0 < T; n0 += 64) {
            const uint32_t n = n0 + lane;
            const int32_t mine = n < T && n > 0 ? sh.parent[n] : -1;
            uint64_t tries = __ballot(mine == (int32_t)w.node && mine >= 0);
            while (tries) {
                const uint32_t c = n0 + (uint32_t)__ffsll((unsigned long long)tries) - 1;
                tries &= tries - 1;
                const double u = (double)sh.u[c];
                double p = sh.p[c];
                bool yes;
                if (v.draft) {
                    yes = u * (double)sh.q[c] < p;
                } else {
                    const int64_t x = sh.token[c];
                    for (uint32_t g = 0; g < w.gone; g += 64)
                        if (__ballot(g + lane < w.gone && sh.gone[g + lane] == x))
                            p = 0.0;
                    yes = p > 0.0 && u * left < p;
                }
                if (yes) {
                    w.node = c;
                    w.refused = false;
                    w.gone = 0;
                    left = 1.0;
                    if (lane == 0)
                        sh.path[found] = (int32_t)c;
                    ++found;
                    tries = __ballot(mine == (int32_t)c);
                } else if (v.draft) {
                    w.refused = true;
                } else {
                    left -= p;
                    if (lane == 0)
                        sh.gone[w.gone] = sh.token[c];
                    ++w.gone;
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                }
            }
        }
        if (lane == 0) {
            sh.found = found;
            out = w;
        }
    }
    __syncthreads();
    return out;
}

// The weights r and p of this thread's tokens of a chunk.
template <int DT>
struct Weights {
    float p[VE_EACH], q[VE_EACH];
    uint32_t gone;          // bit k: token k was refused

    __device__ __forceinline__ void load(const Verify &v, uint32_t b, const Walk &w, const Shared &sh,
                                         uint32_t chunk)
    {
        typedef typename Prob<DT>::one one;
        const uint32_t x0 = chunk * VE_CHUNK + threadIdx.x * VE_EACH;
        const one *pr = (const one *)v.target + (int64_t)b * v.p_seq + (int64_t)w.node * v.p_row;
        const one *qr = w.refused ? (const one *)v.draft + (int64_t)b * v.q_seq + (int64_t)w.node * v.q_row
                                  : nullptr;
        if (x0 + VE_EACH <= v.vocab) {
            one raw[VE_EACH];
            __builtin_memcpy(raw, pr + x0, sizeof(raw));
#pragma unroll
            for (uint32_t k = 0; k < VE_EACH; ++k)
                p[k] = clean(Prob<DT>::of(raw[k]));
            if (qr)
                __builtin_memcpy(raw, qr + x0, sizeof(raw));
#pragma unroll
            for (uint32_t k = 0; k < VE_EACH; ++k)
                q[k] = qr ? clean(Prob<DT>::of(raw[k])) : 0.f;
        } else {
#pragma unroll
            for (uint32_t k = 0; k < VE_EACH; ++k) {
                p[k] = x0 + k < v.vocab ? clean(Prob<DT>::of(pr[x0 + k])) : 0.f;
                q[k] = qr && x0 + k < v.vocab ? clean(Prob<DT>::of(qr[x0 + k])) : 0.f;
            }
        }
        gone = 0;
        for (uint32_t g = 0; g < w.gone; ++g) {
            const uint64_t k = (uint64_t)sh.gone[g] - x0;
            gone |= k < VE_EACH ? 1u << k : 0u;
        }
    }
    __device__ __forceinline__ double r(uint32_t k) const
    {
        const double x = (double)p[k] - (double)q[k];
        return (gone >> k) & 1 || x < 0.0 ? 0.0 : x;
    }
};

// Sum of x over the threads before this one, and over all; always in the same order.
__device__ __forceinline__ double add_before(double x, double *waves, double *all)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double incl = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(incl, o);
        incl += lane >= (uint32_t)o ? y : 0.0;
    }
    __syncthreads();
    if (lane == 63)
        waves[wave] = incl;
    __syncthreads();
    double before = 0.0, total = 0.0;
    for (uint32_t w = 0; w < 4; ++w) {
        before += w < wave ? waves[w] : 0.0;
        total += waves[w];
    }
    *all = total;
    return before + (incl - x);
}

__device__ __forceinline__ void put_sum(double *p, double x)
{
    __hip_atomic_store((uint64_t *)p, __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ double get_sum(const double *p)
{
    return __builtin_bit_cast(double, __hip_atomic_load((const uint64_t *)p, __ATOMIC_RELAXED,
                                                        __HIP_MEMORY_SCOPE_AGENT));
}

// A workgroup sums the weights of one chunk of the vocabulary in double; the last one of a
// sequence to arrive finds the chunk, thread and token where the sums pass the threshold.
template <int DT>
__global__ void __launch_bounds__(256) verify_chunks(const VerifyArgs g)
{
    __shared__ Shared sh;
    __shared__ double waves[4];
    __shared__ uint32_t arrived, hit, last;
    __shared__ double before_hit;
    const Verify &v = g.v;
    const uint32_t id = (uint32_t)(g.first + blockIdx.x);
    const uint32_t b = g.by_chunks.quot(id), chunk = id - b * v.chunks, tid = threadIdx.x;
    const Walk w = walk<DT>(v, b, sh);
    Weights<DT> y;
    double all, all_p;
    if (w.nodes > 0) {
        y.load(v, b, w, sh, chunk);
        double r = 0.0, p = 0.0;
#pragma unroll
        for (uint32_t k = 0; k < VE_EACH; ++k) {
            r += y.r(k);
            p += (double)y.p[k];
        }
        add_before(r, waves, &all);
        add_before(p, waves, &all_p);
    } else {
        all = all_p = 0.0;
    }
    double *sums = v.sums + (uint64_t)b * v.chunks * 2;
    if (tid == 0) {
        put_sum(sums + 2 * chunk, all);
        put_sum(sums + 2 * chunk + 1, all_p);
        __builtin_amdgcn_s_waitcnt(0x0f70);     // (stored before it is counted)
        arrived = __hip_atomic_fetch_add(&v.arrivals[b], 1u, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
        if (arrived == v.chunks - 1)
            __hip_atomic_store(&v.arrivals[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        hit = v.chunks;
        last = 0;
    }
    __syncthreads();
    if (arrived != v.chunks - 1)
        return;
    for (uint32_t n = tid; n < v.t; n += 256)
        v.path[(uint64_t)b * v.t + n] = n < sh.found ? sh.path[n] : -1;
    if (tid == 0)
        v.found[b] = (int32_t)sh.found;
    // the chunks' sums, a run of them a thread
    const uint32_t run = (v.chunks + 255) / 256, c0 = tid * run;
    const uint32_t c1 = c0 + run < v.chunks ? c0 + run : v.chunks;
    double r = 0.0, p = 0.0, total, total_p;
    for (uint32_t c = c0; c < c1; ++c) {
        r += get_sum(sums + 2 * c);
        p += get_sum(sums + 2 * c + 1);
    }
    double begin = add_before(r, waves, &total);
    const double begin_p = add_before(p, waves, &total_p);
    const bool plain = !(total > 0.0);
    if (plain) {
        begin = begin_p;
        total = total_p;
    }
    if (!(total > 0.0)) {
        if (tid == 0)
            v.next[b] = -1;
        return;
    }
    const double threshold = (double)sh.u[0] * total;
    // the first chunk whose sums pass it; where rounding leaves none, the last with a sum
    auto sum_of = [&](uint32_t c) { return get_sum(sums + 2 * c + (plain ? 1 : 0)); };
    double at = begin;
    for (uint32_t c = c0; c < c1; ++c) {
        const double x = sum_of(c);
        if (x > 0.0) {
            atomicMax(&last, c);
            if (at + x > threshold)
                atomicMin(&hit, c);
        }
        at += x;
    }
    __syncthreads();
    const uint32_t there = hit < v.chunks ? hit : last;
    if (there >= c0 && there < c1) {
        at = begin;
        for (uint32_t c = c0; c < there; ++c)
            at += sum_of(c);
        before_hit = at;
    }
    __syncthreads();
    if (tid == 0) {
        hit = 0xffffffffu;
        last = 0;
    }
    __syncthreads();
    y.load(v, b, w, sh, there);
    double mine = 0.0, unused;
#pragma unroll
    for (uint32_t k = 0; k < VE_EACH; ++k)
        mine += plain ? (double)y.p[k] : y.r(k);
    double sum = before_hit + add_before(mine, waves, &unused);
#pragma unroll
    for (uint32_t k = 0; k < VE_EACH; ++k) {
        const double x = plain ? (double)y.p[k] : y.r(k);
        sum += x;
        if (x > 0.0) {
            const uint32_t token = there * VE_CHUNK + tid * VE_EACH + k;
            atomicMax(&last, token);
            if (sum > threshold)
                atomicMin(&hit, token);
        }
    }
    __syncthreads();
    if (tid == 0)
        v.next[b] = (int64_t)(hit != 0xffffffffu ? hit : last);
}

}  // namespace

hipError_t launch_verify(const Verify &v, hipStream_t s)
{
    VerifyArgs g{};
    g.v = v;
    g.by_chunks = PageDiv::of(v.chunks);
    const uint64_t total = (uint64_t)v.batch * v.chunks, step = 1u << 22;
    hipError_t e = hipSuccess;
    for (; g.first < total && e == hipSuccess; g.first += step) {
        const uint64_t left = total - g.first;
        const dim3 grid((uint32_t)(left < step ? left : step));
        if (v.dtype == 5)
            verify_chunks<5><<<grid, 256, 0, s>>>(g);
        else if (v.dtype == sjk::DT_F16)
            verify_chunks<sjk::DT_F16><<<grid, 256, 0, s>>>(g);
        else
            verify_chunks<sjk::DT_BF16><<<grid, 256, 0, s>>>(g);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sjc
