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
    uint32_t found;         // accepted nodes, in path
    bool refused;           // a drafted token was refused there, with draft
    uint32_t gone;          // tokens refused there, without draft
};

// What is known of node n, a lane each.
struct Node {
    float p, q, u;          // probabilities of its token after its parent; random number
    int32_t parent;         // -1: never reached
    int64_t token;
};

__device__ __forceinline__ float number(float u)
{
    return u > 0.f ? (u < 1.f ? u : 0x1.fffffep-1f) : 0.f;
}

template <int DT>
__device__ __forceinline__ Node node_of(const Verify &v, uint32_t b, uint32_t n)
{
    typedef typename Prob<DT>::one one;
    Node k = {0.f, 0.f, 0.f, -1, -1};
    if (n == 0 || n >= v.t)     // (nodes past the sequence's own are looked up beside its count)
        return k;
    const int32_t from = v.parent ? v.parent[(int64_t)b * v.parent_seq + n] : (int32_t)n - 1;
    k.token = v.tokens[(uint64_t)b * v.t + n];
    k.u = number(v.uniform[(uint64_t)b * v.t + n]);
    if ((uint32_t)from >= n)
        return k;
    k.parent = from;
    if ((uint64_t)k.token < v.vocab) {
        const one *p = (const one *)v.target + (int64_t)b * v.p_seq + (int64_t)from * v.p_row;
        k.p = clean(Prob<DT>::of(p[k.token]));
        if (v.draft) {
            const one *q = (const one *)v.draft + (int64_t)b * v.q_seq + (int64_t)from * v.q_row;
            k.q = clean(Prob<DT>::of(q[k.token]));
        }
    }
    return k;
}

__device__ __forceinline__ int64_t shfl_token(int64_t x, uint32_t lane)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, (int)lane);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)x >> 32), (int)lane);
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ float lane_value(float x, uint32_t lane)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), (int)lane));
}

// The sequence's walk, by a wave: 64 nodes at a time, the next ones' values on their way. A chain
// ends at its first refusal; in a tree the wave goes from node to node by ballots of those that
// follow the present one.
template <int DT>
__device__ __forceinline__ Walk walk(const Verify &v, uint32_t b, int32_t *path, int64_t *gone)
{
    const uint32_t lane = threadIdx.x & 63;
    const uint32_t T = v.count ? clamp_rows(v.count[b], v.t) : v.t;
    Walk w = {0, T, T ? 1u : 0u, false, 0};
    if (lane == 0)
        path[0] = 0;
    Node next = node_of<DT>(v, b, lane);
    if (!v.parent) {
        for (uint32_t n0 = 0; n0 < T; n0 += 64) {
            const Node k = next;
            next = node_of<DT>(v, b, n0 + 64 + lane);
            const bool yes = v.draft ? (double)k.u * (double)k.q < (double)k.p : k.u < k.p;
            const uint64_t no = __ballot(n0 + lane > 0 && n0 + lane < T && !yes);
            const uint32_t first = no ? n0 + (uint32_t)__ffsll((unsigned long long)no) - 1 : T;
            if (n0 + lane < first)
                path[n0 + lane] = (int32_t)(n0 + lane);
            if (no) {
                w.node = first - 1;
                w.found = first;
                w.refused = v.draft != nullptr;
                w.gone = v.draft ? 0 : 1;
                if (n0 + lane == first)
                    gone[0] = k.token;
                return w;
            }
        }
        w.node = T ? T - 1 : 0;
        w.found = T;
        return w;
    }
    double left = 1.0;
    for (uint32_t n0 = 0; n0 < T; n0 += 64) {
        const Node k = next;
        next = node_of<DT>(v, b, n0 + 64 + lane);
        const int32_t parent = n0 + lane < T ? k.parent : -1;
        uint64_t tries = __ballot(parent == (int32_t)w.node), refused = 0;
        while (tries) {
            const uint32_t c = (uint32_t)__ffsll((unsigned long long)tries) - 1;
            tries &= tries - 1;
            const int64_t x = shfl_token(k.token, c);
            double p = (double)lane_value(k.p, c);
            uint64_t again = __ballot((refused >> lane) & 1 && k.token == x);
            for (uint32_t g = 0; g < w.gone; g += 64)
                again |= __ballot(g + lane < w.gone && gone[g + lane] == x);
            p = again ? 0.0 : p;
            if (p > 0.0 && (double)lane_value(k.u, c) * left < p) {
                w.node = n0 + c;
                w.gone = 0;
                left = 1.0;
                refused = 0;
                if (lane == 0)
                    path[w.found] = (int32_t)(n0 + c);
                ++w.found;
                tries = __ballot(parent == (int32_t)w.node);
            } else {
                left -= p;
                refused |= (uint64_t)1 << c;
            }
        }
        if ((refused >> lane) & 1)
            gone[w.gone + (uint32_t)__popcll(refused & (((uint64_t)1 << lane) - 1))] = k.token;
        w.gone += (uint32_t)__popcll(refused);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    return w;
}

// The weights r and p of this thread's tokens of a chunk.
template <int DT>
struct Weights {
    float p[VE_EACH], q[VE_EACH];
    uint32_t gone;          // bit k: token k was refused

    __device__ __forceinline__ void load(const Verify &v, uint32_t b, const Walk &w,
                                         const int64_t *refused, uint32_t chunk)
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
            const uint64_t k = (uint64_t)refused[g] - x0;
            gone |= k < VE_EACH ? 1u << k : 0u;
        }
    }
    // r of token k, or p where `plain`
    __device__ __forceinline__ double of(uint32_t k, bool plain) const
    {
        const double x = (double)p[k] - (plain ? 0.0 : (double)q[k]);
        return (!plain && (gone >> k) & 1) || x < 0.0 ? 0.0 : x;
    }
    __device__ __forceinline__ double sum(bool plain) const
    {
        double x = 0.0;
#pragma unroll
        for (uint32_t k = 0; k < VE_EACH; ++k)
            x += of(k, plain);
        return x;
    }
};

// Number of the first thread for which `yes` holds; 256 if none.  (`last`: of the last one.)
__device__ __forceinline__ uint32_t first_thread(bool yes, uint32_t *found)
{
    const uint64_t m = __ballot(yes);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        found[threadIdx.x >> 6] =
            m ? (threadIdx.x & 192) + (uint32_t)__ffsll((unsigned long long)m) - 1 : 256;
    __syncthreads();
    uint32_t x = found[3];
#pragma unroll
    for (int i = 2; i >= 0; --i)
        x = found[i] < 256 ? found[i] : x;
    return x;
}

__device__ __forceinline__ uint32_t last_thread(bool yes, uint32_t *found)
{
    const uint64_t m = __ballot(yes);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        found[threadIdx.x >> 6] =
            m ? (threadIdx.x & 192) + 63 - (uint32_t)__clzll((long long)m) : 256;
    __syncthreads();
    uint32_t x = found[0];
#pragma unroll
    for (int i = 1; i < 4; ++i)
        x = found[i] < 256 ? found[i] : x;
    return x;
}

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

// (Stores count as loads do.)
__device__ __forceinline__ void wait_stores() { __builtin_amdgcn_s_waitcnt(0x0f70); }

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

// A workgroup sums the weights of one chunk of the vocabulary (PARTS x VE_CHUNK tokens) in double,
// after walking through its sequence's nodes (every workgroup for itself); the last one of a sequence to arrive finds the
// chunk, thread and token where the sums pass the threshold, and reads that chunk again.  Bound
// by latency for few sequences (count, tokens, probabilities, row, sums, row: 10 us for a chain over 32768
// tokens); 64 chains over 131072 tokens, 67 MB, in 25 us, of which 6 are the last workgroups'.
template <int DT, uint32_t PARTS>
__global__ void __launch_bounds__(256) verify_chunks(const VerifyArgs g)
{
    extern __shared__ int64_t lists[];      // tokens refused (t), then the path (t)
    __shared__ Walk walked;
    __shared__ double waves[4], before;
    __shared__ uint32_t found[4], at_chunk, arrived;
    const Verify &v = g.v;
    const uint32_t id = (uint32_t)(g.first + blockIdx.x);
    const uint32_t b = g.by_chunks.quot(id), chunk = id - b * v.chunks, tid = threadIdx.x;
    int64_t *const gone = lists;
    int32_t *const path = (int32_t *)(lists + v.t);
    const float u = number(v.uniform[(uint64_t)b * v.t]);
    if (tid < 64) {
        const Walk w = walk<DT>(v, b, path, gone);
        if (tid == 0)
            walked = w;
    }
    __syncthreads();
    const Walk w = walked;
    Weights<DT> y;
    double all = 0.0;
    if (w.nodes > 0) {
        double x = 0.0;
#pragma unroll 1
        for (uint32_t i = 0; i < PARTS; ++i) {
            y.load(v, b, w, gone, chunk * PARTS + i);
            x += y.sum(false);
        }
        add_before(x, waves, &all);
    }
    double *const sums = v.sums + (uint64_t)b * v.chunks;
    if (tid == 0) {
        put_sum(sums + chunk, all);
        wait_stores();      // (before it is counted)
        arrived = __hip_atomic_fetch_add(&v.arrivals[b], 1u, __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
        if (arrived == v.chunks - 1)
            __hip_atomic_store(&v.arrivals[b], 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (arrived != v.chunks - 1)
        return;
    for (uint32_t n = tid; n < v.t; n += 256)
        v.path[(uint64_t)b * v.t + n] = n < w.found ? path[n] : -1;
    if (tid == 0) {
        v.found[b] = (int32_t)w.found;
        if (w.nodes == 0)
            v.next[b] = -1;
    }
    if (w.nodes == 0)
        return;
    // the chunks' sums, a run of them a thread
    const uint32_t run = (v.chunks + 255) / 256, c0 = tid * run;
    const uint32_t c1 = c0 + run < v.chunks ? c0 + run : v.chunks;
    double mine = 0.0, total;
    for (uint32_t c = c0; c < c1; ++c)
        mine += get_sum(sums + c);
    double begin = add_before(mine, waves, &total);
    bool plain = false;
    if (!(total > 0.0)) {
        // nothing left of what may be drawn: p itself, summed here (probabilities that add up
        // to 1 do not come to this, but for rounding)
        plain = true;
        for (uint32_t c = 0; c < v.chunks; ++c) {
            double x = 0.0;
#pragma unroll 1
            for (uint32_t i = 0; i < PARTS; ++i) {
                y.load(v, b, w, gone, c * PARTS + i);
                x += y.sum(true);
            }
            add_before(x, waves, &all);
            if (tid == 0)
                put_sum(sums + c, all);
        }
        wait_stores();
        __syncthreads();
        mine = 0.0;
        for (uint32_t c = c0; c < c1; ++c)
            mine += get_sum(sums + c);
        begin = add_before(mine, waves, &total);
        if (!(total > 0.0)) {
            if (tid == 0)
                v.next[b] = -1;
            return;
        }
    }
    // the first run whose sums pass the threshold and, where rounding leaves none, the last with a
    // sum; in it the chunk, in the chunk the thread, of the thread the token, by the same rule
    const double threshold = (double)u * total;
    uint32_t who = first_thread(mine > 0.0 && begin + mine > threshold, found);
    who = who < 256 ? who : last_thread(mine > 0.0, found);
    if (tid == who && run == 1) {
        at_chunk = c0;
        before = begin;
    } else if (tid == who) {
        uint32_t last = c0;
        double sum = begin, at = begin;
        for (uint32_t c = c0; c < c1; ++c) {
            const double x = get_sum(sums + c);
            if (x > 0.0) {
                last = c;
                at = sum;
                if (sum + x > threshold)
                    break;
            }
            sum += x;
        }
        at_chunk = last;
        before = at;
    }
    __syncthreads();
    // the part of the chunk, likewise
    uint32_t there = at_chunk * PARTS, pick = there;
    double sofar = before, pick_begin = 0.0;
    who = 256;
#pragma unroll 1
    for (const uint32_t end = there + PARTS;; ) {
        y.load(v, b, w, gone, there);
        mine = y.sum(plain);
        begin = sofar + add_before(mine, waves, &all);
        const uint32_t first = first_thread(mine > 0.0 && begin + mine > threshold, found);
        const uint32_t last = last_thread(mine > 0.0, found);
        if (last < 256) {
            pick = there;
            pick_begin = begin;
            who = first < 256 ? first : last;
        }
        if (first < 256 || ++there == end)
            break;
        sofar += all;
    }
    if (pick != there) {
        y.load(v, b, w, gone, pick);
        there = pick;
    }
    begin = pick_begin;
    if (tid == who) {
        uint32_t last = 0;
        double sum = begin;
        bool passed = false;
#pragma unroll
        for (uint32_t k = 0; k < VE_EACH; ++k) {
            const double x = y.of(k, plain);
            if (x > 0.0 && !passed) {
                last = k;
                passed = sum + x > threshold;
            }
            sum += x;
        }
        v.next[b] = (int64_t)there * VE_CHUNK + tid * VE_EACH + last;
    }
}

template <int DT>
void (*verify_kernel(uint32_t parts))(const VerifyArgs)
{
    return parts == 1 ? verify_chunks<DT, 1> : verify_chunks<DT, 2>;
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
        const size_t lds = (size_t)v.t * 12;
        if (v.dtype == 5)
            verify_kernel<5>(v.parts)<<<grid, 256, lds, s>>>(g);
        else if (v.dtype == sjk::DT_F16)
            verify_kernel<sjk::DT_F16>(v.parts)<<<grid, 256, lds, s>>>(g);
        else
            verify_kernel<sjk::DT_BF16>(v.parts)<<<grid, 256, lds, s>>>(g);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sjc
