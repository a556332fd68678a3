// sj_pages.hip -- the pages of a cache: which of them sequences hold that go on, fork or end
// (sj_cache_pages), and copies of their rows (sj_cache_copy, sj_cache8_copy).
#include "sj_cache.h"

namespace sjc {

namespace {

constexpr uint32_t PG_THREADS = 1024, PG_WAVES = PG_THREADS / 64;
constexpr uint32_t PG_ENTRIES = 4096;   // table entries of a workgroup
constexpr uint32_t PG_SEQS = 16;        // sequences of a workgroup at most

// What new sequence i goes on with: n rows, `whole` full pages, and in the table row `from`
// the number of its last, partly filled one (-1: none, or one that does not exist).
struct Heir {
    uint32_t n, whole, ends;    // (pages that it needs in all)
    bool part;
    const int32_t *from;
    int32_t last;
};

__device__ __forceinline__ Heir heir_of(const Pages &p, uint32_t i)
{
    Heir h;
    const int32_t parent = p.parent ? p.parent[i] : (int32_t)(i < p.batch ? i : ~0u);
    const bool real = (uint32_t)parent < p.batch;
    h.n = real ? clamp_rows(p.len[parent], p.room) : 0;
    h.from = p.table + (real ? (int64_t)parent * p.table_row : 0);
    h.whole = p.div.quot(h.n);
    h.part = h.n != h.whole * p.div.page;
    const uint64_t rows = (uint64_t)h.n + p.tokens;
    h.ends = p.div.quot((uint32_t)(rows < p.room ? rows : p.room) + p.div.page - 1);
    h.last = h.part ? h.from[h.whole] : -1;
    if ((uint32_t)h.last >= p.pages)
        h.last = -1;
    return h;
}

__device__ __forceinline__ uint32_t load_again(const uint32_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Waits for the wave's atomics, which are done where all XCDs see them.  (A fence would write back a
// whole cache, in every workgroup: 83 us instead of 15 for 256 sequences.)
__device__ __forceinline__ void wait_marks() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Sum of x over the threads before this one, and over all.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t *waves, uint32_t *all)
{
    const uint32_t incl = sum_upto(x), wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63)
        waves[wave] = incl;
    __syncthreads();
    uint32_t before = 0, total = 0;
    for (uint32_t w = 0; w < PG_WAVES; ++w) {
        before += w < wave ? waves[w] : 0;
        total += waves[w];
    }
    *all = total;
    return before + incl - x;
}

// Who keeps a partly filled page, how many pages each sequence is given and how many before it,
// and the free pages in ascending order, as many as are needed.  Leaves the bits at zero for the
// next call.
__device__ __forceinline__ void give(const Pages &p, uint32_t *waves)
{
    uint32_t needed = 0;
    for (uint32_t i0 = 0; i0 < p.out_batch; i0 += PG_THREADS) {
        const uint32_t i = i0 + threadIdx.x;
        uint32_t need = 0;
        if (i < p.out_batch) {
            const Heir h = heir_of(p, i);
            bool keeps = false;
            if (h.last >= 0) {
                const uint32_t x = (uint32_t)h.last;
                // (only its holder sets the page's bit here, and reads it before)
                keeps = !((load_again(&p.used[x >> 5]) >> (x & 31)) & 1) &&
                        load_again(&p.holder[x]) == ~i;
                if (keeps)
                    atomicOr(&p.used[x >> 5], 1u << (x & 31));
            }
            const uint32_t begins = h.whole + (h.part ? 1 : 0);
            need = (h.last >= 0 && !keeps ? 1 : 0) + (h.ends > begins ? h.ends - begins : 0);
            p.kept[i] = keeps;
        }
        uint32_t all;
        const uint32_t before = sum_before(need, waves, &all);
        if (i < p.out_batch)
            p.base[i] = needed + before;
        needed += all;
    }
    wait_marks();
    __syncthreads();
    // 32 marks a thread, until there are enough (longer runs a thread are written down one by one: 9 us
    // more for 1300 pages in runs of 256)
    const uint32_t words = (uint32_t)(((uint64_t)p.pages + 31) / 32);
    uint32_t found = 0;
    for (uint32_t w0 = 0; w0 < words && found < needed; w0 += PG_THREADS) {
        const uint32_t w = w0 + threadIdx.x;
        uint32_t bits = w < words ? ~load_again(p.used + w) : 0;
        if (w == words - 1 && p.pages % 32)
            bits &= (1u << p.pages % 32) - 1;
        uint32_t all;
        uint32_t at = found + sum_before((uint32_t)__popc(bits), waves, &all);
        for (; bits && at < needed; ++at, bits &= bits - 1)
            p.free[at] = (int32_t)(32 * w + (uint32_t)__ffs(bits) - 1);
        found += all;
    }
    __syncthreads();
    for (uint32_t w = threadIdx.x; w < words; w += PG_THREADS)
        p.used[w] = 0;
    if (threadIdx.x == 0)
        *p.n_free = found;
}

// Marks the pages that sequences share, one bit each, and for the partly filled ones the first
// sequence that holds them (~i at most; 0: none).  A neighbour with the same parent has marked its pages
// already.  The last workgroup to arrive gives the pages out.  A workgroup takes `seqs` sequences, so that
// few are counted.  Bound by latency, of the chain parent, length, table, marks and of one
// workgroup's scans: 32 sequences and 20000 pages 21 us in three launches, 15 in two; 256 sequences
// forked from 16 and 200000 pages 38 and 20.
__global__ void __launch_bounds__(PG_THREADS) pages_give(const Pages p, uint32_t groups, uint32_t seqs)
{
    __shared__ uint32_t waves[PG_WAVES], arrived;
    const uint32_t each = PG_THREADS / seqs, tid = threadIdx.x % each;
    const uint32_t i = blockIdx.x / groups * seqs + threadIdx.x / each;
    const uint32_t w0 = blockIdx.x % groups * PG_ENTRIES;
    if (i < p.out_batch) {
        const Heir h = heir_of(p, i);
        if (w0 == 0 && tid == 0 && h.last >= 0)
            atomicMax(&p.holder[h.last], ~i);
        if (i == 0 || !p.parent || p.parent[i] != p.parent[i - 1]) {
            const uint32_t end = h.whole < w0 + PG_ENTRIES ? h.whole : w0 + PG_ENTRIES;
            for (uint32_t w = w0 + tid; w < end; w += 4 * each) {
                uint32_t x[4];
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    x[k] = w + k * each < end ? (uint32_t)h.from[w + k * each] : ~0u;
#pragma unroll
                for (uint32_t k = 0; k < 4; ++k)
                    if (x[k] < p.pages)
                        atomicOr(&p.used[x[k] >> 5], 1u << (x[k] & 31));
            }
        }
    }
    wait_marks();       // (before the workgroup is counted)
    __syncthreads();
    if (threadIdx.x == 0) {
        arrived = __hip_atomic_fetch_add(p.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (arrived == gridDim.x - 1)
            __hip_atomic_store(p.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (arrived == gridDim.x - 1)
        give(p, waves);
}

// The new table, the copies and the numbers of each sequence; the holders are 0 again.
__global__ void __launch_bounds__(256) pages_table(const Pages p, uint32_t groups)
{
    const uint32_t i = blockIdx.x / groups, w0 = blockIdx.x % groups * PG_ENTRIES;
    const Heir h = heir_of(p, i);
    const uint32_t n_free = *p.n_free, base = p.base[i];
    const bool copy = h.last >= 0 && !p.kept[i];
    const uint32_t begins = h.whole + (h.part ? 1 : 0), first = base + (copy ? 1 : 0);
    const uint32_t end = p.width < w0 + PG_ENTRIES ? p.width : w0 + PG_ENTRIES;
    for (uint32_t w = w0 + threadIdx.x; w < end; w += 256) {
        int32_t x = -1;
        if (copy && w == h.whole) {
            x = base < n_free ? p.free[base] : -1;
        } else if (w < begins) {
            x = h.from[w];
        } else if (w < h.ends) {
            const uint32_t k = first + (w - begins);
            x = k < n_free ? p.free[k] : -1;
        }
        p.out_table[(uint64_t)i * p.width + w] = x;
    }
    if (w0 == 0 && threadIdx.x == 0) {
        const uint32_t need = (copy ? 1 : 0) + (h.ends > begins ? h.ends - begins : 0);
        const uint32_t left = base < n_free ? n_free - base : 0;
        const bool made = copy && left > 0;
        if (h.last >= 0)
            p.holder[h.last] = 0;
        p.new_len[i] = (int32_t)h.n;
        p.lacking[i] = (int32_t)(need - (need < left ? need : left));
        p.copies[3 * (uint64_t)i] = made ? h.last : -1;
        p.copies[3 * (uint64_t)i + 1] = made ? p.free[base] : -1;
        p.copies[3 * (uint64_t)i + 2] = made ? (int32_t)(h.n - h.whole * p.div.page) : 0;
    }
}

// ---------------------------------------------------------------------- copies

constexpr int CP_LOADS = 4;             // 16-byte chunks of k and of v that a thread has under way
constexpr uint32_t CP_ITEMS = 256 * CP_LOADS;

struct CopyArgs {
    Copy c;
    uint32_t parts;         // workgroups of an entry
    uint32_t first;         // entry of the launch
    uint32_t bytes;         // of a row of a head
    uint32_t heads;         // of the exponents
    PageDiv by_row, by_head;    // chunks of a row; of a head
};

__device__ __forceinline__ i32x4 load_bytes(const uint8_t *p, uint32_t left)
{
    i32x4 v = {0, 0, 0, 0};
    if (left >= 16) {
        __builtin_memcpy(&v, p, 16);
    } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (uint32_t e = 0; e < 15; ++e)
            if (e < left)
                w[e >> 2] |= (uint32_t)p[e] << (8 * (e & 3));
        v = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    }
    return v;
}

__device__ __forceinline__ void store_bytes(uint8_t *p, i32x4 v, uint32_t left)
{
    if (left >= 16) {
        __builtin_memcpy(p, &v, 16);
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 15; ++e)
            if (e < left)
                p[e] = (uint8_t)((uint32_t)v[e >> 2] >> (8 * (e & 3)));
    }
}

// A workgroup takes one part of an entry's 16-byte chunks, row by row and head by head.
__global__ void __launch_bounds__(256) copy_pages(const CopyArgs g)
{
    const Cache &c = g.c.c;
    const uint32_t n = g.first + blockIdx.x / g.parts, part = blockIdx.x % g.parts;
    const int32_t *entry = g.c.copies + 3 * (uint64_t)n;
    const uint32_t from = (uint32_t)entry[0], to = (uint32_t)entry[1];
    const int32_t asked = entry[2];
    if (from >= c.pages || to >= c.pages || from == to || asked <= 0)
        return;
    const uint32_t rows = (uint32_t)asked < c.div.page ? (uint32_t)asked : c.div.page;
    const uint32_t size = g.c.size, items = rows * g.by_row.page;
    const uint8_t *k0 = (const uint8_t *)c.k, *v0 = (const uint8_t *)c.v;
    for (uint32_t i0 = part * CP_ITEMS + threadIdx.x; i0 < items; i0 += g.parts * CP_ITEMS) {
        i32x4 k[CP_LOADS], v[CP_LOADS];
        auto offset = [&](uint32_t i, int64_t row, int64_t head, uint32_t *left) -> int64_t {
            const uint32_t r = g.by_row.quot(i), x = i - r * g.by_row.page;
            const uint32_t h = g.by_head.quot(x);
            uint32_t at = 16 * (x - h * g.by_head.page);
            if (g.bytes >= 16 && at + 16 > g.bytes)
                at = g.bytes - 16;      // (the last one moved back onto its neighbour)
            *left = g.bytes - at;
            return ((int64_t)r * row + (int64_t)h * head) * size + at;
        };
#pragma unroll
        for (int y = 0; y < CP_LOADS; ++y) {
            const uint32_t i = i0 + 256 * y;
            uint32_t left;
            if (i < items) {
                int64_t o = offset(i, c.k_row, c.k_head, &left);
                k[y] = load_bytes(k0 + (int64_t)from * c.k_page * size + o, left);
                o = offset(i, c.v_row, c.v_head, &left);
                v[y] = load_bytes(v0 + (int64_t)from * c.v_page * size + o, left);
            }
        }
#pragma unroll
        for (int y = 0; y < CP_LOADS; ++y) {
            const uint32_t i = i0 + 256 * y;
            uint32_t left;
            if (i < items) {
                int64_t o = offset(i, c.k_row, c.k_head, &left);
                store_bytes((uint8_t *)k0 + (int64_t)to * c.k_page * size + o, k[y], left);
                o = offset(i, c.v_row, c.v_head, &left);
                store_bytes((uint8_t *)v0 + (int64_t)to * c.v_page * size + o, v[y], left);
            }
        }
    }
    if (c.ex && part == 0) {
        const uint32_t blocks = c.by_block.quot(rows + c.by_block.page - 1);
        uint16_t *ex = const_cast<uint16_t *>(c.ex);
        const uint64_t step = (uint64_t)c.blocks * g.heads;
        for (uint32_t i = threadIdx.x; i < blocks * g.heads; i += 256)
            ex[to * step + i] = ex[from * step + i];
    }
}

}  // namespace

hipError_t launch_pages(const Pages &p, hipStream_t s)
{
    const uint32_t groups = p.width ? (p.width + PG_ENTRIES - 1) / PG_ENTRIES : 1;
    uint32_t seqs = 1;      // (32 workgroups, or a sequence each)
    while (seqs < PG_SEQS && p.out_batch > 32 * seqs)
        seqs *= 2;
    pages_give<<<dim3((p.out_batch + seqs - 1) / seqs * groups), PG_THREADS, 0, s>>>(p, groups, seqs);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    pages_table<<<dim3(p.out_batch * groups), 256, 0, s>>>(p, groups);
    return hipGetLastError();
}

hipError_t launch_copy(const Copy &c, hipStream_t s)
{
    CopyArgs g{};
    g.c = c;
    g.heads = c.c.heads;
    // (heads side by side are one: 194 pages of 16 heads of 72, 22 -> 11 us)
    Cache &x = g.c.c;
    if (x.k_head == x.d && x.v_head == x.d) {
        x.d *= x.heads;
        x.heads = 1;
    }
    g.bytes = x.d * c.size;
    const uint32_t chunks = (g.bytes + 15) / 16;
    g.by_head = PageDiv::of(chunks);
    g.by_row = PageDiv::of(x.heads * chunks);
    const uint64_t items = (uint64_t)x.div.page * x.heads * chunks;
    const uint64_t most = (items + CP_ITEMS - 1) / CP_ITEMS;
    g.parts = (uint32_t)(most < 4096 ? most : 4096);
    const uint32_t step = (1u << 22) / g.parts;     // entries of a launch
    hipError_t e = hipSuccess;
    for (uint64_t first = 0; first < c.n && e == hipSuccess; first += step) {
        g.first = (uint32_t)first;
        const uint64_t left = c.n - first;
        copy_pages<<<dim3((uint32_t)(left < step ? left : step) * g.parts), 256, 0, s>>>(g);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace sjc
