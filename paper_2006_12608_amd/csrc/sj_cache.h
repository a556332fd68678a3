// sj_cache.h -- the cache of key and value rows as the kernels see it, and the
// interface between the host side (sj_cache_api.cpp) and the kernels on it
// (sj_attend_*.hip, sj_rotary.hip, sj_evict.hip).  Contracts: include/sj.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sj_internal.h"

namespace sjc {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// n / page for 0 <= n < 2^31 as (n * mul) >> shift: with s = ceil(log2 page),
// mul = floor(2^(31 + s) / page) + 1 exceeds the quotient's factor by at most
// 1 / 2^31 of a unit per n, less than the 1 / page that separates quotients.
struct PageDiv {
    uint32_t mul, shift, page;
    static PageDiv of(uint32_t page)
    {
        uint32_t s = 0;
        while (((uint64_t)1 << s) < page)
            ++s;
        return {(uint32_t)(((uint64_t)1 << (31 + s)) / page + 1), 31 + s, page};
    }
    __device__ __forceinline__ uint32_t quot(uint32_t n) const
    {
        return (uint32_t)(((uint64_t)n * mul) >> shift);
    }
};

struct Cache {
    const uint16_t *k, *v;
    int64_t k_page, k_row, k_head, v_page, v_row, v_head;  // strides in elements
    const int32_t *table;   // may be null: sequence b is page b
    int64_t table_row;
    uint32_t width, pages;
    uint32_t room;          // width * page: rows a sequence may hold (< 2^31)
    PageDiv div;
    uint32_t batch, heads, d;
    // of a cache in 8 bits: k and v point at e4m3 elements (strides in elements), and ex at the
    // exponents of each page, block of rows and head, k's in the low byte and v's in the high one
    const uint16_t *ex;
    uint32_t blocks;        // of a page
    PageDiv by_block;       // rows of a block
};

// Page number and place in the page of row n (< room) of sequence b; the number
// is -1 where the page does not exist.
struct Place {
    int32_t page;
    uint32_t slot;
};

__device__ __forceinline__ Place place_of(const Cache &c, uint32_t b, uint32_t n)
{
    const uint32_t w = c.div.quot(n);
    const int32_t p = c.table ? c.table[(int64_t)b * c.table_row + w] : (int32_t)b;
    return {(uint32_t)p < c.pages ? p : -1, n - w * c.div.page};
}

// The same in two steps for loops that load ahead: the entry of row n's page (of the last
// page past the room), loaded and not looked at, and the place it stands for.  Only
// what reads `page` waits for the load, and for all loads before it.
struct Entry {
    int32_t raw;
    uint32_t n;
};

__device__ __forceinline__ Entry entry_of(const Cache &c, const int32_t *any, uint32_t b, uint32_t n)
{
    const uint32_t w = c.div.quot(n), last = c.width - 1;
    const int32_t *row = c.table ? c.table + (int64_t)b * c.table_row : any;
    return {row[c.table ? (w < last ? w : last) : 0], n};
}

__device__ __forceinline__ Place place_of(const Cache &c, uint32_t b, const Entry &e, uint32_t end)
{
    const int32_t p = c.table ? e.raw : (int32_t)b;
    return {e.n < end && (uint32_t)p < c.pages ? p : -1, e.n - c.div.quot(e.n) * c.div.page};
}

// len[b] and the rows of the call's own tokens, clamped to what the cache holds.
__device__ __forceinline__ uint32_t clamp_rows(int32_t len, uint32_t room)
{
    return len < 0 ? 0u : ((uint32_t)len < room ? (uint32_t)len : room);
}

// Eight elements of a row from element c on (p points at them): one 16-byte load at
// the elements' alignment, element by element in the row's last, partial chunk,
// zeros past the row.
__device__ __forceinline__ i32x4 load8(const uint16_t *p, int left)
{
    i32x4 v = {0, 0, 0, 0};
    if (left >= 8) {
        __builtin_memcpy(&v, p, 16);
    } else if (left > 0) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left)
                w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        v = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    }
    return v;
}

__device__ __forceinline__ void store8(uint16_t *p, i32x4 v, int left)
{
    if (left >= 8) {
        __builtin_memcpy(p, &v, 16);
    } else if (left > 0) {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left)
                p[e] = (uint16_t)((uint32_t)v[e >> 1] >> (16 * (e & 1)));
    }
}

// Sum over the lanes up to this one, and over all lanes.
__device__ __forceinline__ uint32_t sum_upto(uint32_t x)
{
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true);   // row_shr 1
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true);
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);  // row 15 on
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);  // row 31 on
    return x;
}

__device__ __forceinline__ uint32_t sum_all(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_readlane((int)sum_upto(x), 63);
}

// ------------------------------------------------------------------- attention

// Blocks of rows that one wave takes at a time, and queries of one matrix tile.
constexpr uint32_t AT_ROWS = 32, AT_Q = 16, AT_WAVES = 4;

struct Attend {
    Cache c;
    const int32_t *len, *count;    // count may be null
    uint32_t t, group, q_heads;    // tokens, query heads per cache head
    PageDiv by_group;
    const uint16_t *q;
    int64_t q_seq, q_tok, q_head;
    const uint64_t *tree;          // may be null (chain)
    int64_t tree_seq, tree_tok;
    float scale2;                  // |scale| * log2(e), above 0
    bool negate;                   // scale < 0
    uint16_t *out;
    float *lse;                    // never null here (scratch where the caller wants none)
    const float *w_in;
    float *w_out;                  // may be null
    uint64_t w_cols;
    // work split: a sequence's rows are cut into shares, one workgroup per share,
    // cache head and tile of query rows
    uint32_t tiles;                // tiles of query rows per cache head
    uint32_t heads_at_once;        // cache heads of a workgroup
    uint32_t want;                 // shares there should be at most
    uint32_t w_want;               // the same for the weights' kernel, a workgroup a share and head
    uint32_t slots;                // most shares there can be
    bool whole;                    // every sequence is one share
    uint32_t *plan;                // per sequence: first share, shares
    uint32_t *arrivals;            // per sequence, head and tile, zeros: shares that have arrived;
                                   // null: attend_join joins the shares, if any
    float *scores;                 // may be null: per head, query row and column (s_cols a row):
    uint32_t s_cols;               // scale2 * score, -inf where the row is not seen
    float *part_o;                 // per share, head, tile: query rows x padded d
    float *part_ml;                // per share, head, tile: query rows x {max, sum}
};

// The kernels for one call; the query rows of a workgroup's tile (16, 32, 64, 128 or 256)
// follow from t * group and d.
uint32_t attend_tile_rows(uint32_t rows, uint32_t d);
// Workgroups of the call's kernel that one CU holds at once.
int attend_occupancy_f16(uint32_t d, uint32_t tile_rows);
int attend_occupancy_bf16(uint32_t d, uint32_t tile_rows);
hipError_t launch_attend_f16(const Attend &a, hipStream_t s);
hipError_t launch_attend_bf16(const Attend &a, hipStream_t s);
// The same over a cache in 8 bits (d a multiple of 8).
int attend8_occupancy_f16(uint32_t d, uint32_t tile_rows, uint32_t heads_at_once);
int attend8_occupancy_bf16(uint32_t d, uint32_t tile_rows, uint32_t heads_at_once);
hipError_t launch_attend8_f16(const Attend &a, hipStream_t s);
hipError_t launch_attend8_bf16(const Attend &a, hipStream_t s);

// --------------------------------------------------------- rotary and appending

struct Turn {
    const int32_t *pos;
    const int64_t *turns;
    uint32_t pairs;
    int layout;
    float factor;
    bool inverse;
};

struct Strided {
    const uint16_t *in;
    uint16_t *out;
    int64_t in_seq, in_tok, in_head, out_seq, out_tok, out_head;
    uint32_t heads;
};

struct Rotary {
    int dtype;
    Turn turn;
    uint32_t batch, t, d;
    Strided x;              // turned into x.out (rotary; an append's queries); heads may be 0
    // an append's keys and values (heads of the cache; c.batch = 0: none)
    Cache c;
    const int32_t *len, *count;
    Strided key, value;     // out unused
};

hipError_t launch_rotary(const Rotary &r, hipStream_t s);

// ------------------------------------------------------------------- eviction

struct Evict {
    Cache src, dst;
    const int32_t *len;
    const float *weight;
    uint32_t sets;
    uint64_t w_cols, w_out_cols;
    uint32_t keep, sink, recent;
    int32_t *index, *new_len;
    float *w_out;           // may be null
    uint32_t chunks;        // of EV_CHUNK rows, where a sequence may have more than EV_ONE
    uint32_t *hist;         // per set, step and chunk: EV_BINS counts
    uint32_t *state;        // per set and chunk: key prefix, rows still needed; keys above
};

// Rows that one workgroup selects from alone, rows of a chunk beyond, bins of a step.
constexpr uint32_t EV_ONE = 32768, EV_CHUNK = 8192, EV_BINS = 2048;

// Scratch of a call: uint32 values of hist and of state (0 where one workgroup does).
inline uint32_t evict_chunks(uint32_t room)
{
    return room <= EV_ONE ? 0 : (room + EV_CHUNK - 1) / EV_CHUNK;
}
inline uint64_t evict_hist_values(uint64_t sets, uint32_t chunks)
{
    return sets * chunks * 3 * EV_BINS;
}
inline uint64_t evict_state_values(uint64_t sets, uint32_t chunks) { return sets * chunks * 8; }

hipError_t launch_evict(const Evict &e, hipStream_t s);

// ------------------------------------------------------------- appending in 8 bits

constexpr uint32_t A8_SINES = 2048;     // rows x pairs of a block that a workgroup turns

struct Append8 {
    int dtype;
    Turn turn;              // of keys (no pairs where a block has more than A8_SINES)
    Cache c;
    uint32_t t, blocks;     // tokens; blocks of a sequence that they may touch
    const int32_t *len, *count;
    Strided key, value;     // out unused
};

hipError_t launch_append8(const Append8 &r, hipStream_t s);

// ------------------------------------------------------------------------- pages

struct Pages {
    const int32_t *table, *len, *parent;    // parent may be null
    int64_t table_row;
    uint32_t batch, width, pages, room, out_batch, tokens;
    PageDiv div;
    int32_t *out_table, *new_len, *copies, *lacking;
    // zeros between calls:
    uint32_t *arrived;      // workgroups
    uint32_t *used;         // a bit a page
    uint32_t *holder;       // a page: ~i for the first sequence i that goes on with it partly filled
    uint32_t *base;         // a sequence: pages given out before it
    int32_t *kept;          // a sequence: whether its last page stays with it
    int32_t *free;          // the pages to give out
    uint32_t *n_free;       // how many were found (enough, or all)
};

hipError_t launch_pages(const Pages &p, hipStream_t s);

struct Copy {
    Cache c;
    uint32_t size;          // bytes of an element
    const int32_t *copies;
    uint32_t n;
};

hipError_t launch_copy(const Copy &c, hipStream_t s);

// ------------------------------------------------------------------ drafted tokens

struct Verify {
    int dtype;
    uint32_t batch, t, vocab;
    const int64_t *tokens;
    const int32_t *parent, *count;      // may be null
    int64_t parent_seq;
    const void *target, *draft;         // draft may be null
    int64_t p_seq, p_row, q_seq, q_row; // strides in elements
    const float *uniform;
    int32_t *path, *found;
    int64_t *next;
    uint32_t parts, chunks;             // of VE_CHUNK tokens; chunks of the vocabulary of so many parts
    double *sums;                       // per sequence and chunk
    uint32_t *arrivals;                 // per sequence, zeros between calls
};

constexpr uint32_t VE_CHUNK = 4096, VE_MOST = 1024;   // tokens that a workgroup takes at once; nodes at most

hipError_t launch_verify(const Verify &v, hipStream_t s);

}  // namespace sjc
