// sj_cache_api.cpp -- host side of the calls on a cache of key and value rows
// (sj_rotary, sj_cache_append, sj_attend, sj_cache_evict, the two for caches in 8 bits, pages and
// their copies, and the verification of drafted tokens; contracts in include/sj.h):
// argument checks, scratch, and the kernels on the context's stream.  Nothing
// here waits for the device but the replacement of scratch that a call outgrows.
#include <hip/hip_runtime.h>

#include <cmath>

#include "sj.h"
#include "sj_cache.h"
#include "sj_host.h"

using namespace sjh;

namespace {

const int64_t kMaxStride = (int64_t)1 << 40;   // elements; extents below stay in 64 bits
const uint64_t kMaxCells = (uint64_t)1 << 31;
const uint64_t kMaxRows = (uint64_t)1 << 30;   // of a sequence

const uint64_t kMaxScores = (uint64_t)1 << 30; // bytes of kept scores

struct Axis {
    uint64_t n;
    int64_t stride;
};

// The device array that element 0 and these strided axes reach, d adjacent elements
// at each place.
int check_strided(const sj_ctx *c, const void *p, const Axis *axes, int n_axes, uint64_t d,
                  const char *name, uint32_t size = 2)
{
    uint64_t last = 0;
    for (int i = 0; i < n_axes; ++i) {
        if (axes[i].n == 0)
            return SJ_OK;
        if (axes[i].stride < 0 || axes[i].stride > kMaxStride)
            return fail(SJ_E_INVAL, "%s: stride %lld is negative or too large", name,
                        (long long)axes[i].stride);
        if (axes[i].n > 1) {
            if ((uint64_t)axes[i].stride > ((uint64_t)1 << 60) / axes[i].n)
                return fail(SJ_E_INVAL, "%s: stride %lld is too large", name,
                            (long long)axes[i].stride);
            last += (axes[i].n - 1) * (uint64_t)axes[i].stride;
        }
    }
    if ((uintptr_t)p % size != 0)
        return fail(SJ_E_INVAL, "%s must be %u-byte aligned", name, size);
    return check_device_ptr(c, p, (size_t)(last + d) * size, name);
}

// Scratch and counters of one call.  While the context's stream is captured nothing may be
// allocated, and the graph keeps what there is.
int grow_both(sj_ctx *c, size_t bytes, size_t counters)
{
    hipStreamCaptureStatus state = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(c->stream, &state) != hipSuccess) {
        (void)hipGetLastError();
        state = hipStreamCaptureStatusNone;
    }
    if (state != hipStreamCaptureStatusNone) {
        if (bytes > c->scratch_bytes || counters > c->arrivals_n)
            return fail(SJ_E_UNSUPPORTED,
                        "scratch would grow during a capture (%zu bytes, %zu there): make the "
                        "call once on the stream before", bytes, c->scratch_bytes);
        c->scratch_held = true;
        c->arrivals_held = c->arrivals_held || counters != 0;
        return SJ_OK;
    }
    const int st = grow_scratch(c, bytes);
    return st == SJ_OK && counters ? grow_arrivals(c, counters) : st;
}

int check_array(const sj_ctx *c, const void *p, uint64_t bytes, uint32_t align, const char *name)
{
    if (bytes == 0)
        return SJ_OK;
    if ((uintptr_t)p % align != 0)
        return fail(SJ_E_INVAL, "%s must be %u-byte aligned", name, align);
    return check_device_ptr(c, p, (size_t)bytes, name);
}

// Checks a cache of elements of `size` bytes and translates it for the kernels.
int check_cache(const sj_ctx *c, const sj_cache *s, const char *name, sjc::Cache *out,
                uint32_t size = 2)
{
    if (!s)
        return fail(SJ_E_INVAL, "%s is NULL", name);
    if (s->dtype != SJ_F16 && s->dtype != SJ_BF16)
        return fail(SJ_E_INVAL, "%s: dtype %d is neither SJ_F16 nor SJ_BF16", name, s->dtype);
    if (s->heads == 0 || s->d == 0 || s->page == 0)
        return fail(SJ_E_INVAL, "%s: heads, d and page must be positive", name);
    if (s->d > 256)
        return fail(SJ_E_UNSUPPORTED, "%s: d = %u is above 256", name, s->d);
    const uint32_t width = s->pages == 0 ? 0 : (s->table ? s->width : 1);
    if ((uint64_t)width * s->page > kMaxRows || s->page >= kMaxCells || s->pages >= kMaxCells)
        return fail(SJ_E_UNSUPPORTED, "%s: %u pages of %u rows are too many", name, width, s->page);
    if ((uint64_t)s->batch * s->heads > 65535)
        return fail(SJ_E_UNSUPPORTED, "%s: batch * heads = %llu is above 65535", name,
                    (unsigned long long)s->batch * s->heads);
    int st;
    const Axis k[3] = {{s->pages, s->k_page}, {s->page, s->k_row}, {s->heads, s->k_head}};
    const Axis v[3] = {{s->pages, s->v_page}, {s->page, s->v_row}, {s->heads, s->v_head}};
    if ((st = check_strided(c, s->k, k, 3, s->d, "k", size)) != SJ_OK ||
        (st = check_strided(c, s->v, v, 3, s->d, "v", size)) != SJ_OK)
        return st;
    if (s->table && s->batch && width) {
        if (s->table_row < 0 || s->table_row > kMaxStride)
            return fail(SJ_E_INVAL, "%s: table_row is negative or too large", name);
        if ((st = check_array(c, s->table,
                              ((uint64_t)(s->batch - 1) * (uint64_t)s->table_row + width) * 4, 4,
                              "table")) != SJ_OK)
            return st;
    }
    *out = sjc::Cache{(const uint16_t *)s->k, (const uint16_t *)s->v, s->k_page, s->k_row, s->k_head,
                      s->v_page, s->v_row, s->v_head, s->table, s->table_row, width, s->pages,
                      width * s->page, sjc::PageDiv::of(s->page), s->batch, s->heads, s->d,
                      nullptr, 1, sjc::PageDiv::of(s->page)};
    return SJ_OK;
}

// The same of a cache in 8 bits.
int check_cache8(const sj_ctx *c, const sj_cache8 *s, const char *name, sjc::Cache *out)
{
    if (!s)
        return fail(SJ_E_INVAL, "%s is NULL", name);
    int st;
    if ((st = check_cache(c, &s->rows, name, out, 1)) != SJ_OK)
        return st;
    if (s->rows.d % 8 != 0)
        return fail(SJ_E_UNSUPPORTED, "%s: d = %u is no multiple of 8", name, s->rows.d);
    if (s->block == 0 || s->rows.page % s->block != 0)
        return fail(SJ_E_INVAL, "%s: blocks of %u rows do not divide pages of %u", name, s->block,
                    s->rows.page);
    out->blocks = s->rows.page / s->block;
    if ((st = check_array(c, s->exponents, (uint64_t)s->rows.pages * out->blocks * s->rows.heads * 2, 2,
                          "exponents")) != SJ_OK)
        return st;
    out->ex = (const uint16_t *)s->exponents;
    out->by_block = sjc::PageDiv::of(s->block);
    return SJ_OK;
}

int check_turn(const sj_ctx *c, uint64_t tokens, const int32_t *pos, const int64_t *turns,
               uint32_t n_pairs, uint32_t d, int layout, double factor)
{
    if (layout != SJ_HALF && layout != SJ_INTERLEAVED)
        return fail(SJ_E_INVAL, "unknown layout %d", layout);
    if (2 * (uint64_t)n_pairs > d)
        return fail(SJ_E_INVAL, "%u pairs do not fit in %u elements", n_pairs, d);
    if (n_pairs > 256)
        return fail(SJ_E_UNSUPPORTED, "%u pairs: 256 at most", n_pairs);
    if (std::isnan(factor))
        return fail(SJ_E_INVAL, "factor is NaN");
    if (n_pairs == 0)
        return SJ_OK;
    int st = check_array(c, pos, tokens * 4, 4, "pos");
    return st != SJ_OK ? st : check_array(c, turns, (uint64_t)n_pairs * 8, 8, "turns");
}

}  // namespace

extern "C" int sj_rotary(sj_ctx *c, int dtype, const void *x, const int64_t x_stride[2], void *y,
                         const int64_t y_stride[2], uint32_t n, uint32_t heads, uint32_t d,
                         const int32_t *pos, const int64_t *turns, uint32_t n_pairs, int layout,
                         double factor, unsigned flags)
{
    g_err.clear();
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    if (dtype != SJ_F16 && dtype != SJ_BF16)
        return fail(SJ_E_INVAL, "dtype %d is neither SJ_F16 nor SJ_BF16", dtype);
    if (flags & ~(unsigned)SJ_FLAG_INVERSE)
        return fail(SJ_E_INVAL, "flags 0x%x: not taken by sj_rotary", flags);
    if (!x_stride || !y_stride)
        return fail(SJ_E_INVAL, "strides are NULL");
    if (n >= kMaxCells || d > 65536 || (uint64_t)heads * ((d + 7) / 8 + 1) >= kMaxCells / 256)
        return fail(SJ_E_UNSUPPORTED, "%u tokens of %u heads of %u elements are too many", n, heads,
                    d);
    int st;
    if ((st = check_turn(c, n, pos, turns, n_pairs, d, layout, factor)) != SJ_OK)
        return st;
    if (n == 0 || heads == 0 || d == 0)
        return SJ_OK;
    const Axis ax[2] = {{n, x_stride[0]}, {heads, x_stride[1]}};
    const Axis ay[2] = {{n, y_stride[0]}, {heads, y_stride[1]}};
    if ((st = check_strided(c, x, ax, 2, d, "x")) != SJ_OK ||
        (st = check_strided(c, y, ay, 2, d, "y")) != SJ_OK)
        return st;
    if (x == y && (x_stride[0] != y_stride[0] || x_stride[1] != y_stride[1]))
        return fail(SJ_E_INVAL, "y is x with other strides");
    SJ_HIP(hipSetDevice(c->device));
    sjc::Rotary r{};
    r.dtype = dtype;
    r.turn = {pos, turns, n_pairs, layout, (float)factor, (flags & SJ_FLAG_INVERSE) != 0};
    r.batch = 1;
    r.t = n;
    r.d = d;
    r.x = {(const uint16_t *)x, (uint16_t *)y, 0, x_stride[0], x_stride[1], 0, y_stride[0],
           y_stride[1], heads};
    SJ_HIP(sjc::launch_rotary(r, c->stream));
    return SJ_OK;
}

namespace {

// sj_cache_append (cache) and sj_cache8_append (cache8).
int append_rows(sj_ctx *c, const sj_cache *cache, const sj_cache8 *cache8, bool eight, const int32_t *len,
                const int32_t *count, uint32_t t, const void *key, const int64_t key_stride[3],
                const void *value, const int64_t value_stride[3], const int32_t *pos,
                const int64_t *turns, uint32_t n_pairs, int layout, double factor, const void *q,
                const int64_t q_stride[3], uint32_t q_heads, void *q_out,
                const int64_t q_out_stride[3])
{
    g_err.clear();
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    sjc::Rotary r{};
    int st;
    if ((st = eight ? check_cache8(c, cache8, "cache", &r.c)
                    : check_cache(c, cache, "cache", &r.c)) != SJ_OK)
        return st;
    const uint32_t B = r.c.batch, d = r.c.d;
    if (!key_stride || !value_stride || (q && (!q_stride || !q_out_stride)))
        return fail(SJ_E_INVAL, "strides are NULL");
    if ((uint64_t)B * t >= kMaxCells ||
        ((uint64_t)q_heads + 2 * r.c.heads) * ((d + 7) / 8 + 1) >= kMaxCells / 256)
        return fail(SJ_E_UNSUPPORTED, "%u x %u tokens of %u heads are too many", B, t, q_heads);
    if ((st = check_turn(c, (uint64_t)B * t, pos, turns, n_pairs, d, layout, factor)) != SJ_OK)
        return st;
    if (B == 0 || t == 0)
        return SJ_OK;
    if ((st = check_array(c, len, (uint64_t)B * 4, 4, "len")) != SJ_OK ||
        (count && (st = check_array(c, count, (uint64_t)B * 4, 4, "count")) != SJ_OK))
        return st;
    auto axes = [&](const int64_t *s, uint32_t heads, Axis *a) {
        a[0] = {B, s[0]};
        a[1] = {t, s[1]};
        a[2] = {heads, s[2]};
    };
    Axis a[3];
    axes(key_stride, r.c.heads, a);
    if ((st = check_strided(c, key, a, 3, d, "key")) != SJ_OK)
        return st;
    axes(value_stride, r.c.heads, a);
    if ((st = check_strided(c, value, a, 3, d, "value")) != SJ_OK)
        return st;
    if (q) {
        axes(q_stride, q_heads, a);
        if ((st = check_strided(c, q, a, 3, d, "q")) != SJ_OK)
            return st;
        axes(q_out_stride, q_heads, a);
        if ((st = check_strided(c, q_out, a, 3, d, "q_out")) != SJ_OK)
            return st;
        if (q == q_out && (q_stride[0] != q_out_stride[0] || q_stride[1] != q_out_stride[1] ||
                           q_stride[2] != q_out_stride[2]))
            return fail(SJ_E_INVAL, "q_out is q with other strides");
        r.x = {(const uint16_t *)q, (uint16_t *)q_out, q_stride[0], q_stride[1], q_stride[2],
               q_out_stride[0], q_out_stride[1], q_out_stride[2], q_heads};
    }
    SJ_HIP(hipSetDevice(c->device));
    r.dtype = eight ? cache8->rows.dtype : cache->dtype;
    r.turn = {pos, turns, n_pairs, layout, (float)factor, false};
    r.batch = B;
    r.t = t;
    r.d = d;
    r.len = len;
    r.count = count;
    r.key = {(const uint16_t *)key, nullptr, key_stride[0], key_stride[1], key_stride[2], 0, 0, 0,
             r.c.heads};
    r.value = {(const uint16_t *)value, nullptr, value_stride[0], value_stride[1], value_stride[2],
               0, 0, 0, r.c.heads};
    if (!eight) {
        SJ_HIP(sjc::launch_rotary(r, c->stream));
        return SJ_OK;
    }
    // (the blocks that t rows may touch, beginning anywhere in the first)
    const uint32_t block = cache8->block, heads = r.c.heads;
    const uint64_t blocks = ((uint64_t)t + block - 2) / block + 1;
    if (B * blocks * 2 * r.c.heads >= kMaxCells)
        return fail(SJ_E_UNSUPPORTED, "%u x %u tokens of %u heads are too many", B, t, r.c.heads);
    sjc::Append8 w{};
    w.dtype = r.dtype;
    w.turn = r.turn;
    w.c = r.c;
    w.t = t;
    w.blocks = (uint32_t)blocks;
    w.len = len;
    w.count = count;
    w.key = r.key;
    w.value = r.value;
    r.c.batch = 0;
    // long blocks, halves that begin inside a chunk: the keys are turned on the way into scratch, which is
    // there before the first launch, since a call that is refused must not have turned the queries
    const bool passes =
        (uint64_t)block * n_pairs > sjc::A8_SINES || (layout == SJ_HALF && n_pairs % 8 != 0);
    if (passes && (st = grow_both(c, (size_t)((uint64_t)B * t * heads * d * 2), 0)) != SJ_OK)
        return st;
    if (q)                  // (the queries alone)
        SJ_HIP(sjc::launch_rotary(r, c->stream));
    if (passes) {
        const int64_t row = (int64_t)heads * d;
        r.x = {(const uint16_t *)key, (uint16_t *)c->scratch, key_stride[0], key_stride[1],
               key_stride[2], row * t, row, d, heads};
        SJ_HIP(sjc::launch_rotary(r, c->stream));
        w.key = {(const uint16_t *)c->scratch, nullptr, row * t, row, d, 0, 0, 0, heads};
        w.turn.pairs = 0;
    }
    if (r.c.room)
        SJ_HIP(sjc::launch_append8(w, c->stream));
    return SJ_OK;
}

}  // namespace

extern "C" int sj_cache_append(sj_ctx *c, const sj_cache *cache, const int32_t *len,
                               const int32_t *count, uint32_t t, const void *key,
                               const int64_t key_stride[3], const void *value,
                               const int64_t value_stride[3], const int32_t *pos,
                               const int64_t *turns, uint32_t n_pairs, int layout, double factor,
                               const void *q, const int64_t q_stride[3], uint32_t q_heads,
                               void *q_out, const int64_t q_out_stride[3])
{
    return append_rows(c, cache, nullptr, false, len, count, t, key, key_stride, value, value_stride, pos,
                       turns, n_pairs, layout, factor, q, q_stride, q_heads, q_out, q_out_stride);
}

extern "C" int sj_cache8_append(sj_ctx *c, const sj_cache8 *cache, const int32_t *len,
                               const int32_t *count, uint32_t t, const void *key,
                               const int64_t key_stride[3], const void *value,
                               const int64_t value_stride[3], const int32_t *pos,
                               const int64_t *turns, uint32_t n_pairs, int layout, double factor,
                               const void *q, const int64_t q_stride[3], uint32_t q_heads,
                               void *q_out, const int64_t q_out_stride[3])
{
    const Alone alone(c);
    return append_rows(c, nullptr, cache, true, len, count, t, key, key_stride, value, value_stride, pos,
                       turns, n_pairs, layout, factor, q, q_stride, q_heads, q_out, q_out_stride);
}


namespace {

// sj_attend (cache) and sj_attend8 (cache8).
int attend_rows(sj_ctx *c, const sj_cache *cache, const sj_cache8 *cache8, bool eight, const int32_t *len,
                const int32_t *count, uint32_t t, const void *q, const int64_t q_stride[3],
                uint32_t q_heads, const uint64_t *tree, const int64_t tree_stride[2], double scale,
                void *out, float *lse, const float *w_in, float *w_out, uint64_t w_cols)
{
    g_err.clear();
    const Alone alone(c);
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    sjc::Attend a{};
    int st;
    if ((st = eight ? check_cache8(c, cache8, "cache", &a.c)
                    : check_cache(c, cache, "cache", &a.c)) != SJ_OK)
        return st;
    const bool f16 = (eight ? cache8->rows.dtype : cache->dtype) == SJ_F16;
    const uint32_t B = a.c.batch, d = a.c.d;
    if (q_heads == 0 || q_heads % a.c.heads != 0)
        return fail(SJ_E_INVAL, "%u query heads do not divide over %u cache heads", q_heads,
                    a.c.heads);
    if (std::isnan(scale))
        return fail(SJ_E_INVAL, "scale is NaN");
    if (!q_stride || (tree && !tree_stride))
        return fail(SJ_E_INVAL, "strides are NULL");
    if ((uint64_t)t * (q_heads / a.c.heads) >= kMaxCells || w_cols >= kMaxCells ||
        (uint64_t)B * t * q_heads >= kMaxCells)
        return fail(SJ_E_UNSUPPORTED, "%u x %u tokens of %u heads are too many", B, t, q_heads);
    if (B == 0)
        return SJ_OK;
    const uint64_t q_rows = (uint64_t)B * t * q_heads;
    const Axis aq[3] = {{B, q_stride[0]}, {t, q_stride[1]}, {q_heads, q_stride[2]}};
    if ((st = check_array(c, len, (uint64_t)B * 4, 4, "len")) != SJ_OK ||
        (count && (st = check_array(c, count, (uint64_t)B * 4, 4, "count")) != SJ_OK) ||
        (st = check_strided(c, q, aq, 3, d, "q")) != SJ_OK ||
        (st = check_array(c, out, q_rows * d * 2, 2, "out")) != SJ_OK ||
        (lse && (st = check_array(c, lse, q_rows * 4, 4, "lse")) != SJ_OK))
        return st;
    if (out == q && q_rows) {
        // each workgroup writes the query rows that it has read, but the weights read q again
        if (w_out && w_cols)
            return fail(SJ_E_INVAL, "out must not be q where weights are asked for");
        if ((B > 1 && (uint64_t)q_stride[0] != (uint64_t)t * q_heads * d) ||
            (t > 1 && (uint64_t)q_stride[1] != (uint64_t)q_heads * d) ||
            (q_heads > 1 && q_stride[2] != d))
            return fail(SJ_E_INVAL, "out is q with other strides");
    }
    const uint64_t w_bytes = (uint64_t)B * a.c.heads * w_cols * 4;
    if (w_out) {
        if ((st = check_array(c, w_out, w_bytes, 4, "w_out")) != SJ_OK ||
            (w_in && (st = check_array(c, w_in, w_bytes, 4, "w_in")) != SJ_OK))
            return st;
    } else if (w_in) {
        return fail(SJ_E_INVAL, "w_in without w_out");
    }
    if (tree && t) {
        const uint64_t words = ((uint64_t)t + 63) / 64;
        for (int i = 0; i < 2; ++i)
            if (tree_stride[i] < 0 || tree_stride[i] > kMaxStride)
                return fail(SJ_E_INVAL, "tree: stride %lld is negative or too large",
                            (long long)tree_stride[i]);
        if ((st = check_array(c, tree,
                              ((uint64_t)(B - 1) * (uint64_t)tree_stride[0] +
                               (uint64_t)(t - 1) * (uint64_t)tree_stride[1] + words) *
                                  8,
                              8, "tree")) != SJ_OK)
            return st;
    }
    a.len = len;
    a.count = count;
    a.t = t;
    a.group = q_heads / a.c.heads;
    a.by_group = sjc::PageDiv::of(a.group);
    a.q_heads = q_heads;
    a.q = (const uint16_t *)q;
    a.q_seq = q_stride[0];
    a.q_tok = q_stride[1];
    a.q_head = q_stride[2];
    a.tree = tree;
    if (tree) {
        a.tree_seq = tree_stride[0];
        a.tree_tok = tree_stride[1];
    }
    // (above 0, so that -inf stays -inf: at 1e-30 every finite score is as good as 0)
    a.scale2 = (float)std::fmax(std::fabs(scale) * 1.4426950408889634074, 1e-30);
    a.negate = scale < 0;
    a.out = (uint16_t *)out;
    a.w_in = w_in;
    a.w_out = w_out;
    a.w_cols = w_cols;
    SJ_HIP(hipSetDevice(c->device));
    // work split and scratch: [plan][lse][maxima and sums][sums of values][scores]
    const uint32_t rows = t * a.group, qt = sjc::attend_tile_rows(rows, d);
    const uint32_t dp = d <= 64 ? 64 : (d <= 128 ? 128 : 256);
    a.tiles = rows == 0 ? 1 : (rows + qt - 1) / qt;
    // Two heads at once where rows are 8 bits and shares of one head each would more than fill the
    // GPU (32 sequences of 200 to 8192 rows of 8 heads of 128: 77 us one at a time, 68 two, 73
    // four; heads of 64: 54, 41, 50; one sequence of 2048 rows of 2 heads, which cannot fill it: 12
    // and 16).  A kernel of its own joins these shares: where the last workgroup does, it reads
    // twice the heads' results alone (2 x 131072 rows 125 and 113 us; 2 x 10865 to 19681 rows of 16
    // heads of 72 with 18 query rows 74 and 38).  The host knows the table's room and not the lengths, so
    // short sequences of a wide table are taken two heads at once too, with the kernel that joins
    // (4 x 500 rows of 8 heads of 128: 11 us with room for 512 rows, 14 for 16384; 2048 rows of one
    // sequence: 12, and 14 for 131072).
    const uint64_t least = sjc::AT_ROWS * sjc::AT_WAVES;
    const bool fills = eight && qt <= 32 &&
                       B * ((a.c.room + least - 1) / least) * a.c.heads * a.tiles > 8 * (uint64_t)c->num_cus;
    a.heads_at_once = fills && a.c.heads % 2 == 0 ? 2 : 1;
    int per_cu;
    if (eight)
        per_cu = (f16 ? sjc::attend8_occupancy_f16 : sjc::attend8_occupancy_bf16)(d, qt, a.heads_at_once);
    else
        per_cu = (f16 ? sjc::attend_occupancy_f16 : sjc::attend_occupancy_bf16)(d, qt);
    const uint64_t units = (uint64_t)a.c.heads * a.tiles, held = (uint64_t)c->num_cus * per_cu;
    const uint64_t groups = units / a.heads_at_once;
    a.want = held / groups > 0 ? (uint32_t)(held / groups) : 1;
    // (no more workgroups than shares of the least size could use)
    const uint64_t room_shares = B * ((a.c.room + least - 1) / least + 1);
    a.slots = a.want > B ? a.want : B;
    a.slots = a.slots < room_shares ? a.slots : (uint32_t)room_shares;
    a.w_want = 2 * c->num_cus / a.c.heads > 0 ? 2 * c->num_cus / a.c.heads : 1;
    const uint64_t parts = a.slots * units;
    if (parts >= kMaxCells)
        return fail(SJ_E_UNSUPPORTED, "%u sequences of %llu query tiles are too many", B,
                    (unsigned long long)units);
    const size_t off_lse = align_up((size_t)B * 8);
    const size_t off_ml = off_lse + align_up(lse ? 0 : (size_t)q_rows * 4);
    // (with as many sequences as shares wanted every sequence is one share, and nothing joins)
    a.whole = B >= a.want;
    const uint64_t kept_parts = a.whole ? 0 : parts;
    const size_t off_o = off_ml + align_up((size_t)kept_parts * qt * 8);
    // Weights need every query row's lse, so the scores a second time.  Up to 16 query
    // rows they are kept (8 bytes written and read again per row of the cache and
    // query row, 128 at most); beyond, and where they would fill too much memory, the
    // keys are multiplied again (2 d bytes per row, 256 for d = 128).
    const size_t off_s = off_o + align_up((size_t)kept_parts * qt * dp * 4);
    const uint64_t cols = w_cols < a.c.room ? w_cols : a.c.room;
    a.s_cols = (uint32_t)((cols + 31) / 32 * 32);
    const uint64_t s_bytes = (uint64_t)B * a.c.heads * rows * a.s_cols * 4;
    const bool keep = w_out && rows <= 16 && s_bytes > 0 && s_bytes <= kMaxScores;
    const bool counted = qt <= 32 && !keep && !a.whole && !fills;
    if ((st = grow_both(c, off_s + (keep ? (size_t)s_bytes : 0), counted ? (size_t)B * units : 0)) !=
        SJ_OK)
        return st;
    uint8_t *s = (uint8_t *)c->scratch;
    a.plan = (uint32_t *)s;
    a.arrivals = counted ? c->arrivals : nullptr;
    a.lse = lse ? lse : (float *)(s + off_lse);
    a.part_ml = (float *)(s + off_ml);
    a.part_o = (float *)(s + off_o);
    a.scores = keep ? (float *)(s + off_s) : nullptr;
    SJ_HIP((eight ? (f16 ? sjc::launch_attend8_f16 : sjc::launch_attend8_bf16)
                  : (f16 ? sjc::launch_attend_f16 : sjc::launch_attend_bf16))(a, c->stream));
    return SJ_OK;
}

}  // namespace

extern "C" int sj_attend(sj_ctx *c, const sj_cache *cache, const int32_t *len, const int32_t *count,
                         uint32_t t, const void *q, const int64_t q_stride[3], uint32_t q_heads,
                         const uint64_t *tree, const int64_t tree_stride[2], double scale, void *out,
                         float *lse, const float *w_in, float *w_out, uint64_t w_cols)
{
    return attend_rows(c, cache, nullptr, false, len, count, t, q, q_stride, q_heads, tree, tree_stride,
                       scale, out, lse, w_in, w_out, w_cols);
}

extern "C" int sj_attend8(sj_ctx *c, const sj_cache8 *cache, const int32_t *len, const int32_t *count,
                         uint32_t t, const void *q, const int64_t q_stride[3], uint32_t q_heads,
                         const uint64_t *tree, const int64_t tree_stride[2], double scale, void *out,
                         float *lse, const float *w_in, float *w_out, uint64_t w_cols)
{
    return attend_rows(c, nullptr, cache, true, len, count, t, q, q_stride, q_heads, tree, tree_stride,
                       scale, out, lse, w_in, w_out, w_cols);
}


extern "C" int sj_cache_evict(sj_ctx *c, const sj_cache *src, const int32_t *len,
                              const float *weight, uint32_t sets, uint64_t w_cols, uint32_t keep,
                              uint32_t sink, uint32_t recent, const sj_cache *dst, int32_t *index,
                              int32_t *new_len, float *w_out, uint64_t w_out_cols)
{
    g_err.clear();
    const Alone alone(c);
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    sjc::Evict e{};
    int st;
    if ((st = check_cache(c, src, "src", &e.src)) != SJ_OK ||
        (st = check_cache(c, dst, "dst", &e.dst)) != SJ_OK)
        return st;
    if (src->dtype != dst->dtype || e.src.heads != e.dst.heads || e.src.d != e.dst.d ||
        e.src.batch != e.dst.batch)
        return fail(SJ_E_INVAL, "src and dst differ in dtype, heads, d or batch");
    if (sets != 1 && sets != e.src.heads)
        return fail(SJ_E_INVAL, "sets = %u is neither 1 nor the number of heads, %u", sets,
                    e.src.heads);
    if ((uint64_t)sink + recent > keep)
        return fail(SJ_E_INVAL, "sink + recent = %llu is above keep = %u",
                    (unsigned long long)sink + recent, keep);
    if (src->k == dst->k && src->table == dst->table && e.src.room)
        return fail(SJ_E_INVAL, "dst must not share rows with src");
    const uint32_t most = keep < e.src.room ? keep : e.src.room;
    if (most > e.dst.room || keep >= kMaxCells || w_cols >= kMaxCells || w_out_cols >= kMaxCells)
        return fail(SJ_E_UNSUPPORTED, "%u rows may stay, dst has room for %u", most, e.dst.room);
    const uint64_t B = e.src.batch;
    if (B == 0)
        return SJ_OK;
    if ((st = check_array(c, len, B * 4, 4, "len")) != SJ_OK ||
        (st = check_array(c, new_len, B * 4, 4, "new_len")) != SJ_OK ||
        (st = check_array(c, weight, B * sets * w_cols * 4, 4, "weight")) != SJ_OK ||
        (st = check_array(c, index, B * sets * keep * 4, 4, "index")) != SJ_OK ||
        (w_out && (st = check_array(c, w_out, B * sets * w_out_cols * 4, 4, "w_out")) != SJ_OK))
        return st;
    if (w_out && w_out == weight && w_cols)
        return fail(SJ_E_INVAL, "w_out must not be weight");
    if (new_len == len)
        return fail(SJ_E_INVAL, "new_len must not be len");
    SJ_HIP(hipSetDevice(c->device));
    e.len = len;
    e.weight = weight;
    e.sets = sets;
    e.w_cols = w_cols;
    e.w_out_cols = w_out_cols;
    e.keep = keep;
    e.sink = sink;
    e.recent = recent;
    e.index = index;
    e.new_len = new_len;
    e.w_out = w_out;
    e.chunks = sjc::evict_chunks(e.src.room);
    if (e.chunks) {
        const size_t off = align_up((size_t)sjc::evict_hist_values(B * sets, e.chunks) * 4);
        if ((st = grow_both(c, off + (size_t)sjc::evict_state_values(B * sets, e.chunks) * 4, 0)) !=
            SJ_OK)
            return st;
        e.hist = (uint32_t *)c->scratch;
        e.state = (uint32_t *)((uint8_t *)c->scratch + off);
    }
    SJ_HIP(sjc::launch_evict(e, c->stream));
    return SJ_OK;
}

extern "C" int sj_cache_pages(sj_ctx *c, const int32_t *table, int64_t table_row, uint32_t batch,
                              uint32_t width, uint32_t pages, uint32_t page, const int32_t *len,
                              const int32_t *parent, uint32_t out_batch, uint32_t tokens,
                              int32_t *out_table, int32_t *new_len, int32_t *copies,
                              int32_t *lacking)
{
    g_err.clear();
    const Alone alone(c);
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    if (page == 0)
        return fail(SJ_E_INVAL, "page must be positive");
    if ((uint64_t)width * page > kMaxRows || page >= kMaxCells || pages >= kMaxCells ||
        batch >= kMaxCells || (uint64_t)out_batch * width >= kMaxCells || out_batch > (1u << 22))
        return fail(SJ_E_UNSUPPORTED, "%u sequences of %u pages of %u rows are too many", out_batch,
                    width, page);
    if (out_batch == 0)
        return SJ_OK;
    int st;
    if (batch && width) {
        if (table_row < 0 || table_row > kMaxStride)
            return fail(SJ_E_INVAL, "table_row is negative or too large");
        if ((st = check_array(c, table, ((uint64_t)(batch - 1) * (uint64_t)table_row + width) * 4, 4,
                              "table")) != SJ_OK)
            return st;
    }
    const uint64_t n = out_batch;
    if ((st = check_array(c, len, (uint64_t)batch * 4, 4, "len")) != SJ_OK ||
        (parent && (st = check_array(c, parent, n * 4, 4, "parent")) != SJ_OK) ||
        (st = check_array(c, out_table, n * width * 4, 4, "out_table")) != SJ_OK ||
        (st = check_array(c, new_len, n * 4, 4, "new_len")) != SJ_OK ||
        (st = check_array(c, copies, n * 12, 4, "copies")) != SJ_OK ||
        (st = check_array(c, lacking, n * 4, 4, "lacking")) != SJ_OK)
        return st;
    if ((out_table == table && width) || new_len == len)
        return fail(SJ_E_INVAL, "out_table must not be table, and new_len not len");
    SJ_HIP(hipSetDevice(c->device));
    // scratch: [base][kept][pages given out][their number]; no more pages are given out than there
    // are, nor than the table's entries.  Counters: [workgroups][bits][holders]
    const uint64_t given = n * width < pages ? n * width : pages, words = ((uint64_t)pages + 31) / 32;
    const size_t off_kept = align_up((size_t)n * 4), off_free = off_kept + align_up((size_t)n * 4);
    const size_t off_n = off_free + align_up((size_t)given * 4);
    if ((st = grow_both(c, off_n + 256, (size_t)(1 + words + pages))) != SJ_OK)
        return st;
    uint8_t *s = (uint8_t *)c->scratch;
    sjc::Pages p{};
    p.table = table;
    p.len = len;
    p.parent = parent;
    p.table_row = table_row;
    p.batch = batch;
    p.width = width;
    p.pages = pages;
    p.room = width * page;
    p.out_batch = out_batch;
    p.tokens = tokens;
    p.div = sjc::PageDiv::of(page);
    p.out_table = out_table;
    p.new_len = new_len;
    p.copies = copies;
    p.lacking = lacking;
    p.arrived = c->arrivals;
    p.used = c->arrivals + 1;
    p.holder = c->arrivals + 1 + words;
    p.base = (uint32_t *)s;
    p.kept = (int32_t *)(s + off_kept);
    p.free = (int32_t *)(s + off_free);
    p.n_free = (uint32_t *)(s + off_n);
    SJ_HIP(sjc::launch_pages(p, c->stream));
    return SJ_OK;
}

namespace {

int copy_rows(sj_ctx *c, sjc::Copy &k, const int32_t *copies, uint32_t n)
{
    const uint64_t chunks = ((uint64_t)k.c.d * k.size + 15) / 16;
    if (k.c.heads > 65535 || (uint64_t)k.c.div.page * k.c.heads * chunks >= kMaxCells - 65536)
        return fail(SJ_E_UNSUPPORTED, "pages of %u rows of %u heads are too long", k.c.div.page,
                    k.c.heads);
    if (n == 0 || k.c.pages == 0)
        return SJ_OK;
    int st;
    if ((st = check_array(c, copies, (uint64_t)n * 12, 4, "copies")) != SJ_OK)
        return st;
    k.copies = copies;
    k.n = n;
    SJ_HIP(hipSetDevice(c->device));
    SJ_HIP(sjc::launch_copy(k, c->stream));
    return SJ_OK;
}

}  // namespace

extern "C" int sj_cache_copy(sj_ctx *c, const sj_cache *cache, const int32_t *copies, uint32_t n)
{
    g_err.clear();
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    if (!cache)
        return fail(SJ_E_INVAL, "cache is NULL");
    sjc::Copy k{};
    k.size = 2;
    sj_cache pool = *cache;     // (whatever sequences there are)
    pool.table = nullptr;
    pool.batch = 0;
    const int st = check_cache(c, &pool, "cache", &k.c);
    return st != SJ_OK ? st : copy_rows(c, k, copies, n);
}

extern "C" int sj_cache8_copy(sj_ctx *c, const sj_cache8 *cache, const int32_t *copies, uint32_t n)
{
    g_err.clear();
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    if (!cache)
        return fail(SJ_E_INVAL, "cache is NULL");
    sjc::Copy k{};
    k.size = 1;
    sj_cache8 pool = *cache;
    pool.rows.table = nullptr;
    pool.rows.batch = 0;
    const int st = check_cache8(c, &pool, "cache", &k.c);
    return st != SJ_OK ? st : copy_rows(c, k, copies, n);
}

extern "C" int sj_verify(sj_ctx *c, int dtype, uint32_t batch, uint32_t t, uint32_t vocab,
                         const int64_t *tokens, const int32_t *parent, int64_t parent_seq,
                         const int32_t *count, const void *target, const int64_t target_stride[2],
                         const void *draft, const int64_t draft_stride[2], const float *uniform,
                         int32_t *path, int32_t *found, int64_t *next)
{
    g_err.clear();
    const Alone alone(c);
    if (!c)
        return fail(SJ_E_INVAL, "context is NULL");
    if (dtype != SJ_F16 && dtype != SJ_BF16 && dtype != SJ_F32)
        return fail(SJ_E_INVAL, "dtype %d is none of SJ_F16, SJ_BF16 and SJ_F32", dtype);
    if (t == 0 || vocab == 0)
        return fail(SJ_E_INVAL, "t and vocab must be positive");
    if (draft && parent)
        return fail(SJ_E_INVAL, "draft goes with chains, not with parent");
    if (!target_stride || (draft && !draft_stride))
        return fail(SJ_E_INVAL, "strides are NULL");
    sjc::Verify v{};
    // Two parts a workgroup where those of one would not all run at once, since each walks through its
    // sequence's nodes first (64 chains of 131072 tokens: 29 us in one part, 25 in two, 27 in four).
    v.chunks = (vocab + sjc::VE_CHUNK - 1) / sjc::VE_CHUNK;
    v.parts = (uint64_t)batch * v.chunks > 6 * (uint64_t)c->num_cus ? 2 : 1;
    v.chunks = (v.chunks + v.parts - 1) / v.parts;
    if (t > sjc::VE_MOST || vocab >= kMaxCells || batch >= kMaxCells / 1024 ||
        (uint64_t)batch * v.chunks >= kMaxCells)
        return fail(SJ_E_UNSUPPORTED, "%u sequences of %u nodes and %u tokens are too many", batch, t,
                    vocab);
    if (batch == 0)
        return SJ_OK;
    const uint64_t n = (uint64_t)batch * t;
    const uint32_t size = dtype == SJ_F32 ? 4 : 2;
    const Axis ap[2] = {{batch, target_stride[0]}, {t, target_stride[1]}};
    int st;
    if ((st = check_array(c, tokens, n * 8, 8, "tokens")) != SJ_OK ||
        (count && (st = check_array(c, count, (uint64_t)batch * 4, 4, "count")) != SJ_OK) ||
        (st = check_strided(c, target, ap, 2, vocab, "target", size)) != SJ_OK ||
        (st = check_array(c, uniform, n * 4, 4, "uniform")) != SJ_OK ||
        (st = check_array(c, path, n * 4, 4, "path")) != SJ_OK ||
        (st = check_array(c, found, (uint64_t)batch * 4, 4, "found")) != SJ_OK ||
        (st = check_array(c, next, (uint64_t)batch * 8, 8, "next")) != SJ_OK)
        return st;
    if (draft && t > 1) {
        const Axis aq[2] = {{batch, draft_stride[0]}, {t - 1, draft_stride[1]}};
        if ((st = check_strided(c, draft, aq, 2, vocab, "draft", size)) != SJ_OK)
            return st;
    }
    if (parent) {
        if (parent_seq < 0 || parent_seq > kMaxStride)
            return fail(SJ_E_INVAL, "parent_seq is negative or too large");
        if ((st = check_array(c, parent, ((uint64_t)(batch - 1) * (uint64_t)parent_seq + t) * 4, 4,
                              "parent")) != SJ_OK)
            return st;
    }
    SJ_HIP(hipSetDevice(c->device));
    if ((st = grow_both(c, (size_t)batch * v.chunks * 8, batch)) != SJ_OK)
        return st;
    v.dtype = dtype;
    v.batch = batch;
    v.t = t;
    v.vocab = vocab;
    v.tokens = tokens;
    v.parent = parent;
    v.count = count;
    v.parent_seq = parent_seq;
    v.target = target;
    v.draft = t > 1 ? draft : nullptr;
    v.p_seq = target_stride[0];
    v.p_row = target_stride[1];
    if (draft) {
        v.q_seq = draft_stride[0];
        v.q_row = draft_stride[1];
    }
    v.uniform = uniform;
    v.path = path;
    v.found = found;
    v.next = next;
    v.sums = (double *)c->scratch;
    v.arrivals = c->arrivals;
    SJ_HIP(sjc::launch_verify(v, c->stream));
    return SJ_OK;
}
