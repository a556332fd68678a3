"""A cache in 8 bits on the GPU: appended rows bit for bit against their definition, and attention
against the definition in 64 bits over the values that the elements stand for, which are values of
the 16-bit type: the tolerances are those of attention over a cache in 16 bits."""
import numpy as np
import pytest

from oracle import cache as ref
from oracle import cache8 as ref8
from test_cache_gpu import SHAPES, Case, chain_tree, check_attend, dev, host, say, tdtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2006_12608_amd  # noqa: F401  (fails loudly when libsj.so is missing)
    yield
    torch.cuda.synchronize()


def dev8(b):
    import torch
    return torch.from_numpy(np.ascontiguousarray(b)).to("cuda").view(torch.float8_e4m3fn)


def bytes_of(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def wide8(t, order):
    """The e4m3 tensor in another order of memory, or inside a wider one at an odd place."""
    import torch
    u = t.view(torch.uint8)
    if order == "heads":
        u = u.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    elif order == "wide":
        big = torch.full((*u.shape[:3], 2 * u.shape[3] + 3), 127, dtype=torch.uint8, device="cuda")
        big[..., 1:u.shape[3] + 1] = u
        u = big[..., 1:u.shape[3] + 1]
    return u.view(torch.float8_e4m3fn)


class Case8(Case):
    """A case of a cache in 16 bits with its rows rounded to 8, blocks of `block` rows; c.k and c.v hold
    the values that the elements stand for."""

    def __init__(self, seed, dtype, B, T, heads, group, d, page, lens, block, order="rows", **kw):
        super().__init__(seed, dtype, B, T, heads, group, d, page, lens, **kw)
        import paper_2006_12608_amd as sj
        page, pages = self.page, self.k.shape[0]
        if page % block:
            block = page
        self.block, nb = block, page // block
        rng = np.random.default_rng(seed + 1)
        self.ex = rng.integers(-6, 3, (pages, nb, heads, 2)).astype(np.int8)
        self.b8 = []
        for i, x in enumerate((self.k, self.v)):
            two = 2.0 ** np.repeat(self.ex[..., i].astype(np.float64), block, 1)[..., None]
            b8 = ref8.to_e4m3(x * 4 / two)
            self.b8.append(b8)
            x[:] = ref8.e4m3(b8) * two
        self.k8, self.v8 = (wide8(dev8(b), order) for b in self.b8)
        self.dex = dev(self.ex)
        self.cache = sj.kv_cache8(self.k8, self.v8, self.dex,
                                  None if self.table is None else dev(self.table),
                                  dtype=tdtype(dtype))


EIGHTS = [s for s in SHAPES if s[4] % 8 == 0]
# heads of 8, of a half chunk of 16, and of few query rows over many rows, whose shares are joined in steps
EIGHTS += [(2, 3, 2, 2, 8, 16, [40, 5]), (1, 20, 2, 2, 8, 16, [300]), (2, 2, 4, 4, 24, 16, [700, 33]),
           (1, 1, 4, 4, 56, 16, [9000]), (2, 1, 2, 4, 128, 64, [9000, 12000]), (1, 3, 4, 4, 72, 64, [20000]),
           (1, 6, 2, 4, 64, 16, [14000]), (1, 1, 3, 4, 128, 64, [30000]), (1, 1, 2, 7, 232, 64, [9000]),
           (1, 1, 16, 8, 64, 64, [6000])]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", EIGHTS, ids=lambda s: "x".join(map(str, s[:6])))
@pytest.mark.parametrize("mask", ["chain", "tree"])
def test_attend8(dtype, shape, mask):
    B, T, heads, group, d, page, lens = shape
    say("attend8", dtype, shape[:6], mask)
    block = {16: 4, 64: 16, 48: 48, 100: 10, 256: 64, 24: 8, 32: 16}.get(page, 1)
    c = Case8(B + T + d, dtype, B, T, heads, group, d, page, lens, block)
    tree = chain_tree(c.rng, B, T) if mask == "tree" else None
    weight = c.rng.random((B, heads, c.cache.room + 5)).astype(np.float32)
    check_attend(c, tree, weight)


def widen_table(c, room):
    """The same rows in a table with room for more, whose further pages do not exist."""
    more = np.full((c.B, -(-room // c.page) - c.table.shape[1]), -1, np.int32)
    c.table = np.concatenate([c.table, more], 1)
    c.cache.table = dev(c.table)
    return c


# Room enough that a workgroup takes two heads (of an odd number: one), of 1 to 32 query rows, in one
# share a sequence or several; heads of every variant
WIDES = [
    # B, T, heads, group, d, page, lens, room
    (4, 1, 32, 4, 64, 64, [0, 1, 700, 310], 2560),
    (3, 3, 32, 2, 128, 64, [300, 650, 33], 3000),
    (3, 8, 16, 4, 72, 16, [40, 500, 0], 6000),
    (2, 5, 16, 4, 256, 64, [400, 10], 9000),
    (2, 2, 16, 8, 136, 48, [47, 300], 9000),
    (2, 3, 32, 1, 8, 16, [200, 5], 5000),
    (2, 7, 32, 3, 24, 16, [333, 128], 5000),
    (1, 1, 31, 4, 56, 64, [900], 9000),
    (2, 20, 31, 1, 64, 7, [300, 20], 5000),
    (300, 1, 16, 2, 64, 16, [(7 * b) % 60 for b in range(300)], 128),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", WIDES, ids=lambda s: "x".join(map(str, s[:6])))
@pytest.mark.parametrize("mask", ["chain", "tree"])
def test_attend8_wide_tables(dtype, shape, mask):
    import torch
    import paper_2006_12608_amd as sj
    B, T, heads, group, d, page, lens, room = shape
    say("attend8 wide", dtype, shape[:6], mask)
    assert B * -(-room // 128) * heads > 8 * 256
    counts = [T, max(T - 2, 0)] * (B // 2) + [T] * (B % 2) if T > 4 else None
    c = widen_table(Case8(31, dtype, B, T, heads, group, d, page, lens, 8 if page % 8 == 0 else 1,
                          counts=counts), room)
    tree = chain_tree(c.rng, B, T) if mask == "tree" else None
    weight = c.rng.random((B, heads, c.cache.room + 5)).astype(np.float32)
    check_attend(c, tree, weight)
    check_attend(c, tree, None)
    # into its queries, on another stream: the same bits
    lens, q = dev(c.lens), c.dq.clone()
    kw = dict(tree=None if tree is None else dev(tree.view(np.int64)),
              counts=None if c.counts is None else dev(c.counts))
    want = sj.attend(c.cache, lens, c.dq, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sj.attend(c.cache, lens, q, out=q, **kw)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("heads,group", [(16, 2), (16, 5), (31, 1)])
def test_attend8_wide_tables_hidden_rows_may_hold_anything(dtype, heads, group):
    """NaN in one head of a drafted token's key and value reaches, of the head that shares its
    workgroup too, nothing but the tokens that see it there."""
    import torch
    import paper_2006_12608_amd as sj
    say("attend8 wide hidden", dtype, heads, group)
    T = 6
    c = widen_table(Case8(32, dtype, 1, T, heads, group, 64, 16, [300], 4), 20000)
    tree = np.zeros((1, T, 1), np.uint64)
    for t in range(T):
        tree[0, t, 0] = sum(1 << w for w in range(t + 1) if w != 2 or t == 2)
    r = ref.row_of(c.table, c.page, c.k.shape[0], 0, 302)
    args = (c.cache, dev(c.lens), c.dq, dev(tree.view(np.int64)))
    plain, _ = sj.attend(*args)
    for x in (c.k8, c.v8):
        x.view(torch.uint8)[r[0], r[1], 4] = 127
    got, lse = sj.attend(*args, weight_out=torch.zeros((1, heads, c.cache.room), device="cuda"))
    again, _ = sj.attend(*args)
    hit = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    hit[:, 2, 4 * group:5 * group] = True
    for x in (got, again):
        assert torch.isnan(x[hit]).all() and torch.equal(x[~hit], plain[~hit])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("order", ["heads", "wide"])
@pytest.mark.parametrize("table", ["mixed", None])
@pytest.mark.parametrize("T,d", [(3, 64), (3, 72), (25, 128), (60, 128), (90, 72)])
def test_attend8_strides(dtype, order, table, T, d):
    say("attend8 strides", dtype, order, table, T, d)
    c = Case8(11, dtype, 2, T, 2, 3, d, 16, [50, 7], 8, order=order, table=table)
    weight = np.zeros((2, 2, c.cache.room), np.float32)
    check_attend(c, chain_tree(c.rng, 2, T), weight)
    check_attend(c, None, weight, dq=c.dq.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("mask", ["chain", "tree", "nothing", "some"])
@pytest.mark.parametrize("group", [2, 6])
def test_attend8_counts_and_empty_rows(dtype, mask, group):
    say("attend8 empty", dtype, mask, group)
    c = Case8(3, dtype, 6, 9, 2, group, 64, 16, [0, 40, 0, 9, -5, 100], 4, counts=[9, 4, 0, 20, 3, -1])
    tree = None
    if mask != "chain":
        tree = chain_tree(c.rng, 6, 9)
        if mask == "nothing":
            tree[:] = 0
        if mask == "some":
            tree[:, ::2] = 0
    check_attend(c, tree, np.ones((6, 2, c.cache.room), np.float32))


@pytest.mark.parametrize("hole", [(0, 0), (1, 2), (1, slice(0, 3))])
@pytest.mark.parametrize("group", [2, 8])
def test_attend8_pages_that_do_not_exist(hole, group):
    say("attend8 hole", hole, group)
    c = Case8(5 + sum(map(ord, str(hole))), "f16", 2, 6, 2, group, 64, 16, [40, 38], 16, hole=hole)
    check_attend(c, chain_tree(c.rng, 2, 6), np.zeros((2, 2, c.cache.room), np.float32))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("group", [1, 4, 8, 12])
def test_attend8_hidden_rows_may_hold_anything(dtype, group):
    """NaN in a drafted token's key and value reaches only the tokens that see it."""
    import torch
    import paper_2006_12608_amd as sj
    say("attend8 hidden", dtype, group)
    T = 6
    c = Case8(21, dtype, 1, T, 2, group, 64, 16, [20], 4)
    tree = np.zeros((1, T, 1), np.uint64)
    for t in range(T):
        tree[0, t, 0] = sum(1 << w for w in range(t + 1) if w != 2 or t == 2)
    r = ref.row_of(c.table, c.page, c.k.shape[0], 0, 22)
    plain, _ = sj.attend(c.cache, dev(c.lens), c.dq, dev(tree.view(np.int64)))
    for x in (c.k8, c.v8):
        x.view(torch.uint8)[r[0], r[1]] = 127
    w = torch.zeros((1, 2, c.cache.room), device="cuda")
    got, lse = sj.attend(c.cache, dev(c.lens), c.dq, dev(tree.view(np.int64)), weight_out=w)
    others = [0, 1, 3, 4, 5]
    assert torch.equal(got[:, others], plain[:, others])
    assert torch.isfinite(lse[:, others]).all()
    assert torch.isnan(got[:, 2]).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_byte_at_every_exponent(dtype):
    """One row a token, which sees nothing else: its output is the row's values, rounded to the
    type where an exponent takes them out of its range."""
    import torch
    import paper_2006_12608_amd as sj
    say("bytes", dtype)
    es = np.array([-128, -127, -126, -118, -117, -100, -20, -16, -15, -10, -1, 0, 3, 7, 8, 60, 118, 119]
                  if dtype == "bf16" else [-15, -14, -13, -9, -8, -7, -1, 0, 1, 5, 6, 7], np.int8)
    B, d = len(es), 256
    b8 = np.tile(np.arange(256, dtype=np.uint8), (B, 16, 1, 1))
    b8[(b8 & 127) == 127] = 0
    ex = np.zeros((B, 1, 1, 2), np.int8)
    ex[:, 0, 0, 1] = es
    cache = sj.kv_cache8(dev8(np.zeros_like(b8)), dev8(b8), dev(ex), dtype=tdtype(dtype))
    q = torch.zeros(B, 1, 1, d, dtype=tdtype(dtype), device="cuda")
    out, _ = sj.attend(cache, torch.zeros(B, dtype=torch.int32, device="cuda"), q)
    want = ref8.e4m3(b8[:, 0, 0]) * 2.0 ** np.maximum(es.astype(np.float64), -126)[:, None]
    small = np.abs(want) < 2.0 ** -126      # (below the matrix cores' least normal number)
    got = host(out)[:, 0, 0]
    assert np.array_equal(got[~small], want[~small])
    assert (np.abs(got[small]) < 2.0 ** -126).all()


def appended(c, key, value, **kw):
    """Runs an append of a Case8 and of its oracle: both's bytes and exponents have to be the same."""
    import paper_2006_12608_amd as sj
    pages = c.k8.shape[0]
    counts = kw.pop("counts", None)
    sj.cache_append(c.cache, dev(c.lens), key, value, counts=None if counts is None else dev(counts), **kw)
    ref8.append(c.b8[0], c.b8[1], c.ex, lambda b, n: ref.row_of(c.table, c.page, pages, b, n), c.lens,
                host(key), host(value), c.block, c.dtype, counts, c.cache.room)
    check_bytes(c)


def check_bytes(c):
    for name, got, want in (("k", c.k8, c.b8[0]), ("v", c.v8, c.b8[1])):
        got = bytes_of(got)
        same = (got == want) | ((got & 127 == 127) & (want & 127 == 127))
        assert same.all(), (name, np.argwhere(~same)[:4], got[~same][:4], want[~same][:4])
    assert np.array_equal(c.dex.cpu().numpy(), c.ex), np.argwhere(c.dex.cpu().numpy() != c.ex)[:4]


APPENDS = [
    # B, T, heads, d, page, block, lens
    (1, 1, 1, 8, 1, 1, [0]),
    (4, 1, 2, 128, 16, 16, [0, 1, 15, 16]),
    (3, 5, 3, 72, 48, 16, [14, 0, 47]),
    (2, 40, 2, 64, 16, 4, [3, 16]),
    (2, 33, 1, 256, 64, 64, [63, 10]),
    (1, 300, 2, 80, 256, 256, [100]),
    (2, 70, 2, 128, 100, 50, [99, 0]),
    (3, 2, 1, 192, 7, 7, [6, 5, 0]),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", APPENDS, ids=lambda s: "x".join(map(str, s[:6])))
def test_append8(dtype, shape):
    """Rows of very different sizes, so that exponents grow and stay; twice, the second time behind
    the first."""
    import torch
    B, T, heads, d, page, block, lens = shape
    say("append8", dtype, shape)
    c = Case8(B + T + d, dtype, B, 2 * T, heads, 1, d, page, lens, block)
    rng = np.random.default_rng(T)
    for _ in range(2):
        x = rng.standard_normal((B, T, 2 * heads, d)) * 2.0 ** rng.integers(-9, 9, (B, T, 2 * heads, 1))
        x[rng.random(x.shape) < 0.1] = 0.0
        key, value = dev(x, dtype).split([heads, heads], 2)
        appended(c, key, value)
        c.lens = c.lens + T
    assert isinstance(c.dex, torch.Tensor)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_append8_values_of_every_kind(dtype):
    """Zeros alone, infinities and NaN, the type's largest and least values, ties of the rounding."""
    say("append8 kinds", dtype)
    c = Case8(8, dtype, 6, 4, 1, 1, 32, 8, [0, 3, 8, 0, 1, 7], 4)
    x = np.zeros((6, 4, 1, 32))
    x[1, :, :, ::3] = np.inf
    x[1, 1, :, 1] = -3.0
    x[2] = np.nan
    x[3] = 65504.0 if dtype == "f16" else 3.3e38
    x[3, :, :, 5:] = 1.0
    x[4] = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133
    x[5, :, 0, :] = 256.0
    x[5, :, 0, 1:] = np.arange(31) + 16.5 + np.arange(4)[:, None] / 4
    t = dev(x, dtype)
    appended(c, t, t.neg())


@pytest.mark.parametrize("e", [127, 126, 125, 119, -118, -126, -127, -128])
def test_append8_behind_rows_of_every_exponent(e):
    """Exponents that the append does not set itself, at the ends of int8 (below -126: as -126): one that is
    not less than the new rows' stays, the others' rows are rounded to the new one; what the rows
    stand for is the same."""
    say("append8 exponents", e)
    c = Case8(20, "bf16", 3, 2, 2, 1, 32, 16, [5, 1, 14], 8)
    for name, b in (("k8", c.b8[0]), ("v8", c.b8[1])):
        b[...] = c.rng.integers(0, 0x40, b.shape)       # (below 2, so that values stay finite)
        getattr(c, name).copy_(dev8(b))
    c.ex[...] = e
    c.dex.copy_(dev(c.ex))
    x = np.zeros((3, 2, 2, 32))
    x[0] = 3.2e38 * np.linspace(-1, 1, 32)
    x[1] = 2.0 ** -120
    key = dev(x, "bf16")
    p, s = c.table[0, 0], slice(0, 5)
    want = ref8.e4m3(c.b8[1][p, s]) * 2.0 ** max(e, -126)
    appended(c, key, key)
    top = 119 if e < 119 else e
    assert (c.ex[p, 0] == top).all()
    got = ref8.e4m3(bytes_of(c.v8)[p, s]) * 2.0 ** int(c.dex[p, 0, 0, 1])
    assert (np.abs(got - want) <= (2.0 ** (top - 10) if e < 119 else 0)).all()


def test_append8_counts_holes_and_the_room():
    say("append8 counts")
    c = Case8(9, "bf16", 7, 9, 2, 1, 64, 16, [0, 15, 20, 3, 14, -7, 30], 8, hole=(2, 1))
    c.lens[6] = c.cache.room - 4        # the last rows do not fit
    counts = np.array([9, 0, 6, 100, -1, 4, 9], np.int32)
    key = dev(c.rng.standard_normal((7, 9, 2, 64)), "bf16")
    appended(c, key, key * 3, counts=counts)


@pytest.mark.parametrize("turn", [False, True])
@pytest.mark.parametrize("page,block,T", [(16, 16, 3), (256, 128, 90)])
def test_append8_idle_sequences_leave_the_pages_they_name(page, block, T, turn):
    """Sequences that append nothing (a count of 0 or less) name the page that another one appends
    much larger rows to, or hold rows at an exponent below the type's: they write nothing."""
    import torch
    import paper_2006_12608_amd as sj
    say("append8 idle", page, block, T, turn)
    heads, d = 16, 64
    lens = [5, 7, 1, 15, 3, 9, 14, 4]
    c = Case8(18, "bf16", 8, T, heads, 1, d, page, lens, block)
    c.table[1:7] = c.table[0]
    c.cache.table = dev(c.table)
    c.ex[c.table[7, 0], 0] = -120
    c.dex.copy_(dev(c.ex))
    counts = np.array([T, 0, 0, -1, 0, -9, 0, 0], np.int32)
    key = dev(c.rng.standard_normal((8, T, heads, d)) * 2.0 ** 14, "bf16")
    before = c.ex.copy()
    kw = {}
    if turn:        # by nothing: turned rows are the rows
        kw = dict(pos=torch.zeros(8, T, dtype=torch.int32, device="cuda"), turns=sj.rotary_turns(32))
    appended(c, key, key.flip(2), counts=counts, **kw)
    assert (c.ex[c.table[0, 0], 0] > before[c.table[0, 0], 0]).all()
    assert (c.ex[c.table[7, 0], 0] == -120).all()


@pytest.mark.parametrize("order", ["heads", "wide"])
def test_append8_strides(order):
    say("append8 strides", order)
    c = Case8(10, "f16", 2, 20, 3, 1, 40, 16, [5, 31], 16, order=order)
    x = c.rng.standard_normal((2, 3, 20, 41))
    key = dev(x, "f16").permute(0, 2, 1, 3)[..., 1:]
    appended(c, key, key.flip(1))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot,T,page,block", [(64, 64, 1, 16, 8), (128, 64, 20, 16, 8), (72, 40, 7, 16, 8),
                                                (80, 38, 33, 16, 8), (256, 252, 3, 16, 8), (128, 128, 70, 64, 16),
                                                (128, 112, 90, 128, 64), (96, 96, 50, 100, 50), (64, 64, 300, 64, 64)])
def test_append8_turned(dtype, layout, d, rot, T, page, block):
    """Turned keys are the ones that a cache in 16 bits gets, rounded to 8; so are the queries."""
    import torch
    import paper_2006_12608_amd as sj
    say("append8 turned", dtype, layout, d, rot, T)
    c = Case8(12, dtype, 3, T, 2, 2, d, page, [0, 9, 16], block)
    turns = sj.rotary_turns(rot)
    key = dev(c.rng.standard_normal((3, T, 2, d)), dtype)
    pos = torch.randint(-5, 100000, (3, T), dtype=torch.int32, device="cuda")
    turned = sj.rotary(key.view(3 * T, 2, d), pos.view(-1), turns, layout=layout, factor=1.25)
    want_q = sj.rotary(c.dq.view(3 * T, 4, d), pos.view(-1), turns, layout=layout, factor=1.25)
    q = sj.cache_append(c.cache, dev(c.lens), key, key, pos=pos, turns=turns, q=c.dq, layout=layout,
                        factor=1.25)
    ref8.append(c.b8[0], c.b8[1], c.ex, lambda b, n: ref.row_of(c.table, c.page, c.k8.shape[0], b, n),
                c.lens, host(turned.view(3, T, 2, d)), host(key), c.block, dtype)
    check_bytes(c)
    assert torch.equal(q.view(want_q.shape), want_q)


@pytest.mark.parametrize("layout,rot,page", [("half", 38, 16), ("interleaved", 64, 256)])
def test_append8_refused_in_a_capture_leaves_the_queries(layout, rot, page):
    """Keys that pass through scratch: where it would grow during a capture the call is refused, and
    nothing of it is in the graph; queries turned in place are turned once, by the call that is not
    refused."""
    import torch
    import paper_2006_12608_amd as sj
    say("append8 refused", layout, rot, page)
    c = Case8(19, "bf16", 2, 5, 2, 2, 80, page, [3, 16], page)
    turns = sj.rotary_turns(rot)
    lens, key = dev(c.lens), c.dq[:, :, :2].clone()
    pos = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5) + 1
    q = c.dq.clone()
    want = sj.rotary(q.view(10, 4, 80), pos.view(-1), turns, layout=layout).view(q.shape)
    turned = sj.rotary(key.view(10, 2, 80), pos.view(-1), turns, layout=layout).view(key.shape)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    ctx = sj.sj_create(torch.cuda.current_device(), stream.cuda_stream)
    args = (c.cache, lens, key, key)
    kw = dict(pos=pos, turns=turns, q=q, q_out=q, layout=layout, ctx=ctx)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        with pytest.raises(sj.SjError, match="capture"):
            sj.cache_append(*args, **kw)
        seen = q + 0
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q, c.dq) and torch.equal(seen, c.dq)
    check_bytes(c)
    with torch.cuda.stream(stream):
        sj.cache_append(*args, **kw)
    torch.cuda.synchronize()
    assert torch.equal(q, want)
    ref8.append(c.b8[0], c.b8[1], c.ex, lambda b, n: ref.row_of(c.table, c.page, c.k8.shape[0], b, n),
                c.lens, host(turned), host(key), c.block, c.dtype)
    check_bytes(c)
    del graph
    sj.sj_destroy(ctx)


def test_append8_then_attend_graph():
    """Append and attend captured together, replayed with other inputs, lengths and pages in place."""
    import torch
    import paper_2006_12608_amd as sj
    say("append8 graph")
    c = Case8(13, "bf16", 3, 4, 2, 4, 64, 16, [30, 5, 44], 8)
    lens, key = dev(c.lens), torch.empty(3, 4, 2, 64, dtype=torch.bfloat16, device="cuda")
    q = torch.empty_like(c.dq)
    w = torch.zeros(3, 2, c.cache.room, device="cuda")

    def both():
        sj.cache_append(c.cache, lens, key, key)
        return sj.attend(c.cache, lens, q, weight_out=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        key.normal_()
        q.normal_()
        both()
    side.synchronize()
    with torch.cuda.graph(g, stream=side):
        out, lse = both()
    saved = [x.view(torch.uint8).clone() for x in (c.k8, c.v8)] + [c.dex.clone()]
    for i in range(4):
        key.normal_(std=2.0 ** i)
        q.normal_()
        lens.copy_(dev((c.lens - i).astype(np.int32)))
        w.fill_(7.0)
        g.replay()
        got = [x.clone() for x in (out, lse, w)] + [x.view(torch.uint8).clone() for x in (c.k8, c.v8)]
        ex = c.dex.clone()
        c.k8.view(torch.uint8).copy_(saved[0])
        c.v8.view(torch.uint8).copy_(saved[1])
        c.dex.copy_(saved[2])
        a, b = both()
        want = [a, b, w] + [x.view(torch.uint8) for x in (c.k8, c.v8)]
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(ex, c.dex)
        saved = [x.view(torch.uint8).clone() for x in (c.k8, c.v8)] + [c.dex.clone()]


def test_refusals():
    import torch
    import paper_2006_12608_amd as sj
    say("refusals8")
    c = Case8(14, "bf16", 2, 2, 2, 2, 64, 16, [3, 4], 8)
    k, v, ex = c.k8, c.v8, c.dex
    with pytest.raises(ValueError):
        sj.kv_cache8(k.view(torch.uint8), v, ex)
    with pytest.raises(ValueError):
        sj.kv_cache8(k, v, ex[:, :1])
    with pytest.raises(ValueError):
        sj.kv_cache8(k[:, :15], v[:, :15], ex)
    with pytest.raises(ValueError):
        sj.kv_cache8(k[..., :60], v[..., :60], ex)
    with pytest.raises(ValueError):
        sj.kv_cache8(k, v, ex, dtype=torch.float32)
    with pytest.raises(ValueError):
        sj.kv_cache(k, v)
    with pytest.raises(ValueError):
        sj.attend(c.cache, dev(c.lens), c.dq.half())
    with pytest.raises(ValueError):
        sj.cache_append(c.cache, dev(c.lens), c.dq[:, :, :2].half(), c.dq[:, :, :2].half())
    w = torch.zeros(2, 2, c.cache.room, device="cuda")
    with pytest.raises(ValueError):
        sj.cache_evict(c.cache, dev(c.lens), w, c.cache, keep=1)
    ex2 = c.dex.clone()
    with pytest.raises(ValueError):
        c.cache.exponents = ex2[:1]
    assert c.cache.exponents is c.dex
    c.cache.exponents = ex2
    assert c.cache.raw.exponents == ex2.data_ptr()
    # the C entries' own checks
    ctx, raw = sj.context(), c.cache.raw
    lens = dev(c.lens)
    args = (lens.data_ptr(), None, 2, c.dq.data_ptr(), c.dq.stride()[:3], 4, None, (0, 0), 1.0,
            c.dq.data_ptr(), None)
    for field, bad, code in (("block", 0, sj.SJ_E_INVAL), ("block", 5, sj.SJ_E_INVAL),
                             ("exponents", None, sj.SJ_E_INVAL),
                             ("exponents", ex2.data_ptr() + 1, sj.SJ_E_INVAL)):
        r = sj.sj_cache8(raw.rows, raw.exponents, raw.block)
        setattr(r, field, bad)
        assert sj.sj_attend8(ctx, r, *args) == code, (field, sj.sj_last_error())
    r = sj.sj_cache8(raw.rows, raw.exponents, raw.block)
    r.rows.d = 60
    assert sj.sj_attend8(ctx, r, *args) == sj.SJ_E_UNSUPPORTED
    r.rows.d, r.rows.dtype = 64, sj.SJ_I8
    assert sj.sj_attend8(ctx, r, *args) == sj.SJ_E_INVAL


def test_pools_without_pages_and_calls_without_tokens():
    import torch
    import paper_2006_12608_amd as sj
    say("empty8")
    none = torch.empty(0, 16, 2, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ex = torch.empty(0, 2, 2, 2, dtype=torch.int8, device="cuda")
    table = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    lens = torch.tensor([0, 5, -1], dtype=torch.int32, device="cuda")
    x = torch.randn(3, 2, 2, 64, device="cuda").bfloat16()
    cache = sj.kv_cache8(none, none, ex, table)
    sj.cache_append(cache, lens, x, x)
    w = torch.full((3, 2, 9), 7.0, device="cuda")
    out, lse = sj.attend(cache, lens, x, weight_out=w)
    assert (out == 0).all() and (lse == -np.inf).all() and (w == 0).all()
    sj.cache_copy(cache, torch.zeros(2, 3, dtype=torch.int32, device="cuda"))
    c = Case8(16, "bf16", 2, 3, 2, 2, 64, 16, [3, 4], 8)
    sj.cache_append(c.cache, dev(c.lens), c.dq[:, :0, :2], c.dq[:, :0, :2])
    check_bytes(c)
    out, lse = sj.attend(c.cache, dev(c.lens), c.dq[:, :0])
    assert out.shape == (2, 0, 4, 64) and lse.shape == (2, 0, 4)


@pytest.mark.parametrize("T,weights", [(1, False), (7, True), (60, True)])
def test_attend8_into_its_queries_and_on_another_stream(T, weights):
    """out may be q where no weights are asked for; a call on a side stream gives the same bits."""
    import torch
    import paper_2006_12608_amd as sj
    say("attend8 streams", T)
    c = Case8(17, "bf16", 4, T, 4, 4, 128, 64, [9000, 30, 7000, 12000], 16)
    lens = dev(c.lens)
    kw = dict(weight_out=torch.empty(4, 4, c.cache.room, device="cuda")) if weights else {}
    want = sj.attend(c.cache, lens, c.dq, **kw)
    first = [x.clone() for x in want] + [x.clone() for x in kw.values()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [*sj.attend(c.cache, lens, c.dq, **kw), *kw.values()]
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(first, got))
    if not weights:
        q = c.dq.clone()
        out, lse = sj.attend(c.cache, lens, q, out=q)
        assert out is q and torch.equal(q, first[0]) and torch.equal(lse, first[1])


def test_gradients_are_not_lost_silently():
    import torch
    import paper_2006_12608_amd as sj
    say("autograd8")
    c = Case8(15, "bf16", 2, 2, 2, 2, 64, 16, [3, 4], 8)
    q = c.dq.clone().requires_grad_()
    out, _ = sj.attend(c.cache, dev(c.lens), q)
    with pytest.raises(RuntimeError):
        out.float().sum().backward()


def test_offsets_past_32_bits():
    """Rows further than 2^32 elements into the pool."""
    import torch
    import paper_2006_12608_amd as sj
    say("far8")
    pages, page, heads, d = 2 ** 16 + 8, 64, 8, 136         # 4.56e9 elements
    k = torch.zeros(pages, page, heads, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros(pages, page, heads, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    ex = torch.zeros(pages, 1, heads, 2, dtype=torch.int8, device="cuda")
    table = torch.tensor([[pages - 1, pages - 2], [pages - 3, 0]], dtype=torch.int32, device="cuda")
    cache = sj.kv_cache8(k, v, ex, table)
    lens = torch.tensor([60, 0], dtype=torch.int32, device="cuda")
    x = torch.randn(2, 20, heads, d, device="cuda").bfloat16()
    sj.cache_append(cache, lens, x, x)
    b8 = np.zeros((3, page, heads, d), np.uint8), np.zeros((3, page, heads, d), np.uint8)
    e = np.zeros((3, 1, heads, 2), np.int8)
    at = {0: [0, 1], 1: [2]}
    ref8.append(b8[0], b8[1], e, lambda b, n: (at[b][n // page], n % page), [60, 0], host(x), host(x), page,
                "bf16")
    far = [pages - 1, pages - 2, pages - 3]
    assert np.array_equal(bytes_of(k[far[0]:].contiguous()), b8[0][:1])
    for i, p in enumerate(far):
        assert np.array_equal(k.view(torch.uint8)[p].cpu().numpy(), b8[0][i])
        assert np.array_equal(ex[p].cpu().numpy(), e[i])
    out, _ = sj.attend(cache, lens, x, torch.tensor([[[1 << u] for u in range(20)]], device="cuda"))
    assert out.shape == x.shape and torch.isfinite(out).all()
    copies = torch.tensor([[pages - 3, 5, 20]], dtype=torch.int32, device="cuda")
    sj.cache_copy(cache, copies)
    assert np.array_equal(k.view(torch.uint8)[5].cpu().numpy(), b8[0][2])
