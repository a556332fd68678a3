"""Pages of a cache on the GPU: tables of sequences that go on, fork and end, and copies of pages,
entry by entry against their definition."""
import numpy as np
import pytest

from oracle import cache8 as ref8
from test_cache_gpu import dev, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2006_12608_amd  # noqa: F401  (fails loudly when libsj.so is missing)
    yield
    torch.cuda.synchronize()


def check(table, lens, tokens, pages, page, parent=None):
    import paper_2006_12608_amd as sj
    table = np.asarray(table, np.int32)
    want = ref8.pages(table, lens, tokens, pages, page, parent)
    got = sj.cache_pages(dev(table), dev(np.asarray(lens, np.int32)), tokens, pages=pages, page=page,
                         parent=None if parent is None else dev(np.asarray(parent, np.int32)))
    for name, x, y in zip(("table", "lengths", "copies", "lacking"), got, want):
        x = x.cpu().numpy()
        assert x.shape == y.shape and np.array_equal(x, y), (name, np.argwhere(x != y)[:4])
    return want


def held(rng, B, width, pages, page, lens):
    table, order = np.full((B, width), -1, np.int32), rng.permutation(pages)
    at = 0
    for b in range(B):
        n = -(-min(max(lens[b], 0), width * page) // page)
        table[b, :n] = order[at:at + n]
        at += n
    return table


@pytest.mark.parametrize("seed", range(12))
def test_sequences_fork_go_on_and_end(seed):
    rng = np.random.default_rng(seed)
    B, page = int(rng.integers(1, 40)), int(rng.choice([1, 2, 16, 48]))
    out, width = int(rng.integers(1, 120)), int(rng.integers(1, 60))
    lens = rng.integers(0, width * page + 1, B)
    pages = int(sum(-(-lens // page)) + rng.integers(0, out * 4))
    pages = max(pages, 1)
    table = held(rng, B, width, pages, page, lens)
    parent = rng.integers(-1, B, out)
    say("pages", seed, B, out, page, width, pages)
    check(table, lens, int(rng.integers(0, 3 * page)), pages, page, parent)
    check(table, lens, int(rng.integers(0, 3 * page)), pages, page)


def test_forks_of_forks():
    """Sequences share pages, fall back into a page that another one has full, and go on."""
    say("forks of forks")
    table, n, _, _ = check([[0, 1, 2, -1]], [9], 4, 30, 4, [0, 0, 0])
    n[1] = 6        # rows taken back: inside a page that 0 and 2 have full
    table, n, copies, _ = check(table, n, 4, 30, 4, [1, 1, 0, 2, 5, -3])
    assert copies[0, 0] == 1 and copies[1, 0] == 1      # nobody may write into it
    check(table, n, 40, 30, 4, [3, 2, 1, 0])


@pytest.mark.parametrize("lens", [[0, 0], [-4, 10 ** 9], [33, 64]])
def test_lengths_outside_the_room_and_pages_that_do_not_exist(lens):
    say("pages odd", lens)
    table = [[3, -1, 2 ** 31 - 1, 9], [8, 4, 5, -2 ** 31]]
    for tokens in (0, 1, 17, 2 ** 31):
        check(table, lens, tokens, 9, 16)
        check(table, lens, tokens, 9, 16, [1, 1, 0])


@pytest.mark.parametrize("pages,out", [(1, 3), (31, 2), (32, 2), (33, 70), (100000, 1500)])
def test_sizes_around_words_and_workgroups(pages, out):
    say("pages sizes", pages, out)
    rng = np.random.default_rng(pages)
    B, page, width = 3, 16, 5000 if pages > 50000 else 9
    lens = [min(pages // 3 * page, width * page) - 5 * b for b in range(B)]
    table = held(rng, B, width, pages, page, lens)
    check(table, lens, 20, pages, page, rng.integers(0, B, out))
    check(table[:, ::-1][:, ::-1], lens, 20, pages, page)


def test_nothing_to_do():
    import torch
    import paper_2006_12608_amd as sj
    say("pages nothing")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    out = sj.cache_pages(none.view(0, 4), none, 3, pages=5, page=2, parent=none)
    assert [tuple(x.shape) for x in out] == [(0, 4), (0,), (0, 3), (0,)]
    check(np.zeros((2, 0), np.int32), [3, 0], 5, 4, 16)
    check([[0]], [5], 3, 0, 16)
    check(np.zeros((0, 3), np.int32), [], 5, 4, 16, [0, 1])


def test_pages_strided_table_refusals_and_graph():
    import torch
    import paper_2006_12608_amd as sj
    say("pages graph")
    wide = torch.arange(40, dtype=torch.int32, device="cuda").view(4, 10)
    lens = dev(np.array([20, 5, 9, 0], np.int32))
    parent = dev(np.array([0, 0, 2], np.int32))
    got = sj.cache_pages(wide[:, 2:8], lens, 6, pages=50, page=4, parent=parent)
    want = ref8.pages(wide[:, 2:8].cpu().numpy(), [20, 5, 9, 0], 6, 50, 4, np.array([0, 0, 2]))
    assert all(np.array_equal(x.cpu().numpy(), y) for x, y in zip(got, want))
    for bad in (dict(tokens=-1), dict(pages=-1), dict(page=0), dict(tokens=2 ** 32), dict(pages=2 ** 33)):
        kw = dict(dict(tokens=1, pages=5, page=2), **bad)
        with pytest.raises(ValueError):
            sj.cache_pages(wide, lens, kw["tokens"], pages=kw["pages"], page=kw["page"])
    with pytest.raises(ValueError):
        sj.cache_pages(wide, lens[:3], 1, pages=5, page=2)
    with pytest.raises(ValueError):
        sj.cache_pages(wide.long(), lens, 1, pages=5, page=2)
    with pytest.raises(ValueError):
        sj.cache_pages(wide, lens, 1, pages=5, page=2, parent=parent.long())
    with pytest.raises(sj.SjError):
        sj.cache_pages(wide, lens, 1, pages=5, page=2 ** 30)
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sj.cache_pages(wide, lens, 6, pages=50, page=4, parent=parent)
    side.synchronize()
    with torch.cuda.graph(g, stream=side):
        out = sj.cache_pages(wide, lens, 6, pages=50, page=4, parent=parent)
    for i in range(4):
        lens.copy_(dev(np.array([20 + i, 5 * i, 9, 3], np.int32)))
        parent.copy_(dev(np.array([0, i % 4, 2], np.int32)))
        g.replay()
        want = sj.cache_pages(wide, lens, 6, pages=50, page=4, parent=parent)
        assert all(torch.equal(x, y) for x, y in zip(out, want)), i


# ---------------------------------------------------------------------- copies

def pool(rng, kind, shape, order):
    import torch
    x = rng.integers(0, 2 ** 16, shape).astype(np.uint16)
    t = torch.from_numpy(x.view(np.int16)).to("cuda").view(torch.float16)
    if kind == "8":
        t = torch.from_numpy((x & 255).astype(np.uint8)).to("cuda")
    if order == "heads":
        t = t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    elif order == "wide":
        big = torch.zeros((*shape[:3], 2 * shape[3] + 3), dtype=t.dtype, device="cuda")
        big[..., 1:shape[3] + 1] = t
        t = big[..., 1:shape[3] + 1]
    return t.view(torch.float8_e4m3fn) if kind == "8" else t


def raw(t):
    import torch
    return t.view(torch.uint8 if t.dtype == torch.float8_e4m3fn else torch.int16).cpu().numpy()


@pytest.mark.parametrize("kind", ["16", "8"])
@pytest.mark.parametrize("order", ["rows", "heads", "wide"])
@pytest.mark.parametrize("page,heads,d,block", [(16, 2, 64, 4), (1, 1, 8, 1), (7, 3, 72, 7), (100, 1, 256, 25),
                                                (300, 16, 128, 100), (64, 1, 24, 64)])
def test_copies(kind, order, page, heads, d, block):
    import torch
    import paper_2006_12608_amd as sj
    say("copies", kind, order, page, heads, d)
    rng = np.random.default_rng(page)
    pages = 12
    k, v = (pool(rng, kind, (pages, page, heads, d), order) for _ in "kv")
    ex = dev(rng.integers(-9, 9, (pages, page // block, heads, 2)).astype(np.int8))
    cache = sj.kv_cache8(k, v, ex) if kind == "8" else sj.kv_cache(k, v)
    copies = np.array([[0, 5, page], [0, 6, 1], [3, 7, page // 2], [-1, -1, 0], [3, 3, page], [2, pages, 4],
                       [pages, 8, 4], [2, 9, 0], [2, 10, -5], [1, 11, 10 ** 9], [-2, 4, 3]], np.int32)
    want = [raw(k), raw(v), ex.cpu().numpy()]
    for a, b, n in copies.tolist():
        if 0 <= a < pages and 0 <= b < pages and n > 0:
            n = min(n, page)
            for x in want[:2]:
                x[b, :n] = x[a, :n]
            if kind == "8":
                want[2][b, :-(-n // block)] = want[2][a, :-(-n // block)]
    sj.cache_copy(cache, dev(copies))
    for x, y in zip((raw(k), raw(v), ex.cpu().numpy()), want):
        assert np.array_equal(x, y), np.argwhere(x != y)[:3]
    sj.cache_copy(cache, torch.empty(0, 3, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        sj.cache_copy(cache, dev(copies[:, :2]))
    with pytest.raises(ValueError):
        sj.cache_copy(cache, dev(copies.astype(np.int64)))


@pytest.mark.parametrize("d", [33, 1, 200])
def test_copies_of_odd_heads(d):
    import paper_2006_12608_amd as sj
    say("copies odd", d)
    rng = np.random.default_rng(d)
    k, v = (pool(rng, "16", (40000, 2, 2, d), "rows") for _ in "kv")
    copies = np.stack([rng.permutation(20000), 20000 + rng.permutation(20000), rng.integers(0, 3, 20000)],
                      1).astype(np.int32)
    want = [raw(k), raw(v)]
    for x in want:
        for n in (1, 2):
            c = copies[copies[:, 2] >= n]
            x[c[:, 1], n - 1] = x[c[:, 0], n - 1]
    sj.cache_copy(sj.kv_cache(k, v), dev(copies))
    assert np.array_equal(raw(k), want[0]) and np.array_equal(raw(v), want[1])


def test_forked_sequences_answer_for_themselves():
    """A prompt in a cache in 8 bits, forked twice and gone on with differently: each fork's attention is that
    of a sequence of its own."""
    import torch
    import paper_2006_12608_amd as sj
    say("forks answer")
    g = torch.Generator("cuda").manual_seed(3)
    page, heads, d, pages = 16, 2, 64, 40

    def cache(table):
        k, v = (torch.zeros(pages, page, heads, d, dtype=torch.uint8, device="cuda")
                .view(torch.float8_e4m3fn) for _ in "kv")
        return sj.kv_cache8(k, v, torch.zeros(pages, 2, heads, 2, dtype=torch.int8, device="cuda"), table)

    def rows(B, T):
        return torch.randn(B, T, heads, d, generator=g, device="cuda").bfloat16()
    lens = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    empty = torch.full((2, 8), -1, dtype=torch.int32, device="cuda")
    table, lens, _, lacking = sj.cache_pages(empty, lens, 53, pages=pages, page=page)
    assert not lacking.any()
    shared = cache(table)
    prompt, value = rows(2, 53), rows(2, 53)
    sj.cache_append(shared, lens, prompt, value)
    lens = torch.tensor([53, 40], dtype=torch.int32, device="cuda")
    parent = torch.tensor([0, 0, 1, 0], dtype=torch.int32, device="cuda")
    table, lens, copies, lacking = sj.cache_pages(table, lens, 9, pages=pages, page=page, parent=parent)
    assert not lacking.any() and (copies[[0, 2], 0] == -1).all() and (copies[[1, 3], 0] >= 0).all()
    sj.cache_copy(shared, copies)
    shared.table = table
    own = cache(torch.arange(32, dtype=torch.int32, device="cuda").view(4, 8))
    counts = torch.tensor([53, 53, 40, 53], dtype=torch.int32, device="cuda")
    at = parent.long()
    sj.cache_append(own, torch.zeros_like(lens), prompt[at].contiguous(), value[at].contiguous(), counts=counts)
    new, q = rows(4, 9), torch.randn(4, 9, 8, d, generator=g, device="cuda").bfloat16()
    outs = []
    for c in (shared, own):
        sj.cache_append(c, lens, new, new)
        outs.append(sj.attend(c, lens, q))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
