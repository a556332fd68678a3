"""Edges of the calls on a cache of key and value rows: infinite keys, long tails of small
weights, launches past 2^32 threads, graphs, threads, autograd and arguments that alias."""
import numpy as np
import pytest

from oracle import cache as ref
from test_cache_gpu import Case, U, chain_tree, dev, host, say, tdtype

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2006_12608_amd  # noqa: F401  (fails loudly when libsj.so is missing)
    yield
    torch.cuda.synchronize()


def check_row_at_minus_infinity(c, tree, w, out, n0):
    """out and w (numpy) against the definition for a cache in which row n0's key scores -inf:
    the row weighs 0, and everything else is as if it did not exist."""
    d = c.q.shape[-1]
    r = ref.row_of(c.table, c.page, c.k.shape[0], 0, n0)
    plain = c.k.copy()
    plain[r] = 0.0
    dots = ref.attend(plain, c.v, c.table, c.lens, c.q, tree, d ** -0.5, c.counts)[4]
    want, lse, want_w, mag, _ = ref.attend(c.k, c.v, c.table, c.lens, c.q, tree, d ** -0.5, c.counts)
    assert np.isfinite(lse).all() and (want_w[0, :, n0] == 0).all()
    u, n = U[c.dtype], c.cache.room
    rho = 4 * (d + 4) * 2.0 ** -24 * dots.max() + n * 2.0 ** -23 + 2.0 ** -19
    tol = u * np.abs(want) + (u + rho) * mag + 2.0 ** -25 + n * 2.0 ** -25 * np.nanmax(np.abs(c.v))
    assert (np.abs(out - want) <= tol).all()
    R = c.q.shape[1] * c.q.shape[2] // c.k.shape[2]
    assert (w[0, :, n0] == 0).all(), w[0, :, n0]
    tol = (rho + (R + 2) * 2.0 ** -24) * want_w + 1e-30
    assert (np.abs(w[..., :want_w.shape[2]] - want_w) <= tol).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T,group,d", [(4, 4, 64), (5, 4, 64), (10, 4, 128), (25, 4, 128), (16, 4, 64),
                                       (5, 5, 256), (31, 3, 256), (33, 5, 72), (70, 4, 64)])
def test_weights_of_a_row_hidden_by_an_infinite_key(dtype, T, group, d):
    """A cached key whose element is -inf where every query's is positive: its score is -inf,
    its weight 0, whatever number of query rows the tiles are padded from."""
    import torch
    import paper_2006_12608_amd as sj
    say("infinite key", dtype, T, group, d)
    c = Case(81, dtype, 1, T, 2, group, d, 16, [300])
    c.dq[..., 3] = 1.0
    c.q = host(c.dq)
    for n0 in (5, 299):     # in a block of cached rows only, and beside the tokens' own
        r = ref.row_of(c.table, c.page, c.k.shape[0], 0, n0)
        kept = c.dk[r[0], r[1]].clone()
        c.dk[r[0], r[1], :, 3] = float("-inf")
        c.k = host(c.dk)
        w = torch.full((1, 2, c.cache.room), float("nan"), device="cuda")
        out, lse = sj.attend(c.cache, dev(c.lens), c.dq, weight_out=w)
        check_row_at_minus_infinity(c, None, host(w), host(out), n0)
        c.dk[r[0], r[1]] = kept


def test_weights_of_an_infinite_key_without_kept_scores():
    """16 query rows over so many columns that their scores are not kept."""
    import torch
    import paper_2006_12608_amd as sj
    say("infinite key, wide")
    page, width = 65536, 257
    c = Case(82, "bf16", 1, 4, 1, 4, 64, 512, [300])
    n0 = 17
    k, v = (torch.zeros(1, page, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    for n in range(304):
        r = ref.row_of(c.table, c.page, c.k.shape[0], 0, n)
        if n == n0:
            c.dk[r[0], r[1], :, 3] = float("-inf")
        k[0, n], v[0, n] = c.dk[r[0], r[1]], c.dv[r[0], r[1]]
    c.dq[..., 3] = 1.0
    c.q, c.k = host(c.dq), host(c.dk)
    w = torch.full((1, 1, page * width), float("nan"), device="cuda")
    out, _ = sj.attend(sj.kv_cache(k, v, table), dev(c.lens), c.dq, weight_out=w)
    assert (w[..., 304:] == 0).all()
    check_row_at_minus_infinity(c, None, host(w[..., :c.cache.room]), host(out), n0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 24, 40, 100, 200])
@pytest.mark.parametrize("x", [16.6, 17.4])
def test_attend_far_tail(dtype, T, x):
    """32768 rows of weight e^-x beside one of weight 1 whose value is 0: the rows are all there
    is of the output.  Their exponentials enter the product as 16-bit values, rounded by u each,
    and the output is rounded once; sums over n rows in fp32 and the exponentials' own error make
    n 2^-24 + 2^-19.  Sequences enough that none is cut: a share without the row of weight 1
    would take its tail's weights as 1."""
    import torch
    import paper_2006_12608_amd as sj
    say("far tail", dtype, T, x)
    n, d, B, page = 32769, 64, 2100, 64
    width = -(-(n + T) // page)
    k = torch.zeros(width, page, 1, d, device="cuda", dtype=tdtype(dtype))
    v = torch.ones_like(k)
    rows = k.view(-1, d)
    rows[:, 0] = -x
    rows[0, 0] = 0
    rows[n:, 0] = -240
    v.view(-1, d)[0] = 0
    x = -float(rows[1, 0])
    q = torch.zeros(B, T, 1, d, device="cuda", dtype=k.dtype)
    q[..., 0] = 1
    table = torch.arange(width, dtype=torch.int32, device="cuda")[None].expand(B, width)
    out, lse = sj.attend(sj.kv_cache(k, v, table), torch.full((B,), n, dtype=torch.int32, device="cuda"),
                         q, scale=1.0)
    w = 32768 * np.exp(-x)
    want = w / (1 + w)
    tol = (2 * U[dtype] + n * 2.0 ** -24 + 2.0 ** -19) * want
    assert float((out.double() - want).abs().max()) <= tol
    assert float((lse.double() - np.log1p(w)).abs().max()) <= n * 2.0 ** -24 + 2.0 ** -19


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("T", [1, 24, 40, 100, 200])
@pytest.mark.parametrize("step", [0.01, 0.2, 3.0])
def test_attend_rising_scores(dtype, T, step):
    """Scores that grow along the rows, so that the running maximum follows again and again:
    nothing overflows, and exponentials below the smallest normal number of fp16 (rounded by
    2^-25) are far below the largest: at most 2^-36 of it a row."""
    import torch
    import paper_2006_12608_amd as sj
    say("rising", dtype, T, step)
    n, d = 700, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    k = torch.zeros(1, n + T, 1, d, device="cuda", dtype=tdtype(dtype))
    v = torch.randn(1, n + T, 1, d, device="cuda", generator=g).to(k.dtype)
    steps = torch.arange(n + T, device="cuda") * step
    k[0, :, 0, 0] = steps.to(k.dtype)
    q = torch.zeros(1, T, 1, d, device="cuda", dtype=k.dtype)
    q[..., 0] = 1
    lens = np.array([n], np.int32)
    out, lse = sj.attend(sj.kv_cache(k, v), dev(lens), q, scale=1.0)
    want, want_lse, _, mag, dots = ref.attend(host(k), host(v), None, lens, host(q), None, 1.0)
    u = U[dtype]
    e = (d + 4) * 2.0 ** -24 * dots
    rho = 4 * e + (n + T) * 2.0 ** -23 + 2.0 ** -19
    tol = u * np.abs(want) + (u + rho[..., None]) * mag + 2.0 ** -25
    tol = tol + (n + T) * 2.0 ** -36 * float(v.abs().max())
    assert (np.abs(host(out) - want) <= tol).all()
    assert (np.abs(host(lse) - want_lse) <= 2 * e + (n + T) * 2.0 ** -24 +
            2.0 ** -20 * (1 + np.abs(want_lse))).all()


def test_rotary_and_append_of_more_tokens_than_a_launch_has_threads():
    """2^27 tokens of one head of 8: 8 tokens a workgroup of 256 would be 2^32 threads."""
    import torch
    import paper_2006_12608_amd as sj
    say("many tokens")
    n, half, d = 2 ** 27 + 1003, 2 ** 26, 8
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-2 ** 14, 2 ** 14, (n, 1, d), generator=g, device="cuda",
                      dtype=torch.int16).view(torch.float16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    turns = sj.rotary_turns(d)
    want = torch.empty_like(x)
    for at in (0, half, 2 * half):
        sj.rotary(x[at:at + half], pos[at:at + half], turns, out=want[at:at + half])
    assert torch.equal(sj.rotary(x, pos, turns).view(torch.int16), want.view(torch.int16))
    k, v = (torch.zeros(1, n + 5, 1, d, dtype=x.dtype, device="cuda") for _ in range(2))
    lens = torch.tensor([5], dtype=torch.int32, device="cuda")
    sj.cache_append(sj.kv_cache(k, v), lens, x[None], x[None], pos=pos[None], turns=turns)
    assert torch.equal(k[0, 5:].view(torch.int16), want.view(torch.int16))
    assert torch.equal(v[0, 5:].view(torch.int16), x.view(torch.int16))
    del x, want, k, v
    torch.cuda.empty_cache()


def test_evict_into_as_many_rows_as_a_cache_may_have():
    """keep = 2^30: workgroups of 64 rows would be 2^32 threads."""
    import torch
    import paper_2006_12608_amd as sj
    say("evict keep 2^30")
    page, width = 2 ** 20, 2 ** 10
    g = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn(2, page, 1, 8, generator=g, device="cuda").half() for _ in range(2))
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 1
    lens = torch.tensor([70000], dtype=torch.int32, device="cuda")
    w = torch.rand(1, 1, 100, generator=g, device="cuda")
    index, n, left = sj.cache_evict(sj.kv_cache(k, v, table), lens, w, sj.kv_cache(k2, v2, table),
                                    keep=2 ** 30, weight_out=torch.empty(1, 1, 200, device="cuda"))
    assert int(n) == 70000
    assert torch.equal(index[0, 0, :70000], torch.arange(70000, dtype=torch.int32, device="cuda"))
    assert (index[0, 0, 70000:] == -1).all()
    assert torch.equal(left[0, 0, :100], w[0, 0]) and (left[0, 0, 100:] == 0).all()
    assert torch.equal(k2[1, :70000], k[1, :70000]) and torch.equal(v2[1, :70000], v[1, :70000])
    assert (k2[0] == 0).all() and (k2[1, 70000:] == 0).all()
    del index
    torch.cuda.empty_cache()


def test_weights_of_more_columns_than_a_launch_has_threads():
    """8 heads of 2^31 - 1 columns: workgroups of 1024 columns would be 2^32 threads."""
    import torch
    import paper_2006_12608_amd as sj
    say("wide weights")
    torch.cuda.empty_cache()
    cols = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 90 * 2 ** 30:
        pytest.skip("needs 90 GB of device memory")
    c = Case(83, "bf16", 1, 2, 8, 2, 64, 16, [100])
    narrow = torch.empty(1, 8, c.cache.room, device="cuda")
    sj.attend(c.cache, dev(c.lens), c.dq, weight_out=narrow)
    w = torch.zeros(1, 8, cols, device="cuda")
    sj.attend(c.cache, dev(c.lens), c.dq, weight=w)
    assert torch.equal(w[..., :c.cache.room], narrow)
    for h in range(8):
        for part in w[0, h, c.cache.room:].split(2 ** 28):
            assert not part.any()
    del w
    torch.cuda.empty_cache()


def test_a_cache_with_a_table_of_no_pages_has_no_rows():
    """A table of width 0 is not the absence of a table: nothing is appended, seen or kept."""
    import torch
    import paper_2006_12608_amd as sj
    say("no pages")
    k, v = (torch.ones(2, 16, 1, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    c = sj.kv_cache(k, v, torch.zeros(2, 0, dtype=torch.int32, device="cuda"))
    assert c.room == 0
    lens = torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    row = torch.full((2, 1, 1, 64), 7.0, dtype=torch.float16, device="cuda")
    sj.cache_append(c, lens, row, row)
    assert (k == 1).all() and (v == 1).all()
    for T in (1, 40):
        w = torch.full((2, 1, 9), 5.0, device="cuda")
        out, lse = sj.attend(c, lens, row.expand(2, T, 1, 64).contiguous(), weight=w)
        assert (out == 0).all() and (lse == -np.inf).all() and (w == 5).all()
    into = sj.kv_cache(k.clone(), v.clone())
    index, n, _ = sj.cache_evict(c, lens, torch.ones(2, 1, 4, device="cuda"), into, keep=4)
    assert (index == -1).all() and (n == 0).all() and (into.k == 1).all()


def test_a_cache_follows_its_tensors():
    """Another table, or other rows, put into a cache is what the next call reads; one that
    does not fit is refused and changes nothing."""
    import torch
    import paper_2006_12608_amd as sj
    say("other table")
    c = Case(84, "f16", 2, 1, 2, 2, 64, 16, [60, 60])
    lens = dev(c.lens)
    want = sj.attend(c.cache, lens, c.dq)[0]
    other = torch.flip(c.cache.table, (0,)).contiguous()
    want_other = sj.attend(sj.kv_cache(c.dk, c.dv, other), lens, c.dq)[0]
    assert not torch.equal(want, want_other)
    first = c.cache.table
    c.cache.table = other
    assert torch.equal(sj.attend(c.cache, lens, c.dq)[0], want_other)
    with pytest.raises(ValueError):
        c.cache.table = other.long()
    with pytest.raises(ValueError):
        c.cache.k = c.dk[..., :32]
    assert torch.equal(sj.attend(c.cache, lens, c.dq)[0], want_other)
    c.cache.table = torch.cat([first, first[:, :1]], 1)      # wider
    assert c.cache.width == first.shape[1] + 1 and c.cache.room == 16 * c.cache.width
    assert torch.equal(sj.attend(c.cache, lens, c.dq)[0], want)
    c.cache.v = torch.zeros_like(c.dv)
    assert (sj.attend(c.cache, lens, c.dq)[0] == 0).all()


def test_evicted_lengths_that_alias_the_lengths_are_refused():
    """new_len = len, which workgroups still read when others write it."""
    import torch
    import paper_2006_12608_amd as sj
    say("aliases: len")
    c = Case(85, "f16", 2, 6, 2, 3, 64, 16, [60, 33])
    k2, v2 = torch.zeros_like(c.dk), torch.zeros_like(c.dv)
    into = sj.kv_cache(k2, v2, c.cache.table)
    lens, ctx = dev(c.lens), sj.context()
    w = torch.rand(2, 2, c.cache.room, device="cuda")
    index = torch.zeros(2, 2, 9, dtype=torch.int32, device="cuda")
    st = sj.sj_cache_evict(ctx, c.cache.raw, lens.data_ptr(), w.data_ptr(), 2, c.cache.room, 9, 0, 0,
                           into.raw, index.data_ptr(), lens.data_ptr())
    assert st == sj.SJ_E_INVAL and "len" in sj.sj_last_error()
    assert lens.tolist() == [60, 33] and (index == 0).all() and (k2 == 0).all()


def test_an_output_that_aliases_the_queries():
    """out = q is refused where the weights read q a second time, and right where they do not."""
    import torch
    import paper_2006_12608_amd as sj
    say("aliases: out")
    for T in (6, 30):
        c = Case(85, "f16", 2, T, 2, 3, 64, 16, [60, 33])
        lens, w = dev(c.lens), torch.rand(2, 2, c.cache.room, device="cuda")
        want = sj.attend(c.cache, lens, c.dq)[0]
        q = c.dq.clone()
        with pytest.raises(sj.SjError, match="out"):
            sj.attend(c.cache, lens, q, out=q, weight=w)
        assert torch.equal(q, c.dq)
        sj.attend(c.cache, lens, q, out=q)
        assert torch.equal(q, want)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary_takes_part_in_autograd(layout, inverse):
    """The gradient of rotary is rotary the other way round, with gradients of any strides,
    and has a gradient itself."""
    import torch
    import paper_2006_12608_amd as sj
    say("autograd", layout, inverse)
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn(9, 3, 20, generator=g, device="cuda").half().requires_grad_()
    pos = torch.arange(9, dtype=torch.int32, device="cuda") * 1001
    turns = sj.rotary_turns(12)
    kw = dict(layout=layout, factor=1.5)
    y = sj.rotary(x, pos, turns, inverse=inverse, **kw)
    assert y.requires_grad
    grad = torch.randn(9, 3, 20, generator=g, device="cuda").half()
    want = sj.rotary(grad, pos, turns, inverse=not inverse, **kw)
    y.backward(grad)
    assert torch.equal(x.grad, want)
    wide = grad.transpose(0, 2).contiguous().transpose(0, 2)     # elements not adjacent
    x.grad = None
    sj.rotary(x, pos, turns, inverse=inverse, **kw).backward(wide)
    assert torch.equal(x.grad, want)
    x.grad = None
    sj.rotary(x, pos, turns, inverse=inverse, **kw).sum().backward()
    assert torch.equal(x.grad, sj.rotary(torch.ones_like(grad), pos, turns, inverse=not inverse, **kw))
    v = grad.clone().requires_grad_()
    first, = torch.autograd.grad(sj.rotary(x, pos, turns, inverse=inverse, **kw), x, v, create_graph=True)
    second, = torch.autograd.grad(first, v, grad)
    assert torch.equal(second, sj.rotary(grad, pos, turns, inverse=inverse, **kw))
    with pytest.raises(ValueError, match="grad"):
        sj.rotary(x, pos, turns, out=torch.empty_like(grad))
    with torch.no_grad():
        assert torch.equal(sj.rotary(x, pos, turns, inverse=inverse, out=torch.empty_like(grad), **kw), y)
        assert not sj.rotary(x, pos, turns).requires_grad


def test_calls_without_a_gradient_say_so():
    """attend, and append's queries: a backward pass through them ends with an error instead of
    a gradient that lacks their part."""
    import torch
    import paper_2006_12608_amd as sj
    say("no gradient")
    c = Case(86, "bf16", 2, 3, 2, 2, 64, 16, [40, 9])
    lens = dev(c.lens)
    want, want_lse = sj.attend(c.cache, lens, c.dq)
    q = c.dq.clone().requires_grad_()
    out, lse = sj.attend(c.cache, lens, q)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    for y in (out, lse):
        with pytest.raises(RuntimeError, match="gradient"):
            y.float().sum().backward(retain_graph=True)
    with pytest.raises(ValueError, match="grad"):
        sj.attend(c.cache, lens, q, out=torch.empty_like(c.dq))
    row = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16, device="cuda")
    turned = sj.cache_append(c.cache, lens, row, row, q=q)
    assert torch.equal(turned, c.dq)
    with pytest.raises(RuntimeError, match="gradient"):
        turned.float().sum().backward()
    with pytest.raises(ValueError, match="grad"):
        sj.cache_append(c.cache, lens, row, row, q=q, q_out=torch.empty_like(c.dq))
    with pytest.raises(ValueError, match="grad"):       # no result to carry it
        sj.cache_append(c.cache, lens, row.clone().requires_grad_(), row)
    with torch.no_grad():
        sj.cache_append(c.cache, lens, row.clone().requires_grad_(), row, q=q, q_out=q)
        sj.attend(c.cache, lens, q, out=torch.empty_like(q))
    assert not sj.attend(c.cache, lens, q.detach())[0].requires_grad
    weight = torch.rand(2, 2, c.cache.room, device="cuda").requires_grad_()
    with pytest.raises(ValueError, match="grad"):
        sj.attend(c.cache, lens, c.dq, weight=weight)
    into = sj.kv_cache(torch.zeros_like(c.dk), torch.zeros_like(c.dv), c.cache.table)
    with pytest.raises(ValueError, match="grad"):
        sj.cache_evict(c.cache, lens, weight, into, keep=4)
    sj.cache_evict(c.cache, lens, weight.detach(), into, keep=4)
    own = sj.kv_cache(c.dk.clone().requires_grad_(), c.dv, c.cache.table)
    for call in (lambda: sj.cache_append(own, lens, row, row, q=c.dq),
                 lambda: sj.cache_evict(own, lens, weight.detach(), into, keep=4)):
        with pytest.raises(ValueError, match="grad"):
            call()
        with torch.no_grad():
            call()
    with pytest.raises(RuntimeError, match="gradient"):
        sj.attend(own, lens, c.dq)[0].float().sum().backward()


def wide_cache(cols):
    """A cache of one sequence with room for `cols` rows, of which one page of 1024 exists."""
    import torch
    import paper_2006_12608_amd as sj
    k = torch.zeros(1, 1024, 1, 64, dtype=torch.float16, device="cuda")
    table = torch.full((1, cols // 1024), -1, dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    return sj.kv_cache(k, k.clone(), table)


def test_scratch_that_no_graph_holds_is_freed():
    """After a capture the scratch that it holds stays; what later calls outgrow in turn is
    freed.  16 query rows keep 64 bytes of scores a column, with a quarter more allocated."""
    import gc
    import torch
    import paper_2006_12608_amd as sj
    say("scratch freed")
    c = Case(87, "f16", 1, 4, 1, 4, 64, 16, [300])
    lens, w = dev(c.lens), torch.zeros(1, 1, c.cache.room, device="cuda")
    want = sj.attend(c.cache, lens, c.dq, weight_out=torch.empty_like(w))
    sizes = [2 ** e for e in range(20, 24)]
    caches = [wide_cache(n) for n in sizes]
    weights = torch.zeros(1, 1, sizes[-1], device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    gc.collect()
    torch.cuda.empty_cache()        # (as a capture does: not to be mistaken for scratch)
    free = torch.cuda.mem_get_info()[0]
    ctx = sj.sj_create(torch.cuda.current_device(), stream.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        sj.attend(c.cache, lens, c.dq, weight_out=w, ctx=ctx)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            out, lse = sj.attend(c.cache, lens, c.dq, weight_out=w, ctx=ctx)
        for cache, n in zip(caches, sizes):
            sj.attend(cache, lens, c.dq, weight_out=weights[..., :n], ctx=ctx)
    torch.cuda.synchronize()
    used = free - torch.cuda.mem_get_info()[0]
    assert used <= 1.25 * 64 * sizes[-1] + 2 ** 27, used
    for _ in range(2):
        out.zero_()
        w.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    del graph
    sj.sj_destroy(ctx)


def test_two_threads_on_one_stream():
    """Threads of a program share their stream's context: their calls do not mix."""
    import threading
    import torch
    import paper_2006_12608_amd as sj
    say("threads")
    cases = [Case(88, "f16", 3, 2, 2, 4, 64, 16, [900, 33, 500]),
             Case(89, "bf16", 2, 40, 1, 2, 128, 16, [50, 1200])]
    rng = np.random.default_rng(3)
    P = dev(rng.integers(-3, 4, (700, 64)), "f16")
    jobs = []
    for c in cases:
        lens = dev(c.lens)

        def job(c=c, lens=lens):
            w = torch.empty(c.B, c.k.shape[2], c.cache.room, device="cuda")
            return (*sj.attend(c.cache, lens, c.dq, weight_out=w), w)
        jobs.append(job)
    jobs.append(lambda: (sj.join_ip(P, P, 150.0, two_pass=True),))
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    wrong, errors = [], []

    def work(i):
        try:
            for _ in range(60):
                got = jobs[i]()
                if not all(torch.equal(x, y) for x, y in zip(got, want[i])):
                    wrong.append(i)
        except Exception as e:      # (shown by the assertion below)
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors and not wrong, (errors, wrong)


def test_a_context_may_be_made_during_a_capture():
    """torch.cuda.graph without a stream captures on one of its own, where the first call makes
    its context.  Calls without scratch are then captured; one that needs scratch is refused,
    and the capture goes on."""
    import torch
    import paper_2006_12608_amd as sj
    say("context in a capture")
    c = Case(90, "f16", 2, 3, 2, 4, 64, 16, [300, 33])
    lens = dev(c.lens)
    pos, turns = torch.arange(6, dtype=torch.int32, device="cuda"), sj.rotary_turns(64)
    x = c.dq.view(6, 8, 64)
    want = sj.rotary(x, pos, turns)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        ctx = sj.sj_create(torch.cuda.current_device(), stream.cuda_stream)
        y = sj.rotary(x, pos, turns, ctx=ctx)
        with pytest.raises(sj.SjError, match="capture"):
            sj.attend(c.cache, lens, c.dq, ctx=ctx)
        z = y + 1
    for _ in range(3):
        y.zero_()
        z.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(z, want + 1)
    with torch.cuda.stream(stream):     # and the context serves as any other
        out = sj.attend(c.cache, lens, c.dq, ctx=ctx)[0]
    torch.cuda.synchronize()
    assert torch.equal(out, sj.attend(c.cache, lens, c.dq)[0])
    del graph
    sj.sj_destroy(ctx)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("T,group,d", [(6, 1, 64), (6, 4, 64), (6, 8, 128), (6, 12, 64), (40, 4, 64),
                                       (30, 2, 256), (70, 4, 72)])
def test_weights_of_hidden_rows_may_hold_anything(dtype, bad, T, group, d):
    """A drafted token whose key and value are not finite and that no token sees: every output
    and weight is that of the definition, and its own weight 0."""
    import torch
    import paper_2006_12608_amd as sj
    say("hidden weights", dtype, bad, T, group, d)
    c = Case(91, dtype, 1, T, 2, group, d, 16, [70])
    tree = chain_tree(c.rng, 1, T)
    tree[0, :, 0] &= np.uint64(2 ** 64 - 1 - 4)         # nobody sees token 2
    r = ref.row_of(c.table, c.page, c.k.shape[0], 0, 72)
    for x in (c.dk, c.dv):
        x[r[0], r[1]] = bad
    c.k[r], c.v[r] = 0.0, 0.0
    want, want_lse, want_w, mag, dots = ref.attend(c.k, c.v, c.table, c.lens, c.q, tree, d ** -0.5)
    w = torch.full((1, 2, c.cache.room), float("nan"), device="cuda")
    out, lse = sj.attend(c.cache, dev(c.lens), c.dq, dev(tree.view(np.int64)), weight_out=w)
    assert np.array_equal(np.isinf(want_lse), np.isinf(host(lse))) and torch.isfinite(out).all()
    w = host(w)
    assert np.isfinite(w).all() and (w[0, :, 72] == 0).all()
    rho = 4 * (d + 4) * 2.0 ** -24 * dots.max() + c.cache.room * 2.0 ** -23 + 2.0 ** -19
    tol = (rho + (T * group + 2) * 2.0 ** -24) * want_w + 1e-30
    assert (np.abs(w - want_w) <= tol).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("n,heads,d,rot", [(9000, 32, 50, 34), (4000, 9, 211, 166), (9000, 12, 135, 50),
                                           (20000, 8, 128, 100)])
def test_rotary_rounds_alike_however_it_is_called(dtype, layout, n, heads, d, rot):
    """In place, out of place and on the way into a cache, which take different loads, the same
    pairs give the same bits."""
    import torch
    import paper_2006_12608_amd as sj
    say("same bits", dtype, layout, n, heads, d, rot)
    g = torch.Generator(device="cuda").manual_seed(8)
    x = (torch.randn(n, heads, d, generator=g, device="cuda") * 3).to(tdtype(dtype))
    pos = torch.randint(-1000, 10 ** 6, (n,), generator=g, device="cuda", dtype=torch.int32)
    turns = sj.rotary_turns(rot)
    want = sj.rotary(x, pos, turns, layout=layout, factor=1.25)
    y = x.clone()
    assert torch.equal(sj.rotary(y, pos, turns, layout=layout, factor=1.25, out=y), want)
    k, v = (torch.zeros(1, n, heads, d, dtype=x.dtype, device="cuda") for _ in range(2))
    q = x[None].clone()
    sj.cache_append(sj.kv_cache(k, v), torch.zeros(1, dtype=torch.int32, device="cuda"), x[None], x[None],
                    pos=pos[None], turns=turns, q=q, q_out=q, layout=layout, factor=1.25)
    assert torch.equal(k[0], want) and torch.equal(q[0], want) and torch.equal(v[0], x)
