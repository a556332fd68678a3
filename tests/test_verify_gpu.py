"""Verification of drafted tokens on the GPU against the rule's words (oracle.cache8.verify).  All
outputs are whole numbers: random numbers nearer to a border than 1e-9 are moved off it before the
first run, which double sums of at most 2^17 terms (error below 2^17 2^-53 = 1.5e-11) resolve."""
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


def tdtype(dtype):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]


def put(x, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to("cuda").to(tdtype(dtype))


def softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def check(tokens, target, uniform, draft=None, parent=None, counts=None):
    """target, draft: device tensors; the rest numpy."""
    import paper_2006_12608_amd as sj
    p = target.double().cpu().numpy()
    q = None if draft is None else draft.double().cpu().numpy()
    uniform = np.asarray(uniform, np.float32)
    # off the borders of the token that is drawn
    for _ in range(20):
        want = ref8.verify(tokens, p, uniform, q, parent, counts)
        near = [ref8.verify(tokens, p, uniform * np.float64(1 + s), q, parent, counts)[2]
                for s in (-1e-9, 1e-9)]
        off = (near[0] != want[2]) | (near[1] != want[2])
        if not off.any():
            break
        uniform[off, 0] = np.random.default_rng(1).random(off.sum()).astype(np.float32)
    else:
        raise AssertionError("no numbers away from the borders")
    got = sj.verify_drafts(dev(tokens), target, dev(uniform), draft=draft,
                           parent=None if parent is None else dev(parent.astype(np.int32)),
                           counts=None if counts is None else dev(np.asarray(counts, np.int32)))
    for name, x, y in zip(("path", "found", "next"), got, want):
        x = x.cpu().numpy()
        assert x.shape == y.shape and np.array_equal(x, y), (name, x[np.argwhere(x != y)[0][0]],
                                                             y[np.argwhere(x != y)[0][0]])
    return want


def drafted(rng, B, T, V, parent=None, chance=True, sharp=2.0):
    """Targets, drafts' distributions and tokens that are often accepted."""
    logits = sharp * rng.standard_normal((B, T, V))
    p = softmax(logits)
    q = softmax(logits + 0.5 * rng.standard_normal((B, T, V)))[:, :T - 1]
    tokens = rng.integers(0, V, (B, T))
    for b in range(B):
        for n in range(1, T):
            up = n - 1 if parent is None else int((parent if parent.ndim == 1 else parent[b])[n])
            if not 0 <= up < n:
                continue
            row = softmax(logits[b, up]) if up >= T - 1 else q[b, up]
            if chance and parent is None:
                tokens[b, n] = rng.choice(V, p=row)
            else:
                rank = sum(1 for m in range(n) if parent is not None and
                           (parent if parent.ndim == 1 else parent[b])[m] == up)
                tokens[b, n] = np.argsort(-row)[min(rank, V - 1)]
    return p, q, tokens, rng.random((B, T))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (3, 2, 5), (4, 5, 4096), (2, 7, 4097), (5, 66, 100), (2, 4, 33001),
                                   (40, 3, 777), (1, 5, 131072), (400, 2, 20000)])
def test_chains(dtype, B, T, V):
    say("chains", dtype, B, T, V)
    rng = np.random.default_rng(B + T + V)
    p, q, tokens, u = drafted(rng, B, T, V)
    counts = rng.integers(0, T + 2, B)
    target = put(p, dtype)
    check(tokens, target, u, put(q, dtype), None, None)
    check(tokens, target, u, put(q, dtype), None, counts)
    _, found, _ = check(tokens, target, u)
    assert found.min() >= 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V,own", [(3, 8, 50, False), (4, 64, 1000, True), (2, 200, 300, False),
                                       (2, 1024, 40, True), (6, 33, 20011, False)])
def test_trees(dtype, B, T, V, own):
    say("trees", dtype, B, T, V, own)
    rng = np.random.default_rng(T)
    parent = np.array([[-1] + [int(rng.integers(max(0, n - 9), n)) for n in range(1, T)]
                       for _ in range(B if own else 1)], np.int32)
    parent[..., -1] = T + 3 if T > 9 else parent[..., -1]       # never reached
    parent = parent if own else parent[0]
    p, _, tokens, u = drafted(rng, B, T, V, parent, sharp=4.0)
    tokens[:, T // 2] = tokens[:, T // 2 - 1]                   # siblings may be alike
    tokens[0, 1] = V + 7                                        # no token of the vocabulary
    tokens[0, T // 3] = -1
    _, found, _ = check(tokens, put(p, dtype), u, None, parent)
    assert found.max() > 1
    check(tokens, put(p, dtype), u, None, parent, rng.integers(0, T + 1, B))


def test_numbers_at_the_ends_and_probabilities_of_every_kind():
    """u of 0, just below 1, outside [0, 1) and NaN; NaN, infinities, negative numbers and zeros among the
    probabilities; drafts as likely as the target's; rows without any probability."""
    say("ends")
    V, T = 9, 3
    rows = [np.full(V, 1 / V), np.eye(V)[4], np.zeros(V), np.array([0, 0, .5, 0, .5, 0, 0, 0, 0]),
            np.array([np.nan, -1, np.inf, .25, -np.inf, .75, 0, np.nan, 0])]
    ends = [0.0, 1 - 2.0 ** -24, 0.3, -2.0, 7.0, np.nan]
    B = len(rows) * len(ends)
    p = np.zeros((B, T, V))
    u = np.zeros((B, T))
    for i, r in enumerate(rows):
        for j, e in enumerate(ends):
            p[i * len(ends) + j] = r
            u[i * len(ends) + j] = e, e, 0.5
    u = np.where(np.isnan(u), 0.0, u)
    tokens = np.tile(np.array([0, 4, 5]), (B, 1))
    import paper_2006_12608_amd as sj
    import torch
    for draft in (None, p[:, :T - 1].copy(), np.tile(rows[0], (B, T - 1, 1))):
        want = ref8.verify(tokens, np.float32(p), u, None if draft is None else np.float32(draft))
        got = sj.verify_drafts(dev(tokens), put(p, "f32"), dev(u.astype(np.float32)),
                               draft=None if draft is None else put(draft, "f32"))
        for x, y in zip(got, want):
            assert np.array_equal(x.cpu().numpy(), y), (x.cpu().numpy(), y)
    nan = sj.verify_drafts(dev(tokens), put(p, "f32"), torch.full((B, T), float("nan"), device="cuda"))
    zero = sj.verify_drafts(dev(tokens), put(p, "f32"), torch.zeros((B, T), device="cuda"))
    assert all(torch.equal(x, y) for x, y in zip(nan, zero))


@pytest.mark.parametrize("B,V", [(3, 9000), (400, 20000)])
def test_nothing_left_but_the_targets_own(B, V):
    """Drafts as likely as the target's, and tokens that neither gives: every one is refused, nothing is
    left of the difference, and the token is drawn from the target itself."""
    say("nothing left", B, V)
    rng = np.random.default_rng(V)
    p = softmax(rng.standard_normal((B, 2, V)))
    p[..., ::3] = 0.0
    p[:, :, :V // 2] *= rng.random((B, 2, 1)) < 0.5
    tokens = 3 * rng.integers(0, V // 3, (B, 2))
    target = put(p, "f32")
    path, found, nxt = check(tokens, target, rng.random((B, 2)), target[:, :1].contiguous())
    assert (found == 1).all() and (nxt % 3 != 0).all()
    if B > 100:     # (three sequences may all be drawn from the upper half)
        assert (nxt >= V // 2).any() and (nxt < V // 2).any()


@pytest.mark.parametrize("kind", ["chain", "certain", "tree"])
def test_the_texts_distribution_is_the_targets(kind):
    """Many sequences with the same probabilities: the first token said, drafted or drawn, is distributed
    as the target's.  The largest of 8 relative frequencies' deviations stays below five standard
    deviations of a binomial."""
    import torch
    import paper_2006_12608_amd as sj
    say("distribution", kind)
    B, V, g = 40000, 8, torch.Generator("cuda").manual_seed(5)
    rng = np.random.default_rng(2)
    p = softmax(rng.standard_normal(V))
    q = softmax(rng.standard_normal(V))
    T = {"chain": 2, "certain": 2, "tree": 4}[kind]
    target = put(np.tile(p, (1, T, 1)), "f32").expand(B, T, V)
    u = torch.rand((B, T), generator=g, device="cuda")
    tokens = torch.zeros((B, T), dtype=torch.int64, device="cuda")
    kw = {}
    if kind == "chain":
        row = torch.from_numpy(q).to("cuda")
        tokens[:, 1] = torch.multinomial(row, B, replacement=True, generator=g)
        kw["draft"] = put(np.tile(q, (1, 1, 1)), "f32").expand(B, 1, V)
    elif kind == "certain":
        tokens[:, 1] = 3
    else:
        tokens[:, 1:] = torch.tensor([5, 2, 5])
        kw["parent"] = torch.tensor([-1, 0, 0, 0], dtype=torch.int32, device="cuda")
    path, found, nxt = sj.verify_drafts(tokens, target, u, **kw)
    at = path[:, 1:2].long()
    said = torch.where(found > 1, tokens.gather(1, at.clamp(min=0))[:, 0], nxt)
    share = torch.bincount(said, minlength=V).double().cpu().numpy() / B
    assert (np.abs(share - p) < 5 * np.sqrt(p * (1 - p) / B)).all(), (share, p)
    assert 0 < (found > 1).sum() < B


def test_strides_refusals_and_graph():
    import torch
    import paper_2006_12608_amd as sj
    say("verify graph")
    rng = np.random.default_rng(7)
    B, T, V = 3, 6, 5000
    p, q, tokens, u = drafted(rng, B, T, V)
    wide = torch.full((T, B, V + 3), float("nan"), device="cuda")
    wide[:, :, 1:V + 1] = put(p, "f32").transpose(0, 1)
    target = wide[:, :, 1:V + 1].transpose(0, 1)
    check(tokens, target, u, put(q, "f32"))
    t, draft, du = dev(tokens), put(q, "f32"), put(u, "f32")
    with pytest.raises(ValueError):
        sj.verify_drafts(t.int(), target, du)
    with pytest.raises(ValueError):
        sj.verify_drafts(t, target.double(), du)
    with pytest.raises(ValueError):
        sj.verify_drafts(t, target, du, draft=draft, parent=torch.zeros(T, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        sj.verify_drafts(t, target, du, draft=draft[:, :-1])
    with pytest.raises(ValueError):
        sj.verify_drafts(t, target, du[:, 1:])
    with pytest.raises(ValueError):
        sj.verify_drafts(t, target.clone().requires_grad_(), du)
    with pytest.raises(sj.SjError):
        sj.verify_drafts(t[:, :0].contiguous(), target[:, :0], du[:, :0].contiguous())
    many = torch.zeros(1, 1025, dtype=torch.int64, device="cuda")
    with pytest.raises(sj.SjError):
        sj.verify_drafts(many, torch.zeros(1, 1025, 4, device="cuda"), many.float())
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sj.verify_drafts(t, target, du, draft=draft)
    side.synchronize()
    with torch.cuda.graph(g, stream=side):
        out = sj.verify_drafts(t, target, du, draft=draft)
    for i in range(4):
        du.uniform_()
        g.replay()
        want = sj.verify_drafts(t, target, du, draft=draft)
        assert all(torch.equal(x, y) for x, y in zip(out, want)), i
