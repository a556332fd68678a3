"""Caches in 8 bits, pages and drafted tokens without a GPU: refusals of the C entries and the
oracle's own definitions by hand."""
import numpy as np
import pytest

from oracle import cache8 as ref


def test_null_context_is_rejected():
    import paper_2006_12608_amd as sj
    no = (0, 0, 0)
    assert sj.sj_cache8_append(None, None, None, None, 0, None, no, None, no, None, None, 0, 0,
                               1.0) == sj.SJ_E_INVAL
    assert "context" in sj.sj_last_error()
    assert sj.sj_attend8(None, None, None, None, 0, None, no, 1, None, (0, 0), 1.0, None,
                         None) == sj.SJ_E_INVAL
    assert sj.sj_cache_pages(None, None, 0, 0, 0, 0, 1, None, None, 0, 0, None, None, None,
                             None) == sj.SJ_E_INVAL
    assert sj.sj_cache_copy(None, None, None, 0) == sj.SJ_E_INVAL
    assert sj.sj_cache8_copy(None, None, None, 0) == sj.SJ_E_INVAL
    assert sj.sj_verify(None, sj.SJ_F32, 0, 1, 1, None, None, 0, None, None, (0, 0), None, (0, 0),
                        None, None, None, None) == sj.SJ_E_INVAL


def test_host_tensors_are_refused():
    import torch
    import paper_2006_12608_amd as sj
    x = torch.zeros(2, 16, 1, 8, dtype=torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        sj.kv_cache8(x, x, torch.zeros(2, 1, 1, 2, dtype=torch.int8))
    with pytest.raises(ValueError):
        sj.kv_cache8(x, x, torch.zeros(2, 1, 1, 2, dtype=torch.int8), dtype=torch.float32)
    i = torch.zeros(2, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        sj.cache_pages(i, i[0], 1, pages=4, page=16)
    with pytest.raises(ValueError):
        sj.verify_drafts(torch.zeros(1, 2, dtype=torch.int64), torch.zeros(1, 2, 4),
                         torch.zeros(1, 2))


def test_e4m3_is_the_types():
    """All 256 bytes as torch reads them, and rounding of numbers around every value and tie."""
    import torch
    b = np.arange(256, dtype=np.uint8)
    t = torch.from_numpy(b).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.e4m3(b), t, equal_nan=True)
    f = ref.e4m3(b[:127])
    x = np.concatenate([f, (f[1:] + f[:-1]) / 2, (f[1:] + f[:-1]) / 2 * (1 + 2.0 ** -20), [500.0, 1e30]])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(np.clip(x, -448, 448)).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.e4m3(ref.to_e4m3(x)), want)
    assert np.isnan(ref.e4m3(ref.to_e4m3([np.nan, np.inf, -np.inf]))).all()


def test_exponents_by_hand():
    assert ref.exponent([448.0], "f16") == 0 and ref.exponent([448.5], "f16") == 1
    assert ref.exponent([0.0], "f16") == -15 and ref.exponent([65504.0], "f16") == 7
    assert ref.exponent([1.75, -np.inf, np.nan], "bf16") == -8
    assert ref.exponent([1e-40], "bf16") == -117 and ref.exponent([3e38], "bf16") == 119


def test_pages_by_hand():
    """Two children of a sequence of 5 rows in pages of 2, one of another, whose pages are free."""
    table = np.array([[7, 3, 5, -1], [0, 1, -1, -1]], np.int32)
    out, n, copies, lacking = ref.pages(table, [5, 3], 2, 9, 2, np.array([0, 0]))
    assert out.tolist() == [[7, 3, 5, 0], [7, 3, 1, 2]] and n.tolist() == [5, 5]
    assert copies.tolist() == [[-1, -1, 0], [5, 1, 1]] and lacking.tolist() == [0, 0]
    out, _, _, lacking = ref.pages(table, [5, 3], 3, 9, 2)
    assert out.tolist() == [[7, 3, 5, 2], [0, 1, 4, -1]] and lacking.tolist() == [0, 0]
    _, _, copies, lacking = ref.pages(table, [5, 3], 4, 4, 2, np.array([1, 1, -1]))
    assert (copies == [-1, -1, 0]).all() and lacking.tolist() == [0, 3, 2]


def test_verify_by_hand():
    p = np.array([[[0.5, 0.25, 0.25], [0.1, 0.8, 0.1], [0.0, 0.0, 1.0]]])
    q = np.array([[[0.25, 0.75, 0.0], [0.2, 0.2, 0.6]]])
    tok = np.array([[9, 1, 2]])
    # token 1 passes with probability 1/3, token 2 after it with 1/6
    got = ref.verify(tok, p, np.array([[0.99, 0.3, 0.1]]), q)
    assert [x.tolist() for x in got] == [[[0, 1, 2]], [3], [2]]
    # refused at once: what is left is (.25, 0, .25)
    got = ref.verify(tok, p, np.array([[0.49, 0.34, 0.1]]), q)
    assert [x.tolist() for x in got] == [[[0, -1, -1]], [1], [0]]
    assert ref.verify(tok, p, np.array([[0.5, 0.34, 0.1]]), q)[2].tolist() == [2]
    # two siblings chosen without chance: 1 passes below .25, then 0 below .5 / .75
    up = np.array([-1, 0, 0])
    tok = np.array([[9, 1, 0]])
    assert ref.verify(tok, p, np.array([[0.5, 0.26, 0.66]]), None, up)[0].tolist() == [[0, 2, -1]]
    got = ref.verify(tok, p, np.array([[0.5, 0.26, 0.67]]), None, up)
    assert [x.tolist() for x in got] == [[[0, -1, -1]], [1], [2]]


def test_the_rule_keeps_the_targets_distribution():
    """By summing over all drafts and integrating over u(1): for a chain of one token, what the text goes on
    with has the target's probabilities."""
    rng = np.random.default_rng(0)
    p, q = rng.random(5), rng.random(5)
    p, q = p / p.sum(), q / q.sum()
    pass_ = np.minimum(1.0, p / q)
    rest = np.maximum(p - q, 0)
    got = q * pass_ + (q * (1 - pass_)).sum() * rest / rest.sum()
    assert np.allclose(got, p)


def test_a_call_that_appends_nothing_changes_nothing():
    """Sequence 0 ends inside a block and appends no row: its bytes and exponents, the least ones of
    int8 among them, stay, also where sequence 1 appends to the same page."""
    rng = np.random.default_rng(1)
    k8, v8 = (rng.integers(0, 126, (2, 4, 1, 8)).astype(np.uint8) for _ in "kv")
    ex = np.full((2, 1, 1, 2), -120, np.int8)
    before = [x.copy() for x in (k8, v8, ex)]
    rows = rng.standard_normal((1, 2, 1, 8))
    for count in (0, -1):
        ref.append(k8, v8, ex, lambda b, n: (0, n), [3], rows, rows, 4, "bf16", [count])
        assert all(np.array_equal(x, y) for x, y in zip((k8, v8, ex), before))
    alone = [x.copy() for x in before]
    rows = np.concatenate([rows * 0, rows * 512])
    ref.append(*alone, lambda b, n: (0, n), [2], rows[1:], rows[1:], 4, "bf16")
    ref.append(k8, v8, ex, lambda b, n: (0, n), [3, 2], rows, rows, 4, "bf16", [0, 2])
    assert all(np.array_equal(x, y) for x, y in zip((k8, v8, ex), alone)) and ex[0, 0, 0, 0] > -10
