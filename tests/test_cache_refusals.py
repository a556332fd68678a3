"""The calls on caches without a GPU: NULL contexts are refused, and the
frequencies of rotary positions are those of the definition."""
import numpy as np

from oracle import cache as ref


def test_null_context_is_rejected():
    import paper_2006_12608_amd as sj
    assert sj.sj_rotary(None, sj.SJ_F16, None, (0, 0), None, (0, 0), 0, 0, 0, None, None, 0, 0,
                        1.0) == sj.SJ_E_INVAL
    assert "context" in sj.sj_last_error()
    assert sj.sj_cache_append(None, None, None, None, 0, None, (0, 0, 0), None, (0, 0, 0), None,
                              None, 0, 0, 1.0) == sj.SJ_E_INVAL
    assert sj.sj_attend(None, None, None, None, 0, None, (0, 0, 0), 1, None, (0, 0), 1.0, None,
                        None) == sj.SJ_E_INVAL
    assert sj.sj_cache_evict(None, None, None, None, 1, 0, 0, 0, 0, None, None,
                             None) == sj.SJ_E_INVAL


def test_turns_are_the_frequencies():
    import paper_2006_12608_amd as sj
    for rot, kw in ((128, {}), (40, {"linear": 4.0}), (64, {"ramp": (8.0, 4096.0, 1.0, 32.0)}),
                    (2, {}), (0, {})):
        t = sj.rotary_turns(rot, 10000.0, device="cpu", **kw).numpy().view(np.uint64)
        want = ref.frequencies(rot, 10000.0, **kw) / (2 * np.pi) if rot else np.zeros(0)
        assert t.shape == (rot // 2,)
        assert np.allclose(t.astype(np.float64) / 2.0 ** 64, want, rtol=1e-14, atol=0)


def test_oracle_rotary_keeps_lengths_and_turns_back():
    rng = np.random.default_rng(1)
    x, pos, f = rng.standard_normal((5, 3, 10)), rng.integers(0, 1000, 5), ref.frequencies(8)
    for layout in ("half", "interleaved"):
        y = ref.rotary(x, pos, f, layout, 2.0)
        assert np.allclose((y[..., :8] ** 2).sum(-1), 4 * (x[..., :8] ** 2).sum(-1))
        assert np.allclose(ref.rotary(y, pos, f, layout, 0.5, inverse=True)[..., :8], x[..., :8])
        assert np.array_equal(y[..., 8:], x[..., 8:])


def test_oracle_eviction_by_hand():
    w = np.array([5.0, 1.0, 3.0, 3.0, np.nan, 9.0, 0.0])
    assert list(ref.evict(w, 7, 4, 1, 1)) == [0, 2, 5, 6]
    assert list(ref.evict(w, 7, 5, 0, 0)) == [0, 1, 2, 3, 5]
    assert list(ref.evict(w, 3, 4, 1, 1)) == [0, 1, 2]


def test_oracle_attention_by_hand():
    """Two rows with scores 0 and log 3, the second one hidden from token 0."""
    k = np.array([0.0, np.log(3.0)]).reshape(1, 2, 1, 1)
    v = np.array([1.0, 5.0]).reshape(1, 2, 1, 1)
    q = np.ones((1, 2, 1, 1))
    out, lse, w, _, _ = ref.attend(k, v, None, [0], q, None, 1.0)
    assert np.allclose(out.ravel(), [1.0, 4.0]) and np.allclose(lse.ravel(), [0.0, np.log(4.0)])
    assert np.allclose(w.ravel(), [1.25, 0.75])
