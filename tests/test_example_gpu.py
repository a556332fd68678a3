"""The example of drafted decoding: the text is the one that token by token decoding writes."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples",
                    "drafted_decoding.py")


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("drafted_decoding", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def turned(x, pos, d):
    import torch
    f = 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64) / d)
    a = pos.double()[:, None, None] * f
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)


def plain_logits(model, text):
    """The whole text at once, with no cache, in 64 bits."""
    import torch

    def unit(x):
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    n = len(text)
    x = model.embed.cpu().double()[text]
    pos = torch.arange(n)
    hidden = torch.ones(n, n).triu(1).bool()
    for i in range(model.layers):
        h = unit(x) @ model.qkv[i].cpu().double()
        q, k, v = h.split([model.q_heads * model.d, model.heads * model.d, model.heads * model.d], -1)
        q = turned(q.view(n, model.q_heads, model.d), pos, model.d)
        k = turned(k.view(n, model.heads, model.d), pos, model.d)
        v = v.view(n, model.heads, model.d)
        group = model.q_heads // model.heads
        o = []
        for j in range(model.q_heads):
            s = q[:, j] @ k[:, j // group].T * model.d ** -0.5
            o.append(s.masked_fill(hidden, -torch.inf).softmax(-1) @ v[:, j // group])
        x = x + torch.cat(o, -1) @ model.out[i].cpu().double()
    return unit(x) @ model.head.cpu().double().T


def prompts_of(lengths, vocab=512):
    import torch
    g = torch.Generator().manual_seed(5)
    return [torch.randint(vocab, (n,), generator=g).tolist() for n in lengths]


@pytest.mark.parametrize("fans", [(), (2,), (3, 2, 1, 1)])
def test_text_is_the_models_own(ex, fans):
    """Every token said is the 64-bit model's choice, up to 16-bit rounding.  A logit is a
    product over 512 elements of about unit size, so of standard deviation 22.6; the
    activations behind it pass through fewer than 32 roundings of 2^-11 each, whose errors
    add to less than 2^-6 of it at worst: two logits are ranked right when they differ by
    more than 2 * 2^-6 * 22.6 * 4 (four standard deviations) = 2.9; independent errors stay
    far below, 2 * 32^0.5 * 2^-11 * 22.6 * 4 = 0.5, which is what is asked."""
    model = ex.Model()
    prompts = prompts_of([150, 2, 65, 64])
    texts, evictions, _ = ex.decode(model, prompts, 12, 512, fans)
    assert evictions == 0
    for text, prompt in zip(texts, prompts):
        assert len(text) >= len(prompt) + 12 and text[:len(prompt)] == prompt
        logits = plain_logits(model, text)[len(prompt) - 1:-1]
        said = logits.gather(1, ex.torch.tensor(text[len(prompt):])[:, None])[:, 0]
        assert (logits.max(-1).values - said).max() <= 0.5


def test_drafts_are_accepted_and_caches_stay_bounded(ex):
    model = ex.Model()
    prompts = prompts_of([90, 40])
    texts, evictions, _ = ex.decode(model, prompts, 60, 128)
    said = sum(len(t) - len(p) for t, p in zip(texts, prompts))
    assert said > 1.2 * 60 * 2
    assert evictions >= 1
