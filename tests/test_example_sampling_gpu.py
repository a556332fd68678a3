"""The example of drafted decoding with sampled text, caches in 8 bits and shared prompts: it runs, a
temperature near 0 says what the model finds likeliest, and forks of a prompt go on from it alone."""
import pytest

from test_example_gpu import ex, plain_logits, prompts_of     # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fans", [(2,), (3, 2, 1, 1)])
def test_cold_samples_are_the_models_choice(ex, fans):      # noqa: F811
    """At temperature 2^-10 a token whose logit is 0.02 below the best has probability below e^-20: the
    bound is that of the greedy text."""
    model = ex.Model()
    prompts = prompts_of([150, 2, 65])
    texts, _, _ = ex.decode(model, prompts, 10, 512, fans, temperature=2.0 ** -10)
    for text, prompt in zip(texts, prompts):
        assert len(text) >= len(prompt) + 10 and text[:len(prompt)] == prompt
        logits = plain_logits(model, text)[len(prompt) - 1:-1]
        said = logits.gather(1, ex.torch.tensor(text[len(prompt):])[:, None])[:, 0]
        assert (logits.max(-1).values - said).max() <= 0.5 + 0.02


@pytest.mark.parametrize("temperature", [0.0, 20.0])
def test_caches_in_8_bits_and_shared_prompts(ex, temperature):      # noqa: F811
    model = ex.Model()
    prompts = prompts_of([70, 33])
    ex.torch.manual_seed(1)
    texts, evictions, _ = ex.decode(model, prompts, 12, 512, temperature=temperature, bits=8, samples=3)
    assert evictions == 0 and len(texts) == 6
    for i, text in enumerate(texts):
        prompt = prompts[i // 3]
        assert text[:len(prompt)] == prompt and len(text) >= len(prompt) + 12
    if temperature == 0.0:      # nothing but their pages tells the forks apart
        assert texts[0] == texts[1] == texts[2] and texts[3] == texts[4] == texts[5]
    else:
        assert texts[0] != texts[1]


def test_pages_come_back(ex):       # noqa: F811
    """Sequences that end give their pages back; a pool too small says how many are lacking."""
    model = ex.Model()
    pool = ex.Pool(model, 3, 64, 7)
    pool.reserve(32)
    assert not pool.lacking.any() and (pool.table >= 0).sum() == 6
    pool.lengths += 20
    pool.reserve(44, ex.torch.tensor([1], dtype=ex.torch.int32, device="cuda"))
    assert pool.table.shape == (1, 4) and not pool.lacking.any() and (pool.table >= 0).all()
    pool.lengths += 20
    pool.reserve(24, ex.torch.tensor([0, 0, 0], dtype=ex.torch.int32, device="cuda"))
    assert pool.lacking.tolist() == [0, 0, 1]
