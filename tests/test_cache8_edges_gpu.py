"""Caches in 8 bits, copies and verification on the GPU where a call takes more workgroups than one
launch, and attention over long heads by more query rows than its kernels hold at once."""
import numpy as np
import pytest

from test_cache8_gpu import Case8
from test_cache_gpu import chain_tree, check_attend, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2006_12608_amd  # noqa: F401  (fails loudly when libsj.so is missing)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape", [(1, 80, 2, 2, 256, 16, [100]), (2, 140, 1, 1, 200, 16, [77, 0]),
                                   (1, 50, 2, 6, 136, 64, [300])], ids=lambda s: "x".join(map(str, s[:6])))
@pytest.mark.parametrize("mask", ["chain", "tree"])
def test_attend8_long_heads_many_query_rows(dtype, shape, mask):
    B, T, heads, group, d, page, lens = shape
    say("attend8 long heads", dtype, shape[:6], mask)
    c = Case8(B + T + d, dtype, B, T, heads, group, d, page, lens, 8)
    tree = chain_tree(c.rng, B, T) if mask == "tree" else None
    check_attend(c, tree, c.rng.random((B, heads, c.cache.room + 5)).astype(np.float32))


def test_append8_of_more_blocks_than_a_launch_takes():
    """2^22 + 300 blocks of one row: the same bytes as in calls of 2^20 rows."""
    import torch
    import paper_2006_12608_amd as sj
    say("append8 launches")
    n = 2 ** 22 + 300
    torch.manual_seed(1)
    x = (torch.randn(1, n, 1, 8, device="cuda") * torch.exp2(torch.randint(-20, 20, (1, n, 1, 1),
                                                                           device="cuda"))).bfloat16()
    pools = []
    for step in (n, 2 ** 20):
        k, v = (torch.zeros(1, n, 1, 8, dtype=torch.uint8, device="cuda") for _ in "kv")
        ex = torch.zeros(1, n, 1, 2, dtype=torch.int8, device="cuda")
        cache = sj.kv_cache8(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), ex)
        for at in range(0, n, step):
            lens = torch.tensor([at], dtype=torch.int32, device="cuda")
            key = x[:, at:at + step]
            sj.cache_append(cache, lens, key, key.flip(3))
        pools.append((k, v, ex))
    assert all(torch.equal(a, b) for a, b in zip(*pools))
    k, _, ex = pools[0]
    held = k.view(torch.float8_e4m3fn).float() * torch.exp2(ex[..., :1].float())
    assert ((held - x.float()).abs() <= 2.0 ** -4 * x.float().abs() + torch.exp2(ex[..., :1].float() - 10)).all()


def test_copies_of_more_entries_than_a_launch_takes():
    import torch
    import paper_2006_12608_amd as sj
    say("copy launches")
    n = 2 ** 22 + 7
    k = torch.randn(9, 4, 1, 8, device="cuda").half()
    v = torch.randn(9, 4, 1, 8, device="cuda").half()
    copies = torch.full((n, 3), -1, dtype=torch.int32, device="cuda")
    copies[0] = torch.tensor([0, 1, 4])
    copies[n // 2] = torch.tensor([2, 3, 1])
    copies[n - 1] = torch.tensor([4, 5, 3])
    want = [x.clone() for x in (k, v)]
    for x in want:
        x[1], x[3, :1], x[5, :3] = x[0], x[2, :1], x[4, :3]
    sj.cache_copy(sj.kv_cache(k, v), copies)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("batch,vocab", [(2 ** 20 + 3, 36000), (1, 2 ** 26 + 5)])
def test_verification_of_more_parts_than_a_launch_takes(batch, vocab):
    """And of a vocabulary with more parts than a workgroup has threads.  Probabilities are multiples of
    2^-40, so that their sums are exact in any order."""
    import torch
    import paper_2006_12608_amd as sj
    say("verify launches", batch, vocab)
    torch.manual_seed(2)
    whole = torch.randint(0, 2 ** 13, (vocab,), device="cuda")
    p = (whole.double() * 2.0 ** -40).float().view(1, 1, vocab).expand(batch, 1, vocab)
    units = torch.randint(0, 2 ** 14, (batch,), device="cuda")
    units[0] = 2 ** 14 - 1
    u = (units.float() * 2.0 ** -14).view(batch, 1)
    tokens = torch.zeros(batch, 1, dtype=torch.int64, device="cuda")
    path, found, following = sj.verify_drafts(tokens, p, u)
    assert (path == 0).all() and (found == 1).all()
    # sum_{y <= x} > u sum, in whole numbers (products below 2^53: exact in double too)
    sums = whole.cumsum(0)
    limit = torch.div(units * sums[-1], 2 ** 14, rounding_mode="floor")
    assert torch.equal(following, torch.searchsorted(sums, limit, right=True))
