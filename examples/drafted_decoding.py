"""Decoding with drafted tokens over a bounded cache of key and value rows.

A small attention model with random weights continues a batch of ragged prompts.  Each step
drafts a tree of likely tokens below the last one, appends their keys (turned by rotary
positions) and values to the paged caches, lets every drafted token attend to the cache and
to its own ancestors, and keeps the path that the model itself would have taken: so several
tokens a step, and the same text as one token at a time.  The softmax weight that each cache
row draws is accumulated, and where a cache is full its heaviest rows move to other pages.

    python examples/drafted_decoding.py [--steps 32] [--batch 4] [--budget 512]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2006_12608_amd as sj                                        # noqa: E402

PAGE = 16


class Tree:
    """The shape of a draft: node 0 is the last token of the text, every node of level i has
    fans[i] children."""

    def __init__(self, fans, device):
        parent, rank, depth, level = [-1], [0], [0], [0]
        for fan in fans:
            below = []
            for p in level:
                for r in range(fan):
                    below.append(len(parent))
                    parent.append(p)
                    rank.append(r)
                    depth.append(depth[p] + 1)
            level = below
        self.size = len(parent)
        if self.size > 64:
            raise ValueError("this example keeps a tree's mask in one word a token")
        self.parent, self.rank = parent, rank
        self.children = [[c for c in range(self.size) if parent[c] == n] for n in range(self.size)]
        sees = []                       # bit w of sees[n]: n sees token w, itself and its ancestors
        for n in range(self.size):
            sees.append((sees[parent[n]] if n else 0) | 1 << n)
        sees = [s - 2 ** 64 if s >= 2 ** 63 else s for s in sees]
        self.mask = torch.tensor(sees, device=device).view(1, self.size, 1)
        self.depth = torch.tensor(depth, dtype=torch.int32, device=device)


class Model:
    """Layers of attention between residuals, with random weights."""

    def __init__(self, vocab=512, layers=2, q_heads=8, heads=2, d=64, dtype=torch.float16, seed=1):
        g = torch.Generator("cuda").manual_seed(seed)
        width = q_heads * d

        def rand(*shape, std=1.0):
            return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)
        self.q_heads, self.heads, self.d, self.layers = q_heads, heads, d, layers
        self.embed = rand(vocab, width)
        self.head = rand(vocab, width)
        self.qkv = [rand(width, (q_heads + 2 * heads) * d, std=width ** -0.5) for _ in range(layers)]
        self.out = [rand(width, width, std=0.5 * width ** -0.5) for _ in range(layers)]
        self.turns = sj.rotary_turns(d)
        # the draft: what would follow a token if attention added nothing
        self.follow = (norm(self.embed) @ self.head.T).topk(8).indices

    def project(self, layer, x):
        q, k, v = (norm(x) @ self.qkv[layer]).split(
            [self.q_heads * self.d, self.heads * self.d, self.heads * self.d], dim=-1)
        return (q.unflatten(-1, (self.q_heads, self.d)), k.unflatten(-1, (self.heads, self.d)),
                v.unflatten(-1, (self.heads, self.d)))


def norm(x):
    f = x.float()
    return (f * torch.rsqrt((f * f).mean(-1, keepdim=True) + 1e-6)).to(x.dtype)


class Caches:
    """Per layer: two sets of pages, of which one is in use, and the rows' weights."""

    def __init__(self, model, batch, room, seed=2):
        g = torch.Generator("cuda").manual_seed(seed)
        width = -(-room // PAGE)
        pages = batch * width
        shape = (pages, PAGE, model.heads, model.d)

        def cache():
            table = torch.randperm(pages, generator=g, device="cuda").int().view(batch, width)
            rows = [torch.empty(shape, dtype=model.embed.dtype, device="cuda") for _ in "kv"]
            return sj.kv_cache(*rows, table)
        self.used = [cache() for _ in range(model.layers)]
        self.spare = [cache() for _ in range(model.layers)]
        self.room = width * PAGE
        self.weight = [torch.zeros(batch, model.heads, self.room, device="cuda")
                       for _ in range(model.layers)]
        self.lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def evict(self, keep, sink, recent):
        for i, w in enumerate(self.weight):
            kept = torch.empty_like(w)
            _, lengths, self.weight[i] = sj.cache_evict(
                self.used[i], self.lengths, w, self.spare[i], keep=keep, sink=sink, recent=recent,
                weight_out=kept)
        self.used, self.spare = self.spare, self.used
        self.lengths = lengths


def forward(model, caches, tokens, pos, counts=None, tree=None):
    """Logits of a block of tokens.  Without a tree the block becomes part of the text and adds
    to the rows' weights; with one, returns also its keys, values and weights per layer."""
    x = model.embed[tokens]
    drafted = []
    for i in range(model.layers):
        q, k, v = model.project(i, x)
        q = sj.cache_append(caches.used[i], caches.lengths, k, v, pos=pos, turns=model.turns, q=q,
                            counts=counts)
        if tree is None:
            o, _ = sj.attend(caches.used[i], caches.lengths, q, counts=counts,
                             weight=caches.weight[i])
        else:
            w = torch.empty_like(caches.weight[i])
            o, _ = sj.attend(caches.used[i], caches.lengths, q, tree.mask, weight_out=w)
            drafted.append((k, v, w))
        x = x + o.flatten(2) @ model.out[i]
    return norm(x) @ model.head.T, drafted


def read_prompts(model, caches, prompts, chunk=64):
    """The prompts' tokens but the last of each, in blocks."""
    sizes = [len(p) - 1 for p in prompts]
    for at in range(0, max(sizes), chunk):
        counts = [min(max(n - at, 0), chunk) for n in sizes]
        block = [(p[at:at + c] + [0] * chunk)[:chunk] for p, c in zip(prompts, counts)]
        pos = torch.arange(at, at + chunk, dtype=torch.int32, device="cuda").expand(len(sizes), -1)
        counts = torch.tensor(counts, dtype=torch.int32, device="cuda")
        forward(model, caches, torch.tensor(block, device="cuda"), pos.contiguous(), counts)
        caches.lengths = caches.lengths + counts


def step(model, caches, tree, last, pos):
    """One draft and its verification: the tokens accepted, per sequence.  last and pos: the
    text's last tokens, not yet in the cache, and their positions."""
    drafts = [last]
    for n in range(1, tree.size):
        drafts.append(model.follow[drafts[tree.parent[n]], tree.rank[n]])
    tokens = torch.stack(drafts, 1)
    where = (pos[:, None] + tree.depth).int()
    logits, drafted = forward(model, caches, tokens, where, tree=tree)
    best = logits.argmax(-1)
    paths, said = [], []
    for tok, nxt in zip(tokens.tolist(), best.tolist()):
        path, n = [0], 0
        while n is not None:
            text = nxt[n]
            n = next((c for c in tree.children[n] if tok[c] == text), None)
            if n is not None:
                path.append(n)
        paths.append(path)
        said.append([tok[n] for n in path[1:]] + [text])
    # the accepted rows close up at the front of the drafted ones
    longest = max(map(len, paths))
    counts = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    path = torch.tensor([p + [0] * (longest - len(p)) for p in paths], device="cuda")
    rows = path[:, :, None, None]
    own = caches.lengths[:, None].long()
    columns = torch.arange(caches.room, device="cuda")
    for i, (k, v, w) in enumerate(drafted):
        shape = (-1, -1, model.heads, model.d)
        sj.cache_append(caches.used[i], caches.lengths, k.gather(1, rows.expand(shape)),
                        v.gather(1, rows.expand(shape)), pos=where.gather(1, path),
                        turns=model.turns, counts=counts)
        old = caches.weight[i]
        accepted = w.gather(2, (own + path)[:, None].expand(-1, model.heads, -1))
        accepted *= torch.arange(longest, device="cuda") < counts[:, None, None]
        new = torch.where(columns < own[:, None], old + w, 0.)
        slots = (own + torch.arange(longest, device="cuda"))[:, None].expand_as(accepted)
        caches.weight[i] = new.scatter(2, slots, accepted)
    caches.lengths = caches.lengths + counts
    return said


def decode(model, prompts, steps, budget, fans=(3, 2, 1, 1), sink=4):
    """Continues the prompts: (texts, evictions, seconds of the steps)."""
    tree = Tree(fans, "cuda")
    chunk = 64
    room = max(budget, max(map(len, prompts)) + chunk) + tree.size
    caches = Caches(model, len(prompts), room)
    read_prompts(model, caches, prompts, chunk)
    texts = [list(p) for p in prompts]
    evictions, upper = 0, max(map(len, prompts)) - 1
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(steps):
        if upper + tree.size > caches.room:
            caches.evict(budget // 2, sink, recent=budget // 8)
            evictions += 1
            upper = budget // 2
        last = torch.tensor([t[-1] for t in texts], device="cuda")
        pos = torch.tensor([len(t) - 1 for t in texts], device="cuda")
        said = step(model, caches, tree, last, pos)
        for t, s in zip(texts, said):
            t += s
        upper += max(map(len, said))
    torch.cuda.synchronize()
    return texts, evictions, time.perf_counter() - begin


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300, help="tokens of the longest prompt")
    ap.add_argument("--budget", type=int, default=512, help="cache rows of a sequence")
    args = ap.parse_args(argv)
    model = Model()
    g = torch.Generator().manual_seed(3)
    vocab = model.embed.shape[0]
    prompts = [torch.randint(vocab, (max(args.prompt - 37 * b, 2),), generator=g).tolist()
               for b in range(args.batch)]
    decode(model, prompts, 2, args.budget)          # loads the libraries
    texts, evictions, seconds = decode(model, prompts, args.steps, args.budget)
    said = sum(len(t) - len(p) for t, p in zip(texts, prompts))
    print(f"{said} tokens in {args.steps} steps of {args.batch} sequences, "
          f"{said / (args.steps * args.batch):.2f} a step and sequence, {evictions} evictions, "
          f"{1e3 * seconds / args.steps:.2f} ms a step")


if __name__ == "__main__":
    main()
