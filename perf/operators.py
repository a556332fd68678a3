"""Performance cases of the operators around a cache of key and value rows:
rotary positions, rows appended to the cache, attention of single tokens and
of trees of drafted tokens over it, and eviction by accumulated attention
weight.

A case is a dict of plain values.  `prepare` makes its inputs on the GPU from
a seed, `run` is one call as a program makes it: of the framework when `own`
is true, of elementary torch operations in 32 bits otherwise.  `work` is the
data and arithmetic a call cannot do without, `exact` the results from the
definitions in 64 bits.

The cache is a pool of pages of rows, k and v (pages, page, heads, d), with a
table (sequences, pages of a sequence).  Sequence b holds `lengths[b]` rows.
"""
import math

import numpy as np
import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}
DEV = "cuda"


def listed():
    return [
        # One user, one token at a time, a small head and a short history:
        # latency alone.
        dict(name="attend_one_f16_d64_n2048", kind="attend", dtype="f16", B=1, T=1, kv=2, group=4,
             d=64, page=64, lo=2048, hi=2048, tree=False, weight=False, joint=False),
        # A batch of ordinary decoding steps, histories of very different
        # lengths, pages of 16 rows with k and v side by side in each page.
        dict(name="attend_batch_bf16_d128_n200_8192", kind="attend", dtype="bf16", B=32, T=1, kv=8,
             group=4, d=128, page=16, lo=200, hi=8192, tree=False, weight=False, joint=True),
        # Speculative decoding: a tree of 16 drafted tokens for each of 16
        # users, with the weights that a later eviction goes by.
        dict(name="attend_tree16_bf16_d128_n1024_6000", kind="attend", dtype="bf16", B=16, T=16,
             kv=8, group=4, d=128, page=64, lo=1024, hi=6000, tree=True, weight=True, joint=False),
        # Two long documents, one token each: the cache's bytes alone.
        dict(name="attend_long_bf16_d128_n131072", kind="attend", dtype="bf16", B=2, T=1, kv=8,
             group=4, d=128, page=64, lo=131000, hi=131072, tree=False, weight=True, joint=False),
        # Large trees over long histories: as much arithmetic as bytes.
        dict(name="attend_tree64_f16_d128_n32768", kind="attend", dtype="f16", B=4, T=64, kv=8,
             group=4, d=128, page=64, lo=30000, hi=32768, tree=True, weight=True, joint=False),
        # Rotated queries and keys of one decoding step of 64 users, the keys
        # and values written to their pages: latency.
        dict(name="append_step_bf16_64x1", kind="append", dtype="bf16", B=64, T=1, kv=8, group=4,
             d=128, rot=128, page=16, lo=100, hi=4000, layout="half", scaling="none"),
        # The same for prompts read in chunks of 2048 tokens, half of each
        # head rotated in adjacent pairs, positions scaled for long contexts.
        dict(name="append_prompt_f16_8x2048", kind="append", dtype="f16", B=8, T=2048, kv=8,
             group=4, d=128, rot=64, page=64, lo=0, hi=5000, layout="interleaved",
             scaling="ramp"),
        # A training step's queries: positions forward.
        dict(name="rotary_bf16_16384x32x128", kind="rotary", dtype="bf16", n=16384, heads=32,
             d=128, rot=128, layout="half", scaling="none", inverse=False, reach=8192),
        # The gradient through them, in the other layout, on part of an odd
        # head at far positions.
        dict(name="rotary_grad_f16_5000x12x80", kind="rotary", dtype="f16", n=5000, heads=12,
             d=80, rot=40, layout="interleaved", scaling="linear", inverse=True, reach=1000000),
        # One user's history cut to a third, each head by its own weights.
        dict(name="evict_one_f16_d64_n3000", kind="evict", dtype="f16", B=1, kv=2, sets=2, d=64,
             page=64, lo=3000, hi=3000, keep=1024, sink=4, recent=128),
        # A serving batch at its budget, each head by its own weights; some
        # sequences are still within it.
        dict(name="evict_batch_bf16_d128_n2500_16000", kind="evict", dtype="bf16", B=16, kv=8,
             sets=8, d=128, page=16, lo=2500, hi=16000, keep=4096, sink=4, recent=512),
        # Long documents, one choice of rows for all heads.
        dict(name="evict_long_bf16_d128_n131072", kind="evict", dtype="bf16", B=2, kv=8, sets=1,
             d=128, page=64, lo=130000, hi=131072, keep=32768, sink=16, recent=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "rotary", "evict", "evict"])
    dtype = rng.choice(["f16", "bf16"])
    page = rng.choice([16, 16, 48, 64, 64, 100, 256])
    if kind == "rotary":
        heads, d = rng.randint(1, 32), 2 * _log_int(rng, 16, 128)
        n = _log_int(rng, 1, max(1, 67108864 // (heads * d)))
        return dict(kind=kind, dtype=dtype, n=n, heads=heads, d=d, rot=2 * rng.randint(1, d // 2),
                    layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "ramp"]),
                    inverse=rng.random() < 0.5, reach=_log_int(rng, 512, 1000000))
    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256])
    kv, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 7, 8])
    if kind == "append":
        B = _log_int(rng, 1, 64)
        T = _log_int(rng, 1, max(1, min(4096, 80000000 // (B * kv * (group + 2) * d))))
        lo = rng.randint(0, 3000)
        return dict(kind=kind, dtype=dtype, B=B, T=T, kv=kv, group=group, d=d,
                    rot=2 * rng.randint(1, d // 2), page=page, lo=lo,
                    hi=lo + rng.randint(0, 3000), layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "ramp"]))
    B = _log_int(rng, 1, 32)
    if kind == "evict":
        most = max(16, min(131072, 200000000 // (B * kv * d)))
        hi = _log_int(rng, 16, most)
        lo = max(1, int(hi * rng.uniform(0.2, 1.0)))
        keep = max(1, int(hi * rng.uniform(0.05, 0.6)))
        sink = rng.randint(0, min(16, keep))
        return dict(kind=kind, dtype=dtype, B=B, kv=kv, sets=rng.choice([1, kv]), d=d, page=page,
                    lo=lo, hi=hi, keep=keep, sink=sink, recent=rng.randint(0, keep - sink))
    T = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
    most = min(131072, 250000000 // (B * kv * d), 16000000000 // (B * T * kv * group * d))
    hi = _log_int(rng, 16, max(16, most))
    return dict(kind=kind, dtype=dtype, B=B, T=T, kv=kv, group=group, d=d, page=page,
                lo=max(1, int(hi * rng.uniform(0.02, 1.0))), hi=hi,
                tree=T > 1 and rng.random() < 0.75, weight=rng.random() < 0.5,
                joint=rng.random() < 0.3)


# ------------------------------------------------------------------- inputs

def _lengths(case):
    """The lengths of a case's sequences, in increasing order: lo .. hi."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    return (x * scale).to(TORCH[dtype])


def _scaling(case):
    """Long-context scaling of the rotary frequencies: none, every position
    divided by 4, or by parts (wavelengths that fit 32 times into 4096
    positions stay, those that do not fit once are divided by 8, a linear
    blend between)."""
    return {"none": {}, "linear": dict(linear=4.0),
            "ramp": dict(ramp=(8.0, 4096.0, 1.0, 32.0))}[case["scaling"]]


def _frequencies(case):
    """Radians a position of each pair, in 64 bits (numpy)."""
    rot = case["rot"]
    f = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if case["scaling"] == "linear":
        f = f / 4.0
    elif case["scaling"] == "ramp":
        s, length, low, high = 8.0, 4096.0, 1.0, 32.0
        r = length * f / (2 * np.pi)
        g = np.clip((r - low) / (high - low), 0.0, 1.0)
        f = f / s * (1 - g) + f * g
    return f


def _factor(case):
    return 0.1 * math.log(8.0) + 1.0 if case["scaling"] == "ramp" else 1.0


def _turns(case):
    """The frequencies as a program keeps them: fixed-point turns a position,
    2^-64 of a turn each, so that whole turns drop out of 64-bit products."""
    t = [int(f / (2 * math.pi) * 2.0 ** 64) for f in _frequencies(case)]
    return torch.tensor(t, dtype=torch.int64, device=DEV)


def _pool(case, g, rows, joint=False, fill=True):
    """k, v and the table of a cache with room for `rows` rows a sequence:
    pages in an order of their own.  Rows that no sequence holds are zeros."""
    B, page, kv, d = case["B"], case["page"], case["kv"], case["d"]
    width = -(-rows // page)
    pages = B * width
    dtype = TORCH[case["dtype"]]
    if joint:
        both = torch.zeros((pages, 2, page, kv, d), dtype=dtype, device=DEV)
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = (torch.zeros((pages, page, kv, d), dtype=dtype, device=DEV) for _ in range(2))
    table = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).view(B, width)
    if fill:
        for x, scale in ((k, 1.0), (v, 1.0)):
            for p in range(0, pages, 4096):
                x[p:p + 4096] = _normal(g, x[p:p + 4096].shape, case["dtype"], scale)
    return k, v, table


def _tree(case, rng):
    """Ancestor masks of random trees of drafted tokens, 64 tokens a word: bit
    s of token t's mask is set when t follows s (t itself included)."""
    B, T = case["B"], case["T"]
    W = -(-T // 64)
    words = np.zeros((B, T, W), np.uint64)
    for b in range(B):
        masks = []
        for t in range(T):
            parent = int(rng.integers(max(-1, t - 8), t)) if t else -1
            masks.append((masks[parent] if parent >= 0 else 0) | (1 << t))
            for w in range(W):
                words[b, t, w] = (masks[t] >> (64 * w)) & 0xFFFFFFFFFFFFFFFF
    return torch.from_numpy(words.view(np.int64)).to(DEV)


def _handle(st, which="k v table"):
    import paper_2006_12608_amd as sj
    k, v, table = which.split()
    return sj.kv_cache(st[k], st[v], st[table])


def prepare(case, seed):
    g, rng = _gen(seed), np.random.default_rng(seed)
    st = {"case": case}
    kind = case["kind"]
    if kind == "rotary":
        st["x"] = _normal(g, (case["n"], case["heads"], case["d"]), case["dtype"])
        st["pos"] = torch.randint(0, case["reach"], (case["n"],), generator=g, device=DEV,
                                  dtype=torch.int32)
        st["turns"] = _turns(case)
        return st
    lens = rng.permutation(_lengths(case))
    st["lengths"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    B, kv, d = case["B"], case["kv"], case["d"]
    if kind == "evict":
        rows = max(lens)
        st["k"], st["v"], st["table"] = _pool(case, g, rows)
        room = min(rows, case["keep"])
        st["k2"], st["v2"], st["table2"] = _pool(case, g, room, fill=False)
        # sums of softmax weights: a few rows hold most, a long tail next to none
        w = torch.randn((B, case["sets"], rows), generator=g, device=DEV)
        st["weight"] = torch.exp(2.0 * w) / rows
        if own:
            st["cache"], st["kept"] = _handle(st), _handle(st, "k2 v2 table2")
        return st
    T, heads = case["T"], kv * case["group"]
    if kind == "append":
        st["k"], st["v"], st["table"] = _pool(case, g, max(lens) + T, fill=False)
        # a fused projection's output: a token's queries, keys, values
        qkv = _normal(g, (B, T, heads + 2 * kv, d), case["dtype"])
        st["q"], st["key"], st["value"] = qkv.split([heads, kv, kv], 2)
        st["pos"] = (st["lengths"][:, None]
                     + torch.arange(T, dtype=torch.int32, device=DEV)).contiguous()
        st["turns"] = _turns(case)
    else:
        st["k"], st["v"], st["table"] = _pool(case, g, max(lens) + T, case["joint"])
        st["q"] = _normal(g, (B, T, heads, d), case["dtype"], 1.5)
        if case["tree"]:
            st["tree"] = _tree(case, rng)
        if case["weight"]:
            st["weight"] = torch.rand((B, kv, max(lens) + T), generator=g, device=DEV)
    if own:
        st["cache"] = _handle(st)
    return st


# ---------------------------------------------------------- framework's calls

def _run_own(st):
    import paper_2006_12608_amd as sj
    case = st["case"]
    kind = case["kind"]
    if kind == "rotary":
        return sj.rotary(st["x"], st["pos"], st["turns"], layout=case["layout"],
                         factor=_factor(case), inverse=case["inverse"])
    cache = st.get("cache") or _handle(st)
    if kind == "append":
        q = sj.cache_append(cache, st["lengths"], st["key"], st["value"], pos=st["pos"],
                            turns=st["turns"], q=st["q"], layout=case["layout"],
                            factor=_factor(case))
        return q, st["k"], st["v"]
    if kind == "evict":
        kept = st.get("kept") or _handle(st, "k2 v2 table2")
        index, lengths, weight = sj.cache_evict(cache, st["lengths"], st["weight"], kept,
                                                keep=case["keep"], sink=case["sink"],
                                                recent=case["recent"])
        return index, lengths, weight, st["k2"], st["v2"]
    if not case["weight"]:
        out, lse = sj.attend(cache, st["lengths"], st["q"], st.get("tree"))
        return out, lse
    weight = torch.empty_like(st["weight"])
    out, lse = sj.attend(cache, st["lengths"], st["q"], st.get("tree"), weight=st["weight"],
                         weight_out=weight)
    return out, lse, weight


# ------------------------------------------------------------------ plain form

def _rotate(x, pos, case, turns):
    """x (..., heads, d), pos (...): fp32 result."""
    rot = case["rot"]
    phase = (pos.to(torch.int64)[..., None] * turns) >> 32
    angle = phase.to(torch.int32).to(torch.float32) * (2 * math.pi / 2.0 ** 32)
    c = (torch.cos(angle) * _factor(case))[..., None, :]
    s = (torch.sin(angle) * _factor(case))[..., None, :]
    if case.get("inverse"):
        s = -s
    x = x.float()
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        r = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        r = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([r, x[..., rot:]], -1)


def _rows(x, table, page, rows):
    """The rows 0 .. rows - 1 of every sequence: (B, rows, heads, d)."""
    at = torch.arange(rows, device=DEV)
    return x[table[:, at // page].long(), (at % page)[None, :]]


def _run_plain(st):
    case = st["case"]
    kind, dtype = case["kind"], TORCH[case["dtype"]]
    if kind == "rotary":
        return _rotate(st["x"], st["pos"], case, st["turns"]).to(dtype)
    page, lens, table = case["page"], st["lengths"].long(), st["table"].long()
    if kind == "append":
        at = lens[:, None] + torch.arange(case["T"], device=DEV)
        p, r = table.gather(1, at // page), at % page
        st["k"][p, r] = _rotate(st["key"], st["pos"], case, st["turns"]).to(dtype)
        st["v"][p, r] = st["value"]
        return _rotate(st["q"], st["pos"], case, st["turns"]).to(dtype), st["k"], st["v"]
    if kind == "evict":
        return _evict_plain(st, case, lens, table)
    B, T, kv, group, d = (case[x] for x in ("B", "T", "kv", "group", "d"))
    n = max(_lengths(case)) + T
    k = _rows(st["k"], table, page, n).permute(0, 2, 3, 1).float()          # B kv d n
    q = st["q"].float().view(B, T, kv, group, d).permute(0, 2, 1, 3, 4)
    q = q.reshape(B, kv, T * group, d) / math.sqrt(d)
    s = torch.matmul(q, k.contiguous()).view(B, kv, T, group, n)
    at = torch.arange(n, device=DEV)
    new = at[None, None, :] - lens[:, None, None]                           # B 1 n
    t = torch.arange(T, device=DEV)[None, :, None]
    if case["tree"]:
        word = st["tree"].gather(2, (new.clamp(0, T - 1) // 64).expand(B, T, n))
        seen = ((word >> (new.clamp(0, T - 1) % 64)) & 1).bool()
        ok = (new < 0) | ((new < T) & seen)
    else:
        ok = new <= t
    s = torch.where(ok[:, None, :, None, :], s, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    p = p / total
    lse = (top + torch.log(total)).squeeze(-1)                              # B kv T group
    v = _rows(st["v"], table, page, n).permute(0, 2, 1, 3).float()          # B kv n d
    out = torch.matmul(p.view(B, kv, T * group, n), v.contiguous())
    out = out.view(B, kv, T, group, d).permute(0, 2, 1, 3, 4).reshape(B, T, kv * group, d)
    out, lse = out.to(dtype), lse.permute(0, 2, 1, 3).reshape(B, T, kv * group)
    if not case["weight"]:
        return out, lse
    return out, lse, st["weight"] + p.sum((2, 3))


def _evict_plain(st, case, lens, table):
    B, sets, keep, page = case["B"], case["sets"], case["keep"], case["page"]
    w = st["weight"]
    rows = w.shape[2]
    at = torch.arange(rows, device=DEV)
    n = lens[:, None]
    forced = (at < case["sink"]) | (at >= n - case["recent"])
    rank = torch.where(at < n, torch.where(forced, 2, 1), 0)[:, None, :].expand(B, sets, rows)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, descending=True,
                                        stable=True).indices)
    room = min(keep, rows)
    size = torch.clamp(lens, max=keep)
    held = torch.arange(room, device=DEV)[None, None, :] < size[:, None, None]
    pick = torch.where(held, order[..., :room], rows).sort(-1).values
    src = pick.clamp(max=rows - 1)
    index = torch.full((B, sets, keep), -1, dtype=torch.int32, device=DEV)
    index[..., :room] = torch.where(held, pick, -1).to(torch.int32)
    weight = torch.zeros((B, sets, keep), device=DEV)
    weight[..., :room] = torch.where(held, w.gather(-1, src), 0.0)
    kv = case["kv"]
    src, held = src.expand(B, kv, room), held.expand(B, kv, room)[..., None]
    j = torch.arange(room, device=DEV)
    head = torch.arange(kv, device=DEV)[None, :, None]
    p = table.gather(1, (src // page).flatten(1)).view(src.shape)
    p2 = st["table2"].long()[:, j // page][:, None, :].expand(B, kv, room)
    for x, y in (("k", "k2"), ("v", "v2")):
        moved = st[x][p, src % page, head]
        st[y][p2, j % page, head] = torch.where(held, moved, st[y][p2, j % page, head])
    return index, size.to(torch.int32), weight, st["k2"], st["v2"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------ work

def work(case):
    kind = case["kind"]
    if kind == "rotary":
        cells = case["n"] * case["heads"] * case["d"]
        return {"bytes": 4 * cells + 4 * case["n"],
                "flops": 3 * case["n"] * case["heads"] * case["rot"]}
    B, kv, d = case["B"], case["kv"], case["d"]
    lens = _lengths(case)
    if kind == "evict":
        kept = sum(min(n, case["keep"]) for n in lens)
        # read and written: rows of k and of v; read: weights; written: kept
        # weights and indexes
        return {"bytes": 8 * kept * kv * d + 4 * case["sets"] * (sum(lens) + 2 * kept),
                "flops": case["sets"] * sum(lens)}
    T, heads = case["T"], kv * case["group"]
    if kind == "append":
        return {"bytes": 4 * B * T * (heads + 2 * kv) * d + 4 * B * T,
                "flops": 3 * B * T * (heads + kv) * case["rot"]}
    n = sum(lens) + B * T
    size = 4 * n * kv * d + 4 * B * T * heads * d + 4 * B * T * heads
    if case["weight"]:
        size += 8 * B * kv * (max(lens) + T)
    return {"bytes": size, "flops": 4 * heads * T * n * d}


# ----------------------------------------------------------------------- exact

def _exact_rotate(x, pos, case):
    rot = case["rot"]
    f = torch.from_numpy(_frequencies(case)).to(DEV)
    angle = pos.double().unsqueeze(-1) * f
    e = torch.polar(torch.full_like(angle, _factor(case)),
                    -angle if case.get("inverse") else angle).unsqueeze(-2)
    y = x.double().clone()
    if case["layout"] == "half":
        z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * e
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.view_as_complex(y[..., :rot].unflatten(-1, (-1, 2)).contiguous()) * e
        y[..., :rot] = torch.view_as_real(z).flatten(-2)
    return y


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotary":
        return _exact_rotate(st["x"], st["pos"], case)
    page, lens = case["page"], st["lengths"].tolist()
    table = st["table"].tolist()
    B, kv = case["B"], case["kv"]

    def pages(b, n):
        return torch.tensor(table[b][:-(-n // page)], device=DEV)

    if kind == "append":
        key = _exact_rotate(st["key"], st["pos"], case)
        k, v = st["k"].double(), st["v"].double()
        for b in range(B):
            at = range(lens[b], lens[b] + case["T"])
            p = torch.tensor([table[b][i // page] for i in at], device=DEV)
            r = torch.tensor([i % page for i in at], device=DEV)
            k[p, r], v[p, r] = key[b], st["value"][b].double()
        return _exact_rotate(st["q"], st["pos"], case), k, v
    if kind == "evict":
        keep, sets = case["keep"], case["sets"]
        weight = st["weight"].cpu().numpy()
        index = np.full((B, sets, keep), -1, np.int32)
        left = np.zeros((B, sets, keep), np.float64)
        k2, v2 = st["k2"].double(), st["v2"].double()
        table2 = st["table2"].tolist()
        for b, n in enumerate(lens):
            m = min(n, keep)
            at = np.arange(n)
            forced = (at < case["sink"]) | (at >= n - case["recent"])
            for s in range(sets):
                w = weight[b, s, :n].astype(np.float64)
                order = np.lexsort((at, -w, ~forced))
                index[b, s, :m] = np.sort(order[:m])
                left[b, s, :m] = w[index[b, s, :m]]
            for h in range(kv):
                rows = torch.from_numpy(index[b, h % sets, :m].astype(np.int64)).to(DEV)
                p = torch.tensor(table[b], device=DEV)[rows // page]
                j = torch.arange(m, device=DEV)
                p2 = torch.tensor(table2[b], device=DEV)[j // page]
                for x, y in ((st["k"], k2), (st["v"], v2)):
                    y[p2, j % page, h] = x[p, rows % page, h].double()
        return (torch.from_numpy(index), torch.tensor([min(n, keep) for n in lens],
                                                      dtype=torch.int32),
                torch.from_numpy(left), k2, v2)
    T, group, d = case["T"], case["group"], case["d"]
    out = torch.empty((B, T, kv * group, d), dtype=torch.float64, device=DEV)
    lse = torch.empty((B, T, kv * group), dtype=torch.float64, device=DEV)
    weight = st["weight"].double() if case["weight"] else None
    tree = st["tree"].cpu().numpy().view(np.uint64) if case["tree"] else None
    for b, n in enumerate(lens):
        ok = torch.ones((T, n + T), dtype=torch.bool)
        for t in range(T):
            for u in range(T):
                ok[t, n + u] = bool((int(tree[b, t, u // 64]) >> (u % 64)) & 1) \
                    if tree is not None else u <= t
        ok = ok.to(DEV)
        at = pages(b, n + T)
        for h in range(kv):
            k = st["k"][at, :, h].reshape(-1, d)[:n + T].double()
            v = st["v"][at, :, h].reshape(-1, d)[:n + T].double()
            mine = slice(h * group, (h + 1) * group)
            for t0 in range(0, T, 16):
                some = slice(t0, t0 + 16)
                q = st["q"][b, some, mine].double()                          # t group d
                s = (q.reshape(-1, d) @ k.T.contiguous()).view(-1, group, n + T) / math.sqrt(d)
                s = s.masked_fill(~ok[some, None, :], -math.inf)
                a = torch.softmax(s, -1)
                out[b, some, mine] = (a.reshape(-1, n + T) @ v).view(-1, group, d)
                lse[b, some, mine] = torch.logsumexp(s, -1)
                if weight is not None:
                    weight[b, h, :n + T] += a.sum((0, 1))
    return (out, lse) if weight is None else (out, lse, weight)
