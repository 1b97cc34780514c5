"""Cases of attention with scored masks (tanh cap, distance bias, documents, prefix) and of the normalised, rotated heads
that feed it.

Each case is what a program does with one layer:

  fwd    the output alone: generation one token at a time, prefill, an encoder's inference
  train  the output, then the gradients of the layer's inputs (and of the norms' weights) for a given upstream gradient
  hvp    those gradients with a graph, and the gradients of their product with given directions: the layer's part of a
         Hessian-vector product, with respect to the inputs, the weights and the upstream gradient

The layer is `score` or `rotary`.

`score` is attention over the scores cap tanh(s / cap) (cap 0: s itself) minus slope_h times the distance of the positions
(slopes), under one of the masks full, causal, documents (packed documents, causal inside each; `docs` of them, the last
`pad` positions belong to none) and prefix (`prefix` leading positions see each other both ways, the rest is causal;
with documents, those of each document).  It holds entry, dtype ("bf16" or "f32"), B, H, Hkv (key/value heads), Nq, Nk, d,
short (the batch's valid lengths are spread evenly from `short` to 1 times the padded length) and loud (the scores'
standard deviation).  Nq < Nk continues sequences whose keys lie in a cache of Nk rows.

`rotary` takes the queries and keys of a projection, [B, N, heads, d], to the heads of an attention, [B, heads, N, d]:
each head vector is divided by its root mean square and multiplied by a weight (norm), then the pairs of its first `rot`
dims are rotated by angles of position, pairs of (i, i + rot / 2) or (interleaved) (2 i, 2 i + 1).  `grid` names the
positions: "n" (text) for n consecutive tokens from `far` on, "hxw" or "txhxw" for the rows and columns of an image or
the frames of a video, whose axes share the pairs as `sections` says ("16,24,24").
"""
import math

import torch

own = False


def _score(name, entry, B, H, Nq, Nk, d, dtype="bf16", Hkv=None, mask="causal", cap=0.0, slopes=False, docs=1, pad=0,
           prefix=0, short=1.0, loud=3.0):
    return {"name": name, "layer": "score", "entry": entry, "dtype": dtype, "B": B, "H": H, "Hkv": Hkv or H, "Nq": Nq,
            "Nk": Nk, "d": d, "mask": mask, "cap": cap, "slopes": slopes, "docs": docs, "pad": pad, "prefix": prefix,
            "short": short, "loud": loud}


def _rotary(name, entry, B, H, grid, d, dtype="bf16", Hkv=None, norm=True, rot=None, sections=None, far=0,
            interleaved=False, base=10000.0, weights="bf16"):
    rot = rot or d
    return {"name": name, "layer": "rotary", "entry": entry, "dtype": dtype, "B": B, "H": H, "Hkv": Hkv or H,
            "grid": grid, "d": d, "norm": norm, "rot": rot, "sections": sections or str(rot // 2), "far": far,
            "interleaved": interleaved, "base": base, "weights": weights}


def listed():
    return [
        # one decoding step of a capped layer with grouped heads over ragged caches: memory bandwidth
        _score("score_token_capped", "fwd", 16, 16, 1, 4096, 128, Hkv=4, cap=50.0, short=0.3),
        # prefill of one long prompt with a distance bias a head
        _score("score_prefill_slopes", "fwd", 1, 16, 8192, 8192, 128, slopes=True),
        # a training step on packed documents with a padded tail, at the benchmark's B4 H12 N4096 shape
        _score("score_train_documents", "train", 4, 12, 4096, 4096, 64, mask="documents", docs=9, pad=100),
        # a training step of a wide capped causal layer, the largest case
        _score("score_train_capped", "train", 4, 16, 4096, 4096, 128, Hkv=8, cap=50.0),
        # verification in fp32 on odd lengths, everything at once on a prefix
        _score("score_train_f32_prefix", "train", 2, 6, 333, 333, 64, dtype="f32", mask="prefix", prefix=100, cap=20.0,
               slopes=True, short=0.6),
        # a curvature probe through a capped causal layer
        _score("score_hvp_capped", "hvp", 1, 12, 1024, 1024, 64, cap=30.0),
        # the same through packed documents with prefixes and a distance bias, ragged
        _score("score_hvp_documents", "hvp", 2, 8, 2047, 2047, 64, mask="documents", docs=7, pad=61, prefix=40,
               slopes=True),
        # heads of one new token of a serving batch at far positions: latency
        _rotary("rotary_token", "fwd", 16, 32, "1", 128, Hkv=8, far=120000, base=1000000.0),
        # a training step's heads, normalised, from a projection's output
        _rotary("rotary_train_norm", "train", 4, 16, "4096", 128, Hkv=8),
        # a curvature probe through the norms, odd length, rotation of half the dims
        _rotary("rotary_hvp_norm", "hvp", 2, 12, "2047", 64, rot=32, weights="f32"),
        # heads of a video model's inference, positions of three axes, no norm
        _rotary("rotary_video", "fwd", 2, 16, "9x30x44", 128, sections="16,24,24", norm=False),
        # a training step on images in fp32, positions of two axes, neighbours paired
        _rotary("rotary_image_train_f32", "train", 8, 6, "31x45", 64, dtype="f32", sections="16,16", interleaved=True,
                weights="f32"),
    ]


# ---------------------------------------------------------------------------
# Work
# ---------------------------------------------------------------------------
def _spread(n, B, short):
    """Valid lengths of a batch: B values spread evenly from `short` n to n."""
    return [max(1, round(n * (1 - (1 - short) * b / max(1, B - 1)))) for b in range(B)]


def _lengths(c):
    """(valid query rows, valid key rows, position of the first query) of each batch entry."""
    kl = _spread(c["Nk"], c["B"], c["short"])
    if c["Nq"] == c["Nk"]:
        return kl, kl, [0] * c["B"]
    kl = [max(n, c["Nq"]) for n in kl]
    return [c["Nq"]] * c["B"], kl, [n - c["Nq"] for n in kl]


def _document_lengths(c):
    """Lengths of an entry's documents, 1 : 2 : ... : docs of the positions that are not padding."""
    total, n = c["Nk"] - c["pad"], c["docs"]
    ends = [round(total * i * (i + 1) / (n * (n + 1))) for i in range(n + 1)]
    return [b - a for a, b in zip(ends, ends[1:])]


def _pairs(c):
    """Valid (query, key) pairs of one head over the batch."""
    def square(n, prefix):
        p = min(n, prefix)
        return n * (n + 1) // 2 + p * (p - 1) // 2

    if c["mask"] == "documents":
        return c["B"] * sum(square(n, c["prefix"]) for n in _document_lengths(c))
    total = 0
    for ql, kl, start in zip(*_lengths(c)):
        if c["mask"] == "full":
            total += ql * kl
        elif c["mask"] == "prefix":
            total += square(kl, c["prefix"])
        else:  # row i sees start + i + 1 keys
            total += ql * (start + 1) + ql * (ql - 1) // 2
    return total


def _rotary_inputs(c):
    return ["q", "k"] + (["wq", "wk"] if c["norm"] else [])


def _rotary_outputs(c):
    names = _rotary_inputs(c)
    first = [] if c["entry"] == "fwd" else ["d" + n for n in names]
    second = ["hgq", "hgk"] + ["h" + n for n in names] if c["entry"] == "hvp" else []
    return ["q", "k"] + first + second


def _tokens(c):
    return math.prod(int(x) for x in c["grid"].split("x"))


_CONTRACTIONS = {"fwd": 2, "train": 2 + 5, "hvp": 2 + 5 + 12}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["layer"] == "rotary":
        elements = case["B"] * _tokens(case) * (case["H"] + case["Hkv"]) * case["d"]
        # matrices read and written: inputs and outputs, then upstream and input gradients, then directions and the
        # second gradients of both
        return {"bytes": {"fwd": 2, "train": 4, "hvp": 7}[case["entry"]] * elements * size,
                "flops": {"fwd": 8, "train": 24, "hvp": 60}[case["entry"]] * elements}
    ql, kl, _ = _lengths(case)
    q_in, k_in = case["H"] * sum(ql), case["Hkv"] * sum(kl)                       # valid rows
    q_out, k_out = case["B"] * case["H"] * case["Nq"], case["B"] * case["Hkv"] * case["Nk"]
    # (query-side, key-side) matrices read, then written
    rq, rk, wq, wk = {"fwd": (1, 2, 1, 0), "train": (2, 2, 2, 2), "hvp": (3, 4, 4, 4)}[case["entry"]]
    return {"bytes": (rq * q_in + rk * k_in + wq * q_out + wk * k_out) * case["d"] * size,
            "flops": case["H"] * _pairs(case) * 2 * case["d"] * _CONTRACTIONS[case["entry"]]}


def _cost(c):
    """Work in units that compare the two data types (fp32 MFMA runs at 1/16 of the bf16 rate)."""
    return work(c)["flops"] * (16 if c["dtype"] == "f32" else 1)


def draw(rng):
    top = max(_cost(c) for c in listed() if c["layer"] == "score")
    top_bytes = max(work(c)["bytes"] for c in listed() if c["layer"] == "rotary")

    def log_uniform(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, n // 64 * 64) if n > 128 and rng.random() < 0.3 else n

    while True:
        layer = rng.choice(("score", "score", "score", "rotary", "rotary"))
        entry = rng.choice(("fwd", "train", "train", "hvp"))
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        G = rng.choice((1, 1, 1, 2, 4, 8))
        Hkv = rng.choice((1, 2, 4, 6, 8, 12, 16))
        c = {"layer": layer, "entry": entry, "dtype": dtype, "B": rng.choice((1, 1, 2, 4, 8, 16)), "H": Hkv * G,
             "Hkv": Hkv}
        if c["H"] > 48:
            continue
        if layer == "rotary":
            d = c["d"] = rng.choice((32, 64, 64, 128, 128, 256))
            c["rot"] = rng.choice((d, d, d // 2))
            c["norm"] = entry == "hvp" or rng.random() < 0.6
            c["interleaved"] = rng.random() < 0.3
            c["base"] = rng.choice((10000.0, 500000.0, 1000000.0))
            c["weights"] = "f32" if dtype == "f32" else rng.choice(("bf16", "f32"))
            c["far"] = rng.choice((0, 0, 1000, 300000))
            axes = rng.choice((1, 1, 2, 3))
            pairs = c["rot"] // 2
            if axes == 1:
                c["grid"], c["sections"] = str(1 if rng.random() < 0.15 else log_uniform(2, 16384)), str(pairs)
            else:
                c["far"] = 0
                first = pairs // 2 if axes == 2 else pairs // 4
                cut = (first, pairs - first) if axes == 2 else (first, (pairs - first) // 2,
                                                                pairs - first - (pairs - first) // 2)
                c["sections"] = ",".join(str(x) for x in cut)
                c["grid"] = "x".join(str(log_uniform(2, 90 if axes == 2 or i else 16)) for i in range(axes))
            if work(c)["bytes"] <= top_bytes:
                return c
            continue
        c["d"] = rng.choice((32, 64, 64, 64, 128, 128) if dtype == "f32" else (32, 64, 64, 64, 128, 128, 256))
        c["cap"] = rng.choice((0.0, 20.0, 30.0, 50.0))
        c["slopes"] = rng.random() < 0.4
        c["docs"], c["pad"], c["prefix"], c["short"] = 1, 0, 0, 1.0
        c["loud"] = rng.choice((1.0, 3.0, 6.0))
        if entry == "fwd" and rng.random() < 0.5:  # a decoding step, of one token or a few
            c["Nq"], c["Nk"], c["mask"] = rng.choice((1, 1, 1, 2, 5)), log_uniform(64, 16384), "causal"
            c["short"] = rng.choice((0.25, 0.5, 0.8, 1.0))
        else:
            c["Nq"] = c["Nk"] = n = log_uniform(32, 8192)
            c["mask"] = rng.choice(("full", "causal", "documents", "documents", "prefix"))
            if c["mask"] == "documents":
                c["docs"] = rng.choice((2, 3, 5, 9, 17))
                c["pad"] = rng.choice((0, n // 30, n // 5))
                c["prefix"] = rng.choice((0, 0, max(1, n // 30)))
            else:
                c["short"] = rng.choice((0.25, 0.5, 0.8, 1.0))
                if c["mask"] == "prefix":
                    c["prefix"] = max(1, int(n * rng.uniform(0.05, 0.7)))
        if not (c["cap"] or c["slopes"] or c["mask"] in ("documents", "prefix")):
            continue
        elements = c["B"] * c["H"] * c["Nq"] * c["Nk"]
        cache = c["B"] * c["Hkv"] * c["Nk"] * c["d"] * (4 if dtype == "f32" else 2)
        if _cost(c) <= top and elements <= 1.1e9 and cache <= 3e8:
            return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _documents(case, seed):
    """Document of every position, [B, Nk], -1 for padding: each entry's documents in another order."""
    gen = torch.Generator().manual_seed(int(seed))
    lens = torch.tensor(_document_lengths(case))
    rows = []
    for _ in range(case["B"]):
        order = torch.randperm(case["docs"], generator=gen)
        ids = torch.repeat_interleave(torch.arange(case["docs"]), lens[order])
        rows.append(torch.cat([ids, torch.full((case["pad"],), -1)]))
    return torch.stack(rows).to(torch.int32)


def _slopes(H):
    """2^(-8 (h + 1) / H): a geometric series of falling slopes."""
    return [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]


def _frequencies(case):
    """Radians a position of every pair, falling from 1 by powers of 1 / base, and the pair's axis."""
    pairs = case["rot"] // 2
    sections = [int(s) for s in case["sections"].split(",")]
    assert sum(sections) == pairs
    freq = [case["base"] ** (-i / pairs) for i in range(pairs)]
    return freq, [a for a, n in enumerate(sections) for _ in range(n)]


def _positions(case, seed):
    """[axes, B, N]: consecutive ones from a start of each entry's own, or the coordinates of a grid's cells."""
    dims = [int(x) for x in case["grid"].split("x")]
    if len(dims) == 1:
        starts = torch.randint(0, max(1, case["far"]) + 1, (case["B"], 1),
                               generator=torch.Generator().manual_seed(int(seed)))
        return (torch.arange(dims[0])[None, :] + starts * (case["far"] > 0))[None].to(torch.int32)
    cells = torch.stack([x.reshape(-1) for x in torch.meshgrid(*map(torch.arange, dims), indexing="ij")])
    return cells[:, None, :].expand(-1, case["B"], -1).contiguous().to(torch.int32)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    B, H, Hkv, d = (case[n] for n in ("B", "H", "Hkv", "d"))
    x = {}

    def randn(name, *shape, dtype=dt, mean=0.0, by=1.0):
        x[name] = (torch.randn(*shape, generator=gen, device="cuda") * by + mean).to(dtype)

    if case["layer"] == "rotary":
        N = _tokens(case)
        randn("q", B, N, H, d)
        randn("k", B, N, Hkv, d)
        wt = torch.float32 if case["weights"] == "f32" else torch.bfloat16
        if case["norm"]:
            randn("wq", d, dtype=wt, mean=1.0, by=0.2)
            randn("wk", d, dtype=wt, mean=1.0, by=0.2)
        if case["entry"] != "fwd":
            randn("gq", B, H, N, d)
            randn("gk", B, Hkv, N, d)
        if case["entry"] == "hvp":
            randn("uq", B, N, H, d)
            randn("uk", B, N, Hkv, d)
            randn("uwq", d, dtype=wt)
            randn("uwk", d, dtype=wt)
        freq, axes = _frequencies(case)
        x["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        x["axes"] = torch.tensor(axes, dtype=torch.int32, device="cuda")
        x["positions"] = _positions(case, seed).cuda()
        return x

    for n in ("q", "k", "v", "dO", "uq", "uk", "uv"):
        if case["entry"] == "fwd" and n not in ("q", "k", "v") or case["entry"] == "train" and n.startswith("u"):
            continue
        keys = n in ("k", "v", "uk", "uv")
        randn(n, B, Hkv if keys else H, case["Nk"] if keys else case["Nq"], d, by=case["loud"] if n == "q" else 1.0)
    order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed)))
    for n, values in zip(("q_lens", "kv_lens", "q_starts"), _lengths(case)):
        x[n] = torch.tensor(values, dtype=torch.int32)[order].cuda()
    if case["slopes"]:
        x["slopes"] = torch.tensor(_slopes(H), dtype=torch.float32, device="cuda")
    if case["mask"] == "documents":
        x["documents"] = _documents(case, seed).cuda()
    if case["prefix"]:
        x["prefix_lens"] = torch.full((B,), case["prefix"], dtype=torch.int32, device="cuda")
    return x


def prepare(case, seed):
    st = {"case": dict(case), **_inputs(case, seed)}
    if case["layer"] == "score":
        leaves = ("q", "k", "v") + (("dO",) if case["entry"] == "hvp" else ())
        # a batch whose sequences are all whole passes no lengths
        if case["short"] == 1.0:
            st["q_lens"] = st["kv_lens"] = None
        elif case["Nq"] < case["Nk"]:
            st["q_lens"] = None
        if case["Nq"] == case["Nk"]:
            st["q_starts"] = None
        st["spans"] = None
        if own and case["mask"] in ("documents", "prefix"):  # once a batch, for every layer of a model
            import paper_2609_24089_amd as fb
            st["spans"] = fb.attention_spans(case["B"], case["Nk"], documents=st.get("documents"),
                                             prefix_lens=st.get("prefix_lens"), device="cuda")
    else:
        leaves = ("q", "k", "wq", "wk") + (("gq", "gk") if case["entry"] == "hvp" else ())
    if case["entry"] != "fwd":
        for n in leaves:
            if n in st:
                st[n].requires_grad_(True)
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(st):
    if own:
        return _own_rotary(st) if st["case"]["layer"] == "rotary" else _own_score(st)
    with torch.no_grad():
        return _plain_rotary(st) if st["case"]["layer"] == "rotary" else _plain_score(st)


def _own_score(st):
    import paper_2609_24089_amd as fb
    c = st["case"]

    def layer():
        return fb.scored_attention(st["q"], st["k"], st["v"], causal=c["mask"] == "causal", cap=c["cap"] or None,
                                   slopes=st.get("slopes"), spans=st["spans"], kv_lens=st["kv_lens"],
                                   q_lens=st["q_lens"], q_starts=st["q_starts"])

    if c["entry"] == "fwd":
        with torch.no_grad():
            return {"O": layer()}
    leaves = [st[n] for n in ("q", "k", "v")]
    O = layer()
    if c["entry"] == "train":
        return {"O": O.detach(), **dict(zip(("dq", "dk", "dv"), torch.autograd.grad(O, leaves, st["dO"])))}
    g = torch.autograd.grad(O, leaves, st["dO"], create_graph=True)
    h = torch.autograd.grad(g, [st["dO"], *leaves], [st[n] for n in ("uq", "uk", "uv")])
    return {"O": O.detach(), **{n: t.detach() for n, t in zip(("dq", "dk", "dv"), g)},
            **dict(zip(("hO", "hq", "hk", "hv"), h))}


def _own_rotary(st):
    import paper_2609_24089_amd as fb
    c = st["case"]

    def layer():
        return fb.rotate_heads(st["q"].transpose(1, 2), st["k"].transpose(1, 2), st["positions"],
                               (st["freq"], st["axes"]), q_weight=st.get("wq"), k_weight=st.get("wk"),
                               interleaved=c["interleaved"])

    if c["entry"] == "fwd":
        with torch.no_grad():
            return dict(zip(("q", "k"), layer()))
    names = _rotary_inputs(c)
    leaves, up = [st[n] for n in names], [st["gq"], st["gk"]]
    y = layer()
    g = torch.autograd.grad(y, leaves, up, create_graph=c["entry"] == "hvp")
    h = torch.autograd.grad(g, up + leaves, [st["u" + n] for n in names]) if c["entry"] == "hvp" else ()
    return dict(zip(_rotary_outputs(c), [t.detach() for t in (*y, *g, *h)]))


def _valid(st, c, B, Nq, Nk, dev):
    """Which pairs count, [B, Nq, Nk], or None for all; and the rows' positions."""
    keys = torch.arange(Nk, device=dev)
    rows = torch.arange(Nq, device=dev)[None, :] + (0 if st["q_starts"] is None else st["q_starts"][:, None])
    rows = rows.expand(B, Nq)
    valid = None
    if c["short"] < 1 or c["mask"] != "full":
        valid = torch.ones(B, Nq, Nk, dtype=torch.bool, device=dev)
    if st["kv_lens"] is not None:
        valid &= keys < st["kv_lens"][:, None, None]
    if st["q_lens"] is not None:
        valid &= torch.arange(Nq, device=dev)[:, None] < st["q_lens"][:, None, None]
    if c["mask"] == "full":
        return valid, rows
    seen = keys <= rows[:, :, None]
    if c["mask"] == "documents":
        ids = st["documents"]
        valid &= (ids[:, :, None] == ids[:, None, :]) & (ids >= 0)[:, :, None]
        if c["prefix"]:  # a key's place in its document
            first = (ids[:, 1:] != ids[:, :-1]).nonzero()
            place = torch.zeros_like(ids, dtype=torch.long)
            place[first[:, 0], first[:, 1] + 1] = first[:, 1] + 1
            place = keys - place.cummax(1).values
            seen = seen | (place < st["prefix_lens"][:, None])[:, None, :]
    elif c["mask"] == "prefix":
        seen = seen | (keys < st["prefix_lens"][:, None])[:, None, :]
    valid &= seen
    return valid, rows


def _plain_score(st):
    c = st["case"]
    B, H, Hkv, Nq, Nk = (c[n] for n in ("B", "H", "Hkv", "Nq", "Nk"))
    G, dev, tau = H // Hkv, st["q"].device, c["d"] ** -0.5
    f = {n: st[n].detach().float() for n in ("q", "k", "v", "dO", "uq", "uk", "uv") if n in st}
    for n in ("k", "v", "uk", "uv"):
        if n in f:
            f[n] = f[n].repeat_interleave(G, 1) if G > 1 else f[n]
    mm = lambda a, b: torch.matmul(a, b.transpose(-1, -2).contiguous())  # noqa: E731
    tm = lambda a, b: torch.matmul(a.transpose(-1, -2).contiguous(), b)  # noqa: E731
    group = lambda x: x.reshape(B, Hkv, G, Nk, -1).sum(2)  # noqa: E731
    qt, kt = st["q"].dtype, st["k"].dtype

    valid, rows = _valid(st, c, B, Nq, Nk, dev)
    S = mm(f["q"] * tau, f["k"])
    t = None
    if c["cap"]:
        t = torch.tanh(S / c["cap"])
        S = c["cap"] * t
    if c["slopes"]:
        far = (torch.arange(Nk, device=dev) - rows[:, :, None]).abs().float()
        S = S - st["slopes"][None, :, None, None] * far[:, None]
    if valid is not None:
        S = S.masked_fill(~valid[:, None], -math.inf)
    top = S.amax(-1, keepdim=True)
    P = (S - torch.where(top == -math.inf, 0.0, top)).exp()
    total = P.sum(-1, keepdim=True)
    P = P / torch.where(total == 0, 1.0, total)
    out = {"O": torch.matmul(P, f["v"]).to(qt)}
    if c["entry"] == "fwd":
        return out

    dP = mm(f["dO"], f["v"])
    D = (P * dP).sum(-1, keepdim=True)
    dZ = P * (dP - D)                               # by the capped scores
    slope = 1 - t * t if t is not None else 1.0     # of the cap
    dS = dZ * slope
    out["dq"] = (tau * torch.matmul(dS, f["k"])).to(qt)
    out["dk"] = (tau * group(tm(dS, f["q"]))).to(kt)
    out["dv"] = group(tm(P, f["dO"])).to(kt)
    if c["entry"] == "train":
        return out

    Fs = tau * (mm(f["uq"], f["k"]) + mm(f["q"], f["uk"]))
    F = Fs * slope
    alpha = (P * F).sum(-1, keepdim=True)
    Pt = mm(f["dO"], f["uv"]) + F * (dP - D) - alpha * dP
    E = (P * Pt).sum(-1, keepdim=True)
    St = P * (Pt - E) * slope
    if t is not None:
        St = St - dZ * Fs * (2 / c["cap"]) * t * slope
    Ph = P * (F - alpha)
    out["hO"] = (torch.matmul(P, f["uv"]) + torch.matmul(Ph, f["v"])).to(qt)
    out["hq"] = (tau * (torch.matmul(St, f["k"]) + torch.matmul(dS, f["uk"]))).to(qt)
    out["hk"] = (tau * group(tm(St, f["q"]) + tm(dS, f["uq"]))).to(kt)
    out["hv"] = group(tm(Ph, f["dO"])).to(kt)
    return out


_EPS = 1e-6


def _plain_rotary(st):
    c = st["case"]
    rot, d = c["rot"], c["d"]
    angle = st["positions"].double()[st["axes"].long()] * st["freq"][:, None, None]  # [pairs, B, N]
    cos, sin = (f(angle).permute(1, 2, 0)[:, :, None].float() for f in (torch.cos, torch.sin))
    if c["interleaved"]:
        a, b = slice(0, rot, 2), slice(1, rot, 2)
    else:
        a, b = slice(0, rot // 2), slice(rot // 2, rot)

    def turn(x, sine):
        y = x.clone()
        y[..., a] = x[..., a] * cos - x[..., b] * sine
        y[..., b] = x[..., a] * sine + x[..., b] * cos
        return y

    out = {}
    for n in ("q", "k"):
        x, dt = st[n].detach().float(), st[n].dtype
        wt = st.get("w" + n)
        w = wt.detach().float() if wt is not None else None
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) if w is not None else None
        y = x * r * w if w is not None else x
        out[n] = turn(y, sin).transpose(1, 2).to(dt).contiguous()
        if c["entry"] == "fwd":
            continue
        g = turn(st["g" + n].detach().float().transpose(1, 2), -sin)
        if w is None:
            out["d" + n] = g.to(dt)
            continue
        aw = g * w
        ax = (aw * x).sum(-1, keepdim=True) / d
        out["d" + n] = (r * aw - r ** 3 * ax * x).to(dt)
        out["dw" + n] = (g * x * r).sum((0, 1, 2), dtype=torch.float64).to(wt.dtype)
        if c["entry"] == "train":
            continue
        u, uw = st["u" + n].float(), st["uw" + n].float()
        ux = (u * x).sum(-1, keepdim=True) / d
        both = ((aw * u).sum(-1, keepdim=True) + (uw * g * x).sum(-1, keepdim=True)) / d
        out["h" + n] = (r * uw * g - r ** 3 * (both * x + aw * ux + u * ax) + 3 * r ** 5 * ax * ux * x).to(dt)
        out["hw" + n] = (r * g * u - r ** 3 * ux * g * x).sum((0, 1, 2), dtype=torch.float64).to(wt.dtype)
        out["hg" + n] = turn(r * w * u - r ** 3 * ux * w * x + r * uw * x, sin).transpose(1, 2).to(dt).contiguous()
    return {n: out[n] for n in _rotary_outputs(c)}


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    return _exact_rotary(case, seed) if case["layer"] == "rotary" else _exact_score(case, seed)


def _exact_rotary(case, seed):
    """Complex multiplication of the pairs; the derivatives by torch's automatic differentiation, once and twice."""
    x = {n: t.double() if t.is_floating_point() else t for n, t in _inputs(case, seed).items()}
    entry, rot = case["entry"], case["rot"]
    steps = x["positions"].double().permute(1, 2, 0)[:, :, x["axes"].long()] * x["freq"]   # [B, N, pairs]
    turn = torch.polar(torch.ones_like(steps), steps)[:, :, None]
    out = {}
    for n in ("q", "k"):
        leaves = [x[n].clone().requires_grad_(entry != "fwd")]
        if case["norm"]:
            leaves.append(x["w" + n].clone().requires_grad_(entry != "fwd"))
        y = leaves[0]
        if case["norm"]:
            y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + _EPS) * leaves[1]
        pairs = y[..., :rot]
        pairs = (pairs.unflatten(-1, (rot // 2, 2)) if case["interleaved"]
                 else pairs.unflatten(-1, (2, rot // 2)).transpose(-1, -2))
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        pairs = pairs.flatten(-2) if case["interleaved"] else pairs.transpose(-1, -2).flatten(-2)
        y = torch.cat([pairs, y[..., rot:]], -1).transpose(1, 2)
        out[n] = y.detach().contiguous()
        if entry == "fwd":
            continue
        names = [n, "w" + n][:len(leaves)]
        up = x["g" + n].clone().requires_grad_(True)
        g = torch.autograd.grad(y, leaves, up, create_graph=entry == "hvp")
        out.update({"d" + m: t.detach() for m, t in zip(names, g)})
        if entry == "hvp":
            h = torch.autograd.grad(g, [up] + leaves, [x["u" + m] for m in names])
            out.update(dict(zip(["hg" + n] + ["h" + m for m in names], h)))
    return {n: out[n] for n in _rotary_outputs(case)}


def _exact_score(case, seed):
    """A batch entry, a document and a key/value head at a time on its valid rows alone: the output by its definition,
    the derivatives by torch's automatic differentiation of it, once and twice."""
    x = {n: t.double() if t.is_floating_point() else t for n, t in _inputs(case, seed).items()}
    entry, G = case["entry"], case["H"] // case["Hkv"]
    names = {"fwd": ("O",), "train": ("O", "dq", "dk", "dv"),
             "hvp": ("O", "dq", "dk", "dv", "hO", "hq", "hk", "hv")}[entry]
    r = {n: torch.zeros_like(x["q" if n[-1] in "Oq" else n[-1]]) for n in names}
    ql, kl, start = (x[n].tolist() for n in ("q_lens", "kv_lens", "q_starts"))
    for b in range(case["B"]):
        # (rows, keys) of what sees each other
        blocks = [(slice(0, ql[b]), slice(0, kl[b]))]
        if case["mask"] == "documents":
            ids, counts = torch.unique_consecutive(x["documents"][b], return_counts=True)
            ends = counts.cumsum(0).tolist()
            blocks = [(slice(e - n, e),) * 2 for i, n, e in zip(ids.tolist(), counts.tolist(), ends) if i >= 0]
        for rs, ks in blocks:
            if rs.stop == rs.start:
                continue
            pos = torch.arange(rs.start, rs.stop, device="cuda") + start[b]
            key = torch.arange(ks.start, ks.stop, device="cuda")
            gap = key[None, :] - pos[:, None]
            hidden = None
            if case["mask"] != "full":
                hidden = gap > 0
                if case["prefix"]:
                    hidden &= key[None, :] >= ks.start + case["prefix"]
            for hk in range(case["Hkv"]):
                h = slice(hk * G, hk * G + G)
                diff = [t.clone().requires_grad_(entry != "fwd") for t in
                        (x["q"][b, h, rs], x["k"][b, hk, ks], x["v"][b, hk, ks])]
                dO = x["dO"][b, h, rs].clone().requires_grad_(True) if entry != "fwd" else None
                with torch.set_grad_enabled(entry != "fwd"):
                    S = torch.matmul(diff[0], diff[1].t()) * case["d"] ** -0.5
                    if case["cap"]:
                        S = torch.tanh(S / case["cap"]) * case["cap"]
                    if case["slopes"]:
                        S = S - x["slopes"][h][:, None, None] * gap.abs()
                    if hidden is not None:
                        S = S.masked_fill(hidden, -math.inf)
                    O = torch.matmul(torch.softmax(S, -1), diff[2])
                r["O"][b, h, rs] = O.detach()
                if entry == "fwd":
                    continue
                g = torch.autograd.grad(O, diff, dO, create_graph=entry == "hvp")

                def put(names, values):
                    for n, t in zip(names, values):
                        if n[1] in "kv":
                            r[n][b, hk, ks] = t.detach()
                        else:
                            r[n][b, h, rs] = t.detach()

                put(("dq", "dk", "dv"), g)
                if entry == "hvp":
                    u = [x["uq"][b, h, rs], x["uk"][b, hk, ks], x["uv"][b, hk, ks]]
                    put(("hO", "hq", "hk", "hv"), torch.autograd.grad(g, [dO, *diff], u))
    return r
