"""Cases of attention between sequences of two lengths and of attention with a learned relative position bias.

Each case is what a program does with one layer:

  fwd    the output alone: generation one token at a time, prefill, an encoder's inference
  train  the output, then the gradients of q, k, v (and of the bias table) for a given upstream gradient
  hvp    those gradients with a graph, and the gradients of their product with given directions: the layer's part of a
         Hessian-vector product, with respect to q, k, v, the upstream gradient (and the bias table)

The layer is `cross` (queries attend to another sequence, padded to a common length) or `bias` (self-attention with a
bias that depends on the bucket of the key's position minus the query's).  A case holds: layer, entry, dtype ("bf16" or
"f32"), B, H, Hkv (key/value heads), Nq, Nk, d, short (the batch's valid lengths are spread evenly from `short` to 1
times the padded length), and for `bias` causal, buckets, far (the distance from which all keys share a bucket) and
table ("f32" or "bf16").  A `bias` case with Nq < Nk continues sequences whose keys lie in a cache of Nk rows.
"""
import math

import torch

own = False


def _cross(name, entry, B, H, Nq, Nk, d, dtype="bf16", Hkv=None, short=1.0):
    return {"name": name, "layer": "cross", "entry": entry, "dtype": dtype, "B": B, "H": H, "Hkv": Hkv or H, "Nq": Nq,
            "Nk": Nk, "d": d, "short": short}


def _bias(name, entry, B, H, Nq, Nk, d, dtype="bf16", Hkv=None, short=1.0, causal=False, buckets=32, far=128,
          table="f32"):
    return {"name": name, "layer": "bias", "entry": entry, "dtype": dtype, "B": B, "H": H, "Hkv": Hkv or H, "Nq": Nq,
            "Nk": Nk, "d": d, "short": short, "causal": causal, "buckets": buckets, "far": far, "table": table}


def listed():
    return [
        # one decoding step of a small model over a ragged batch of encoder states: latency
        _cross("cross_token", "fwd", 4, 12, 1, 1500, 64, short=0.3),
        # one decoding step of a serving batch with grouped heads over long contexts: memory bandwidth
        _cross("cross_token_grouped_batch", "fwd", 32, 32, 1, 4096, 128, Hkv=8, short=0.5),
        # a decoder's inference on whole targets against padded encoder states
        _cross("cross_forward_padded", "fwd", 8, 16, 512, 2048, 64, short=0.5),
        # a training step of a wide decoder layer, the largest case
        _cross("cross_train", "train", 4, 16, 2048, 4096, 128, short=0.75),
        # verification in fp32, odd lengths on both sides
        _cross("cross_train_f32_odd", "train", 2, 6, 333, 777, 64, dtype="f32", short=0.6),
        # a curvature probe through a decoder layer, ragged
        _cross("cross_hvp_ragged", "hvp", 2, 8, 1000, 2047, 64, short=0.7),
        # one decoding step with the bias over ragged caches
        _bias("bias_token_cache", "fwd", 16, 16, 1, 4096, 64, short=0.25, causal=True),
        # prefill of one long prompt
        _bias("bias_prefill", "fwd", 1, 16, 8192, 8192, 128, causal=True),
        # a training step of a bidirectional encoder on a padded batch
        _bias("bias_train_padded", "train", 8, 12, 512, 512, 64, short=0.4),
        # a training step of a causal layer at the benchmark's B4 H12 N4096 shape, the table in bf16
        _bias("bias_train_causal", "train", 4, 12, 4096, 4096, 64, causal=True, table="bf16"),
        # a Hessian-vector product through a 12-head causal layer
        _bias("bias_hvp_causal", "hvp", 1, 12, 1024, 1024, 64, causal=True),
        # the same in fp32 on a short odd sequence with narrow heads: verification, latency
        _bias("bias_hvp_f32_short", "hvp", 1, 4, 201, 201, 32, dtype="f32", buckets=16, far=40),
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
    if c["layer"] == "cross":
        ql = _spread(c["Nq"], c["B"], c["short"]) if c["Nq"] > 1 else [1] * c["B"]
        return ql[::-1], kl, [0] * c["B"]
    if c["Nq"] == c["Nk"]:
        return kl, kl, [0] * c["B"]
    kl = [max(n, c["Nq"]) for n in kl]
    return [c["Nq"]] * c["B"], kl, [n - c["Nq"] for n in kl]


def _pairs(c):
    """Valid (query, key) pairs of one head over the batch."""
    total = 0
    for ql, kl, start in zip(*_lengths(c)):
        # row i of a causal layer sees min(kl, start + i + 1) keys
        whole = max(0, min(ql, kl - start - 1)) if c.get("causal") else 0
        total += whole * (start + 1) + whole * (whole - 1) // 2 + (ql - whole) * kl
    return total


_CONTRACTIONS = {"fwd": 2, "train": 2 + 5, "hvp": 2 + 5 + 12}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
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
    top = max(_cost(c) for c in listed())

    def log_uniform(lo, hi):
        n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        return max(lo, n // 64 * 64) if n > 128 and rng.random() < 0.3 else n

    while True:
        layer = rng.choice(("cross", "bias"))
        entry = rng.choice(("fwd", "train", "train", "hvp"))
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        d = rng.choice((32, 64, 64, 64, 128, 128) if dtype == "f32" else (32, 64, 64, 64, 128, 128, 256))
        G = rng.choice((1, 1, 1, 2, 4, 8))
        Hkv = rng.choice((1, 2, 4, 6, 8, 12, 16))
        c = {"layer": layer, "entry": entry, "dtype": dtype, "B": rng.choice((1, 1, 2, 4, 8, 16)), "H": Hkv * G,
             "Hkv": Hkv, "d": d, "short": rng.choice((0.25, 0.5, 0.8, 1.0))}
        if entry == "fwd" and rng.random() < 0.5:  # a decoding step, of one token or a few
            c["Nq"], c["Nk"] = rng.choice((1, 1, 1, 2, 5)), log_uniform(64, 16384)
        elif layer == "cross":
            c["Nq"], c["Nk"] = log_uniform(32, 4096), log_uniform(32, 8192)
        else:
            c["Nq"] = c["Nk"] = log_uniform(32, 8192)
        if layer == "bias":
            c["causal"] = c["Nq"] < c["Nk"] or rng.random() < 0.5
            c["buckets"], c["far"] = rng.choice(((32, 128), (32, 128), (16, 40), (64, 500)))
            c["table"] = rng.choice(("f32", "bf16"))
        elements = c["B"] * c["H"] * c["Nq"] * c["Nk"]
        cache = c["B"] * c["Hkv"] * c["Nk"] * d * (4 if dtype == "f32" else 2)
        if c["H"] <= 48 and _cost(c) <= top and elements <= 1.1e9 and cache <= 3e8:
            return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _bucket_map(buckets, far, bidirectional):
    """Bucket of every key position minus query position from -far to far.  Short distances have a bucket each, longer
    ones share buckets whose borders grow by a constant factor up to `far`; keys after the query have the upper half of
    the buckets (bidirectional) or the bucket of distance 0.  Distance n > half lies in bucket half + k for the largest
    k with (n / half)^(m) >= (far / half)^k, m = per_side - half, in whole numbers."""
    per_side = buckets // 2 if bidirectional else buckets
    half = per_side // 2
    m = per_side - half
    side = []
    for n in range(far + 1):
        c = n
        if n >= half:
            c = half
            while c + 1 < per_side and n ** m * half ** (c + 1 - half) >= far ** (c + 1 - half) * half ** m:
                c += 1
        side.append(c)
    after = [per_side + c for c in side] if bidirectional else [side[0]] * (far + 1)
    return side[:0:-1] + [side[0]] + after[1:]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    x = {}
    for n in ("q", "k", "v", "dO", "uq", "uk", "uv"):
        if case["entry"] == "fwd" and n not in ("q", "k", "v") or case["entry"] == "train" and n.startswith("u"):
            continue
        keys = n in ("k", "v", "uk", "uv")
        shape = (case["B"], case["Hkv"] if keys else case["H"], case["Nk"] if keys else case["Nq"], case["d"])
        x[n] = torch.randn(shape, generator=gen, device="cuda").to(dt)
    order = torch.randperm(case["B"], generator=torch.Generator().manual_seed(int(seed)))
    for n, values in zip(("q_lens", "kv_lens", "q_starts"), _lengths(case)):
        x[n] = torch.tensor(values, dtype=torch.int32)[order].cuda()
    if case["layer"] == "bias":
        tt = torch.float32 if case["table"] == "f32" else torch.bfloat16
        x["table"] = torch.randn(case["buckets"], case["H"], generator=gen, device="cuda").to(tt)
        if case["entry"] == "hvp":
            x["ut"] = torch.randn(case["buckets"], case["H"], generator=gen, device="cuda").to(tt)
        x["buckets"] = torch.tensor(_bucket_map(case["buckets"], case["far"], not case["causal"]), dtype=torch.int32,
                                    device="cuda")
    return x


def prepare(case, seed):
    st = {"case": dict(case), "scale": case["d"] ** -0.5, **_inputs(case, seed)}
    if case["entry"] != "fwd":
        for n in ("q", "k", "v", "table") + (("dO",) if case["entry"] == "hvp" else ()):
            if n in st:
                st[n].requires_grad_(True)
    # a batch whose sequences are all whole passes no lengths
    if case["short"] == 1.0:
        st["q_lens"] = st["kv_lens"] = None
    elif case["Nq"] == 1:
        st["q_lens"] = None
    if case["Nq"] == case["Nk"] or case["layer"] == "cross":
        st["q_starts"] = None
    return st


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2609_24089_amd as fb
    c = st["case"]

    def layer():
        if c["layer"] == "cross":
            return fb.cross_attention(st["q"], st["k"], st["v"], st["scale"], kv_lens=st["kv_lens"],
                                      q_lens=st["q_lens"])
        return fb.biased_attention(st["q"], st["k"], st["v"], st["table"], st["buckets"], st["scale"],
                                   causal=c["causal"], kv_lens=st["kv_lens"], q_lens=st["q_lens"],
                                   q_starts=st["q_starts"])

    if c["entry"] == "fwd":
        with torch.no_grad():
            return {"O": layer()}
    leaves = [st[n] for n in ("q", "k", "v", "table") if n in st]
    O = layer()
    if c["entry"] == "train":
        g = torch.autograd.grad(O, leaves, st["dO"])
        return {"O": O.detach(), **dict(zip(("dq", "dk", "dv", "dt"), g))}
    g = torch.autograd.grad(O, leaves, st["dO"], create_graph=True)
    u = [st[n] for n in ("uq", "uk", "uv", "ut") if n in st]
    h = torch.autograd.grad(g, [st["dO"], *leaves], u)
    return {"O": O.detach(), **{n: t.detach() for n, t in zip(("dq", "dk", "dv", "dt"), g)},
            **dict(zip(("hO", "hq", "hk", "hv", "ht"), h))}


def _by_bucket(x, st, rows, keys):
    """Sum x [B, H, Nq, Nk] over the pairs of each bucket: [buckets, H] in 64 bits."""
    B, H, Nq, Nk = x.shape
    # row i of the flipped rows, padded by Nq and read again one column shorter, is shifted right by i
    skew = torch.nn.functional.pad(x.flip(2), (0, Nq)).reshape(B, H, Nq * (Nk + Nq))[:, :, :Nq * (Nk + Nq - 1)]
    diag = skew.reshape(B, H, Nq, Nk + Nq - 1).sum(2, dtype=torch.float64)  # by key row - query row + Nq - 1
    far = (st["buckets"].numel() - 1) // 2
    step = torch.arange(Nk + Nq - 1, device=x.device) - (Nq - 1) - rows[:, :1]
    bucket = st["buckets"][(step.clamp(-far, far) + far).long()]
    one = (bucket[:, :, None] == torch.arange(st["table"].shape[0], device=x.device)).double()
    return torch.matmul(diag, one).sum(0).t()


def _run_plain(st):
    with torch.no_grad():
        c, tau = st["case"], st["scale"]
        B, H, Hkv, Nq, Nk = (c[n] for n in ("B", "H", "Hkv", "Nq", "Nk"))
        G, dev = H // Hkv, st["q"].device
        f = {n: t.detach().float() for n, t in st.items() if torch.is_tensor(t) and t.is_floating_point()}
        for n in ("k", "v", "uk", "uv"):
            if n in f:
                f[n] = f[n].repeat_interleave(G, 1) if G > 1 else f[n]
        mm = lambda a, b: torch.matmul(a, b.transpose(-1, -2).contiguous())  # noqa: E731
        tm = lambda a, b: torch.matmul(a.transpose(-1, -2).contiguous(), b)  # noqa: E731
        group = lambda x: x.reshape(B, Hkv, G, Nk, -1).sum(2)  # noqa: E731

        keys = torch.arange(Nk, device=dev)
        rows = torch.arange(Nq, device=dev)[None, :] + (0 if st["q_starts"] is None else st["q_starts"][:, None])
        valid = torch.ones(B, Nq, Nk, dtype=torch.bool, device=dev) if c["short"] < 1 or c.get("causal") else None
        if st["kv_lens"] is not None:
            valid &= keys < st["kv_lens"][:, None, None]
        if st["q_lens"] is not None:
            valid &= torch.arange(Nq, device=dev)[:, None] < st["q_lens"][:, None, None]
        if c.get("causal"):
            valid &= keys <= rows[:, :, None]

        S = mm(f["q"] * tau, f["k"])
        if c["layer"] == "bias":
            rows = rows.expand(1 if st["q_starts"] is None else B, Nq)
            step = (keys - rows[:, :, None]).clamp(-c["far"], c["far"]) + c["far"]
            bucket = st["buckets"][step]
            S += f["table"][bucket].permute(0, 3, 1, 2)
        if valid is not None:
            S.masked_fill_(~valid[:, None], -math.inf)
        top = S.amax(-1, keepdim=True)
        P = S.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = P.sum(-1, keepdim=True)
        P /= torch.where(total == 0, 1.0, total)
        O = torch.matmul(P, f["v"])
        out = {"O": O.to(st["q"].dtype)}
        if c["entry"] == "fwd":
            return out

        dP = mm(f["dO"], f["v"])
        D = (P * dP).sum(-1, keepdim=True)
        dS = P * (dP - D)
        out["dq"] = (tau * torch.matmul(dS, f["k"])).to(st["q"].dtype)
        out["dk"] = (tau * group(tm(dS, f["q"]))).to(st["k"].dtype)
        out["dv"] = group(tm(P, f["dO"])).to(st["v"].dtype)
        if c["layer"] == "bias":
            out["dt"] = _by_bucket(dS, st, rows, keys).to(st["table"].dtype)
        if c["entry"] == "train":
            return out

        F = tau * (mm(f["uq"], f["k"]) + mm(f["q"], f["uk"]))
        if c["layer"] == "bias":
            F += f["ut"][bucket].permute(0, 3, 1, 2)
        alpha = (P * F).sum(-1, keepdim=True)
        Pt = mm(f["dO"], f["uv"]) + F * (dP - D) - alpha * dP
        E = (P * Pt).sum(-1, keepdim=True)
        St = P * (Pt - E)
        Ph = P * (F - alpha)
        out["hO"] = (torch.matmul(P, f["uv"]) + torch.matmul(Ph, f["v"])).to(st["q"].dtype)
        out["hq"] = (tau * (torch.matmul(St, f["k"]) + torch.matmul(dS, f["uk"]))).to(st["q"].dtype)
        out["hk"] = (tau * group(tm(St, f["q"]) + tm(dS, f["uq"]))).to(st["k"].dtype)
        out["hv"] = group(tm(Ph, f["dO"])).to(st["v"].dtype)
        if c["layer"] == "bias":
            out["ht"] = _by_bucket(St, st, rows, keys).to(st["table"].dtype)
        return out


# ---------------------------------------------------------------------------
# The definition in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    """A batch entry and a key/value head at a time on its valid rows alone: the output by its definition, the
    derivatives by torch's automatic differentiation of it, once and twice."""
    x = {n: t.double() if t.is_floating_point() else t for n, t in _inputs(case, seed).items()}
    entry, G = case["entry"], case["H"] // case["Hkv"]
    biased, causal = case["layer"] == "bias", case.get("causal", False)
    names = {"fwd": ("O",), "train": ("O", "dq", "dk", "dv", "dt"),
             "hvp": ("O", "dq", "dk", "dv", "dt", "hO", "hq", "hk", "hv", "ht")}[entry]
    like = {"O": "q", "hO": "q"}
    r = {n: torch.zeros_like(x[like.get(n) or {"q": "q", "k": "k", "v": "v", "t": "table"}[n[1]]]) for n in names
         if biased or not n.endswith("t")}
    ql, kl, start = (x[n].tolist() for n in ("q_lens", "kv_lens", "q_starts"))
    for b in range(case["B"]):
        pos = torch.arange(ql[b], device="cuda") + start[b]
        key = torch.arange(kl[b], device="cuda")
        gap = key[None, :] - pos[:, None]
        for hk in range(case["Hkv"]):
            h = slice(hk * G, hk * G + G)
            q, k, v = x["q"][b, h, :ql[b]], x["k"][b, hk, :kl[b]], x["v"][b, hk, :kl[b]]
            leaves = [q, k, v]
            if biased:
                leaves.append(x["table"][:, h])
            diff = [t.clone().requires_grad_(entry != "fwd") for t in leaves]
            dO = x["dO"][b, h, :ql[b]].clone().requires_grad_(True) if entry != "fwd" else None
            with torch.set_grad_enabled(entry != "fwd"):
                S = torch.matmul(diff[0], diff[1].t()) * case["d"] ** -0.5
                if biased:
                    R = case["far"]
                    # the bias of each step of position first, then that of every pair
                    by_step = torch.nn.functional.embedding(x["buckets"].long(), diff[3])
                    S = S + by_step.t()[:, gap.clamp(-R, R) + R]
                if causal:
                    S = S.masked_fill(gap > 0, -math.inf)
                O = torch.matmul(torch.softmax(S, -1), diff[2])
            r["O"][b, h, :ql[b]] = O.detach()
            if entry == "fwd":
                continue
            g = torch.autograd.grad(O, diff, dO, create_graph=entry == "hvp")

            def put(names, values):
                for n, t in zip(names, values):
                    if n == "dt" or n == "ht":
                        r[n][:, h] += t.detach()
                    elif n[1] in "kv":
                        r[n][b, hk, :kl[b]] = t.detach()
                    else:
                        r[n][b, h, :ql[b]] = t.detach()

            put(("dq", "dk", "dv", "dt"), g)
            if entry == "hvp":
                u = [x["uq"][b, h, :ql[b]], x["uk"][b, hk, :kl[b]], x["uv"][b, hk, :kl[b]]]
                if biased:
                    u.append(x["ut"][:, h])
                put(("hO", "hq", "hk", "hv", "ht"), torch.autograd.grad(g, [dO, *diff], u))
    return r
