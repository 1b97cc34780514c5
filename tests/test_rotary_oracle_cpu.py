"""Pins of the oracle of normalised, rotated heads (oracle/rotary_oracle.py): torch's own double backward in float64
through a forward written with complex numbers, and central differences.  And of the frequencies."""
import numpy as np
import pytest
import torch

from oracle import rotary_oracle
from paper_2609_24089_amd import rotary_frequencies

# d, pairs, norm, interleaved, axes
CASES = [(16, 8, True, False, 1), (16, 8, True, True, 1), (20, 4, True, False, 2), (12, 6, False, True, 3),
         (12, 4, False, False, 1)]


def inputs(case, seed):
    d, pairs, norm, interleaved, axes = case
    rng = np.random.default_rng(seed)
    x = {n: rng.standard_normal((2, 3, 4, d)) for n in ("x", "dy", "u")}
    x.update({n: rng.standard_normal(d) if norm else None for n in ("w", "uw")})
    freqs, axis = rng.uniform(0.01, 1.0, pairs), rng.integers(0, axes, pairs)
    return x, rotary_oracle.angles(rng.integers(-5, 40, (axes, 2, 4)), freqs, axis)


def torch_forward(x, w, angle, eps, interleaved):
    pairs = angle.shape[-1]
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w
    head, tail = x[..., :2 * pairs], x[..., 2 * pairs:]
    z = torch.complex(head[..., 0::2], head[..., 1::2]) if interleaved else torch.complex(head[..., :pairs],
                                                                                         head[..., pairs:])
    z = z * torch.polar(torch.ones_like(angle), angle)[:, None]
    y = torch.stack([z.real, z.imag], -1).flatten(-2) if interleaved else torch.cat([z.real, z.imag], -1)
    return torch.cat([y, tail], -1)


@pytest.mark.parametrize("case", CASES, ids=range(len(CASES)))
def test_matches_torch_double_backward(case):
    x, angle = inputs(case, 2)
    eps, interleaved = 0.01, case[3]
    got = rotary_oracle.run(x["x"], angle, x["w"], eps, interleaved, x["dy"], x["u"], x["uw"])
    t = {n: torch.tensor(v, requires_grad=True) for n, v in x.items() if v is not None}
    y = torch_forward(t["x"], t.get("w"), torch.tensor(angle), eps, interleaved)
    leaves = [t[n] for n in ("x", "w") if n in t]
    g = torch.autograd.grad(y, leaves, t["dy"], create_graph=True)
    h = torch.autograd.grad(g, [t["dy"], *leaves], [t[n].detach() for n in ("u", "uw") if n in t], allow_unused=True)
    want = {"y": y, "dx": g[0], "dyt": h[0], "xt": torch.zeros_like(y) if h[1] is None else h[1]}
    if case[2]:
        want.update(dw=g[1], wt=h[2])
    assert set(want) == set(got)
    for n, v in want.items():
        np.testing.assert_allclose(got[n], v.detach().numpy(), rtol=0, atol=1e-12, err_msg=n)


def test_matches_central_differences():
    """Step 1e-5: off by the step's square times a third derivative and by rounding over the step, below 1e-7."""
    x, angle = inputs(CASES[0], 3)
    rng = np.random.default_rng(4)
    h = 1e-5
    run = lambda y: rotary_oracle.run(y["x"], angle, y["w"], 0.01, False, y["dy"], x["u"], x["uw"])  # noqa: E731
    got = run(x)

    def phi(y):
        r = run(y)
        return (r["y"] * y["dy"]).sum(), (r["dx"] * x["u"]).sum() + (r["dw"] * x["uw"]).sum()

    for name, first, second in (("x", "dx", "xt"), ("w", "dw", "wt"), ("dy", "y", "dyt")):
        v = rng.standard_normal(x[name].shape)
        hi, lo = phi({**x, name: x[name] + h * v}), phi({**x, name: x[name] - h * v})
        assert abs((hi[0] - lo[0]) / (2 * h) - (got[first] * v).sum()) < 1e-7, name
        assert abs((hi[1] - lo[1]) / (2 * h) - (got[second] * v).sum()) < 1e-7, name


def test_frequencies():
    freqs, axes = rotary_frequencies(64, base=500.0)
    assert freqs.dtype == torch.float64 and axes.dtype == torch.int32 and int(axes.max()) == 0
    np.testing.assert_allclose(freqs.numpy(), 500.0 ** (-np.arange(32) / 32), rtol=1e-15)
    freqs, axes = rotary_frequencies(64, sections=(8, 14, 10))
    assert axes.tolist() == [0] * 8 + [1] * 14 + [2] * 10
    np.testing.assert_allclose(freqs.numpy(), 10000.0 ** (-np.arange(32) / 32), rtol=1e-15)
    freqs, axes = rotary_frequencies(32, sections=(6, 10), apart=True)
    np.testing.assert_allclose(freqs.numpy(), np.concatenate([10000.0 ** (-np.arange(6) / 6),
                                                              10000.0 ** (-np.arange(10) / 10)]), rtol=1e-15)
    for bad in (dict(dims=24), dict(dims=0), dict(dims=32, sections=(8, 9)), dict(dims=32, sections=(-1, 17)),
                dict(dims=32, base=0.0)):
        with pytest.raises(ValueError):
            rotary_frequencies(**bad)
