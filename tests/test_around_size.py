"""The norm-wise bounds of tests/_around_size.py tell the roundings that the kernels make from mistakes, on a
64-bit emulation of the roundings (CPU): the emulation lies within them, with a mistake planted it does not."""

import pytest
import torch

from tests import _around_size as S

F64, BF = torch.float64, torch.bfloat16


def emulated(q, k, v, do, mistake=None):
    """One head's outputs with the kernels' roundings to fewer bits; fp32 sums are taken as exact."""
    scale = q.shape[-1] ** -0.5
    Q, K, V, dO = (t[0, 0].to(F64) for t in (q, k, v, do))
    bf = lambda x: x.to(BF).to(F64)
    s = scale * Q @ K.t()
    lse = torch.logsumexp(s, -1, keepdim=True)
    p = torch.exp(s - lse)
    part = torch.exp(s - s.amax(-1, keepdim=True))
    live = torch.ones(K.shape[0], dtype=F64)
    if mistake == "key":  # one key left out of the walks
        live[K.shape[0] // 2] = 0
    o = bf((bf(part) * live) @ V / part.sum(-1, keepdim=True))
    dp = dO @ V.t()
    D = (dO * o).sum(-1, keepdim=True) if mistake == "D from O" else (p * dp).sum(-1, keepdim=True)
    ds = p * (dp - D) * live
    two = bf(ds) if mistake == "one term" else bf(ds) + bf(ds - bf(ds))
    half = lambda x, e: torch.ldexp(torch.ldexp(x, torch.tensor(e)).half().to(F64), torch.tensor(-e))
    ph = half(p, 0 if mistake == "P unscaled" else 15)
    out = dict(o=o, dq=bf(scale * two @ K), dk=bf(scale * bf(ph * (dp - D)).t() @ Q), dv=bf(bf(p).t() @ dO))
    if mistake in out:
        out[mistake] = out[mistake] * 1.01
    return {n: x[None, None] for n, x in out.items()}


CASES = [("plain", 200, 4000), ("offset", 200, 4000), ("sink", 200, 4000), ("plain", 40, 60000)]


@pytest.mark.parametrize("kind,Nq,Nk", CASES)
def test_the_kernels_roundings_pass(kind, Nq, Nk):
    x = S.inputs(kind, 1, 1, 1, Nq, Nk)
    S.check(emulated(*x), S.reference(*x[:3], None, False, 128 ** -0.5, x[3]))


@pytest.mark.parametrize("mistake,kind,Nq,Nk,seen_in", [
    ("o", "plain", 200, 4000, "o"), ("dq", "plain", 200, 4000, "dq"), ("dk", "plain", 200, 4000, "dk"),
    ("dv", "plain", 200, 4000, "dv"), ("key", "plain", 200, 4000, "o"), ("key", "plain", 200, 4000, "dq"),
    ("D from O", "offset", 200, 4000, "dq"), ("one term", "offset", 200, 4000, "dq"),
    ("P unscaled", "sink", 200, 4000, "dk"), ("P unscaled", "plain", 16, 300000, "dk"),
])
def test_a_mistake_does_not(mistake, kind, Nq, Nk, seen_in):
    x = S.inputs(kind, 1, 1, 1, Nq, Nk)
    ref = S.reference(*x[:3], None, False, 128 ** -0.5, x[3])
    with pytest.raises(AssertionError, match=f"'{seen_in}'"):
        S.check({seen_in: emulated(*x, mistake)[seen_in]}, ref)
