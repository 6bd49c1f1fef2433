"""Layer and RMS norm with their gradients against 64 bits (tests/_around.py), on the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402
from tests import _around as A  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


def _inputs(B, N, d, dt, wdt, per_sample, packed, seed, offset=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    x = (offset + rn(B, N, d * packed) * (1 + 5 * (torch.arange(d * packed, device="cuda") % 37 == 0)))
    x = x.to(dt)[..., (packed // 2) * d:(packed // 2 + 1) * d]
    ws = (B, d) if per_sample else (d,)
    return x, (1 + 0.2 * rn(*ws)).to(wdt), (0.3 * rn(*ws)).to(wdt), rn(B, N, d).to(dt)


def _expand(w, x):
    return None if w is None else (w if w.dim() == 1 else w.unsqueeze(1))


CASES = [  # B, N, d, per_sample, packed
    (1, 1, 8, False, 1), (1, 1, 1536, False, 1), (3, 1, 64, True, 1), (2, 5, 504, True, 1),
    (1, 257, 520, False, 3), (1, 700, 1536, False, 3), (2, 301, 2048, True, 1), (1, 130, 2056, False, 1),
    (2, 77, 5120, True, 1), (1, 300, 8192, False, 1), (1, 19, 8200, False, 1), (2, 9, 16384, True, 1),
    (1, 4100, 256, False, 1), (5, 1030, 128, True, 1),
]


@pytest.mark.parametrize("dt,wdt", [(BF, F32), (BF, BF), (F32, F32)])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("B,N,d,per_sample,packed", CASES)
def test_norm_and_gradients(B, N, d, per_sample, packed, kind, dt, wdt):
    x, w, b, dy = _inputs(B, N, d, dt, wdt, per_sample, packed, 7 * N + d)
    out = torch.full((B, N, d), float("nan"), dtype=dt, device="cuda")
    y, mean, rstd = R.rola_norm(x, w, b, kind=kind, out=out, want_stats=True)
    assert y is out
    dx = torch.full((B, N, d), float("nan"), dtype=dt, device="cuda")
    got, dw, db = R.rola_norm_backward(x, w, mean, rstd, dy, kind=kind, out=dx)
    wx, bx = _expand(w, x), _expand(b, x)
    ry, _, mu, rs, ey, _ = A.norm(x, wx, bx, kind)
    A.check("y", y, ry, ey)
    A.check("rstd", rstd, rs.squeeze(-1), 256 * A.E32 * rs.squeeze(-1) * (1 + x.to(A.F64).abs().amax(-1) * rs.squeeze(-1)))
    if kind == "layer":
        A.check("mean", mean, mu.squeeze(-1), 64 * A.E32 * x.to(A.F64).abs().mean(-1))
    else:
        assert mean is None
    over = (1,) if per_sample else (0, 1)
    want, bound = A.norm_grad(x, wx, kind, dy, over)
    for name, g, r, e in zip(("dx", "dw", "db"), (got, dw, db), want, bound):
        assert g.shape == r.shape, name
        A.check(name, g, r, e)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_without_parameters(kind):
    x, _, _, dy = _inputs(2, 33, 96, F32, F32, False, 1, 5)
    y, mean, rstd = R.rola_norm(x, kind=kind, want_stats=True)
    ry, _, _, _, ey, _ = A.norm(x, None, None, kind)
    A.check("y", y, ry, ey)
    assert torch.equal(R.rola_norm(x, kind=kind)[0], y)
    for per_sample in (False, True):
        dx, dw, db = R.rola_norm_backward(x, None, mean, rstd, dy, kind=kind, want_bias=False,
                                          per_sample=per_sample)
        want, bound = A.norm_grad(x, None, kind, dy, (1,) if per_sample else (0, 1))
        assert db is None
        A.check("dx", dx, want[0], bound[0])
        A.check("dw", dw, want[1], bound[1])


def test_constant_rows_and_large_offsets():
    """A constant row has xh = 0 (rstd = eps^-1/2); a mean far above the spread keeps the spread."""
    x = torch.full((3, 4, 1536), 1000.0, device="cuda")
    x[1] += torch.randn((4, 1536), device="cuda")
    y, mean, rstd = R.rola_norm(x, want_stats=True)
    ry, _, _, _, ey, _ = A.norm(x, None, None, "layer")
    A.check("y", y, ry, ey)
    assert bool((y[0] == 0).all()) and bool((mean[0] == 1000).all())
    assert bool(((rstd[0] - 1e3).abs() <= 1e3 * 4 * A.E32).all())


def test_gradient_against_differences():
    """<dY, Y> by central differences along random directions, the difference quotient taken in 64 bits from the
    reference that the kernel is checked against: ties that reference to the function itself."""
    x, w, b, dy = _inputs(1, 6, 64, F32, F32, False, 1, 3)
    _, mean, rstd = R.rola_norm(x, w, b, want_stats=True)
    dx, dw, db = R.rola_norm_backward(x, w, mean, rstd, dy)
    f = lambda x_, w_, b_: float((A.norm(x_, w_, b_, "layer")[0] * dy.to(A.F64)).sum())
    A.U[torch.float64] = 0.0
    h = 1e-5
    x, w, b = (t.to(A.F64) for t in (x, w, b))
    for k in range(3):
        vx, vw, vb = (torch.randn(t.shape, dtype=A.F64, device="cuda") for t in (x, w, b))
        want = (f(x + h * vx, w + h * vw, b + h * vb) - f(x - h * vx, w - h * vw, b - h * vb)) / (2 * h)
        got = float((dx.to(A.F64) * vx).sum() + (dw.to(A.F64) * vw).sum() + (db.to(A.F64) * vb).sum())
        # fp32 gradients of 384 + 128 terms of size ~1: 2^-20 each; the quotient's h^2 term
        assert abs(got - want) <= 1e-3 * (1 + abs(want)), (got, want)


def test_other_stream_and_two_calls_at_once():
    x, w, b, dy = _inputs(2, 513, 1536, BF, F32, True, 1, 11)
    want = R.rola_norm(x, w, b)[0]
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for st in s:
        with torch.cuda.stream(st):
            got.append(R.rola_norm(x, w, b)[0])
    st = torch.cuda.Stream()
    got.append(R.rola_norm(x, w, b, out=torch.empty_like(want), stream=st)[0])
    torch.cuda.synchronize()
    for g in got:
        assert torch.equal(g, want)
