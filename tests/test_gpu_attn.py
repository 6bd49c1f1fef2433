"""Softmax attention over another set of tokens with its gradients against 64 bits (tests/_around.py), on
the GPU."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402
from tests import _around as A  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


def _inputs(B, H, Hkv, Nq, Nk, d, dt, packed=False, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def heads(h, n, s=1.0):
        x = (s * torch.randn((B, h, n, d), generator=g, device="cuda")).to(dt)
        return x.transpose(1, 2).contiguous().transpose(1, 2) if packed else x

    return heads(H, Nq, spread), heads(Hkv, Nk), heads(Hkv, Nk), heads(H, Nq)


def _nan_like(x):
    return torch.full_like(x, float("nan"))


def _run(B, H, Hkv, Nq, Nk, lens, causal, dt, d, packed=False, seed=0, spread=1.0, poison=True, grads=True):
    q, k, v, do = _inputs(B, H, Hkv, Nq, Nk, d, dt, packed, seed, spread)
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    scale = d ** -0.5
    want, bound = A.attention(q, k, v, lens, causal, scale, do if grads else None)
    if lens is not None and poison:  # what lies behind a sample's keys is never used
        for b, n in enumerate(lens):
            k[b, :, max(0, n):] = float("nan")
            v[b, :, max(0, n):] = float("inf")
    o, lse = R.rola_attn(q, k, v, kv_len=kv_len, causal=causal, out=_nan_like(q),
                         lse=torch.full((B, H, Nq), float("nan"), device="cuda"))
    got = [o, lse]
    if grads:
        got += R.rola_attn_backward(q, k, v, o, lse, do, kv_len=kv_len, causal=causal, dQ=_nan_like(q),
                                    dK=_nan_like(v), dV=_nan_like(v))
    for name, x, r, e in zip(("o", "lse", "dq", "dk", "dv"), got, want, bound):
        A.check(name, x, r, e)
    return got


SHAPES = [  # B, H, Hkv, Nq, Nk, lens, causal
    (1, 1, 1, 1, 1, None, False),
    (1, 1, 1, 1, 1, [0], False),
    (2, 2, 1, 1, 33, [33, 1], False),
    (1, 5, 1, 1, 700, None, False),
    (2, 8, 2, 3, 1100, [1100, 517], True),
    (1, 2, 2, 31, 32, None, False),
    (1, 2, 2, 32, 31, None, True),
    (1, 2, 2, 33, 65, None, True),
    (1, 3, 3, 64, 1, None, False),
    (2, 2, 2, 127, 129, [129, 0], False),
    (1, 2, 2, 128, 128, None, True),
    (2, 4, 2, 129, 97, [97, 40], True),      # fewer keys than queries: rows without a key
    (3, 6, 3, 200, 300, [300, 31, 64], True),
    (1, 12, 12, 390, 512, [77], False),
    (2, 4, 1, 257, 640, [640, 333], False),
    (1, 2, 2, 1000, 37, None, False),
    (1, 2, 2, 20, 1500, None, True),         # few rows, split over the keys, causal
    (1, 1, 1, 40, 1500, [1411], False),
    (1, 2, 1, 2600, 96, None, False),        # few keys, the queries split
]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,lens,causal", SHAPES)
def test_bf16(B, H, Hkv, Nq, Nk, lens, causal, packed):
    _run(B, H, Hkv, Nq, Nk, lens, causal, BF, 128, packed, seed=Nq + 3 * Nk)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,lens,causal", SHAPES)
def test_f32(B, H, Hkv, Nq, Nk, lens, causal, d):
    _run(B, H, Hkv, Nq, Nk, lens, causal, F32, d, packed=d == 64, seed=Nq + 5 * Nk)


@pytest.mark.parametrize("dt", [BF, F32])
def test_spiky_scores(dt):
    """Scores of some hundred (a one-hot softmax): the running maximum moves often and far."""
    _run(1, 2, 2, 150, 400, None, False, dt, 128, seed=5, spread=20.0)
    _run(1, 2, 1, 150, 400, [311], True, dt, 128, seed=6, spread=20.0)


def test_long_cache_ragged():
    _run(3, 10, 2, 1, 20011, [20011, 7000, 1], False, BF, 128, seed=9, grads=False)
    _run(1, 2, 2, 300, 9000, [8999], True, BF, 128, seed=10, grads=False)


def test_offsets_past_32_bits():
    """A packed cache of 2.9 GB whose last tokens lie behind 2^31 bytes."""
    Nk, width = 70000, 20480
    cache = torch.zeros((Nk, width), dtype=BF, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = torch.randn((2, Nk, 128), generator=g, device="cuda").to(BF)
    cache[:, 20224:20352], cache[:, 20352:] = k, v
    K, V = (cache[:, c:c + 128].unflatten(1, (1, 128)).transpose(0, 1).unsqueeze(0) for c in (20224, 20352))
    assert K.stride(2) * 2 * Nk > 2 ** 31
    for Nq in (1, 200):
        q = torch.randn((1, 1, Nq, 128), generator=g, device="cuda").to(BF)
        o, lse = R.rola_attn(q, K, V, causal=True)
        wo, wl = R.rola_attn(q, k.view(1, 1, Nk, 128), v.view(1, 1, Nk, 128), causal=True)
        assert torch.equal(o, wo) and torch.equal(lse, wl)


def test_parts_of_one_packed_tensor():
    """q, k, v and their gradients as parts of packed [B, N, 3, H, d] tensors, broadcast dO."""
    B, N, H, d = 2, 150, 3, 128
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.randn((B, N, 3, H, d), generator=g, device="cuda").to(BF)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    do = torch.randn((B, 1, N, d), generator=g, device="cuda").to(BF).expand(B, H, N, d)
    want, bound = A.attention(q, k, v, None, False, d ** -0.5, do)
    o, lse = R.rola_attn(q, k, v)
    assert o.transpose(1, 2).is_contiguous()  # token after token, as q
    dqkv = _nan_like(qkv)
    R.rola_attn_backward(q, k, v, o, lse, do, dQ=dqkv[:, :, 0].transpose(1, 2), dK=dqkv[:, :, 1].transpose(1, 2),
                         dV=dqkv[:, :, 2].transpose(1, 2))
    A.check("o", o, want[0], bound[0])
    for i in range(3):
        A.check("dq dk dv"[3 * i:3 * i + 2], dqkv[:, :, i].transpose(1, 2), want[2 + i], bound[2 + i])


def test_same_as_the_dense_reference():
    """The square call against this library's dense attention (another kernel)."""
    q, k, v, _ = _inputs(1, 2, 2, 390, 390, 128, BF, seed=8)
    want, bound = A.attention(q, k, v, None, False, 128 ** -0.5)
    o, _ = R.rola_attn(q, k, v)
    dense = R.rola_dense_attn(q, k, v, (3, 10, 13))
    A.check("dense", dense, want[0], 2 * bound[0])
    A.check("o", o, dense.to(A.F64), 3 * bound[0])


def test_gradients_against_differences():
    q, k, v, do = _inputs(1, 2, 1, 9, 17, 64, F32, seed=2)
    o, lse = R.rola_attn(q, k, v, causal=True)
    grads = R.rola_attn_backward(q, k, v, o, lse, do, causal=True)
    A.U[torch.float64] = 0.0
    f = lambda *t: float((A.attention(*t, None, True, 0.125)[0][0] * do.to(A.F64)).sum())
    x, h = [t.to(A.F64) for t in (q, k, v)], 1e-5
    for _ in range(3):
        dirs = [torch.randn(t.shape, dtype=A.F64, device="cuda") for t in x]
        want = (f(*(t + h * s for t, s in zip(x, dirs))) - f(*(t - h * s for t, s in zip(x, dirs)))) / (2 * h)
        got = sum(float((g.to(A.F64) * s).sum()) for g, s in zip(grads, dirs))
        assert abs(got - want) <= 1e-3 * (1 + abs(want)), (got, want)


def test_captured_and_replayed():
    """Forward and backward in a graph, replayed with new inputs between eager work, against eager results."""
    q, k, v, do = _inputs(2, 4, 2, 40, 900, 128, BF, seed=3)
    kv_len = torch.tensor([900, 450], dtype=torch.int32, device="cuda")
    x = torch.randn((2, 40, 512), device="cuda").to(BF)

    def step():
        y, mean, rstd = R.rola_norm(x, kind="layer", want_stats=True)
        o, lse = R.rola_attn(q, k, v, kv_len=kv_len)
        g = R.rola_attn_backward(q, k, v, o, lse, do, kv_len=kv_len)
        n = R.rola_norm_backward(x, None, mean, rstd, y)
        return [y, o, lse, *g, *n]

    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        outs = step()
    for r in range(4):
        q.copy_(torch.randn(q.shape, device="cuda"))
        x.copy_(torch.randn(x.shape, device="cuda"))
        kv_len.copy_(torch.tensor([900 - 100 * r, 450 - 150 * r], device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for a, b in zip(got, step()):
            assert torch.equal(a, b), r


def test_same_result_every_time():
    q, k, v, do = _inputs(1, 4, 2, 300, 700, 128, BF, seed=13)
    first = None
    for _ in range(3):
        o, lse = R.rola_attn(q, k, v)
        out = [o, lse, *R.rola_attn_backward(q, k, v, o, lse, do)]
        first = first or out
        assert all(torch.equal(a, b) for a, b in zip(first, out))


def test_rows_and_guard_zones_untouched():
    """Nothing outside a view is written: outputs inside a larger tensor keep what lies around them."""
    q, k, v, do = _inputs(1, 2, 2, 45, 70, 128, BF, seed=14)
    big = [torch.full((1, 4, t.shape[2] + 6, 128), 7.0, dtype=BF, device="cuda") for t in (q, q, k, k)]
    o, dq, dk, dv = (t[:, 1:3, 3:-3] for t in big)
    _, lse = R.rola_attn(q, k, v, out=o)
    R.rola_attn_backward(q, k, v, o, lse, do, dQ=dq, dK=dk, dV=dv)
    want, bound = A.attention(q, k, v, None, False, 128 ** -0.5, do)
    for t, view, i in zip(big, (o, dq, dk, dv), (0, 2, 3, 4)):
        A.check(str(i), view, want[i], bound[i])
        view.fill_(7.0)
        assert bool((t == 7.0).all())


def test_f32_gradients_of_more_rows_than_one_turn_of_the_row_products():
    """2^20 + 37 queries over two keys: the last rows' products come from a second turn."""
    N = 2 ** 20 + 37
    q, k, v, do = _inputs(1, 1, 1, N, 2, 64, F32, seed=9)
    o, lse = R.rola_attn(q, k, v)
    dq = R.rola_attn_backward(q, k, v, o, lse, do, dQ=_nan_like(q))[0]
    tail = slice(N - 101, N)
    want, bound = A.attention(q[:, :, tail], k, v, None, False, 64 ** -0.5, do[:, :, tail])
    A.check("dq", dq[:, :, tail], want[2], bound[2])


def test_workspace_of_another_stream_is_not_given_out_again(monkeypatch):
    """After a call on a given stream, the current stream's next allocations are not the call's workspace."""
    from paper_2609_06712_amd import rola

    taken = []

    class Calls:
        def __getattr__(self, name):
            fn = getattr(lib, name)

            def call(*args):
                if name in ("rola_attn", "rola_attn_backward"):
                    taken.append((args[-3], args[-2]))
                return fn(*args)
            return call

    lib = rola.LIB
    q, k, v, do = _inputs(1, 2, 1, 20, 1500, 128, BF, seed=12)
    want = R.rola_attn(q, k, v)
    want += R.rola_attn_backward(q, k, v, *want, do)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    monkeypatch.setattr(rola, "LIB", Calls())
    st = torch.cuda.Stream()
    got = R.rola_attn(q, k, v, stream=st)
    got += R.rola_attn_backward(q, k, v, *got, do, stream=st)
    again = [torch.empty(n, dtype=torch.uint8, device="cuda") for _, n in taken for _ in range(3)]
    torch.cuda.synchronize()
    assert len(taken) == 2 and all(n > 0 for _, n in taken)
    for x in again:
        for p, n in taken:
            assert x.data_ptr() + x.numel() <= p or p + n <= x.data_ptr()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("B,H,Hkv,Nq,Nk,d,lens,causal", [
    (1, 3, 3, 700, 2900, 128, None, False),      # 64-row tiles, cut: forward and gradients
    (2, 4, 2, 309, 3100, 128, [3100, 1777], False),
    (1, 4, 2, 1201, 1190, 128, None, True),      # 64-row tiles in the gradients only
    (1, 4, 4, 1500, 1600, 64, [1533], False),    # d 64: 16-row tiles forward, 64 in the gradients
    (1, 2, 1, 1100, 1500, 128, [1100], True),    # 16-row tiles in both
])
def test_f32_tiles_by_the_amount_of_work(B, H, Hkv, Nq, Nk, d, lens, causal):
    _run(B, H, Hkv, Nq, Nk, lens, causal, F32, d, packed=True, seed=13)
