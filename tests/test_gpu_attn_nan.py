"""What NaN and infinite scores leave: the rows that see one are NaN in every output, and no other row or key
changes, on the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
# few and many rows, each whole and cut over its keys
SHAPES = [(1, 2, 2, 20, 40), (1, 4, 2, 5, 3000), (1, 2, 1, 300, 90), (2, 2, 2, 900, 1700), (1, 12, 12, 1500, 1100)]
FORMS = [(BF, 128), (F32, 64), (F32, 128)]


def _inputs(B, H, Hkv, Nq, Nk, dt, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda h, n: torch.randn((B, h, n, d), generator=g, device="cuda").to(dt)
    return rn(H, Nq), rn(Hkv, Nk), rn(Hkv, Nk), rn(H, Nq)


@pytest.mark.parametrize("dt,d", FORMS)
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk", SHAPES)
def test_nan_query(B, H, Hkv, Nq, Nk, dt, d):
    """One query is NaN: its row is, and what sums over its head's queries; the other rows and heads stay as they were."""
    q, k, v, do = _inputs(B, H, Hkv, Nq, Nk, dt, d, Nq)
    n = Nk - 3
    kv_len = torch.full((B,), n, dtype=torch.int32, device="cuda")
    clean_o, clean_lse = R.rola_attn(q, k, v, kv_len=kv_len)
    clean = R.rola_attn_backward(q, k, v, clean_o, clean_lse, do, kv_len=kv_len)
    row = Nq // 2
    q[0, 1, row, 5] = float("nan")
    o, lse = R.rola_attn(q, k, v, kv_len=kv_len)
    hit = torch.zeros((B, H, Nq), dtype=torch.bool, device="cuda")
    hit[0, 1, row] = True
    assert torch.equal(lse.isnan(), hit)
    assert torch.equal(o.isnan().all(-1), hit) and torch.equal(o.isnan().any(-1), hit)
    assert torch.equal(o[~hit], clean_o[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])
    dq, dk, dv = R.rola_attn_backward(q, k, v, o, lse, do, kv_len=kv_len)
    assert bool(dq[hit].isnan().all()) and torch.equal(dq[~hit], clean[0][~hit])
    head = torch.zeros((B, Hkv, Nk), dtype=torch.bool, device="cuda")
    head[0, Hkv // H, :n] = True  # the key head of query head 1
    for x, c in ((dk, clean[1]), (dv, clean[2])):
        assert bool(x[head].isnan().all()) and torch.equal(x[~head], c[~head])
        assert bool((x[:, :, n:] == 0).all())  # a key that is not there


@pytest.mark.parametrize("dt,d", FORMS)
@pytest.mark.parametrize("B,H,Hkv,Nq,Nk", SHAPES)
def test_infinite_key(B, H, Hkv, Nq, Nk, dt, d):
    """A key with an infinite channel: rows whose score is +inf have no softmax (NaN), those of -inf go without it."""
    q, k, v, do = _inputs(B, H, Hkv, Nq, Nk, dt, d, Nq + 1)
    q[..., 7] += (q[..., 7] == 0).to(dt)
    k[:, :, Nk // 2, 7] = float("inf")
    up = q[..., 7] > 0
    o, lse = R.rola_attn(q, k, v)
    assert torch.equal(lse.isnan(), up) and torch.equal(o.isnan().any(-1), up)
    assert bool(lse[~up].isfinite().all())
    dq, dk, dv = R.rola_attn_backward(q, k, v, o, lse, do)
    assert bool(dq[up].isnan().all()) and bool(dk.isnan().all()) and bool(dv.isnan().all())
