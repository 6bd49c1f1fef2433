"""Attention with its inputs and gradients as parts of packed tensors of every order, against separate tensors, on
the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dt,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("B,H,Nq,Nk", [(2, 3, 150, 150), (1, 2, 4, 700), (2, 2, 1, 1)])
@pytest.mark.parametrize("order", ["bphnd", "bhpnd", "bhnpd", "bnphd", "bnhpd", "bpnhd", "phbnd"])
def test_packed_in_and_out(order, B, H, Nq, Nk, dt, d):
    """K and V in one packed tensor and their gradients in another of the same order; Q, O and dQ with them where the
    lengths are equal."""
    g = torch.Generator(device="cuda").manual_seed(Nq)
    parts = 3 if Nq == Nk else 2
    sizes = dict(b=B, h=H, n=Nk, p=parts, d=d)
    like = lambda fill: torch.full([sizes[x] for x in order], fill, dtype=dt, device="cuda")

    def views(t):
        t = t.permute(*(order.index(x) for x in "pbhnd"))
        return [t[i] for i in range(parts)]

    kv, dkv = like(0.0).normal_(generator=g), like(float("nan"))
    x, dx = views(kv), views(dkv)
    new = lambda: torch.randn((B, H, Nq, d), generator=g, device="cuda").to(dt)
    q, do = x[2] if parts == 3 else new(), new()
    k, v = x[:2]
    o, lse = R.rola_attn(q, k, v)
    want_o, want_lse = R.rola_attn(q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(o, want_o) and torch.equal(lse, want_lse)
    want = R.rola_attn_backward(q.contiguous(), k.contiguous(), v.contiguous(), o.contiguous(), lse, do)
    got = R.rola_attn_backward(q, k, v, o, lse, do, dQ=dx[2] if parts == 3 else None, dK=dx[0], dV=dx[1])
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert not bool(dkv.isnan().any())
