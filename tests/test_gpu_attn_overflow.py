"""Attention gradients beyond fp32's range, on the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402


@pytest.mark.parametrize("dt,d", [(torch.float32, 64), (torch.float32, 128), (torch.bfloat16, 128)])
@pytest.mark.parametrize("Nq,Nk", [(64, 40), (9000, 3000)])
def test_keys_that_are_not_there_get_zero_beside_a_gradient_that_overflows(Nq, Nk, dt, d):
    """The one key's gradients overflow fp32; those of the keys behind it are zero all the same."""
    B = 1 if Nk == 40 else 24  # (fewer and more than one tile of keys per CU)
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn((B, 1, n, d), generator=g, device="cuda").to(dt) for n in (Nq, Nk, Nk))
    do = torch.full_like(q, 3e38)
    kv_len = torch.ones(B, dtype=torch.int32, device="cuda")
    o, lse = R.rola_attn(q, k, v, kv_len=kv_len)
    _, dk, dv = R.rola_attn_backward(q, k, v, o, lse, do, kv_len=kv_len)
    assert bool(dv[:, :, 0].isinf().all())
    assert bool((dk[:, :, 1:] == 0).all()) and bool((dv[:, :, 1:] == 0).all())


@pytest.mark.parametrize("power", [-60, 40, 90])
@pytest.mark.parametrize("Nq,Nk", [(64, 40), (1500, 3000)])
def test_bf16_gradients_scale_exactly_with_the_output_gradient(Nq, Nk, power):
    """dO times a power of two, up to gradients of some 2^100: every bit of the gradients moves with it."""
    g = torch.Generator(device="cuda").manual_seed(Nq)
    q, k, v, do = (torch.randn((1, 2, n, 128), generator=g, device="cuda").to(torch.bfloat16) for n in (Nq, Nk, Nk, Nq))
    o, lse = R.rola_attn(q, k, v, causal=True)
    want = R.rola_attn_backward(q, k, v, o, lse, do, causal=True)
    got = R.rola_attn_backward(q, k, v, o, lse, do * 2.0 ** power, causal=True)
    for a, b in zip(got, want):
        assert torch.equal(a, b * 2.0 ** power)
