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
