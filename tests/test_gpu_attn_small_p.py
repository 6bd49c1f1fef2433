"""dK where the probabilities are small: the bf16 gradients in the norm of the whole tensors and of each key's row
(tests/_around_size.py) beside a key that takes nearly all of every row, and over long key sets, on the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402
from tests import _around_size as S  # noqa: E402


@pytest.mark.parametrize("kind,H,Hkv,Nq,Nk,causal", [
    ("sink", 2, 2, 512, 8400, False), ("sink", 4, 2, 130, 512, False), ("sink", 2, 1, 900, 1100, True),
    ("plain", 1, 1, 200, 75600, False), ("plain", 1, 1, 64, 300000, False),
])
def test_gradients_of_small_probabilities(kind, H, Hkv, Nq, Nk, causal):
    q, k, v, do = S.inputs(kind, 1, H, Hkv, Nq, Nk, seed=Nq + Nk, device="cuda")
    o, lse = R.rola_attn(q, k, v, causal=causal)
    dq, dk, dv = R.rola_attn_backward(q, k, v, o, lse, do, causal=causal)
    ref = S.reference(q, k, v, None, causal, 128 ** -0.5, do)
    S.check(dict(o=o, dq=dq, dk=dk, dv=dv), ref)


def test_spread_scores_lose_no_key():
    """Scores of some hundred: every key whose gradient bf16 can hold has one that is not zero."""
    g = torch.Generator(device="cuda").manual_seed(5)
    rn = lambda n, s=1.0: (s * torch.randn((1, 1, n, 128), generator=g, device="cuda")).to(torch.bfloat16)
    q, k, v, do = rn(150, 20.0), rn(400), rn(400), rn(150)
    o, lse = R.rola_attn(q, k, v)
    dk = R.rola_attn_backward(q, k, v, o, lse, do)[1]
    want, err, worst, _ = S.reference(q, k, v, None, False, 128 ** -0.5, do)["dk"]
    size = want.norm(dim=-1)
    live = size > 2.0 ** -30
    assert int(live.sum()) > 390
    assert bool(((dk.double() - want).norm(dim=-1) <= 0.5 * size + 4 * S.U * (err + worst).sqrt())[live].all())
