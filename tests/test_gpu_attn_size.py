"""The bf16 attention and its gradients against 64 bits in the norm of the whole tensors and of their rows
(tests/_around_size.py), on the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402
from tests import _around_size as S  # noqa: E402


@pytest.mark.parametrize("kind,B,H,Hkv,Nq,Nk,lens,causal", [
    ("plain", 2, 4, 2, 300, 4000, [4000, 2500], False),
    ("plain", 1, 2, 2, 1500, 1500, None, True),
    ("plain", 2, 8, 2, 3, 20000, [20000, 311], False),   # few rows, split over the keys
    ("plain", 1, 3, 3, 2600, 77, None, False),           # few keys, split over the queries
    ("offset", 1, 2, 1, 256, 4096, None, False),
    ("offset", 2, 2, 1, 700, 3001, [3001, 900], True),
])
def test_bf16_in_the_norm(kind, B, H, Hkv, Nq, Nk, lens, causal):
    q, k, v, do = S.inputs(kind, B, H, Hkv, Nq, Nk, seed=Nq + Nk, device="cuda")
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, lse = R.rola_attn(q, k, v, kv_len=kv_len, causal=causal)
    dq, dk, dv = R.rola_attn_backward(q, k, v, o, lse, do, kv_len=kv_len, causal=causal)
    ref = S.reference(q, k, v, lens, causal, 128 ** -0.5, do)
    S.check(dict(o=o, dq=dq, dk=dk, dv=dv), ref)
