"""Layer and RMS norm at the widths on either side of each change of the kernels' form (pieces per thread, threads
per row), few rows and many, against 64 bits (tests/_around.py), on the GPU."""

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import rola as R  # noqa: E402
from tests import _around as A  # noqa: E402


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [5, 300])
@pytest.mark.parametrize("d", [512, 520, 1024, 1032, 1536, 1544, 2048, 2056, 4096, 4104, 6144, 6152, 8192, 8200,
                               12288, 12296, 16384])
def test_widths(d, rows, dt):
    g = torch.Generator(device="cuda").manual_seed(d + rows)
    rn = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, w, b, dy = (0.5 + rn(1, rows, d)).to(dt), 1 + 0.2 * rn(d), rn(d), rn(1, rows, d).to(dt)
    for kind in ("layer", "rms"):
        y, mean, rstd = R.rola_norm(x, w, b, kind=kind, want_stats=True)
        ry, _, _, _, ey, _ = A.norm(x, w, b, kind)
        A.check("y", y, ry, ey)
        got = R.rola_norm_backward(x, w, mean, rstd, dy, kind=kind)
        want, bound = A.norm_grad(x, w, kind, dy, (0, 1))
        for name, a, r, e in zip(("dx", "dw", "db"), got, want, bound):
            A.check(name, a, r, e)
