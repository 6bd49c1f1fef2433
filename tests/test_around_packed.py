"""Outputs that are parts of one packed tensor, in every order of its dimensions: the overlap check of the attention
gradients against the sets of bytes themselves (host checks, no launch)."""

import itertools

import pytest
import torch

R = pytest.importorskip("paper_2609_06712_amd.rola")

no_gpu = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="host-validation test: CPU only")
GB = 1 << 36
ROW = 256  # bytes of a row: d 128 in bf16


def _parts(order, sizes, parts):
    """Byte strides of B, H, N and the offsets of the parts of a packed tensor with the dimensions in `order`."""
    stride, s = {}, ROW
    for dim in reversed(order):
        stride[dim] = s
        s *= parts if dim == "p" else sizes[dim]
    return [stride[x] for x in "bhn"], [i * stride["p"] for i in range(parts)]


def _bytes(sizes, stride, off):
    """The 16-byte pieces that a part holds."""
    rows = (off + b * stride[0] + h * stride[1] + n * stride[2]
            for b, h, n in itertools.product(*(range(sizes[x]) for x in "bhn")))
    return {r + 16 * i for r in rows for i in range(ROW // 16)}


def _refused(sizes, stride, offs):
    """The message of a backward call with dQ, dK, dV at these places of one buffer. Where they pass, the call is
    stopped by a workspace that lies on Q."""
    N = sizes["n"]
    p = R.AttnProblem(sizes["b"], sizes["h"], sizes["h"], N, N, 128, 1, 0)
    el = [s // 2 for s in stride]
    far = lambda k: R.Heads((k + 1) * GB, *(s // 2 for s in (sizes["h"] * N * ROW, N * ROW, ROW)))
    grads = [R.Heads(9 * GB + o, *el) for o in offs]
    st = R.LIB.rola_attn_backward(p, far(0), far(1), far(2), None, 0.1, far(3), 5 * GB, far(5), *grads, GB, 1 << 32,
                                  None)
    assert st == R.ROLA_ERR_INVALID_ARGUMENT
    return R.LIB.rola_last_error().decode()


@no_gpu
@pytest.mark.parametrize("order", ["".join(o) for o in itertools.permutations("bhnp")])
@pytest.mark.parametrize("B,H,N", [(1, 2, 5), (2, 3, 4), (1, 1, 3), (3, 1, 1), (2, 4, 1)])
def test_parts_of_a_packed_tensor_pass(order, B, H, N):
    sizes = dict(b=B, h=H, n=N)
    stride, offs = _parts(order, sizes, 3)
    assert "output ws" in _refused(sizes, stride, offs)


@no_gpu
@pytest.mark.parametrize("order", ["".join(o) for o in itertools.permutations("bhnp")])
def test_shifted_parts_do_not(order):
    """Part 1 moved by some 16-byte pieces: accepted only where no byte is shared, refused wherever one is."""
    sizes = dict(b=2, h=3, n=4)
    stride, offs = _parts(order, sizes, 3)
    mine = _bytes(sizes, stride, offs[0]) | _bytes(sizes, stride, offs[2])
    for move in (-offs[1], -ROW, -ROW // 2, -16, 16, ROW // 2, ROW, offs[1] - ROW):
        if _bytes(sizes, stride, offs[1] + move) & mine:
            assert "outputs d" in _refused(sizes, stride, [offs[0], offs[1] + move, offs[2]]), move
