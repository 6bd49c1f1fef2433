"""The norms and the attention together, as they are used: the text cross-attention with its gradients
(train.cross_forward, cross_backward) against 64-bit autograd, and the DiT block with the library's norms
and cross-attention around the module, on the GPU."""

import math

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU hosts too; every test here is skipped there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2609_06712_amd import dit_block as DB  # noqa: E402
from paper_2609_06712_amd import rola as R  # noqa: E402
from paper_2609_06712_amd import train as T  # noqa: E402

F64 = torch.float64


def _reference(x, ctx, w, heads, lens, dout, eps=1e-6):
    """Output and gradients in 64 bits by differentiating the definition."""
    leaves = {"x": x, "ctx": ctx, **w}
    leaves = {k: v.to(F64).requires_grad_() for k, v in leaves.items() if v is not None}
    x, ctx = leaves["x"], leaves["ctx"]
    B, N, d = x.shape
    mu = x.mean(-1, keepdim=True)
    h = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(-1, keepdim=True) + eps)
    pick = lambda t: t if t.dim() == 1 else t.unsqueeze(1)
    h = h * pick(leaves["ln_w"]) + pick(leaves["ln_b"])
    rms = lambda t, g: t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps) * g
    q, k, v = rms(h @ leaves["Wq"].t(), leaves["nq"]), rms(ctx @ leaves["Wk"].t(), leaves["nk"]), ctx @ leaves["Wv"].t()
    outs = []
    for b in range(B):
        qs, ks, vs = (t[b].view(-1, heads, d // heads).transpose(0, 1) for t in (q, k, v))
        n = ctx.shape[1] if lens is None else lens[b]
        if n == 0:
            outs.append(torch.zeros_like(x[b]))
            continue
        s = qs @ ks[:, :n].transpose(1, 2) / math.sqrt(d // heads)
        outs.append((torch.softmax(s, -1) @ vs[:, :n]).transpose(0, 1).reshape(N, d))
    out = torch.stack(outs) @ leaves["Wo"].t()
    names = list(leaves)
    g = torch.autograd.grad(out, [leaves[n] for n in names], dout.to(F64), allow_unused=True)
    return out.detach(), dict(zip(names, g))


def _case(dt, d, B, N, L, per_sample, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s, scale=1.0, off=0.0: (off + scale * torch.randn(s, generator=g, device="cuda"))
    x, ctx, dout = rn(B, N, d).to(dt), rn(B, L, d).to(dt), rn(B, N, d).to(dt)
    w = {k: rn(d, d, scale=d ** -0.5).to(dt) for k in ("Wq", "Wk", "Wv", "Wo")}
    w.update({k: rn(d, scale=0.1, off=1.0).to(dt) for k in ("nq", "nk")})
    shape = (B, d) if per_sample else (d,)
    w.update(ln_w=rn(*shape, scale=0.1, off=1.0), ln_b=rn(*shape, scale=0.1))
    return x, ctx, w, dout


# Chains of roundings: each of the about eight bf16 tensors between an input and a gradient is off by at
# most 2^-8 of its values, at random, so 3 u in the norm covers sqrt(8) of them; fp32 chains of matrix products
# over up to 260 terms lose some hundred units of 2^-24.
@pytest.mark.parametrize("dt,d,heads,tol", [(torch.bfloat16, 256, 2, 3 * 2.0 ** -8), (torch.float32, 256, 4, 1e-5)])
@pytest.mark.parametrize("per_sample,lens", [(False, None), (True, [77, 31]), (True, [0, 40])])
def test_cross_attention_and_gradients(dt, d, heads, tol, per_sample, lens):
    x, ctx, w, dout = _case(dt, d, 2, 130, 77, per_sample)
    kv_len = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, saved = T.cross_forward(x, ctx, w, heads, kv_len=kv_len)
    grads = T.cross_backward(x, ctx, w, saved, dout)
    want, ref = _reference(x, ctx, w, heads, lens, dout)
    rel = lambda a, b: float((a.to(F64) - b).norm() / b.norm())
    assert rel(out, want) < tol
    for name, r in ref.items():
        assert grads["d" + name].shape == r.shape, name
        assert rel(grads["d" + name], r) < tol, (name, rel(grads["d" + name], r))


def test_views_of_the_projections_are_taken_in_place():
    x, ctx, w, dout = _case(torch.bfloat16, 256, 2, 64, 77, False)
    _, saved = T.cross_forward(x, ctx, w, 2)
    assert saved["q"].transpose(1, 2).is_contiguous() and saved["o"].transpose(1, 2).is_contiguous()
    out = saved["o"].transpose(1, 2).reshape(2, 64, 256)
    assert out.data_ptr() == saved["o"].data_ptr()


@pytest.mark.parametrize("attn", ["rola", "dense"])
def test_dit_block_with_the_kernels_around(attn):
    """The same block in both settings: they differ by the roundings of the torch path (its probabilities and
    scores in bf16) and of the kernels."""
    shape = DB.DiTShape("tiny", 256, 2, 512, 1, 16, (3, 10, 13))
    x, ctx = DB.inputs(shape, seed=4)
    outs = [DB.DiTBlock(shape, attn=attn, block=64, sparsity=0.5, r=32, seed=3, around=a).forward(x, ctx)
            for a in ("torch", "rola")]
    a, b = (o.to(F64) for o in outs)
    assert float((a - b).norm() / a.norm()) < 2e-2
    with pytest.raises(ValueError):
        DB.DiTBlock(shape, around="other")


def test_captured_step():
    """A training step of the cross-attention in a graph while eager results of the same tensors live."""
    x, ctx, w, dout = _case(torch.bfloat16, 256, 2, 96, 77, True, seed=5)

    def step():
        out, saved = T.cross_forward(x, ctx, w, 2)
        return [out, *T.cross_backward(x, ctx, w, saved, dout).values()]

    eager = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        outs = step()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))
        x.copy_(torch.randn(x.shape, device="cuda"))
        eager = step()
        torch.cuda.synchronize()
