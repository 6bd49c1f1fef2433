"""64-bit references of the norms and of the attention over another set of tokens, with bounds on what
rounding may add. u(t) = half a step of type t, relative; 2^-24 that of fp32, in which the kernels compute."""

import math

import torch

F64 = torch.float64
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
E32 = 2.0 ** -24


def norm(x, w, b, kind, eps=1e-6):
    """(y, xh, mu, rstd, bound on y); x [B, N, d], w and b broadcastable to it or None. A statistic is a sum
    of d terms added pairwise over lanes and waves after at most 32 in a row: 64 steps bound it, and its
    error reaches x - mu relative to the largest |x|."""
    u = U[x.dtype]
    x = x.to(F64)
    mu = x.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(x[..., :1])
    rstd = ((x - mu).square().mean(-1, keepdim=True) + eps).rsqrt()
    xh = (x - mu) * rstd
    w = torch.ones_like(x) if w is None else w.to(F64).expand_as(x)
    b = torch.zeros_like(x) if b is None else b.to(F64).expand_as(x)
    y = xh * w + b
    dxh = 64 * E32 * (xh.abs() + x.abs().amax(-1, keepdim=True) * rstd)
    return y, xh, mu, rstd, u * y.abs() + w.abs() * dxh + 4 * E32 * (y.abs() + b.abs()), dxh


def norm_grad(x, w, kind, dy, over, eps=1e-6):
    """(dx, dw, db) and their bounds; `over`: the dimensions that W's gradient is summed over. The sums over
    rows are at most 64 + rows / 64 steps of fp32 long."""
    u = U[x.dtype]
    _, xh, mu, rstd, _, dxh = norm(x, w, None, kind, eps)
    dy = dy.to(F64)
    wf = torch.ones_like(dy) if w is None else w.to(F64).expand_as(dy)
    g = dy * wf
    c2 = (g * xh).mean(-1, keepdim=True)
    c1 = g.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(c2)
    dx = rstd * (g - c1 - xh * c2)
    size = g.abs() + g.abs().mean(-1, keepdim=True) + xh.abs() * (g * xh).abs().mean(-1, keepdim=True)
    e = rstd * (64 * E32 * size + dxh * c2.abs() + xh.abs() * (g.abs() * dxh).mean(-1, keepdim=True))
    steps = (64 + dy.shape[0] * dy.shape[1] / 64) * E32
    dw, db = (dy * xh).sum(over), dy.sum(over)
    ew = (steps * (dy * xh).abs() + dy.abs() * dxh).sum(over)
    return (dx, dw, db), (u * dx.abs() + e, ew, steps * dy.abs().sum(over))


def attention(q, k, v, lens, causal, scale, do=None):
    """(o, lse[, dq, dk, dv]) and their bounds, [B, H, ...] with k, v [B, Hkv, ...]."""
    u, bf = U[q.dtype], q.dtype == torch.bfloat16
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1:3]
    G = H // Hkv
    q, k, v = (t.to(F64).reshape(B, -1, t.shape[2], d) for t in (q, k, v))
    do = None if do is None else do.to(F64)
    z = lambda *s: torch.zeros(s, dtype=F64, device=q.device)
    o, lse = z(B, H, Nq, d), torch.full((B, H, Nq), -math.inf, dtype=F64, device=q.device)
    eo, el = z(B, H, Nq, d), z(B, H, Nq)
    grads = [z(B, H, Nq, d), z(B, Hkv, Nk, d), z(B, Hkv, Nk, d)]
    errs = [torch.zeros_like(t) for t in grads]
    for b in range(B):
        n = Nk if lens is None else max(0, min(int(lens[b]), Nk))
        if n == 0:
            continue
        i = torch.arange(Nq, device=q.device).view(-1, 1)
        j = torch.arange(n, device=q.device)
        seen = j <= i + n - Nq if causal else torch.ones((Nq, n), dtype=torch.bool, device=q.device)
        rows = seen.any(-1)
        if not rows.any():
            continue
        for h in range(H):
            Q, K, V = q[b, h], k[b, h // G, :n], v[b, h // G, :n]
            s = torch.where(seen, scale * Q @ K.t(), torch.full((), -math.inf, dtype=F64, device=q.device))
            m = torch.where(rows, s.amax(-1), torch.zeros_like(s[:, 0])).unsqueeze(-1)
            p = torch.exp(s - m)
            l = p.sum(-1, keepdim=True)
            p = torch.where(rows.unsqueeze(-1), p / l, torch.zeros_like(p))
            o[b, h] = p @ V
            lse[b, h] = torch.where(rows, ((m + l.log()) / math.log(2)).squeeze(-1), lse[b, h])
            # a score: d products added in fp32; the exponent's argument rounds once more
            ds_ = (d + 8) * E32 * scale * (Q.abs() @ K.abs().t()).amax() + 8 * E32 * s[seen].abs().max()
            el[b, h] = 2 * ds_ / math.log(2) + (n + 64) * E32
            # a probability: twice a score's error (the denominator's too), the row sum's n additions, and
            # its rounding for the product
            r = 2 * ds_ + (n + 64) * E32 + (u if bf else 0.0)
            eo[b, h] = r * (p @ V.abs()) + u * o[b, h].abs()
            if do is None:
                continue
            dO = do[b, h]
            dp = dO @ V.t()
            D = (p * dp).sum(-1, keepdim=True)
            dS = p * (dp - D)
            # P's own error without its rounding; handed over as fp16 (2^-11) for dS, rounded for dV
            rp = 2 * ds_ + (n + 64) * E32
            edp = (d + 8) * E32 * (dO.abs() @ V.abs().t())
            eD = (dO.abs() * (eo[b, h] + d * E32 * o[b, h].abs())).sum(-1, keepdim=True)
            edS = p * (edp + eD) + (rp + (u + 2.0 ** -11 + 2.0 ** -24 if bf else 4 * E32)) * dS.abs()
            if bf:
                edS = edS + 2.0 ** -24 * (dp - D).abs()  # fp16 below its normal range: 2^-25 absolute
            grads[0][b, h] = scale * dS @ K
            grads[1][b, h // G, :n] += scale * dS.t() @ Q
            grads[2][b, h // G, :n] += p.t() @ dO
            sums = (n + Nq * G) * E32
            errs[0][b, h] = scale * (edS + sums * dS.abs()) @ K.abs()
            errs[1][b, h // G, :n] += scale * (edS + sums * dS.abs()).t() @ Q.abs()
            errs[2][b, h // G, :n] += (rp + sums + (u if bf else 0.0)) * p.t() @ dO.abs()
    if do is None:
        return (o, lse), (eo, el)
    return (o, lse, *grads), (eo, el, *(e + u * g.abs() for e, g in zip(errs, grads)))


def check(name, got, want, bound):
    """Every value within its bound; infinities equal."""
    got = got.detach().to(F64)
    same = (got == want) | ((got - want).abs() <= bound + 1e-30)
    assert bool(same.all()), (name, int((~same).sum()),
                              float(((got - want).abs() / (bound + 1e-30)).nan_to_num(math.inf)[~same].max()))
