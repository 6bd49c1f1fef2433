"""Norm-wise bounds on the bf16 attention of tests/_around.py, beside its bounds on single values: those add up every
rounding's worst case over a row or a key, so that what grows like a root (roundings are independent) is allowed to
grow like the count. Here they add as squares.

A rounding to bf16 is off by at most U = 2^-8 of the value; over values of all mantissas m the error is uniform
within a half-step, so its mean square is U^2 / 3 times the mean of 1 / m^2 = 3 / (8 ln 2): RMS = 0.425 U.
What is rounded: every result once; P for O and dV; dS for dK, from a P that is off by half a step of fp16 or by
half of that type's least step over 2^15; dS in two terms (U^2) for dQ.

D is an fp32 sum over a row's n keys, and its error d_i is the same for all of them, so dQ_i is off by
d_i scale |sum_j P_ij K_j|, and dK_j by the d_i scale P_ij |Q_i| of independent rows. In units of 2^-24 of sum_j P |dP|, which no partial sum exceeds: a lane adds half a row's
terms one after the other, n / 2 roundings of at most one unit each; the probabilities' sum adds eight at a time,
n / 16; the log-sum-exp is rounded at |lse| 2^-24, ln 2 times that in P; the scores, exp2 and the last sums 16. That
is the bound for one row (where one key holds most of it, each of the others may round the same way: an emulation
of the sum in fp32 is off by up to 654 units at 8400 keys, the bound being about 4760). Over all rows the roundings are
independent: sqrt(n / 2) and sqrt(n / 16) for the sums, the others as before.
"""

import math

import torch

F64 = torch.float64
U, U16, E32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24
RMS = math.sqrt(0.125 / math.log(2.0))
NAMES = ("o", "dq", "dk", "dv")


def reference(q, k, v, lens, causal, scale, do):
    """{name: (value, squared error of each of its rows from what was rounded within, the same from D at its worst and
    over all rows)}, the errors in units of U^2. q, do [B, H, Nq, d], k and v [B, Hkv, Nk, d]."""
    B, H, Nq, d = q.shape
    Hkv, Nk = k.shape[1:3]
    G = H // Hkv
    q, k, v, do = (t.to(F64) for t in (q, k, v, do))
    val = dict(o=torch.zeros_like(q), dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(k))
    err = {n: torch.zeros(x.shape[:-1], dtype=F64, device=q.device) for n, x in val.items()}
    worst, usual = ({n: torch.zeros_like(x) for n, x in err.items()} for _ in range(2))
    sq = lambda x: x.square().sum(-1)
    for b in range(B):
        n = Nk if lens is None else lens[b]
        i = torch.arange(Nq, device=q.device).view(-1, 1)
        seen = (torch.arange(n, device=q.device) <= i + n - Nq) | (not causal)
        assert bool(seen.any(-1).all())  # (rows without a key: the bounds on single values)
        for h in range(H):
            Q, K, V, dO, g = q[b, h], k[b, h // G, :n], v[b, h // G, :n], do[b, h], h // G
            s = (scale * Q @ K.t()).masked_fill(~seen, -math.inf)
            p = torch.softmax(s, -1)
            dp = dO @ V.t()
            D = (p * dp).sum(-1, keepdim=True)
            ds = scale * p * (dp - D)
            val["o"][b, h], err["o"][b, h] = p @ V, p.square() @ sq(V)
            val["dq"][b, h] = ds @ K
            err["dq"][b, h] = (U * ds).square() @ sq(K)
            unit = E32 / U * scale * (p * dp.abs()).sum(-1)
            rest, sums = torch.logsumexp(s, -1).abs() + 16, n / 2 + n / 16
            for to, units in ((worst, (sums + rest).square()), (usual, sums + rest.square())):
                d2 = units * unit.square()
                to["dq"][b, h] = d2 * sq(p @ K)
                to["dk"][b, g, :n] += p.square().t() @ (d2 * sq(Q))
            val["dk"][b, g, :n] += ds.t() @ Q
            low = 2.0 ** -40 * scale * (dp - D)
            err["dk"][b, g, :n] += ((1 + U16 / U) * ds).square().t() @ sq(Q) + (low / U).square().t() @ sq(Q)
            val["dv"][b, g, :n] += p.t() @ dO
            err["dv"][b, g, :n] += p.square().t() @ sq(dO)
    return {name: (val[name], err[name], worst[name], usual[name]) for name in val}


def excess(got, ref):
    """(error of the whole tensor, error of the worst row), each over its bound.
    Whole: independent roundings at their root mean square, and a quarter above.
    A row of d_h values: the roundings within at their worst (few of them may carry the row); its own d_h
    independent ones at 0.75 U, where 0.425 U is their root mean square and the norm of 128 of them strays by a tenth."""
    want, err, worst, usual = ref
    diff = got.detach().to(F64) - want
    own = want.square().sum(-1)
    whole = 1.25 * RMS * U * float((own + err + usual).sum()) ** 0.5
    row = U * (0.75 ** 2 * own + err + worst).sqrt() + 1e-30
    return float(diff.norm()) / whole, float((diff.norm(dim=-1) / row).max())


def check(got, ref):
    for name, x in got.items():
        whole, row = excess(x, ref[name])
        assert whole <= 1 and row <= 1, (name, whole, row)


def inputs(kind, B, H, Hkv, Nq, Nk, seed=0, d=128, device="cpu"):
    """q, k, v, do in bf16. "plain": independent values. "offset": the keys, and the values, have a part in common,
    which dQ must cancel. "sink": one key per key head takes all but about a thousandth of every row."""
    gen = torch.Generator().manual_seed(seed)
    rn = lambda *s: torch.randn(s, generator=gen)
    q, k, v, do = rn(B, H, Nq, d), rn(B, Hkv, Nk, d), rn(B, Hkv, Nk, d), rn(B, H, Nq, d)
    if kind == "offset":
        k += 2 * rn(B, Hkv, 1, d)
        v += 2 * rn(B, Hkv, 1, d)
    if kind == "sink":
        c = rn(d)
        c /= c.norm()
        q += 8 * c  # the score of the sink: ln Nk + 1/2, the other keys' log-sum-exp, and 7 above
        k[:, :, Nk // 3] = c * (math.log(Nk) + 7.5) * d ** 0.5 / 8
    return [t.to(torch.bfloat16).to(device) for t in (q, k, v, do)]
