"""Forward and backward of the module for fine-tuning (Sec. 4.5: P_q, P_k, W_g, b_g are trained jointly
with the backbone), composed from the library's entry points.

forward() keeps what the backward needs: the rotated Q^r, K^r (Algorithm step 3), the block lists,
O^s with its per-query log-sum-exp, and the summary C. backward() runs the low-rank/fusion backward
(which also yields dO^s and the gate-logit gradient), the block-sparse attention backward, and maps
dQ^r, dK^r back through the backbone rotation (R(p)^T = R(-p)); the two branches' shares of dQ^n,
dK^n and dV are added. Every step, the additions included, runs in the library's kernels.

cross_forward() and cross_backward() do the same for the block's text cross-attention beside the module: layer
norm of the hidden states, projections (library GEMMs), RMS norm of q and k, attention over each sample's text
tokens, output projection. q, k, v and their gradients stay views of the projections' rows: nothing is transposed.
"""

from __future__ import annotations

import torch

from . import rola as R


def forward(Qn, Kn, V, Pq, Pk, logits, grid, split, block=64, sparsity=0.9, r=32, base=10000.0):
    prob = R.problem_of(Qn, grid)
    cos, sin = R.rola_rope_tables(prob, split, base)
    # the rotation fused with the selection's pooling: bitwise rola_rope_apply and rola_block_select
    qr, qbar = R.rola_rope_pool(Qn, cos, sin, grid, block)
    kr, kbar = R.rola_rope_pool(Kn, cos, sin, grid, block)
    idx = R.rola_block_select_pooled(qbar, kbar, kr, grid, block, sparsity)
    os_, lse = R.rola_sparse_attn_lse(qr, kr, V, grid, block, sparsity, idx)
    C, _ = R.rola_lowrank_summary(Kn, V, Pk, r, cos, sin, grid, want_z=False)
    out = R.rola_lowrank_readout_combine(Qn, Pq, r, cos, sin, C, os_, logits, grid)
    saved = dict(cos=cos, sin=sin, qr=qr, kr=kr, idx=idx, os=os_, lse=lse, C=C, grid=grid,
                 block=block, sparsity=sparsity, r=r)
    return out, saved


def backward(Qn, Kn, V, Pq, Pk, logits, saved, dO):
    """Gradients of <dO, O>: dict of dQn, dKn, dV (fp32 [B, H, N, d]), dPq, dPk (fp32 [H, r, d]) and
    dlogits (fp32 [B, N])."""
    g, r = saved["grid"], saved["r"]
    cos, sin = saved["cos"], saved["sin"]
    dOs, dQn, dKn, dV, dPq, dPk, dlog = R.rola_lowrank_backward(
        Qn, Kn, V, Pq, Pk, r, cos, sin, saved["C"], saved["os"], logits, dO, g)
    # dQ^n += R(p)^T dQ^r, dK^n += R(p)^T dK^r, dV += the sparse branch's share
    R.rola_sparse_attn_backward_accumulate(saved["qr"], saved["kr"], V, g, saved["block"],
                                           saved["sparsity"], saved["idx"], saved["os"], saved["lse"],
                                           dOs, cos, sin, dQn, dKn, dV)
    return dict(dQn=dQn, dKn=dKn, dV=dV, dPq=dPq, dPk=dPk, dlogits=dlog)


def cross_forward(x, ctx, w, heads, kv_len=None, eps=1e-6):
    """Text cross-attention: x [B, N, d] hidden states, ctx [B, L, d] text tokens, kv_len (int32 [B], on the
    device) the valid ones per sample. w: dict of the layer norm's ln_w, ln_b ([d], or [B, d] per sample;
    None for neither), the projections Wq, Wk, Wv, Wo [d, d] and the RMS norms' nq, nk [d]. Returns
    (out [B, N, d], what cross_backward takes)."""
    B, N, d = x.shape
    L = ctx.shape[1]
    h, mean, rstd = R.rola_norm(x, w["ln_w"], w["ln_b"], kind="layer", eps=eps, want_stats=True)
    q0, k0, v = h @ w["Wq"].t(), ctx @ w["Wk"].t(), ctx @ w["Wv"].t()
    qn, _, rq = R.rola_norm(q0, w["nq"], kind="rms", eps=eps, want_stats=True)
    kn, _, rk = R.rola_norm(k0, w["nk"], kind="rms", eps=eps, want_stats=True)
    q, k, vh = (t.view(B, n, heads, d // heads).transpose(1, 2) for t, n in ((qn, N), (kn, L), (v, L)))
    o, lse = R.rola_attn(q, k, vh, kv_len=kv_len)
    out = o.transpose(1, 2).reshape(B, N, d) @ w["Wo"].t()
    saved = dict(h=h, mean=mean, rstd=rstd, q0=q0, k0=k0, rq=rq, rk=rk, q=q, k=k, v=vh, o=o, lse=lse,
                 kv_len=kv_len)
    return out, saved


def cross_backward(x, ctx, w, saved, dout):
    """Gradients of <dout, out>: dict of dx, dctx in the inputs' type, the projections' dWq, dWk, dWv, dWo in
    theirs, and the norms' dln_w, dln_b, dnq, dnk in fp32."""
    s = saved
    B, N, d = x.shape

    def rows(t):
        return t.reshape(-1, t.shape[-1])

    def merged(t):  # [B, heads, n, d_h] -> [B, n, d], a view when the heads lie inside the tokens
        return t.transpose(1, 2).reshape(B, t.shape[2], d)

    g = {}
    heads = s["q"].shape[1]
    g["dWo"] = rows(dout).t() @ rows(merged(s["o"]))
    do = (dout @ w["Wo"]).view(B, N, heads, d // heads).transpose(1, 2)
    dq, dk, dv = R.rola_attn_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], do, kv_len=s["kv_len"])
    dq0, g["dnq"], _ = R.rola_norm_backward(s["q0"], w["nq"], None, s["rq"], merged(dq), kind="rms",
                                            want_bias=False)
    dk0, g["dnk"], _ = R.rola_norm_backward(s["k0"], w["nk"], None, s["rk"], merged(dk), kind="rms",
                                            want_bias=False)
    dv = merged(dv)
    g["dWq"], g["dWk"], g["dWv"] = (rows(a).t() @ rows(b) for a, b in ((dq0, s["h"]), (dk0, ctx), (dv, ctx)))
    g["dctx"] = dk0 @ w["Wk"] + dv @ w["Wv"]
    per_sample = w["ln_w"] is not None and w["ln_w"].dim() == 2
    g["dx"], g["dln_w"], g["dln_b"] = R.rola_norm_backward(x, w["ln_w"], s["mean"], s["rstd"], dq0 @ w["Wq"],
                                                           kind="layer", per_sample=per_sample)
    return g
