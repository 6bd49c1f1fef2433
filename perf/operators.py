"""Performance cases of the operators around the attention module: layer and RMS norm, and softmax attention
of one set of tokens over another, each with its gradients.

A case is a dict of plain values: its kind and its sizes and options. Kinds:

  norm        rola_norm alone.
  norm_train  rola_norm and, from the output's gradient, rola_norm_backward.
  attn        rola_attn alone.
  attn_train  rola_attn and, from the output's gradient, rola_attn_backward.

With `own` false the same operators are computed in their plain form, elementary torch operations in 32 bits.

Sizes: the tiny fp32 layer, single tokens over a cache of a 480p video's length, one latent frame over the
frames before it, text cross-attention (512 text tokens) of the Wan-shaped 480p and 720p layers, dense self
attention of the 8400-token grid, ragged batches between them; hidden sizes 128 to 5120.
"""

import math

import torch

own = False  # whether run() makes the framework's calls

EPS = 1e-6
LOG2E = math.log2(math.e)
F32, F64 = torch.float32, torch.float64
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attn(name, kind, B, H, Hkv, Nq, Nk, d=128, dtype="bf16", causal=False, lens="full", packed=True):
    case = dict(name=name, kind=kind, B=B, H=H, Hkv=Hkv, Nq=Nq, Nk=Nk, d=d, dtype=dtype, causal=causal,
                lens=lens, packed=packed)
    if name is None:
        del case["name"]
    return case


def _norm(name, kind, B, N, d, norm="layer", dtype="bf16", wdtype="f32", per_sample=False, bias=True,
          packed=1):
    case = dict(name=name, kind=kind, B=B, N=N, d=d, norm=norm, dtype=dtype, wdtype=wdtype,
                per_sample=per_sample, bias=bias, packed=packed)
    if name is None:
        del case["name"]
    return case


def listed():
    return [
        # the smallest call: the RMS norm of one token's queries, launch-bound
        _norm("norm-one-token", "norm", 1, 1, 1536, norm="rms", wdtype="bf16", bias=False),
        # the modulated layer norm before the attention of the 14B-shaped 720p model
        _norm("norm-720p", "norm", 1, 75600, 5120),
        # the modulated layer norm of a 480p training step, two samples with their own modulation
        _norm("norm-train-480p", "norm_train", 2, 32760, 1536, per_sample=True),
        # the RMS norm of the queries inside a packed projection, an odd frame size
        _norm("norm-train-packed-odd", "norm_train", 1, 17 * 37 * 61, 1536, norm="rms", wdtype="bf16",
              bias=False, packed=3),
        # the attention of the fp32 layer used to bring a model up and check it
        _attn("attn-tiny-f32", "attn", 1, 2, 2, 256, 256, d=64, dtype="f32", packed=False),
        # one new token per sample over a cache as long as a 480p video, five query heads per key head
        _attn("attn-token-cache", "attn", 8, 40, 8, 1, 32760, lens="ragged", packed=False),
        # one latent frame of a causal video model over itself and the 20 frames before it
        _attn("attn-frame-causal", "attn", 1, 12, 12, 1560, 32760, causal=True, packed=False),
        # text cross-attention of the 14B-shaped 720p model
        _attn("attn-text-720p", "attn", 1, 40, 40, 75600, 512),
        # text cross-attention of a 480p training step, prompts padded to 512 tokens
        _attn("train-text-480p", "attn_train", 2, 12, 12, 32760, 512, lens="ragged"),
        # dense self attention of the 8400-token grid with its gradients: the teacher of the sparse module
        _attn("train-self-8400", "attn_train", 1, 12, 12, 8400, 8400, packed=False),
        # a padded causal batch with shared key heads; two samples have fewer keys than queries
        _attn("train-causal-grouped-odd", "attn_train", 3, 8, 2, 1111, 1337, causal=True, lens="ragged"),
        # the fp32 path of a gradient check at odd sizes
        _attn("train-f32-odd", "attn_train", 2, 4, 4, 777, 333, d=64, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    """Seconds-like measure that orders cases: matrix work of fp32 counts sixteen times bf16's."""
    w = work(case)
    return w["flops"] * (16 if case["dtype"] == "f32" and "H" in case else 1) / 1e15 + w["bytes"] / 5e12


def draw(rng):
    """One more case of the same ranges."""
    while True:
        kind = rng.choice(["norm", "norm_train", "attn", "attn_train"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        if kind.startswith("norm"):
            d = 8 * _log(rng, 8, 640)
            norm = rng.choice(["layer", "rms"])
            case = _norm(None, kind, rng.choice([1, 1, 2, 3]), _log(rng, 1, 75600), d, norm=norm,
                         dtype=dtype, wdtype=rng.choice([dtype, "f32"]), per_sample=rng.random() < 0.5,
                         bias=rng.random() < 0.5, packed=rng.choice([1, 1, 3]))
        else:
            Hkv = rng.choice([1, 2, 4, 5, 8, 12])
            H = Hkv * rng.choice([1, 1, 2, 5])
            causal = rng.random() < 0.3
            if kind == "attn" and rng.random() < 0.4:  # few queries over a cache
                Nq, Nk = _log(rng, 1, 64), _log(rng, 256, 32760)
            else:
                Nq, Nk = _log(rng, 16, 32760), _log(rng, 16, 8400)
            case = _attn(None, kind, rng.choice([1, 1, 2, 4]), H, Hkv, Nq, Nk,
                         d=rng.choice([64, 128]) if dtype == "f32" else 128, dtype=dtype, causal=causal,
                         lens=rng.choice(["full", "ragged"]), packed=rng.random() < 0.5)
        if _cost(case) <= max(_cost(c) for c in listed() if ("H" in c) == ("H" in case)):
            return case


def _lens(case):
    """Keys per sample: all of them, or from all down to a seventh of them."""
    B, Nk = case["B"], case["Nk"]
    if case["lens"] == "full":
        return None
    return [max(1, Nk - (Nk * 6 * b) // (7 * max(1, B - 1)) - (b % 2)) if B > 1 else max(1, Nk - Nk // 3)
            for b in range(B)]


def _pairs(case):
    """Visible (query, key) pairs of one head, over the batch."""
    total = 0
    for n in _lens(case) or [case["Nk"]] * case["B"]:
        Nq = case["Nq"]
        if not case["causal"]:
            total += Nq * n
        else:  # query i sees max(0, n - Nq + i + 1) keys
            first = max(0, Nq - n)
            rows = Nq - first
            total += rows * (n - Nq + first + 1 + n) // 2
    return total


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"].startswith("norm"):
        rows, d = case["B"] * case["N"], case["d"]
        train = case["kind"] == "norm_train"
        wrows = case["B"] if case["per_sample"] else 1
        we = 2 if case["wdtype"] == "bf16" else 4
        params = wrows * d * (1 + case["bias"])
        nbytes = rows * d * e * (4 if train else 2) + params * (we + (4 if train else 0))
        return {"bytes": nbytes, "flops": rows * d * (20 if train else 8)}
    B, H, Hkv, Nq, d = case["B"], case["H"], case["Hkv"], case["Nq"], case["d"]
    keys = sum(_lens(case) or [case["Nk"]] * B)
    train = case["kind"] == "attn_train"
    # Q, O (and dO, dQ) once, K, V (and dK, dV, whole) once, the log-sum-exp
    nbytes = B * H * Nq * d * e * (4 if train else 2) + 2 * keys * Hkv * d * e + B * H * Nq * 4
    if train:
        nbytes += 2 * B * case["Nk"] * Hkv * d * e
    return {"bytes": nbytes, "flops": _pairs(case) * H * d * (14 if train else 4)}


def _tokens(gen, shape, dt, spread):
    """Rows as a q/k norm leaves them: unit RMS, drawn around a few directions (softmax rows are spiky)."""
    B, H, N, d = shape
    centres = torch.randn((8, d), generator=gen, device="cuda")
    which = torch.randint(0, 8, (B, H, N), generator=gen, device="cuda")
    x = torch.randn(shape, generator=gen, device="cuda") + spread * centres[which]
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True))).to(dt)


def _placed(x, packed):
    """The tensor as the path has it: [B, H, N, d] contiguous, or a view of the packed [B, N, H d]."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if packed else x


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    state = {"case": case}
    if case["kind"].startswith("norm"):
        B, N, d, wdt = case["B"], case["N"], case["d"], DTYPE[case["wdtype"]]
        # hidden states with a mean and a few strong channels
        x = randn(B, N, d * case["packed"])
        x *= 1 + 3 * (torch.rand((d * case["packed"],), generator=gen, device="cuda") < 0.02)
        x += 0.3 * randn(B, 1, d * case["packed"])
        wshape = (B, d) if case["per_sample"] else (d,)
        state["x"] = x.to(dt)[..., :d]
        state["w"] = (1 + 0.1 * randn(*wshape)).to(wdt)
        state["b"] = (0.1 * randn(*wshape)).to(wdt) if case["bias"] else None
        if case["kind"] == "norm_train":
            state["dy"] = randn(B, N, d).to(dt)
        return state
    B, H, Hkv, Nq, Nk, d = (case[k] for k in ("B", "H", "Hkv", "Nq", "Nk", "d"))
    centre_seed = torch.Generator(device="cuda").manual_seed(seed)  # q and k share their directions
    state["q"] = _placed(_tokens(centre_seed, (B, H, Nq, d), dt, 0.7), case["packed"])
    centre_seed.manual_seed(seed)
    state["k"] = _placed(_tokens(centre_seed, (B, Hkv, Nk, d), dt, 0.7), case["packed"])
    state["v"] = _placed(randn(B, Hkv, Nk, d).to(dt), case["packed"])
    lens = _lens(case)
    state["lens"] = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    if case["kind"] == "attn_train":
        state["do"] = _placed(randn(B, H, Nq, d).to(dt), case["packed"])
    return state


# ---- the framework's calls ------------------------------------------------------------------------

def _run_own(state):
    from paper_2609_06712_amd import rola as R
    case = state["case"]
    if case["kind"].startswith("norm"):
        x, w, b = state["x"], state["w"], state["b"]
        train = case["kind"] == "norm_train"
        y, mean, rstd = R.rola_norm(x, w, b, kind=case["norm"], eps=EPS, want_stats=train)
        if not train:
            return (y,)
        dx, dw, db = R.rola_norm_backward(x, w, mean, rstd, state["dy"], kind=case["norm"],
                                          want_bias=b is not None)
        return (y, dx, dw) if b is None else (y, dx, dw, db)
    q, k, v, lens = state["q"], state["k"], state["v"], state["lens"]
    o, lse = R.rola_attn(q, k, v, kv_len=lens, causal=case["causal"])
    if case["kind"] == "attn":
        return o, lse
    dq, dk, dv = R.rola_attn_backward(q, k, v, o, lse, state["do"], kv_len=lens, causal=case["causal"])
    return o, lse, dq, dk, dv


# ---- the plain forms ------------------------------------------------------------------------------

def _rows(w, x):
    """A weight [d] or [B, d] against x [B, N, d]."""
    return w.float() if w.dim() == 1 else w.float().unsqueeze(1)


def _plain_norm(state):
    case, dt = state["case"], state["x"].dtype
    x = state["x"].float()
    if case["norm"] == "layer":
        x = x - x.mean(-1, keepdim=True)
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh = x * rstd
    w = _rows(state["w"], x)
    y = xh * w
    if state["b"] is not None:
        y = y + _rows(state["b"], x)
    y = y.to(dt)
    if case["kind"] == "norm":
        return (y,)
    dy = state["dy"].float()
    g = dy * w
    dx = g - xh * (g * xh).mean(-1, keepdim=True)
    if case["norm"] == "layer":
        dx = dx - g.mean(-1, keepdim=True)
    dx = (dx * rstd).to(dt)
    over = (1,) if state["w"].dim() == 2 else (0, 1)
    dw = (dy * xh).sum(over)
    return (y, dx, dw) if state["b"] is None else (y, dx, dw, dy.sum(over))


def _hidden(case, lens):
    """True where a query may not see a key: [B, 1, 1 or Nq, Nk], or None."""
    Nq, Nk = case["Nq"], case["Nk"]
    if lens is None and not case["causal"]:
        return None
    j = torch.arange(Nk, device="cuda")
    n = torch.full((case["B"],), Nk, device="cuda") if lens is None else lens
    n = n.view(-1, 1, 1, 1)
    hidden = j >= n
    if case["causal"]:
        i = torch.arange(Nq, device="cuda").view(-1, 1)
        hidden = hidden | (j > i + n - Nq)
    return hidden


def _plain_attn(state):
    case, dt = state["case"], state["q"].dtype
    B, H, Hkv, Nq, Nk, d = (case[k] for k in ("B", "H", "Hkv", "Nq", "Nk", "d"))
    G, scale = H // Hkv, d ** -0.5

    def grouped(t):  # the query heads of a key head beside each other
        return t.float().reshape(B, Hkv, G * Nq, d)

    def split(t):
        return t.view(B, Hkv, G, Nq, Nk)

    q, k, v = grouped(state["q"]), state["k"].float().contiguous(), state["v"].float().contiguous()
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale
    hidden = _hidden(case, state["lens"])
    if hidden is not None:
        split(s).masked_fill_(hidden.unsqueeze(2), -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)  # rows that see no key
    p = torch.exp(s - m)
    del s
    l = p.sum(-1, keepdim=True)
    lse = ((m + torch.log(l)) * LOG2E).view(B, H, Nq)
    p = p / torch.where(l == 0, torch.ones_like(l), l)
    o = torch.matmul(p, v)
    out = o.view(B, H, Nq, d).to(dt)
    if case["kind"] == "attn":
        return out, lse
    do = grouped(state["do"])
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    dp = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = p * (dp - (do * o).sum(-1, keepdim=True)) * scale
    del dp, p
    dq = torch.matmul(ds, k).view(B, H, Nq, d)
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q)
    return out, lse, dq.to(dt), dk.to(dt), dv.to(dt)


def run(state):
    if own:
        return _run_own(state)
    return _plain_norm(state) if state["case"]["kind"].startswith("norm") else _plain_attn(state)


# ---- the definition in 64 bits --------------------------------------------------------------------

def _exact_norm(case, state):
    """Sample by sample; the gradients by differentiation of the definition."""
    train = case["kind"] == "norm_train"
    w0 = state["w"].to(F64).requires_grad_(train)
    b0 = None if state["b"] is None else state["b"].to(F64).requires_grad_(train)
    leaves = [w0] + ([b0] if b0 is not None else [])
    ys, dxs, sums = [], [], None
    for n in range(case["B"]):
        x = state["x"][n].to(F64).requires_grad_(train)
        w = w0 if w0.dim() == 1 else w0[n]
        b = b0 if b0 is None or b0.dim() == 1 else b0[n]
        if case["norm"] == "layer":
            var, mu = torch.var_mean(x, dim=-1, unbiased=False, keepdim=True)
        else:
            var, mu = (x ** 2).mean(-1, keepdim=True), 0.0
        y = w * ((x - mu) / torch.sqrt(var + EPS))
        y = y if b is None else y + b
        ys.append(y.detach())
        if train:
            g = torch.autograd.grad(y, [x] + leaves, state["dy"][n].to(F64))
            dxs.append(g[0])
            sums = list(g[1:]) if sums is None else [a + c for a, c in zip(sums, g[1:])]
    return (torch.stack(ys),) + ((torch.stack(dxs), *sums) if train else ())


def _exact_attn(case, state):
    """Head by head over the keys that exist; the gradients by differentiation of the definition."""
    B, H, Hkv, Nq, Nk, d = (case[k] for k in ("B", "H", "Hkv", "Nq", "Nk", "d"))
    train = case["kind"] == "attn_train"
    dev = "cuda"
    o = torch.zeros((B, H, Nq, d), dtype=F64, device=dev)
    lse = torch.full((B, H, Nq), -math.inf, dtype=F64, device=dev)
    dq = torch.zeros_like(o)
    dk = torch.zeros((B, Hkv, Nk, d), dtype=F64, device=dev)
    dv = torch.zeros_like(dk)
    for b, n in enumerate(_lens(case) or [Nk] * B):
        first = max(0, Nq - n) if case["causal"] else 0  # earlier queries see no key
        if first == Nq or n == 0:
            continue
        for h in range(H):
            q = state["q"][b, h, first:].to(F64).requires_grad_(train)
            k = state["k"][b, h * Hkv // H, :n].to(F64).requires_grad_(train)
            v = state["v"][b, h * Hkv // H, :n].to(F64).requires_grad_(train)
            s = (q @ k.t()) / math.sqrt(d)
            if case["causal"]:
                past = torch.ones(s.shape, dtype=torch.bool, device=dev).tril(n - Nq + first)
                s = torch.where(past, s, torch.full_like(s, -math.inf))
            a = torch.softmax(s, dim=-1) @ v
            o[b, h, first:] = a.detach()
            lse[b, h, first:] = torch.logsumexp(s.detach(), -1) / math.log(2.0)
            if train:
                g = torch.autograd.grad(a, (q, k, v), state["do"][b, h, first:].to(F64))
                dq[b, h, first:] = g[0]
                dk[b, h * Hkv // H, :n] += g[1]
                dv[b, h * Hkv // H, :n] += g[2]
    return (o, lse, dq, dk, dv) if train else (o, lse)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"].startswith("norm"):
        return _exact_norm(case, state)
    if work(case)["flops"] > 8e12:  # beyond about 20 seconds in 64 bits
        return None
    return _exact_attn(case, state)
