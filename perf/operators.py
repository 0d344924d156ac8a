"""The attention block of a training step, as measured: rotary positions, attention with its
backward pass and each head's largest logit, and the clip of the query and key weights by it.

`own` selects what `run` does: False computes the operators in their plain form (elementary
torch operations in 32 bits, angles in 64, rounded once at the end), True makes the calls
that a user of the library makes (`Muon.rotary`, `Muon.attention`, `Muon.attention_backward`,
`Muon.qk_clip`).

A case is a dict of plain values.  `op` is one of
  rotary    the query and key heads of one layer turned by their positions
  forward   attention; outputs, log-sum-exps and, with `track`, each head's largest logit
  backward  the gradients of queries, keys and values
  clip      the query and key weights of `layers` layers
Attention is dense (`batch` sequences of `sq` queries and `sk` keys), padded (`lens`: every
sequence has a length of its own below that) or packed (`docs` sequences one behind the other
on one token axis of `sq` tokens).  `fused`: queries, keys and values are slices of one tensor.
"""
import functools
import math
import random

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}
INF = float("inf")
TAU = 20.0  # the clip's threshold


def _rotary(name=None, batch=1, s=1, q=32, kv=8, d=128, rot=128, layout="half", dtype="bf16", inverse=False, far=4096,
            factor=1.0):
    c = dict(op="rotary", batch=batch, s=s, q=q, kv=kv, d=d, rot=rot, layout=layout, dtype=dtype, inverse=inverse,
             far=far, factor=factor)
    return dict(c, name=name) if name else c


def _attention(op, name=None, batch=1, sq=1, sk=1, q=32, kv=8, d=128, dtype="bf16", causal=True, window=0, docs=0,
               lens=False, fused=False, track=False, size=1.0):
    c = dict(op=op, batch=batch, sq=sq, sk=sk, q=q, kv=kv, d=d, dtype=dtype, causal=causal, window=window, docs=docs,
             lens=lens, fused=fused, track=track, size=size)
    return dict(c, name=name) if name else c


def _clip(name=None, layers=1, q=32, kv=8, d=128, hidden=4096, hot=2, dtype="bf16"):
    c = dict(op="clip", layers=layers, q=q, kv=kv, d=d, hidden=hidden, hot=hot, dtype=dtype)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token of each of 8 sequences, far into their contexts: a call's latency
        _rotary("rotary-tokens", batch=8, s=1, far=131072, factor=4.0),
        # one layer's queries and keys of a long training sequence
        _rotary("rotary-layer-8k", s=8192, far=8192),
        # the gradient through a rotation of half of every head, neighbouring pairs, fp32, an odd length
        _rotary("rotary-part-gradient-f32", batch=2, s=2047, q=12, kv=12, d=96, rot=48, layout="interleaved",
                dtype="f32", inverse=True, far=32768, factor=8.0),
        # a small model's full attention over a short odd batch, fp32 throughout
        _attention("forward", "forward-short-f32", batch=3, sq=77, sk=77, q=12, kv=12, d=64, dtype="f32",
                   causal=False),
        # one layer of the 4096-wide model of the benchmark, grouped keys and values, its logits tracked
        _attention("forward", "forward-layer-4k", sq=4096, sk=4096, track=True),
        # a token looking back at a long context: few rows, many keys
        _attention("forward", "forward-token-16k", batch=4, sq=1, sk=16385),
        # documents packed on one axis, a sliding window, queries keys and values from one fused projection
        _attention("forward", "forward-packed-window", sq=8191, sk=8191, q=16, kv=16, d=64, window=1024, docs=11,
                   fused=True, track=True),
        # a small fp32 model's backward pass, shared heads
        _attention("backward", "backward-short-f32", batch=2, sq=129, sk=129, q=8, kv=4, d=64, dtype="f32"),
        # one layer of the 4096-wide model
        _attention("backward", "backward-layer-4k", sq=4096, sk=4096),
        # a padded batch of ragged sequences, heads of an odd width, larger logits
        _attention("backward", "backward-padded-ragged", batch=6, sq=1021, sk=1021, q=12, kv=12, d=80, lens=True,
                   size=2.0),
        # the clip of one layer of a small fp32 model: latency
        _clip("clip-layer-f32", q=12, kv=12, d=64, hidden=768, hot=3, dtype="f32"),
        # the clip of a whole 4096-wide model's queries and keys, a quarter of the heads above the threshold
        _clip("clip-model-h4096", layers=32),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    kv = rng.choice((1, 2, 4, 6, 8, 16))
    return kv * rng.choice([g for g in (1, 1, 2, 3, 4, 8) if kv * g <= 32]), kv


def draw(rng):
    op = rng.choice(("rotary", "forward", "forward", "backward", "backward", "clip"))
    q, kv = _heads(rng)
    d = rng.choice((16, 32, 64, 64, 72, 80, 96, 128, 128))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "rotary":
        batch, s = rng.choice(((_log_int(rng, 1, 64), 1), (rng.randint(1, 4), _log_int(rng, 2, 4096))))
        return _rotary(batch=batch, s=s, q=q, kv=kv, d=d, rot=2 * rng.randint(1, d // 2) if rng.random() < 0.4 else d,
                       layout=rng.choice(("half", "interleaved")), dtype=dtype, inverse=rng.random() < 0.5,
                       far=_log_int(rng, 4096, 1000000), factor=rng.choice((1.0, 4.0, 32.0)))
    if op == "clip":
        layers = _log_int(rng, 1, 24)
        return _clip(layers=layers, q=q, kv=kv, d=d, hidden=_log_int(rng, 64, 4096), hot=rng.randint(0, kv),
                     dtype=dtype)
    form = rng.choice(("dense", "dense", "lens", "docs", "token" if op == "forward" else "dense"))
    causal = rng.random() < 0.7
    window = _log_int(rng, 16, 2048) if causal and rng.random() < 0.25 else 0
    opts = dict(q=q, kv=kv, d=d, dtype=dtype, causal=causal, window=window, fused=False, track=op == "forward" and
                rng.random() < 0.5, size=rng.choice((0.5, 1.0, 2.0)))
    if form == "token":
        return _attention(op, batch=_log_int(rng, 1, 16), sq=rng.choice((1, 1, 2, 5)), sk=_log_int(rng, 64, 16384),
                          **opts)
    if form == "docs":
        s = _log_int(rng, 64, 4096)
        return _attention(op, sq=s, sk=s, docs=rng.randint(1, 12), **dict(opts, fused=rng.random() < 0.5))
    batch, s = rng.randint(1, 4), _log_int(rng, 1, 2048 if dtype == "bf16" else 1500)
    if form == "lens":
        return _attention(op, batch=batch, sq=s, sk=s, lens=True, **dict(opts, fused=rng.random() < 0.5))
    sk = s if rng.random() < 0.7 else _log_int(rng, max(1, s // 2), 2 * s)
    return _attention(op, batch=batch, sq=s, sk=sk, **dict(opts, fused=sk == s and rng.random() < 0.5))


def _lengths(case):
    """(query, key) lengths of every sequence, from the case alone."""
    rng = random.Random(1000 * case["sq"] + 10 * case["batch"] + case["docs"])
    if case["docs"]:
        cuts = sorted(rng.randint(0, case["sq"]) for _ in range(case["docs"] - 1))
        lens = [b - a for a, b in zip([0] + cuts, cuts + [case["sq"]])]
        return lens, lens
    if case["lens"]:
        lens = [rng.randint((case["sq"] + 3) // 4, case["sq"]) for _ in range(case["batch"])]
        return lens, lens
    return [case["sq"]] * case["batch"], [case["sk"]] * case["batch"]


def _pairs(case):
    """Visible (query, key) pairs of all sequences, for one head."""
    total = 0
    for nq, nk in zip(*_lengths(case)):
        if not case["causal"]:
            total += nq * nk
            continue
        for i in range(nq):
            last = min(nk - 1, i + nk - nq)
            first = max(0, i + nk - nq - case["window"] + 1) if case["window"] else 0
            total += max(0, last - first + 1)
    return total


def work(case):
    es = ES[case["dtype"]]
    if case["op"] == "rotary":
        n = case["batch"] * case["s"] * (case["q"] + case["kv"])
        return {"bytes": 2.0 * n * case["d"] * es, "flops": 3.0 * n * case["rot"]}
    if case["op"] == "clip":
        group = case["q"] // case["kv"]
        n = case["layers"] * case["hot"] * (group + 1) * case["d"] * case["hidden"]
        return {"bytes": 2.0 * n * es + 4.0 * case["layers"] * case["q"], "flops": float(n)}
    nq, nk = (sum(x) for x in _lengths(case))
    rows, cols = nq * case["q"] * case["d"] * es, nk * case["kv"] * case["d"] * es
    flops = float(_pairs(case)) * case["q"] * case["d"]
    if case["op"] == "forward":
        return {"bytes": 2.0 * rows + 2.0 * cols + 4.0 * nq * case["q"], "flops": 4 * flops}
    return {"bytes": 4.0 * rows + 4.0 * cols + 4.0 * nq * case["q"], "flops": 10 * flops}


def _frequencies(rot, factor):
    """Radians a position of each pair, in 64 bits: base 10000, positions interpolated by `factor`."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    return (10000.0 ** (-2.0 * i / rot) / factor).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape, size=1.0, dtype=DTYPE[case["dtype"]]):
        return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)

    st = {"case": case}
    if case["op"] == "rotary":
        st["q"] = normal(case["batch"], case["s"], case["q"], case["d"])
        st["k"] = normal(case["batch"], case["s"], case["kv"], case["d"])
        start = torch.randint(0, max(1, case["far"] - case["s"] + 1), (case["batch"], 1), generator=g, device="cuda")
        st["positions"] = start + torch.arange(case["s"], device="cuda")
        st["freqs"] = _frequencies(case["rot"], case["factor"])
        st["scale"] = 1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0
        return st
    if case["op"] == "clip":
        rows_q, rows_k = case["q"] * case["d"], case["kv"] * case["d"]
        st["wq"] = [normal(rows_q, case["hidden"], size=0.02) for _ in range(case["layers"])]
        st["wk"] = [normal(rows_k, case["hidden"], size=0.02) for _ in range(case["layers"])]
        # `hot` groups of heads of every layer have logits above the threshold, the others below
        m = torch.rand(case["layers"], case["kv"], case["q"] // case["kv"], generator=g, device="cuda")
        hot = torch.rand(case["layers"], case["kv"], generator=g, device="cuda").argsort(-1) < case["hot"]
        m = torch.where(hot[..., None], TAU * (1.001 + 4 * m), TAU * (0.999 * m))
        st["logits"] = list(m.reshape(case["layers"], case["q"]).unbind(0))
        return st
    shape = (case["sq"],) if case["docs"] else (case["batch"], case["sq"])
    kshape = (case["sk"],) if case["docs"] else (case["batch"], case["sk"])
    if case["fused"]:
        x = normal(*shape, case["q"] + 2 * case["kv"], case["d"], size=case["size"])
        st["q"], st["k"], st["v"] = x.split([case["q"], case["kv"], case["kv"]], dim=-2)
    else:
        st["q"] = normal(*shape, case["q"], case["d"], size=case["size"])
        st["k"] = normal(*kshape, case["kv"], case["d"], size=case["size"])
        st["v"] = normal(*kshape, case["kv"], case["d"])
    nq, nk = _lengths(case)
    if case["docs"]:
        ends = torch.tensor([0] + nq, device="cuda").cumsum(0).to(torch.int32)
        st["where"] = {"q_offsets": ends, "k_offsets": ends}
    elif case["lens"]:
        lens = torch.tensor(nq, device="cuda", dtype=torch.int32)
        st["where"] = {"q_lens": lens, "k_lens": lens}
    else:
        st["where"] = {}
    if case["op"] == "backward":
        # what the forward pass left: outputs, what their rounding took from them, log-sum-exps
        out, lse, _ = _plain_forward(st)
        st["out"], st["lse"] = out.to(DTYPE[case["dtype"]]), lse
        st["residual"] = (out - st["out"].float()).to(torch.bfloat16) if case["dtype"] == "bf16" else None
        st["dout"] = normal(*shape, case["q"], case["d"])
    return st


# ---------------------------------------------------------------- the plain forms

def _turn(x, cos, sin, case):
    """The rotation of x [batch, s, heads, d], in 32 bits."""
    x32, rot = x.float(), case["rot"]
    if case["layout"] == "half":
        a, b = x32[..., : rot // 2], x32[..., rot // 2: rot]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), -1)
    else:
        a, b = x32[..., 0:rot:2], x32[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2)
    return torch.cat((turned, x32[..., rot:]), -1).to(x.dtype)


def _plain_rotary(st):
    case = st["case"]
    angle = st["positions"].double()[..., None, None] * st["freqs"]
    cos, sin = (st["scale"] * angle.cos()).float(), (st["scale"] * angle.sin()).float()
    sin = -sin if case["inverse"] else sin
    return _turn(st["q"], cos, sin, case), _turn(st["k"], cos, sin, case)


def _visible(st):
    """[batch or 1, sq, sk]: which key each query sees."""
    case, where = st["case"], st["where"]
    i, j = torch.arange(case["sq"], device="cuda")[:, None], torch.arange(case["sk"], device="cuda")[None, :]
    if case["docs"]:
        ends = where["q_offsets"].long()
        doc_i = torch.searchsorted(ends, i.contiguous(), right=True)
        doc_j = torch.searchsorted(ends, j.contiguous(), right=True)
        see, shift = (doc_i == doc_j)[None], 0
    elif case["lens"]:
        lens = where["q_lens"].long()[:, None, None]
        see, shift = (i < lens) & (j < lens), 0
    else:
        see, shift = torch.ones(1, case["sq"], case["sk"], dtype=torch.bool, device="cuda"), case["sk"] - case["sq"]
    if case["causal"]:
        see = see & (j <= i + shift)
        if case["window"]:
            see = see & (i + shift - j < case["window"])
    return see


def _grouped(x, case):
    """[.., s, heads, d] as fp32 [batch, kv, heads // kv, s, d]."""
    x = x.float() if x.dim() == 4 else x.float()[None]
    return x.permute(0, 2, 1, 3).reshape(x.shape[0], case["kv"], -1, x.shape[1], x.shape[3])


def _plain_logits(st, q, k):
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(st["case"]["d"])
    return s.masked_fill(~_visible(st)[:, None, None], -INF)


def _tokens(x, like):
    """Back from [batch, kv, group, s, d] to the layout of `like`."""
    return x.flatten(1, 2).permute(0, 2, 1, 3).reshape(*like.shape[:-2], -1, like.shape[-1]).contiguous()


def _plain_forward(st):
    case = st["case"]
    q, k, v = (_grouped(st[x], case) for x in "qkv")
    s = _plain_logits(st, q, k)
    top = s.amax(-1, keepdim=True)
    p = (s - top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.clamp(min=torch.finfo(torch.float32).tiny)
    lse = (top + total.log()).squeeze(-1).flatten(1, 2)
    lse = lse[0] if case["docs"] else lse
    return _tokens(out, st["q"]), lse, top.flatten(1, 2).amax((0, 2, 3))


def _plain_backward(st):
    case = st["case"]
    q, k, v, do = (_grouped(st[x], case) for x in ("q", "k", "v", "dout"))
    s = _plain_logits(st, q, k)
    p = (s - s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
    p = p / p.sum(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).tiny)
    dp = torch.matmul(do, v.transpose(-1, -2))
    ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(case["d"])
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(2, keepdim=True)
    dv = torch.matmul(p.transpose(-1, -2), do).sum(2, keepdim=True)
    return tuple(_tokens(x, st[y]).to(st[y].dtype) for x, y in ((dq, "q"), (dk, "k"), (dv, "v")))


def _plain_clip(st):
    case = st["case"]
    m = torch.stack(st["logits"]).reshape(case["layers"], case["kv"], -1)
    gamma = torch.where(m > TAU, TAU / m, torch.ones_like(m))
    key = gamma.amin(-1, keepdim=True).sqrt()
    for_q, for_k = (x.flatten(1).repeat_interleave(case["d"], 1)[..., None] for x in (gamma / key, key))
    wq, wk = torch.stack(st["wq"]), torch.stack(st["wk"])
    wq, wk = (wq.float() * for_q).to(wq.dtype), (wk.float() * for_k).to(wk.dtype)
    torch._foreach_copy_(st["wq"] + st["wk"], list(wq.unbind(0)) + list(wk.unbind(0)))


@functools.lru_cache(maxsize=None)
def _muon():
    """The library handle of a program's process."""
    from paper_2609_21594_amd.binding import Muon
    return Muon(torch.cuda.current_device())


def run(st):
    case = st["case"]
    if case["op"] == "rotary":
        if not own:
            q, k = _plain_rotary(st)
        else:
            q, k = _muon().rotary([st["q"], st["k"]], st["freqs"], positions=st["positions"],
                                     layout=case["layout"], scale=st["scale"], inverse=case["inverse"])
        return {"q": q, "k": k}
    if case["op"] == "forward":
        if not own:
            out, lse, top = _plain_forward(st)
            out = out.to(st["q"].dtype)
        else:
            top = torch.full((case["q"],), -INF, device="cuda") if case["track"] else None
            out, lse = _muon().attention(st["q"], st["k"], st["v"], causal=case["causal"], window=case["window"],
                                            max_logits=top, **st["where"])
        return {"out": out, "lse": lse, "top": top} if case["track"] else {"out": out, "lse": lse}
    if case["op"] == "backward":
        if not own:
            dq, dk, dv = _plain_backward(st)
        else:
            dq, dk, dv = _muon().attention_backward(st["dout"], st["q"], st["k"], st["v"], st["out"], st["lse"],
                                                       residual=st["residual"], causal=case["causal"],
                                                       window=case["window"], **st["where"])
        return {"dq": dq, "dk": dk, "dv": dv}
    if not own:
        _plain_clip(st)
    else:
        _muon().qk_clip(st["wq"], st["wk"], st["logits"], TAU)
    # three layers stand for all: a case's outputs are few
    pick = sorted({0, case["layers"] // 2, case["layers"] - 1})
    return {"wq": [st["wq"][i] for i in pick], "wk": [st["wk"][i] for i in pick]}


# ---------------------------------------------------------------- the definitions, in 64 bits

def _exact_rotary(st, x):
    case, x = st["case"], x.double()
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
    freq = torch.exp(-math.log(10000.0) * 2 * i / case["rot"]) / case["factor"]
    angle = st["positions"].double()[..., None] * freq
    turn = torch.polar(torch.full_like(angle, st["scale"]), -angle if case["inverse"] else angle)[:, :, None]
    out = x.clone()
    n = case["rot"] // 2
    re, im = (slice(0, n), slice(n, 2 * n)) if case["layout"] == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    z = torch.complex(x[..., re].contiguous(), x[..., im].contiguous()) * turn
    out[..., re], out[..., im] = z.real, z.imag
    return out


def _exact_sequence(st, q, k, v, dout):
    """One sequence of one head: outputs, log-sum-exps, the largest logit and, with dout, the
    gradients of sum(out * dout)."""
    case = st["case"]
    back = dout is not None
    q, k, v = (x.double().requires_grad_(back) for x in (q, k, v))
    s = q @ k.T / math.sqrt(case["d"])
    if case["causal"]:
        gap = torch.arange(len(q), device="cuda")[:, None] + len(k) - len(q) - torch.arange(len(k), device="cuda")
        hidden = (gap < 0) | (gap >= case["window"]) if case["window"] else gap < 0
        s = s.masked_fill(hidden, -INF)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse.masked_fill(lse == -INF, 0.0)[:, None])
    out = p @ v
    grads = torch.autograd.grad((out * dout.double()).sum(), (q, k, v)) if back else None
    top = s.detach().max() if s.numel() else torch.tensor(-INF, dtype=torch.float64, device="cuda")
    return out.detach(), lse.detach(), top, grads


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rotary":
        return {"q": _exact_rotary(st, st["q"]), "k": _exact_rotary(st, st["k"])}
    if case["op"] == "clip":
        pick, group = sorted({0, case["layers"] // 2, case["layers"] - 1}), case["q"] // case["kv"]
        wq, wk = [], []
        for layer in pick:
            a, b = st["wq"][layer].double(), st["wk"][layer].double()
            m = st["logits"][layer].tolist()
            for g in range(case["kv"]):
                gamma = [min(1.0, TAU / m[g * group + h]) if m[g * group + h] > 0 else 1.0 for h in range(group)]
                b[g * case["d"]:(g + 1) * case["d"]] *= math.sqrt(min(gamma))
                for h in range(group):
                    row = (g * group + h) * case["d"]
                    a[row:row + case["d"]] *= gamma[h] / math.sqrt(min(gamma))
            wq.append(a)
            wk.append(b)
        return {"wq": wq, "wk": wk}
    nq, nk = _lengths(case)
    group, back = case["q"] // case["kv"], case["op"] == "backward"
    full = [st[x] if st[x].dim() == 4 else st[x][None] for x in "qkv"] + ([st["dout"].view(-1, *st["dout"].shape[-3:])]
                                                                         if back else [])
    q, k, v = full[:3]
    out, dk, dv = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (q, k, v))
    dq = torch.zeros_like(out)
    lse = torch.full((q.shape[0], case["q"], q.shape[1]), -INF, dtype=torch.float64, device="cuda")
    top = torch.full((case["q"],), -INF, dtype=torch.float64, device="cuda")
    at = 0
    for n in range(len(nq)):
        b, i, j = (0, at, at) if case["docs"] else (n, 0, 0)
        at += nq[n]
        if not nq[n] or not nk[n]:
            continue
        for h in range(case["q"]):
            rows, keys = (b, slice(i, i + nq[n]), h), (b, slice(j, j + nk[n]), h // group)
            o, l, t, grads = _exact_sequence(st, q[rows], k[keys], v[keys], full[3][rows] if back else None)
            out[rows], lse[b, h, i:i + nq[n]], top[h] = o, l, torch.maximum(top[h], t)
            if back:
                dq[rows] = grads[0]
                dk[keys] += grads[1]
                dv[keys] += grads[2]
    if back:
        return {x: y.view(st[x[1]].shape) for x, y in (("dq", dq), ("dk", dk), ("dv", dv))}
    got = {"out": out.view(st["q"].shape), "lse": lse[0] if case["docs"] else lse}
    return dict(got, top=top) if case["track"] else got
