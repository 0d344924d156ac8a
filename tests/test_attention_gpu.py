"""Attention and its gradients on the GPU against the fp64 oracle, whose
elementwise error bounds are derived in oracle/attention_ref.py."""
import numpy as np
import pytest

from oracle import attention_ref as ref
from tests.gpu_util import require_gpu, to_bits, to_host

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def muon():
    require_gpu()
    from paper_2609_21594_amd.binding import Muon
    m = Muon(0)
    yield m
    m.close()


def tensor(rng, shape, dtype, size=1.0):
    import torch
    t = torch.from_numpy((rng.standard_normal(shape) * size).astype(np.float32)).cuda()
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def close(got, want, what):
    val, bound = want
    got = to_host(got).reshape(val.shape) if not isinstance(got, np.ndarray) else got
    if val.size == 0:
        return
    same = np.isneginf(val) & np.isneginf(got)
    assert np.isfinite(got[~same]).all(), what
    off = np.where(same, 0.0, np.abs(np.where(same, 0.0, got) - np.where(same, 0.0, val)))
    worst = np.unravel_index(np.argmax(off - bound), off.shape)
    assert (off <= bound + 1e-37).all(), (what, worst, got[worst], val[worst], bound[worst])


def saved(want, dtype):
    """What the forward pass leaves, from the oracle's results: (out, residual, lse)."""
    import torch
    o = torch.from_numpy(want["out"][0]).cuda()
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    out = o.to(t)
    res = (o - out.double()).to(torch.bfloat16) if dtype == "bf16" else None
    return out, res, torch.from_numpy(want["lse"][0]).float().cuda()


# batch, queries, keys, query heads, key heads, head size, causal, window
SHAPES = [
    (1, 1, 1, 1, 1, 8, False, 0),
    (2, 1, 33, 2, 1, 16, True, 0),
    (1, 2, 1, 2, 2, 64, True, 0),
    (1, 31, 31, 3, 3, 40, True, 0),
    (2, 33, 63, 4, 2, 64, False, 0),
    (1, 64, 64, 2, 2, 128, True, 0),
    (1, 65, 129, 4, 4, 72, True, 0),
    (1, 128, 128, 1, 1, 128, False, 0),
    (1, 129, 70, 2, 1, 64, True, 0),      # the first 59 queries see nothing
    (2, 200, 257, 6, 2, 80, True, 0),
    (1, 300, 300, 2, 1, 128, True, 7),
    (1, 257, 400, 2, 2, 64, True, 100),
    (1, 90, 90, 2, 2, 64, True, 1),       # each query its own key
    (1, 520, 515, 2, 1, 128, True, 0),
    (1, 140, 600, 8, 8, 32, False, 0),
    (1, 400, 40, 3, 1, 96, False, 0),
]
# few queries, many keys: the key axis is split, heads of a group share a tile
LONG = [
    (1, 1, 1500, 4, 1, 128, True, 0),
    (2, 1, 1025, 8, 2, 64, False, 0),
    (1, 5, 1300, 6, 2, 80, True, 0),
    (1, 17, 2100, 8, 1, 64, True, 0),     # 136 rows: more than one tile of 128
    (1, 40, 900, 1, 1, 128, True, 0),
    (1, 3, 513, 3, 1, 16, True, 0),
]


def make(case, dtype, size=1.0, seed=0):
    b, sq, sk, hq, hkv, d, causal, window = case
    rng = np.random.default_rng([seed, b, sq, sk, hq, hkv, d])
    return [tensor(rng, s, dtype, z) for s, z in (((b, sq, hq, d), size), ((b, sk, hkv, d), size), ((b, sk, hkv, d), 1.0),
                                                 ((b, sq, hq, d), 1.0))]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SHAPES + LONG, ids=str)
def test_forward(muon, case, dtype):
    import torch
    q, k, v, _ = make(case, dtype, 1.5)
    kw = dict(causal=case[6], window=case[7])
    want = ref.attention(*map(to_host, (q, k, v)), dtype, **kw)
    top = torch.full((case[3],), -INF, device="cuda")
    res = torch.full_like(q, NAN) if dtype == "bf16" else None
    out, lse = muon.attention(q, k, v, max_logits=top, residual=res, **kw)
    close(out, want["out"], "out")
    close(lse, want["lse"], "lse")
    close(top, want["top"], "top")
    if res is not None:
        # out and residual together lose 2^-16; the probabilities' rounding
        # (2^-8 of the weighted sizes) remains in both
        r, o = to_host(res), to_host(out)
        assert (np.abs(r) <= ref.HALF_STEP["bf16"] * np.abs(o + r) * (1 + 2.0 ** -7)).all()
    again, lse2 = muon.attention(q, k, v, **kw)
    assert np.array_equal(to_bits(again), to_bits(out)) and np.array_equal(to_bits(lse2), to_bits(lse))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", SHAPES + LONG[:3], ids=str)
def test_backward(muon, case, dtype):
    q, k, v, do = make(case, dtype, 1.5)
    kw = dict(causal=case[6], window=case[7])
    want = ref.attention(*map(to_host, (q, k, v)), dtype, dout=to_host(do), **kw)
    out, res, lse = saved(want, dtype)
    got = muon.attention_backward(do, q, k, v, out, lse, residual=res, **kw)
    for name, x in zip(("dq", "dk", "dv"), got):
        close(x, want[name], name)
    again = muon.attention_backward(do, q, k, v, out, lse, residual=res, **kw)
    for x, y in zip(got, again):
        assert np.array_equal(to_bits(x), to_bits(y))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_one_key_have_no_gradient(muon, dtype):
    for b, s, h, hk, d, window in ((3, 1, 4, 2, 72, 0), (1, 300, 2, 1, 128, 1), (2, 40, 3, 3, 16, 1)):
        q, k, v, do = make((b, s, s, h, hk, d, True, window), dtype)
        want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=True, window=window)
        out, res, lse = saved(want, dtype)   # out is the value row, bit for bit
        dq, dk, dv = muon.attention_backward(do, q, k, v, out, lse, residual=res, causal=True, window=window)
        assert not dq.any() and not dk.any() and dv.any()


def test_large_logits(muon):
    # logits of several hundred: one key takes nearly everything
    case = (1, 130, 130, 2, 2, 64, True, 0)
    for dtype in ("bf16", "f32"):
        q, k, v, do = make(case, dtype, 8.0)
        want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=True, dout=to_host(do))
        out, lse = muon.attention(q, k, v, causal=True)
        close(out, want["out"], "out")
        close(lse, want["lse"], "lse")
        o, res, l = saved(want, dtype)
        for name, x in zip(("dq", "dk", "dv"), muon.attention_backward(do, q, k, v, o, l, residual=res, causal=True)):
            close(x, want[name], name)


def test_without_residual_only_the_rounding_of_out_is_lost(muon):
    case = (1, 130, 130, 2, 2, 64, True, 0)
    q, k, v, do = make(case, "bf16", 1.0)
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", causal=True, dout=to_host(do))
    out, _, lse = saved(want, "bf16")
    dq, dk, dv = muon.attention_backward(do, q, k, v, out, lse, causal=True)
    # dout . out is off by up to 2^-8 sum |dout out|; that times p k (p q) goes into dq (dk)
    host = [to_host(x)[0] for x in (q, k, v, do)]
    for h in range(2):
        qh, kh, vh, dh = (x[:, h] for x in host)
        s = np.where(ref.visible(130, 130, True), 0.125 * qh @ kh.T, -np.inf)
        p = np.exp(s - want["lse"][0][0, h][:, None])
        extra = p * (2.0 ** -8 * (np.abs(dh) * np.abs(want["out"][0][0, :, h])).sum(1))[:, None]
        for name, got, more in (("dq", dq, 0.125 * extra @ np.abs(kh)), ("dk", dk, 0.125 * extra.T @ np.abs(qh))):
            val, bound = (x[0, :, h] for x in want[name])
            close(to_host(got)[0, :, h], (val, bound + more * (1 + 2.0 ** -7)), name)
    close(dv, want["dv"], "dv")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch_ignores_what_lies_behind_the_lengths(muon, dtype):
    import torch
    case = (5, 150, 140, 4, 2, 64, True, 0)
    q, k, v, do = make(case, dtype)
    nq, nk = [150, 1, 0, 77, 40], [140, 1, 64, 0, 90]
    want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=True, dout=to_host(do),
                         seqs=[(b, 0, nq[b], 0, nk[b]) for b in range(5)])
    out, res, lse = saved(want, dtype)
    for b in range(5):  # whatever padding holds
        for t in (q, do, out):
            t[b, nq[b]:] = NAN
        lse[b, :, nq[b]:] = NAN
        for t in (k, v):
            t[b, nk[b]:] = INF
    ql, kl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (nq, nk))
    top = torch.full((4,), -INF, device="cuda")
    o, l = muon.attention(q, k, v, causal=True, q_lens=ql, k_lens=kl, max_logits=top)
    close(o, want["out"], "out")
    close(l, want["lse"], "lse")
    close(top, want["top"], "top")
    got = muon.attention_backward(do, q, k, v, out, lse, residual=res, causal=True, q_lens=ql, k_lens=kl)
    for name, x in zip(("dq", "dk", "dv"), got):
        close(x, want[name], name)
    # lengths beyond the axes are cut to them, negative ones to 0
    ql2 = torch.tensor([1000, 1, -5, 77, 40], dtype=torch.int32, device="cuda")
    kl2 = torch.tensor([1 << 30, 1, 64, -(1 << 31), 90], dtype=torch.int32, device="cuda")
    o2, l2 = muon.attention(q, k, v, causal=True, q_lens=ql2, k_lens=kl2)
    assert np.array_equal(to_bits(o), to_bits(o2)) and np.array_equal(to_bits(l), to_bits(l2))


def test_padded_batch_of_single_tokens(muon):
    # the split of the key axis and the shared tile of a group, with lengths
    import torch
    case = (3, 2, 1200, 4, 2, 64, True, 0)
    q, k, v, _ = make(case, "bf16")
    nq, nk = [2, 1, 0], [1200, 700, 3]
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", causal=True, seqs=[(b, 0, nq[b], 0, nk[b]) for b in range(3)])
    ql, kl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (nq, nk))
    k[1, 700:] = NAN
    top = torch.full((4,), -INF, device="cuda")
    o, l = muon.attention(q, k, v, causal=True, q_lens=ql, k_lens=kl, max_logits=top)
    close(o, want["out"], "out")
    close(l, want["lse"], "lse")
    close(top, want["top"], "top")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 20)])
def test_packed_sequences_leave_other_rows_alone(muon, dtype, causal, window):
    import torch
    nq = [0, 130, 1, 0, 257, 3] + [2] * 70    # more sequences than a wave counts at once
    nk = [5, 130, 1, 4, 200, 0] + [3] * 70
    qo, ko = np.cumsum([7] + nq), np.cumsum([2] + nk)
    sq, sk = int(qo[-1]) + 9, int(ko[-1]) + 4
    q, k, v, do = make((1, sq, sk, 4, 2, 64, causal, window), dtype)
    seqs = [(0, int(a), n, int(b), m) for a, n, b, m in zip(qo, nq, ko, nk)]
    want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=causal, window=window, seqs=seqs, dout=to_host(do))
    out, res, lse = saved(want, dtype)
    off = [torch.from_numpy(x.astype(np.int32)).cuda() for x in (qo, ko)]
    kw = dict(causal=causal, window=window, q_offsets=off[0], k_offsets=off[1])
    q, k, v, do = (t[0] for t in (q, k, v, do))
    for t in (q, do, out[0]):                 # rows of no sequence
        t[:7] = NAN
        t[qo[-1]:] = NAN
    for t in (k, v):
        t[:2] = NAN
        t[ko[-1]:] = NAN
    top = torch.full((4,), -INF, device="cuda")
    o, l = muon.attention(q, k, v, max_logits=top, **kw)
    close(o, want["out"], "out")
    close(l, want["lse"], "lse")
    close(top, want["top"], "top")
    args = (do, q, k, v, out[0], lse[0])
    res = None if res is None else res[0]
    got = muon.attention_backward(*args, residual=res, **kw)
    for name, x in zip(("dq", "dk", "dv"), got):
        close(x, want[name], name)
    # results given by the caller: rows of no sequence stay as they were
    given = [torch.full_like(t, 3.0) for t in (q, q, k, v)]
    muon.attention(q, k, v, out=given[0], **kw)
    muon.attention_backward(*args, residual=res, dq=given[1], dk=given[2], dv=given[3], **kw)
    for t, like, lo, hi in zip(given, (o, *got), (7, 7, 2, 2), (qo[-1], qo[-1], ko[-1], ko[-1])):
        assert (t[:lo] == 3).all() and (t[hi:] == 3).all()
        assert np.array_equal(to_bits(t[lo:hi].contiguous()), to_bits(like[lo:hi].contiguous()))
    # offsets beyond the axis are cut to it
    far = off[0].clone()
    far[-1] = sq + 1000
    o3, _ = muon.attention(q, k, v, **dict(kw, q_offsets=far))
    assert o3.shape == o.shape


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["fused", "heads first", "padded rows"])
def test_strided_tensors(muon, dtype, layout):
    import torch
    b, sq, hq, hkv, d = 2, 133, 4, 2, 72
    q, k, v, do = make((b, sq, sq, hq, hkv, d, True, 0), dtype)
    want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=True, dout=to_host(do))
    out, res, lse = saved(want, dtype)

    def places(sizes):
        """Tensors [b, sq, n, d] in one buffer of the layout, filled with a mark."""
        if layout == "fused":
            buf = torch.full((b, sq, sum(sizes) + 1, d), 5.0, dtype=q.dtype, device="cuda")
            return buf, list(buf[:, :, :-1].split(sizes, 2))
        if layout == "heads first":
            buf = torch.full((sum(sizes) + 1, b, sq, d), 5.0, dtype=q.dtype, device="cuda")
            return buf, [x.permute(1, 2, 0, 3) for x in buf[:-1].split(sizes, 0)]
        buf = torch.full((b, sum(sizes) + 1, sq, d + 8), 5.0, dtype=q.dtype, device="cuda")
        return buf, [x.transpose(1, 2)[..., :d] for x in buf[:, :-1].split(sizes, 1)]
    _, (q2, k2, v2, do2, o2) = places([hq, hkv, hkv, hq, hq])
    for t, s in ((q2, q), (k2, k), (v2, v), (do2, do), (o2, out)):
        t.copy_(s)
    obuf, (o, r) = places([hq, hq])
    muon.attention(q2, k2, v2, causal=True, out=o, residual=r if dtype == "bf16" else None)
    close(o.contiguous(), want["out"], "out")
    gbuf, (dq, dk, dv) = places([hq, hkv, hkv])
    muon.attention_backward(do2, q2, k2, v2, o2, lse, residual=res, causal=True, dq=dq, dk=dk, dv=dv)
    for name, x in zip(("dq", "dk", "dv"), (dq, dk, dv)):
        close(x.contiguous(), want[name], name)
    # nothing outside the views was written
    o.fill_(5.0)
    r.fill_(5.0)
    for t in (dq, dk, dv):
        t.fill_(5.0)
    assert (obuf == 5).all() and (gbuf == 5).all()


def test_broadcast_keys_and_values(muon):
    import torch
    q, k, v, do = make((2, 70, 70, 4, 1, 64, True, 0), "bf16")
    kx, vx = k[:1].expand(2, -1, 4, -1), v[:1].expand(2, -1, 4, -1)
    want = ref.attention(*map(to_host, (q, kx, vx)), "bf16", causal=True, dout=to_host(do))
    out, lse = muon.attention(q, kx, vx, causal=True)
    close(out, want["out"], "out")
    o, res, l = saved(want, "bf16")
    got = muon.attention_backward(do, q, kx, vx, o, l, residual=res, causal=True)
    for name, x in zip(("dq", "dk", "dv"), got):
        assert x.is_contiguous()
        close(x, want[name], name)


def test_offsets_beyond_32_bits(muon):
    # keys and values 16 MiB a token apart, the second batch beyond 2^31 elements
    import torch
    d, tokens = 64, 140
    q, k, v, do = make((2, 96, tokens, 2, 1, d, True, 0), "bf16")
    step = 1 << 23
    big = torch.empty(2 * tokens * step, dtype=torch.bfloat16, device="cuda")
    place = [big.as_strided((2, tokens, 1, d), (tokens * step, step, d, 1), at) for at in (0, 4096, 8192, 12288)]
    assert tokens * step > 1 << 30 and big.numel() > 1 << 31
    place[0].copy_(k)
    place[1].copy_(v)
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", causal=True, dout=to_host(do))
    out, lse = muon.attention(q, place[0], place[1], causal=True)
    close(out, want["out"], "out")
    o, res, l = saved(want, "bf16")
    dq, dk, dv = muon.attention_backward(do, q, place[0], place[1], o, l, residual=res, causal=True, dk=place[2],
                                         dv=place[3])
    for name, x in (("dq", dq), ("dk", dk.contiguous()), ("dv", dv.contiguous())):
        close(x, want[name], name)


def test_empty_requests(muon):
    import torch
    z = lambda *s: torch.ones(*s, dtype=torch.bfloat16, device="cuda")
    out, lse = muon.attention(z(0, 4, 2, 64), z(0, 4, 2, 64), z(0, 4, 2, 64))
    assert out.shape == (0, 4, 2, 64)
    out, lse = muon.attention(z(2, 0, 2, 64), z(2, 4, 2, 64), z(2, 4, 2, 64))
    assert out.numel() == 0
    out, lse = muon.attention(z(2, 5, 2, 64), z(2, 0, 2, 64), z(2, 0, 2, 64))
    assert not out.any() and (lse == -INF).all()
    dq, dk, dv = muon.attention_backward(z(2, 5, 2, 64), z(2, 5, 2, 64), z(2, 0, 2, 64), z(2, 0, 2, 64), out, lse)
    assert not dq.any() and dk.numel() == 0
    e = z(2, 0, 2, 64)
    dq, dk, dv = muon.attention_backward(e, e, z(2, 70, 2, 64), z(2, 70, 2, 64), e, torch.empty(2, 2, 0, device="cuda"))
    assert not dk.any() and not dv.any()
    off = torch.zeros(1, dtype=torch.int32, device="cuda")  # no sequence at all
    out, lse = muon.attention(z(3, 2, 64), z(4, 2, 64), z(4, 2, 64), q_offsets=off, k_offsets=off)
    assert not out.any() and (lse == -INF).all()


def test_max_logits_accumulate_and_pass_over_nan(muon):
    import torch
    q, k, v, _ = make((1, 70, 70, 2, 2, 64, True, 0), "bf16")
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", causal=True)["top"]
    top = torch.tensor([1000.0, -1000.0], device="cuda")
    muon.attention(q, k, v, causal=True, max_logits=top)
    assert top[0] == 1000.0 and abs(float(top[1]) - want[0][1]) <= want[1][1]
    q[0, 3, 1] = NAN
    top.fill_(-INF)
    out, _ = muon.attention(q, k, v, causal=True, max_logits=top)
    assert torch.isfinite(top).all() and torch.isnan(out[0, 3, 1]).all() and torch.isfinite(out[0, :3]).all()
    # all logits negative
    q, k = torch.ones_like(q), -torch.ones_like(k)
    top.fill_(-INF)
    muon.attention(q, k, v, causal=True, max_logits=top)
    assert torch.equal(top.cpu(), torch.full((2,), -8.0))


def test_refusals_leave_buffers_alone(muon):
    import torch
    from paper_2609_21594_amd.binding import MuonError
    q, k, v, do = make((1, 70, 70, 4, 2, 64, True, 0), "bf16")
    out = torch.full_like(q, 3.0)
    for kw in (dict(window=5), dict(scale=-1.0), dict(scale=INF)):
        with pytest.raises(MuonError):
            muon.attention(q, k, v, out=out, **kw)
    with pytest.raises(MuonError, match="overlap"):
        muon.attention(q, k, v, out=q)
    with pytest.raises(MuonError, match="overlap"):
        muon.attention(q, k, v, out=out[:, :1].expand(1, 70, 4, 64))
    with pytest.raises(MuonError, match="aligned"):
        shifted = torch.empty(q.numel() + 1, dtype=q.dtype, device="cuda")[1:].view(q.shape)
        muon.attention(shifted, k, v, out=out)
    with pytest.raises(MuonError, match="head_dim"):
        muon.attention(q[..., :12].contiguous(), k[..., :12].contiguous(), v[..., :12].contiguous())
    with pytest.raises(ValueError):
        muon.attention(q.cpu(), k, v)
    with pytest.raises(ValueError):
        muon.attention(q, k, v, out=out[:, :5])
    with pytest.raises(ValueError):
        muon.attention(q, k, v, max_logits=torch.zeros(3, device="cuda"))
    with pytest.raises(ValueError):
        muon.attention_backward(do, q, k, v, out, torch.zeros(1, 4, 71, device="cuda"))
    with pytest.raises(ValueError):
        muon.attention_backward(do[:, :5], q, k, v, out, torch.zeros(1, 4, 70, device="cuda"))
    torch.cuda.synchronize()
    assert (out == 3).all()


@pytest.mark.parametrize("case", [(2, 70, 90, 2, 1, 16, False, 0), (1, 300, 300, 2, 2, 128, True, 0),
                                  (40, 65, 100, 16, 8, 64, False, 0)], ids=str)
def test_gradients_do_not_feel_the_rounding_of_lse(muon, case):
    """fp32: a step of lse (here 2^-18, lse being 40 to 64) would be a common
    factor 1 + 3.8e-6 of a row's probabilities.  They sum to 1 by themselves up
    to exp2's own 2^-23 and that of its argument near the maximum, so that
    gradients agree to a few 2^-23 of their norm.  A sum that lse itself puts
    elsewhere stays: half a unit more scales by exp(-1/2)."""
    import torch
    q, k, v, do = make(case, "f32", 2.0)
    scale = 3.0 / case[5] ** 0.5
    kw = dict(causal=case[6], scale=scale)
    out, lse = muon.attention(q, k, v, **kw)
    assert lse[:, :, -1].max() > 8
    ref_ = muon.attention_backward(do, q, k, v, out, lse, **kw)
    step = 2.0 ** -18
    near = muon.attention_backward(do, q, k, v, out, lse + step, **kw)
    far = muon.attention_backward(do, q, k, v, out, lse + 0.5, **kw)
    for x, y, z in zip(ref_, near, far):
        x, y, z = (t.double().cpu() for t in (x, y, z))
        assert (x - y).norm() <= 1e-6 * x.norm()
        assert (x * np.exp(-0.5) - z).norm() <= 2e-5 * x.norm()


@pytest.mark.parametrize("dtype,limit", [("bf16", 3 * 2.0 ** -8), ("f32", 1e-5)])
def test_gradients_of_a_part_of_the_keys(muon, dtype, limit):
    """lse and out of all keys: each part's dk and dv are those of the whole
    call, the parts' dq add up to its own.  bf16: probabilities and two results
    rounded, 2^-8 each."""
    import torch
    q, k, v, do = make((2, 150, 260, 4, 2, 64, False, 0), dtype, 1.5)
    res = torch.empty_like(q) if dtype == "bf16" else None
    out, lse = muon.attention(q, k, v, residual=res)
    whole = muon.attention_backward(do, q, k, v, out, lse, residual=res)
    cuts = (slice(0, 70), slice(70, 260))
    parts = [muon.attention_backward(do, q, k[:, c], v[:, c], out, lse, residual=res) for c in cuts]
    joined = (sum(p[0].double() for p in parts), *(torch.cat([p[i] for p in parts], 1).double() for i in (1, 2)))
    for x, y in zip(whole, joined):
        assert (x.double() - y).norm() <= limit * x.double().norm()
