"""Attention requests at values where rounding or the order of sums shows, and at
values that are not finite, on every way that a launch can take."""
import numpy as np
import pytest

from oracle import attention_ref as ref
from tests.gpu_util import to_bits, to_host
from tests.test_attention_gpu import close, make, muon, tensor  # noqa: F401

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


# one part, parts of one token and of a group's heads, parts of many queries
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 70, 70, 4, 2, 64, True, 0), (1, 1, 1500, 4, 1, 128, True, 0),
                                  (2, 3, 1100, 6, 2, 80, False, 0), (1, 200, 4100, 4, 2, 128, True, 0)], ids=str)
def test_a_query_that_is_no_number_stays_none(muon, case, dtype):  # noqa: F811
    import torch
    q, k, v, _ = make(case, dtype)
    kw = dict(causal=case[6])
    row = (case[0] - 1, case[1] // 2, 1)
    want = ref.attention(*map(to_host, (q, k, v)), dtype, **kw)
    q[row][3] = NAN
    top = torch.full((case[3],), -INF, device="cuda")
    res = torch.zeros_like(q) if dtype == "bf16" else None
    out, l = muon.attention(q, k, v, max_logits=top, residual=res, **kw)
    lse = l.transpose(1, 2)
    assert torch.isnan(out[row]).all() and torch.isnan(lse[row])
    assert res is None or torch.isnan(res[row]).all()
    # the other rows are as without it
    other = np.ones((case[0], case[1], case[3]), dtype=bool)
    other[row] = False
    close(to_host(out)[other], tuple(x[other] for x in want["out"]), "out")
    close(to_host(lse)[other], tuple(x.transpose(0, 2, 1)[other] for x in want["lse"]), "lse")
    # NaN raises no largest logit: a head whose only row that is has none
    assert np.array_equal(np.isfinite(to_host(top)), other.any(axis=(0, 1)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_that_are_no_numbers_reach_every_row_that_sees_them(muon, dtype):  # noqa: F811
    """Whatever part of a split key axis they fill: one key, some of a part's, all
    of one part's (which then has no maximum) or of several."""
    import torch
    q, k, v, _ = make((1, 1, 1500, 4, 1, 128, True, 0), dtype)
    for n in (1, 64, 128, 320, 384, 640, 1024, 1500):
        for lo in range(0, 1500 - n + 1, 64):
            bad = k.clone()
            bad[:, lo:lo + n, :, 7] = NAN
            out, lse = muon.attention(q, bad, v, causal=True)
            assert torch.isnan(out).all() and torch.isnan(lse).all(), (n, lo)


@pytest.mark.parametrize("heads,d", [(16, 8), (8, 72), (1, 8), (1, 72)], ids=str)
def test_rows_of_equal_probabilities_sum_to_one(muon, heads, d):  # noqa: F811
    """fp32, logits all 0: one query on n keys has p = 1 / n, and dv of a gradient of
    ones is p.  The gradient pass normalises rows by their own sums, so that what is
    left of a common factor is those sums' rounding, in half steps of 2^-24: 4 for 16
    values by pairs, 2 for the steps with their carries, 1 for the halves of a wave, 3
    for up to four waves a row; 1 each for the reciprocal, its product with p, and
    dv's product and its sum with zeros."""
    import torch
    b, s = 64, 1600
    nk = torch.linspace(200, 1598, b).to(torch.int32).cuda()   # odd and even, whole tiles and not
    one = torch.ones_like(nk)
    rng = np.random.default_rng(4)
    q = torch.zeros(b, 1, heads, d, device="cuda")
    k, v = (torch.from_numpy(rng.standard_normal((b, s, heads, d)).astype(np.float32)).cuda() for _ in "kv")
    out, lse = muon.attention(q, k, v, q_lens=one, k_lens=nk)
    _, _, dv = muon.attention_backward(torch.ones_like(q), q, k, v, out, lse, q_lens=one, k_lens=nk)
    for i, n in enumerate(nk.tolist()):
        off = (dv[i, :n].double() * n - 1).abs().max()
        assert off <= 14 * 2.0 ** -24, (n, float(off))
        assert not dv[i, n:].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 70, 70, 2, 2, 64, True, 0), (1, 2, 1500, 4, 1, 128, False, 0)], ids=str)
def test_infinite_values_reach_the_rows_that_see_them(muon, case, dtype):  # noqa: F811
    """As infinity or NaN."""
    import torch
    q, k, v, _ = make(case, dtype)
    at = case[2] // 2
    v[0, at, :, 5] = INF
    out, lse = muon.attention(q, k, v, causal=case[6])
    seen = out[0, at if case[6] else 0:, :, 5]
    assert not torch.isfinite(seen).any()
    rest = torch.arange(case[5], device="cuda") != 5
    assert torch.isfinite(out[..., rest]).all() and torch.isfinite(lse).all()


def seen_keys(nq, nk, causal, window):
    """(first, last) key of each query."""
    i = np.arange(nq)
    last = np.minimum(nk - 1, i + nk - nq) if causal else np.full(nq, nk - 1)
    return np.maximum(0, i + nk - nq - window + 1) if causal and window else np.zeros(nq, dtype=int), last


# batch, queries, keys, query heads, key heads, head size, causal, window, lengths of queries and keys
ONE_KEY = [
    (3, 1, 1, 4, 2, 72, True, 0, None),
    (1, 300, 300, 2, 1, 128, True, 1, None),
    (2, 40, 40, 3, 3, 16, True, 1, None),
    (2, 200, 1, 4, 4, 64, False, 0, None),
    (4, 130, 130, 4, 2, 96, True, 0, None),                                  # the first query alone
    (2, 70, 33, 2, 2, 32, True, 0, None),
    (40, 150, 150, 4, 4, 64, True, 1, None),                                 # one plane
    (3, 1, 1500, 4, 1, 128, True, 0, ([1, 1, 0], [1, 1500, 1])),             # parts, heads of a group in a tile
    (2, 5, 900, 4, 4, 80, False, 0, ([5, 3], [1, 900])),
    (2, 200, 4100, 4, 2, 64, True, 0, ([200, 150], [100, 1])),               # parts of many queries
    (8, 2050, 130, 8, 8, 128, True, 1, ([2050, 1, 0, 5, 600, 7, 8, 9], [130, 1, 4, 0, 130, 7, 8, 9])),  # 8 waves
    (0, 260, 200, 4, 2, 64, True, 0, ([1, 130, 0, 129], [1, 130, 3, 66])),   # packed
    (0, 70, 70, 2, 2, 40, False, 0, ([1] * 70, [1] * 70)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", ONE_KEY, ids=str)
def test_rows_that_see_one_key_have_its_value_and_no_gradient(muon, case, dtype):  # noqa: F811
    """From the library's own results, logits well above 1: out is the value row bit
    for bit, and every dS of the row is exactly 0."""
    import torch
    b, sq, sk, hq, hkv, d, causal, window, lens = case
    q, k, v, do = make((max(1, b), sq, sk, hq, hkv, d, causal, window), dtype, 3.0)
    kw = dict(causal=causal, window=window)
    if b:
        nq, nk = lens or ([sq] * b, [sk] * b)
        seqs = [(n, 0, x, 0, y) for n, (x, y) in enumerate(zip(nq, nk))]
        if lens:
            kw.update((n, torch.tensor(x, dtype=torch.int32, device="cuda")) for n, x in (("q_lens", nq), ("k_lens", nk)))
    else:
        qo, ko = (np.cumsum([0] + list(x)) for x in lens)
        seqs = [(0, int(i), x, int(j), y) for i, x, j, y in zip(qo, lens[0], ko, lens[1])]
        q, k, v, do = (t[0] for t in (q, k, v, do))
        kw.update((n, torch.from_numpy(x.astype(np.int32)).cuda()) for n, x in (("q_offsets", qo), ("k_offsets", ko)))
    res = torch.full_like(q, NAN) if dtype == "bf16" else None
    out, lse = muon.attention(q, k, v, residual=res, **kw)
    dq, dk, dv = muon.attention_backward(do, q, k, v, out, lse, residual=res, **kw)
    row = (lambda t, n: t[n]) if b else (lambda t, n: t)
    value = v.repeat_interleave(hq // hkv, -2)
    rows = 0
    for n, i, x, j, y in seqs:
        first, last = seen_keys(x, y, causal, window)
        at = np.flatnonzero(first == last)
        rows += len(at)
        mine, theirs = torch.from_numpy(i + at).cuda(), torch.from_numpy(j + first[at]).cuda()
        assert np.array_equal(to_bits(row(out, n)[mine]), to_bits(row(value, n)[theirs])), n
        assert not row(dq, n)[mine].any(), n
        assert res is None or not row(res, n)[mine].any(), n
        lone = np.setdiff1d(first[at], [c for f, l in zip(first, last) if l > f for c in range(f, l + 1)])
        assert not row(dk, n)[torch.from_numpy(j + lone).cuda()].any(), n
    assert rows and dv.any()


@pytest.mark.parametrize("case", [(2, 1, 1000, 4, 2, 64, True, 0), (1, 200, 200, 2, 2, 64, True, 50),
                                  (1, 90, 40, 2, 1, 64, True, 0), (1, 90, 40, 2, 1, 64, True, 7),
                                  (1, 30, 70, 2, 2, 64, True, 50), (1, 30, 70, 2, 2, 64, True, 10),
                                  (3, 30, 70, 2, 2, 64, False, 0)], ids=str)
def test_profile_counts_visible_pairs(muon, case):  # noqa: F811
    b, sq, sk, hq, _, d, causal, window = case
    q, k, v, do = make(case, "bf16")
    kw = dict(causal=causal, window=window)
    muon.profile(True)
    out, lse = muon.attention(q, k, v, **kw)
    muon.attention_backward(do, q, k, v, out, lse, **kw)
    got = muon.profile_read()
    muon.profile(False)
    pairs = b * hq * int(ref.visible(sq, sk, causal, window).sum())
    assert got["attention_forward"]["flops"] == 4 * pairs * d
    assert got["attention_backward"]["flops"] == 10 * pairs * d


def test_profile_leaves_captured_calls_out(muon):  # noqa: F811
    import torch
    from paper_2609_21594_amd.attention import rotary_frequencies
    q, k, v, do = make((1, 40, 40, 2, 2, 64, True, 0), "bf16")
    freqs = rotary_frequencies(64).cuda()
    w = [torch.ones(128, 8, device="cuda") for _ in range(2)]
    top = torch.zeros(2, device="cuda")

    def work():
        a, b = muon.rotary([q, k], freqs)
        out, lse = muon.attention(a, b, v, causal=True)
        grads = muon.attention_backward(do, a, b, v, out, lse, causal=True)
        muon.qk_clip([w[0]], [w[1]], [top], 1.0)
        return [out, *grads]
    eager = work()
    torch.cuda.synchronize()
    muon.profile(True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = work()
    for _ in range(3):
        for t in res:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(res, eager):
            assert np.array_equal(to_bits(x), to_bits(y))
    names = ("rotary", "attention_forward", "attention_backward", "qk_clip")
    got = muon.profile_read()
    assert all(got[n]["launches"] == 0 for n in names)
    work()
    got = muon.profile_read()
    muon.profile(False)
    assert all(got[n]["launches"] == 1 and got[n]["total_ms"] > 0 for n in names)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_gradients_of_any_alignment(muon, dtype):  # noqa: F811
    """Broadcast, sliced off their alignment and transposed ones, as autograd hands them over."""
    import torch
    from paper_2609_21594_amd.attention import rotary, rotary_frequencies
    rng = np.random.default_rng(9)
    freqs = rotary_frequencies(14).cuda()
    x, wide, do = (tensor(rng, (2, 37, 3, n), dtype) for n in (20, 21, 20))
    for g in (do, do[:, :1, :1].expand(2, 37, 3, 20), wide[..., 1:], do.transpose(2, 3).contiguous().transpose(2, 3)):
        leaf = x.clone().requires_grad_()
        rotary(muon, leaf, freqs, scale=1.5).backward(g)
        close(leaf.grad, ref.rotary(to_host(g.contiguous()), np.broadcast_to(np.arange(37), (2, 37)), freqs.cpu().numpy(),
                                    dtype, scale=1.5, inverse=True), "gradient")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", [1e2, 1e3, 1e4])
def test_one_key_far_above_the_others(muon, dtype, size):  # noqa: F811
    """Logits of the size of diverged weights: out is that key's value, its dv the sum
    of dout up to P's own rounding (two bf16 terms, 2^-16; fp32 2^-24), lse's (a
    factor up to exp(2^-23 |lse|); fp32: divided out), the result's and that of a sum
    of 20 rows."""
    import torch
    nq, n, d = 20, 70, 16
    q, _, v, do = make((1, nq, n, 1, 1, d, False, 0), dtype)
    k = torch.zeros_like(v)
    q.zero_()
    q[..., 0] = 1
    k[0, :, 0, 0] = torch.linspace(-1, 0.5, n, device="cuda").to(k.dtype) * size
    k[0, 35, 0, 0] = 1.0173 * size
    res = torch.empty_like(q) if dtype == "bf16" else None
    out, lse = muon.attention(q, k, v, scale=1.0, residual=res)
    _, _, dv = muon.attention_backward(do, q, k, v, out, lse, residual=res, scale=1.0)
    # scaled by log2 e and back: two constants, two products and a sum
    top = float(k[0, 35, 0, 0])
    assert (np.abs(to_host(lse) - top) <= 5 * 2.0 ** -24 * top).all()
    u = ref.HALF_STEP[dtype]
    # out: p of the key is 1 up to 2^-22 (exponential and sum), rounded
    value = to_host(v)[0, 35, 0]
    assert (np.abs(to_host(out)[0, :, 0] - value) <= (u + 2.0 ** -22) * np.abs(value)).all()
    sums, sizes = to_host(do)[0, :, 0].sum(0), np.abs(to_host(do)[0, :, 0]).sum(0)
    factor = np.expm1(2.0 ** -23 * float(lse.abs().max())) + 2.0 ** -16 if dtype == "bf16" else 14 * 2.0 ** -24
    assert (np.abs(to_host(dv)[0, 35, 0] - sums) <= (factor + 24 * 2.0 ** -24) * sizes + u * np.abs(sums)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outputs_between_broadcast_inputs(muon, dtype):  # noqa: F811
    """All in one tensor, one head of keys and values for all query heads."""
    import torch
    q, k, v, do = make((2, 70, 70, 4, 1, 64, True, 0), dtype)
    want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=True, dout=to_host(do))
    buf = torch.full((2, 70, 22, 64), 5.0, dtype=q.dtype, device="cuda")
    q2, k2, v2, do2, out, dq = (buf[:, :, a:b] for a, b in ((0, 4), (4, 5), (5, 6), (6, 10), (10, 14), (14, 18)))
    for t, s in ((q2, q), (k2, k), (v2, v), (do2, do)):
        t.copy_(s)
    kx, vx = k2.expand(2, 70, 4, 64), v2.expand(2, 70, 4, 64)
    res = torch.empty_like(q) if dtype == "bf16" else None
    _, lse = muon.attention(q2, kx, vx, causal=True, out=out, residual=res)
    close(out.contiguous(), want["out"], "out")
    exact = torch.from_numpy(want["out"][0]).cuda()
    out.copy_(exact)
    res = (exact - out.double()).to(torch.bfloat16) if res is not None else None
    lse = torch.from_numpy(want["lse"][0]).float().cuda()
    _, dk, dv = muon.attention_backward(do2, q2, kx, vx, out, lse, residual=res, causal=True, dq=dq)
    close(dq.contiguous(), want["dq"], "dq")
    # a gradient for each head that sees the one: together its own
    for name, x in (("dk", dk), ("dv", dv)):
        val, bound = want[name]
        each = to_host(x)
        slack = ref.HALF_STEP[dtype] * np.abs(each).sum(2, keepdims=True)
        assert (np.abs(each.sum(2, keepdims=True) - val) <= bound + slack * (1 + 2.0 ** -7)).all(), name
    assert (buf[:, :, 18:] == 5).all() and torch.equal(q2, q) and torch.equal(do2, do)
