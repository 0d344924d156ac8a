"""Attention requests at values where rounding or the order of sums shows, and at
values that are not finite, on every way that a launch can take."""
import numpy as np
import pytest

from oracle import attention_ref as ref
from tests.gpu_util import to_host
from tests.test_attention_gpu import close, make, muon  # noqa: F401

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
