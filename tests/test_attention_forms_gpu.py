"""Attention requests for the forms of a launch that the lists of sizes elsewhere do
not reach: long key axes whose parts are many keys each (four waves to a row), parts
of requests of more than 4096 rows (two waves or one, one plane), heads of 65 to 96
and few rows."""
import numpy as np
import pytest

from oracle import attention_ref as ref
from tests.gpu_util import to_bits, to_host
from tests.test_attention_gpu import close, make, muon, saved  # noqa: F401

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")

# dtype and batch, queries, keys, query heads, key heads, head size, causal, window
PARTS = [
    ("bf16", 1, 1, 33000, 4, 1, 64, True, 0),       # 64 parts of 515 keys
    ("bf16", 1, 3, 33100, 2, 1, 96, False, 0),
    ("bf16", 1, 1, 32900, 1, 1, 128, True, 0),
    ("bf16", 8, 20, 600, 32, 8, 64, True, 0),       # 5120 rows, 128 workgroups
    ("bf16", 8, 20, 600, 32, 8, 96, False, 0),
    ("bf16", 8, 20, 600, 32, 8, 128, True, 0),
    ("bf16", 16, 20, 520, 32, 8, 80, True, 0),      # 256 workgroups
    ("f32", 16, 2, 520, 32, 8, 128, True, 0),
]


@pytest.mark.parametrize("case", PARTS, ids=str)
@pytest.mark.parametrize("padded", [False, True])
def test_parts(muon, case, padded):  # noqa: F811
    import torch
    dtype, case = case[0], case[1:]
    b, sq, sk, hq, _, _, causal, _ = case
    q, k, v, _ = make(case, dtype, 1.5)
    kw, seqs = dict(causal=causal), None
    if padded:  # lengths that leave parts, and whole sequences, without a key
        nq = [sq, 0, 1, sq - sq // 3][:b] + [sq] * (b - 4)
        nk = [sk - 300, 40, sk, 0][:b] + [sk - 1] * (b - 4)
        seqs = [(i, 0, n, 0, m) for i, (n, m) in enumerate(zip(nq, nk))]
        kw.update((n, torch.tensor(x, dtype=torch.int32, device="cuda")) for n, x in (("q_lens", nq), ("k_lens", nk)))
    want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=causal, seqs=seqs)
    top = torch.full((hq,), -INF, device="cuda")
    res = torch.full_like(q, NAN) if dtype == "bf16" else None
    out, lse = muon.attention(q, k, v, max_logits=top, residual=res, **kw)
    close(out, want["out"], "out")
    close(lse, want["lse"], "lse")
    close(top, want["top"], "top")
    if res is not None:
        r, o = to_host(res), to_host(out)
        assert (np.abs(r) <= ref.HALF_STEP["bf16"] * np.abs(o + r) * (1 + 2.0 ** -7)).all()
    again, lse2 = muon.attention(q, k, v, **kw)
    assert np.array_equal(to_bits(again), to_bits(out)) and np.array_equal(to_bits(lse2), to_bits(lse))


@pytest.mark.parametrize("case", [(1, 600, 600, 2, 1, 96, True, 0), (2, 520, 700, 2, 2, 72, False, 0)], ids=str)
def test_few_rows_of_heads_of_up_to_96(muon, case):  # noqa: F811
    import torch
    q, k, v, do = make(case, "bf16", 1.5)
    kw = dict(causal=case[6], window=case[7])
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", dout=to_host(do), **kw)
    top = torch.full((case[3],), -INF, device="cuda")
    out, lse = muon.attention(q, k, v, max_logits=top, **kw)
    close(out, want["out"], "out")
    close(lse, want["lse"], "lse")
    close(top, want["top"], "top")
    out, res, lse = saved(want, "bf16")
    got = muon.attention_backward(do, q, k, v, out, lse, residual=res, **kw)
    for name, x in zip(("dq", "dk", "dv"), got):
        close(x, want[name], name)
