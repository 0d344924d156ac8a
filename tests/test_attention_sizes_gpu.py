"""Attention requests of the sizes from which a launch takes another form: many
rows (probabilities in one bf16 plane), many and few workgroups (a wave to a row
or several), heads of a group in parts or added up at once, many sequences."""
import numpy as np
import pytest

from oracle import attention_ref as ref
from tests.gpu_util import to_bits, to_host
from tests.test_attention_gpu import close, make, muon, saved  # noqa: F401

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")

# dtype and batch, queries, keys, query heads, key heads, head size, causal, window
SIZES = [
    # bf16, more than 4096 rows
    ("bf16", 20, 130, 130, 16, 4, 64, True, 0),     # 640 workgroups of queries
    ("bf16", 20, 130, 130, 16, 4, 32, False, 0),
    ("bf16", 22, 129, 70, 16, 16, 96, True, 0),
    ("bf16", 10, 131, 140, 16, 2, 128, True, 50),
    ("bf16", 4, 300, 301, 4, 2, 64, True, 0),       # 48, over 301 keys
    ("bf16", 4, 300, 301, 4, 4, 128, False, 0),
    ("bf16", 9, 400, 260, 8, 8, 24, True, 0),       # 288
    ("bf16", 5, 500, 490, 4, 4, 96, True, 0),       # 80, over 490
    ("bf16", 2, 600, 700, 4, 2, 64, True, 0),       # 40, over 700
    ("bf16", 2, 600, 700, 4, 1, 96, True, 0),
    ("bf16", 2, 533, 520, 4, 2, 128, False, 0),
    ("bf16", 1, 1100, 1100, 4, 2, 80, True, 200),
    ("bf16", 2, 4097, 1, 1, 1, 16, False, 0),       # one key
    # the heads of a group: each by itself, two parts, all at once
    ("bf16", 32, 33, 130, 32, 8, 16, True, 0),
    ("bf16", 16, 33, 130, 32, 8, 16, True, 0),
    ("f32", 16, 33, 130, 32, 8, 24, True, 20),
    ("bf16", 8, 600, 128, 16, 4, 128, False, 0),
    ("bf16", 64, 40, 130, 16, 8, 16, True, 0),
    ("f32", 32, 33, 130, 32, 8, 16, True, 0),
    ("f32", 64, 40, 130, 16, 8, 16, False, 0),
    # fp32: 512 workgroups and more
    ("f32", 32, 65, 100, 16, 4, 64, True, 0),
    ("f32", 32, 40, 99, 16, 16, 72, False, 0),
    ("f32", 32, 40, 99, 16, 4, 128, True, 30),
    ("f32", 1, 600, 500, 2, 1, 96, True, 0),
]


@pytest.mark.parametrize("case", SIZES, ids=str)
def test_sizes(muon, case):
    dtype, case = case[0], case[1:]
    q, k, v, do = make(case, dtype, 1.5)
    kw = dict(causal=case[6], window=case[7])
    want = ref.attention(*map(to_host, (q, k, v)), dtype, dout=to_host(do), **kw)
    got, lse = muon.attention(q, k, v, **kw)
    close(got, want["out"], "out")
    close(lse, want["lse"], "lse")
    out, res, lse = saved(want, dtype)
    got = muon.attention_backward(do, q, k, v, out, lse, residual=res, **kw)
    for name, x in zip(("dq", "dk", "dv"), got):
        close(x, want[name], name)
    again = muon.attention_backward(do, q, k, v, out, lse, residual=res, **kw)
    for x, y in zip(got, again):
        assert np.array_equal(to_bits(x), to_bits(y))


# lengths of the sequences (keys: the same, or those after the colon), heads of queries and keys, head size
PACKED = [
    ([1, 500, 0, 3, 129, 128, 127], None, 4, 2, 64),
    ([300] + [0] * 62 + [5], None, 4, 4, 32),                         # 64
    ([2, 0, 1] * 21 + [140, 7], None, 4, 1, 72),                      # 65
    ([3, 0, 9, 131, 1] * 40, [2, 4, 0, 140, 7] * 40, 4, 2, 32),       # 200
    ([4] * 130, None, 16, 8, 64),                                     # the heads of a group added up at once
    ([1] * 4000 + [0] * 90 + [3] * 30, None, 2, 1, 16),               # two rounds of a search
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 100)])
@pytest.mark.parametrize("index", range(len(PACKED)))
def test_packed(muon, index, causal, window, dtype):
    import torch
    nq, nk, hq, hkv, d = PACKED[index]
    nk = nk or nq
    qo, ko = np.cumsum([3] + nq), np.cumsum([0] + nk)
    sq, sk = int(qo[-1]) + 2, int(ko[-1]) + 5
    q, k, v, do = make((1, sq, sk, hq, hkv, d, causal, window), dtype)
    seqs = [(0, int(a), n, int(b), m) for a, n, b, m in zip(qo, nq, ko, nk)]
    want = ref.attention(*map(to_host, (q, k, v)), dtype, causal=causal, window=window, seqs=seqs, dout=to_host(do))
    out, res, lse = saved(want, dtype)
    kw = dict(causal=causal, window=window, q_offsets=torch.from_numpy(qo.astype(np.int32)).cuda(),
              k_offsets=torch.from_numpy(ko.astype(np.int32)).cuda())
    q, k, v, do = (t[0] for t in (q, k, v, do))
    o, l = muon.attention(q, k, v, **kw)
    close(o, want["out"], "out")
    close(l, want["lse"], "lse")
    got = muon.attention_backward(do, q, k, v, out[0], lse[0], residual=None if res is None else res[0], **kw)
    for name, x in zip(("dq", "dk", "dv"), got):
        close(x, want[name], name)


def test_offsets_out_of_order_stay_inside_the_tensors(muon):
    """Not a sequence list, so no result is right; nothing beyond the tensors is written."""
    import torch
    rng = np.random.default_rng(3)
    t = 700
    for n in (5, 64, 65, 300):
        q, k, v, do = (torch.full((t + 200, 2, 32), 3.0, device="cuda", dtype=torch.bfloat16) for _ in range(4))
        bad = [torch.from_numpy(rng.integers(-900, 1500, n + 1).astype(np.int32)).cuda() for _ in range(2)]
        kw = dict(causal=True, q_offsets=bad[0], k_offsets=bad[1])
        given = [torch.full_like(q, 5.0) for _ in range(4)]
        part = slice(100, 100 + t)
        _, lse = muon.attention(q[part], k[part], v[part], out=given[0][part], **kw)
        lse.zero_()
        muon.attention_backward(do[part], q[part], k[part], v[part], q[part], lse, dq=given[1][part], dk=given[2][part],
                                dv=given[3][part], **kw)
        for x in given:
            assert (x[:100] == 5).all() and (x[100 + t:] == 5).all()


# few rows of many heads, or more than 128 queries, on a long key axis in parts
PARTS = [
    ("bf16", 16, 1, 600, 16, 16, 64, True, 0),      # 256 workgroups
    ("bf16", 32, 2, 520, 32, 8, 96, True, 0),
    ("bf16", 1, 200, 4100, 8, 2, 128, True, 0),
    ("bf16", 1, 515, 4121, 12, 12, 40, False, 0),
    ("bf16", 1, 1030, 4200, 4, 1, 128, True, 0),
    ("bf16", 5, 129, 4096, 4, 4, 72, True, 0),
    ("f32", 1, 200, 4100, 4, 2, 128, True, 0),
    ("f32", 2, 300, 4096, 3, 3, 64, False, 0),
]


@pytest.mark.parametrize("case", PARTS, ids=str)
@pytest.mark.parametrize("padded", [False, True])
def test_parts_of_the_keys(muon, case, padded):
    import torch
    dtype, case = case[0], case[1:]
    b, sq, sk, hq, _, _, causal, _ = case
    q, k, v, _ = make(case, dtype, 1.5)
    kw, seqs = dict(causal=causal), None
    if padded:  # lengths that leave parts, and whole sequences, without a key
        nq = [sq, 0, 1, sq - sq // 3, sq, 3][:b] + [sq] * (b - 6)
        nk = [sk - 300, 40, sk, sk // 2, 0, 17][:b] + [sk - 1] * (b - 6)
        seqs = [(i, 0, min(n, sq), 0, m) for i, (n, m) in enumerate(zip(nq, nk))]  # (the kernels cut them too)
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


# batch (0: packed, two sequences), queries, keys, query heads, key heads, head size, causal, window: forward
# workgroups of 8 waves
EIGHT = [
    (4, 513, 600, 16, 16, 64, False, 0),
    (4, 600, 129, 16, 4, 128, False, 0),
    (4, 520, 257, 16, 8, 96, False, 0),
    (8, 2050, 300, 8, 8, 128, True, 0),
    (8, 2050, 2200, 8, 2, 72, True, 0),
    (16, 2049, 140, 8, 8, 24, True, 0),
    (4, 2050, 2050, 8, 2, 64, True, 100),
    (0, 4300, 310, 16, 16, 40, False, 0),
]


@pytest.mark.parametrize("case", EIGHT, ids=str)
def test_many_rows_and_long_sequences(muon, case):
    import torch
    batch, sq, sk, hq, hkv, d, causal, window = case
    q, k, v, _ = make((max(1, batch), *case[1:]), "bf16", 1.5)
    kw, rng = dict(causal=causal, window=window), np.random.default_rng(5)
    if batch:
        # lengths of 0, of all and others
        nq, nk = ([0, n] + [int(x) for x in rng.integers(1, n + 1, batch - 2)] for n in (sq, sk))
        seqs = [(b, 0, n, 0, m) for b, (n, m) in enumerate(zip(nq, nk))]
        kw.update((n, torch.tensor(x, dtype=torch.int32, device="cuda")) for n, x in (("q_lens", nq), ("k_lens", nk)))
    else:
        seqs = [(0, 3, 2000, 0, 300), (0, 2003, sq - 2003, 300, 5)]
        kw.update((n, torch.tensor(x, dtype=torch.int32, device="cuda")) for n, x in (("q_offsets", [3, 2003, sq]),
                                                                                 ("k_offsets", [0, 300, 305])))
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", causal=causal, window=window, seqs=seqs)
    if not batch:
        q, k, v = q[0], k[0], v[0]
    top, res = torch.full((hq,), -INF, device="cuda"), torch.full_like(q, NAN)
    out, lse = muon.attention(q, k, v, max_logits=top, residual=res, **kw)
    close(out, want["out"], "out")
    close(lse, want["lse"], "lse")
    close(top, want["top"], "top")
    r, o = to_host(res), to_host(out)
    held = np.s_[:] if batch else np.s_[3:]
    assert (np.abs(r) <= ref.HALF_STEP["bf16"] * np.abs(o + r) * (1 + 2.0 ** -7))[held].all()
    again, lse2 = muon.attention(q, k, v, **kw)
    assert np.array_equal(to_bits(again), to_bits(out)) and np.array_equal(to_bits(lse2), to_bits(lse))
