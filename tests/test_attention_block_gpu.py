"""Rotary positions, the clip of query and key weights, and the whole block as
a training step uses it, on the GPU."""
import gc

import numpy as np
import pytest

from oracle import attention_ref as ref
from tests.gpu_util import require_gpu, to_bits, to_host
from tests.test_attention_gpu import close, make, tensor

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.fixture(scope="module")
def muon():
    require_gpu()
    from paper_2609_21594_amd.binding import Muon
    m = Muon(0)
    yield m
    m.close()


# ---------------------------------------------------------------- rotary positions

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("b,s,h,hk,d,r", [(1, 1, 1, 1, 2, 2), (3, 1, 8, 2, 128, 128), (2, 37, 4, 4, 64, 32),
                                          (1, 130, 3, 1, 80, 80), (2, 9, 2, 2, 20, 14), (1, 5, 1, 0, 96, 48),
                                          (1, 700, 2, 1, 256, 256), (2, 3, 2, 1, 1024, 1000)])
def test_rotary(muon, dtype, layout, b, s, h, hk, d, r):
    import torch
    from paper_2609_21594_amd.attention import rotary_frequencies
    rng = np.random.default_rng([b, s, h, d, r])
    q, k = tensor(rng, (b, s, h, d), dtype), tensor(rng, (b, s, hk, d), dtype)
    freqs = rotary_frequencies(r, 10000.0, 4.0, "linear").cuda()
    for pos in (None, rng.integers(0, 1 << 20, (b, s)), rng.integers(-5, 1 << 30, (b, s))):
        for inverse, scale in ((False, 1.0), (True, 1.25)):
            at = np.broadcast_to(np.arange(s), (b, s)) if pos is None else pos
            p = None if pos is None else torch.from_numpy(pos).cuda()
            if p is not None and not inverse:
                p = p.to(torch.int32)
            got = muon.rotary([q, k], freqs, positions=p, layout=layout, scale=scale, inverse=inverse)
            for x, y in ((q, got[0]), (k, got[1])):
                close(y, ref.rotary(to_host(x), at, freqs.cpu().numpy(), dtype, layout, scale, inverse), "rotary")
            # in place, the same bits
            q2, k2 = q.clone(), k.clone()
            muon.rotary([q2, k2], freqs, positions=p, layout=layout, scale=scale, inverse=inverse, outs=[q2, k2])
            assert np.array_equal(to_bits(q2), to_bits(got[0])) and np.array_equal(to_bits(k2), to_bits(got[1]))


def test_rotary_strides_positions_and_alignment(muon):
    import torch
    from paper_2609_21594_amd.attention import rotary_frequencies
    rng = np.random.default_rng(3)
    freqs = rotary_frequencies(48).cuda()
    base = tensor(rng, (2, 6, 41, 65), "bf16")           # [b, h, s, d + 1]: odd rows
    x = base.transpose(1, 2)[..., 1:]                    # [2, 41, 6, 64], 2-byte aligned
    pos = torch.from_numpy(rng.integers(0, 5000, (41, 2))).cuda().t()
    want = ref.rotary(to_host(x.contiguous()), pos.cpu().numpy(), freqs.cpu().numpy(), "bf16")
    close(muon.rotary(x, freqs, positions=pos), want, "strided")
    y = torch.full((2, 6, 41, 65), 7.0, dtype=torch.bfloat16, device="cuda")
    muon.rotary(x, freqs, positions=pos, outs=y.transpose(1, 2)[..., 1:])
    close(y.transpose(1, 2)[..., 1:].contiguous(), want, "strided result")
    assert (y[..., 0] == 7).all()
    # one position for all of a batch, a start, no batch axis
    one = torch.tensor([[9], [4]], device="cuda").expand(2, 41)
    close(muon.rotary(x, freqs, positions=one),
          ref.rotary(to_host(x.contiguous()), one.cpu().numpy(), freqs.cpu().numpy(), "bf16"), "expanded positions")
    close(muon.rotary(x[0], freqs, first=1000),
          ref.rotary(to_host(x[:1].contiguous()), 1000 + np.arange(41)[None], freqs.cpu().numpy(), "bf16"), "start")


def test_rotary_refusals(muon):
    import torch
    from paper_2609_21594_amd.binding import MuonError
    x = torch.ones(1, 4, 2, 16, device="cuda")
    f = torch.ones(8, dtype=torch.float64, device="cuda")
    for kw in (dict(layout="other"), dict(positions=torch.zeros(1, 3, dtype=torch.int64, device="cuda")),
               dict(outs=x[:, :2]), dict(xs=[x, x[..., :8]]), dict(xs=[x] * 5), dict(xs=x[0, 0])):
        with pytest.raises(ValueError):
            muon.rotary(**{**dict(xs=x, freqs=f), **kw})
    for kw in (dict(freqs=f.float()), dict(positions=torch.zeros(1, 4, device="cuda")), dict(xs=[x, x.bfloat16()])):
        with pytest.raises(TypeError):
            muon.rotary(**{**dict(xs=x, freqs=f), **kw})
    with pytest.raises(MuonError, match="rotary_dim"):
        muon.rotary(x, torch.ones(9, dtype=torch.float64, device="cuda"))
    with pytest.raises(MuonError, match="overlap"):
        buf = torch.ones(1, 5, 2, 16, device="cuda")
        muon.rotary(buf[:, :4], f, outs=buf[:, 1:])
    assert (x == 1).all()


# ---------------------------------------------------------------- the clip

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,hd,cols", [(1, 1, 1, 1), (4, 4, 3, 7), (8, 2, 64, 256), (6, 3, 20, 1001), (2, 1, 128, 96)])
def test_qk_clip(muon, dtype, hq, hkv, hd, cols):
    import torch
    rng = np.random.default_rng([hq, hkv, hd, cols])
    weights, logits = [], []
    for values in (rng.uniform(1, 30, hq), np.full(hq, -INF), np.full(hq, np.nan), np.full(hq, INF), np.full(hq, 5.0),
                   np.where(np.arange(hq) % 2 == 0, 500.0, 0.1)):
        weights.append((tensor(rng, (hq * hd, cols), dtype), tensor(rng, (hkv * hd, cols), dtype)))
        logits.append(torch.from_numpy(values.astype(np.float32)).cuda())
    before = [(q.clone(), k.clone()) for q, k in weights]
    want = [ref.qk_clip(to_host(q), to_host(k), m.cpu().numpy(), 5.0, dtype) for (q, k), m in zip(weights, logits)]
    muon.qk_clip([w[0] for w in weights], [w[1] for w in weights], logits, 5.0)
    for (q, k), (wq, wk) in zip(weights, want):
        close(q, wq, "wq")
        close(k, wk, "wk")
    for i in (1, 2, 3, 4):  # nothing above the threshold, or no number: the same bits
        for a, b in zip(weights[i], before[i]):
            assert np.array_equal(to_bits(a), to_bits(b))
    assert not torch.isneginf(logits[0]).any()
    muon.qk_clip([weights[0][0]], [weights[0][1]], [logits[0]], 1e9, reset=True)
    assert torch.isneginf(logits[0]).all() and not torch.isneginf(logits[4]).any()


def test_qk_clip_of_packed_weights_and_many_layers(muon):
    import torch
    rng = np.random.default_rng(8)
    packed = tensor(rng, (40, 8 * 16, 96), "bf16")  # 40 layers: more than one launch takes; columns of q, k, rest
    wq, wk = [p[:, :32] for p in packed], [p[:64, 32:64] for p in packed]
    logits = list(torch.from_numpy(rng.uniform(1, 20, (40, 8)).astype(np.float32)).cuda())
    want = [ref.qk_clip(to_host(q.contiguous()), to_host(k.contiguous()), m.cpu().numpy(), 5.0, "bf16")
            for q, k, m in zip(wq, wk, logits)]
    rest = to_bits(packed[..., 64:].contiguous()), to_bits(packed[:, 64:, 32:64].contiguous())
    muon.qk_clip(wq, wk, logits, 5.0, reset=True)
    for q, k, (a, b) in zip(wq, wk, want):
        close(q.contiguous(), a, "wq")
        close(k.contiguous(), b, "wk")
    assert np.array_equal(rest[0], to_bits(packed[..., 64:].contiguous()))
    assert np.array_equal(rest[1], to_bits(packed[:, 64:, 32:64].contiguous()))
    assert all(torch.isneginf(m).all() for m in logits)


# ---------------------------------------------------------------- together

def reference_block(x, w, freqs, hq, hkv, d):
    """out of rotary + causal attention of x through the weights, in fp64, by
    elementary operations."""
    import torch
    b, s, _ = x.shape
    q, k, v = ((x @ m.t()).view(b, s, -1, d) for m in w)
    angle = torch.arange(s, dtype=torch.float64)[:, None] * freqs
    c, sn = angle.cos()[:, None], angle.sin()[:, None]

    def turn(t):
        a, e = t[..., : d // 2], t[..., d // 2:]
        return torch.cat((a * c - e * sn, a * sn + e * c), -1)
    q, k = turn(q).transpose(1, 2), turn(k).transpose(1, 2).repeat_interleave(hq // hkv, 1)
    v = v.transpose(1, 2).repeat_interleave(hq // hkv, 1)
    logits = (q @ k.transpose(-1, -2)) / d ** 0.5
    logits = logits.masked_fill(torch.ones(s, s, dtype=torch.bool).triu(1), -INF)
    return (logits.softmax(-1) @ v).transpose(1, 2).reshape(b, s, -1), logits.amax((0, 2, 3))


def test_block_gradients_and_training_step(muon):
    """Projections, rotary, attention, gradients of the weights, Muon and the
    clip, as one training step."""
    import torch
    from paper_2609_21594_amd.attention import attention, rotary, rotary_frequencies
    from paper_2609_21594_amd.optim import MuonAdamW
    torch.manual_seed(0)
    b, s, hidden, hq, hkv, d = 2, 100, 96, 4, 2, 32
    x = torch.randn(b, s, hidden)
    ws = [torch.nn.Parameter((torch.randn(n * d, hidden) * 0.25).cuda()) for n in (hq, hkv, hkv)]
    freqs = rotary_frequencies(d)
    top = torch.full((hq,), -INF, device="cuda")
    up = torch.randn(b, s, hq * d)

    def forward():
        q, k, v = ((x.cuda() @ w.t()).view(b, s, -1, d) for w in ws)
        q, k = rotary(muon, [q, k], freqs.cuda())
        return attention(muon, q, k, v, causal=True, max_logits=top).flatten(2)
    out = forward()
    (out * up.cuda()).sum().backward()
    r = [w.detach().cpu().double().requires_grad_() for w in ws]
    want, logits = reference_block(x.double(), r, freqs, hq, hkv, d)
    (want * up.double()).sum().backward()
    # fp32 throughout: products over 96 and sums over up to 200 rows, each
    # within 2^-24 times its length of its terms' size; 1e-4 is far above that
    # for values of size 1 to 100 relative to the norm
    assert (out.detach().cpu().double() - want).norm() <= 1e-5 * want.norm()
    for w, g in zip(ws, r):
        assert (w.grad.cpu().double() - g.grad).norm() <= 1e-5 * g.grad.norm()
    assert torch.allclose(top.cpu().double(), logits, rtol=1e-5)

    threshold = float(logits.detach().median())
    opt = MuonAdamW(ws, lr=0.0, adamw_lr=0.0)       # the clip alone changes the weights
    opt.clip_query_keys(ws[0], ws[1], top, threshold)
    before = [w.detach().clone() for w in ws]
    opt.step()
    wq, wk = ref.qk_clip(to_host(before[0]), to_host(before[1]), logits.detach().numpy(), threshold, "f32")
    # the factor's relative error adds that of the logit (1e-5 above)
    close(ws[0], (wq[0], wq[1] + 2e-5 * np.abs(wq[0])), "wq")
    close(ws[1], (wk[0], wk[1] + 2e-5 * np.abs(wk[0])), "wk")
    assert torch.equal(ws[2], before[2]) and torch.isneginf(top).all()
    forward()
    assert (top <= threshold * (1 + 1e-4)).all() and (top > 0).all()
    with pytest.raises(Exception):
        opt.clip_query_keys(ws[0], ws[1], top, threshold)      # the same weights twice
    with pytest.raises(ValueError):
        opt.clip_query_keys(torch.zeros(128, 96, device="cuda"), ws[1], top)
    opt.step()
    opt.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_qk_clip_of_factors_below_binary32(muon, dtype):
    """1e-30 / 1e20 has no binary32 value; the weights stay numbers."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    wq, wk = torch.ones(16, 8, device="cuda", dtype=t), torch.ones(8, 8, device="cuda", dtype=t)
    muon.qk_clip([wq], [wk], [torch.tensor([1e20, 1e-31], device="cuda")], 1e-30)
    # 2^-126 split as 2^-63 and 2^-63, exact; the other head keeps its logits
    assert (wk == 2.0 ** -63).all() and (wq[:8] == 2.0 ** -63).all() and (wq[8:] == 2.0 ** 63).all()


def test_weights_that_share_logits_are_clipped_by_thresholds_of_their_own(muon):
    import torch
    from paper_2609_21594_amd.optim import MuonAdamW
    ws = [torch.nn.Parameter(torch.ones(16, 24, device="cuda")) for _ in range(4)]
    top = torch.tensor([8.0, 1.0], device="cuda")
    opt = MuonAdamW(ws, lr=0.0, adamw_lr=0.0)
    opt.clip_query_keys(ws[0], ws[1], top, 2.0)
    opt.clip_query_keys(ws[2], ws[3], top, 4.0)
    opt.step()
    # factors 2 / 8 and 4 / 8 of head 0, their square roots to queries and keys:
    # 0.5 is exact, 0.5 ** 0.5 off by at most one rounding of the root and one of the product
    for w, f in zip(ws, (0.5, 0.5, 0.5 ** 0.5, 0.5 ** 0.5)):
        assert ((w[:8] - f).abs() <= 2 * 2.0 ** -24).all() and (w[8:] == 1).all()
    assert torch.isneginf(top).all()
    opt.close()


def test_clip_of_views_of_a_packed_parameter(muon):
    import torch
    from paper_2609_21594_amd.optim import MuonAdamW
    w = torch.nn.Parameter(torch.ones(48, 24, device="cuda"))
    top = torch.tensor([8.0, 1.0], device="cuda")
    opt = MuonAdamW([w], lr=0.0, adamw_lr=0.0)
    opt.clip_query_keys(w[:16], w[16:32], top, 2.0)       # views with a graph
    (3 * w).sum().backward()
    assert torch.equal(w.grad, torch.full_like(w, 3.0))
    opt.step()
    half = torch.ones(48, 24)
    half[:8] = half[16:24] = 0.5                          # 2 / 8 in two factors of a half, exact
    assert torch.equal(w.detach().cpu(), half)
    assert all(t.grad_fn is None for entry in opt._clips for t in entry[:2])
    opt.close()


def test_gradients_against_differences(muon):
    import torch
    from paper_2609_21594_amd.attention import attention, rotary, rotary_frequencies
    rng = np.random.default_rng(1)
    q, k, v = (tensor(rng, (1, 50, h, 16), "f32").requires_grad_() for h in (4, 2, 2))
    up = tensor(rng, (1, 50, 4, 16), "f32")
    freqs = rotary_frequencies(8).cuda()

    def loss(q, k, v):
        a, b = rotary(muon, [q, k], freqs, layout="interleaved", scale=1.1)
        return (attention(muon, a, b, v, causal=True, window=20) * up).sum(dtype=torch.float64)
    loss(q, k, v).backward()
    for t, i in ((q, 0), (k, 1), (v, 2)):
        way = tensor(rng, t.shape, "f32")
        h = 2.0 ** -7
        ends = [float(loss(*[x.detach() + (sign * h * way if j == i else 0) for j, x in enumerate((q, k, v))]))
                for sign in (1, -1)]
        slope = float((t.grad.double() * way.double()).sum())
        # the loss (size up to 100) is known to about 1e-5, so its slope to
        # 1e-5 / h; third derivatives of size up to 1e3 give h^2 / 6 of that
        assert abs((ends[0] - ends[1]) / (2 * h) - slope) <= 1e-5 / h + 1e3 * h * h / 6, i


def test_autograd_forms(muon):
    """Results no gradient reaches, broadcast gradients, lse, packed sequences."""
    import torch
    from paper_2609_21594_amd.attention import attention, rotary, rotary_frequencies
    q, k, v, do = make((1, 40, 40, 4, 2, 64, True, 0), "bf16")
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    out, lse = attention(muon, *leaves, causal=True, return_lse=True)
    assert not lse.requires_grad
    out.sum().backward()                                   # an expanded gradient
    want = ref.attention(*map(to_host, (q, k, v)), "bf16", causal=True, dout=np.ones(q.shape))
    for name, t in zip(("dq", "dk", "dv"), leaves):
        val, bound = want[name]
        # out and lse are the GPU's here: out's own error (rounded probabilities,
        # 2^-8 of sum p |v| <= max |v|) moves dout . out, 64 terms, by `moved`;
        # a probability times that reaches dq with k, and dk, summed over at
        # most 40 rows of 2 heads, with q
        moved = 2.0 ** -8 * 1.01 * 64 * np.abs(to_host(v)).max()
        slack = {"dq": 0.125 * moved * np.abs(to_host(k)).max(), "dk": 0.125 * moved * np.abs(to_host(q)).max() * 80,
                 "dv": 0.0}[name]
        assert (np.abs(to_host(t.grad) - val) <= bound + slack).all(), name
    off = torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")
    a = [t[0].clone().requires_grad_() for t in (q, k, v)]
    attention(muon, *a, causal=True, q_offsets=off, k_offsets=off).backward(do[0])
    for i, lo, hi in ((0, 0, 15), (1, 15, 40)):            # each sequence as if alone
        c = [t[:, lo:hi].clone().requires_grad_() for t in (q, k, v)]
        attention(muon, *c, causal=True).backward(do[:, lo:hi])
        for x, y in zip(a, c):
            assert torch.allclose(x.grad[lo:hi].float(), y.grad[0].float(), rtol=2.0 ** -6, atol=2.0 ** -6)
    f = rotary_frequencies(64).cuda()
    x, y = q.clone().requires_grad_(), k.clone().requires_grad_()
    a, b = rotary(muon, [x, y], f)
    a.backward(do)                                         # no gradient reaches the keys
    assert y.grad is None
    close(x.grad, ref.rotary(to_host(do), np.arange(40)[None], f.cpu().numpy(), "bf16", inverse=True), "gradient")
    with torch.no_grad():
        assert not attention(muon, x, y, v).requires_grad


def test_other_stream(muon):
    import torch
    q, k, v, do = make((2, 200, 200, 4, 2, 128, True, 0), "bf16")
    out, lse = muon.attention(q, k, v, causal=True)
    grads = muon.attention_backward(do, q, k, v, out, lse, causal=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        out2, lse2 = muon.attention(q, k, v, causal=True, stream=side)
        grads2 = muon.attention_backward(do, q, k, v, out2, lse2, causal=True, stream=side)
        torch.empty(1 << 24, dtype=torch.uint8, device="cuda").fill_(255)  # would land in freed scratch
    side.synchronize()
    for a, b in zip((out, lse, *grads), (out2, lse2, *grads2)):
        assert np.array_equal(to_bits(a), to_bits(b))
    # two streams at once, each call with scratch of its own
    others = [torch.cuda.Stream() for _ in range(3)]
    got = [muon.attention(q[:, :2], k, v, causal=True, stream=s) for s in others]
    torch.cuda.synchronize()
    for o, l in got[1:]:
        assert np.array_equal(to_bits(o), to_bits(got[0][0])) and np.array_equal(to_bits(l), to_bits(got[0][1]))


def test_captured_and_replayed(muon):
    import torch
    from paper_2609_21594_amd.attention import rotary_frequencies
    shapes = ((1, 150, 4, 64), (1, 150, 2, 64), (1, 150, 2, 64), (1, 150, 4, 64))
    ins = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    one, cache = torch.zeros(2, 1, 4, 64, dtype=torch.bfloat16, device="cuda"), [torch.zeros(2, 900, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    freqs = rotary_frequencies(64).cuda()
    wq, wk = torch.ones(256, 32, device="cuda"), torch.ones(128, 32, device="cuda")

    def work():
        q, k = muon.rotary(ins[:2], freqs)
        top = torch.full((4,), -INF, device="cuda")
        out, lse = muon.attention(q, k, ins[2], causal=True, max_logits=top)
        grads = muon.attention_backward(ins[3], q, k, ins[2], out, lse, causal=True)
        split = muon.attention(one, *cache, causal=True)
        wq.fill_(1.0)
        wk.fill_(1.0)
        muon.qk_clip([wq], [wk], [top], 1.0)
        return [out, lse, top, *grads, *split, wq, wk]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):                              # two graphs share the handle, not their scratch
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = work()
        graphs.append((g, res))
    rng = np.random.default_rng(2)
    for turn in range(3):
        for t in (*ins, one, *cache):
            t.copy_(tensor(rng, t.shape, "bf16"))
        for g, res in graphs:
            g.replay()
            torch.cuda.synchronize()
            got = [to_bits(t) for t in res]
            for a, b in zip(got, work()):
                assert np.array_equal(a, to_bits(b)), turn
    del graphs, g, res
    gc.collect()


def test_captures_that_autograd_cannot_follow_are_refused(muon):
    import torch
    from paper_2609_21594_amd.attention import attention
    q, k, v, _ = make((1, 40, 40, 2, 2, 64, True, 0), "bf16")
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    attention(muon, *leaves, causal=True).sum()
    alive = attention(muon, *leaves, causal=True)   # an eager graph of the leaves
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="eager autograd graph"):
        with torch.cuda.graph(g):
            attention(muon, *leaves, causal=True)
    torch.cuda.synchronize()
    del alive
    gc.collect()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = attention(muon, *leaves, causal=True)
        grads = torch.autograd.grad(out.sum(), leaves)
    for _ in range(2):
        g.replay()
    torch.cuda.synchronize()
    got = [to_bits(t) for t in grads]
    del out
    out = attention(muon, *leaves, causal=True)
    for a, b in zip(got, torch.autograd.grad(out.sum(), leaves)):
        assert np.array_equal(a, to_bits(b))


def test_profile_names_the_calls(muon):
    import torch
    q, k, v, do = make((1, 64, 64, 2, 2, 64, True, 0), "bf16")
    muon.profile(True)
    out, lse = muon.attention(q, k, v, causal=True)
    muon.attention_backward(do, q, k, v, out, lse, causal=True)
    got = muon.profile_read()
    muon.profile(False)
    assert got["attention_forward"]["launches"] == 1 and got["attention_backward"]["launches"] == 1
    assert got["attention_forward"]["total_ms"] > 0 and got["rotary"]["launches"] == 0
    del torch


def test_inference_is_captured_beside_an_eager_graph(muon):
    """Without gradients there is nothing to accumulate, so nothing to refuse."""
    import torch
    from paper_2609_21594_amd.attention import attention, rotary, rotary_frequencies
    q, k, v = (torch.randn(1, 20, 2, 16, device="cuda", dtype=torch.bfloat16, requires_grad=True) for _ in range(3))
    freqs = rotary_frequencies(16).cuda()

    def run():
        return attention(muon, *rotary(muon, [q, k], freqs), v, causal=True)
    eager = run()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.no_grad(), torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(to_bits(out), to_bits(eager.detach()))
    assert not out.requires_grad
    eager.sum().backward()
    assert torch.isfinite(q.grad).all()
