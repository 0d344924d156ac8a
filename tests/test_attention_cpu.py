"""The attention block on the CPU: the oracle against differences, packed
requests, refusals (through the library's host-only checks, on addresses that
nothing dereferences) and the frequencies."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import attention_ref as ref  # noqa: E402
from paper_2609_21594_amd import binding as B  # noqa: E402
from paper_2609_21594_amd.attention import rotary_frequencies  # noqa: E402

BASE = 1 << 40


def call(fn, *args):
    msg = ctypes.create_string_buffer(256)
    st = fn(*args, msg, 256)
    return st, msg.value.decode()


# ---------------------------------------------------------------- the oracle

@pytest.mark.parametrize("causal,window", [(False, 0), (True, 0), (True, 3)])
def test_oracle_gradients_match_differences(causal, window):
    rng = np.random.default_rng(5)
    q, k, v, do = (rng.standard_normal(s) for s in ((1, 6, 4, 5), (1, 7, 2, 5), (1, 7, 2, 5), (1, 6, 4, 5)))
    got = ref.attention(q, k, v, "f32", causal=causal, window=window, dout=do)

    def loss(q, k, v):
        return float((ref.attention(q, k, v, "f32", causal=causal, window=window)["out"][0] * do).sum())
    h = 1e-5
    for name, at in (("dq", 0), ("dk", 1), ("dv", 2)):
        xs = [q, k, v]
        for _ in range(8):
            i = tuple(rng.integers(0, n) for n in xs[at].shape)
            ends = []
            for sign in (1, -1):
                ys = [x.copy() for x in xs]
                ys[at][i] += sign * h
                ends.append(loss(*ys))
            # second differences are below 1e2 here: the truncation is below 1e2 h^2
            assert abs((ends[0] - ends[1]) / (2 * h) - got[name][0][i]) < 1e-7


def test_oracle_rows_without_keys_are_zero():
    q, k = np.ones((1, 5, 1, 4)), np.ones((1, 2, 1, 4))
    got = ref.attention(q, k, k, "f32", causal=True, dout=q)
    assert not got["out"][0][0, :3].any() and np.isneginf(got["lse"][0][0, 0, :3]).all()
    assert not got["dq"][0][0, :3].any() and got["out"][0][0, 3:].all()


def test_oracle_rotation_turns_back():
    rng = np.random.default_rng(6)
    x, pos = rng.standard_normal((2, 3, 2, 10)), rng.integers(0, 1000, (2, 3))
    f = rotary_frequencies(6).numpy()
    for layout in ("half", "interleaved"):
        y, _ = ref.rotary(x, pos, f, "f32", layout)
        z, _ = ref.rotary(y, pos, f, "f32", layout, inverse=True)
        assert np.abs(z - x).max() < 1e-13 and (y[..., 6:] == x[..., 6:]).all()


# ---------------------------------------------------------------- frequencies

def test_frequencies():
    f = rotary_frequencies(8, base=100.0)
    assert f.dtype == torch.float64
    assert torch.allclose(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64), rtol=1e-14)
    assert torch.allclose(rotary_frequencies(8, 100.0, 4.0, "linear"), f / 4, rtol=1e-14)
    g = rotary_frequencies(8, 100.0, 4.0, "base")
    assert g[0] == 1.0 and math.isclose(g[-1], f[-1] / 4, rel_tol=1e-12)
    h = rotary_frequencies(64, 10000.0, 8.0, "ramp", original_length=4096)
    f = rotary_frequencies(64, 10000.0)
    turns = 4096 * f / (2 * math.pi)
    assert (h[turns >= 32] == f[turns >= 32]).all() and torch.allclose(h[turns <= 1], f[turns <= 1] / 8, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and ((h < f) & (h > f / 8))[mid].all()


@pytest.mark.parametrize("kw", [dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, factor=2.0),
                                dict(rotary_dim=8, method="ramp", factor=2.0), dict(rotary_dim=8, method="other"),
                                dict(rotary_dim=2, method="base", factor=2.0), dict(rotary_dim=8, base=0.0),
                                dict(rotary_dim=8, method="linear", factor=float("inf"))])
def test_frequencies_refuse(kw):
    with pytest.raises(ValueError):
        rotary_frequencies(**kw)


# ---------------------------------------------------------------- requests

def test_packed_records_have_the_structs_layouts():
    for rec, cls in ((B._ATTENTION_PACK, B.MuonAttention), (B._GRAD_PACK, B.MuonAttentionGrad),
                     (B._ROTARY_PACK, B.MuonRotary), (B._ROTARY_TENSOR_PACK, B.MuonRotaryTensor),
                     (B._CLIP_PACK, B.MuonQKClip)):
        assert rec.size == ctypes.sizeof(cls)
    q = torch.zeros(2, 5, 4, 16, dtype=torch.bfloat16)
    k = torch.zeros(2, 7, 3, 2, 16, dtype=torch.bfloat16)[:, :, 1]
    a = B._Attention(q, k, k, None, True, 3, None, None, None, None)
    out, lse = torch.zeros_like(q), torch.zeros(a.lse_shape)
    rec = B.MuonAttention.from_buffer_copy(a.record(out, out, lse, lse, 256, 99))
    assert (rec.dtype, rec.head_dim, rec.q_heads, rec.kv_heads, rec.causal, rec.window) == (B.BF16, 16, 4, 2, 1, 3)
    assert (rec.batch, rec.q_tokens, rec.k_tokens, rec.sequences, rec.scale) == (2, 5, 7, 0, 0.25)
    assert (rec.k.data, rec.k.batch_stride, rec.k.token_stride, rec.k.head_stride) == (k.data_ptr(), 7 * 96, 96, 16)
    assert (rec.out.data, rec.residual.data, rec.lse, rec.max_logits, rec.scratch, rec.scratch_bytes) == (
        out.data_ptr(), out.data_ptr(), lse.data_ptr(), lse.data_ptr(), 256, 99)
    off = torch.tensor([0, 2, 5], dtype=torch.int32)
    rec = B.MuonAttention.from_buffer_copy(B._Attention(q[0], k[0], k[0], 2.0, False, 0, off, off, None, None).sizes())
    assert (rec.batch, rec.sequences, rec.q_tokens, rec.q_offsets, rec.q.token_stride) == (1, 2, 5, off.data_ptr(), 64)


def heads(i, h, t, d=64):
    return B.MuonHeads(BASE + (i << 32), t * h * d, h * d, d)


def request(**kw):
    a = B.MuonAttention(dtype=B.BF16, head_dim=64, q_heads=8, kv_heads=2, causal=1, scale=0.125, batch=2, q_tokens=96,
                        k_tokens=96, q=heads(0, 8, 96), k=heads(1, 2, 96), v=heads(2, 2, 96), out=heads(3, 8, 96),
                        lse=BASE + (4 << 32), scratch=BASE + (5 << 32), scratch_bytes=1 << 30)
    for n, v in kw.items():
        at = a
        *path, last = n.split("__")
        for p in path:
            at = getattr(at, p)
        setattr(at, last, v)
    return a


def grads():
    return B.MuonAttentionGrad(heads(6, 8, 96), heads(7, 8, 96), heads(8, 2, 96), heads(9, 2, 96))


def check(a, g=None):
    return call(B.load_library().muon_validate_attention, ctypes.byref(a) if a else None,
                ctypes.byref(g) if g else None)


def test_good_requests_pass():
    assert check(request()) == (0, "")
    assert check(request(), grads()) == (0, "")
    assert check(request(residual=heads(10, 8, 96)), grads())[0] == 0
    # broadcast keys, strides of single dimensions, a fused tensor with outputs beside inputs
    assert check(request(k__head_stride=0, v__token_stride=0))[0] == 0
    assert check(request(batch=1, q__batch_stride=-3))[0] == 0
    fused = {f"{n}__token_stride": 20 * 64 for n in ("q", "k", "v", "out")}
    fused.update({f"{n}__batch_stride": 96 * 20 * 64 for n in ("q", "k", "v", "out")})
    fused.update(q__data=BASE, k__data=BASE + 8 * 128, v__data=BASE + 10 * 128, out__data=BASE + 12 * 128)
    assert check(request(**fused))[0] == 0
    # head-major storage
    assert check(request(out__head_stride=96 * 64, out__token_stride=64))[0] == 0
    # nothing to do
    assert check(request(batch=0, q__data=0, k__data=0, v__data=0, out__data=0, lse=0))[0] == 0


BAD = [
    (dict(dtype=7), "dtype"), (dict(q_heads=7), "multiple"), (dict(kv_heads=0), "multiple"),
    (dict(head_dim=0), "head_dim"), (dict(head_dim=60), "head_dim"), (dict(head_dim=136), "head_dim"),
    (dict(scale=0.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=-1.0), "scale"),
    (dict(causal=2), "causal"), (dict(causal=0, window=4), "window"), (dict(window=-1), "window"),
    (dict(batch=-1), "range"), (dict(q_tokens=1 << 31), "range"), (dict(q_tokens=1 << 26), "too many"),
    (dict(q_offsets=BASE, sequences=1), "together"), (dict(q_lengths=BASE), "together"),
    (dict(q_offsets=BASE, k_offsets=BASE, sequences=3), "batch 1"), (dict(sequences=2), "sequences"),
    (dict(q_offsets=BASE, k_offsets=BASE, q_lengths=BASE, k_lengths=BASE, batch=1), "exclude"),
    (dict(fill_rest=1), "fill_rest"), (dict(fill_rest=2), "fill_rest"), (dict(reserved=1), "reserved"),
    (dict(q__data=0), "q is NULL"), (dict(k__data=BASE + 2), "k is not 16"), (dict(v__token_stride=130), "v: strides"),
    (dict(v__token_stride=-128), "v: stride"), (dict(q__token_stride=1 << 24), "token stride"),
    (dict(out__token_stride=64), "overlap"), (dict(out__batch_stride=0), "overlap"), (dict(out__data=BASE), "overlaps"),
    (dict(out__data=BASE + (1 << 32)), "overlaps"), (dict(lse=BASE), "overlaps"), (dict(lse=0), "lse"),
    (dict(lse=BASE + 2), "lse"), (dict(max_logits=BASE + (3 << 32)), "overlaps"), (dict(max_logits=BASE + 1), "max_logits"),
    (dict(dtype=B.F32, residual=heads(10, 8, 96)), "residual"), (dict(residual=heads(3, 8, 96)), "overlaps"),
    (dict(q_lengths=BASE + 1, k_lengths=BASE), "aligned"),
    (dict(q_lengths=BASE + (3 << 32), k_lengths=BASE), "overlaps"),
]


@pytest.mark.parametrize("kw,word", BAD, ids=[f"{i}-{w}" for i, (_, w) in enumerate(BAD)])
def test_bad_requests_are_refused(kw, word):
    st, msg = check(request(**kw))
    assert st in (1, 2) and word in msg, (st, msg)


def test_backward_refusals():
    for i, name in enumerate(("dq", "dk", "dv")):
        g = grads()
        getattr(g, name).data = BASE  # the queries
        st, msg = check(request(), g)
        assert st == 1 and "overlaps" in msg
        getattr(g, name).data = 0
        assert name in check(request(), g)[1]
    st, msg = check(request(scratch_bytes=100), grads())
    assert st == 1 and "scratch has 100 bytes" in msg
    assert "aligned" in check(request(scratch=BASE + (5 << 32) + 16), grads())[1]
    assert check(request(scratch=BASE), grads())[1].startswith("an output or the scratch")
    assert check(None)[0] == 1
    n = ctypes.c_size_t()
    lib = B.load_library()
    assert lib.muon_attention_scratch(ctypes.byref(request()), 1, ctypes.byref(n)) == 0 and n.value > 0
    assert check(request(scratch_bytes=n.value - 1), grads())[0] == 1
    assert check(request(scratch_bytes=n.value), grads())[0] == 0
    assert lib.muon_attention_scratch(ctypes.byref(request(head_dim=3)), 1, ctypes.byref(n)) == 2


def rot(**kw):
    r = B.MuonRotary(dtype=B.BF16, head_dim=64, rotary_dim=64, scale=1.0, batch=2, tokens=96, freqs=BASE + (9 << 32),
                     n_tensors=2)
    for n, v in kw.items():
        setattr(r, n, v)
    return r


def rot_tensors(**kw):
    t = (B.MuonRotaryTensor * 4)()
    for i in range(4):
        t[i] = B.MuonRotaryTensor(heads(2 * i, 8, 96), heads(2 * i + 1, 8, 96), 8)
    for n, v in kw.items():
        setattr(t[0].y if n == "data" else t[0], n, v)
    return t


def test_rotary_refusals():
    fn = B.load_library().muon_validate_rotary

    def st(r, t=None):
        return call(fn, ctypes.byref(r), t or rot_tensors())
    assert st(rot()) == (0, "")
    assert st(rot(positions=BASE + (10 << 32), position_batch_stride=96, position_token_stride=1))[0] == 0
    for kw, word in ((dict(dtype=3), "dtype"), (dict(rotary_dim=63), "rotary_dim"), (dict(rotary_dim=0), "rotary_dim"),
                     (dict(rotary_dim=66), "rotary_dim"), (dict(head_dim=2000), "head_dim"), (dict(layout=2), "layout"),
                     (dict(inverse=5), "inverse"), (dict(scale=float("inf")), "scale"), (dict(n_tensors=5), "tensors"),
                     (dict(n_tensors=0), "tensors"), (dict(freqs=0), "freqs"), (dict(freqs=BASE + 4), "freqs"),
                     (dict(tokens=1 << 31), "range"), (dict(tokens=1 << 23), "too many"),
                     (dict(positions=BASE + 2), "positions"),
                     (dict(positions=BASE + (10 << 32), position_token_stride=-1), "stride"),
                     (dict(positions=BASE + (1 << 32)), "overlaps")):
        code, msg = st(rot(**kw))
        assert code in (1, 2) and word in msg, (kw, code, msg)
    assert st(rot(), rot_tensors(data=BASE))[0] == 0  # in place
    same = rot_tensors(data=BASE)
    same[0].y.token_stride *= 2
    assert "same strides" in st(rot(), same)[1]
    assert "overlaps" in st(rot(), rot_tensors(data=BASE + 128))[1]
    assert "overlaps" in st(rot(), rot_tensors(data=BASE + (3 << 32)))[1]
    assert call(fn, None, rot_tensors())[0] == 1


def clip(**kw):
    c = B.MuonQKClip(BASE, BASE + (1 << 32), BASE + (2 << 32), 0, 0, 256, 8, 2, 64, B.BF16, 10.0, 0)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def test_clip_refusals():
    fn = B.load_library().muon_validate_qk_clip

    def st(*cs):
        return call(fn, (B.MuonQKClip * len(cs))(*cs), len(cs))
    assert st(clip()) == (0, "") and st()[0] == 0
    assert st(clip(), clip(wq=BASE + (3 << 32), wk=BASE + (4 << 32)))[0] == 0  # shared logits
    # query and key weights side by side in one packed weight
    assert st(clip(wk=BASE + 512, q_ld=512, k_ld=512))[0] == 0
    for kw, word in ((dict(dtype=9), "dtype"), (dict(q_heads=7), "multiple"), (dict(kv_heads=0), "multiple"),
                     (dict(head_dim=0), "range"), (dict(cols=0), "range"), (dict(threshold=0.0), "threshold"),
                     (dict(threshold=float("nan")), "threshold"), (dict(q_ld=200), "stride"), (dict(wk=0), "NULL"),
                     (dict(max_logits=0), "NULL"), (dict(wq=BASE + 1), "aligned"), (dict(max_logits=BASE + (2 << 32) + 2), "aligned"),
                     (dict(wk=BASE), "overlap"), (dict(max_logits=BASE + 16), "overlap"), (dict(reserved=1), "reserved"),
                     (dict(q_heads=65536, kv_heads=65536, head_dim=8192, q_ld=0), "too many")):
        code, msg = st(clip(**kw))
        assert code in (1, 2) and word in msg, (kw, code, msg)
    assert "overlap" in st(clip(), clip())[1]  # the same weights twice
    assert call(fn, None, 1)[0] == 1


# ---------------------------------------------------------------- the binding's own checks

def test_binding_refuses_shapes_and_types():
    q, k = torch.zeros(2, 5, 4, 16), torch.zeros(2, 7, 2, 16)
    off = torch.tensor([0, 5], dtype=torch.int32)
    lens = torch.tensor([5, 5], dtype=torch.int32)

    def a(q=q, k=k, v=k, **kw):
        args = dict(scale=None, causal=False, window=0, q_offsets=None, k_offsets=None, q_lens=None, k_lens=None)
        args.update(kw)
        return B._Attention(q, k, v, **args)
    a()
    a(q_lens=lens, k_lens=lens)
    for kw in (dict(q=q[0]), dict(v=k[:, :5]), dict(k=k[..., :8], v=k[..., :8]), dict(k=k[:1], v=k[:1]),
               dict(q_offsets=off, k_offsets=off), dict(q_lens=lens[:1], k_lens=lens),
               dict(q=q.transpose(2, 3), k=k, v=k),
               dict(q=q[0], k=k[0], v=k[0], q_offsets=off, k_offsets=torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            a(**kw)
    for kw in (dict(k=k.bfloat16(), v=k), dict(q=q.half(), k=k.half(), v=k.half()), dict(q_lens=lens.long(), k_lens=lens)):
        with pytest.raises(TypeError):
            a(**kw)
    with pytest.raises(ValueError):
        B.clip_records([torch.zeros(10, 4)], [torch.zeros(8, 4)], [torch.zeros(4)], 1.0)
    with pytest.raises(ValueError):
        B.clip_records([torch.zeros(8, 4)], [torch.zeros(3, 4)], [torch.zeros(4)], 1.0)
    with pytest.raises(ValueError):
        B.clip_records([torch.zeros(4, 8).t()], [torch.zeros(8, 4)], [torch.zeros(4)], 1.0)
    with pytest.raises(TypeError):
        B.clip_records([torch.zeros(8, 4)], [torch.zeros(8, 4)], [torch.zeros(4).double()], 1.0)
    w = torch.zeros(8, 4)
    with pytest.raises(B.MuonError):
        B.validate_qk_clip([w], [w], [torch.zeros(4)], 1.0)
    B.validate_qk_clip([w], [torch.zeros(4, 4)], [torch.zeros(4)], 1.0)
