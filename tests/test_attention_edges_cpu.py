"""The attention block's autograd functions and host-only checks on the CPU, with a
stand-in for the library where tensors would need a device."""
import pytest

torch = pytest.importorskip("torch")

import torch.autograd.forward_ad as fwd  # noqa: E402

from paper_2609_21594_amd.attention import attention, rotary  # noqa: E402


class StandIn:
    """Results of the right shapes; says whether it was called."""
    calls = 0

    def attention(self, q, k, v, max_logits=None, residual=None, **kw):
        self.calls += 1
        return q.detach().clone(), torch.zeros(q.shape[0], q.shape[2], q.shape[1])

    def rotary(self, xs, freqs, positions=None, **kw):
        self.calls += 1
        return [x.detach().clone() for x in xs]


# ---------------------------------------------------------------- forward-mode tangents

@pytest.mark.parametrize("grad", [True, False])
@pytest.mark.parametrize("which", range(3))
def test_attention_refuses_tangents(grad, which):
    """There is no forward-mode derivative; no_grad does not turn that mode off, so a
    result without a tangent would be a wrong derivative of zero."""
    xs = [torch.ones(1, 3, 2, 8) for _ in range(3)]
    with fwd.dual_level(), torch.set_grad_enabled(grad):
        xs[which] = fwd.make_dual(xs[which], torch.ones(1, 3, 2, 8))
        lib = StandIn()
        with pytest.raises(RuntimeError, match="jvp"):
            attention(lib, *xs)
        assert lib.calls == 0


@pytest.mark.parametrize("grad", [True, False])
def test_rotary_refuses_tangents(grad):
    x, freqs = torch.ones(1, 3, 2, 8), torch.ones(4, dtype=torch.float64)
    with fwd.dual_level(), torch.set_grad_enabled(grad):
        dual = fwd.make_dual(x, torch.ones_like(x))
        with pytest.raises(RuntimeError, match="jvp"):
            rotary(StandIn(), dual, freqs)
        with pytest.raises(RuntimeError, match="jvp"):
            rotary(StandIn(), [x, dual], freqs)
        with pytest.raises(RuntimeError, match="jvp"):
            rotary(StandIn(), x, fwd.make_dual(freqs, torch.ones_like(freqs)))


def test_transformed_functions_refuse_tangents():
    def f(x):
        with torch.no_grad():
            return attention(StandIn(), x, x, x)
    x = torch.ones(1, 3, 2, 8)
    with pytest.raises(RuntimeError, match="jvp"):
        torch.func.jvp(f, (x,), (x,))


def test_without_tangents_no_grad_skips_autograd():
    lib, x = StandIn(), torch.ones(1, 3, 2, 8, requires_grad=True)
    with fwd.dual_level(), torch.no_grad():
        assert not attention(lib, x, x, x).requires_grad
        assert not rotary(lib, x, torch.ones(4, dtype=torch.float64)).requires_grad
    assert lib.calls == 2


# ---------------------------------------------------------------- gradients that do not exist

def test_rotary_refuses_frequencies_that_want_a_gradient():
    """It has none for them; silence would leave them untrained."""
    lib, x = StandIn(), torch.ones(1, 3, 2, 8)
    freqs = torch.ones(4, dtype=torch.float64, requires_grad=True)
    with pytest.raises(RuntimeError, match="freqs"):
        rotary(lib, x, freqs)
    with torch.no_grad():
        rotary(lib, x, freqs)
    assert lib.calls == 1


# ---------------------------------------------------------------- requests

def test_scales_that_binary32_cannot_hold_in_base_2_are_refused():
    """The kernels take scale * log2(e), which must be finite: with infinity a logit
    of 0 becomes NaN."""
    from tests.test_attention_cpu import check, grads, request
    assert check(request(scale=2.3e38))[0] == 0
    for g in (None, grads()):
        st, msg = check(request(scale=3e38), g)
        assert st == 1 and "scale" in msg


# ---------------------------------------------------------------- copies of weights on several ranks

def _clip_rank(rank, world, port, out):
    import os
    import numpy as np
    import torch.distributed as dist
    from oracle import attention_ref as ref
    os.environ.update(MASTER_ADDR="127.0.0.1", MASTER_PORT=str(port))
    dist.init_process_group("gloo", rank=rank, world_size=world)
    rng = np.random.default_rng(1)
    wq, wk = rng.standard_normal((16, 4)), rng.standard_normal((8, 4))     # the same on every rank
    top = torch.tensor([[8.0, 1.0], [2.0, 5.0]])[rank]                     # of the rank's batch
    own = ref.qk_clip(wq, wk, top.numpy(), 4.0, "f32")
    dist.all_reduce(top, dist.ReduceOp.MAX)
    both = ref.qk_clip(wq, wk, top.numpy(), 4.0, "f32")
    for name, res in (("own", own), ("both", both)):
        mine = torch.from_numpy(np.concatenate([x[0].ravel() for x in res]))
        all_ = [torch.empty_like(mine) for _ in range(world)]
        dist.all_gather(all_, mine)
        out[rank, name] = all(torch.equal(x, mine) for x in all_)
    dist.destroy_process_group()


def test_copies_of_weights_need_the_largest_logits_of_all_ranks():
    """What `clip_query_keys` tells data-parallel programs to do, on the oracle."""
    import socket
    import torch.multiprocessing as mp
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    with mp.Manager() as m:
        out = m.dict()
        mp.spawn(_clip_rank, (2, port, out), nprocs=2)
        assert all(out[r, "both"] for r in range(2)) and not any(out[r, "own"] for r in range(2))


# ---------------------------------------------------------------- gradients as the library takes them

def test_gradients_far_apart_are_copied():
    """Tokens more than 2^24 bytes apart are refused by the library; autograd may hand
    over such a gradient of an ordinary result."""
    from paper_2609_21594_amd.attention import _plain
    far = torch.zeros(2, (1 << 23) + 8, dtype=torch.bfloat16)
    g = far[None, :, None, :64]
    assert g.stride(1) * 2 > 1 << 24
    assert _plain(g).is_contiguous()
    near = torch.zeros(2, 1 << 12, dtype=torch.bfloat16).as_strided((1, 2, 2, 64), (4096, 128, 64, 1))
    assert _plain(near) is near


def test_rotary_copies_only_gradients_it_has_to():
    """Its library call takes heads of any alignment, broadcast ones too, as long as
    their elements are contiguous."""
    class Rotary(StandIn):
        def rotary(self, xs, freqs, positions=None, **kw):
            self.got = xs
            return super().rotary(xs, freqs, positions, **kw)
    lib, seen = Rotary(), []
    freqs = torch.ones(3, dtype=torch.float64)
    from paper_2609_21594_amd import attention as A

    class Ctx:
        captured, kw, saved_tensors, needs_input_grad = False, dict(inverse=False), (freqs, None), (False,) * 4 + (True,)
    Ctx.lib = lib
    odd = torch.zeros(1, 5, 2, 7, dtype=torch.bfloat16)[..., 1:]             # 12-byte heads, 2-byte aligned
    wide = torch.zeros(1, 1, 1, 6, dtype=torch.bfloat16).expand(1, 5, 2, 6)
    turned = torch.zeros(1, 5, 6, 2, dtype=torch.bfloat16).transpose(2, 3)
    capturing, A._enter_backward = A._enter_backward, lambda ctx: None       # (asks the device)
    try:
        for g in (odd, wide, turned):
            A._Rotary.backward(Ctx, g)
            seen.append(lib.got[0])
    finally:
        A._enter_backward = capturing
    assert seen[0] is odd and seen[1] is wide
    assert seen[2] is not turned and seen[2].is_contiguous()


def test_broadcast_inputs_may_lie_between_outputs():
    """Slices of one tensor, the keys' one head for all: no byte is shared."""
    from tests.test_attention_cpu import BASE, check, grads, request
    row = 20 * 64
    fused = {f"{n}__{s}": x for n in ("q", "k", "v", "out") for s, x in (("token_stride", row), ("batch_stride", 96 * row))}
    fused.update(q__data=BASE, k__data=BASE + 8 * 128, v__data=BASE + 9 * 128, out__data=BASE + 10 * 128,
                 k__head_stride=0, v__head_stride=0)
    assert check(request(**fused)) == (0, "")
    # one sequence's keys for both
    assert check(request(**dict(fused, k__batch_stride=0, v__batch_stride=0))) == (0, "")
    # the keys' head is the last of the outputs'
    assert "overlap" in check(request(**dict(fused, k__data=BASE + 17 * 128)))[1]
    assert "overlap" in check(request(**dict(fused, k__data=BASE + 96 * row * 2 + 12 * 128, k__batch_stride=0)))[1]
    g = grads()
    for name, at in (("dq", 10), ("dk", 18)):
        h = getattr(g, name)
        h.data, h.token_stride, h.batch_stride = BASE + at * 128, row, 96 * row
    assert check(request(**dict(fused, out__data=BASE + (40 << 32))), g) == (0, "")
