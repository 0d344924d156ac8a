"""Autograd over the attention block of the library: rotary positions and
softmax attention whose largest logits feed the clip of the query and key
weights (`MuonAdamW.clip_query_keys`).

    lib = Muon(0)
    freqs = rotary_frequencies(128, base=10000.0).cuda()
    q, k = rotary(lib, [q, k], freqs)
    out = attention(lib, q, k, v, causal=True, max_logits=largest)

`lib` is a handle of the tensors' device.  Forward and backward run on the
streams that autograd gives them.  A handle serves one host thread at a time:
autograd's own thread may use it while the thread that called `backward`
waits, a second training thread needs a handle of its own.

Under graph capture, forward and backward belong in the capture together, and
no eager graph of the same leaves may still live: autograd would accumulate
their gradients on the eager graph's stream, which ends a capture and the
process with it.  Both are refused with a RuntimeError where these functions
can see them: a captured backward pass of an eager forward pass, and leaves
given to them that an earlier call of theirs on another stream still holds.
(`Muon.attention` and `Muon.attention_backward` know no autograd.)

Forward-mode tangents are refused with a RuntimeError, with gradients enabled or not.
"""
from __future__ import annotations

import math

import torch
from torch.autograd import forward_ad


def rotary_frequencies(rotary_dim, base=10000.0, factor=1.0, method="none", original_length=None, low=1.0, high=32.0):
    """fp64 [rotary_dim / 2] radians a position: base ** (-2 i / rotary_dim),
    scaled for contexts `factor` times longer than trained:
      "none"     as they are (factor must be 1)
      "linear"   every frequency / factor (positions interpolated)
      "base"     the base raised to base * factor ** (r / (r - 2)), so that the
                 slowest pair is interpolated by `factor` and the fastest not at all
      "ramp"     by how many turns t a pair makes over `original_length`
                 positions: t <= low interpolated, t >= high kept, linear in t
                 between"""
    r = int(rotary_dim)
    if r < 2 or r % 2:
        raise ValueError("rotary_dim must be even and >= 2")
    if not (math.isfinite(base) and base > 0 and math.isfinite(factor) and factor > 0):
        raise ValueError("base and factor must be finite and > 0")
    i = torch.arange(r // 2, dtype=torch.float64)
    if method == "base":
        if r == 2:
            raise ValueError('method "base" needs rotary_dim > 2')
        base = base * factor ** (r / (r - 2))
    freqs = torch.as_tensor(base, dtype=torch.float64) ** (-2.0 * i / r)
    if method == "none":
        if factor != 1.0:
            raise ValueError('a factor needs method "linear", "base" or "ramp"')
    elif method == "linear":
        freqs = freqs / factor
    elif method == "ramp":
        if original_length is None or not high > low:
            raise ValueError('method "ramp" needs original_length and high > low')
        turns = original_length * freqs / (2 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0.0, 1.0)
        freqs = freqs * keep + freqs / factor * (1.0 - keep)
    elif method != "base":
        raise ValueError(f"unknown method {method!r}")
    return freqs


def _refuse_tangents(*tensors):
    """There are no forward-mode derivatives here, and `no_grad` leaves that mode on:
    without this a result would come back without its tangent."""
    for t in tensors:
        if t is not None and forward_ad.unpack_dual(t).tangent is not None:
            raise RuntimeError("rotary and attention have no forward-mode derivative (jvp)")


def _enter(ctx, tensors):
    """Notes on which stream each leaf's gradient will be accumulated (in the
    leaf's accumulator, which lives as long as a graph holds it), and refuses a
    capture that would accumulate elsewhere."""
    ctx.captured = torch.cuda.is_current_stream_capturing()
    for t in tensors:
        if t.requires_grad and t.is_leaf:
            notes = torch.autograd.graph.get_gradient_edge(t).node.metadata
            here = torch.cuda.current_stream(t.device).cuda_stream
            if ctx.captured and notes.get("muon_stream", here) != here:
                raise RuntimeError("a graph capture meets leaves that an eager autograd graph still holds: "
                                   "delete the eager results first")
            notes.setdefault("muon_stream", here)


def _enter_backward(ctx):
    if torch.cuda.is_current_stream_capturing() and not ctx.captured:
        raise RuntimeError("a captured backward pass needs its forward pass in the same capture")


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, lib, freqs, positions, kw, *xs):
        _enter(ctx, xs)
        ctx.lib, ctx.kw = lib, kw
        ctx.save_for_backward(freqs, positions)
        ctx.set_materialize_grads(False)
        return tuple(lib.rotary(list(xs), freqs, positions=positions, **kw))

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *gs):
        _enter_backward(ctx)
        freqs, positions = ctx.saved_tensors
        kw = dict(ctx.kw, inverse=not ctx.kw["inverse"])  # the transpose: scale stays
        need = [i for i, g in enumerate(gs) if g is not None and ctx.needs_input_grad[4 + i]]
        out = [None] * len(gs)
        if need:
            for i, g in zip(need, ctx.lib.rotary([_near(gs[i]) for i in need], freqs, positions=positions, **kw)):
                out[i] = g
        return (None, None, None, None, *out)


def _near(g):
    """A gradient as the rotation takes it: contiguous heads, tokens at most 2^24
    bytes apart (autograd also hands over transposed and sliced ones)."""
    if g.stride(-1) == 1 and g.stride(-3) * g.element_size() <= 1 << 24:
        return g
    return g.clone(memory_format=torch.contiguous_format)


def _plain(g):
    """A gradient as attention takes it: 16-byte aligned heads besides, none of them
    expanded."""
    es = g.element_size()
    if g.data_ptr() % 16 == 0 and all(s * es % 16 == 0 and s > 0 for s in g.stride()[:-1]):
        return _near(g)
    return g.clone(memory_format=torch.contiguous_format)


def rotary(lib, xs, freqs, positions=None, first=0, layout="half", scale=1.0, inverse=False):
    """`Muon.rotary` with gradients: a tensor, or a list of up to 4.  freqs have
    none, and are refused where they ask for one."""
    one = torch.is_tensor(xs)
    xs = [xs] if one else list(xs)
    _refuse_tangents(*xs, freqs)
    kw = dict(first=first, layout=layout, scale=scale, inverse=inverse)
    if torch.is_grad_enabled():
        if freqs.requires_grad:
            raise RuntimeError("rotary has no gradient for freqs: detach them")
        ys = _Rotary.apply(lib, freqs, positions, kw, *xs)
    else:
        ys = lib.rotary(xs, freqs, positions=positions, **kw)
    return ys[0] if one else list(ys)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, lib, q, k, v, max_logits, kw):
        _enter(ctx, (q, k, v))
        ctx.lib, ctx.kw = lib, kw
        residual = None
        if q.dtype == torch.bfloat16 and any(ctx.needs_input_grad):
            residual = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        out, lse = lib.attention(q, k, v, max_logits=max_logits, residual=residual, **kw)
        ctx.save_for_backward(q, k, v, out, lse, residual, *(kw[n] for n in _LISTS))
        ctx.mark_non_differentiable(lse)
        ctx.set_materialize_grads(False)
        return out, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, _):
        _enter_backward(ctx)
        if dout is None:
            return None, None, None, None, None, None
        q, k, v, out, lse, residual, *lists = ctx.saved_tensors
        kw = dict(ctx.kw, **dict(zip(_LISTS, lists)))
        dq, dk, dv = ctx.lib.attention_backward(_plain(dout), q, k, v, out, lse, residual=residual, **kw)
        return None, dq, dk, dv, None, None


_LISTS = ("q_offsets", "k_offsets", "q_lens", "k_lens")


def attention(lib, q, k, v, scale=None, causal=False, window=0, q_offsets=None, k_offsets=None, q_lens=None,
              k_lens=None, max_logits=None, return_lse=False):
    """`Muon.attention` with gradients for q, k and v (lse and max_logits carry
    none).  bf16 outputs keep what their rounding took for the backward pass."""
    _refuse_tangents(q, k, v)
    kw = dict(scale=scale, causal=causal, window=window, q_offsets=q_offsets, k_offsets=k_offsets, q_lens=q_lens,
              k_lens=k_lens)
    if torch.is_grad_enabled():
        out, lse = _Attention.apply(lib, q, k, v, max_logits, kw)
    else:
        out, lse = lib.attention(q, k, v, max_logits=max_logits, **kw)
    return (out, lse) if return_lse else out
