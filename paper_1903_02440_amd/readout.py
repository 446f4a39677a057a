"""Binding of the readout operators (``include/libspyke_readout.h``): the gated
delta rule, its single-sample form and its gradients, and winners drawn from
scores.

The functions have the names of the C entry points and, as those of the package,
only marshal: dtype and shape checks, outputs and workspaces that are not given,
raw pointers and the stream.  The call runs on the tensors' device, on its
current stream unless one is given (keyword ``stream``).
"""
from __future__ import annotations

import functools

import torch

from . import _F, _I, _P, _Z, _check, _lib, _need, _out, _ws

_SIGS = {
    "spk_delta_rule_workspace_size": (_Z, [_I] * 7),
    "spk_delta_rule": (_I, [_P] * 5 + [_I] * 7 + [_F] + [_P] * 5 + [_Z, _P]),
    "spk_delta_rule_step": (_I, [_P] * 5 + [_I] * 6 + [_F] + [_P] * 3),
    "spk_delta_rule_backward_workspace_size": (_Z, [_I] * 7),
    "spk_delta_rule_backward": (_I, [_P] * 5 + [_I] * 7 + [_F] + [_P] * 11 + [_Z, _P]),
    "spk_sample_winners_workspace_size": (_Z, [_I] * 5),
    "spk_sample_winners": (_I, [_P, _I, _P, _P] + [_I] * 5 + [_F, _I, _F, _F] + [_P] * 3 + [_Z, _P]),
}
for _name, (_res, _args) in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _res
    _fn.argtypes = _args

SPK_F32, SPK_BF16 = 0, 1
_DTYPES = {torch.float32: SPK_F32, torch.bfloat16: SPK_BF16}

__all__ = ["SPK_F32", "SPK_BF16"] + list(_SIGS)


def _dtype(t, name):
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name}: expected torch.float32 or torch.bfloat16, got {t.dtype}")
    return code


def _at(dev, name, t):
    """Address of a tensor on the call's device (None and False: NULL)."""
    if t is None or t is False:
        return None
    if t.device != dev:
        raise ValueError(f"{name}: on {t.device}, the call's tensors are on {dev}")
    if not t.is_contiguous():
        raise ValueError("libspyke needs contiguous tensors")
    return t.data_ptr()


def _on(dev, call):
    """call(stream handle) on the current stream of `dev`, with `dev` current (a launch goes to the current device)."""
    if dev.index == torch.cuda.current_device():
        _check(call(torch._C._cuda_getCurrentRawStream(dev.index)))
        return
    with torch.cuda.device(dev):
        _check(call(torch.cuda.current_stream(dev).cuda_stream))


def _with_stream(fn):
    """Adds the keyword `stream`: the call runs with it current, so that outputs and workspaces made here are its too."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        for t in (*args, *kw.values()):
            if isinstance(t, torch.Tensor) and t.device != stream.device:
                raise ValueError(f"stream on {stream.device}, a tensor of the call on {t.device}")
        with torch.cuda.stream(stream):
            return fn(*args, **kw)
    return call


# ---------------------------------------------------------------- delta rule
def spk_delta_rule_workspace_size(dtype, B, L, Hk, Hv, dk, dv) -> int:
    return int(_lib.spk_delta_rule_workspace_size(dtype, B, L, Hk, Hv, dk, dv))


def spk_delta_rule_backward_workspace_size(dtype, B, L, Hk, Hv, dk, dv) -> int:
    return int(_lib.spk_delta_rule_backward_workspace_size(dtype, B, L, Hk, Hv, dk, dv))


def _delta_args(q, k, v, g, beta, lengths, initial_state):
    """Checks the inputs of a batch call; (dtype code, B, L, Hk, Hv, dk, dv)."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dim() != 4:
            raise ValueError(f"{name}: expected [B, L, heads, size], got shape {tuple(t.shape)}")
    dt = _dtype(q, "q")
    B, L, Hk, dk = q.shape
    Hv, dv = v.shape[2:]
    _need(q, q.dtype, (B, L, Hk, dk), "q")
    _need(k, q.dtype, (B, L, Hk, dk), "k")
    _need(v, q.dtype, (B, L, Hv, dv), "v")
    _need(g, torch.float32, (B, L, Hv), "g")
    _need(beta, torch.float32, (B, L, Hv), "beta")
    if lengths is not None:
        _need(lengths, torch.int32, (B,), "lengths")
    if initial_state is not None:
        _need(initial_state, torch.float32, (B, Hv, dk, dv), "initial_state")
    return dt, B, L, Hk, Hv, dk, dv


def _rows(t, like, dtype, lengths, name):
    """An output of rows per sample; a new one is 0 behind the sequences' lengths."""
    if t is None and lengths is not None:
        return torch.zeros(like.shape, dtype=dtype, device=like.device)
    return _out(t, like.shape, dtype, like.device, name)


@_with_stream
def spk_delta_rule(q, k, v, g, beta, scale=1.0, initial_state=None, lengths=None, out=None, final_state=None,
                   workspace=None):
    """Gated delta rule over a batch of sequences: q, k [B,L,Hk,dk] and v [B,L,Hv,dv] of one dtype (float32 or
    bfloat16), g, beta f32 [B,L,Hv] -> (out [B,L,Hv,dv], final_state f32 [B,Hv,dk,dv] or None).  lengths i32 [B]
    gives each sequence's samples; rows of a given `out` behind them are left as they were, those of a new one
    are 0.  final_state may be initial_state.  g is a log decay, at most 0: calls of more than 10 samples answer the
    growth of a state by more than e within 64 samples with NaN."""
    dt, B, L, Hk, Hv, dk, dv = _delta_args(q, k, v, g, beta, lengths, initial_state)
    dev = q.device
    out = _rows(out, v, q.dtype, lengths, "out")
    final_state = _out(final_state, (B, Hv, dk, dv), torch.float32, dev, "final_state")
    n = spk_delta_rule_workspace_size(dt, B, L, Hk, Hv, dk, dv)
    ws = _ws(workspace, n, dev)
    args = (_at(dev, "q", q), _at(dev, "k", k), _at(dev, "v", v), _at(dev, "g", g), _at(dev, "beta", beta), dt, B, L,
            Hk, Hv, dk, dv, scale, _at(dev, "lengths", lengths), _at(dev, "initial_state", initial_state),
            _at(dev, "out", out), _at(dev, "final_state", final_state), _at(dev, "workspace", ws), n)
    _on(dev, lambda st: _lib.spk_delta_rule(*args, st))
    return out, (final_state if final_state is not False else None)


@_with_stream
def spk_delta_rule_step(q, k, v, g, beta, state, scale=1.0, out=None):
    """One sample of every sequence: q, k [B,Hk,dk], v [B,Hv,dv], g, beta f32 [B,Hv]; state f32 [B,Hv,dk,dv] is
    updated in place -> out [B,Hv,dv]."""
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.dim() != 3:
            raise ValueError(f"{name}: expected [B, heads, size], got shape {tuple(t.shape)}")
    dt = _dtype(q, "q")
    B, Hk, dk = q.shape
    Hv, dv = v.shape[1:]
    _need(q, q.dtype, (B, Hk, dk), "q")
    _need(k, q.dtype, (B, Hk, dk), "k")
    _need(v, q.dtype, (B, Hv, dv), "v")
    _need(g, torch.float32, (B, Hv), "g")
    _need(beta, torch.float32, (B, Hv), "beta")
    _need(state, torch.float32, (B, Hv, dk, dv), "state")
    dev = q.device
    out = _out(out, (B, Hv, dv), q.dtype, dev, "out")
    args = (_at(dev, "q", q), _at(dev, "k", k), _at(dev, "v", v), _at(dev, "g", g), _at(dev, "beta", beta), dt, B, Hk,
            Hv, dk, dv, scale, _at(dev, "state", state), _at(dev, "out", out))
    _on(dev, lambda st: _lib.spk_delta_rule_step(*args, st))
    return out


@_with_stream
def spk_delta_rule_backward(q, k, v, g, beta, d_out, d_final_state=None, scale=1.0, initial_state=None, lengths=None,
                            d_q=None, d_k=None, d_v=None, d_g=None, d_beta=None, d_initial_state=None, workspace=None):
    """Gradients of spk_delta_rule's (out, final_state) -> (d_q, d_k, d_v, d_g, d_beta, d_initial_state or None)
    from d_out [B,L,Hv,dv] and d_final_state f32 [B,Hv,dk,dv] (None: zeros).  Rows behind a sequence's length are as in
    spk_delta_rule, and so is growth (g above 0), for any number of samples.  d_initial_state may be
    d_final_state."""
    dt, B, L, Hk, Hv, dk, dv = _delta_args(q, k, v, g, beta, lengths, initial_state)
    dev, f32, state = q.device, torch.float32, (B, Hv, dk, dv)
    _need(d_out, q.dtype, (B, L, Hv, dv), "d_out")
    if d_final_state is not None:
        _need(d_final_state, f32, state, "d_final_state")
    d_q = _rows(d_q, q, q.dtype, lengths, "d_q")
    d_k = _rows(d_k, q, q.dtype, lengths, "d_k")
    d_v = _rows(d_v, v, q.dtype, lengths, "d_v")
    d_g = _rows(d_g, g, f32, lengths, "d_g")
    d_beta = _rows(d_beta, g, f32, lengths, "d_beta")
    d_initial_state = _out(d_initial_state, state, f32, dev, "d_initial_state")
    n = spk_delta_rule_backward_workspace_size(dt, B, L, Hk, Hv, dk, dv)
    ws = _ws(workspace, n, dev)
    args = (_at(dev, "q", q), _at(dev, "k", k), _at(dev, "v", v), _at(dev, "g", g), _at(dev, "beta", beta), dt, B, L,
            Hk, Hv, dk, dv, scale, _at(dev, "lengths", lengths), _at(dev, "initial_state", initial_state),
            _at(dev, "d_out", d_out), _at(dev, "d_final_state", d_final_state), _at(dev, "d_q", d_q),
            _at(dev, "d_k", d_k), _at(dev, "d_v", d_v), _at(dev, "d_g", d_g), _at(dev, "d_beta", d_beta),
            _at(dev, "d_initial_state", d_initial_state), _at(dev, "workspace", ws), n)
    _on(dev, lambda st: _lib.spk_delta_rule_backward(*args, st))
    return d_q, d_k, d_v, d_g, d_beta, (d_initial_state if d_initial_state is not False else None)


# ---------------------------------------------------------------- drawing
def spk_sample_winners_workspace_size(dtype, B, C, H, W) -> int:
    return int(_lib.spk_sample_winners_workspace_size(dtype, B, C, H, W))


def check_draw(T, C, H, W, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Raises what spk_sample_winners raises for these settings (a call of no images: nothing is enqueued)."""
    _check(_lib.spk_sample_winners(None, SPK_F32, None, None, 0, T, C, H, W, temperature, top_k, top_p, min_p, None, None,
                                   None, 0, None))


@_with_stream
def spk_sample_winners(scores, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, t_first=None, T=1, winners=None,
                       n_winners=None, workspace=None):
    """One winner per image drawn from scores (float32 or bfloat16) [B,C,H,W] with u f32 [B] in [0, 1) ->
    (winners i32 [B,1,4] = (f,t,y,x), n_winners i32 [B]).  t_first u8 [B,C,H,W] masks the silent neurons
    (t_first >= T)."""
    if scores.dim() != 4:
        raise ValueError(f"scores: expected [B, C, H, W], got shape {tuple(scores.shape)}")
    dt = _dtype(scores, "scores")
    B, C, H, W = scores.shape
    dev = scores.device
    _need(scores, scores.dtype, (B, C, H, W), "scores")
    _need(u, torch.float32, (B,), "u")
    if t_first is not None:
        _need(t_first, torch.uint8, (B, C, H, W), "t_first")
    winners = _out(winners, (B, 1, 4), torch.int32, dev, "winners")
    n_winners = _out(n_winners, (B,), torch.int32, dev, "n_winners")
    n = spk_sample_winners_workspace_size(dt, B, C, H, W)
    ws = _ws(workspace, n, dev)
    args = (_at(dev, "scores", scores), dt, _at(dev, "t_first", t_first), _at(dev, "u", u), B, T, C, H, W, temperature,
            top_k, top_p, min_p, _at(dev, "winners", winners), _at(dev, "n_winners", n_winners),
            _at(dev, "workspace", ws), n)
    _on(dev, lambda st: _lib.spk_sample_winners(*args, st))
    return winners, n_winners
