"""The readout operators' C ABI and binding: symbols, and bad arguments rejected
on the host before any HIP call -- CPU only."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import readout_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "libspyke_readout.h")

spk = pytest.importorskip("paper_1903_02440_amd")

P = ctypes.c_void_p(0x1000)  # never dereferenced: every call fails validation first


def test_every_declared_symbol_is_bound():
    names = re.findall(r"^SPK_API\s+[\w\s\*]*?\b(spk_\w+)\s*\(", open(HEADER).read(), flags=re.M)
    from paper_1903_02440_amd import readout
    assert names and sorted(names) == sorted(readout._SIGS)
    for n in names:
        assert hasattr(spk.lib(), n) and hasattr(spk, n)


def _rule(dtype=0, B=2, L=5, Hk=2, Hv=4, dk=8, dv=6, scale=1.0, q=P, out=P, ws=P, n=1 << 40):
    return spk.lib().spk_delta_rule(q, P, P, P, P, dtype, B, L, Hk, Hv, dk, dv, scale, None, None, out, P, ws, n, None)


def _step(dtype=0, B=2, Hk=2, Hv=4, dk=8, dv=6, scale=1.0, state=P):
    return spk.lib().spk_delta_rule_step(P, P, P, P, P, dtype, B, Hk, Hv, dk, dv, scale, state, P, None)


@pytest.mark.parametrize("call", [_rule, _step], ids=["rule", "step"])
def test_delta_refusals(call):
    assert call(dtype=2) == spk.SPK_E_ARG and b"SPK_BF16" in spk.lib().spk_last_error()
    assert call(dk=0) == spk.SPK_E_SHAPE
    assert call(dv=0) == spk.SPK_E_SHAPE
    assert call(Hk=0) == spk.SPK_E_SHAPE
    assert call(Hv=3) == spk.SPK_E_SHAPE
    assert call(B=-1) == spk.SPK_E_SHAPE
    assert call(dk=257) == spk.SPK_E_RANGE
    assert call(dv=4097) == spk.SPK_E_RANGE
    assert call(B=16385) == spk.SPK_E_RANGE
    assert call(scale=math.inf) == spk.SPK_E_ARG
    assert call(scale=math.nan) == spk.SPK_E_ARG
    assert call(B=0) == spk.SPK_OK


def test_delta_buffers():
    assert _rule(L=-1) == spk.SPK_E_SHAPE
    assert _rule(L=(1 << 24) + 1, B=1) == spk.SPK_E_RANGE
    assert _rule(q=None) == spk.SPK_E_ARG
    assert _rule(out=None) == spk.SPK_E_ARG
    assert _step(state=None) == spk.SPK_E_ARG


def _draw(dtype=0, B=2, T=1, C=10, H=1, W=1, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=P, scores=P, ws=P,
          n=1 << 40):
    return spk.lib().spk_sample_winners(scores, dtype, None, u, B, T, C, H, W, temperature, top_k, top_p, min_p, P, P,
                                        ws, n, None)


def test_sample_refusals():
    assert _draw(dtype=7) == spk.SPK_E_ARG
    assert _draw(C=0) == spk.SPK_E_SHAPE
    assert _draw(T=0) == spk.SPK_E_SHAPE
    assert _draw(T=256) == spk.SPK_E_RANGE
    assert _draw(C=(1 << 24) + 1) == spk.SPK_E_RANGE
    assert _draw(C=1 << 16, H=1 << 15, W=1 << 15) == spk.SPK_E_RANGE
    for t in (-1.0, math.inf, math.nan):
        assert _draw(temperature=t) == spk.SPK_E_ARG
    assert _draw(top_k=-1) == spk.SPK_E_ARG
    for p in (0.0, -0.5, 1.5, math.nan):
        assert _draw(top_p=p) == spk.SPK_E_ARG
    for p in (-0.1, 1.1, math.nan):
        assert _draw(min_p=p) == spk.SPK_E_ARG
    assert _draw(u=None) == spk.SPK_E_ARG
    assert _draw(scores=None) == spk.SPK_E_ARG
    assert _draw(B=0, scores=None, u=None) == spk.SPK_OK


def test_binding_refuses_before_the_call():
    z = torch.zeros
    with pytest.raises(TypeError):  # half precision has no kernel
        spk.spk_sample_winners(z(2, 3, 1, 1, dtype=torch.float16), z(2))
    with pytest.raises(ValueError, match="device tensor"):
        spk.spk_sample_winners(z(2, 3, 1, 1), z(2))
    with pytest.raises(ValueError, match="scores"):
        spk.spk_sample_winners(z(2, 3), z(2))
    with pytest.raises(ValueError, match="q: expected"):
        spk.spk_delta_rule(z(2, 3, 4), z(2, 3, 4), z(2, 3, 4), z(2, 3), z(2, 3))
    with pytest.raises(TypeError):
        spk.spk_delta_rule_step(z(2, 3, 4, dtype=torch.float64), z(2, 3, 4), z(2, 3, 4), z(2, 3), z(2, 3),
                                z(2, 3, 4, 4))


def test_reference_of_one_sample():
    """The reference itself: one sample by hand (S = [[2],[0]], k = (1,0), v = 5, e^g = 1/2, beta = 1/2)."""
    one = torch.ones(1, 1, 1)
    out, s = ref.delta_rule(torch.tensor([[[[1.0, 1.0]]]]), torch.tensor([[[[1.0, 0.0]]]]), 5 * one[..., None],
                            math.log(0.5) * one, 0.5 * one, 2.0, torch.tensor([[[[2.0], [0.0]]]]))
    # S -> (1, 0); u = (5 - 1) / 2 = 2; S -> (3, 0); out = 2 * 3
    assert s.flatten().tolist() == pytest.approx([3.0, 0.0], abs=1e-6) and out.item() == pytest.approx(6.0, abs=1e-6)


def test_reference_of_a_draw():
    x = np.log(np.array([[1.0, 4.0, 2.0, 1.0]])).reshape(1, 4, 1, 1)
    for u, f in ((0.0, 0), (0.1, 0), (0.2, 1), (0.6, 1), (0.65, 2), (0.9, 3), (1.5, 3), (math.nan, 0)):
        assert ref.sample_winners(x, [u])[0][0, 0, 0] == f
    assert ref.sample_winners(x, [0.99], top_k=3)[0][0, 0, 0] == 2  # the later of two equal scores goes
    assert ref.sample_winners(x, [0.0], top_p=0.7)[0][0, 0, 0] == 1
    assert ref.sample_winners(x, [0.99], min_p=0.3)[0][0, 0, 0] == 2


def _back(dtype=0, B=2, L=5, Hk=2, Hv=4, dk=8, dv=6, scale=1.0, q=P, dq=P, ws=P, n=1 << 40):
    return spk.lib().spk_delta_rule_backward(q, P, P, P, P, dtype, B, L, Hk, Hv, dk, dv, scale, None, None, P, None, dq,
                                             P, P, P, P, None, ws, n, None)


def test_backward_refusals():
    assert _back(dtype=2) == spk.SPK_E_ARG
    assert _back(dk=0) == spk.SPK_E_SHAPE
    assert _back(Hv=3) == spk.SPK_E_SHAPE
    assert _back(L=-1) == spk.SPK_E_SHAPE
    assert _back(dk=257) == spk.SPK_E_RANGE
    assert _back(dv=4097) == spk.SPK_E_RANGE
    assert _back(B=16385) == spk.SPK_E_RANGE
    assert _back(scale=math.nan) == spk.SPK_E_ARG
    assert _back(q=None) == spk.SPK_E_ARG
    assert _back(dq=None) == spk.SPK_E_ARG
    assert _back(ws=None) == spk.SPK_E_WORKSPACE
    assert _back(n=1024) == spk.SPK_E_WORKSPACE and b"needed" in spk.lib().spk_last_error()
    assert _back(B=0) == spk.SPK_OK
    assert _rule(L=500, ws=None) == spk.SPK_E_WORKSPACE
    assert _rule(L=500, n=64) == spk.SPK_E_WORKSPACE


def test_workspace_sizes():
    size, back = spk.spk_delta_rule_workspace_size, spk.spk_delta_rule_backward_workspace_size
    assert size(0, 2, 1, 1, 2, 64, 64) == 0  # a few samples run one after another
    assert 0 < size(1, 2, 500, 1, 2, 64, 64) < size(1, 4, 500, 1, 2, 64, 64)
    assert size(1, 2, 500, 1, 3, 64, 64) > size(1, 2, 500, 1, 1, 64, 64)
    assert size(5, 2, 500, 1, 2, 64, 64) == 0 and size(0, 2, 500, 2, 3, 64, 64) == 0
    # the states of every chunk, twice, and two rows a sample
    assert back(0, 1, 320, 1, 1, 64, 64) >= 4 * (2 * 10 * 64 * 64 + 2 * 320 * 64)
    assert back(0, 0, 320, 1, 1, 64, 64) == 0 and back(0, 1, 0, 1, 1, 64, 64) == 0


def test_workspaces_on_16_bytes():
    odd = ctypes.c_void_p(0x1008)
    assert _rule(L=500, ws=odd) == spk.SPK_E_ARG and b"aligned" in spk.lib().spk_last_error()
    assert _back(ws=odd) == spk.SPK_E_ARG and b"aligned" in spk.lib().spk_last_error()
    assert _draw(C=50000, ws=odd) == spk.SPK_E_ARG and b"aligned" in spk.lib().spk_last_error()
    assert _draw(C=50000, n=64) == spk.SPK_E_WORKSPACE
    assert spk.spk_sample_winners_workspace_size(0, 2, 10, 1, 1) == 0
    assert 0 < spk.spk_sample_winners_workspace_size(0, 2, 50000, 1, 1) < spk.spk_sample_winners_workspace_size(
        0, 4, 50000, 1, 1)


def test_large_counts_are_refused():
    assert _draw(B=(1 << 21) + 1) == spk.SPK_E_RANGE
    assert _draw(B=65536, C=16385) == spk.SPK_E_RANGE
    assert _rule(B=1, Hk=1, Hv=2048, dv=4096) == spk.SPK_E_RANGE  # rows of more than 2^22 values


def test_stream_of_another_device_is_refused():
    class Other:
        device = torch.device("cuda", 1)
    z = torch.zeros
    with pytest.raises(ValueError, match="stream on cuda:1"):
        spk.spk_sample_winners(z(2, 3, 1, 1), z(2), stream=Other)
    with pytest.raises(ValueError, match="stream on cuda:1"):
        spk.spk_delta_rule(q=z(2, 3, 1, 4), k=z(2, 3, 1, 4), v=z(2, 3, 1, 4), g=z(2, 3, 1), beta=z(2, 3, 1), stream=Other)
