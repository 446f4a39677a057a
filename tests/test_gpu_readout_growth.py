"""Log decays above 0: the batch calls and the gradients serve states that grow by up to e within 64 samples and
answer more with NaN; up to 10 samples and single steps serve any finite growth."""
import math

import pytest
import torch

import readout_ref as ref
from test_gpu_readout import BF16, F32, close, make, seeded, size_of
from test_gpu_readout_grad import NAMES, close as close_grad, reference, upstream

spk = pytest.importorskip("paper_1903_02440_amd")

pytestmark = pytest.mark.gpu

GRADS = ("d_q", "d_k", "d_v", "d_g", "d_beta", "d_state")


def repeated(B, L, Hk, Hv, dk, dv, dtype, seed):
    """The same key over and over at beta = 1: the state along it is replaced, not grown, sample after sample, where
    the chunks' terms grow and cancel."""
    x, s0 = make(B, L, Hk, Hv, dk, dv, dtype, seed)
    x["k"] = x["k"][:, :1].expand(-1, L, -1, -1).contiguous()
    x["beta"] = torch.ones_like(x["beta"])
    return x, s0


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", [(1, 200, 1, 2, 40, 24), (2, 130, 2, 2, 128, 64), (1, 97, 1, 1, 200, 10)])
@pytest.mark.parametrize("keys", [repeated, make])
def test_growth_that_is_served(keys, B, L, Hk, Hv, dk, dv, dtype):
    """g = 1/64 throughout.  What is summed grows by up to e in a chunk, and once more by what multiplies it: e^2
    times the bounds of the decaying rule."""
    x, s0 = keys(B, L, Hk, Hv, dk, dv, dtype, 7)
    x["g"] = torch.full_like(x["g"], 1.0 / 64)
    out, last = spk.spk_delta_rule(**x, initial_state=s0)
    want, final = ref.delta_rule(**x, scale=1.0, state=s0)
    m = size_of(x, s0, final) * math.e ** 2
    close(out, want, dk, L, dtype, m, "out")
    close(last, final, dk, L, F32, m, "state")
    d_out, d_last = upstream(x, s0)
    got = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0)
    grads = reference(x, s0, 1.0, None, d_out, d_last)
    for name, a, b in zip(GRADS, got, grads):
        tol = 6 * 2.0 ** -24 * math.sqrt((dk + dv + 16) * (L + 1)) * (4 if name == "d_g" else 1) * math.e ** 2
        err, norm = (a.double().cpu() - b).norm().item(), b.norm().item()
        assert err <= (tol + torch.finfo(a.dtype).eps / 2) * norm, (name, err / norm, tol)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("g", [0.25, 3.0, math.inf])
def test_growth_that_is_not(dtype, g):
    """One head of one sequence grows from sample 70 on: NaN there from sample 64 on at the latest and in its state,
    everything else as if it did not; a length that ends before the growth leaves it out."""
    B, L, Hk, Hv, dk, dv = 3, 200, 1, 2, 40, 24
    x, s0 = repeated(B, L, Hk, Hv, dk, dv, dtype, 9)
    plain = spk.spk_delta_rule(**x, initial_state=s0)
    d_out, d_last = upstream(x, s0)
    a = [x[n] for n in NAMES]
    grads = spk.spk_delta_rule_backward(*a, d_out, d_final_state=d_last, initial_state=s0)
    x["g"] = x["g"].clone()
    x["g"][1:, 70:150, 1] = g
    lens = torch.tensor([L, L, 70], dtype=torch.int32).cuda()
    out, last = spk.spk_delta_rule(**x, initial_state=s0, lengths=lens)
    assert bool(out[1, 150:, 1].isnan().all()) and bool(last[1, 1].isnan().all())
    assert torch.equal(out[1, :64, 1], plain[0][1, :64, 1]) and torch.equal(out[1, :, 0], plain[0][1, :, 0])
    assert torch.equal(out[0], plain[0][0]) and torch.equal(last[0], plain[1][0]) and torch.equal(last[1, 0], plain[1][1, 0])
    assert torch.equal(out[2, :64], plain[0][2, :64]) and bool(torch.isfinite(last[2]).all())
    a[3] = x["g"]
    got = spk.spk_delta_rule_backward(*a, d_out, d_final_state=d_last, initial_state=s0, lengths=lens)
    for name, t, p in zip(GRADS, got, grads):
        assert torch.equal(t[0], p[0]) and bool(torch.isfinite(t[2]).all()), name
        assert name in ("d_q", "d_state") or bool(t[1, :64].isnan().any()), name
    assert bool(got[5][1, 1].isnan().all()) and torch.equal(got[5][1, 0], grads[5][1, 0])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("g", [0.25, 2.0])
def test_growth_sample_by_sample(dtype, g):
    """Ten samples and single steps, from zero states.  A rounding of the state is multiplied by e^g at each later
    sample, but for its part along the repeated key, which is replaced: off by up to the sum of e^(g j), j < L, below
    e^(g (L - 1)) / (1 - e^-g), times the decaying rule's bound.  What is stored along the key takes the last samples'
    roundings only, of the state as it is by then, grown once."""
    B, L, Hk, Hv, dk, dv = 2, 10, 1, 2, 40, 24
    x, s0 = repeated(B, L, Hk, Hv, dk, dv, dtype, 11)
    x["g"] = torch.full_like(x["g"], g)
    s0 = torch.zeros_like(s0)
    out, last = spk.spk_delta_rule(**x, initial_state=s0)
    want, final = ref.delta_rule(**x, scale=1.0, state=s0)
    m = size_of(x, None, final) * math.exp(g)  # (the state is grown before what is along the key is replaced)
    grown = m * math.exp(g * (L - 1)) / (1 - math.exp(-g))
    state = s0.clone()
    outs = [spk.spk_delta_rule_step(*(x[n][:, t].contiguous() for n in NAMES), state) for t in range(L)]
    key = x["k"][:, 0].double().cpu()  # (of 16 bits: its norm is off 1 by 2^-8, which leaves e^g 2^-8 of earlier roundings)
    for o, s in ((out, last), (torch.stack(outs, 1), state)):
        close(o, want, dk, L, dtype, grown, "out")
        close(s, final, dk, L, F32, grown, "state")
        along = [torch.einsum("bhk,bhkv->bhv", key.expand(-1, Hv, -1), t.double().cpu()) for t in (s, final)]
        bound = 6 * 2.0 ** -24 * math.sqrt((dk + 16) * 2) * 2 * math.exp(g) * size_of(x, s, final)
        assert bool(((along[0] - along[1]).abs() <= bound).all())
