"""The batch calls' products hold what float holds: cases in which fewer bits show."""
import math

import pytest
import torch

import readout_ref as ref
from test_gpu_readout import BF16, F32, seeded

spk = pytest.importorskip("paper_1903_02440_amd")

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,Hv,dk,dv,L", [(1, 1, 64, 16, 64), (1, 1, 250, 10, 70), (2, 4, 128, 128, 130),
                                          (1, 16, 256, 256, 90), (64, 4, 32, 40, 33), (64, 4, 200, 70, 33)])
def test_what_was_stored_is_read_back_over_a_large_state(B, Hv, dk, dv, L, dtype):
    """Keys are unit vectors e_0, e_1, ... in turn, queries the keys, beta = 1, no decay: out_t = v_t by the
    definition, and in chunks the sum of S[t] and v_t - S[t], which cancel.  S is 2^10 times the values.  The
    difference is rounded once, a second one for a row that a chunk meets twice is a sum of up to six products, and
    the sum takes the three terms of each: below sixteen roundings by 2^-24 of |S[t]| + |v_t|, besides the half step
    of a 16-bit result.  (A state or difference of two terms would be off by 2^-17 of it.)"""
    randn, _ = seeded(101)
    S = randn(B, Hv, dk, dv) * 1024
    at = torch.arange(L) % dk
    k = torch.nn.functional.one_hot(at, dk).to(dtype)[None, :, None].repeat(B, 1, 1, 1)
    v = randn(B, L, Hv, dv).to(dtype)
    g, beta = torch.zeros(B, L, Hv), torch.ones(B, L, Hv)
    out, last = spk.spk_delta_rule(k.cuda(), k.cuda(), v.cuda(), g.cuda(), beta.cuda(), initial_state=S.cuda())
    want, final = ref.delta_rule(k, k, v, g, beta, 1.0, S)
    was = S.double()[:, :, at].transpose(1, 2).abs()  # (rows met again hold a value by then: smaller)
    tol = 16 * 2.0 ** -24 * (was + want.abs())
    half = torch.finfo(dtype).eps / 2
    err = (out.double().cpu() - want).abs()
    assert bool((err <= tol + half * (want.abs() + tol)).all()), float((err - tol - half * want.abs()).max())
    err = (last.double().cpu() - final).abs()
    assert bool((err <= 16 * 2.0 ** -24 * (S.double().abs() + final.abs() + 8)).all())


def worst():
    """A number whose second and third bfloat16 terms are as large as they get when each is cut off, not rounded."""
    return 1 + 2.0 ** -7 - 2.0 ** -23


@pytest.mark.parametrize("dk", [1, 40, 200])
def test_float_products(dk):
    """beta = 0 and no decay: out_t = q_t . S, one product here, of floats held as sums of three bfloat16 terms.  The
    products of terms that are made are exact, and adding them rounds: the sums before the last are below 2^-5 of
    the product, so all roundings together are below 2^-23 of it; 2^-22 leaves as much again for products of terms
    that are not made.  (Of terms that are cut off, not rounded, these are 2^-21 here.)"""
    B, L, dv = 1, 40, 20
    q = torch.zeros(B, L, 1, dk)
    q[..., dk // 2] = worst()
    S = torch.zeros(B, 1, dk, dv)
    S[:, :, dk // 2] = worst() * 2.0 ** torch.arange(dv)
    zero = torch.zeros(B, L, 1)
    out, last = spk.spk_delta_rule(q.cuda(), q.cuda(), torch.zeros(B, L, 1, dv).cuda(), zero.cuda(), zero.cuda(),
                                   initial_state=S.cuda())
    want = (q.double() @ S.double()[:, 0]).reshape(out.shape)
    assert bool(((out.double().cpu() - want).abs() <= 2.0 ** -22 * want).all())
    assert torch.equal(last.cpu(), S)


def test_float_values_up_to_the_largest():
    """The terms of the largest floats are finite: the states and queries up to the type's end give finite products."""
    B, L, dk, dv = 1, 33, 4, 5
    q = torch.zeros(B, L, 1, dk)
    q[:, :, :, 1] = torch.finfo(F32).max
    k = torch.zeros(B, L, 1, dk)
    k[..., 0] = 1.0
    S = torch.full((B, 1, dk, dv), 2.0 ** -10)
    S[:, :, 2] = torch.finfo(F32).max
    zero = torch.zeros(B, L, 1)
    out, last = spk.spk_delta_rule(q.cuda(), k.cuda(), torch.zeros(B, L, 1, dv).cuda(), zero.cuda(), zero.cuda(),
                                   initial_state=S.cuda())
    want = torch.full((B, L, 1, dv), torch.finfo(F32).max * 2.0 ** -10, dtype=torch.float64)
    assert bool(((out.double().cpu() - want).abs() <= 2.0 ** -22 * want).all())
    assert torch.equal(last.cpu(), S)
