"""Gradients of the delta rule on the GPU against the 64-bit definition's own and
against differences."""
import math

import pytest
import torch

import readout_ref as ref
from test_gpu_readout import BF16, F32, close as near, make, seeded, size_of

spk = pytest.importorskip("paper_1903_02440_amd")

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "g", "beta")


def reference(x, s0, scale, lens, d_out, d_last):
    leaf = {n: x[n].double().cpu().requires_grad_() for n in NAMES}
    s = torch.zeros(d_last.shape, dtype=torch.float64) if s0 is None else s0.double().cpu()
    s.requires_grad_()
    out, last = ref.delta_rule(**leaf, scale=scale, state=s, lengths=lens)
    return torch.autograd.grad([out, last], [*leaf.values(), s], [d_out.double().cpu(), d_last.double().cpu()])


def close(got, want, dk, dv, n, what):
    """In the 2-norm of the whole tensor: every value is a chain of sums over dk, dv and the samples whose
    roundings (2^-24 of what is summed, about (dk + dv + 16) * (n + 1) of them) have no preferred sign and are not
    amplified by the contracting rule; six standard deviations, and d_g, a difference of three such sums, four
    times that.  16-bit results are rounded once more, by half a step."""
    tol = 6 * 2.0 ** -24 * math.sqrt((dk + dv + 16) * (n + 1)) * (4 if what == "d_g" else 1)
    tol += torch.finfo(got.dtype).eps / 2
    assert torch.isfinite(got).all(), what
    err, norm = (got.double().cpu() - want).norm().item(), want.norm().item()
    assert err <= tol * norm + 1e-30, f"{what}: off by {err / max(norm, 1e-300)} of its norm, {tol} allowed"


def upstream(x, s0, seed=77):
    randn, _ = seeded(seed)
    return randn(*x["v"].shape).to(x["v"].dtype).cuda(), randn(*s0.shape).cuda()


CASES = [  # B, L, Hk, Hv, dk, dv
    (1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 5, 3), (1, 17, 2, 2, 16, 16), (2, 65, 2, 4, 31, 10), (1, 64, 1, 3, 64, 48),
    (1, 129, 1, 1, 200, 10), (2, 70, 2, 2, 128, 128), (1, 40, 1, 2, 256, 130), (1, 31, 1, 1, 129, 260),
    (1, 200, 1, 3, 72, 36),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", CASES)
def test_gradients(B, L, Hk, Hv, dk, dv, dtype):
    x, s0 = make(B, L, Hk, Hv, dk, dv, dtype, 31, features=dv == 10)
    d_out, d_last = upstream(x, s0)
    got = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, scale=0.5, initial_state=s0)
    want = reference(x, s0, 0.5, None, d_out, d_last)
    for name, a, b in zip(("d_q", "d_k", "d_v", "d_g", "d_beta", "d_state"), got, want):
        close(a, b, dk, dv, L, name)
    again = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, scale=0.5,
                                        initial_state=s0)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_gradients_of_padded_sequences(dtype):
    B, L, dk, dv = 6, 140, 40, 24
    x, s0 = make(B, L, 1, 2, dk, dv, dtype, 33)
    d_out, d_last = upstream(x, s0)
    lens = torch.tensor([0, 1, 63, 140, 65, 500], dtype=torch.int32)
    want = reference(x, s0, 1.0, lens, d_out, d_last)
    dead = (torch.arange(L)[None] >= lens[:, None]).cuda()
    bad = {n: t.clone() for n, t in x.items()}
    for t in [*bad.values(), d_out]:
        t[dead] = math.nan
    outs = {"d_" + n: torch.full_like(x[n], 7.0) for n in NAMES}
    got = spk.spk_delta_rule_backward(*(bad[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0,
                                      lengths=lens.cuda(), **outs)
    for name, a, b in zip(NAMES, got, want):
        assert bool((a[dead] == 7.0).all()), name
        a[dead] = 0.0
        close(a, b, dk, dv, L, "d_" + name)
    close(got[5], want[5], dk, dv, L, "d_state")
    assert torch.equal(got[5][0], d_last[0])
    new = spk.spk_delta_rule_backward(*(bad[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0,
                                      lengths=lens.cuda())
    assert all(torch.equal(a, b) for a, b in zip(got, new))


def test_gradient_forms():
    """No initial state, no gradient of the final one, none wanted of the initial one, in place, no samples."""
    x, s0 = make(2, 70, 1, 2, 33, 18, F32, 35)
    a = [x[n] for n in NAMES]
    d_out, d_last = upstream(x, s0)
    got = spk.spk_delta_rule_backward(*a, d_out)
    want = reference(x, None, 1.0, None, d_out, torch.zeros_like(d_last))
    for name, p, r in zip(("d_q", "d_k", "d_v", "d_g", "d_beta", "d_state"), got, want):
        close(p, r, 33, 18, 70, name)
    zero = spk.spk_delta_rule_backward(*a, d_out, initial_state=torch.zeros_like(s0),
                                       d_final_state=torch.zeros_like(s0), d_initial_state=False)
    assert zero[5] is None and all(torch.equal(p, r) for p, r in zip(got[:5], zero))
    full = spk.spk_delta_rule_backward(*a, d_out, d_final_state=d_last, initial_state=s0)
    same = d_last.clone()
    place = spk.spk_delta_rule_backward(*a, d_out, d_final_state=same, initial_state=s0, d_initial_state=same)
    assert place[5] is same and all(torch.equal(p, r) for p, r in zip(full, place))
    e = [t[:, :0].contiguous() for t in a]
    none = spk.spk_delta_rule_backward(*e, d_out[:, :0].contiguous(), d_final_state=d_last)
    assert torch.equal(none[5], d_last) and none[0].numel() == 0


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_gradients_through_gates(dtype):
    x, s0 = make(1, 150, 1, 2, 48, 20, dtype, 37)
    x["g"][0, 70:73] = -math.inf
    x["g"][0, 100] = -90.0
    x["g"][0, 120:] = 0.0
    x["beta"][0, 5:9] = 0.0
    x["beta"][0, 110:] = 1.0
    d_out, d_last = upstream(x, s0)
    got = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0)
    want = reference(x, s0, 1.0, None, d_out, d_last)
    want = [torch.nan_to_num(w) for w in want]  # (0 * inf of the definition's e^g where g is -inf)
    for name, a, b in zip(("d_q", "d_k", "d_v", "d_g", "d_beta", "d_state"), got, want):
        close(a, b, 48, 20, 150, name)


def test_gradient_against_differences():
    """Along one direction in all inputs: the central difference of the loss, in 64 bits, with h = 2^-13, is off by
    h^2 / 6 of its third derivative, which terms of order 1 keep below 2^-20 of the slope; the gradient by its own
    rounding (some 2^-24 * 2^10)."""
    x, s0 = make(1, 80, 1, 2, 24, 12, F32, 39)
    d_out, d_last = upstream(x, s0)
    got = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0)
    randn, _ = seeded(5)
    way = [randn(*t.shape).double() * 0.1 for t in (*(x[n] for n in NAMES), s0)]
    slope = sum((a.double().cpu() * w).sum().item() for a, w in zip(got, way))
    h, loss = 2.0 ** -13, []
    for sign in (1, -1):
        y = {n: x[n].double().cpu() + sign * h * w for n, w in zip(NAMES, way)}
        out, last = ref.delta_rule(**y, scale=1.0, state=s0.double().cpu() + sign * h * way[5])
        loss.append(((out * d_out.double().cpu()).sum() + (last * d_last.double().cpu()).sum()).item())
    norm = math.sqrt(sum((a.double().norm().item() * w.norm().item()) ** 2 for a, w in zip(got, way)))
    assert abs(slope - (loss[0] - loss[1]) / (2 * h)) <= 2.0 ** -14 * norm


def test_gradients_unaligned():
    x, s0 = make(2, 67, 1, 2, 64, 32, BF16, 41)
    d_out, d_last = upstream(x, s0)

    def shifted(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    a = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0)
    outs = {"d_" + n: shifted(torch.zeros_like(x[n])) for n in NAMES}
    b = spk.spk_delta_rule_backward(*(shifted(x[n]) for n in NAMES), shifted(d_out), d_final_state=shifted(d_last),
                                    initial_state=shifted(s0), d_initial_state=shifted(torch.zeros_like(s0)), **outs)
    want = reference(x, s0, 1.0, None, d_out, d_last)
    for name, p, r, w in zip(("d_q", "d_k", "d_v", "d_g", "d_beta", "d_state"), a, b, want):
        close(p, w, 64, 32, 67, name)
        close(r, w, 64, 32, 67, name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dk", [20, 64, 128, 250])
@pytest.mark.parametrize("B,dv", [(65, 40), (30, 40), (50, 10), (25, 10)])
def test_many_memories(B, dv, dk, dtype):
    """Enough heads that a tile of columns has fewer waves, and workgroups several tiles; the results of a few
    sequences, padded ones among them, against the definition on them alone."""
    L, Hk, Hv, some = 70, 2, 4, [0, 1, B // 2, B - 1]
    x, s0 = make(B, L, Hk, Hv, dk, dv, dtype, 91)
    d_out, d_last = upstream(x, s0)
    lens = torch.full((B,), L, dtype=torch.int32)
    lens[1], lens[B // 2] = 0, 33
    out, last = spk.spk_delta_rule(**x, initial_state=s0, lengths=lens.cuda())
    got = spk.spk_delta_rule_backward(*(x[n] for n in NAMES), d_out, d_final_state=d_last, initial_state=s0,
                                      lengths=lens.cuda())
    few = {n: t[some].contiguous() for n, t in x.items()}
    want, final = ref.delta_rule(**few, scale=1.0, state=s0[some], lengths=lens[some])
    m = size_of(few, s0[some], final)
    near(out[some], want, dk, L, dtype, m, "out")
    near(last[some], final, dk, L, F32, m, "state")
    grads = reference(few, s0[some], 1.0, lens[some], d_out[some], d_last[some])
    for name, a, b in zip(("d_q", "d_k", "d_v", "d_g", "d_beta", "d_state"), got, grads):
        close(a[some], b, dk, dv, L, name)
    assert all(bool(torch.isfinite(t).all()) for t in (out, last, *got))


def test_offsets_beyond_32_bits():
    """The last sequence (row) of a call whose tensors hold more than 2^32 (2^31) elements, as alone."""
    r = torch.Generator(device="cuda").manual_seed(5)
    B, L, Hv, dk, dv = 2, 33000, 16, 16, 4096
    k = torch.nn.functional.normalize(torch.randn(B, L, 1, dk, generator=r, device="cuda"), dim=-1).to(BF16)
    v = torch.randn(B, L, Hv, dv, generator=r, device="cuda", dtype=BF16)
    g, beta = -torch.rand(B, L, Hv, generator=r, device="cuda"), torch.rand(B, L, Hv, generator=r, device="cuda")
    assert v.numel() > 2 ** 32
    out, last = spk.spk_delta_rule(k, k, v, g, beta)
    alone = spk.spk_delta_rule(k[1:], k[1:], v[1:], g[1:], beta[1:])
    assert torch.equal(out[1:], alone[0]) and torch.equal(last[1:], alone[1])
    grads = spk.spk_delta_rule_backward(k, k, v, g, beta, out, d_initial_state=False)
    alone = spk.spk_delta_rule_backward(k[1:], k[1:], v[1:], g[1:], beta[1:], out[1:], d_initial_state=False)
    assert all(torch.equal(a[1:], b) for a, b in zip(grads[:5], alone[:5]))
    del v, out, grads, alone
    x = torch.randn(130, 1 << 24, 1, 1, generator=r, device="cuda", dtype=BF16)
    u = torch.rand(130, generator=r, device="cuda")
    assert x.numel() > 2 ** 31
    for kw in (dict(top_p=0.5), dict(top_k=40)):
        w, n = spk.spk_sample_winners(x, u, **kw)
        w1, _ = spk.spk_sample_winners(x[129:], u[129:], **kw)
        assert torch.equal(w[129:], w1) and bool((n == 1).all())
    torch.cuda.empty_cache()
