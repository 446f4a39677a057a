"""The readout operators on the GPU against plain 64-bit forms."""
import math

import numpy as np
import pytest
import torch

import readout_ref as ref

spk = pytest.importorskip("paper_1903_02440_amd")

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def seeded(seed):
    r = torch.Generator().manual_seed(seed)
    return lambda *s: torch.randn(s, generator=r), lambda *s: torch.rand(s, generator=r)


def make(B, L, Hk, Hv, dk, dv, dtype, seed=0, features=False):
    """Inputs of unit key norm, rates in (0, 1) and decays below 1: the rule contracts."""
    randn, rand = seeded(seed)
    k, q = randn(B, L, Hk, dk), randn(B, L, Hk, dk)
    if features:
        k, q = k.clamp(min=0), q.clamp(min=0)
    k, q = (x / x.norm(dim=-1, keepdim=True).clamp(min=1e-6) for x in (k, q))
    x = [k.to(dtype), q.to(dtype), randn(B, L, Hv, dv).to(dtype)]
    return dict(q=x[1].cuda(), k=x[0].cuda(), v=x[2].cuda(), g=-torch.exp(rand(B, L, Hv) * 7 - 8).cuda(),
                beta=torch.sigmoid(randn(B, L, Hv)).cuda()), randn(B, Hv, dk, dv).cuda()


def close(got, want, dk, n, dtype, size, what, extra=0.0):
    """Rounding only.  A value is a sum over dk or the samples; each of about
    (dk + 16) * (n + 1) roundings is off by at most 2^-24 of the size of what is
    summed, with no preferred sign, and the rule with keys of norm 1 and rates
    below 1 does not amplify earlier errors: six standard deviations of their sum.
    A result of 16 bits is rounded once more, by half its step.  `extra`: what
    else the case adds, as a share of `size`."""
    tol = (6 * 2.0 ** -24 * math.sqrt((dk + 16) * (n + 1)) + extra) * size
    half = torch.finfo(dtype).eps / 2
    err = (got.double().cpu() - want).abs()
    bound = tol + half * (want.abs() + tol)
    assert got.dtype == dtype and torch.isfinite(got).all(), what
    assert bool((err <= bound).all()), f"{what}: off by {float((err - bound).max())} over the bound {float(tol)}"


def size_of(x, state, final):
    """The largest column of the memories, or value: what the sums add up."""
    cols = [s.double().norm(dim=2).max().item() for s in (state, final) if s is not None and s.numel()]
    return max(cols + [x["v"].abs().max().item() if x["v"].numel() else 0.0]) * 2


CASES = [  # B, L, Hk, Hv, dk, dv
    (1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 5, 3), (1, 17, 2, 2, 16, 16), (2, 65, 2, 4, 31, 10), (1, 64, 1, 3, 64, 48),
    (1, 129, 1, 1, 200, 10), (3, 70, 2, 2, 128, 128), (1, 40, 1, 2, 256, 130), (2, 33, 1, 1, 250, 20),
    (1, 200, 2, 6, 72, 36), (1, 31, 1, 1, 129, 260), (1, 300, 1, 1, 32, 32),
]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,L,Hk,Hv,dk,dv", CASES)
def test_delta_rule(B, L, Hk, Hv, dk, dv, dtype):
    x, s0 = make(B, L, Hk, Hv, dk, dv, dtype, features=dv == 10)
    out, last = spk.spk_delta_rule(**x, scale=0.5, initial_state=s0)
    want, final = ref.delta_rule(**x, scale=0.5, state=s0)
    m = size_of(x, s0, final)
    close(out, want, dk, L, dtype, m, "out")
    close(last, final, dk, L, F32, m, "state")
    again = spk.spk_delta_rule(**x, scale=0.5, initial_state=s0)
    assert torch.equal(out, again[0]) and torch.equal(last, again[1])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_delta_rule_of_padded_sequences(dtype):
    B, L, Hk, Hv, dk, dv = 7, 140, 1, 2, 40, 24
    x, s0 = make(B, L, Hk, Hv, dk, dv, dtype, 3)
    lens = torch.tensor([0, 1, 63, 64, 140, 65, 500], dtype=torch.int32)
    want, final = ref.delta_rule(**x, scale=1.0, state=s0, lengths=lens)
    # rows behind a sequence's length hold what no kernel may read or touch
    dead = torch.arange(L)[None] >= lens[:, None]
    bad = {n: t.clone() for n, t in x.items()}
    for t in bad.values():
        t[dead.cuda()] = math.nan
    out = torch.full_like(x["v"], 7.0)
    _, last = spk.spk_delta_rule(**bad, initial_state=s0, lengths=lens.cuda(), out=out)
    assert bool((out[dead.cuda()] == 7.0).all())
    m = size_of(x, s0, final)
    want[dead] = 7.0
    close(out, want, dk, L, dtype, m, "out")
    close(last, final, dk, L, F32, m, "state")
    assert torch.equal(last[0], s0[0])
    new, _ = spk.spk_delta_rule(**bad, initial_state=s0, lengths=lens.cuda())
    assert bool((new[dead.cuda()] == 0.0).all()) and torch.equal(new[~dead.cuda()], out[~dead.cuda()])


def test_delta_rule_forms():
    """No initial state, no final state, the state in place, no samples."""
    x, s0 = make(2, 70, 1, 2, 33, 18, F32, 5)
    out, last = spk.spk_delta_rule(**x, initial_state=s0)
    same = s0.clone()
    o2, l2 = spk.spk_delta_rule(**x, initial_state=same, final_state=same)
    assert l2 is same and torch.equal(same, last) and torch.equal(o2, out)
    o3, l3 = spk.spk_delta_rule(**x, initial_state=s0, final_state=False)
    assert l3 is None and torch.equal(o3, out)
    zo, zl = spk.spk_delta_rule(**x)
    ro, rl = spk.spk_delta_rule(**x, initial_state=torch.zeros_like(s0))
    assert torch.equal(zo, ro) and torch.equal(zl, rl)
    e = {n: t[:, :0].contiguous() for n, t in x.items()}
    o, l = spk.spk_delta_rule(**e, initial_state=s0)
    assert o.numel() == 0 and torch.equal(l, s0)
    assert bool((spk.spk_delta_rule(**e)[1] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_delta_rule_gates(dtype):
    """Forgetting of all (g = -inf), of next to nothing and of nothing, rates of 0 and 1."""
    x, s0 = make(1, 150, 1, 2, 48, 20, dtype, 9)
    x["g"][0, 70:73] = -math.inf
    x["g"][0, 100] = -90.0
    x["g"][0, 101] = -1e30
    x["g"][0, 120:] = 0.0
    x["beta"][0, 5:9] = 0.0
    x["beta"][0, 110:] = 1.0
    out, last = spk.spk_delta_rule(**x, initial_state=s0)
    want, final = ref.delta_rule(**x, scale=1.0, state=s0)
    m = size_of(x, s0, final)
    close(out, want, 48, 150, dtype, m, "out")
    close(last, final, 48, 150, F32, m, "state")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,Hk,Hv,dk,dv", [(1, 1, 1, 1, 1), (3, 2, 4, 7, 5), (2, 1, 8, 250, 10), (4, 2, 4, 128, 128),
                                           (1, 1, 1, 256, 300), (5, 3, 3, 100, 36), (1, 2, 2, 17, 130), (2, 1, 2, 70, 129),
                                           (1, 1, 1, 256, 3), (2, 2, 2, 30, 131), (3, 1, 1, 200, 257)])
def test_delta_step(B, Hk, Hv, dk, dv, dtype):
    """Sample after sample with the state in place, against the batch definition."""
    L = 6
    x, s0 = make(B, L, Hk, Hv, dk, dv, dtype, 11)
    state = s0.clone()
    outs = [spk.spk_delta_rule_step(*(x[n][:, t].contiguous() for n in ("q", "k", "v", "g", "beta")), state, scale=2.0)
            for t in range(L)]
    want, final = ref.delta_rule(**x, scale=2.0, state=s0)
    m = 2 * size_of(x, s0, final)
    close(torch.stack(outs, 1), want, dk, L, dtype, m, "out")
    close(state, final, dk, L, F32, m, "state")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_delta_unaligned(dtype):
    """Tensors that start one element into their allocation give the same values."""
    x, s0 = make(2, 67, 1, 2, 64, 32, dtype, 13)

    def shifted(t):
        flat = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    out, last = spk.spk_delta_rule(**x, initial_state=s0)
    o2, l2 = torch.empty(out.numel() + 1, dtype=dtype, device="cuda"), torch.empty(last.numel() + 1, device="cuda")
    o2, l2 = o2[1:].view(out.shape), l2[1:].view(last.shape)
    spk.spk_delta_rule(**{n: shifted(t) for n, t in x.items()}, initial_state=shifted(s0), out=o2, final_state=l2)
    want, final = ref.delta_rule(**x, scale=1.0, state=s0)
    m = size_of(x, s0, final)
    close(o2, want, 64, 67, dtype, m, "out")
    close(l2, final, 64, 67, F32, m, "state")
    st, s2 = s0.clone(), shifted(s0)
    one = {n: t[:, 0].contiguous() for n, t in x.items()}
    a = spk.spk_delta_rule_step(**one, state=st)
    b = spk.spk_delta_rule_step(**{n: shifted(t) for n, t in one.items()}, state=s2)
    want, final = ref.delta_rule(**{n: t[:, :1] for n, t in x.items()}, scale=1.0, state=s0)
    for o, s in ((a, st), (b, s2)):
        close(o, want[:, 0], 64, 1, dtype, m, "out")
        close(s, final, 64, 1, F32, m, "state")


# ---------------------------------------------------------------- drawing
def check_draw(scores, u, **kw):
    tf = kw.get("t_first")
    got = spk.spk_sample_winners(scores.cuda(), u.cuda(), **{**kw, "t_first": None if tf is None else tf.cuda()})
    want = ref.sample_winners(scores.double().numpy(), u.numpy(),
                              **{**kw, "t_first": None if tf is None else tf.numpy()})
    np.testing.assert_array_equal(got[0].cpu().numpy(), want[0])
    np.testing.assert_array_equal(got[1].cpu().numpy(), want[1])


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.5, top_k=1), dict(top_k=7), dict(top_p=0.75),
            dict(min_p=0.25), dict(temperature=2.0, top_k=50, top_p=0.9375, min_p=0.03125),
            dict(temperature=0.25, top_k=20, top_p=0.5)]


@pytest.mark.parametrize("kw", SETTINGS, ids=[str(i) for i in range(len(SETTINGS))])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,C,H,W", [(3, 1, 1, 1), (4, 10, 1, 1), (7, 65, 3, 5), (2, 200, 4, 4), (3, 33001, 1, 1)])
def test_sample_winners(B, C, H, W, dtype, kw):
    """bfloat16 scores hold many equal ones: their order by index shows in every boundary."""
    randn, rand = seeded(C + H)
    check_draw((randn(B, C, H, W) * 2).to(dtype), rand(B), **kw)


@pytest.mark.parametrize("kw", SETTINGS, ids=[str(i) for i in range(len(SETTINGS))])
def test_sample_of_masked_neurons(kw):
    randn, rand = seeded(4)
    x = randn(9, 30, 5, 3)
    tf = torch.where(rand(9, 30, 5, 3) < 0.5, 3, 4).to(torch.uint8)
    tf[2] = 4        # no neuron fired
    tf[3] = 255
    tf[4, 1:] = 4    # one map
    x[5] = -math.inf  # nothing to draw
    x[6, :29] = math.nan
    x[7, 3:6] = math.inf  # they share the draw
    tf[7, 4] = 0
    x[8] = torch.finfo(F32).min  # the type's lowest is a score like others
    check_draw(x, rand(9), t_first=tf, T=4, **kw)


def test_sample_of_equal_scores_and_ends_of_u():
    x = torch.zeros(6, 40, 1, 1)
    x[3:] = -3.0
    u = torch.tensor([0.0, 0.5, 1.0 - 2.0 ** -24, 1.0, math.nan, -2.0])
    for kw in (dict(), dict(top_k=8), dict(top_p=0.5), dict(top_k=16, top_p=0.25), dict(min_p=1.0)):
        check_draw(x, u, **kw)


def test_sample_of_long_rows():
    """Rows beyond what a workgroup keeps, one and several; an odd length."""
    randn, rand = seeded(8)
    for B, C in ((1, 131072), (5, 70001), (1, 1 << 20)):
        x, u = randn(B, C, 1, 1) * 3, rand(B)
        got = [spk.spk_sample_winners(x.cuda(), u.cuda(), temperature=0.75, top_k=k, top_p=0.9375)
               for k in (0, 50, 3000)]
        for k, (w, n) in zip((0, 50, 3000), got):
            v, order = x.double().reshape(B, -1).sort(dim=1, descending=True, stable=True)
            e = torch.exp((v - v[:, :1]) / 0.75)
            e[:, k or C:] = 0
            c = e.cumsum(1)
            e = torch.where(c - e < 0.9375 * c[:, -1:], e, 0.0)
            e = torch.zeros_like(e).scatter_(1, order, e)
            c = e.cumsum(1)
            at = (c <= u.double()[:, None] * c[:, -1:]).sum(1)
            assert torch.equal(w[:, 0, 0].cpu().long(), at) and bool((n == 1).all())


def in_order(x, u, temperature, top_k, top_p, min_p):
    """The definition on whole rows at once (x f64 [B,N], -inf = cannot win), in 64 bits."""
    v, order = x.sort(dim=1, descending=True, stable=True)
    e = torch.where(v == v[:, :1], 1.0, torch.exp((v - v[:, :1]) / temperature))
    e[:, top_k or x.shape[1]:] = 0
    c = e.cumsum(1)
    e = torch.where((c - e < top_p * c[:, -1:]) & (e >= min_p), e, 0.0)
    e = torch.zeros_like(e).scatter_(1, order, e)
    c = e.cumsum(1)
    return (c <= u.double()[:, None] * c[:, -1:]).sum(1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,C,H,W", [(3, 50001, 1, 1), (2, 333, 9, 17), (700, 16385, 1, 1)])
def test_sample_of_long_masked_rows(B, C, H, W, dtype):
    """Rows of several workgroups, of odd lengths (so that every row starts at another alignment), with silent
    neurons; scores of few steps, so that a boundary's bin holds more equal ones than LDS takes."""
    randn, rand = seeded(B)
    N = C * H * W
    fine = (randn(B, C, H, W) * 3).to(dtype)
    for x in (fine, (fine.float() * 2).round().to(dtype) / 2):
        u = rand(B)
        tf = torch.where(rand(B, C, H, W) < 0.5, 6, 7).to(torch.uint8)
        tf[0] = 7
        flat = torch.where(tf < 7, x.double(), -math.inf).reshape(B, N)
        some = flat.max(1).values > -math.inf
        for kw in (dict(top_p=0.75), dict(temperature=5.0, top_p=0.5, min_p=0.25), dict(top_k=40), dict(),
                   dict(top_k=9000, top_p=0.9375), dict(temperature=0.5, top_k=60, top_p=0.5, min_p=0.125),
                   dict(top_k=N - 1, top_p=0.875)):
            w, n = spk.spk_sample_winners(x.cuda(), u.cuda(), t_first=tf.cuda(), T=7, **kw)
            at = in_order(flat.cuda(), u.cuda(), **{"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, **kw})
            at = at.clamp(max=N - 1).cpu()
            want = torch.stack([at // (H * W), torch.full_like(at, 6), at // W % H, at % W], 1)
            want = torch.where(some[:, None], want, -1)
            assert torch.equal(w[:, 0].cpu().long(), want) and torch.equal(n.cpu().bool(), some), kw


def test_sample_of_long_rows_at_the_ends():
    """All equal, all masked, infinities, the type's lowest value, greedy; u at its ends."""
    N = 40000
    x = torch.zeros(8, N, 1, 1)
    x[1] = -math.inf
    x[2] = math.nan
    x[3, 7:9] = math.inf
    x[4] = torch.finfo(F32).min
    x[5, 1:] = torch.finfo(F32).min
    x[6] = -0.0
    x[6, 20000:] = 0.0
    x[7, ::2] = -1e30
    u = torch.tensor([1.0 - 2.0 ** -24, 0.5, 0.5, 0.75, 0.5, 0.999, 1.0, math.nan])
    first = lambda kw: spk.spk_sample_winners(x.cuda(), u.cuda(), **kw)[0][:, 0, 0].tolist()  # noqa: E731
    assert first(dict()) == [N - 1, -1, -1, 8, N // 2, 0, N - 1, 1]
    assert first(dict(temperature=0.0)) == [0, -1, -1, 7, 0, 0, 0, 1]
    assert first(dict(top_k=2)) == [1, -1, -1, 8, 1, 0, 1, 1]
    assert first(dict(top_p=0.5)) == [N // 2 - 1, -1, -1, 7, N // 4, 0, N // 2 - 1, 1]


# ---------------------------------------------------------------- together
def test_readout_learns_draws_and_rewards():
    """As a program uses them: a layer's potentials as features, a readout learnt over the images in order,
    decisions drawn from its scores, and the reward they earn fed to the reward-modulated update."""
    B, C, classes, T = 40, 20, 10, 15
    randn, rand = seeded(21)
    tf = torch.where(rand(B, C, 2, 2) < 0.7, T - 1, T).to(torch.uint8).cuda()
    vf = (randn(B, C, 2, 2).abs() * 3).cuda() * (tf < T)
    feat = spk.spk_pool_potentials(vf[:, None].contiguous(), 2).reshape(B, C)
    key = (feat / feat.norm(dim=1, keepdim=True).clamp(min=1e-6)).reshape(1, B, 1, C)
    labels = torch.randint(0, classes, (B,), generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda()
    v = torch.nn.functional.one_hot(labels.long(), classes).float().reshape(1, B, 1, classes)
    g, beta = torch.zeros(1, B, 1).cuda(), torch.full((1, B, 1), 0.5).cuda()
    scores, S = spk.spk_delta_rule(key, key, v, g, beta)
    step = torch.zeros_like(S)
    for t in range(B):
        o = spk.spk_delta_rule_step(key[:, t], key[:, t], v[:, t], g[:, t], beta[:, t], step)
        want = scores[:, t].double().cpu()
        close(o, want, C, B, F32, 2.0, "step against batch")
    close(step, S.double().cpu(), C, B, F32, 2.0, "state of the steps")
    u = rand(B).cuda()
    win, nw = spk.spk_sample_winners(scores.reshape(B, classes, 1, 1), u, temperature=0.25, top_p=0.9375)
    rwin, rnw = ref.sample_winners(scores.reshape(B, classes, 1, 1).double().cpu().numpy(), u.cpu().numpy(),
                                   temperature=0.25, top_p=0.9375)
    np.testing.assert_array_equal(win.cpu().numpy(), rwin)
    decision, reward = spk.spk_decide(win, nw, labels, classes)
    assert torch.equal(decision.cpu(), torch.from_numpy(rwin[:, 0, 0]))
    assert torch.equal(reward.cpu().int(), torch.where(decision == labels, 1, -1).cpu().int())
    # the deciding layer's own drawn winners under that reward
    lw, ln = spk.spk_sample_winners(vf, u, temperature=2.0, t_first=tf, T=T)
    W = torch.full((C, 3, 3, 3), 0.5, device="cuda")
    pre = torch.zeros(B, 3, 2, 2, dtype=torch.uint8, device="cuda")
    spk.spk_rstdp_first_spike(W, 1, pre, T, lw, ln, reward, 0.01, -0.01)
    drawn = torch.unique(lw[ln > 0][:, 0, 0]).long()
    changed = (W != 0.5).flatten(1).any(1)
    assert bool(changed[drawn].any()) and not bool(changed[[c for c in range(C) if c not in drawn.tolist()]].any())


@pytest.mark.parametrize("top_k", [1, 2, 300, 1024, 1025, 4096])
@pytest.mark.parametrize("steps", [1.0, 8.0, 1e6])
def test_sample_of_long_rows_by_count(top_k, steps):
    """Boundaries with few and many equal scores on both sides of what one list takes, and rows of few scores that
    can win."""
    randn, rand = seeded(top_k)
    B, N = 4, 60001
    x, u = (randn(B, N, 1, 1) * 2 * steps).round() / steps, rand(B)
    x[1, 700:] = -math.inf
    x[2, 3:] = math.nan
    flat = torch.where(x.isnan(), -math.inf, x.double()).reshape(B, N).cuda()
    for kw in (dict(), dict(top_p=0.75), dict(top_p=0.5, min_p=0.125), dict(min_p=0.9375), dict(min_p=2.0 ** -40)):
        w, n = spk.spk_sample_winners(x.cuda(), u.cuda(), temperature=1.5, top_k=top_k, **kw)
        at = in_order(flat, u.cuda(), **{"temperature": 1.5, "top_k": top_k, "top_p": 1.0, "min_p": 0.0, **kw})
        assert torch.equal(w[:, 0, 0].long(), at) and bool((n == 1).all()), kw
