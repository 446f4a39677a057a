"""Drawn winners in the chain and the online trainer, readout calls in captured
graphs and on other streams."""
import numpy as np
import pytest
import torch

import readout_ref as ref
import synth
from paper_1903_02440_amd.pipeline import Chain, chain_for, online_for
from test_gpu_readout import BF16, F32, make, seeded

spk = pytest.importorskip("paper_1903_02440_amd")

pytestmark = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def loaded(wl, inp, **kw):
    ch = chain_for(wl, inp["bank"], **kw)
    ch.set_weights([dev(w) for w in inp["weights"]])
    ch.set_input(image=dev(inp["image"]), labels=dev(inp["labels"]))
    return ch


@pytest.mark.parametrize("kw", [{}, {"fused": True, "want_waves": False, "want_spikes": False,
                                     "want_potentials": False}], ids=["full", "fused"])
def test_chain_draws_its_decision(kw):
    wl = synth.mnist_3layer(24)
    inp = synth.make_inputs(wl)
    u = torch.rand(24, generator=torch.Generator().manual_seed(3))
    draw = dict(temperature=4.0, top_k=60, top_p=0.9375)
    plain, greedy, drawn = (loaded(wl, inp, sample=s, **kw) for s in (None, dict(temperature=0.0), draw))
    for ch in (greedy, drawn):
        ch.set_input(uniform=u.cuda())
    for ch in (plain, greedy, drawn):
        ch.step()
    torch.cuda.synchronize()
    last = plain.conv_stages()[-1]
    b = drawn.bufs[last]
    win, nw = ref.sample_winners(b["vf"].double().cpu().numpy(), u.numpy(), t_first=b["tf"].cpu().numpy(), T=wl.T,
                                 **draw)
    np.testing.assert_array_equal(b["win"].cpu().numpy(), win)
    np.testing.assert_array_equal(b["nw"].cpu().numpy(), nw)
    want = np.where(nw > 0, win[:, 0, 0] % wl.n_classes, -1)
    np.testing.assert_array_equal(drawn.decision.cpu().numpy(), want)
    # the best of the order is the kWTA's winner where every neuron fires at one step
    assert torch.equal(greedy.bufs[last]["win"], plain.bufs[last]["win"])
    assert all(torch.equal(a, c) for a, c in zip(greedy.weights(), plain.weights()))
    assert not torch.equal(b["win"], plain.bufs[last]["win"])


def test_chain_refuses_a_draw_by_time():
    wl = synth.mnist_single(2)
    with pytest.raises(ValueError, match="infinite threshold"):
        Chain(wl.stages, 2, wl.T, wl.H, wl.W, wl.cin, filter_bank=torch.zeros(6, 3, 3), sample={})


def test_online_draws_replay_as_eager():
    wl = synth.mnist_3layer(12)
    inp = synth.make_inputs(wl)
    draw = dict(temperature=3.0, top_p=0.875)
    u = torch.rand(12, generator=torch.Generator().manual_seed(4)).cuda()
    trainers = [online_for(wl, inp["bank"], sample=draw, **kw) for kw in (dict(steps_per_graph=4), dict(use_graph=False))]
    imgs, labs = dev(inp["image"]), dev(inp["labels"])
    for tr in trainers:
        tr.set_weights([dev(w) for w in inp["weights"]])
    for a, b in ((0, 4), (4, 8), (8, 12)):
        for tr in trainers:
            tr.run(imgs[a:b], labs[a:b], u[a:b])
            torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(*(tr.weights() for tr in trainers))), (a, b)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_readout_calls_replay(dtype):
    """A batch, its gradients, a step and a draw of a long row in one graph, replayed on new inputs."""
    x, s0 = make(2, 100, 1, 2, 40, 24, dtype, 51)
    randn, rand = seeded(52)
    d_out, u = randn(*x["v"].shape).to(dtype).cuda(), rand(3).cuda()
    scores = (randn(3, 20011, 1, 1) * 2).to(dtype).cuda()
    one = {n: t[:, 0].contiguous() for n, t in x.items()}
    names = ("q", "k", "v", "g", "beta")

    def work(state):
        out, last = spk.spk_delta_rule(**x, initial_state=s0)
        grads = spk.spk_delta_rule_backward(*(x[n] for n in names), d_out, initial_state=s0)
        step = spk.spk_delta_rule_step(**one, state=state)
        return [out, last, *grads, step, *spk.spk_sample_winners(scores, u, top_k=30, top_p=0.875)]

    state = s0.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(s0.clone())
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = work(state)
    for k in range(3):
        new = make(2, 100, 1, 2, 40, 24, dtype, 60 + k)
        for n in names:
            x[n].copy_(new[0][n])
        u.copy_(rand(3))
        scores.copy_((randn(3, 20011, 1, 1) * 2).to(dtype))
        state.copy_(new[1])
        g.replay()
        torch.cuda.synchronize()
        again = new[1].clone()
        want = work(again)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k
        assert torch.equal(state, again)


def test_readout_calls_on_two_streams():
    """Two calls at once, each with a workspace of its own."""
    calls = [make(1, 400, 2, 4, 96, 72, BF16, 71 + k) for k in range(2)]
    want = [spk.spk_delta_rule(**x, initial_state=s) for x, s in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    got = []
    for st, (x, s) in zip(streams, calls):
        st.wait_stream(torch.cuda.current_stream())
        n = spk.spk_delta_rule_workspace_size(spk.SPK_BF16, 1, 400, 2, 4, 96, 72)
        ws, out, last = (torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(x["v"]), torch.empty_like(s))
        torch.cuda.synchronize()
        got.append((out, last, ws))
    for _ in range(3):
        for st, (x, s), (out, last, ws) in zip(streams, calls, got):
            spk.spk_delta_rule(**x, initial_state=s, out=out, final_state=last, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for (o, l), (out, last, _) in zip(want, got):
        assert torch.equal(o, out) and torch.equal(l, last)


def test_readout_calls_on_a_given_stream_make_their_buffers_there():
    """Outputs and workspaces made by calls on side streams are not handed to other work while those run."""
    x, s0 = make(2, 300, 2, 4, 64, 48, F32, 81)
    want = spk.spk_delta_rule(**x, initial_state=s0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(4):
        got = [spk.spk_delta_rule(**x, initial_state=s0, stream=st) for st in streams]
        noise = [torch.full_like(want[0], 7.0) for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[0]) and torch.equal(l, want[1]) for o, l in got)
        assert all(bool((t == 7.0).all()) for t in noise)
