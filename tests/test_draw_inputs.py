"""The numbers that a draw in the chain and the online trainer needs: asked for on the host before anything is
enqueued -- CPU only."""
import pytest
import torch

import synth

spk = pytest.importorskip("paper_1903_02440_amd")
from paper_1903_02440_amd.pipeline import chain_for, online_for  # noqa: E402

WL = synth.mnist_3layer(4)
BANK = torch.zeros(WL.stages[0].cin, 3, 3)


def chain(**kw):
    return chain_for(WL, BANK, device="cpu", concurrent_learn=False, **kw)


def trainer(**kw):
    return online_for(WL, BANK, device="cpu", **kw)


def test_a_chain_does_not_draw_without_numbers():
    ch = chain(sample=dict(temperature=2.0))
    with pytest.raises(ValueError, match="uniform"):
        ch.forward()
    with pytest.raises(ValueError, match="uniform"):
        ch.step()
    u = torch.rand(4)
    ch.set_input(uniform=u)
    assert torch.equal(ch.uniform, u)


@pytest.mark.parametrize("u", [torch.rand(1), torch.rand(3), torch.rand(4, 1), torch.rand(())], ids=lambda t: str(tuple(t.shape)))
def test_a_chain_takes_a_number_an_image(u):
    with pytest.raises(ValueError, match="uniform"):
        chain(sample={}).set_input(uniform=u)


def test_numbers_without_a_draw_are_refused():
    with pytest.raises(ValueError, match="sample"):
        chain().set_input(uniform=torch.rand(4))
    with pytest.raises(ValueError, match="sample"):
        trainer().run(torch.zeros(2, WL.H, WL.W, dtype=torch.uint8), uniform=torch.rand(2))


def test_a_trainer_does_not_draw_without_numbers():
    images, labels = torch.zeros(5, WL.H, WL.W, dtype=torch.uint8), torch.zeros(5, dtype=torch.int32)
    tr = trainer(sample=dict(top_p=0.5), steps_per_graph=2)
    for u in (None, torch.rand(4), torch.rand(6), torch.rand(1), torch.rand(5, 1)):
        with pytest.raises(ValueError, match="uniform"):
            tr.run(images, labels, u)
    tr.run(images[:0], labels[:0])
