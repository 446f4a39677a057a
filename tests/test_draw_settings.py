"""The settings of a draw are checked when a chain or an online trainer is made -- CPU only."""
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


@pytest.mark.parametrize("make", [chain, trainer], ids=["chain", "online"])
@pytest.mark.parametrize("bad", [dict(temperature=-1.0), dict(temperature=float("inf")), dict(top_k=-2), dict(top_p=0.0),
                                 dict(top_p=1.5), dict(min_p=-0.25), dict(topk=5), dict(T=3), dict(winners=None)],
                         ids=str)
def test_settings_are_checked_when_they_are_given(make, bad):
    with pytest.raises((TypeError, spk.SpykeError)):
        make(sample=bad)


def test_settings_that_are_fine():
    for ok in ({}, dict(temperature=0.0), dict(temperature=2.0, top_k=5, top_p=0.5, min_p=0.25)):
        assert chain(sample=ok).sample == ok
