"""The feed-forward blocks on the host (no GPU needed): what they keep of a user's
tensors, and what they refuse before anything has changed."""
import os

import pytest
import torch

from paper_2309_17224_amd import feedforward as FF
from paper_2309_17224_amd import fp8lin as F

BF, F32 = torch.bfloat16, torch.float32
D, FFN = 8, 16


@pytest.fixture
def gpt(monkeypatch):
    """A GPT block whose casts (which need a GPU) are noted instead."""
    if not os.path.exists(F.LIB_PATH):
        from paper_2309_17224_amd import build
        build.build()
    block = FF.GptFeedForward(4, D, FFN, "cpu")
    block.casts = []
    monkeypatch.setattr(block, "_quantise", lambda x, t, fmt, predict=True: block.casts.append(x))
    return block


def weights(seed=0, **other):
    g = torch.Generator().manual_seed(seed)
    w = dict(W1=torch.randn(D, FFN, generator=g), b1=torch.randn(FFN, generator=g), W2=torch.randn(FFN, D, generator=g),
             b2=torch.randn(D, generator=g), g=torch.randn(D, generator=g), b=torch.randn(D, generator=g))
    return dict({k: v.to(BF) for k, v in w.items()}, **other)


def test_parameters_are_copied_without_their_graph(gpt):
    """Updated from parameters step after step, the block holds values alone: no history that grows with every update."""
    for step in range(3):
        w = {k: torch.nn.Parameter(v) for k, v in weights(step).items()}
        gpt.set_weights(**w)
        for name in ("b1", "b2", "g", "b"):
            t = getattr(gpt, name)
            assert not t.requires_grad and t.grad_fn is None and torch.equal(t, w[name])
