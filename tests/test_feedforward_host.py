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


def refused(block, error, match, **other):
    """set_weights raises, and has neither cast nor copied anything."""
    before = {n: None if getattr(block, n, None) is None else getattr(block, n).clone() for n in ("b1", "b2", "g", "b")}
    casts = len(block.casts)
    with pytest.raises(error, match=match):
        block.set_weights(**weights(7, **other))
    assert len(block.casts) == casts
    for n, t in before.items():
        now = getattr(block, n, None)
        assert (now is None) == (t is None) and (t is None or torch.equal(now, t)), n


@pytest.mark.parametrize("again", [False, True])
def test_unusable_weights_are_refused_before_anything_changes(gpt, again):
    if again:
        gpt.set_weights(**weights())
    v = lambda n, dt=BF: torch.ones(n, dtype=dt)  # noqa: E731
    refused(gpt, TypeError, "g and b", g=v(D, F32))
    refused(gpt, TypeError, "g and b", b=v(D, F32))
    for name, n in (("b1", FFN), ("b2", D), ("g", D), ("b", D)):
        refused(gpt, TypeError, name, **{name: v(n, torch.float16)})
        refused(gpt, ValueError, name, **{name: v(n + 1)})
    for name, shape in (("W1", (D, FFN)), ("W2", (FFN, D))):
        refused(gpt, TypeError, name, **{name: torch.ones(shape, dtype=torch.float16)})
        refused(gpt, ValueError, name, **{name: torch.ones(shape[::-1], dtype=BF).t()})   # columns contiguous, not rows
        refused(gpt, ValueError, name, **{name: torch.ones((shape[0], 1), dtype=BF).expand(shape)})


def test_biases_keep_their_types(gpt):
    """Each bias of its own type; what the block was set up with stays, since a captured graph has its tensors."""
    gpt.set_weights(**weights(b1=torch.ones(FFN, dtype=F32), g=torch.ones(D), b=torch.ones(D)))
    assert gpt.db1.dtype == F32 and gpt.db2.dtype == BF
    refused(gpt, TypeError, "b1", b1=torch.ones(FFN, dtype=BF))
    refused(gpt, TypeError, "b", g=torch.ones(D, dtype=BF), b=torch.ones(D, dtype=BF))


def test_gated_weights_are_refused_before_either_is_cast(monkeypatch):
    block = FF.GatedFeedForward(4, D, FFN, "cpu")
    casts = []
    monkeypatch.setattr(block, "_quantise", lambda x, t, fmt, predict=True: casts.append(x))
    good = torch.ones((D, 2 * FFN), dtype=BF), torch.ones((FFN, D), dtype=BF)
    for error, bad in ((TypeError, torch.ones((FFN, D), dtype=torch.float16)), (ValueError, torch.ones((D, FFN), dtype=BF)),
                       (ValueError, torch.ones((D, FFN), dtype=BF).t())):
        with pytest.raises(error, match="Wd"):
            block.set_weights(good[0], bad)
    assert not casts
    block.set_weights(*good)
    assert len(casts) == 2


def test_calls_out_of_order_are_refused(gpt):
    x = torch.ones((4, D), dtype=BF)
    gated = FF.GatedFeedForward(4, D, FFN, "cpu")
    for block in (gpt, gated):
        with pytest.raises(RuntimeError, match="set_weights"):
            block.forward(x)
        with pytest.raises(RuntimeError, match="forward"):
            block.backward(x)
        with pytest.raises(RuntimeError, match="capture"):
            block.replay()
    gpt.set_weights(**weights())
    with pytest.raises(RuntimeError, match="forward"):
        gpt.backward(x)
    infer = FF.GatedFeedForward(4, D, FFN, "cpu", train=False)
    with pytest.raises(RuntimeError, match="inference"):
        infer.backward(x)


def test_a_block_of_another_gpu_is_refused(gpt, monkeypatch):
    """Calls run on the current GPU's stream: a block on another is refused before any is made."""
    x = torch.ones((4, D), dtype=BF)
    gpt.set_weights(**weights())
    casts = len(gpt.casts)
    gpt.ran = True
    monkeypatch.setattr(FF, "_index", lambda dev: 1)
    monkeypatch.setattr(F, "_current", lambda: 0)
    for call in (lambda: gpt.set_weights(**weights(1)), lambda: gpt.forward(x), lambda: gpt.backward(x)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
    assert len(gpt.casts) == casts and torch.equal(gpt.b1, weights()["b1"])
