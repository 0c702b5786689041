"""The example of examples/recogniser.py: it learns, its stream follows its
sequences, and the gradients it passes on are those of its losses."""
import os
import sys

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def recogniser():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import recogniser
    finally:
        sys.path.pop(0)
    return recogniser


def test_learns_and_streams(recogniser):
    losses, apart = recogniser.main(steps=30)
    first, last = np.mean(losses[:3], 0), np.mean(losses[-3:], 0)
    assert last[0] < 0.8 * first[0] and last[1] < first[1], (first, last)
    # states in [-8, 8] rounded to bfloat16 on both sides: two spacings of 2^-5
    assert apart <= 2.0 ** -4


def test_gradients_of_the_whole(recogniser):
    """In float32, along random directions of every layer, against differences
    of both losses."""
    import torch
    from paper_2110_02848_amd import gpu, synth
    rng = np.random.default_rng(1)
    comp = gpu.Composer(0)
    graph, spellings = synth.lexicon(rng, 30, 8, 2, 4)
    net = recogniser.Recogniser(comp, gpu.to_device(graph), 8, 30, 12, 20, torch.float32, 1)
    batch = recogniser.utterances(rng, 3, spellings, 8, 12)
    _, _, grads = net.loss_and_grads(batch)
    g = torch.Generator(device="cuda").manual_seed(2)
    for k, grad in grads.items():
        d = torch.randn(grad.shape, generator=g, device="cuda")
        keep, vals = net.layers[k], []
        for s in (1, -1):
            net.layers[k] = keep + s * 1e-2 * d
            a, b, _ = net.loss_and_grads(batch)
            vals.append(a + b)
        net.layers[k] = keep
        want = (vals[0] - vals[1]) / 2e-2
        got = float((grad.double() * d.double()).sum())
        # steps of 1e-2: their third order, and losses of 1e-7 over 2e-2
        assert abs(got - want) <= 1e-2 * float((grad * d).abs().sum()) + 1e-4, (k, got, want)
    comp.close()
