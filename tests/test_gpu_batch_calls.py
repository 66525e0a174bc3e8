"""Generation of several requests, with and without drafted trees, as callers may call it."""
import numpy as np
import pytest

import synth
from gpu_util import gpu_engine

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def engine():
    eng = gpu_engine(synth.SHAPES["tiny_f32"], 100, seed=2)
    yield eng
    eng.close()


def prompts_of(*lens):
    return [np.random.default_rng(6).integers(0, 200, size=n).astype(np.int32) for n in lens]


@pytest.mark.parametrize("tree", [False, True])
def test_prompts_of_any_stride(engine, tree):
    """A prompt that is a view of another array, backwards or every second token, or that may not be written."""
    a, b = prompts_of(9, 12)
    fixed = b.copy()
    fixed.flags.writeable = False
    go = (lambda p: engine.generate_tree(p, 4, lambda texts: [None] * 3)) if tree else (lambda p: engine.generate_batch(p, 4))
    want, _ = go([a[::-1].copy(), b[::2].copy(), b])
    got, _ = go([a[::-1], b[::2], fixed])
    assert np.array_equal(got, want)
