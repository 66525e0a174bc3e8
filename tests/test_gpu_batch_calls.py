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


PENALTIES = [{}, dict(repetition=1.3), dict(presence=0.2), dict(frequency=0.2), dict(bias={3: 2.0})]


@pytest.mark.parametrize("penalty", PENALTIES)
@pytest.mark.parametrize("tree", [False, True])
def test_tokens_are_kept_where_penalties_want_them_alone(engine, penalty, tree, monkeypatch):
    """Without penalties of occurred tokens no step copies tokens; with them they stay in one place."""
    from paper_2602_16760_amd import engine as E
    places, append = [], E._Batch.append

    def watched(self, *args):
        append(self, *args)
        places.append(self.tokens.data_ptr())

    monkeypatch.setattr(E._Batch, "append", watched)
    sampling = dict(temperature=0.8, seed=1, **penalty)
    if tree:
        engine.generate_tree(prompts_of(5, 9), 6, lambda texts: [([7], [0])] * 2, sampling=sampling)
    else:
        engine.generate_batch(prompts_of(5, 9), 6, sampling=sampling)
    if set(penalty) & {"repetition", "presence", "frequency"}:
        assert places and len(set(places)) == 1
    else:
        assert not places


def test_a_draft_for_every_text(engine):
    for trees in ([], [None], [([7], [0])], [None] * 3):
        with pytest.raises(ValueError):
            engine.generate_tree(prompts_of(5, 9), 4, lambda texts: trees)


def test_a_draft_that_writes_into_its_texts(engine):
    """What a draft does with the lists that it is given is its own affair."""
    prompts = prompts_of(5, 9)
    want, _ = engine.generate_batch(prompts, 8)

    def draft(texts):
        out = []
        for text in texts:
            out.append(None if text is None else ([text[-1]], [0]))
            if text is not None:
                text += [1, 2, 3]
        return out

    got, st = engine.generate_tree(prompts, 8, draft)
    assert np.array_equal(got, want) and st["free_pages"] == st["pages"]


@pytest.mark.parametrize("R,max_rows,pages", [(2, 64, 3), (40, 16, 1), (1, 64, 5)])
def test_pages_for_the_rows_that_a_request_has(engine, R, max_rows, pages):
    """64 rows are shared by the requests: positions of a request's last step are its prompt's, the tokens in front of the last one's, and its rows'."""
    prompts, per = prompts_of(*[5] * R), min(max_rows, 64 // R)
    assert -(-(4 + 5 + per) // 16) == pages
    draft = lambda texts: [None if t is None else (list(range(100, 163)), [0] * 63) for t in texts]
    tokens, st = engine.generate_tree(prompts, 6, draft, max_rows=max_rows, n_pages=pages * R)
    assert st["pages"] == st["free_pages"] == pages * R and np.array_equal(tokens, engine.generate_batch(prompts, 6)[0])
    assert engine.generate_tree(prompts, 6, draft, max_rows=max_rows)[1]["pages"] == pages * R
    from paper_2602_16760_amd import binding as B
    with pytest.raises(B.LaError):
        engine.generate_tree(prompts, 6, draft, max_rows=max_rows, n_pages=pages * R - 1)
