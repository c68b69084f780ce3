"""What the small server refuses: configurations of the other server, copies that the pool has no page for."""
import types

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2601_21758_amd import _lib as L  # noqa: E402
from paper_2601_21758_amd import serve  # noqa: E402


@pytest.mark.parametrize("beams", [0, -1, 2, 4])
def test_greedy_server_has_one_beam(beams):
    """Server keeps one slot a request: more beams than that are BeamServer's, and none are nobody's."""
    model = types.SimpleNamespace(c=serve.Config(beams=beams))
    with pytest.raises(ValueError, match="beam"):
        serve.Server(model, [], [[1]], device="cpu")


@pytest.mark.parametrize("beams", [0, -1, L.MAX_BEAMS + 1])
def test_beams_of_a_search(beams):
    model = types.SimpleNamespace(c=serve.Config(beams=beams, slots=100))
    with pytest.raises(ValueError, match="beam"):
        serve.BeamServer(model, [], [[1]], device="cpu")


def small(**kw):
    c = dict(layers=1, q_heads=2, kv_heads=1, head_dim=64, vocab=64, dtype=torch.float16, n_pages=40, slots=6, admit=2,
             answer=4)
    return serve.Config(**dict(c, **kw))


@pytest.mark.gpu
@pytest.mark.parametrize("lost", [1, 2])
def test_refused_copies_end_the_search(lost):
    """A reordering that refuses a beam's copy empties its slot: the search does not go on without the beam's tokens."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    server = serve.BeamServer(serve.Model(small(beams=3)), [5] * 3, [[1, 2, 3], [4]])
    reorder, calls = server.cache.reorder, []

    def refuse(slot, parent, **kw):
        granted = reorder(slot, parent, **kw)
        calls.append(granted)
        if len(calls) == lost:
            server.cache.release(slot[1:2])
            granted[1] = 0
        return granted

    server.cache.reorder = refuse
    with pytest.raises(RuntimeError, match="out of pages"):
        server.run()
    assert len(calls) == lost


@pytest.mark.gpu
def test_beams_without_a_parent_are_no_refusal():
    """Fewer tokens than beams: the beams that nothing continues are empty, and the search goes on."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    server = serve.BeamServer(serve.Model(small(vocab=2, beams=5)), [1, 0], [[1, 0, 1], [0]])
    answers = server.run()
    assert sorted(answers) == [0, 1] and all(len(a) == 4 and set(a) <= {0, 1} for a in answers.values())
    assert all(np.isfinite(list(server.scores.values())))


@pytest.mark.gpu
@pytest.mark.parametrize("prompt,answer,prefix", [(7, 20, 0), (16, 33, 5), (1, 50, 40), (31, 18, 16)])
def test_reserved_pages_are_enough(prompt, answer, prefix):
    """A pool with just the pages that a request's beams may come to hold refuses none of their copies."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    beams, page = 4, 16
    own = -(-(prefix + prompt + answer) // page) - prefix // page
    c = small(beams=beams, answer=answer, n_pages=-(-prefix // page) + beams * own, slots=beams)
    rng = np.random.default_rng(prompt)
    prompts = [rng.integers(0, c.vocab, prompt).tolist() for _ in range(2)]
    server = serve.BeamServer(serve.Model(c), rng.integers(0, c.vocab, prefix).tolist(), prompts)
    answers = server.run()
    assert sorted(len(a) for a in answers.values()) == [answer] * 2
