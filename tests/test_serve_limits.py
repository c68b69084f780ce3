"""What the small server refuses: configurations of the other server."""
import types

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
