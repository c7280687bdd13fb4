"""The limits by which the orthogonalisation is tested, on a model of its arithmetic (no GPU
needed): the documented arithmetic is within them, and a diagonal rounded to fp16, which
costs most of a result's error, is not."""
import pytest

from tests import ortho_model as M

SHAPES = [(16, 16), (17, 90), (64, 64), (129, 63), (128, 300), (200, 70), (257, 256), (130, 1000),
          (33, 2050), (512, 768)]


@pytest.mark.parametrize("shape", SHAPES)
def test_limits(shape):
    g = M.gradient(shape[0] * 31 + shape[1], *shape)
    assert M.error(M.model(g), g) <= M.ONE
    assert M.error(M.model(g, diagonals_rounded=True), g) > 1.2 * M.ONE
    limit = M.three(g)
    assert M.error(M.model(g, 3), g) <= limit / 2
    assert M.error(M.model(g), g) > 10 * limit  # products left out
