"""Arguments of orthogonalised updates in forms that Python programs have them in: what the binding makes of them, or refuses.  Without
matrices, so that nothing is launched."""
import numpy as np
import pytest

import paper_1906_08879_amd as pl
from tests.test_losses_host import lib  # noqa: F401  (a fixture)

USUAL = (3.4445, -4.7750, 2.0315)


def test_iterations_that_can_be_read_once(lib):  # noqa: F811
    """A generator's steps are checked as those of a list are: numbers of steps of two would be read as others of three."""
    pl.orthogonal_update([], out=[], iteration=(USUAL for _ in range(5)))
    pl.orthogonal_update([], out=[], iteration=(iter(USUAL) for _ in range(5)))
    pl.orthogonal_update([], out=[], iteration=np.array([USUAL] * 5))
    for bad in ([(1.0, 2.0)] * 3, [(1.0,)] * 3, [USUAL, ()], [USUAL + (1.0,)], [USUAL, 1.0], 1.0, None, [("a", "b", "c")]):
        with pytest.raises(pl.PlacetoError):
            pl.orthogonal_update([], out=[], iteration=bad)
        if isinstance(bad, list):
            with pytest.raises(pl.PlacetoError):
                pl.orthogonal_update([], out=[], iteration=(step for step in bad))


def test_scales_of_other_types(lib):  # noqa: F811
    for scales in (2, 0.5, np.float32(0.5), np.float64(0.5), np.int64(2), [], (), np.zeros(0)):
        pl.orthogonal_update([], out=[], scales=scales)
    for bad in (None, "1", ["a"], [1.0], np.array(0.5), np.float32([0.5]), object()):
        with pytest.raises(pl.PlacetoError):
            pl.orthogonal_update([], out=[], scales=bad)
