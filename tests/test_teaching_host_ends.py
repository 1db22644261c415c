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


@pytest.mark.parametrize("shape", [(1, 1), (1, 4096), (1, 4097), (1, 1 << 21), (4097, 1), (8, 50000), (5, 6000), (17, 2049), (32, 1 << 21), (33, 1024), (33, 1025), (64, 1024), (65, 64),
                                   (65, 1024), (333, 1111), (1000, 3000), (1024, 1024), (4096, 4096), (3000, 100000)])
def test_workspace_is_as_large_as_documented(lib, shape):  # noqa: F811
    """Sides padded to 32 where there are many rows; small matrices have rooms of a few sizes."""
    k, n = min(shape), max(shape)
    k32, n32, tiles = -(-k // 32) * 32, -(-n // 32) * 32, -(-k // 64)
    size = pl.orthogonal_workspace_bytes([shape])
    if k <= 32:
        least, most = (0, 0) if n <= (4096 if k <= 16 else 2048) else (1, 2 << 20)
    elif k <= 64 and n <= 1024:
        least, most = 32 << 10, 256 << 10
    else:
        least = 4 * k * n32 + 8 * n * k32 + 8 * k * k32
        most = least + tiles * (tiles + 1) // 2 * -(-n // 256) * (16 << 10)
    assert least <= size <= most + (16 << 10)
    assert size == pl.orthogonal_workspace_bytes([shape[::-1]])
    assert pl.orthogonal_workspace_bytes([shape] * 5) <= 5 * (most + (16 << 10))
