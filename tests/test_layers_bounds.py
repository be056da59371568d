"""Bounds of runs as the binding takes them: whole numbers, however they are held, and nothing that would have to be rounded."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_1902_01981_amd import layers  # noqa: E402


@pytest.mark.parametrize("bounds", [[0, 3, 9], (0, 3, 9), np.array([0, 3, 9], dtype=np.int32), np.array([0, 3, 9], dtype=np.uint16), np.array([0.0, 3.0, 9.0]),
                                    np.array([0, 7, 3, 7, 9, 7])[::2], torch.tensor([0, 3, 9])], ids=str)
def test_whole_numbers(bounds):
    at, runs, held = layers._bounds(bounds)
    assert runs == 2 and held.tolist() == [0, 3, 9] and held.dtype == np.int64 and at == held.ctypes.data


@pytest.mark.parametrize("bounds", [[0, 2.5, 9], np.array([0.0, 3.0, 9.25]), np.array([0.0, np.nan, 9.0]), [0.0, 1e30], [0], [], [[0, 9]], 9], ids=str)
def test_what_is_refused(bounds):
    with pytest.raises(ValueError):
        layers._bounds(bounds)
