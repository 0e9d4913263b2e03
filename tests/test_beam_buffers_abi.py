"""Host-side checks of the beams' buffers (no GPU): which may be the same, before anything is launched."""
import pytest

from paper_2609_34977_gb300 import _native as N
from tests.test_abi import lib  # noqa: F401  (the fixture that builds the library)
from tests.test_pages_abi import _At, _refused, _tensor


class _FloatAt(_At):
    def __init__(self, at, *shape):
        super().__init__(at, *shape)
        self.dtype = _tensor("float32", 1).dtype


@pytest.mark.parametrize("n_in,n_out", [(1, 4), (4, 3), (32, 31)])
def test_scores_in_place_of_another_number_of_beams(lib, n_in, n_out):  # noqa: F811
    # one request's totals would be written over another's scores, which may not have been read
    f, i = lambda *s: _tensor("float32", *s), lambda *s: _tensor("int32", *s)  # noqa: E731
    B = 2
    _refused(N.SPD_EINVAL, "scores_out may be scores", N.spd_beam_select, f(B * n_in, 100), _FloatAt(1 << 22, B, n_in), 5, i(B, n_out),
             i(B, n_out), _FloatAt(1 << 22, B, n_out), None, _tensor("uint8", 1 << 20))
