"""Host-side checks of the calls for answers from the cache (no GPU): what they refuse, and that they read no further than the
arrays they are given."""
import numpy as np
import pytest

from paper_2609_34977_gb300 import _native as N
from tests.test_abi import _FakeCuda, lib  # noqa: F401  (the fixture that builds the library)


class _Somewhere(_FakeCuda):
    def data_ptr(self):
        return 1 << 20


@pytest.mark.parametrize("cu", [[0, 5, 3], [0, 2, 4, 1, 3], [0, 4, 0, 3]])
def test_lists_are_not_read_past_their_end(lib, cu):  # noqa: F811
    # cu's last entry says that there are 3 entries. What lies behind them would be refused for itself, if it were read
    whole = np.array([-1, 0, 1, 9, 9], np.int32)
    with pytest.raises(N.SpiderError, match="q_cu decreases") as e:
        N.spd_tree_mask(whole[:3], cu, words=1)
    assert e.value.code == N.SPD_EINVAL
    n, ws = len(cu) - 1, _Somewhere("uint8", 1 << 12)
    whole = np.array([0, 1, 2, 0, 0], np.int32)
    with pytest.raises(N.SpiderError, match="path_cu decreases") as e:
        N.spd_tree_commit(_Somewhere("bfloat16", n * 16 * 256), 1, whole[:3], cu, [1] * n, 16, 2, 64, ws, stream=0)
    assert e.value.code == N.SPD_EINVAL


class _Rows(_Somewhere):
    def __init__(self, dtype, *shape):
        super().__init__(dtype, int(np.prod(shape)))
        self.shape = shape

    def stride(self):
        return self.shape[-1], 1


@pytest.mark.parametrize("shape", [(4, 4), (2, 6), (1, 4), (13,), (2, 2, 10)])
def test_grammars_of_another_width_are_refused(lib, shape):  # noqa: F811
    # 150 tokens are 5 words; a row stride of 4, 6 or 10 would put every grammar but the first in the wrong place
    z, rule = _Rows("float32", 3, 150), _Rows("int32", 3)
    with pytest.raises(ValueError, match="allow"):
        N.spd_logits_process(z, z, allow=_Rows("int32", *shape), rule=rule, stream=0)
