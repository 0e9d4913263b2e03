"""Host-side checks of the paged cache's and the beams' calls (no GPU): what they refuse, before anything is launched."""
import numpy as np
import pytest

from paper_2609_34977_gb300 import _native as N
from tests.test_abi import lib  # noqa: F401  (the fixture that builds the library)
from tests.test_answer_abi import _Rows


def _tensor(dtype, *shape):
    return _Rows(dtype, *shape)


class _Odd(_Rows):
    def data_ptr(self):
        return (1 << 20) + 4


def _refused(code, match, call, *args, **kw):
    with pytest.raises(N.SpiderError, match=match) as e:
        call(*args, stream=0, **kw)
    assert e.value.code == code


def _rope(**kw):
    a = dict(h=4, g=2, d=64, new=[2, 3], lens=[2, 30], pages=8, page=16, theta=1e4, width=4, n_axes=1)
    a.update(kw)
    n = max(1, sum(a["new"]))
    q = a.get("q") or _tensor("bfloat16", n, a["h"] * a["d"])
    kv = a.get("kv") or _tensor("bfloat16", n, 2 * a["g"] * a["d"])
    return (q, kv, _tensor("int32", a["n_axes"], sum(a["new"])), None, a["theta"], np.cumsum([0] + a["new"]), a["lens"],
            a.get("table") or _tensor("int32", len(a["new"]), a["width"]),
            a.get("pool") or _tensor("bfloat16", a["pages"], a["page"], 2 * a["g"] * a["d"]), a["h"], a["g"], a["d"],
            a.get("out") or _tensor("bfloat16", n, a["h"] * a["d"]))


@pytest.mark.parametrize("code,match,kw", [
    (N.SPD_EINVAL, "rows do not hold", dict(lens=[1, 30])),             # fewer rows than new ones
    (N.SPD_EINVAL, "rows do not hold", dict(lens=[2, 65])),             # more than the table holds
    (N.SPD_EINVAL, "rows do not hold", dict(lens=[2, -1])),
    (N.SPD_EINVAL, "theta", dict(theta=0.0)),
    (N.SPD_EINVAL, "theta", dict(theta=float("nan"))),
    (N.SPD_EINVAL, "theta", dict(theta=float("inf"))),
    (N.SPD_EINVAL, "bad rotary", dict(h=3)),                            # heads no multiple of K/V heads
    (N.SPD_EUNSUPPORTED, "head_dim", dict(d=96)),
    (N.SPD_EUNSUPPORTED, "page_size", dict(page=24)),
    (N.SPD_EUNSUPPORTED, "2\\^31", dict(pages=1 << 27)),
    (N.SPD_EINVAL, "16-byte aligned", dict(q=_Odd("bfloat16", 5, 256))),
    (N.SPD_EINVAL, "aligned", dict(pool=_Odd("bfloat16", 8, 16, 256))),
])
def test_rope_refusals(lib, code, match, kw):  # noqa: F811
    _refused(code, match, N.spd_rope_pages, *_rope(**kw))


def test_rope_strides(lib):  # noqa: F811
    class Wide(_Rows):
        def stride(self):
            return 260, 1

    _refused(N.SPD_EINVAL, "multiples of 8", N.spd_rope_pages, *_rope(q=Wide("bfloat16", 5, 256)))
    same = type("Same", (_Rows,), dict(stride=lambda self: (264, 1)))("bfloat16", 5, 256)
    _refused(N.SPD_EINVAL, "in place", N.spd_rope_pages, *_rope(q=same))  # (both lie at the same place)
    with pytest.raises(ValueError, match="pos"):
        a = list(_rope())
        a[2] = _tensor("int32", 1, 4)
        N.spd_rope_pages(*a, stream=0)
    with pytest.raises(ValueError, match="pool"):
        N.spd_rope_pages(*_rope(pool=_tensor("bfloat16", 8, 16, 128)), stream=0)
    with pytest.raises(ValueError, match="axis"):
        a = list(_rope())
        a[3] = np.zeros(31, np.uint8)
        N.spd_rope_pages(*a, stream=0)
    with pytest.raises(ValueError, match="table"):
        N.spd_rope_pages(*_rope(table=_tensor("int32", 1, 4)), stream=0)


@pytest.mark.parametrize("cu", [[0, 5, 3], [0, 2, 4, 1, 3], [0, 4, 0, 3]])
def test_lists_that_decrease(lib, cu):  # noqa: F811
    n = len(cu) - 1
    ws = _tensor("uint8", 1 << 27)
    _refused(N.SPD_EINVAL, "q_cu decreases", N.spd_paged_attention, _tensor("bfloat16", 3, 256), cu, [30] * n,
             _tensor("int32", n, 4), _tensor("bfloat16", 8, 16, 256), 4, 2, 64, _tensor("bfloat16", 3, 256), None, ws)


@pytest.mark.parametrize("prefix", [[-1, 0], [0, 31], [3, 0]])
def test_prefixes_outside_the_rows(lib, prefix):  # noqa: F811
    _refused(N.SPD_EINVAL, "prefix of sequence", N.spd_paged_attention, _tensor("bfloat16", 3, 256), [0, 1, 3], [2, 30],
             _tensor("int32", 2, 4), _tensor("bfloat16", 8, 16, 256), 4, 2, 64, _tensor("bfloat16", 3, 256), None,
             _tensor("uint8", 1 << 27), prefix=prefix)


def test_workspaces(lib):  # noqa: F811
    _refused(N.SPD_ENOSPC, "workspace too small", N.spd_paged_attention, _tensor("bfloat16", 3, 256), [0, 1, 3], [2, 30],
             _tensor("int32", 2, 4), _tensor("bfloat16", 8, 16, 256), 4, 2, 64, _tensor("bfloat16", 3, 256), None, _tensor("uint8", 64))
    assert N.spd_paged_attention_workspace_size(1, 1, 4, 3, 64) == 0 and N.spd_paged_attention_workspace_size(1, 1, 4, 2, 80) == 0
    assert N.spd_pages_workspace_size(0, 1) == 0 and N.spd_beam_select_workspace_size(1, 33, 1, 10) == 0


def _update(n_in=2, n_out=3, width=4, pages=8, page=16, **kw):
    i = lambda *s: _tensor("int32", *s)  # noqa: E731
    a = dict(pool=_tensor("bfloat16", 2, pages, page, 256), ref=i(pages), table=i(n_in, width), lens=i(n_in), parent=i(n_out),
             grow=i(n_out), ref_out=i(pages), table_out=_At(1 << 21, n_out, width), len_out=_At(1 << 22, n_out), ws=_tensor("uint8", 1 << 16))
    a.update(kw)
    return a["pool"], 2, 64, a["ref"], a["table"], a["lens"], a["parent"], a["grow"], a["ref_out"], a["table_out"], a["len_out"], a["ws"]


class _At(_Rows):
    def __init__(self, at, *shape):
        super().__init__("int32", *shape)
        self.at = at

    def data_ptr(self):
        return self.at


def test_update_refusals(lib):  # noqa: F811
    _refused(N.SPD_EINVAL, "without parents", N.spd_pages_update, *_update(parent=None))
    _refused(N.SPD_EINVAL, "in place", N.spd_pages_update, *_update(table_out=_tensor("int32", 3, 4)))
    _refused(N.SPD_EINVAL, "in place", N.spd_pages_update, *_update(len_out=_tensor("int32", 3)))
    _refused(N.SPD_ENOSPC, "workspace", N.spd_pages_update, *_update(ws=_tensor("uint8", 300)))
    _refused(N.SPD_EUNSUPPORTED, "page_size", N.spd_pages_update, *_update(page=8))
    _refused(N.SPD_EUNSUPPORTED, "table entries", N.spd_pages_update, *_update(width=1 << 30))
    with pytest.raises(ValueError, match="table_out"):
        N.spd_pages_update(*_update(table_out=_At(1 << 21, 3, 5)), stream=0)
    with pytest.raises(ValueError, match="ref_in"):
        N.spd_pages_update(*_update(ref=_tensor("int32", 7)), stream=0)
    i = lambda *s: _tensor("int32", *s)  # noqa: E731
    _refused(N.SPD_ENOSPC, "workspace", N.spd_pages_compact, _tensor("bfloat16", 2, 8, 16, 256), 2, 64, i(8), i(2, 4), i(8), i(2, 4), i(1),
             _tensor("uint8", 300))


@pytest.mark.parametrize("code,match,kw", [
    (N.SPD_EUNSUPPORTED, "beams", dict(n_in=33)),
    (N.SPD_EUNSUPPORTED, "beams", dict(n_out=33)),
    (N.SPD_EUNSUPPORTED, "65535", dict(B=1 << 14, n_in=5)),
    (N.SPD_EINVAL, "eos", dict(eos=100)),
    (N.SPD_EINVAL, "eos", dict(eos=-2)),
    (N.SPD_ENOSPC, "workspace", dict(ws=300)),
])
def test_beam_refusals(lib, code, match, kw):  # noqa: F811
    a = dict(B=2, n_in=3, n_out=4, eos=5, ws=1 << 20)
    a.update(kw)
    f = lambda *s: _tensor("float32", *s)  # noqa: E731
    i = lambda *s: _tensor("int32", *s)  # noqa: E731
    B, n_in, n_out = a["B"], a["n_in"], a["n_out"]
    _refused(code, match, N.spd_beam_select, f(B * n_in, 100), f(B, n_in), a["eos"], i(B, n_out), i(B, n_out), f(B, n_out), f(B, n_in),
             _tensor("uint8", a["ws"]))


def test_beam_shapes(lib):  # noqa: F811
    f = lambda *s: _tensor("float32", *s)  # noqa: E731
    i = lambda *s: _tensor("int32", *s)  # noqa: E731
    for z, scores, parent in ((f(5, 100), f(2, 3), i(2, 4)), (f(6, 100), f(6), i(2, 4)), (f(6, 100), f(2, 3), i(1, 4))):
        with pytest.raises(ValueError):
            N.spd_beam_select(z, scores, 5, parent, i(2, 4), f(2, 4), None, _tensor("uint8", 1 << 20), stream=0)
