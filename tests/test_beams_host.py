"""The host side of beam search (no GPU): tensors on the CPU, the library's calls as stand-ins, its size functions as they are."""
import numpy as np
import pytest
import torch

from paper_2609_34977_gb300 import _native as N
from paper_2609_34977_gb300 import beams
from paper_2609_34977_gb300.beams import BeamAnswer
from tests.test_abi import lib  # noqa: F401  (the fixture that builds the library)

CALLS = ("spd_pages_update", "spd_decode_paged", "spd_beam_select", "spd_pages_compact")


class _Library:
    """Stand-ins that record their calls and arguments; `fails` maps a call to the status that it leaves in its workspace. Selection r
    (from 0) takes the beams 0, 1, ... of every request (all of them beam 0 of the prompts) and token r."""

    def __init__(self, monkeypatch):
        self.calls, self.args, self.fails, self.ended = [], [], {}, None

        class Torch:
            def __getattr__(self, name):
                f = getattr(torch, name)
                if name in ("zeros", "empty", "full", "arange", "tensor"):
                    return lambda *a, **k: f(*a, **{x: y for x, y in k.items() if x != "device"})
                return f
        monkeypatch.setattr(beams, "torch", Torch())
        monkeypatch.setattr(torch.Tensor, "cuda", lambda t: t)
        for name in CALLS:
            monkeypatch.setattr(N, name, self._stand_in(name))
        monkeypatch.setattr(N, "spd_decode_paged_workspace_size", lambda model, n, seqs: 64)
        monkeypatch.setattr(N, "spd_workspace_status", self._status)

    @staticmethod
    def _status(ws):  # reads and clears
        code = int(ws[:4].view(torch.int32))
        ws[:4] = 0
        return code

    def of(self, name):
        return [a for c, a in zip(self.calls, self.args) if c == name]

    def _stand_in(self, name):
        ws_at = dict(spd_pages_update=11, spd_decode_paged=8, spd_beam_select=7, spd_pages_compact=8)[name]

        def call(*a, **k):
            if name == "spd_decode_paged":
                assert a[4].is_contiguous()  # (positions)
            if name == "spd_beam_select":
                logits, scores, _, parent, token, out, ended, ws = a
                (R, n_in), W = scores.shape, parent.shape[1]
                assert ws.numel() >= N.spd_beam_select_workspace_size(R, n_in, W, logits.shape[1])
                parent.copy_(torch.arange(R)[:, None] * n_in + torch.arange(W)[None] % n_in)
                token.fill_(len(self.of(name)))
                out.fill_(-float(len(self.of(name)) + 1))
                ended.fill_(-float("inf") if self.ended is None else self.ended)
            self.calls.append(name)
            self.args.append((a, k))
            if name in self.fails:
                a[ws_at][:4] = torch.tensor([self.fails[name]], dtype=torch.int32).view(torch.uint8)
        return call


def _answer(n=2, W=3, vocab=8, **kw):
    class Model:
        cfg = dict(n_layers=2, n_kv_heads=1, head_dim=64, n_heads=2, vocab=vocab, d_model=64)
    return BeamAnswer(Model, torch.zeros(vocab, 64), n, W, n_pages=32, max_pages=8, page_size=16, **kw)


def _prompt(run, lens=(20, 7), **kw):
    return run.start(torch.zeros(sum(lens), 64), np.concatenate([[0], np.cumsum(lens)]), **kw)


@pytest.mark.parametrize("vocab", [8, 32000, 152064, 262144])
def test_the_workspace_holds_both_selections(lib, vocab):  # noqa: F811
    for R in range(1, 129):
        for W in range(1, 33):
            size = beams.select_workspace_size(R, W, vocab)
            assert size >= N.spd_beam_select_workspace_size(R, 1, W, vocab) and size >= N.spd_beam_select_workspace_size(R, W, W, vocab)


def test_a_search_of_many_requests_and_a_large_vocabulary_begins(lib, monkeypatch):  # noqa: F811
    _Library(monkeypatch)
    run = _answer(16, 8, 152064)  # the stand-in looks at the workspace
    _prompt(run, [1] * 16)
    run.step()
    assert run.texts.shape == (128, 2) and run.status() == 0


def test_positions_with_several_axes_pass_chunk_by_chunk(lib, monkeypatch):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer(chunk=8, axis=np.arange(32) % 3)
    pos = np.arange(3 * 27).reshape(3, 27) % 50
    _prompt(run, pos=pos)
    run.step()
    passes = [a for a, _ in L.of("spd_decode_paged")]
    want = [list(range(8)) + list(range(20, 27)), list(range(8, 16)), list(range(16, 20))]
    for a, idx in zip(passes, want):
        np.testing.assert_array_equal(a[4].numpy(), pos[:, idx])
    first = [pos[:, :20].max() + 1, pos[:, 20:].max() + 1]
    np.testing.assert_array_equal(passes[3][4].numpy(), np.tile(np.repeat(first, 3), (3, 1)))


def _state(run):
    return (run.texts.tolist(), run.scores.tolist(), run.lens.tolist(), run.next_pos.tolist(), [list(a) for a in run.answers])


@pytest.mark.parametrize("call,code", [("spd_decode_paged", N.SPD_EINVAL), ("spd_beam_select", -6), ("spd_pages_update", N.SPD_ENOSPC)])
def test_a_step_that_failed_takes_over_nothing_and_every_later_call_says_so(lib, monkeypatch, call, code):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer(eos=5)
    _prompt(run)
    run.step()
    was = _state(run)
    L.fails[call], L.ended = code, -3.0  # (ends that the failed step would add)
    with pytest.raises(N.SpiderError) as e:
        run.step()
    assert e.value.code == code == run.status() and _state(run) == was
    L.fails.clear()
    n = len(L.calls)
    for later in (run.step, run.best, run.compact, lambda: _prompt(run)):
        with pytest.raises(N.SpiderError) as e:
            later()
        assert e.value.code == code
    assert len(L.calls) == n and _state(run) == was and run.status() == code


@pytest.mark.parametrize("call,code", [("spd_decode_paged", N.SPD_EINVAL), ("spd_beam_select", -6), ("spd_pages_update", N.SPD_ENOSPC)])
def test_prompts_that_failed_give_no_answers(lib, monkeypatch, call, code):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer(eos=5)
    L.fails[call], L.ended = code, -3.0
    with pytest.raises(N.SpiderError):
        _prompt(run)
    assert run.answers == [[], []] and run.texts.shape[1] == 0
    L.fails.clear()
    for later in (run.best, run.compact, run.step):
        with pytest.raises(N.SpiderError):
            later()


def test_a_compaction_that_failed_says_so(lib, monkeypatch):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer()
    _prompt(run)
    L.fails["spd_pages_compact"] = N.SPD_EINVAL
    with pytest.raises(N.SpiderError):
        run.compact()
    with pytest.raises(N.SpiderError):
        run.step()


@pytest.mark.parametrize("match,lens,kw,rows", [
    ("prompt for", [20, 7], {}, 26),                                   # fewer rows than cu says: they would be read past the end
    ("prompt for", [20, 0], {}, 20),
    ("128 rows", [20, 129], {}, 149),                               # more than a table holds
    ("prefix", [20, 7], dict(prefix=[0, 8]), 27),
    ("prefix", [20, 7], dict(prefix=[-1, 0]), 27),
    ("prefix", [20, 7], dict(prefix=[3]), 27),
    ("pos", [20, 7], dict(pos=np.zeros((3, 26))), 27),
    ("pos", [20, 7], dict(pos=np.zeros(27)), 27),
])
def test_prompts_are_refused_before_anything_changes(lib, monkeypatch, match, lens, kw, rows):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer()
    _prompt(run)
    run.step()
    was, n = _state(run), len(L.calls)
    with pytest.raises(ValueError, match=match):
        run.start(torch.zeros(rows, 64), np.concatenate([[0], np.cumsum(lens)]), **kw)
    assert _state(run) == was and len(L.calls) == n
    run.step()


@pytest.mark.parametrize("cu", [[-3, 20, 27], [1, 20, 27], [0, 27], [0, 20, 27, 30]])
def test_prompts_that_do_not_begin_at_0(lib, monkeypatch, cu):  # noqa: F811
    _Library(monkeypatch)
    run = _answer()
    with pytest.raises(ValueError, match="prompt"):
        run.start(torch.zeros(30, 64), cu, pos=np.zeros((1, 27)))


def test_a_refused_pass_leaves_room_for_other_prompts(lib, monkeypatch):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer(chunk=8)
    with monkeypatch.context() as m:
        def refuse(*a, **k):
            if len(L.of("spd_decode_paged")) == 1:  # the second chunk, of one of two requests
                raise N.SpiderError(N.SPD_EINVAL, "refused")
            L._stand_in("spd_decode_paged")(*a, **k)
        m.setattr(N, "spd_decode_paged", refuse)
        with pytest.raises(N.SpiderError, match="refused"):
            _prompt(run)
    for early in (run.step, run.best):
        with pytest.raises(ValueError, match="start"):
            early()
    _prompt(run)
    run.step()
    assert run.texts.shape == (6, 2) and len(run.best()) == 2


def test_a_full_table_is_told_before_a_step_and_the_answers_stay(lib, monkeypatch):  # noqa: F811
    L = _Library(monkeypatch)
    run = _answer()
    with pytest.raises(ValueError, match="128 rows"):  # (no row for the first token)
        _prompt(run, [128, 7])
    _prompt(run, [126, 7])
    run.step()
    was, best, n = _state(run), run.best(), len(L.calls)
    for _ in range(2):
        with pytest.raises(N.SpiderError, match="128 rows") as e:
            run.step()
        assert e.value.code == N.SPD_EINVAL
    assert _state(run) == was and run.best() == best and run.status() == 0 and len(L.calls) == n
    _prompt(run)  # and others may follow
    run.step()
