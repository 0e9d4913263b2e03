"""The host side of answers (no GPU): tensors on the CPU, the library's calls as stand-ins."""
import numpy as np
import pytest
import torch

from paper_2609_34977_gb300 import _native as N
from paper_2609_34977_gb300.answer import TreeAnswer


class _Library:
    """Stand-ins that record their calls; `fails` maps a call to the status that it leaves in its workspace."""

    def __init__(self, monkeypatch):
        from paper_2609_34977_gb300 import answer
        self.calls, self.fails, self.best = [], {}, 3

        class Torch:
            def __getattr__(self, name):
                f = getattr(torch, name)
                if name in ("zeros", "empty", "arange", "tensor"):
                    return lambda *a, **k: f(*a, **{x: y for x, y in k.items() if x != "device"})
                return f
        monkeypatch.setattr(answer, "torch", Torch())
        monkeypatch.setattr(torch.Tensor, "cuda", lambda t: t)
        N = answer.N
        for name, at in (("spd_prefill_kv", 9), ("spd_decode_tree", 9), ("spd_logits_process", None), ("spd_tree_commit", None),
                         ("spd_cache_weights", 13), ("spd_cache_evict", None)):
            monkeypatch.setattr(N, name, self._stand_in(name, at))
        for name in ("prefill", "decode_tree", "tree_commit", "cache_evict"):
            monkeypatch.setattr(N, f"spd_{name}_workspace_size", lambda *a: 64)
        monkeypatch.setattr(N, "spd_workspace_status", self._status)

    @staticmethod
    def _status(ws):  # reads and clears
        code = int(ws[:4].view(torch.int32))
        ws[:4] = 0
        return code

    def _stand_in(self, name, at):
        def call(*a, **k):
            self.calls.append(name)
            if name == "spd_logits_process":
                a[2].fill_(self.best)
            if name == "spd_cache_evict":
                return np.minimum(a[1], a[5])
            if name in self.fails:
                a[at][:4] = torch.tensor([self.fails[name]], dtype=torch.int32).view(torch.uint8)
        return call


def _answer(n=1, **kw):
    class Model:
        cfg = dict(n_layers=2, n_kv_heads=1, head_dim=64, n_heads=2, vocab=8, d_model=64)
    return TreeAnswer(Model, torch.zeros(8, 64), n, 128, **kw)


def _prompt(run, n=10, **kw):
    return run.start(torch.zeros(n, 64), [0, n], np.arange(n) % 8, **kw)


@pytest.mark.parametrize("call,code", [("spd_prefill_kv", -7), ("spd_decode_tree", -6)])
def test_a_prompt_whose_device_work_failed_says_so(monkeypatch, call, code):
    lib = _Library(monkeypatch)
    run = _answer()
    lib.fails[call] = code
    with pytest.raises(N.SpiderError) as e:
        _prompt(run)
    assert e.value.code == code == run.status() and run.pending == [None] and "spd_tree_commit" not in lib.calls


def test_a_step_whose_device_work_failed_takes_over_no_token(monkeypatch):
    lib = _Library(monkeypatch)
    run = _answer(budget=64)
    assert _prompt(run) == [3] and run.step() == [[3]] and run.status() == 0
    lens, hist = run.lens.tolist(), list(run.hist[0])
    lib.fails["spd_decode_tree"] = -6
    lib.calls.clear()
    with pytest.raises(N.SpiderError):
        run.step([[(5, 0)]])
    assert run.lens.tolist() == lens and run.hist[0] == hist and "spd_tree_commit" not in lib.calls
    lib.fails.clear()
    with pytest.raises(N.SpiderError):
        run.step()
    assert run.status() == -6


def test_weights_that_failed_show_in_the_next_step(monkeypatch):
    lib = _Library(monkeypatch)
    run = _answer(budget=64)
    lib.fails["spd_cache_weights"] = -5
    _prompt(run)
    assert run.status() == -5
    with pytest.raises(N.SpiderError):
        run.step()


def test_a_larger_workspace_keeps_what_the_smaller_one_recorded(monkeypatch):
    _Library(monkeypatch)
    run = _answer(max_nodes=4)
    small = run.ws
    small[:4] = torch.tensor([-6], dtype=torch.int32).view(torch.uint8)
    run._room(40)
    assert run.ws is not small and run.status() == -6
    run.ws[:4] = torch.tensor([-7], dtype=torch.int32).view(torch.uint8)
    assert run.status() == -6  # the first one
