"""Passes over a paged cache (spd_decode_paged) against the fp64 oracle and against each other, and beam search over it (BeamAnswer).

Tolerances: hidden states and logits of the bf16 pipeline are compared with the oracle at 2e-2 of a row's largest, as the prefill's; Q
and K are rounded to bf16 once more (before their rotation), 2^-8 of a value at most, which the attention averages. A score of an
answer of s tokens is a sum of s logarithms of probabilities, each off by at most twice the logits' error."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2609_34977_gb300 import _native as N
from paper_2609_34977_gb300 import synth
from paper_2609_34977_gb300.beams import BeamAnswer
from tests.gpu_util import bf16_np, rowwise_rel

pytestmark = pytest.mark.gpu
TOL = 2e-2


@pytest.fixture(autouse=True)
def fixed_order():
    """The GEMMs' sums in a fixed order: some tests compare bits."""
    N.spd_set_deterministic(True)
    yield
    N.spd_set_deterministic(False)


def _model(seed=1, **kw):
    cfg = dict(synth.TINY_DECODER, **kw)
    w = synth.decoder_weights(seed, cfg, std=0.05)
    wd = {k: v.cuda() for k, v in w.items() if k != "layers"}
    wd["layers"] = [{k: v.cuda() for k, v in lw.items()} for lw in w["layers"]]
    return cfg, w, N.SpdModel(cfg, wd)


def _embed(cfg, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(cfg["vocab"], cfg["d_model"], generator=g).to(torch.bfloat16).cuda()


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _cu(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def _passes(model, cfg, x, lens, chunks, page=16, axes=1, axis=None, prefix=None, seed=0):
    """The prompts in passes of chunks[i] tokens a sequence; the logits after the last."""
    r = np.random.default_rng(seed)
    B, cu = len(lens), _cu(lens)
    need = [-(-n // page) for n in lens]
    order = r.permutation(sum(need) + 3)
    table = np.full((B, max(need)), -1, np.int32)
    for b, at in enumerate(_cu(need)[:-1]):
        table[b, :need[b]] = order[at:at + need[b]]
    pool = torch.full((cfg["n_layers"], len(order), page, 2 * cfg["n_kv_heads"] * cfg["head_dim"]), float("nan"), dtype=torch.bfloat16,
                      device="cuda")  # nobody may read what was not written
    t = torch.from_numpy(table).cuda()
    logits = torch.full((B, cfg["vocab"]), float("nan"), device="cuda")
    done = np.zeros(B, int)
    for step in chunks:
        idx = np.concatenate([np.arange(cu[b] + done[b], cu[b] + done[b] + step[b]) for b in range(B)])
        pos = np.concatenate([np.arange(done[b], done[b] + step[b]) for b in range(B)])
        done += step
        ws = torch.zeros(N.spd_decode_paged_workspace_size(model, len(idx), B), dtype=torch.uint8, device="cuda")
        N.spd_decode_paged(model, x[torch.from_numpy(idx).cuda()], _cu(step), done, torch.from_numpy(np.tile(pos, (axes, 1))).int().cuda(),
                           t, pool, logits, ws, axis=axis, prefix=prefix)
        torch.cuda.synchronize()
        assert N.spd_workspace_status(ws) == 0
    assert (done == lens).all()
    return logits


@pytest.mark.parametrize("lens,chunks", [
    ([37], [[37]]),
    ([37], [[20], [16], [1]]),
    ([70, 5, 130], [[70, 5, 130]]),
    ([70, 9, 130], [[64, 7, 64], [5, 1, 65], [1, 1, 1]]),
])
def test_passes_against_the_oracle(lens, chunks):
    cfg, w, model = _model()
    x = _embed(cfg)[:sum(lens)]
    got = _passes(model, cfg, x, lens, chunks).cpu().numpy()
    _, want = od.prefill(od.model_from_torch(w, cfg), bf16_np(x), _cu(lens), np.zeros((cfg["n_layers"], sum(lens)), np.uint8))
    assert rowwise_rel(got, want) < TOL


def test_equal_axes_are_one_axis_and_prompts_without_an_image_have_no_prefix():
    cfg, _, model = _model()
    lens, x = [50, 33], _embed(cfg)[:83]
    one = _passes(model, cfg, x, lens, [[40, 30], [10, 3]])
    d = cfg["head_dim"]
    three = _passes(model, cfg, x, lens, [[40, 30], [10, 3]], axes=3, axis=np.arange(d // 2) % 3)
    assert torch.equal(one, three)
    assert torch.equal(one, _passes(model, cfg, x, lens, [[40, 30], [10, 3]], prefix=[0, 0]))
    other = _passes(model, cfg, x, lens, [[40, 30], [10, 3]], prefix=[40, 30])
    assert not torch.equal(one, other) and torch.isfinite(other).all()


def test_pass_refusals():
    cfg, _, model = _model()
    B, page = 2, 16
    kvd = cfg["n_kv_heads"] * cfg["head_dim"]
    pool = torch.zeros(cfg["n_layers"], 4, page, 2 * kvd, dtype=torch.bfloat16, device="cuda")
    t = torch.zeros(B, 2, dtype=torch.int32, device="cuda")
    x, pos = _embed(cfg)[:3], torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    ws = torch.zeros(N.spd_decode_paged_workspace_size(model, 3, B), dtype=torch.uint8, device="cuda")
    for cu, lens, size, code, match in (([0, 3, 3], [3, 5], None, N.SPD_EINVAL, "no new token"), ([0, 1, 3], [1, 33], None, N.SPD_EINVAL, "rows"),
                                        ([0, 1, 3], [1, 1], None, N.SPD_EINVAL, "rows"), ([0, 1, 3], [1, 2], 1 << 12, N.SPD_ENOSPC, "workspace")):
        with pytest.raises(N.SpiderError, match=match) as e:
            N.spd_decode_paged(model, x, cu, lens, pos, t, pool, None, ws[:size], prefix=None)
        assert e.value.code == code
    with pytest.raises(ValueError, match="layers"):
        N.spd_decode_paged(model, x, [0, 1, 3], [1, 2], pos, t, pool[:cfg["n_layers"] - 1], None, ws)


def test_a_pass_is_not_captured():
    # it uploads lists from host memory, which a replay would find changed
    cfg, _, model = _model()
    pool = torch.zeros(cfg["n_layers"], 2, 16, 2 * cfg["n_kv_heads"] * cfg["head_dim"], dtype=torch.bfloat16, device="cuda")
    t, x, pos = _i32([[0]]), _embed(cfg)[:3], torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    ws = torch.zeros(N.spd_decode_paged_workspace_size(model, 3, 1), dtype=torch.uint8, device="cuda")
    y = torch.zeros(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(N.SpiderError, match="captured") as e:
            N.spd_decode_paged(model, x, [0, 3], [3], pos, t, pool, None, ws)
        y += 1  # the capture goes on
    assert e.value.code == N.SPD_EUNSUPPORTED
    graph.replay()
    torch.cuda.synchronize()
    assert float(y) == 1 and (pool == 0).all()


def _logprobs(model, cfg, embed, tokens, n_prompt):
    """Sum of the log-probabilities of tokens[n_prompt:], from prefills of every prefix."""
    total = 0.0
    for k in range(n_prompt, len(tokens)):
        x = embed[torch.tensor(tokens[:k], device="cuda")]
        h, lg = torch.empty(k, cfg["d_model"], device="cuda"), torch.empty(1, cfg["vocab"], device="cuda")
        ws = torch.zeros(N.spd_prefill_workspace_size(model, k, 1), dtype=torch.uint8, device="cuda")
        N.spd_prefill(model, x, k, [0, k], None, h, lg, ws)
        total += float(torch.log_softmax(lg[0].double(), 0)[tokens[k]])
    return total


def _search(model, cfg, embed, prompts, W, steps, compact=False, chunk=32, eos=-1):
    run = BeamAnswer(model, embed, len(prompts), W, n_pages=200, max_pages=8, page_size=16, eos=eos, chunk=chunk)
    run.start(embed[torch.tensor(sum(prompts, []), device="cuda")], _cu([len(p) for p in prompts]))
    for _ in range(steps - 1):
        if compact:
            run.compact()
        run.step()
    # the reference counts are what the tables list
    t, ref = run.tables[run.now][:run.B].cpu().numpy(), run.ref.cpu().numpy()
    listed = np.zeros_like(ref)
    for row in t:
        np.add.at(listed, row[row >= 0], 1)
    np.testing.assert_array_equal(ref, listed)
    return run


def test_beam_search():
    cfg, _, model = _model()
    embed = _embed(cfg)
    r = np.random.default_rng(4)
    prompts = [r.integers(0, cfg["vocab"], n).tolist() for n in (45, 16, 33)]
    W, steps = 4, 7
    run = _search(model, cfg, embed, prompts, W, steps)
    scores, texts = run.scores.cpu().numpy(), run.texts.cpu().numpy().reshape(3, W, steps)
    for b, p in enumerate(prompts):
        assert (np.diff(scores[b]) <= 0).all() and len({tuple(t) for t in texts[b]}) == W
        for w in (0, W - 1):
            want = _logprobs(model, cfg, embed, p + texts[b, w].tolist(), len(p))
            assert abs(want - scores[b, w]) < 0.05 * steps, (b, w, want, scores[b, w])
    # compaction between the steps and other chunks move rows and nothing else
    again = _search(model, cfg, embed, prompts, W, steps, compact=True)
    assert torch.equal(again.texts, run.texts) and torch.equal(again.scores, run.scores)
    assert again.compact() == int((run.ref > 0).sum())
    whole = _search(model, cfg, embed, prompts, W, steps, chunk=500)
    np.testing.assert_allclose(whole.scores.cpu().numpy(), scores, atol=0.05 * steps)
    # one beam is the greedy answer
    one = _search(model, cfg, embed, prompts, 1, 3)
    assert one.texts.shape == (3, 3) and torch.isfinite(one.scores).all()


def test_answers_end_and_requests_begin_anew():
    cfg, _, model = _model()
    embed = _embed(cfg)
    r = np.random.default_rng(5)
    prompts = [r.integers(0, cfg["vocab"], n).tolist() for n in (20, 31)]
    free = _search(model, cfg, embed, prompts, 3, 4)
    eos = int(free.texts.cpu().numpy().reshape(2, 3, 4)[0, 0, 2])  # a token that the best beam says
    run = _search(model, cfg, embed, prompts, 3, 5, eos=eos)
    assert run.answers[0] and all(eos not in t for b in run.best() for _, t in b)
    for s, t in run.answers[0][:2]:
        want = _logprobs(model, cfg, embed, prompts[0] + t + [eos], len(prompts[0]))
        assert abs(want - s) < 0.05 * (len(t) + 1)
    first = run.best()
    run.start(embed[torch.tensor(sum(prompts, []), device="cuda")], _cu([len(p) for p in prompts]))
    for _ in range(4):
        run.step()
    assert run.best() == first


def test_a_pool_that_is_too_small():
    cfg, _, model = _model()
    embed = _embed(cfg)
    run = BeamAnswer(model, embed, 1, 4, n_pages=4, max_pages=8, page_size=16)
    with pytest.raises(N.SpiderError) as e:
        run.start(embed[:60], [0, 60])
        for _ in range(20):
            run.step()
    assert e.value.code == N.SPD_ENOSPC
    with pytest.raises(N.SpiderError):
        run.step()
