"""A generation step over drafted tokens (spd_decode_tree) and answers made of such steps (TreeAnswer), against the
oracle's prefill of the sequence that each node ends.

Tolerances are those of the decode steps: logits within 2e-2 of each row's largest magnitude (bf16 operands through the
layers). A chosen token is right where the oracle's logit for it is within twice that of the oracle's best."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2609_34977_gb300 import _native as N
from paper_2609_34977_gb300 import synth
from paper_2609_34977_gb300.answer import TreeAnswer
from tests.gpu_util import bf16_np, rowwise_rel

pytestmark = pytest.mark.gpu
TOL = 2e-2


def _model(seed, **over):
    cfg = dict(synth.TINY_DECODER, n_layers=3, **over)
    w = synth.decoder_weights(seed, cfg, std=0.05)
    wd = {k: v.cuda() for k, v in w.items() if k != "layers"}
    wd["layers"] = [{k: v.cuda() for k, v in lw.items()} for lw in w["layers"]]
    return cfg, N.SpdModel(cfg, wd), od.model_from_torch(w, cfg)


def _rows(n, d, seed):
    return torch.randn(n, d, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


@pytest.mark.parametrize("lens,parents,over", [
    ([30], [[-1]], {}),                                                     # one token
    ([30, 45], [[-1, 0, 0, 1, 1, 2], [-1]], {}),
    ([5, 70, 33], [[-1, 0, 1, 2, 3], [-1, 0, 0, 0, -1], []], {}),           # a chain, a forest, a sequence without drafts
    ([20, 64], [[-1, 0, 0], [-1, 0, 1]], dict(n_heads=4, n_kv_heads=2, head_dim=128)),
    ([40], [[-1] + [i // 2 for i in range(30)]], dict(n_heads=8, n_kv_heads=2)),
])
def test_tree_step_equals_prefill_of_every_path(lens, parents, over):
    cfg, model, om = _model(61, **over)
    D, B, L, max_len = cfg["d_model"], len(lens), cfg["n_layers"], 112
    T, n = sum(lens), sum(len(p) for p in parents)
    x, new = _rows(T, D, 62), _rows(n, D, 63)
    cu, q_cu = np.cumsum([0] + lens).astype(np.int32), np.cumsum([0] + [len(p) for p in parents]).astype(np.int32)
    vis = np.zeros(T, bool)
    mask = np.zeros((L, T), np.uint8)
    for b, k in enumerate(lens):
        vis[cu[b]:cu[b] + k // 2] = True
    mask[:, vis] = np.random.default_rng(64).integers(0, 3, (L, int(vis.sum())))
    cache = torch.zeros(N.spd_kv_cache_bytes(model, B, max_len) // 2, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(N.spd_prefill_workspace_size(model, T, B), dtype=torch.uint8, device="cuda")
    N.spd_prefill_kv(model, x.cuda(), T, cu, mask, torch.zeros(T, D, device="cuda"), None, cache, max_len, ws)
    bits, depth = N.spd_tree_mask(np.concatenate([np.asarray(p, np.int32) for p in parents]), q_cu)
    pos = np.repeat(lens, [len(p) for p in parents]) + depth
    H, hd, G = cfg["n_heads"], cfg["head_dim"], cfg["n_kv_heads"]
    logits = torch.full((n, cfg["vocab"]), float("nan"), device="cuda")
    q = torch.zeros(L, n, H * hd, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((L, n, H), float("nan"), device="cuda")
    tws = torch.zeros(N.spd_decode_tree_workspace_size(model, n), dtype=torch.uint8, device="cuda")
    N.spd_decode_tree(model, new.cuda(), q_cu, lens, pos, torch.from_numpy(bits.view(np.int32)).cuda(), cache, max_len, logits,
                      tws, q_out=q, lse_out=lse)
    torch.cuda.synchronize()
    assert N.spd_workspace_status(tws) == 0
    got, want = logits.cpu().numpy(), []
    for b, ps in enumerate(parents):
        xb = bf16_np(x[cu[b]:cu[b + 1]])
        for i in range(len(ps)):
            path, at = [], i
            while at >= 0:
                path.insert(0, at)
                at = ps[at]
            full = np.concatenate([xb] + [bf16_np(new[q_cu[b] + j:q_cu[b] + j + 1]) for j in path])
            m = np.concatenate([mask[:, cu[b]:cu[b + 1]], np.zeros((L, len(path)), np.uint8)], 1)
            want.append(od.prefill(om, full, [0, len(full)], m)[1][0])
    assert np.isfinite(got).all() and rowwise_rel(got, np.array(want)) < TOL
    # q and lse are what the weights need: the first node of a sequence spreads one unit a head over the rows it sees
    first = [int(q_cu[b]) for b in range(B) if parents[b]]
    r_cu = np.cumsum([0] + [int(bool(p)) for p in parents]).astype(np.int32)
    acc = torch.zeros(L, B, G, max_len, device="cuda")
    N.spd_cache_weights(q, lse, torch.tensor(first, dtype=torch.int32, device="cuda"), r_cu, cache, np.array(lens) + 1, max_len, H,
                        G, hd, 1.0, acc, acc)
    total = acc.sum(-1).cpu().numpy()
    for b in range(B):
        np.testing.assert_allclose(total[:, b], H // G if parents[b] else 0.0, rtol=1e-4)


def _answers(seed, lens, **kw):
    cfg, model, om = _model(seed)
    embed = _rows(cfg["vocab"], cfg["d_model"], seed + 1)
    tokens = np.random.default_rng(seed).integers(0, cfg["vocab"], sum(lens))
    cu = np.cumsum([0] + lens)
    run = TreeAnswer(model, embed.cuda(), len(lens), 160, **kw)
    return cfg, om, embed, tokens, cu, run


def _start(run, embed, tokens, cu, **kw):
    return run.start(embed[tokens].cuda(), cu, tokens, **kw)


def _check_greedy(om, embed, prompt, said, layers):
    """Every token of `said` is the oracle's best after the prompt and the tokens before it (or as good as)."""
    for k in range(len(said)):
        xb = bf16_np(embed[np.concatenate([prompt, said[:k]]).astype(np.int64)])
        z = od.prefill(om, xb, [0, len(xb)], np.zeros((layers, len(xb)), np.uint8))[1][0]
        assert z[said[k]] >= z.max() - 2 * TOL * np.abs(z).max(), k


def test_answers_with_and_without_drafts():
    lens = [40, 23]
    cfg, om, embed, tokens, cu, run = _answers(71, lens, max_nodes=8)
    said = [[t] for t in _start(run, embed, tokens, cu, window=8)]
    for _ in range(9):
        for s, new in zip(said, run.step()):
            assert len(new) == 1
            s.extend(new)
    assert run.status() == 0
    for b in range(2):
        _check_greedy(om, embed, tokens[cu[b]:cu[b + 1]], said[b], cfg["n_layers"])
    # the same again with drafts: what was said, behind wrong ones, two or three tokens deep
    run2 = _answers(71, lens, max_nodes=8)[5]
    got = [[t] for t in _start(run2, embed, tokens, cu, window=8)]
    steps = 0
    while min(len(g) for g in got) < 10:
        drafts = []
        for b in range(2):
            rest = said[b][len(got[b]):len(got[b]) + 3] if got[b] == said[b][:len(got[b])] else []
            d = [((t + 7) % cfg["vocab"], 0) for t in rest[:1]]
            for k, t in enumerate(rest):
                d.append((t, 0 if k == 0 else len(d)))
            drafts.append(d)
        for g, new in zip(got, run2.step(drafts)):
            g.extend(new)
        steps += 1
    assert run2.status() == 0 and run2.lens.tolist() == [lens[b] + len(got[b]) - 1 for b in range(2)]
    for b in range(2):
        _check_greedy(om, embed, tokens[cu[b]:cu[b + 1]], got[b], cfg["n_layers"])
    if all(g[:10] == s[:10] for g, s in zip(got, said)):
        assert steps <= 4  # nine tokens, up to four a step


def test_answers_refuse_prompts_without_a_window():
    _, _, embed, tokens, _, run = _answers(71, [5, 1])
    for cu, kw in (([0, 5, 6], {}), ([0, 6], {}), ([0, 3, 6], dict(window=0))):
        with pytest.raises(ValueError, match="start"):
            _start(run, embed, tokens, cu, **kw)
    with pytest.raises(ValueError, match="drafts"):
        run.pending = [1, 1]
        run.step([[(1, 0)] * 40, []])


def test_answers_refuse_drafts_outside_the_vocabulary():
    cfg, _, embed, tokens, cu, run = _answers(71, [40, 23])
    _start(run, embed, tokens, cu, window=8)
    for t in (-1, cfg["vocab"]):
        with pytest.raises(ValueError, match="vocabulary"):
            run.step([[], [(3, 0), (t, 1)]])
    assert run.lens.tolist() == [40, 23] and all(len(x) == 1 for x in run.step())


def test_a_second_answer_begins_afresh():
    N.spd_set_deterministic(True)
    try:
        kw = dict(max_nodes=4, budget=64, n_recent=16)
        _, _, embed, tokens, cu, run = _answers(91, [120, 50], **kw)
        _start(run, embed, tokens, cu, window=16)
        for _ in range(3):
            run.step([[(5, 0)], [(3, 0)]])
        said = [_start(r, embed, tokens, cu, window=16) for r in (run, _answers(91, [120, 50], **kw)[5])]
        new = _answers(91, [120, 50], **kw)[5]
        assert said[0] == said[1] == _start(new, embed, tokens, cu, window=16)
        assert run.lens.tolist() == new.lens.tolist() and run.next_pos.tolist() == new.next_pos.tolist()
        for b, n in enumerate(run.lens):
            assert torch.equal(run.acc[:, b, :, :n], new.acc[:, b, :, :n])
            assert torch.equal(run.pos[:, b, :, :n], new.pos[:, b, :, :n])
            assert torch.equal(run.kv[:, b, :n].view(torch.int16), new.kv[:, b, :n].view(torch.int16))
    finally:
        N.spd_set_deterministic(False)


def test_answers_within_a_budget():
    # the rows that stay are rows of the whole cache, at the positions that the bookkeeping says
    N.spd_set_deterministic(True)
    try:
        lens, budget = [120, 50], 64
        cfg, om, embed, tokens, cu, whole = _answers(81, lens, max_nodes=4)
        cut = _answers(81, lens, max_nodes=4, budget=budget, n_recent=16)[5]
        a, b = _start(whole, embed, tokens, cu, window=16), _start(cut, embed, tokens, cu, window=16)
        assert a == b and cut.lens.tolist() == [64, 50] and cut.next_pos.tolist() == lens
        L, G, d = cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"]
        full = whole.kv.view(torch.int16).cpu().numpy().reshape(L, 2, 160, 2, G, d)
        left = cut.kv.view(torch.int16).cpu().numpy().reshape(L, 2, 160, 2, G, d)
        pos, acc = cut.pos.cpu().numpy(), cut.acc.cpu().numpy()
        for l, s, g in np.ndindex(L, 2, G):
            n = cut.lens[s]
            p = pos[l, s, g, :n]
            assert len(set(p.tolist())) == n and set(range(4)) <= set(p.tolist())
            assert set(range(lens[s] - 16, lens[s])) <= set(p.tolist())
            np.testing.assert_array_equal(left[l, s, :n, :, g], full[l, s, p][:, :, g])
            assert (acc[l, s, g, n:lens[s]] == 0).all()
        # the total that the window gave, over evicted rows too, is a unit a row and head: what is left is less
        assert (acc.sum(-1) <= 16 * cfg["n_heads"] // G * (1 + 1e-4)).all() and (acc.sum(-1) > 0).all()
        for k in range(12):
            new = cut.step([[(5, 0), (9, 0)], [(3, 0)]])
            assert all(len(x) >= 1 for x in new) and (cut.lens <= budget).all()
        assert cut.status() == 0 and (cut.next_pos >= np.array(lens) + 12).all()
    finally:
        N.spd_set_deterministic(False)


def test_answers_keep_to_their_rules():
    lens = [20, 20]
    cfg, model, om = _model(91)
    words = (cfg["vocab"] + 31) // 32
    allow = np.zeros((2, words), np.int32)
    allow[0] = 0x55555555            # even tokens
    allow[1, 3] = -1                 # tokens 96 to 127
    rules = dict(repetition=torch.tensor([1e6, 1.0], device="cuda"), presence=torch.tensor([1e6, 0.0], device="cuda"),
                 allow=torch.from_numpy(allow).cuda(), rule=lambda b, said: b)
    _, _, embed, tokens, cu, run = _answers(91, lens, max_nodes=4, rules=rules)
    said = [[t] for t in _start(run, embed, tokens, cu)]
    for _ in range(10):
        for s, new in zip(said, run.step([[(said[0][-1], 0)], []])):
            s.extend(new)
    assert all(t % 2 == 0 for t in said[0]) and all(96 <= t < 128 for t in said[1])
    assert len(set(said[0])) == len(said[0])  # a repeated token costs more than any logit
    none = dict(rules, allow=torch.zeros(1, words, dtype=torch.int32, device="cuda"), rule=lambda b, said: 0 if b else -1)
    run = _answers(91, lens, max_nodes=4, rules=none)[5]
    assert _start(run, embed, tokens, cu)[1] == -1
    assert run.step()[1] == [] and run.lens.tolist() == [21, 20]
