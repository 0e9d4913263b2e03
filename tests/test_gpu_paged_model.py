"""Passes and beam search over pages against a plain decoder in 64 bits: grouped heads of 128, positions with three axes (time, height,
width), prefixes that see themselves whole, through spd_decode_paged and through BeamAnswer; a search of many requests over a large
vocabulary.

Tolerances: logits of the bf16 pipeline are off by at most 2e-2 of a row's largest, as the prefill's. A logarithm of a probability is a
logit less a logarithm of a sum of exponentials, either off by at most the logits' error e: 2 e a token, added up over an answer's."""
import numpy as np
import pytest
import torch

from oracle import decoder as od
from paper_2609_34977_gb300.beams import BeamAnswer
from tests.gpu_util import bf16_np, rowwise_rel
from tests.test_gpu_beams import TOL, _cu, _embed, _model, fixed_order, pytestmark  # noqa: F401

GROUPED = dict(n_layers=3, d_model=512, n_heads=14, n_kv_heads=2, head_dim=128, d_ffn=768, vocab=1016, rope_theta=1e6, rms_eps=1e-6)
AXIS = np.repeat([0, 1, 2], [16, 24, 24]).astype(np.uint8)


def _plain(model, x, pos, axis, prefix):
    """Logits of the last token of one sequence: x [n][d_model], pos [axes][n]."""
    cfg, n, rnd = model["cfg"], len(x), od.bf16_round
    H, G, d, eps = cfg["n_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["rms_eps"]
    angle = np.asarray(pos, np.float64)[axis].T * cfg["rope_theta"] ** (-2.0 * np.arange(d // 2) / d)  # [n][d / 2]
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    sees = np.arange(n)[None] < np.maximum(np.arange(n) + 1, prefix)[:, None]

    def turn(a, heads):
        a = a.reshape(n, heads, d)
        lo, hi = a[..., :d // 2], a[..., d // 2:]
        return rnd(np.concatenate([lo * c - hi * s, lo * s + hi * c], -1))

    h = np.array(x, np.float64)
    for w in model["layers"]:
        a = rnd(od.rmsnorm(h, w["attn_norm"], eps))
        q, k, v = turn(a @ w["wq"].T, H), turn(a @ w["wk"].T, G), rnd(a @ w["wv"].T).reshape(n, G, d)
        o = np.zeros((n, H, d))
        for i in range(H):
            z = np.where(sees, q[:, i] @ k[:, i // (H // G)].T / np.sqrt(d), -np.inf)
            p = np.exp(z - z.max(1, keepdims=True))
            o[:, i] = p / p.sum(1, keepdims=True) @ v[:, i // (H // G)]
        h = h + rnd(o.reshape(n, H * d)) @ w["wo"].T
        y = rnd(od.rmsnorm(h, w["ffn_norm"], eps))
        h = h + rnd(od.silu(y @ w["w_gate"].T) * (y @ w["w_up"].T)) @ w["w_down"].T
    return rnd(od.rmsnorm(h[-1:], model["final_norm"], eps)) @ model["lm_head"].T


def _positions(n, image):
    """An image of `image` tokens, seven a row, and text behind it: [3][n]."""
    at = np.arange(image)
    pos = np.stack([np.zeros(image, int), at // 7, at % 7])
    text = np.arange(n - image) + (pos.max() + 1 if image else 0)
    return np.concatenate([pos, np.tile(text, (3, 1))], 1)


LENS, IMAGES = [90, 33, 150], [41, 0, 112]


@pytest.mark.parametrize("chunks", [[[90, 33, 150]], [[64, 30, 130], [25, 2, 19], [1, 1, 1]], [[41, 16, 112]] + [[7, 2, 5]] * 7 + [[0, 3, 3]]])
@pytest.mark.parametrize("prefix", [None, IMAGES])
def test_passes_with_grouped_heads_axes_and_prefixes(chunks, prefix):
    cfg, w, model = _model(3, **GROUPED)
    x, cu, ref = _embed(cfg)[:sum(LENS)], _cu(LENS), od.model_from_torch(w, cfg)
    pos = [_positions(n, k) for n, k in zip(LENS, IMAGES)]
    want = np.concatenate([_plain(ref, bf16_np(x[cu[b]:cu[b + 1]]), pos[b], AXIS, prefix[b] if prefix else 0) for b in range(3)])
    got = _run(model, cfg, x, pos, chunks, prefix)
    assert rowwise_rel(got, want) < TOL
    # positions and prefixes count: without them the answers are others
    flat = [np.tile(np.arange(n), (3, 1)) for n in LENS]
    for other in ([_plain(ref, bf16_np(x[cu[b]:cu[b + 1]]), flat[b], AXIS, prefix[b] if prefix else 0) for b in (0, 2)],
                  [_plain(ref, bf16_np(x[cu[b]:cu[b + 1]]), pos[b], AXIS, 0 if prefix else IMAGES[b]) for b in (0, 2)]):
        assert rowwise_rel(np.concatenate(other), want[[0, 2]]) > 2 * TOL


def _run(model, cfg, x, pos, chunks, prefix):
    """The prompts in passes; a sequence without a token in a chunk is left out of its pass. Logits of the last tokens."""
    from paper_2609_34977_gb300 import _native as N
    B, page, cu = len(pos), 16, _cu(LENS)
    r = np.random.default_rng(1)
    need = [-(-n // page) for n in LENS]
    order = r.permutation(sum(need) + 2)
    table = np.full((B, max(need)), -1, np.int32)
    for b, at in enumerate(_cu(need)[:-1]):
        table[b, :need[b]] = order[at:at + need[b]]
    pool = torch.full((cfg["n_layers"], len(order), page, 2 * cfg["n_kv_heads"] * cfg["head_dim"]), float("nan"),
                      dtype=torch.bfloat16, device="cuda")
    out, done = np.zeros((B, cfg["vocab"])), np.zeros(B, int)
    for step in chunks:
        live = [b for b in range(B) if step[b]]
        idx = np.concatenate([np.arange(cu[b] + done[b], cu[b] + done[b] + step[b]) for b in live])
        at = np.concatenate([pos[b][:, done[b]:done[b] + step[b]] for b in live], 1)
        done += step
        logits = torch.full((len(live), cfg["vocab"]), float("nan"), device="cuda")
        ws = torch.zeros(N.spd_decode_paged_workspace_size(model, len(idx), len(live)), dtype=torch.uint8, device="cuda")
        N.spd_decode_paged(model, x[torch.from_numpy(idx).cuda()], _cu([step[b] for b in live]), done[live],
                           torch.from_numpy(np.ascontiguousarray(at, dtype=np.int32)).cuda(), torch.from_numpy(table[live]).cuda(), pool,
                           logits, ws, axis=AXIS, prefix=[prefix[b] for b in live] if prefix else None)
        torch.cuda.synchronize()
        assert N.spd_workspace_status(ws) == 0
        out[live] = logits.cpu().numpy()
    assert (done == LENS).all()
    return out


def _logprob(ref, embed, prompt, pos, axis, prefix, said):
    """Logarithm of the probability of the tokens `said` behind a prompt's embeddings, and the bound of a pipeline's error."""
    total = tol = 0.0
    nxt = np.asarray(pos).max() + 1
    for k, t in enumerate(said):
        x = np.concatenate([prompt, embed[said[:k]]])
        at = np.concatenate([pos, np.tile(nxt + np.arange(k), (len(pos), 1))], 1)
        z = _plain(ref, x, at, axis, prefix)[0]
        total += z[t] - z.max() - np.log(np.exp(z - z.max()).sum())
        tol += 2 * TOL * np.abs(z).max()
    return total, tol


@pytest.mark.parametrize("chunk", [32, 500])
def test_a_search_behind_images(chunk):
    cfg, w, model = _model(3, **GROUPED)
    embed, ref, cu = _embed(cfg), od.model_from_torch(w, cfg), _cu(LENS)
    x = _embed(cfg, 7)[:sum(LENS)]
    pos = [_positions(n, k) for n, k in zip(LENS, IMAGES)]
    run = BeamAnswer(model, embed, 3, 3, n_pages=120, max_pages=12, page_size=16, axis=AXIS, chunk=chunk)
    run.start(x, cu, pos=np.concatenate(pos, 1), prefix=IMAGES)
    for _ in range(4):
        run.step()
    assert run.compact() <= 120
    run.step()
    e = bf16_np(embed)
    for b, answers in enumerate(run.best()):
        assert len({tuple(t) for _, t in answers}) == 3 and all(len(t) == 6 for _, t in answers)
        for score, said in answers[::2]:
            want, tol = _logprob(ref, e, bf16_np(x[cu[b]:cu[b + 1]]), pos[b], AXIS, IMAGES[b], said)
            assert abs(score - want) <= tol, (b, score, want, tol)
            other, _ = _logprob(ref, e, bf16_np(x[cu[b]:cu[b + 1]]), pos[b], AXIS, 0, said)
            assert not IMAGES[b] or abs(want - other) > 1e-3  # (the prefix counts)


def test_a_search_of_many_requests_over_a_large_vocabulary():
    # one row a request is cut into more slices than its eight beams have together
    cfg, w, model = _model(2, vocab=152064)
    r = np.random.default_rng(6)
    embed = _embed(cfg)
    lens = [int(n) for n in r.integers(1, 40, 16)]
    tokens = r.integers(0, cfg["vocab"], sum(lens))
    cu = _cu(lens)
    run = BeamAnswer(model, embed, 16, 8, n_pages=600, max_pages=8, page_size=16)
    run.start(embed[torch.from_numpy(tokens).cuda()], cu)
    for _ in range(3):
        run.step()
    ref, e = od.model_from_torch(w, cfg), bf16_np(embed)
    one = np.zeros(cfg["head_dim"] // 2, int)
    best = run.best()
    for b in (0, 7, 15):
        assert len({tuple(t) for _, t in best[b]}) == 8
        for score, said in (best[b][0], best[b][7]):
            want, tol = _logprob(ref, e, e[tokens[cu[b]:cu[b + 1]]], np.arange(lens[b])[None], one, 0, said)
            assert abs(score - want) <= tol, (b, score, want, tol)
