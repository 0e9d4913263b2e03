"""Drafted-token attention over the cache, received weights, eviction, commit and logit rules against plain
implementations in 64 bits (numpy on the host).

Tolerances, from the arithmetic of the operators:
  scores    fp32 sums of d exact bf16 products: |error| <= e_s = d 2^-24 max_j sum_c |q_c k_jc| / sqrt(d)
  lse       e_s, the exponentials' and the logarithm's few units (2^-20) and the rounding of the result (2^-22 |lse|)
  o         one rounding to bf16 (2^-8 |o|, twice the half unit), weights off by e_s twice (score and normaliser) and held in at
            least 16 bits: (2 e_s + 2^-15) sum_j p_j |v_j|
  weights   each e^(s - lse) off by (e_s + 2^-20) of itself and of the exponent's rounding (2^-23 |s - lse|, below
            2^-18 here), the sum by 2^-20 of itself
Integers, moved rows and weights are equal bit for bit. Logits: the steps are single fp32 operations, at most 6 of
them on a value: 6 2^-24 of the sum of the magnitudes that enter.
"""
import math

import numpy as np
import pytest
import torch

from paper_2609_34977_gb300 import _native as N
from tests.gpu_util import bf16_np

pytestmark = pytest.mark.gpu


def _rand(shape, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(torch.bfloat16)


def _cu(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def _see(r, n, form):
    """[n][n] which drafts a node sees."""
    if form == "any":  # any set of drafts at all, the empty one included
        see = r.random((n, n)) < 0.3
        see[::3] = False
        return see
    see = np.eye(n, dtype=bool)
    for i in range(1, n):
        see[i] |= see[i - 1 if form == "chain" else r.integers(0, i)]
    return see


def _words(see, words):
    full = np.zeros((see.shape[0], 32 * words), np.uint8)
    full[:, :see.shape[1]] = see
    return np.packbits(full, axis=1, bitorder="little").view(np.int32)


def _plain_rows(q, kv, see, g, m, d):
    """Rows q [n][g m d] over keys kv [k][2 g d] (float64), see [n][k]: o, lse, the bounds of their errors."""
    n, k = see.shape
    o, lse = np.zeros((n, g * m * d)), np.full((n, g * m), -np.inf)
    tol_o, tol_l = np.zeros_like(o), np.zeros_like(lse)
    for h in range(g * m):
        K, V = kv[:, (h // m) * d:(h // m + 1) * d], kv[:, (g + h // m) * d:(g + h // m + 1) * d]
        for i in range(n):
            at = np.flatnonzero(see[i])
            if not len(at):
                continue
            qi = q[i, h * d:(h + 1) * d]
            s = K[at] @ qi / math.sqrt(d)
            e_s = d * 2.0 ** -24 * (np.abs(K[at]) @ np.abs(qi)).max() / math.sqrt(d)
            top = s.max()
            w = np.exp(s - top)
            lse[i, h] = top + np.log(w.sum())
            p = w / w.sum()
            sl = slice(h * d, (h + 1) * d)
            o[i, sl] = p @ V[at]
            tol_o[i, sl] = 2.0 ** -8 * np.abs(o[i, sl]) + (2 * e_s + 2.0 ** -15) * (p @ np.abs(V[at]))
            tol_l[i, h] = e_s + 2.0 ** -20 + 2.0 ** -22 * abs(lse[i, h])
    return o, lse, tol_o, tol_l


def _tree_case(seed, g, m, d, ctx, nodes, form, max_len=None, past=float("nan")):
    r = np.random.default_rng(seed)
    slots = max_len or max(c + n for c, n in zip(ctx, nodes)) + 3
    words = max(1, (max(nodes) + 31) // 32)
    q = _rand((sum(nodes), g * m * d), seed, 2.0)
    kv = _rand((len(ctx), slots, 2 * g * d), seed + 1)
    for b, (c, n) in enumerate(zip(ctx, nodes)):
        kv[b, c + n:] = past  # rows past the sequence are not its own
    see = [_see(r, n, form) for n in nodes]
    mask = np.concatenate([_words(s, words) for s in see if len(s)])
    return q, kv, see, mask, slots


def _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d, lse=True, stream=None):
    n = sum(nodes)
    o = torch.full((n, g * m * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    ls = torch.full((n, g * m), float("nan"), device="cuda") if lse else None
    ws = torch.zeros(N.spd_tree_attention_workspace_size(n, len(ctx), g * m, g, d), dtype=torch.uint8, device="cuda")
    N.spd_tree_attention(q.cuda(), _cu(nodes), ctx, None if mask is None else torch.from_numpy(mask).cuda(), kv.cuda(), slots,
                         g * m, g, d, o, ls, ws, stream=stream)
    torch.cuda.synchronize()
    assert N.spd_workspace_status(ws) == 0
    return o, ls


def _check_tree(q, kv, see, o, ls, ctx, nodes, g, m, d):
    cu, q, got, gl = _cu(nodes), bf16_np(q), bf16_np(o), ls.cpu().numpy().astype(np.float64)
    for b, (c, n) in enumerate(zip(ctx, nodes)):
        if not n:
            continue
        full = np.concatenate([np.ones((n, c), bool), see[b]], 1)
        want, wl, to, tl = _plain_rows(q[cu[b]:cu[b + 1]], bf16_np(kv[b, :c + n]), full, g, m, d)
        rows = slice(cu[b], cu[b + 1])
        np.testing.assert_array_equal(np.isneginf(gl[rows]), np.isneginf(wl))
        fin = np.isfinite(wl)
        assert (np.abs(gl[rows][fin] - wl[fin]) <= tl[fin]).all()
        bad = np.abs(got[rows] - want) > to
        assert not bad.any() and np.isfinite(got[rows]).all(), (b, bad.sum(), np.abs(got[rows] - want).max())


@pytest.mark.parametrize("g,m,d,ctx,nodes,form", [
    (4, 1, 128, [100], [1], "tree"),                       # a decode step
    (2, 7, 128, [1], [1], "tree"),
    (4, 7, 128, [0, 63, 64, 65, 300], [5, 1, 33, 20, 64], "tree"),   # no context; block borders; several tiles a sequence
    (2, 1, 128, [500, 0, 129], [130, 40, 0], "tree"),      # more nodes than a tile has rows; a sequence without drafts
    (2, 2, 64, [127, 128, 700], [64, 3, 17], "chain"),
    (1, 16, 64, [1000], [9], "tree"),
    (1, 3, 128, [61, 190], [43, 44], "any"),               # any masks, rows that see no draft
    (2, 4, 64, [0, 0], [40, 1], "any"),                    # rows that see nothing at all
    (1, 71, 64, [70], [5], "chain"),                       # one node a tile of 128 rows
    (1, 128, 128, [3], [3], "chain"),
    (1, 200, 64, [130], [2], "tree"),                      # a group wider than a tile
    (3, 5, 128, [2500], [12], "tree"),                     # split over the keys
    (1, 1, 64, [4097], [2], "chain"),
])
def test_tree_attention(g, m, d, ctx, nodes, form):
    q, kv, see, mask, slots = _tree_case(len(ctx) + 10 * m + d, g, m, d, ctx, nodes, form)
    o, ls = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    _check_tree(q, kv, see, o, ls, ctx, nodes, g, m, d)


def test_tree_attention_of_chains_needs_no_mask_and_lse_is_optional():
    g, m, d, ctx, nodes = 2, 3, 128, [77, 200], [21, 64]
    q, kv, see, mask, slots = _tree_case(5, g, m, d, ctx, nodes, "chain")
    o, ls = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    _check_tree(q, kv, see, o, ls, ctx, nodes, g, m, d)
    plain, none = _run_tree(q, kv, None, slots, ctx, nodes, g, m, d, lse=False)
    assert none is None and torch.equal(plain, o)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf"), torch.finfo(torch.bfloat16).min])
def test_tree_attention_ignores_what_a_row_does_not_see(what):
    # draft 4 is nobody's ancestor; its own row alone may show its values
    g, m, d, ctx, nodes = 2, 2, 128, [90], [9]
    q, kv, see, mask, slots = _tree_case(6, g, m, d, ctx, nodes, "chain")
    see = [see[0].copy()]
    see[0][5:, 4] = False
    mask = _words(see[0], 1)
    clean = kv.clone()
    kv[0, 94] = what
    o, ls = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    rows = [i for i in range(9) if i != 4]
    want, _ = _run_tree(q, clean, mask, slots, ctx, nodes, g, m, d)
    assert torch.isfinite(o[rows].float()).all() and torch.isfinite(ls[rows]).all()
    np.testing.assert_allclose(bf16_np(o[rows]), bf16_np(want[rows]), rtol=2.0 ** -7, atol=2.0 ** -14)


def test_tree_attention_shows_a_seen_draft_that_is_not_finite():
    g, m, d, ctx, nodes = 1, 2, 64, [66], [6]
    q, kv, see, mask, slots = _tree_case(8, g, m, d, ctx, nodes, "chain")
    kv[0, 66 + 3, g * d + 5] = float("inf")  # one value of V of draft 3, which drafts 3 to 5 see
    o, _ = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    o = bf16_np(o).reshape(6, 2, d)
    assert np.isfinite(o[:3]).all() and np.isposinf(o[3:, :, 5]).all()
    assert np.isfinite(np.delete(o, 5, axis=2)).all()


def test_tree_attention_scores_far_apart():
    # one key far above the others wins outright, whatever block it lies in; weights underflow to zero elsewhere
    g, m, d, ctx, nodes = 1, 2, 128, [333], [4]
    for at in (0, 64, 200, 332, 335):
        q, kv, see, mask, slots = _tree_case(9, g, m, d, ctx, nodes, "chain")
        kv[0, at, :d] = q[3, :d] * 16
        o, ls = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
        _check_tree(q, kv, see, o, ls, ctx, nodes, g, m, d)


def test_tree_attention_past_32_bit_offsets():
    # the second sequence's rows begin 2.46e9 elements into the cache
    g, m, d, slots, ctx, nodes = 8, 1, 128, 1_200_000, [70, 150], [3, 20]
    free, _ = torch.cuda.mem_get_info()
    if free < 16 << 30:
        pytest.skip("needs 16 GB of device memory")
    q, small, see, mask, _ = _tree_case(11, g, m, d, ctx, nodes, "tree")
    kv = torch.empty(2, slots, 2 * g * d, dtype=torch.bfloat16, device="cuda")
    for b in range(2):
        kv[b, :small.shape[1]] = small[b].cuda()
    o, ls = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    _check_tree(q, small, see, o, ls, ctx, nodes, g, m, d)


@pytest.mark.parametrize("g,m,d,most,n", [(4, 7, 128, 2500, 16), (2, 4, 64, 6000, 24), (2, 1, 128, 9000, 5)])
def test_tree_attention_of_very_different_lengths(g, m, d, most, n):
    # sequences split over clusters of different sizes, in launches that share the GPU; repeated calls overlap
    r = np.random.default_rng(n)
    ctx = [int(x) for x in np.exp(r.uniform(np.log(20), np.log(most), n))] + [most]
    nodes = [int(x) for x in r.integers(1, 6, n + 1)]
    q, kv, see, mask, slots = _tree_case(21, g, m, d, ctx, nodes, "tree")
    total = sum(nodes)
    qd, kd, md = q.cuda(), kv.cuda(), torch.from_numpy(mask).cuda()
    ws = torch.zeros(N.spd_tree_attention_workspace_size(total, n + 1, g * m, g, d), dtype=torch.uint8, device="cuda")
    outs = []
    for k in range(6):  # other queries every other time, through the same buffer
        src = qd if k % 2 == 0 else qd.flip(0).contiguous()
        buf = src.clone() if k == 0 else buf.copy_(src)
        o = torch.full((total, g * m * d), float("nan"), dtype=torch.bfloat16, device="cuda")
        ls = torch.full((total, g * m), float("nan"), device="cuda")
        N.spd_tree_attention(buf, _cu(nodes), ctx, md, kd, slots, g * m, g, d, o, ls, ws)
        outs.append((o, ls))
    torch.cuda.synchronize()
    assert N.spd_workspace_status(ws) == 0
    _check_tree(q, kv, see, *outs[0], ctx, nodes, g, m, d)
    _check_tree(q.flip(0), kv, see, *outs[1], ctx, nodes, g, m, d)
    for k in range(2, 6):
        assert torch.equal(outs[k][0], outs[k % 2][0]) and torch.equal(outs[k][1], outs[k % 2][1])


def test_many_sequences_take_several_launches():
    g, m, d = 1, 2, 64
    r = np.random.default_rng(3)
    ctx, nodes = [int(x) for x in r.integers(0, 40, 500)], [int(x) for x in r.integers(0, 4, 500)]
    q, kv, see, mask, slots = _tree_case(12, g, m, d, ctx, nodes, "tree")
    o, ls = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    _check_tree(q, kv, see, o, ls, ctx, nodes, g, m, d)


def test_tree_attention_on_a_stream_of_its_own_and_outputs_between_guards():
    g, m, d, ctx, nodes = 2, 7, 128, [257, 640], [19, 6]
    q, kv, see, mask, slots = _tree_case(13, g, m, d, ctx, nodes, "tree")
    n, w = 25, g * m * d
    o = torch.full((n + 2, w), 7.0, dtype=torch.bfloat16, device="cuda")
    ls = torch.full((n + 2, g * m), 7.0, device="cuda")
    qd, kd, md = q.cuda(), kv.cuda(), torch.from_numpy(mask).cuda()
    ws = torch.zeros(N.spd_tree_attention_workspace_size(n, 2, g * m, g, d), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for _ in range(3):
        N.spd_tree_attention(qd, _cu(nodes), ctx, md, kd, slots, g * m, g, d, o[1:n + 1], ls[1:n + 1], ws, stream=st.cuda_stream)
    st.synchronize()
    assert N.spd_workspace_status(ws) == 0
    _check_tree(q, kv, see, o[1:n + 1], ls[1:n + 1], ctx, nodes, g, m, d)
    assert (o[[0, n + 1]] == 7).all() and (ls[[0, n + 1]] == 7).all()


def test_tree_attention_repeats_bit_for_bit():
    g, m, d, ctx, nodes = 4, 7, 128, [3001, 40], [30, 3]
    q, kv, _, mask, slots = _tree_case(14, g, m, d, ctx, nodes, "tree")
    a = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
    for _ in range(3):
        b = _run_tree(q, kv, mask, slots, ctx, nodes, g, m, d)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- received weights ------------------------------------------------------------------------------
@pytest.mark.parametrize("L,g,m,d,lens,rows", [
    (1, 1, 1, 64, [1], [1]),
    (2, 4, 7, 128, [130, 64, 257, 1], [1, 1, 1, 1]),         # a decode step
    (2, 2, 1, 128, [300, 40], [32, 40]),                     # a window; every cached token a row
    (1, 2, 5, 64, [127, 129, 0], [7, 0, 0]),                 # no rows, no tokens
    (3, 1, 16, 64, [513], [21]),
    (1, 1, 40, 128, [200, 31], [13, 9]),                     # more rows a K/V head than a pass takes
])
@pytest.mark.parametrize("alias", [False, True])
def test_cache_weights(L, g, m, d, lens, rows, alias):
    seed, B, n = 7 * L + m, len(lens), sum(rows)
    r = np.random.default_rng(seed)
    slots = max(lens) + 2
    q, kv = _rand((L, n + 2, g * m * d), seed, 2.0), _rand((L, B, slots, 2 * g * d), seed + 1)
    for b in range(B):
        kv[:, b, lens[b]:] = float("nan")
    pick = r.permutation(n + 2)[:n].astype(np.int32)
    lse = (4.0 + 2.0 * r.random((L, n + 2, g * m))).astype(np.float32)
    if n:
        lse[0, pick[0], 0] = -np.inf  # a row that saw nothing adds nothing
    acc = r.random((L, B, g, slots)).astype(np.float32)
    acc_in = torch.from_numpy(acc).cuda()
    out = acc_in if alias else torch.full_like(acc_in, -5.0)
    rows_dev = torch.from_numpy(pick).cuda()
    N.spd_cache_weights(q.cuda(), torch.from_numpy(lse).cuda(), rows_dev, _cu(rows), kv.cuda(), lens, slots, g * m, g, d, 0.75,
                        acc_in, out)
    got = out.cpu().numpy().astype(np.float64)
    q, kv, cu = bf16_np(q), bf16_np(kv), _cu(rows)
    for l in range(L):
        for b in range(B):
            k = lens[b]
            for h in range(g):
                want, tol = 0.75 * acc[l, b, h, :k].astype(np.float64), np.zeros(k)
                for i in range(rows[b]):
                    for j in range(h * m, (h + 1) * m):
                        at = pick[cu[b] + i]
                        z = float(lse[l, at, j])
                        if z == -np.inf:
                            continue
                        K, qi = kv[l, b, :k - rows[b] + i + 1, h * d:(h + 1) * d], q[l, at, j * d:(j + 1) * d]
                        w = np.exp(K @ qi / math.sqrt(d) - z)
                        e_s = d * 2.0 ** -24 * (np.abs(K) @ np.abs(qi)) / math.sqrt(d)
                        want[:len(w)] += w
                        tol[:len(w)] += w * (e_s + 2.0 ** -18)
                assert (np.abs(got[l, b, h, :k] - want) <= tol + 2.0 ** -20 * np.abs(want)).all()
            np.testing.assert_array_equal(got[l, b, :, k:], acc[l, b, :, k:] if alias else -5.0)


@pytest.mark.parametrize("d,m,n", [(64, 3, 2), (128, 4, 20), (64, 8, 16)])
def test_cache_weights_of_keys_and_normalisers_that_are_not_finite(d, m, n):
    # K/V head 0: q > 0. Row 0's normaliser is -inf, row 1's +inf, the others' finite: infinite and NaN keys show in the others
    # alone, and where there are none (head 1) nothing shows at all
    k, slots = 200, 256
    q = torch.rand(1, n, 2 * m * d) + 0.5
    lse = torch.zeros(1, n, 2, m)
    lse[:, 0], lse[:, 1] = -np.inf, np.inf
    lse[:, 2:, 1] = -np.inf
    kv = torch.zeros(1, 1, slots, 2, 2, d)
    for slot, x in ((3, -np.inf), (70, np.inf), (130, np.nan)):
        kv[:, :, slot, 0] = x
    kv[:, :, k:] = np.nan  # past the cached rows
    acc = torch.full((1, 1, 2, slots), 2.0, device="cuda")
    N.spd_cache_weights(q.to(torch.bfloat16).cuda(), lse.view(1, n, 2 * m).cuda(), None, [0, n],
                        kv.to(torch.bfloat16).view(1, 1, slots, 4 * d).cuda(), [k], slots, 2 * m, 2, d, 0.5, acc, acc)
    got = acc.cpu().numpy()[0, 0]
    finite = m * (n - 2)
    want = np.full(k, 1.0 + finite)
    want[k - n + 1:] = [1.0 + m * max(0, n - max(2, i)) for i in range(1, n)]
    if finite:
        want[[3, 70, 130]] = 1.0, np.inf, np.nan
    np.testing.assert_array_equal(got[0, :k], want)
    np.testing.assert_array_equal(got[1, :k], 1.0)
    assert (got[:, k:] == 2.0).all()


def test_cache_weights_without_a_row_list_and_indices_outside_the_queries():
    g, m, d, lens, rows = 2, 2, 64, [90, 20], [3, 2]
    q, kv = _rand((1, 5, g * m * d), 1, 2.0), _rand((1, 2, 95, 2 * g * d), 2)
    lse, acc = torch.full((1, 5, g * m), 5.0, device="cuda"), torch.zeros(1, 2, g, 95, device="cuda")
    a, b, c = (torch.zeros_like(acc) for _ in range(3))
    args = (_cu(rows), kv.cuda(), lens, 95, g * m, g, d, 1.0, acc)
    N.spd_cache_weights(q.cuda(), lse, None, *args, a)
    N.spd_cache_weights(q.cuda(), lse, torch.arange(5, dtype=torch.int32, device="cuda"), *args, b)
    assert torch.equal(a, b)
    N.spd_cache_weights(q.cuda(), lse, torch.tensor([0, -1, 2, 5, 1 << 30], dtype=torch.int32, device="cuda"), *args, c)
    assert float(c[0, 1].abs().max()) == 0.0 and 0 < float(c[0, 0].sum()) < float(a[0, 0].sum())


# ---- eviction --------------------------------------------------------------------------------------
def _plain_evict(kv, acc, pos, lens, budget, sink, recent, nxt, g, d):
    """Expected (kv, acc, pos, src) of an eviction, on numpy copies (kv as int16 [L][B][slots][2][g][d])."""
    kv, acc_o, pos_o = kv.copy(), acc.copy(), pos.copy()
    src_o = np.full(acc.shape[:3] + (budget,), -3, np.int32)
    for l, b, u in np.ndindex(acc.shape[:3]):
        n = lens[b]
        w, p = acc[l, b, u, :n].astype(np.float64), pos[l, b, u, :n]
        w = np.where(np.isnan(w), -np.inf, w)
        held = (p < sink) | (p >= nxt[b] - recent)
        kept = np.sort(np.lexsort((np.arange(n), np.where(held, 0.0, -w), ~held))[:min(n, budget)])
        take = len(kept)
        src = np.arange(take)
        src[np.setdiff1d(src, kept)] = kept[kept >= take]
        kv[l, b, :take, :, u] = kv[l, b, src, :, u]
        acc_o[l, b, u, :take], pos_o[l, b, u, :take], src_o[l, b, u, :take] = acc[l, b, u, src], pos[l, b, u, src], src
        acc_o[l, b, u, take:n], pos_o[l, b, u, take:n] = 0.0, -1
    return kv, acc_o, pos_o, src_o


@pytest.mark.parametrize("L,g,d,lens,budget,sink,recent,weights", [
    (1, 1, 64, [1], 1, 0, 0, "rand"),
    (1, 2, 128, [2, 5], 1, 0, 0, "rand"),
    (2, 4, 128, [33, 40, 32, 0], 32, 4, 8, "rand"),         # a few over, one at the budget, one empty
    (2, 3, 64, [1000, 77, 1029], 200, 4, 50, "rand"),
    (1, 2, 128, [700], 300, 0, 0, "ties"),                  # many equal weights: the lower slots stay
    (1, 2, 128, [700], 300, 5, 20, "equal"),                # all weights equal
    (1, 2, 64, [500], 120, 3, 9, "odd"),                    # NaN, infinities, both zeros, negative weights
    (1, 1, 64, [300], 50, 40, 200, "rand"),                 # more protected rows than the budget
    (1, 1, 64, [20011], 5000, 4, 64, "rand"),               # a cluster of two
    (1, 1, 64, [70001], 30000, 4, 64, "ties"),              # a cluster of eight
    (1, 1, 64, [70001], 69990, 4, 64, "rand"),
])
@pytest.mark.parametrize("alias", [False, True])
def test_cache_evict(L, g, d, lens, budget, sink, recent, weights, alias):
    B, slots = len(lens), max(lens) + 4
    r = np.random.default_rng(sum(lens) + budget)
    shape = (L, B, g, slots)
    acc = {"rand": lambda: np.exp(2 * r.standard_normal(shape)), "ties": lambda: r.integers(0, 4, shape) / 4.0,
           "equal": lambda: np.full(shape, 0.5),
           "odd": lambda: r.choice([np.nan, np.inf, -np.inf, 0.0, -0.0, -1.5, 1e-42, 3.0], shape)}[weights]().astype(np.float32)
    pos = np.stack([r.permutation(slots) for _ in range(L * B * g)]).reshape(shape).astype(np.int32)
    nxt = np.full(B, slots, np.int32)
    kv = torch.randint(-30000, 30000, (L, B, slots, 2 * g * d), dtype=torch.int16)
    want = _plain_evict(kv.numpy().reshape(L, B, slots, 2, g, d), acc, pos, lens, budget, sink, recent, nxt, g, d)
    kvd, a, p = kv.cuda().view(torch.bfloat16), torch.from_numpy(acc).cuda(), torch.from_numpy(pos).cuda()
    ao, po = (a, p) if alias else (torch.from_numpy(acc).cuda().clone(), torch.from_numpy(pos).cuda().clone())
    src = torch.full((L, B, g, budget), -3, dtype=torch.int32, device="cuda")
    ws = torch.zeros(N.spd_cache_evict_workspace_size(L, B, g, budget), dtype=torch.uint8, device="cuda")
    new = N.spd_cache_evict(kvd, lens, slots, g, d, budget, sink, recent, nxt, a, p, ao, po, src, ws)
    np.testing.assert_array_equal(new, np.minimum(lens, budget))
    got_kv = kvd.view(torch.int16).cpu().numpy().reshape(L, B, slots, 2, g, d)
    np.testing.assert_array_equal(src.cpu().numpy(), want[3])
    np.testing.assert_array_equal(got_kv, want[0])
    np.testing.assert_array_equal(ao.cpu().numpy().view(np.int32), want[1].view(np.int32))
    np.testing.assert_array_equal(po.cpu().numpy(), want[2])


def test_cache_evict_by_slots_without_positions():
    L, g, d, lens, budget = 1, 2, 64, [120, 30], 50
    r = np.random.default_rng(4)
    acc = r.random((L, 2, g, 128)).astype(np.float32)
    pos = np.broadcast_to(np.arange(128, dtype=np.int32), acc.shape).copy()
    kv = torch.randint(-30000, 30000, (L, 2, 128, 2 * g * d), dtype=torch.int16)
    want = _plain_evict(kv.numpy().reshape(L, 2, 128, 2, g, d), acc, pos, lens, budget, 4, 10, np.array(lens), g, d)
    kvd, a = kv.cuda().view(torch.bfloat16), torch.from_numpy(acc).cuda()
    ws = torch.zeros(N.spd_cache_evict_workspace_size(L, 2, g, budget), dtype=torch.uint8, device="cuda")
    N.spd_cache_evict(kvd, lens, 128, g, d, budget, 4, 10, None, a, None, a, None, None, ws)
    np.testing.assert_array_equal(a.cpu().numpy(), want[1])
    np.testing.assert_array_equal(kvd.view(torch.int16).cpu().numpy().reshape(want[0].shape), want[0])


def test_many_sequences_of_weights_and_evictions_take_several_launches():
    B, g, d, slots = 300, 1, 64, 40
    r = np.random.default_rng(9)
    lens = r.integers(0, slots + 1, B).astype(np.int32)
    rows = np.minimum(r.integers(0, 3, B), lens)
    n = int(rows.sum())
    q, kv = _rand((2, n, 2 * d), 31, 2.0), _rand((2, B, slots, 2 * g * d), 32)
    lse = torch.full((2, n, 2), 3.0)
    acc = torch.rand(2, B, g, slots, generator=torch.Generator().manual_seed(33))
    out = torch.zeros(2, B, g, slots, device="cuda")
    N.spd_cache_weights(q.cuda(), lse.cuda(), None, _cu(rows), kv.cuda(), lens, slots, 2, g, d, 0.5, acc.cuda(), out)
    got, cu, qn, kn = out.cpu().numpy(), _cu(rows), bf16_np(q), bf16_np(kv)
    for l in range(2):
        for b in range(B):
            k = lens[b]
            want = 0.5 * acc[l, b, 0, :k].numpy().astype(np.float64)
            for i in range(rows[b]):
                K = kn[l, b, :k - rows[b] + i + 1, :d]
                for j in range(2):
                    want[:len(K)] += np.exp(K @ qn[l, cu[b] + i, j * d:(j + 1) * d] / 8.0 - 3.0)
            np.testing.assert_allclose(got[l, b, 0, :k], want, rtol=1e-4)
            assert (got[l, b, 0, k:] == 0).all()
    pos = np.broadcast_to(np.arange(slots, dtype=np.int32), acc.shape).copy()
    ints = torch.randint(-30000, 30000, (2, B, slots, 2 * g * d), dtype=torch.int16)
    want = _plain_evict(ints.numpy().reshape(2, B, slots, 2, g, d), acc.numpy(), pos, lens, 17, 2, 5, lens, g, d)
    kvd, a = ints.cuda().view(torch.bfloat16), acc.cuda()
    ws = torch.zeros(N.spd_cache_evict_workspace_size(2, B, g, 17), dtype=torch.uint8, device="cuda")
    N.spd_cache_evict(kvd, lens, slots, g, d, 17, 2, 5, None, a, None, a, None, None, ws)
    np.testing.assert_array_equal(a.cpu().numpy(), want[1])
    np.testing.assert_array_equal(kvd.view(torch.int16).cpu().numpy().reshape(want[0].shape), want[0])


# ---- commit ----------------------------------------------------------------------------------------
def test_tree_commit():
    L, g, d, ctx, slots = 2, 3, 64, [10, 0, 33], 80
    paths = [[0, 2, 3, 7, 8, 9, 11, 12, 13, 20, 21, 40], [], [0]]
    kv = torch.randint(-30000, 30000, (L, 3, slots, 2 * g * d), dtype=torch.int16)
    want = kv.clone()
    for b, pa in enumerate(paths):
        for i, node in enumerate(pa):
            want[:, b, ctx[b] + i] = kv[:, b, ctx[b] + node]
    kvd = kv.cuda().view(torch.bfloat16)
    pos = torch.full((L, 3, g, slots), 9, dtype=torch.int32, device="cuda")
    acc = torch.full((L, 3, g, slots), 9.0, device="cuda")
    cu, flat = _cu([len(p) for p in paths]), [x for p in paths for x in p]
    ws = torch.zeros(N.spd_tree_commit_workspace_size(3, len(flat)), dtype=torch.uint8, device="cuda")
    N.spd_tree_commit(kvd, L, flat, cu, ctx, slots, g, d, ws, next_pos=[100, 0, 50], pos=pos, acc=acc)
    assert torch.equal(kvd.view(torch.int16).cpu(), want)
    p, a = pos.cpu().numpy(), acc.cpu().numpy()
    for b, pa in enumerate(paths):
        new = slice(ctx[b], ctx[b] + len(pa))
        assert (p[:, b, :, new] == [100, 0, 50][b] + np.arange(len(pa))).all() and (a[:, b, :, new] == 0).all()
        assert (np.delete(p[:, b], np.r_[new], axis=-1) == 9).all() and (np.delete(a[:, b], np.r_[new], axis=-1) == 9).all()


# ---- logit rules -----------------------------------------------------------------------------------
def _plain_logits(z, seq_of, hist, gen, path, rep, freq, pres, bias, allow, rule):
    """float64 rows and the magnitudes that enter them."""
    n, v = z.shape
    z = z.astype(np.float64)
    out, size = z.copy(), np.abs(np.where(np.isfinite(z), z, 0.0))
    for i in range(n):
        b = seq_of[i]
        made, seen = np.zeros(v), np.zeros(v, bool)
        if 0 <= b < len(hist):
            h = np.asarray(hist[b])
            ok = (h >= 0) & (h < v)
            new = np.arange(len(h)) >= gen[b]
            np.add.at(made, h[ok & new], 1)
            seen[h[ok]] = True
        for t in path[i]:
            made[t] += 1
        seen |= made > 0
        r, f, p = (float(x[b]) if 0 <= b < len(hist) else d for x, d in ((rep, 1.0), (freq, 0.0), (pres, 0.0)))
        out[i] = np.where(seen, np.where(z[i] > 0, z[i] / r, z[i] * r), z[i])
        size[i] *= max(r, 1 / r)
        out[i] -= np.where(made > 0, f * made + p, 0.0)
        size[i] += np.where(made > 0, abs(f) * made + abs(p), 0.0)
        if 0 <= b < len(hist):
            for t, x in bias[b]:
                out[i, t] += x
                size[i, t] += abs(x)
        if 0 <= rule[i] < len(allow):
            out[i][~allow[rule[i]]] = -np.inf
    return out, size


def _logit_case(seed, v, seqs, rows_of, hist_len, n_bias):
    r = np.random.default_rng(seed)
    n = len(rows_of)
    hist = [np.where(r.random(k) < 0.2, -200, (v * r.random(k) ** 3).astype(np.int64)) for k in hist_len]
    gen = [int(r.integers(0, len(h) + 1)) for h in hist]
    path = [list(r.integers(0, v, r.integers(0, 4))) for _ in range(n)]
    bias = []
    for b in range(seqs):
        ids = np.sort(r.choice(v, min(v, n_bias), replace=False))
        if len(ids) > 1:
            ids[1] = ids[0]  # a token listed twice
        bias.append([(int(t), np.float32(x)) for t, x in zip(ids, 3 * r.standard_normal(len(ids)))])
    allow = r.random((3, v)) < np.array([0.01, 0.5, 0.0])[:, None]
    rule = r.integers(-1, 4, n)
    rep, freq, pres = (x.astype(np.float32) for x in (r.uniform(0.7, 1.5, seqs), r.uniform(-0.2, 0.5, seqs), r.uniform(0, 1, seqs)))
    z = (3 * r.standard_normal((n, v))).astype(np.float32)
    z[:, ::7] = 0.25  # equal values: the first of the largest wins
    z[0, v // 2] = -np.inf
    return z, hist, gen, path, bias, allow, rule, rep, freq, pres


def _flat(lists, dt):
    return torch.from_numpy(np.concatenate([np.asarray(x, dt) for x in lists] or [np.zeros(0, dt)]).astype(dt)).cuda()


@pytest.mark.parametrize("v,rows_of,hist_len,n_bias", [
    (1, [0], [3], 1),
    (31, [0, 1], [0, 5], 2),
    (100, [0, 0, 1, 5], [40, 1], 7),             # a row without a sequence
    (1000, [1, 0, 1], [300, 10], 33),            # rows in another order than their sequences
    (8193, [0, 1, 2, 2], [1, 900, 0], 64),       # an odd vocabulary: rows of other alignments
    (32000, [0, 1], [5000, 20], 300),
    (152064, [0, 1, 1], [3000, 700], 500),
    (512000, [0], [2000], 50),                   # sixteen CTAs a row
])
@pytest.mark.parametrize("in_place", [False, True])
def test_logit_rules(v, rows_of, hist_len, n_bias, in_place):
    seqs, n = len(hist_len), len(rows_of)
    z, hist, gen, path, bias, allow, rule, rep, freq, pres = _logit_case(v + n, v, seqs, rows_of, hist_len, n_bias)
    want, size = _plain_logits(z, rows_of, hist, gen, path, rep, freq, pres, bias, allow, rule)
    words = (v + 31) // 32
    h_cu, b_cu, p_cu = _cu([len(h) for h in hist]), _cu([len(b) for b in bias]), _cu([len(p) for p in path])
    wide = torch.full((n + 2, v + 4), 5.0, device="cuda")  # guards around and between the rows
    out = wide[1:n + 1, :v]
    src = out if in_place else torch.from_numpy(z).cuda()
    if in_place:
        out.copy_(torch.from_numpy(z))
    best = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    N.spd_logits_process(
        src, out, best, seq_of=_flat([rows_of], np.int32), hist=_flat(hist, np.int32), hist_cu=torch.from_numpy(h_cu).cuda(),
        gen_start=torch.from_numpy((h_cu[:-1] + gen).astype(np.int32)).cuda(), path=_flat(path, np.int32),
        path_cu=torch.from_numpy(p_cu).cuda(), repetition=_flat([rep], np.float32), frequency=_flat([freq], np.float32),
        presence=_flat([pres], np.float32), bias_cu=torch.from_numpy(b_cu).cuda(),
        bias_id=_flat([[t for t, _ in b] for b in bias], np.int32), bias=_flat([[x for _, x in b] for b in bias], np.float32),
        allow=torch.from_numpy(_words(allow, words)).cuda(), rule=_flat([rule], np.int32))
    got = out.cpu().numpy().astype(np.float64)
    inf = np.isinf(want)
    np.testing.assert_array_equal(np.where(inf, want, 0.0), np.where(np.isinf(got), got, 0.0))
    assert (np.abs(got[~inf] - want[~inf]) <= 6 * 2.0 ** -24 * size[~inf]).all()
    top = got.max(1)
    np.testing.assert_array_equal(best.cpu().numpy(), np.where(np.isneginf(top), -1, got.argmax(1)))
    assert (wide[[0, n + 1]] == 5).all() and (wide[:, v:] == 5).all()


@pytest.mark.parametrize("v,n", [(20000, 120), (152064, 30), (32003, 100)])
def test_logit_rules_of_more_rows_than_fit_at_once(v, n):
    # CTAs on their own, that offer their best to the row: equal bests in many slices, the first one wins every time
    rows_of, hist_len = [i % 3 for i in range(n)], [900, 40, 3000]
    z, hist, gen, path, bias, allow, rule, rep, freq, pres = _logit_case(v + n, v, 3, rows_of, hist_len, 40)
    z[:, 4001::977] = 90.0
    z[7] = -np.inf
    rule[7] = -1
    want, size = _plain_logits(z, rows_of, hist, gen, path, rep, freq, pres, bias, allow, rule)
    h_cu, b_cu, p_cu = _cu([len(h) for h in hist]), _cu([len(b) for b in bias]), _cu([len(p) for p in path])
    zd, out = torch.from_numpy(z).cuda(), torch.zeros(n, v, device="cuda")
    kw = dict(seq_of=_flat([rows_of], np.int32), hist=_flat(hist, np.int32), hist_cu=torch.from_numpy(h_cu).cuda(),
              gen_start=torch.from_numpy((h_cu[:-1] + gen).astype(np.int32)).cuda(), path=_flat(path, np.int32),
              path_cu=torch.from_numpy(p_cu).cuda(), repetition=_flat([rep], np.float32), frequency=_flat([freq], np.float32),
              presence=_flat([pres], np.float32), bias_cu=torch.from_numpy(b_cu).cuda(),
              bias_id=_flat([[t for t, _ in b] for b in bias], np.int32), bias=_flat([[x for _, x in b] for b in bias], np.float32),
              allow=torch.from_numpy(_words(allow, (v + 31) // 32)).cuda(), rule=_flat([rule], np.int32))
    bests = []
    for _ in range(4):
        best = torch.full((n,), 5, dtype=torch.int32, device="cuda")
        N.spd_logits_process(zd, out, best, **kw)
        bests.append(best.cpu().numpy())
    got = out.cpu().numpy().astype(np.float64)
    inf = np.isinf(want)
    np.testing.assert_array_equal(np.where(inf, want, 0.0), np.where(np.isinf(got), got, 0.0))
    assert (np.abs(got[~inf] - want[~inf]) <= 6 * 2.0 ** -24 * size[~inf]).all()
    top = got.max(1)
    assert (top > 40).sum() > n // 3 and bests[0][7] == -1
    for b in bests:
        np.testing.assert_array_equal(b, np.where(np.isneginf(top), -1, got.argmax(1)))
    N.spd_logits_process(zd, out, None, **kw)  # without the best token
    np.testing.assert_array_equal(out.cpu().numpy().astype(np.float64), got)


def test_logit_rules_all_off_is_a_copy_and_nan_never_wins():
    z = torch.randn(3, 5000, device="cuda")
    z[1, 77] = float("nan")
    z[2] = float("nan")
    out, best = torch.zeros_like(z), torch.zeros(3, dtype=torch.int32, device="cuda")
    N.spd_logits_process(z, out, best)
    assert torch.equal(out.view(torch.int32), z.view(torch.int32))
    want = torch.where(torch.isnan(z), -torch.inf, z).argmax(1).tolist()
    assert best.tolist() == [want[0], want[1], -1]


# ---- refusals --------------------------------------------------------------------------------------
def _refused(code, f, *a, **k):
    with pytest.raises(N.SpiderError) as e:
        f(*a, **k)
    assert e.value.code == code


def test_calls_refuse_what_they_cannot_do_before_any_launch():
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    f = lambda *s: torch.full(s, 3.0, device="cuda")  # noqa: E731
    q, kv, o, ls = bf(4, 256), bf(2, 32, 512), torch.full((4, 256), 3.0, dtype=torch.bfloat16, device="cuda"), f(4, 4)
    ws = torch.zeros(N.spd_tree_attention_workspace_size(4, 2, 4, 4, 64), dtype=torch.uint8, device="cuda")
    mask = torch.zeros(4, 1, dtype=torch.int32, device="cuda")
    call = lambda cu, ctx, w=ws, h=4, g=4, d=64: N.spd_tree_attention(q, cu, ctx, mask, kv, 32, h, g, d, o, ls, w)  # noqa: E731
    _refused(N.SPD_EINVAL, call, [0, 3, 2, 4][:1] + [5, 4], [1, 1])            # q_cu decreases
    _refused(N.SPD_EINVAL, call, [0, 2, 4], [31, 0])                           # drafts past max_len
    _refused(N.SPD_EINVAL, call, [0, 2, 4], [-1, 0])
    _refused(N.SPD_ENOSPC, call, [0, 2, 4], [1, 0], ws[:8])
    _refused(N.SPD_EUNSUPPORTED, call, [0, 2, 4], [1, 0], d=32)
    assert N.spd_tree_attention_workspace_size(4, 2, 4, 3, 64) == 0 and N.spd_tree_attention_workspace_size(0, 2, 4, 4, 64) == 0
    acc, pos = f(1, 2, 4, 32), torch.zeros(1, 2, 4, 32, dtype=torch.int32, device="cuda")
    wt = lambda cu, lens: N.spd_cache_weights(q[None], ls[None], None, cu, kv[None], lens, 32, 4, 4, 64, 1.0, acc, acc)  # noqa: E731
    _refused(N.SPD_EINVAL, wt, [0, 2, 4], [33, 4])
    _refused(N.SPD_EINVAL, wt, [0, 2, 4], [1, 4])                              # more rows than cached tokens
    ew = torch.zeros(N.spd_cache_evict_workspace_size(1, 2, 4, 8), dtype=torch.uint8, device="cuda")
    ev = lambda lens, bud=8, nxt=(9, 9), w=ew: N.spd_cache_evict(kv[None], lens, 32, 4, 64, bud, 0, 0, nxt, acc, pos, acc, pos, None, w)  # noqa: E731
    _refused(N.SPD_EINVAL, ev, [33, 4])
    _refused(N.SPD_EINVAL, ev, [20, 4], nxt=None)
    _refused(N.SPD_EINVAL, ev, [20, 4], bud=0)
    _refused(N.SPD_ENOSPC, ev, [20, 4], w=ew[:300])
    cw = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    cm = lambda path, cu: N.spd_tree_commit(kv[None], 1, path, cu, [5, 5], 32, 4, 64, cw)  # noqa: E731
    _refused(N.SPD_EINVAL, cm, [1, 0, 2], [0, 2, 3])                           # a path out of order
    _refused(N.SPD_EINVAL, cm, [0, 1, 27], [0, 2, 3])                          # a node past max_len
    _refused(N.SPD_EINVAL, call, [0, 2, 4], [1, 0], ws[4:])                    # workspaces off their 16 bytes
    _refused(N.SPD_EINVAL, ev, [20, 4], w=ew[8:])
    _refused(N.SPD_EINVAL, lambda: N.spd_tree_commit(kv[None], 1, [0], [0, 1, 1], [5, 5], 32, 4, 64, cw[1:]))
    z = f(2, 64)
    _refused(N.SPD_EINVAL, N.spd_logits_process, z, z, hist=mask.view(-1), seq_of=mask.view(-1)[:2])  # no hist_cu
    _refused(N.SPD_EUNSUPPORTED, N.spd_logits_process, f(1, 819201), f(1, 819201))
    torch.cuda.synchronize()
    assert (o == 3).all() and (ls == 3).all() and (acc == 3).all() and (z == 3).all()
