"""Drafted-token attention where the values are hard: weights that have to keep their bits, NaN in queries and keys,
infinite values.
Plain values in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_34977_gb300 import _native as N
from tests.gpu_util import bf16_np
from tests.test_gpu_answer import _plain_rows, _tree_case

pytestmark = pytest.mark.gpu
LONG = {64: 9000, 128: 9000}  # contexts whose states go through memory (asserted where it matters)


def _cu(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def _call(q, kv, ctx, nodes, g, m, d, mask=None):
    """o and lse in float64, and whether the workspace holds states (of rows merged through memory)."""
    n = sum(nodes)
    o = torch.full((n, g * m * d), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((n, g * m), 7.0, device="cuda")
    ws = torch.zeros(N.spd_tree_attention_workspace_size(n, len(ctx), g * m, g, d), dtype=torch.uint8, device="cuda")
    N.spd_tree_attention(q.to(torch.bfloat16).cuda(), _cu(nodes), ctx, mask, kv.to(torch.bfloat16).cuda(), kv.shape[1], g * m, g,
                         d, o, lse, ws)
    torch.cuda.synchronize()
    assert N.spd_workspace_status(ws) == 0
    return bf16_np(o), lse.cpu().numpy().astype(np.float64), bool((ws[256:] != 0).any())


def _bf16(x):
    return torch.as_tensor(np.asarray(x, np.float32)).to(torch.bfloat16).double().numpy()


def _hard_scores(scale):
    """Four bf16 keys a > 0 whose weights e^(-a scale) lose most in two bf16 terms, all downwards (and by less than 0.85 of the
    second term's half unit, so that the exponential's own rounding does not turn the loss over)."""
    a = np.unique(_bf16(np.linspace(0.05, 2.5, 4000)))
    p = np.exp(-a * scale).astype(np.float32).astype(np.float64)
    first = p - _bf16(p)
    loss = first - _bf16(first)
    safe = np.abs(loss) < 0.85 * 2.0 ** (np.floor(np.log2(np.abs(first))) - 8)
    return a[np.argsort(-np.where(safe, loss / p, -1.0))[:4]]


@pytest.mark.parametrize("d,ctx,at,memory", [(128, 7, 0, False), (64, 7, 0, False), (128, 300, 130, False), (64, 700, 449, False),
                                             (128, LONG[128], 4100, True), (64, LONG[64], 6000, True)])
def test_weights_keep_their_24_bits(d, ctx, at, memory):
    # Scores are exact (one column of q and k); four keys have weights that two bf16 terms do not hold, three keys of weight 1
    # take their sum away again down to 2^-25 of it, all other weights are below 2^-60. What is left shows a weight's bits.
    # Tolerance, of sum p |v|: the exponential 2^-22 and its argument 2^-22, products and sums 3 x 2^-23 (three terms, one
    # slice of 16 keys at most two): below 2^-20; and the output's rounding to bf16. Two terms would lose 2^-18.4.
    scale = 8.0 / math.sqrt(d)
    a = _hard_scores(scale)
    p = np.exp(-a * scale)
    r = np.random.default_rng(d + ctx)
    v = _bf16(r.uniform(1.0, 2.0, (4, d)))
    rest, back = p @ v, []
    for _ in range(3):
        back.append(_bf16(-rest))
        rest = rest + back[-1]
    q = torch.zeros(1, d)
    q[0, 0] = 8.0
    kv = torch.from_numpy(r.standard_normal((1, ctx + 1, 2 * d)).astype(np.float32))
    kv[0, :, :d] = 0.0
    kv[0, :, 0] = -64.0
    kv[0, at:at + 7, 0] = torch.from_numpy(np.concatenate([-a, np.zeros(3)]))
    kv[0, at:at + 7, d:] = torch.from_numpy(np.concatenate([v, np.stack(back)]))
    o, _, through_memory = _call(q, kv, [ctx], [1], 1, 1, d)
    assert through_memory == memory
    total = p.sum() + 3.0
    want, size = rest / total, (p @ np.abs(v) + np.abs(np.stack(back)).sum(0)) / total
    tol = 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size
    two = _bf16(p) + _bf16(p - _bf16(p))
    assert (np.abs((two - p) @ v / total) > tol).all()  # what this test is about
    assert (np.abs(o[0] - want) <= tol).all(), np.abs(o[0] - want).max() / size.max()


# heads, contexts, nodes, and whether the states go through memory: one CTA, a cluster, several tiles a sequence
PLANS = [(2, 2, 64, [50], [3], False), (32, 1, 128, [321], [1], False), (2, 2, 64, [700, 20], [5, 2], False),
         (4, 7, 128, [4096], [1], True), (1, 2, 64, [9000], [5], True), (1, 7, 128, [9000], [40], True),
         (4, 7, 128, [3000, 6000, 40], [4, 9, 1], True)]


def _random(seed, g, m, d, ctx, nodes):
    r = torch.Generator().manual_seed(seed)
    slots = max(c + n for c, n in zip(ctx, nodes)) + 1
    q = torch.randn(sum(nodes), g * m * d, generator=r).to(torch.bfloat16)
    return q, torch.randn(len(ctx), slots, 2 * g * d, generator=r).to(torch.bfloat16)


@pytest.mark.parametrize("g,m,d,ctx,nodes,memory", PLANS)
def test_a_query_that_is_nan_shows_in_its_row_and_head(g, m, d, ctx, nodes, memory):
    q, kv = _random(1, g, m, d, ctx, nodes)
    want, want_lse, through_memory = _call(q, kv, ctx, nodes, g, m, d)
    assert through_memory == memory
    row, head = sum(nodes) - 1, g * m - 1
    q[row, head * d + 3] = float("nan")
    o, lse, _ = _call(q, kv, ctx, nodes, g, m, d)
    bad = np.zeros_like(want, bool)
    bad[row, head * d:] = True
    assert np.isnan(o[bad]).all() and np.isnan(lse[row, head])
    lse[row, head] = want_lse[row, head]
    np.testing.assert_array_equal(o[~bad], want[~bad])
    np.testing.assert_array_equal(lse, want_lse)


@pytest.mark.parametrize("g,m,d,ctx,nodes,memory", PLANS)
@pytest.mark.parametrize("first,last", [(0.0, 0.0), (0.0, 0.3), (0.5, 0.5), (0.6, 1.0), (0.0, 1.0)])
def test_committed_keys_that_are_nan_show_in_every_row_of_their_head(g, m, d, ctx, nodes, memory, first, last):
    # single keys, whole parts of a row's keys, all of them; the other K/V heads and sequences do not see them
    q, kv = _random(2, g, m, d, ctx, nodes)
    want, want_lse, _ = _call(q, kv, ctx, nodes, g, m, d)
    kv[0, int(first * (ctx[0] - 1)):int(last * (ctx[0] - 1)) + 1, :d] = float("nan")
    o, lse, through_memory = _call(q, kv, ctx, nodes, g, m, d)
    assert through_memory == memory
    bad = np.zeros_like(want, bool)
    bad[:nodes[0], :m * d] = True
    assert np.isnan(o[bad]).all() and np.isnan(lse[:nodes[0], :m]).all()
    lse[:nodes[0], :m] = want_lse[:nodes[0], :m]
    np.testing.assert_array_equal(o[~bad], want[~bad])
    np.testing.assert_array_equal(lse, want_lse)


@pytest.mark.parametrize("g,m,d,ctx,nodes,memory", PLANS)
def test_infinite_committed_values_show_as_what_they_are(g, m, d, ctx, nodes, memory):
    # columns of the first K/V head's V: one infinity early, one in every slot (the row's largest weight too, whose first term
    # is the whole weight), the other sign late, both signs, NaN. Weights of a row are within 2^15 of each other.
    q, kv = _random(3, g, m, d, ctx, nodes)
    q = (0.3 * q).to(torch.bfloat16)
    want, want_lse, through_memory = _call(q, kv, ctx, nodes, g, m, d)
    assert through_memory == memory
    v, n, inf = kv[0, :, g * d:], ctx[0], float("inf")
    v[1, 5] = inf
    v[:n, 17] = inf
    v[n - 1, d - 1] = -inf
    v[0, 20], v[n - 2, 20] = inf, -inf
    v[n // 2, 33] = float("nan")
    o, lse, _ = _call(q, kv, ctx, nodes, g, m, d)
    for h in range(m):
        for c, x in ((5, inf), (17, inf), (d - 1, -inf), (20, np.nan), (33, np.nan)):
            np.testing.assert_array_equal(o[:nodes[0], h * d + c], x)
            o[:nodes[0], h * d + c] = want[:nodes[0], h * d + c]
    np.testing.assert_array_equal(o, want)
    np.testing.assert_array_equal(lse, want_lse)


@pytest.mark.parametrize("d,ctx,at", [(128, 7, 3), (64, 300, 140), (128, 9000, 4107)])
def test_an_infinite_value_under_a_small_weight(d, ctx, at):
    # e^-62 = 2^-89.4 of the weight of its neighbour, which is the row's largest
    q, kv = torch.zeros(1, d), torch.ones(1, ctx + 1, 2 * d)
    q[0, 0] = 8.0
    kv[0, :, 0] = -80.0 * math.sqrt(d) / 8.0
    kv[0, at - 1, 0] = 0.0
    kv[0, at, 0] = -62.0 * math.sqrt(d) / 8.0
    kv[0, at, d + 7] = float("inf")
    o, _, _ = _call(q, kv, [ctx], [1], 1, 1, d)
    assert np.isposinf(o[0, 7]) and (np.delete(o[0], 7) == 1.0).all()


@pytest.mark.parametrize("g,m,d,ctx,nodes,memory", PLANS)
def test_infinite_values_of_drafts_show_in_the_rows_that_see_them(g, m, d, ctx, nodes, memory):
    q, kv = _random(4, g, m, d, ctx, nodes)
    q = (0.3 * q).to(torch.bfloat16)
    want, want_lse, through_memory = _call(q, kv, ctx, nodes, g, m, d)
    assert through_memory == memory
    at = nodes[0] // 2  # a chain: the nodes from `at` on see it
    kv[0, ctx[0] + at, g * d + 9] = -float("inf")
    o, lse, _ = _call(q, kv, ctx, nodes, g, m, d)
    for h in range(m):
        assert np.isneginf(o[at:nodes[0], h * d + 9]).all()
        o[at:nodes[0], h * d + 9] = want[at:nodes[0], h * d + 9]
    # the draft's other values enter in fp32 products of their own: the outputs' two roundings to bf16 at most
    np.testing.assert_allclose(o, want, rtol=2.0 ** -7, atol=2.0 ** -12)
    np.testing.assert_array_equal(lse, want_lse)


@pytest.mark.parametrize("g,m,d,ctx,nodes,form", [
    (1, 7, 128, [9000], [40], "tree"),           # three tiles of 18 nodes a part
    (1, 200, 64, [6000], [3], "tree"),           # a group of heads wider than a tile: two tiles a node
    (1, 2, 64, [9000], [130], "chain"),          # three tiles of 64 nodes
    (2, 3, 128, [7000, 5000, 30], [60, 3, 90], "any"),  # sequences of several parts and of one, each of several tiles
])
def test_merge_through_memory_of_several_tiles(g, m, d, ctx, nodes, form):
    q, kv, see, mask, _ = _tree_case(17, g, m, d, ctx, nodes, form)
    o, lse, through_memory = _call(q, kv, ctx, nodes, g, m, d, torch.from_numpy(mask).cuda())
    assert through_memory
    cu, q = _cu(nodes), bf16_np(q)
    for b, (c, n) in enumerate(zip(ctx, nodes)):
        rows = slice(cu[b], cu[b + 1])
        full = np.concatenate([np.ones((n, c), bool), see[b]], 1)
        want, want_lse, tol, tol_lse = _plain_rows(q[rows], bf16_np(kv[b, :c + n]), full, g, m, d)
        assert (np.abs(lse[rows] - want_lse) <= tol_lse).all()
        bad = np.abs(o[rows] - want) > tol
        assert not bad.any(), (b, bad.sum(), np.abs(o[rows] - want).max())
