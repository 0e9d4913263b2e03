"""The paged cache against plain implementations in 64 bits (numpy on the host): rotary positions with several axes and the rows'
way into pages, attention of new tokens, page tables that fork, grow, end and are compacted.

Tolerances, from the arithmetic of the operators:
  rotation  the angle is off by a rounding to 24 bits of half a turn (2^-23) and the fraction's own (2^-53 a position, below 2^-32
            here), sine and cosine by two units (2^-22), products and sum by three roundings (3 2^-24): 2^-21 (|x| + |y|), and one
            rounding to bf16 (2^-8 |x'|)
  scores    fp32 sums of d exact bf16 products: |error| <= e_s = d 2^-24 max_j sum_c |q_c k_jc| / sqrt(d)
  lse       e_s, the exponentials' and the logarithm's few units (2^-20) and the rounding of the result (2^-22 |lse|)
  o         one rounding to bf16 (2^-8 |o|, twice the half unit), weights off by e_s twice (score and normaliser) and by fp32
            roundings (2^-18): (2 e_s + 2^-18) sum_j p_j |v_j|
Integers and moved rows are equal bit for bit.
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


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _table(r, lens, page, extra=2, width=None):
    """Pages handed out in no order, garbage behind every sequence's."""
    n = [-(-x // page) for x in lens]
    order = r.permutation(sum(n) + extra)
    t = np.full((len(lens), width or max(n) + 1), 1 << 30, np.int32)
    at = 0
    for b, k in enumerate(n):
        t[b, :k] = order[at:at + k]
        at += k
    return t, len(order)


def _rows(table, page, lo, hi):
    """Pool rows of a sequence's rows lo .. hi - 1."""
    x = np.arange(lo, hi)
    return table[x // page] * page + x % page


# ---- rotary positions, K/V into pages -------------------------------------------------------------
def _axis(kind, d):
    if kind == "one":
        return None
    if kind == "sections":
        return np.repeat([0, 1, 2], [d // 8, 3 * d // 16, 3 * d // 16]).astype(np.uint8)
    if kind == "turns":
        return (np.arange(d // 2) % 2).astype(np.uint8)
    return np.where(np.arange(d // 2) < d // 4, 0, 200).astype(np.uint8)  # the other half does not turn


@pytest.mark.parametrize("h,g,d,page,new,old,kind,far,theta", [
    (4, 4, 128, 16, [1], [0], "one", 0, 1e4),
    (28, 4, 128, 32, [1] * 7, [31, 32, 33, 0, 5, 64, 100], "sections", 0, 1e6),
    (7, 1, 64, 48, [50, 0, 3, 129], [0, 7, 46, 15], "turns", 0, 1e4),
    (16, 8, 64, 16, [33, 1], [16, 300], "half", 1 << 20, 1e4),
    (2, 2, 128, 64, [70], [1], "sections", (1 << 31) - 200, 1e6),
    (3, 3, 128, 16, [40], [2], "one", -300000, 0.5),
    (32, 32, 128, 64, [257, 100], [3, 0], "one", 5000, 1e4),
    (33, 1, 128, 64, [2860, 40], [5, 0], "sections", 0, 1e6),  # eight heads a thread, numbers of heads that eight does not divide
    (15, 3, 64, 32, [9600], [11], "turns", 1 << 20, 1e4),
])
def test_rope_pages(h, g, d, page, new, old, kind, far, theta):
    r = np.random.default_rng(len(new) + d + page)
    n, lens, cu = sum(new), [a + b for a, b in zip(new, old)], _cu(new)
    table, pages = _table(r, lens, page)
    axis = _axis(kind, d)
    axes = 1 if axis is None else 3 if kind == "sections" else 2 if kind == "turns" else 1
    pos = (r.integers(0, 150, (axes, n)) + far).astype(np.int32)
    # rows of q and kv within wider ones
    qw, kw = _rand((n, h * d + 16), 1, 2.0), _rand((n, 2 * g * d + 8), 2)
    q, kv = qw.cuda()[:, 8:8 + h * d], kw.cuda()[:, :2 * g * d]
    pool = _rand((pages, page, 2 * g * d), 3).cuda()
    before, q_out = pool.clone(), torch.full((n + 1, h * d), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = torch.zeros(64, dtype=torch.int32, device="cuda")
    N.spd_rope_pages(q, kv, _i32(pos), axis, theta, cu, lens, _i32(table), pool, h, g, d, q_out, ws)
    torch.cuda.synchronize()
    assert N.spd_workspace_status(ws) == 0
    ax = np.zeros(d // 2, int) if axis is None else axis.astype(int)
    theta = float(np.float32(theta))
    angle = np.zeros((n, d // 2))
    for j in range(d // 2):
        if ax[j] < axes:
            # far positions: the product modulo 2 pi in extended precision of two parts
            f = theta ** (-2.0 * j / d)
            hi = np.floor(pos[ax[j]].astype(np.float64) / 65536) * 65536
            angle[:, j] = np.fmod(hi * f, 2 * math.pi) + (pos[ax[j]] - hi) * f

    def want(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        tol = 2.0 ** -21 * np.abs(np.concatenate([np.abs(a) + np.abs(b)] * 2, -1))
        return np.concatenate([a * c - b * s, a * s + b * c], -1), tol

    # the reference's own angle: 2^-53 of itself
    slack = 4 * 2.0 ** -53 * np.abs(pos.astype(np.float64)).max() * max(1.0, theta ** (-1.0)) * 8
    for x, got in ((bf16_np(q).reshape(n, h, d), bf16_np(q_out[:n]).reshape(n, h, d)),
                   (bf16_np(kv)[:, :g * d].reshape(n, g, d),
                    bf16_np(pool.view(-1, 2 * g * d)[np.concatenate([_rows(table[b], page, old[b], lens[b]) for b in range(len(new))])]
                            )[:, :g * d].reshape(n, g, d))):
        w, tol = want(x)
        assert (np.abs(got - w) <= tol + slack * np.abs(x).max() + 2.0 ** -8 * np.abs(w)).all(), np.abs(got - w).max()
    written = np.concatenate([_rows(table[b], page, old[b], lens[b]) for b in range(len(new))]).astype(int)
    flat, was = pool.view(-1, 2 * g * d), before.view(-1, 2 * g * d)
    assert torch.equal(flat[written][:, g * d:], kv[:, g * d:])  # V as it is
    rest = np.setdiff1d(np.arange(pages * page), written)
    assert torch.equal(flat[rest], was[rest]) and (q_out[n] == 7.0).all()


def test_rope_in_place_and_many_sequences():
    h, g, d, page, B = 4, 2, 64, 16, 900  # more sequences than a launch holds
    r = np.random.default_rng(0)
    new = [int(x) for x in r.integers(0, 3, B)]
    lens = [x + int(y) for x, y in zip(new, r.integers(0, 40, B))]
    table, pages = _table(r, [max(1, x) for x in lens], page)
    n = sum(new)
    q, kv = _rand((n, h * d), 1).cuda(), _rand((n, 2 * g * d), 2).cuda()
    pos = _i32(r.integers(0, 500, (1, n)))
    pool, out, ws = torch.zeros(pages, page, 2 * g * d, dtype=torch.bfloat16, device="cuda"), torch.empty_like(q), torch.zeros(64, device="cuda")
    args = (pos, None, 1e4, _cu(new), lens, _i32(table))
    N.spd_rope_pages(q, kv, *args, pool, h, g, d, out, ws)
    pool2 = torch.zeros_like(pool)
    N.spd_rope_pages(q, kv, *args, pool2, h, g, d, q, ws)
    torch.cuda.synchronize()
    assert torch.equal(q, out) and torch.equal(pool, pool2) and N.spd_workspace_status(ws) == 0
    rows = np.concatenate([_rows(table[b], page, lens[b] - new[b], lens[b]) for b in range(B)]).astype(int)
    assert torch.equal(pool.view(-1, 2 * g * d)[rows][:, g * d:], kv[:, g * d:])


def test_bad_pages_are_reported_and_not_touched():
    h, g, d, page = 2, 1, 64, 16
    q, kv = _rand((2, h * d), 1).cuda(), _rand((2, 2 * g * d), 2).cuda()
    pool = torch.zeros(3, page, 2 * g * d, dtype=torch.bfloat16, device="cuda")
    for bad in (-1, 3, 1 << 30, -(1 << 31)):
        table = _i32([[0, bad], [1, 2]])
        ws = torch.zeros(N.spd_paged_attention_workspace_size(2, 2, h, g, d), dtype=torch.uint8, device="cuda")
        N.spd_rope_pages(q, kv, _i32([[16, 16]]), None, 1e4, [0, 1, 2], [17, 17], table, pool, h, g, d, torch.empty_like(q), ws)
        assert N.spd_workspace_status(ws) == N.SPD_EINVAL
        assert torch.equal(pool[2, 0, g * d:], kv[1, g * d:]) and (pool[:2] == 0).all()
        N.spd_paged_attention(q, [0, 1, 2], [17, 17], table, pool, h, g, d, torch.empty_like(q), None, ws)
        assert N.spd_workspace_status(ws) == N.SPD_EINVAL


# ---- attention ------------------------------------------------------------------------------------
def _plain_rows(q, kv, limit, g, m, d):
    """Rows q [n][g m d] over keys kv [k][2 g d] (float64), row i sees the first limit[i]: o, lse, the bounds of their errors."""
    n = len(limit)
    o, lse = np.zeros((n, g * m * d)), np.full((n, g * m), -np.inf)
    tol_o, tol_l = np.zeros_like(o), np.zeros_like(lse)
    see = np.arange(len(kv))[None] < np.asarray(limit)[:, None]
    for h in range(g * m):
        K, V = kv[:, (h // m) * d:(h // m + 1) * d], kv[:, (g + h // m) * d:(g + h // m + 1) * d]
        sl = slice(h * d, (h + 1) * d)
        s = np.where(see, q[:, sl] @ K.T / math.sqrt(d), -np.inf)
        e_s = d * 2.0 ** -24 * np.where(see, np.abs(q[:, sl]) @ np.abs(K).T, 0).max(1) / math.sqrt(d)
        top = s.max(1, keepdims=True)
        w = np.exp(s - top)
        lse[:, h] = top[:, 0] + np.log(w.sum(1))
        p = w / w.sum(1, keepdims=True)
        o[:, sl] = p @ V
        # a weight w is held as t + u, t = bf16(w), u = bf16(w - t): |w - t| <= 2^-8 w, |w - t - u| <= 2^-8 |w - t| <= 2^-16 w
        tol_o[:, sl] = 2.0 ** -8 * np.abs(o[:, sl]) + (2 * e_s + 2.0 ** -16 + 2.0 ** -18)[:, None] * (p @ np.abs(V))
        tol_l[:, h] = e_s + 2.0 ** -20 + 2.0 ** -22 * np.abs(lse[:, h])
    return o, lse, tol_o, tol_l


def _case(seed, g, m, d, new, lens, page, std=2.0, past=float("nan"), extra=2):
    r = np.random.default_rng(seed)
    table, pages = _table(r, [max(1, x) for x in lens], page, extra)
    q = _rand((sum(new), g * m * d), seed, std)
    pool = torch.full((pages * page, 2 * g * d), past, dtype=torch.bfloat16)  # rows that are no sequence's
    fill = _rand((sum(lens), 2 * g * d), seed + 1)
    at = 0
    for b, ln in enumerate(lens):
        pool[_rows(table[b], page, 0, ln)] = fill[at:at + ln]
        at += ln
    return q, pool.view(pages, page, 2 * g * d), table


def _attend(q, pool, table, new, lens, g, m, d, prefix=None, lse=True, stream=None):
    n = sum(new)
    o = torch.full((n + 1, g * m * d), 7.0, dtype=torch.bfloat16, device="cuda")
    ls = torch.full((n + 1, g * m), 7.0, device="cuda") if lse else None
    ws = torch.zeros(N.spd_paged_attention_workspace_size(n, len(new), g * m, g, d), dtype=torch.uint8, device="cuda")
    N.spd_paged_attention(q.cuda(), _cu(new), lens, _i32(table), pool.cuda(), g * m, g, d, o, ls, ws, prefix=prefix, stream=stream)
    torch.cuda.synchronize()
    assert N.spd_workspace_status(ws) == 0
    assert (o[n] == 7.0).all() and (ls is None or (ls[n] == 7.0).all())  # rows behind the last are left alone
    return o[:n], None if ls is None else ls[:n]


def _check(q, pool, table, new, lens, g, m, d, prefix, o, ls):
    cu, q, got, gl = _cu(new), bf16_np(q), bf16_np(o), ls.cpu().numpy().astype(np.float64)
    flat, page = pool.view(-1, 2 * g * d), pool.shape[1]
    for b, (n, ln) in enumerate(zip(new, lens)):
        if not n:
            continue
        kv = bf16_np(flat[_rows(table[b], page, 0, ln)])
        limit = [max(ln - n + i + 1, prefix[b] if prefix else 0) for i in range(n)]
        rows = slice(cu[b], cu[b + 1])
        want, wl, to, tl = _plain_rows(q[rows], kv, limit, g, m, d)
        assert (np.abs(gl[rows] - wl) <= tl).all(), (b, np.abs(gl[rows] - wl).max())
        bad = np.abs(got[rows] - want) > to
        assert not bad.any() and np.isfinite(got[rows]).all(), (b, bad.sum(), np.abs(got[rows] - want).max())


@pytest.mark.parametrize("g,m,d,new,lens,page,prefix", [
    (4, 1, 128, [1], [1], 16, None),                              # the first token of all
    (1, 1, 64, [1], [2], 16, None),
    (4, 1, 128, [1], [100], 16, None),                            # a decode step
    (2, 7, 128, [1, 1, 1], [63, 64, 65], 32, None),               # around a block
    (2, 7, 128, [1] * 5, [1, 500, 1000, 33, 257], 48, None),      # ragged, pages that end inside a block
    (8, 2, 64, [1] * 40, list(range(1, 1601, 40)), 16, None),
    (1, 8, 128, [1], [9000], 128, None),                          # split over many CTAs
    (1, 1, 128, [3], [5000], 64, None),
    (2, 1, 128, [130], [130], 16, None),                          # a prompt, just over a tile
    (4, 7, 128, [37, 0, 19, 1], [37, 5, 300, 65], 32, None),      # chunks of several lengths, one sequence without
    (2, 4, 64, [200, 65], [200, 700], 48, None),
    (2, 4, 64, [200, 65, 64], [200, 700, 90], 16, [100, 650, 90]),  # prefixes within the new, over both, and all of it
    (1, 1, 128, [64], [64], 64, [64]),
    (1, 16, 128, [50], [999], 16, [0]),
    (1, 200, 64, [3], [70], 32, None),                            # more heads a group than a tile has rows
    (3, 1, 64, [300], [1111], 16 * 7, None),                      # a page that is no power of two
    (1, 28, 128, [17], [400], 64, None),
    (32, 1, 128, [256], [256], 64, None),                         # a unit a CTA
    (32, 2, 64, [100], [130], 32, [50]),
    (2, 16, 64, [1, 1, 3], [129, 1, 700], 16, None),              # single tokens beside others
    (2, 9, 128, [1, 1, 1], [128, 127, 300], 16, [0, 100, 300]),   # (a prefix tells a last token nothing)
    (1, 17, 128, [1], [500], 16, None),                           # one head too many for the single tokens' form
    (32, 1, 128, [1] * 3, [384, 1, 200], 16, None),               # single tokens, a unit a CTA,
    (4, 7, 64, [1] * 30, [1150 - 7 * i for i in range(30)], 48, None),
    (32, 1, 128, [1], [385], 64, None),                           # and in parts
    (32, 1, 128, [1300], [1300], 64, None),                       # more units than the GPU holds at once, the longest first
    (40, 1, 64, [130, 700, 0, 260], [400, 700, 9, 260], 48, [0, 600, 0, 0]),
    (150, 2, 64, [40, 3], [40, 900], 16, None),
])
def test_attention(g, m, d, new, lens, page, prefix):
    q, pool, table = _case(5, g, m, d, new, lens, page)
    o, ls = _attend(q, pool, table, new, lens, g, m, d, prefix)
    _check(q, pool, table, new, lens, g, m, d, prefix, o, ls)
    again, _ = _attend(q, pool, table, new, lens, g, m, d, prefix, lse=False)
    assert torch.equal(again, o)


def test_attention_of_many_sequences():
    g, m, d, page = 1, 2, 64, 16
    r = np.random.default_rng(3)
    new = [int(x) for x in r.choice([0, 1, 1, 2, 40], 260)]
    lens = [n + int(x) for n, x in zip(new, r.integers(0, 150, 260))]
    q, pool, table = _case(6, g, m, d, new, lens, page)
    o, ls = _attend(q, pool, table, new, lens, g, m, d)
    _check(q, pool, table, new, lens, g, m, d, None, o, ls)


@pytest.mark.parametrize("g,m,d,new,ln", [(2, 3, 128, 40, 700), (2, 1, 64, 300, 900)])
def test_a_row_does_not_hang_on_its_neighbours(g, m, d, new, ln):
    # the scores of the other rows of a tile grow from block to block: the row's bits stay
    q, pool, table = _case(31, g, m, d, [new], [ln], 16)
    o, ls = _attend(q, pool, table, [new], [ln], g, m, d)
    keep = torch.arange(new) % 7 == 3
    other = q.clone()
    other[~keep] *= 20
    o2, ls2 = _attend(other, pool, table, [new], [ln], g, m, d)
    assert torch.equal(o[keep], o2[keep]) and torch.equal(ls[keep], ls2[keep])
    assert not torch.equal(o[~keep], o2[~keep])


@pytest.mark.parametrize("d,new,ln", [(128, 1, 777), (64, 90, 400)])
def test_sequences_share_pages(d, new, ln):
    # beams: the same pages in several tables, last pages of their own
    g, m, page = 2, 4, 16
    q, pool, table = _case(7, g, m, d, [new] * 3, [ln] * 3, page)
    shared = (ln - new) // page
    table[1:, :shared] = table[0, :shared]
    o, ls = _attend(q, pool, table, [new] * 3, [ln] * 3, g, m, d)
    _check(q, pool, table, [new] * 3, [ln] * 3, g, m, d, None, o, ls)


@pytest.mark.parametrize("new,ln", [(1, 300), (100, 300)])
def test_large_scores_and_cancelling_values(new, ln):
    # scores of hundreds: weights that are 0 or 1 and maxima that move from block to block; values whose sums cancel
    g, m, d, page = 2, 2, 128, 32
    q, pool, table = _case(8, g, m, d, [new], [ln], page, std=40.0)
    flat = pool.view(-1, 2 * g * d)
    rows = _rows(table[0], page, 0, ln)
    flat[rows, g * d:] = torch.where((torch.arange(ln) % 2 == 0)[:, None], 3.0e4, -3.0e4).to(torch.bfloat16)
    o, ls = _attend(q, pool, table, [new], [ln], g, m, d)
    _check(q, pool, table, [new], [ln], g, m, d, None, o, ls)
    small = torch.zeros_like(q)  # equal weights: the values cancel but for one
    o, ls = _attend(small, pool, table, [new], [ln], g, m, d)
    _check(small, pool, table, [new], [ln], g, m, d, None, o, ls)


@pytest.mark.parametrize("new,ln,prefix", [(1, 200, 0), (70, 200, 0), (70, 200, 150), (200, 200, 30)])
@pytest.mark.parametrize("what", ["nan_v", "inf_v", "nan_k", "inf_k"])
def test_values_that_are_not_finite_show_only_where_they_are_seen(new, ln, prefix, what):
    g, m, d, page = 2, 3, 128, 16
    q, pool, table = _case(9, g, m, d, [new], [ln], page)
    clean, _ = _attend(q, pool, table, [new], [ln], g, m, d, [prefix])
    flat = pool.view(-1, 2 * g * d)
    for at in (ln - 1, ln - new // 2 - 1):  # the last key, and one in the middle of the new ones
        bad = flat.clone()
        row = _rows(table[0], page, at, at + 1)[0]
        col = d + 5 if "k" in what else g * d + d + 5  # of the second K/V head
        bad[row, col] = float("nan") if "nan" in what else float("inf")
        o, ls = _attend(q, bad.view(pool.shape), table, [new], [ln], g, m, d, [prefix])
        o, ls = o.view(new, g, m, d).float(), ls.view(new, g, m)
        sees = np.array([at < max(ln - new + i + 1, prefix) for i in range(new)])
        ref = clean.view(new, g, m, d).float()
        assert torch.equal(o[:, 0], ref[:, 0])                                # the other head
        assert torch.equal(o[~sees, 1], ref[~sees, 1])                        # rows that do not see it
        hit = o[sees, 1]
        if "k" in what:  # a score of NaN or +-inf
            qc = q.view(new, g, m, d)[:, 1, :, 5].float().cuda()[sees]
            if what == "nan_k":
                assert torch.isnan(hit).all() and torch.isnan(ls[sees, 1]).all()
            else:
                assert torch.isnan(hit[qc > 0]).all() and torch.isfinite(hit[qc < 0]).all()
        else:
            other = torch.arange(d) != 5
            assert torch.equal(hit[..., other.cuda()], ref[sees, 1][..., other.cuda()])
            assert (torch.isnan if what == "nan_v" else torch.isinf)(hit[..., 5]).all()


def test_pools_of_more_than_two_to_the_32_elements():
    # rows at element offsets past 2^32: written, read and copied there
    h, g, d, page = 32, 32, 128, 64
    pages = (1 << 32) // (page * 2 * g * d) + 40
    pool = torch.full((1, pages, page, 2 * g * d), float("nan"), dtype=torch.bfloat16, device="cuda")
    new, lens = [100, 130], [100, 130]
    table = np.array([[pages - 1, 3, -1, -1], [pages - 20, pages - 7, 1, -1]], np.int32)
    fill, q = _rand((230, 2 * g * d), 1), _rand((230, h * d), 2, 2.0)
    pos, turned = torch.zeros(1, 230, dtype=torch.int32, device="cuda"), torch.empty(230, h * d, dtype=torch.bfloat16, device="cuda")
    N.spd_rope_pages(q.cuda(), fill.cuda(), pos, None, 1e4, _cu(new), lens, _i32(table), pool[0], h, g, d, turned)
    assert torch.equal(turned.cpu(), q)  # position 0 turns nothing
    for b, n in enumerate(lens):
        rows = torch.from_numpy(_rows(table[b], page, 0, n)).cuda()
        assert torch.equal(pool.view(-1, 2 * g * d)[rows].cpu(), fill[100 * b:100 * b + n])
    small = torch.cat([fill[:100], torch.zeros(28, 2 * g * d).bfloat16(), fill[100:], torch.zeros(62, 2 * g * d).bfloat16()])
    near = np.array([[0, 1, -1], [2, 3, 4]], np.int32)
    for k in ([100, 130], [1, 1]):  # tiles, and the single tokens' form
        sub = torch.cat([q[100 - k[0]:100], q[230 - k[1]:]])
        ws = torch.zeros(N.spd_paged_attention_workspace_size(sum(k), 2, h, g, d), dtype=torch.uint8, device="cuda")
        o = torch.empty(sum(k), h * d, dtype=torch.bfloat16, device="cuda")
        N.spd_paged_attention(sub.cuda(), _cu(k), lens, _i32(table), pool[0], h, g, d, o, None, ws)
        want, _ = _attend(sub, small.view(5, page, 2 * g * d), near, k, lens, h, 1, d)
        assert torch.equal(o, want) and N.spd_workspace_status(ws) == 0
    ref = np.ones(pages, np.int32)  # everything is held but three pages at the end, and the tables' pages by their tables
    ref[[pages - 2, pages - 3, pages - 4]] = 0
    r, t, _, status = _run_update(pool, ref, table, lens, [0, 0, 1], [1, 1, 0], g, d)
    assert status == 0 and t[1, 1] == pages - 4 and t[0, 1] == 3
    assert torch.equal(pool[0, pages - 4, :36].cpu(), fill[64:100])
    compacted, used = _i32(table), _i32([0])
    live = np.zeros(pages, np.int32)
    live[table[table >= 0]] = 1
    ws = torch.zeros(N.spd_pages_workspace_size(pages, 2), dtype=torch.uint8, device="cuda")
    N.spd_pages_compact(pool, g, d, _i32(live), compacted, _i32(live), compacted, used, ws)
    assert int(used) == 5 and compacted.max() < 5
    for b, n in enumerate(lens):
        rows = torch.from_numpy(_rows(compacted.cpu().numpy()[b], page, 0, n)).cuda()
        assert torch.equal(pool.view(-1, 2 * g * d)[rows].cpu(), fill[100 * b:100 * b + n])


def test_two_streams_and_a_graph():
    g, m, d, page, new, lens = 2, 4, 128, 32, [1, 40], [500, 90]
    q, pool, table = _case(10, g, m, d, new, lens, page)
    want, _ = _attend(q, pool, table, new, lens, g, m, d)
    qc, pc, tc = q.cuda(), pool.cuda(), _i32(table)
    size = N.spd_paged_attention_workspace_size(sum(new), 2, g * m, g, d)
    outs, keep = [], []
    for _ in range(2):  # at the same time, a workspace each
        st, o = torch.cuda.Stream(), torch.empty_like(qc)
        ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        for _ in range(5):
            N.spd_paged_attention(qc, _cu(new), lens, tc, pc, g * m, g, d, o, None, ws, stream=st.cuda_stream)
        outs.append(o)
        keep.append((st, ws))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    o, ws = torch.zeros_like(qc), torch.zeros(size, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        N.spd_paged_attention(qc, _cu(new), lens, tc, pc, g * m, g, d, o, None, ws)
    for _ in range(3):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)


# ---- page tables ----------------------------------------------------------------------------------
def _update(ref, table, lens, parent, grow, page):
    """The definition, one sequence after another."""
    ref, width = list(ref), table.shape[1]
    need = lambda n: -(-n // page)  # noqa: E731
    src = [lens[q] if 0 <= q < len(lens) else 0 for q in parent]
    mine = [[int(x) for x in table[q][:need(n)]] if n else [] for q, n in zip(parent, src)]
    for b, n in enumerate(lens):
        for x in table[b][:need(n)]:
            ref[x] -= 1
    for t in mine:
        for x in t:
            ref[x] += 1
    ends = {}
    for b, n in enumerate(src):
        if n % page:
            ends.setdefault(mine[b][-1], []).append((-(n % page), b))
    copies = {}
    for x, who in ends.items():
        keeps = min(who)[1] if ref[x] == len(who) else -1
        copies.update({b: x for _, b in who if b != keeps and grow[b] > 0})
    for x in copies.values():
        ref[x] -= 1
    free, moved, short = [x for x in range(len(ref)) if ref[x] <= 0], [], False
    take = lambda: free.pop(0) if free else -1  # noqa: E731
    for b, n in enumerate(src):
        fresh = need(n + grow[b]) - need(n)
        if b in copies:
            to = take()
            mine[b][-1] = to
            moved.append((copies[b], to, n % page))
        mine[b] += [take() for _ in range(fresh)]
        for x in mine[b][need(n) - (b in copies):]:
            short |= x < 0
            if x >= 0:
                ref[x] = 1
    out = np.array([t + [-1] * (width - len(t)) for t in mine], np.int32).reshape(len(parent), width)
    return ref, out, [n + g for n, g in zip(src, grow)], moved, short


def _run_update(pool, ref, table, lens, parent, grow, g, d, in_place=False):
    n_out = len(parent) if parent is not None else len(lens)
    ri = _i32(ref)
    ro = ri if in_place else torch.full_like(ri, -9)
    to = torch.full((n_out, table.shape[1]), -9, dtype=torch.int32, device="cuda")
    lo = torch.full((n_out,), -9, dtype=torch.int32, device="cuda")
    ws = torch.zeros(N.spd_pages_workspace_size(len(ref), max(n_out, len(lens))), dtype=torch.uint8, device="cuda")
    N.spd_pages_update(pool, g, d, ri, _i32(table), _i32(lens), None if parent is None else _i32(parent),
                       None if grow is None else _i32(grow), ro, to, lo, ws)
    torch.cuda.synchronize()
    return ro.cpu().numpy(), to.cpu().numpy(), lo.cpu().numpy(), N.spd_workspace_status(ws)


def _pool_of(layers, pages, page, g, d, seed=0):
    return _rand((layers, pages, page, 2 * g * d), seed).cuda()


def _ref_of(table, lens, page, pages):
    ref = np.zeros(pages, np.int32)
    for b, n in enumerate(lens):
        np.add.at(ref, table[b][:-(-n // page)], 1)
    return ref


def _check_update(pool, ref, table, lens, parent, grow, g, d, page, **kw):
    n_out = len(parent) if parent is not None else len(lens)
    before = pool.clone()
    par = parent if parent is not None else list(range(len(lens)))
    w_ref, w_table, w_len, moved, short = _update(ref, table, lens, par, grow if grow is not None else [0] * n_out, page)
    r, t, ln, status = _run_update(pool, ref, table, lens, parent, grow, g, d, **kw)
    np.testing.assert_array_equal(t, w_table)
    np.testing.assert_array_equal(r, w_ref)
    np.testing.assert_array_equal(ln, w_len)
    assert status == (N.SPD_ENOSPC if short else 0)
    for a, b, rows in moved:
        if b >= 0:
            before[:, b, :rows] = before[:, a, :rows]
    assert torch.equal(pool, before)
    return r, t, ln


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("page,g,d", [(16, 2, 64), (48, 1, 128)])
def test_updates_one_after_another(seed, page, g, d):
    # beams fork, end and grow from step to step; pages come back to the pool
    r = np.random.default_rng(seed)
    pages, width, layers, B = 90, 9, 2, 3
    pool = _pool_of(layers, pages, page, g, d)
    lens = [int(x) for x in r.integers(0, 2 * page, B)]
    table, used = _table(r, lens, page, extra=pages - sum(-(-x // page) for x in lens), width=width)
    assert used == pages
    ref = _ref_of(table, lens, page, pages)
    for step in range(8):
        n_out = int(r.integers(1, 9))
        parent = [int(x) for x in r.integers(-1, len(lens) + (step == 3), n_out)]  # -1 and (once) one past the end: empty
        room = [width * page - (lens[q] if 0 <= q < len(lens) else 0) for q in parent]
        grow = [int(min(r.choice([0, 1, 1, page // 2, page, 2 * page + 3]), x)) for x in room]
        ref, table, lens = _check_update(pool, ref, table, lens, parent, grow, g, d, page, in_place=step % 2 == 0)
        lens = [int(x) for x in lens]
        np.testing.assert_array_equal(ref, _ref_of(table, lens, page, pages))


def test_update_without_parents_or_growth():
    page, g, d = 16, 1, 64
    r = np.random.default_rng(1)
    lens = [0, 1, 16, 17, 100]
    table, pages = _table(r, lens, page, extra=12, width=10)
    ref = _ref_of(table, lens, page, pages)
    _check_update(_pool_of(1, pages, page, g, d), ref, table, lens, None, None, g, d, page)
    _check_update(_pool_of(1, pages, page, g, d), ref, table, lens, None, [16, 15, 1, 0, 60], g, d, page)


def test_a_last_page_that_others_hold():
    page, g, d = 16, 1, 64
    # 0 and 1 share their last page, 1 has more rows of it; 2 went on from it into a page of its own; 3 shares with 4 and nobody else
    table = np.array([[0, -1, -1], [0, -1, -1], [0, 1, -1], [2, -1, -1], [2, -1, -1], [3, -1, -1]], np.int32)
    lens = [5, 9, 20, 7, 7, 4]
    ref = np.array([3, 1, 2, 2] + [0] * 8, np.int32)  # page 3 is also held by somebody outside
    pool = _pool_of(3, 12, page, g, d)
    _check_update(pool, ref, table, lens, None, [1] * 6, g, d, page)
    _check_update(pool, ref, table, lens, [0, 1, 3, 3, 4, 5, 5], [1, 1, 0, 1, 1, 1, 0], g, d, page)


def test_update_with_no_pages_left_and_bad_lists():
    page, g, d = 16, 1, 64
    table = np.array([[0, 1, -1], [2, -1, -1]], np.int32)
    pool = _pool_of(1, 4, page, g, d)
    r, t, ln = _check_update(pool, [1, 1, 1, 0], table, [20, 16], [0, 0, 1], [1, 20, 1], g, d, page)  # one page for four
    # lengths that no table holds, entries outside the pool, references that do not count: reported, nothing faults
    for lens, tab, ref in (([20, 1000], table, [1, 1, 1, 0]), ([-5, 16], table, [1, 1, 1, 0]),
                           ([20, 16], np.array([[0, 77, -1], [-3, -1, -1]], np.int32), [1, 1, 1, 0]),
                           ([20, 16], table, [0, 0, 0, 0])):
        r, t, ln, status = _run_update(_pool_of(1, 4, page, g, d), ref, tab, lens, [1, 0], [1, 1], g, d)
        assert status in (N.SPD_EINVAL, N.SPD_ENOSPC) or ref == [0, 0, 0, 0]
        assert ((t >= -1) & (t < 4)).all()


def test_a_large_pool():
    page, g, d, B, W = 16, 1, 64, 300, 5
    r = np.random.default_rng(2)
    lens = [int(x) for x in r.integers(1, 400, B)]
    table, pages = _table(r, lens, page, extra=5000, width=30)
    ref = _ref_of(table, lens, page, pages)
    parent = [int(x) for x in r.integers(0, B, B * W)]
    pool = _pool_of(1, pages, page, g, d)
    ref, table, lens = _check_update(pool, ref, table, lens, parent, [int(x) for x in r.integers(0, 30, B * W)], g, d, page)


@pytest.mark.parametrize("pages,share", [(1, 1.0), (7, 0.0), (40, 0.5), (1500, 0.3), (5000, 0.9), (3000, 1.0)])
@pytest.mark.parametrize("in_place", [False, True])
def test_compaction(pages, share, in_place):
    page, g, d, layers = 16, 1, 64, 2
    r = np.random.default_rng(pages)
    ref = (r.random(pages) < share).astype(np.int32) * r.integers(1, 4, pages).astype(np.int32)
    live = np.flatnonzero(ref)
    table = np.full((3, max(1, len(live))), -1, np.int32)
    for b in range(3):
        k = r.permutation(live)[:int(r.integers(0, len(live) + 1))]
        table[b, :len(k)] = k
    pool = _pool_of(layers, pages, page, g, d)
    before = pool.clone()
    ri, ti = _i32(ref), _i32(table)
    ro, to = (ri, ti) if in_place else (torch.full_like(ri, -9), torch.full_like(ti, -9))
    used = torch.full((1,), -9, dtype=torch.int32, device="cuda")
    ws = torch.zeros(N.spd_pages_workspace_size(pages, 3), dtype=torch.uint8, device="cuda")
    N.spd_pages_compact(pool, g, d, ri, ti, ro, to, used, ws)
    torch.cuda.synchronize()
    assert N.spd_workspace_status(ws) == 0 and int(used) == len(live)
    to_page = dict(zip(live[live >= len(live)], np.flatnonzero(ref[:len(live)] == 0)))
    w_ref = np.where(np.arange(pages) < len(live), ref, 0)
    for a, b in to_page.items():
        w_ref[b] = ref[a]
        before[:, b] = before[:, a]
    np.testing.assert_array_equal(ro.cpu().numpy(), w_ref)
    np.testing.assert_array_equal(to.cpu().numpy(), np.vectorize(lambda x: to_page.get(x, x))(table))
    assert torch.equal(pool, before)


def test_compaction_reports_pages_that_nobody_counts():
    pool = _pool_of(1, 4, 16, 1, 64)
    ws = torch.zeros(N.spd_pages_workspace_size(4, 1), dtype=torch.uint8, device="cuda")
    t, used = _i32([[3, 1, 99, -1]]), _i32([0])
    N.spd_pages_compact(pool, 1, 64, _i32([0, 0, 1, 1]), t, _i32([0] * 4), t, used, ws)
    assert N.spd_workspace_status(ws) == N.SPD_EINVAL
    assert t.cpu().tolist() == [[1, 1, 99, -1]] and int(used) == 2
