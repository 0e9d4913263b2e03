"""Beam search's selection against a plain implementation in 64 bits (numpy on the host).

Tolerance of a total: the sum of exponentials is off by 2^-20 of itself (few units an exponential, fp32 sums of up to some hundred
positive terms in a tree), its logarithm by as much, and the total is rounded to fp32 (2^-24 of itself). Where candidates lie closer
together than twice that, their order is not asked for; the tests' seeds have none but exact ties, whose order is defined.
"""
import numpy as np
import pytest
import torch

from paper_2609_34977_gb300 import _native as N

pytestmark = pytest.mark.gpu


def _plain(z, scores, eos, n_out):
    B, n_in = scores.shape
    v = z.shape[1]
    parent, token = np.full((B, n_out), -1), np.full((B, n_out), -1)
    out, ended = np.full((B, n_out), -np.inf), np.full((B, n_in), -np.inf)
    gap = np.inf
    for b in range(B):
        cand = []
        for w in range(n_in):
            row = z[b * n_in + w].astype(np.float64)
            if not np.isfinite(scores[b, w]) or np.isnan(row).any() or np.isposinf(row).any() or np.isneginf(row).all():
                continue
            top = row.max()
            # (the maximum first: a logit of -3e38 would swallow the logarithm, in 64 bits too)
            t = float(scores[b, w]) + ((row - top) - np.log(np.exp(row - top).sum()))
            keep = np.argsort(-t, kind="stable")[:n_out + 2]
            cand += [(-t[i], w, int(i)) for i in np.union1d(keep, [eos] if eos >= 0 else []).astype(int) if t[i] > -np.inf]
        cand.sort()
        go = [c for c in cand if c[2] != eos][:n_out]
        for k, c in enumerate(go):
            parent[b, k], token[b, k], out[b, k] = b * n_in + c[1], c[2], -c[0]
        for k, c in enumerate(cand[:n_out]):
            if c[2] == eos:
                ended[b, c[1]] = -c[0]
        t = np.array([c[0] for c in cand[:2 * n_out + 2]])
        if len(t) > 1:
            step = np.diff(t)
            gap = min([gap] + [x for x in step if x != 0])
    return parent, token, out, ended, gap


def _run(z, scores, eos, n_out, ended=True, stream=None):
    B, n_in = scores.shape
    zc, sc = (x if isinstance(x, torch.Tensor) else torch.from_numpy(x).cuda() for x in (z, scores))
    parent = torch.full((B, n_out), -9, dtype=torch.int32, device="cuda")
    token, out = torch.full_like(parent, -9), torch.full((B, n_out), -9.0, device="cuda")
    end = torch.full((B, n_in), -9.0, device="cuda") if ended else None
    ws = torch.zeros(N.spd_beam_select_workspace_size(B, n_in, n_out, zc.shape[1]), dtype=torch.uint8, device="cuda")
    N.spd_beam_select(zc, sc, eos, parent, token, out, end, ws, stream=stream)
    torch.cuda.synchronize()
    return parent.cpu().numpy(), token.cpu().numpy(), out.cpu().numpy(), None if end is None else end.cpu().numpy()


def _check(z, scores, eos, n_out, got=None, apart=True):
    parent, token, out, ended, gap = _plain(z, scores, eos, n_out)
    tol = 2.0 ** -19 + 2.0 ** -23 * np.abs(out[np.isfinite(out)]).max(initial=0.0)
    assert gap > 2 * tol or not apart, gap
    p, t, s, e = got or _run(z, scores, eos, n_out)
    np.testing.assert_array_equal(p, parent)
    np.testing.assert_array_equal(t, token)
    for a, b in ((s, out), (e, ended)):
        np.testing.assert_array_equal(np.isneginf(a), np.isneginf(b))
        fin = np.isfinite(b)
        assert (np.abs(a[fin] - b[fin]) <= tol).all()


def _rand(seed, B, n_in, v, std=3.0):
    r = np.random.default_rng(seed)
    return (std * r.standard_normal((B * n_in, v))).astype(np.float32), (-5 * r.random((B, n_in))).astype(np.float32)


@pytest.mark.parametrize("B,n_in,n_out,v,eos", [
    (1, 1, 1, 1, -1),
    (1, 1, 1, 2, 0),
    (1, 4, 4, 32000, 2),
    (3, 1, 5, 1001, 7),          # the first step: one row forks
    (5, 3, 2, 4097, 4096),       # fewer beams out than in; a token in a batch of its own
    (2, 32, 32, 3001, 11),
    (16, 8, 8, 20000, 5),
    (40, 4, 4, 152064, 151643),  # rows beyond one wave
    (1, 16, 16, 7, 3),           # fewer tokens than beams
    (2, 2, 32, 9, -1),           # fewer candidates than places
])
def test_selection(B, n_in, n_out, v, eos):
    z, scores = _rand(1, B, n_in, v)
    if eos >= 0:
        z[::2, eos] = z[::2].max(1) + 1  # ends that come first
    _check(z, scores, eos, n_out)


@pytest.mark.parametrize("n_in,n_out,v,eos", [(12, 12, 152064, 3), (32, 32, 60001, 9), (9, 32, 152064, -1), (6, 1, 152064, 5)])
def test_one_request_over_many_lists(n_in, n_out, v, eos):
    z, scores = _rand(11, 1, n_in, v)
    _check(z, scores, eos, n_out)
    # equal rows, twenty equal bests all over them
    r = np.random.default_rng(12)
    row = np.zeros(v, np.float32)
    best = np.sort(r.choice(np.arange(16, v), 20, replace=False))
    row[best] = 3.0
    p, t, _, _ = _run(row[None].repeat(n_in, 0), np.zeros((1, n_in), np.float32), eos, n_out)
    np.testing.assert_array_equal(p[0], (np.arange(n_out) // 20).astype(int))
    np.testing.assert_array_equal(t[0], np.tile(best, 2)[:n_out])


def test_ties_go_to_the_lower_beam_and_token():
    z = np.zeros((6, 5000), np.float32)
    z[:, 4100:4110] = 2.0  # ten equal bests across two batches of a slice, in equal rows
    z[:, 4999] = 2.0
    scores = np.zeros((2, 3), np.float32)
    p, t, s, e = _run(z, scores, 4105, 16)
    want_t = [x for x in list(range(4100, 4110)) + [4999] if x != 4105]
    for b in range(2):
        np.testing.assert_array_equal(p[b], [3 * b] * 10 + [3 * b + 1] * 6)
        np.testing.assert_array_equal(t[b], want_t + want_t[:6])
        assert np.isfinite(e[b, 0]) and np.isneginf(e[b, 2])
    # everything is equal; -0 and 0 too
    z = np.where(np.arange(9000) % 2 == 0, 0.0, -0.0).astype(np.float32)[None].repeat(2, 0)
    p, t, s, e = _run(z, np.zeros((1, 2), np.float32), 1, 32)
    np.testing.assert_array_equal(t[0], [0] + list(range(2, 33)))
    assert (p == 0).all() and (s == s[0, 0]).all()


@pytest.mark.parametrize("rising", [True, False])
def test_sorted_logits(rising):
    v = 30000
    z = np.linspace(-9, 9, v).astype(np.float32)[::1 if rising else -1][None].repeat(2, 0).copy()
    _check(z, np.array([[-1.0, -2.0]], np.float32), 17, 24)


def test_masked_and_broken_rows():
    z, scores = _rand(3, 6, 4, 6000)
    z[0] = -np.inf                       # a grammar leaves nothing
    z[5, :5990] = -np.inf                # almost nothing
    z[6, 17] = np.nan
    z[7, 3] = np.inf
    z[8:12, 2:] = -np.inf                # fewer than n_out candidates in all
    scores[3, 1:] = -np.inf              # a request whose first step this is
    scores[4, 0] = np.nan
    scores[4, 2] = np.inf
    scores[5] = -np.inf                  # a request without a live beam
    z[16:20, 4] = z[16:20].max(1) + 2
    _check(z, scores, 4, 4)
    _check(z, scores, -1, 8)


def test_wide_and_negative_logits():
    z, scores = _rand(4, 2, 3, 5003, std=1.0)
    z = z * 200 - 9000
    scores = scores * 300
    _check(z.astype(np.float32), scores.astype(np.float32), 0, 6)
    _check(np.full((3, 4000), -3e38, np.float32), np.zeros((1, 3), np.float32), 5, 3)


@pytest.mark.parametrize("v,ld", [(4000, 4004), (4001, 4001), (4002, 4100), (999, 1003)])
def test_strides_and_alignment(v, ld):
    z, scores = _rand(5, 2, 2, v)
    wide = torch.full((4, ld + 3), float("nan"), device="cuda")
    view = wide.flatten()[1:1 + 4 * ld].view(4, ld)[:, :v]  # rows at any 4 bytes
    view.copy_(torch.from_numpy(z))
    _check(z, scores, 3, 5, got=_run(view, torch.from_numpy(scores).cuda(), 3, 5))


def test_the_same_in_every_run_without_ends_and_in_a_graph():
    z, scores = _rand(6, 8, 8, 50000)
    first = _run(z, scores, 9, 8)
    for _ in range(3):
        assert all(np.array_equal(a, b) for a, b in zip(first, _run(z, scores, 9, 8)))
    again = _run(z, scores, 9, 8, ended=False)
    assert again[3] is None and all(np.array_equal(a, b) for a, b in zip(first[:3], again[:3]))
    zc, sc = torch.from_numpy(z).cuda(), torch.from_numpy(scores).cuda()
    parent = torch.zeros(8, 8, dtype=torch.int32, device="cuda")
    token, out, end = torch.zeros_like(parent), torch.zeros(8, 8, device="cuda"), torch.zeros(8, 8, device="cuda")
    ws = torch.zeros(N.spd_beam_select_workspace_size(8, 8, 8, 50000), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        N.spd_beam_select(zc, sc, 9, parent, token, out, end, ws)
    other, _ = _rand(7, 8, 8, 50000)
    zc.copy_(torch.from_numpy(other))
    graph.replay()
    torch.cuda.synchronize()
    _check(other, scores, 9, 8, got=tuple(x.cpu().numpy() for x in (parent, token, out, end)))
