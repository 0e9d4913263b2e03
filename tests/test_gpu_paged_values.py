"""Attention over pages where values that are not finite lie in many tiles' masked keys at once: CTAs that go from unit to unit, with
warps a unit apart, show each value in the rows that see it and in no other, the same bits in every run."""
import numpy as np
import pytest
import torch

from paper_2609_34977_gb300 import _native as N
from tests.test_gpu_pages import _attend, _case, _cu, _i32, _rows, pytestmark  # noqa: F401


@pytest.mark.parametrize("g,m,d,new,lens,prefix", [
    (8, 2, 64, [600, 300, 37], [2600, 2300, 400], None),   # equal stretches: parts, and several units a CTA
    (4, 7, 128, [500, 129], [4500, 3000], None),
    (8, 2, 64, [700, 260], [700, 260], [0, 100]),          # a unit a CTA
    (2, 3, 128, [200, 64, 3], [260, 64, 900], [230, 0, 0]),
])
def test_many_tiles_with_values_that_are_not_finite(g, m, d, new, lens, prefix):
    page, cu = 16, _cu(new)
    q, pool, table = _case(17, g, m, d, new, lens, page)
    clean, lse = _attend(q, pool, table, new, lens, g, m, d, prefix)
    r = np.random.default_rng(d)
    bad, flat = [], pool.clone().view(-1, 2 * g * d)
    want = clean.clone().view(-1, g, m, d)
    for b, (n, ln) in enumerate(zip(new, lens)):
        limit = np.array([max(ln - n + i + 1, prefix[b] if prefix else 0) for i in range(n)])
        for h in range(g):
            # keys that some of the rows see, one in every other column
            for c, key in zip(range(int(r.integers(0, 2)), d, 2), r.integers(ln - n, ln, d)):
                x = (float("nan"), float("inf"), -float("inf"))[int(r.integers(0, 3))]
                flat[_rows(table[b], page, key, key + 1)[0], g * d + h * d + c] = x
                rows = torch.from_numpy(cu[b] + np.flatnonzero(limit > key)).cuda()
                want[rows, h, :, c] = x
                bad.append(len(rows))
    assert max(bad) > 1 and min(bad) >= 1
    pc, tc, qc = flat.view(pool.shape).cuda(), _i32(table), q.cuda()
    size = N.spd_paged_attention_workspace_size(sum(new), len(new), g * m, g, d)
    for _ in range(30):
        o, ls, ws = torch.empty_like(clean), torch.empty_like(lse), torch.zeros(size, dtype=torch.uint8, device="cuda")
        N.spd_paged_attention(qc, cu, lens, tc, pc, g * m, g, d, o, ls, ws, prefix=prefix)
        torch.cuda.synchronize()
        assert N.spd_workspace_status(ws) == 0 and torch.equal(ls, lse)
        got = o.view(want.shape)
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got, nan=0.0, posinf=7e30, neginf=-7e30), torch.nan_to_num(want, nan=0.0, posinf=7e30, neginf=-7e30))
