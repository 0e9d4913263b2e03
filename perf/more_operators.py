"""A paged cache with chunked prompts and beams: the operators, in plain torch and as this library's calls, with the sizes
that are measured.

    rope     rotary positions with one to three axes on new rows of Q and K, and their K/V into the pages of the cache
    attn     attention of new tokens (one a sequence, a chunk of a prompt, a whole prompt) over a layer's pages
    update   sequences fork, end and grow: page tables, reference counts, shared last pages copied (all layers)
    compact  the pages in use move to the front of the pool (all layers)
    beam     the best continuations over beams and vocabulary

A pool is bf16 [layer][page][row of the page][K of every K/V head | V of every K/V head]. The shapes are those of the
repository's LLaVA-1.5 (32 heads of 128, 32000 words) and Qwen2-style decoders (28 heads on 4 of 128, 152064 words; positions
in time, height and width), and a small one with heads of 64 whose pairs take turns between height and width.
"""
import math

import numpy as np
import torch

own = False

BF16 = torch.bfloat16
SHAPES = {  # heads, K/V heads, head width, vocabulary, rotary base, axis of every rotary pair
    "llava": dict(h=32, g=32, d=128, vocab=32000, theta=1e4, axes=1, axis=[0] * 64),
    "qwen": dict(h=28, g=4, d=128, vocab=152064, theta=1e6, axes=3, axis=[0] * 16 + [1] * 24 + [2] * 24),
    "small": dict(h=16, g=8, d=64, vocab=32003, theta=1e4, axes=2, axis=[0, 1] * 16),
}
POOL = 8e8     # bytes of a drawn pool
SCORES = 2e9   # bytes that a drawn attention case's scores may take in fp32, padded


def listed():
    return [
        # the next token of 64 answers: latency
        dict(name="rope_step", kind="rope", shape="qwen", new=_join([1] * 64), old=_join(300 + 37 * i for i in range(64)), page=32,
             far=0),
        # the prompts of three requests, images and text, in one pass
        dict(name="rope_prompt", kind="rope", shape="llava", new="1301,2047,700", old="0,33,64", page=64, far=0),
        # the next token of one request: latency
        dict(name="attn_token", kind="attn", shape="llava", new="1", old="321", prefix="0", page=16),
        # a serving batch, one token each, at different depths of their contexts
        dict(name="attn_batch", kind="attn", shape="qwen", new=_join([1] * 48), old=_join(300 + 173 * i for i in range(48)),
             prefix=_join([0] * 48), page=32),
        # prompts of one image and text each (the image sees all of itself), one of them behind cached rows
        dict(name="attn_prompts", kind="attn", shape="small", new="700,581,1131,64", old="0,0,257,2000", prefix="577,577,0,0",
             page=48),
        # a chunk of a long prompt over what came before it
        dict(name="attn_chunk", kind="attn", shape="qwen", new="2048", old="14333", prefix="0", page=64),
        # a beam step of 16 requests with four beams each, all 28 layers: shared prompts, answers of their own
        dict(name="update_step", kind="update", shape="qwen", layers=28, requests=16, beams=4, prompt=700, answer=90, page=32,
             fork=0),
        # four prompts fork into eight beams each: their last pages are copied
        dict(name="update_fork", kind="update", shape="llava", layers=32, requests=4, beams=8, prompt=640, answer=1, page=64,
             fork=1),
        # a small pool after one answer of three has ended
        dict(name="compact_small", kind="compact", shape="small", layers=2, requests=3, rows=200, page=16, ended=1),
        # half of 24 answers have ended, their pages all over the pool
        dict(name="compact_pool", kind="compact", shape="qwen", layers=28, requests=24, rows=1200, page=64, ended=12),
        # one request with four beams
        dict(name="beam_one", kind="beam", shape="llava", requests=1, beams=4),
        # sixteen requests with eight beams each over a large vocabulary
        dict(name="beam_batch", kind="beam", shape="qwen", requests=16, beams=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _join(v):
    return ",".join(str(int(x)) for x in v)


def _ints(s):
    return [int(v) for v in str(s).split(",")]


def draw(rng):
    kind = rng.choice(["rope", "attn", "attn", "attn", "update", "compact", "beam"])
    shape = rng.choice(["llava", "qwen", "qwen", "small"])
    c = SHAPES[shape]
    page = rng.choice([16, 32, 48, 64, 128])
    if kind == "beam":
        beams = _log(rng, 1, 16)
        return dict(kind=kind, shape=shape, requests=_log(rng, 1, max(1, 128 // beams)), beams=beams)
    if kind in ("rope", "attn"):
        b = _log(rng, 1, 48)
        one = rng.random() < 0.5
        rows = int(POOL / (4 * c["g"] * c["d"])) // (4 * b)
        top = 1 if one else (4000 if kind == "rope" else 1500)
        new = [_log(rng, 1, max(1, min(top, rows))) for _ in range(b)]
        if kind == "rope":
            scale = min(1.0, 4000 / sum(new))
            new = [max(1, int(n * scale)) for n in new]
            return dict(kind=kind, shape=shape, new=_join(new), old=_join(_log(rng, 1, min(4000, rows)) - 1 for _ in range(b)),
                        page=page, far=rng.choice([0, 0, 250000]))
        keys = min(rows, 65000, int(SCORES / (4 * c["h"] * b * max(new))), int(8e9 / (c["h"] * c["d"] * sum(new))) + 64)
        old = [_log(rng, 1, max(1, keys - max(new))) - 1 for _ in range(b)]
        prefix = [rng.choice([0, 0, rng.randint(0, n + o)]) for n, o in zip(new, old)]
        return dict(kind=kind, shape=shape, new=_join(new), old=_join(old), prefix=_join(prefix), page=page)
    layers = _log(rng, 1, 28)
    row = 4 * c["g"] * c["d"] * layers
    if kind == "update":
        beams, fork = _log(rng, 1, 8), rng.choice([0, 0, 1])
        requests = _log(rng, 1, 32 // beams)
        rows = int(POOL / row)
        answer = _log(rng, 1, max(1, min(300, rows // (3 * requests * beams))))
        prompt = _log(rng, 1, max(1, min(4000, rows // (3 * requests))))
        return dict(kind=kind, shape=shape, layers=layers, requests=requests, beams=beams, prompt=prompt, answer=answer, page=page,
                    fork=fork)
    requests = _log(rng, 2, 24)
    rows = _log(rng, 1, max(1, min(4000, int(POOL / row) // requests)))
    return dict(kind=kind, shape=shape, layers=layers, requests=requests, rows=rows, page=page, ended=rng.randint(1, requests - 1))


# ---- inputs -----------------------------------------------------------------------------------
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt) % (1 << 62))


def _randn(shape, g, std=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(std)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _pages_of(rows, page):
    return (np.asarray(rows) + page - 1) // page


def _tables(r, lens, page, spare=3):
    """A pool whose pages were handed out in no order: tables [seq][most pages], -1 behind a sequence's pages."""
    n = _pages_of(lens, page)
    order = r.permutation(int(n.sum()) + spare)
    table = np.full((len(lens), int(n.max()) + 1), -1, np.int32)
    at = 0
    for b, k in enumerate(n):
        table[b, :k] = order[at:at + k]
        at += k
    return table, len(order)


def _positions(r, new, old, axes, far):
    """Rotary positions of a multimodal prompt: stretches of text, where all axes go on together, and images, which go
    through rows and columns of a grid; the next stretch begins behind the largest position. far: where a long video ended."""
    out = []
    for n, o in zip(new, old):
        at, got = int(o) + far, []
        while sum(x.shape[1] for x in got) < n:
            left = n - sum(x.shape[1] for x in got)
            if axes > 1 and left > 8 and r.random() < 0.5:
                w = int(r.integers(2, 40))
                k = min(left, w * int(r.integers(2, 40)))
                i = np.arange(k)
                p = np.stack([np.zeros(k, int), i // w, i % w][3 - axes:]) + at
            else:
                k = min(left, int(r.integers(1, 400)))
                p = np.tile(np.arange(k) + at, (axes, 1))
            got.append(p)
            at = int(p.max()) + 1
        out.append(np.concatenate(got, 1)[:, :n])
    return np.concatenate(out, 1).astype(np.int32)


def prepare(case, seed):
    k, c = case["kind"], SHAPES[case["shape"]]
    g, r = _gen(seed, 2), np.random.default_rng(seed)
    e = lambda shape, dt: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    s = dict(case=case, c=c)
    qd, kvd = c["h"] * c["d"], c["g"] * c["d"]
    if k == "beam":
        n, v = case["requests"] * case["beams"], c["vocab"]
        s.update(z=_randn((n, v), g, 3.0), scores=-5.0 * torch.rand((case["requests"], case["beams"]), generator=g, device="cuda"),
                 eos=int(r.integers(0, v)))
        s["z"][::2, s["eos"]] = 12.0  # half of the beams are about to end
        m = (case["requests"], case["beams"])
        return dict(s, parent=e(m, torch.int32), token=e(m, torch.int32), out=e(m, torch.float32), ended=e(m, torch.float32),
                    ws=e(_ws("spd_beam_select_workspace_size", case["requests"], case["beams"], case["beams"], v), torch.uint8))
    page = case["page"]
    if k in ("rope", "attn"):
        new, old = np.array(_ints(case["new"])), np.array(_ints(case["old"]))
        n, lens = int(new.sum()), (new + old).astype(np.int32)
        table, pages = _tables(r, lens, page)
        s.update(new=new, lens=lens, q_cu=np.concatenate([[0], np.cumsum(new)]).astype(np.int32), table=_i32(table), page=page,
                 pool=_randn((pages, page, 2 * kvd), g, 1.0, BF16), q=_randn((n, qd), g, 2.5, BF16))
        if k == "rope":
            return dict(s, kv=_randn((n, 2 * kvd), g, 1.0, BF16), pos=_i32(_positions(r, new, old, c["axes"], case["far"])),
                        axis=np.array(c["axis"], np.uint8), q_out=e((n, qd), BF16), ws=e(1024, torch.uint8))
        prefix = np.array(_ints(case["prefix"]), np.int32)
        return dict(s, prefix=prefix if prefix.any() else None, o=e((n, qd), BF16), lse=e((n, c["h"]), torch.float32),
                    ws=e(_ws("spd_paged_attention_workspace_size", n, len(new), c["h"], c["g"], c["d"]), torch.uint8))
    layers = case["layers"]
    if k == "update":
        R, W, fork = case["requests"], case["beams"], case["fork"]
        # a prompt's whole pages are shared by its beams; behind them every beam has pages of its own
        prompt = np.array([max(1, case["prompt"] * (R + i) // (2 * R)) for i in range(R)])
        shared = _pages_of(prompt, page) if fork else prompt // page
        lens = np.repeat(prompt, 1 if fork else W) + (0 if fork else case["answer"])
        own_pages = np.zeros(R * W, int) if fork else _pages_of(lens, page) - np.repeat(shared, W)
        spare = R * W * 2 + 7
        order = r.permutation(int(shared.sum() + own_pages.sum()) + spare)
        at, B = 0, len(lens)
        most = int(_pages_of(lens + 1, page).max()) + 1
        table, ref = np.full((B, most), -1, np.int32), np.zeros(len(order), np.int32)
        for i in range(R):
            rows = [i] if fork else range(i * W, (i + 1) * W)
            for b in rows:
                table[b, :shared[i]] = order[at:at + shared[i]]
            ref[order[at:at + shared[i]]] = len(rows)
            at += shared[i]
            for b in [] if fork else rows:
                table[b, shared[i]:shared[i] + own_pages[b]] = order[at:at + own_pages[b]]
                ref[order[at:at + own_pages[b]]] = 1
                at += own_pages[b]
        parent = np.repeat(np.arange(R), W) if fork else np.concatenate([i * W + np.sort(r.integers(0, W, W)) for i in range(R)])
        s.update(table=_i32(table), ref=_i32(ref), lens=_i32(lens), parent=_i32(parent), grow=_i32(np.ones(R * W)), B=B)
        n_out = R * W
    else:
        R = case["requests"]
        lens = np.array([max(1, case["rows"] * (R + i) // (2 * R)) for i in range(R)])
        table, pages = _tables(r, lens, page)
        gone = r.permutation(R)[:case["ended"]]
        ref = np.zeros(pages, np.int32)
        table[gone] = -1
        ref[table[table >= 0]] = 1
        s.update(table=_i32(table), ref=_i32(ref), used=e(1, torch.int32))
        n_out = R
    pages = len(ref)
    return dict(s, pool=_randn((layers, pages, page, 2 * kvd), g, 1.0, BF16), page=page,
                table_out=e((n_out, table.shape[1]), torch.int32), len_out=e(n_out, torch.int32), ref_out=e(pages, torch.int32),
                ws=e(_ws("spd_pages_workspace_size", pages, n_out), torch.uint8))


def _ws(name, *sizes):
    """Workspace bytes of a call (the plain forms need none)."""
    if not own:
        return 16
    from paper_2609_34977_gb300 import _native as N
    return getattr(N, name)(*sizes)


# ---- the library's calls ----------------------------------------------------------------------
def _run_own(s):
    from paper_2609_34977_gb300 import _native as N
    k, c = s["case"]["kind"], s["c"]
    if k == "rope":
        N.spd_rope_pages(s["q"], s["kv"], s["pos"], s["axis"], c["theta"], s["q_cu"], s["lens"], s["table"], s["pool"], c["h"],
                         c["g"], c["d"], s["q_out"], s["ws"])
        return dict(q=s["q_out"], pool=s["pool"])
    if k == "attn":
        N.spd_paged_attention(s["q"], s["q_cu"], s["lens"], s["table"], s["pool"], c["h"], c["g"], c["d"], s["o"], s["lse"],
                              s["ws"], prefix=s["prefix"])
        return dict(o=s["o"], lse=s["lse"])
    if k == "update":
        N.spd_pages_update(s["pool"], c["g"], c["d"], s["ref"], s["table"], s["lens"], s["parent"], s["grow"], s["ref_out"],
                           s["table_out"], s["len_out"], s["ws"])
        return dict(pool=s["pool"], table=s["table_out"], lens=s["len_out"], ref=s["ref_out"])
    if k == "compact":
        N.spd_pages_compact(s["pool"], c["g"], c["d"], s["ref"], s["table"], s["ref_out"], s["table_out"], s["used"], s["ws"])
        # (what the pages behind those in use hold is nobody's)
        return dict(pool=s["pool"], table=s["table_out"], ref=s["ref_out"], used=s["used"])
    N.spd_beam_select(s["z"], s["scores"], s["eos"], s["parent"], s["token"], s["out"], s["ended"], s["ws"])
    return dict(parent=s["parent"], token=s["token"], scores=s["out"], ended=s["ended"])


# ---- the plain forms --------------------------------------------------------------------------
def _dev(a):
    return torch.as_tensor(np.asarray(a, np.int64), device="cuda")


def _plain_rope(s):
    c = s["c"]
    h, g, d = c["h"], c["g"], c["d"]
    j = torch.arange(d // 2, device="cuda", dtype=torch.float64)
    freq = torch.exp(j * (-2.0 / d * math.log(c["theta"])))
    angle = s["pos"][_dev(s["axis"])].double() * freq[:, None]                 # [pair][token]
    cos, sin = torch.cos(angle).T.float()[:, None], torch.sin(angle).T.float()[:, None]

    def turn(x):
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)

    n = s["q"].shape[0]
    q = turn(s["q"].float().view(n, h, d)).to(BF16).view(n, h * d)
    k = turn(s["kv"][:, :g * d].float().view(n, g, d)).to(BF16).view(n, g * d)
    seq = torch.repeat_interleave(torch.arange(len(s["new"]), device="cuda"), _dev(s["new"]), output_size=n)
    slot = torch.arange(n, device="cuda") - _dev(s["q_cu"])[seq + 1] + _dev(s["lens"])[seq]
    page = s["table"][seq, slot // s["page"]].long()
    s["pool"][page, slot % s["page"]] = torch.cat([k, s["kv"][:, g * d:]], 1)
    return dict(q=q, pool=s["pool"])


def _plain_attn(s):
    c = s["c"]
    h, g, d = c["h"], c["g"], c["d"]
    b, most = len(s["new"]), int(s["new"].max())
    lens, new = _dev(s["lens"]), _dev(s["new"])
    i = torch.arange(most, device="cuda")
    real = i[None] < new[:, None]
    rows = torch.where(real, _dev(s["q_cu"][:-1])[:, None] + i[None], 0)
    keys = int(s["lens"].max())
    kv = s["pool"][s["table"].clamp(min=0).long()].view(b, -1, 2 * g * d)[:, :keys].float().view(b, keys, 2, g, d)
    q = s["q"].float().view(-1, g, h // g, d)[rows]                            # [b][n][g][m][d]
    score = torch.einsum("bngmd,bkgd->bgmnk", q, kv[:, :, 0]) / math.sqrt(d)
    limit = lens[:, None] - new[:, None] + i[None] + 1
    if s["prefix"] is not None:
        limit = torch.maximum(limit, _dev(s["prefix"])[:, None])
    seen = torch.arange(keys, device="cuda") < limit[..., None]
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - top)
    total = w.sum(-1, keepdim=True)
    v = torch.where((torch.arange(keys, device="cuda") < lens[:, None])[..., None, None], kv[:, :, 1], 0.0)
    o = torch.einsum("bgmnk,bkgd->bngmd", w / total, v)
    lse = (torch.log(total) + top)[..., 0].permute(0, 3, 1, 2)
    return dict(o=o[real].reshape(-1, h * d).to(BF16), lse=lse[real].reshape(-1, h))


def _plain_update(s):
    page, n_in = s["page"], s["B"]
    pages, (n, most) = s["ref"].shape[0], s["table_out"].shape
    k = torch.arange(most, device="cuda")
    parent, grow, lens = s["parent"].long(), s["grow"].long(), s["lens"].long()
    kids = torch.zeros(n_in, dtype=torch.int64, device="cuda").scatter_add_(0, parent, torch.ones_like(parent))
    listed_in = k[None] < ((lens + page - 1) // page)[:, None]
    ref = s["ref"].long().scatter_add(0, s["table"].clamp(min=0).long().flatten(),
                                      torch.where(listed_in, (kids - 1)[:, None], 0).flatten())
    held = lens[parent]
    have = (held + page - 1) // page
    table = torch.where(k[None] < have[:, None], s["table"][parent], -1).long()
    # a last page that is not full belongs to the sequence that holds most of it (the first of them); others that grow copy it
    part, b = held % page, torch.arange(n, device="cuda")
    tail = table.gather(1, (held // page)[:, None])[:, 0].clamp(min=0)
    key = torch.where(part > 0, part * (n + 1) + n - b, 0)
    owner = torch.zeros(pages, dtype=torch.int64, device="cuda").scatter_reduce(0, tail, key, "amax")
    count = torch.zeros(pages, dtype=torch.int64, device="cuda").scatter_add(0, tail, (part > 0) * 1)
    copy = (part > 0) & (grow > 0) & ~((owner[tail] == key) & (ref[tail] == count[tail]))
    ref = ref.scatter_add(0, tail, torch.where(copy, -1, 0))
    want = (held + grow + page - 1) // page
    fresh = want - have + copy * 1
    first = torch.cumsum(fresh, 0) - fresh
    free = torch.argsort(ref > 0, stable=True)  # free pages first, in their order
    at = torch.where(copy, have - 1, have)
    made = (k[None] >= at[:, None]) & (k[None] < want[:, None])
    got = free[(first[:, None] + k[None] - at[:, None]).clamp(0, pages - 1)]
    table = torch.where(made, got, table)
    ref = ref + (torch.arange(pages, device="cuda")[None] == torch.where(made, got, -1).flatten()[:, None]).sum(0)
    c = torch.nonzero(copy)[:, 0]
    row = (torch.arange(page, device="cuda")[None] < part[c][:, None])[None, :, :, None]
    to, of = table[c, held[c] // page], tail[c]
    s["pool"][:, to] = torch.where(row, s["pool"][:, of], s["pool"][:, to])
    return dict(pool=s["pool"], table=table.int(), lens=(held + grow).int(), ref=ref.int())


def _plain_compact(s):
    pages = s["ref"].shape[0]
    p, live = torch.arange(pages, device="cuda"), s["ref"] > 0
    used = live.sum()
    fill, hole = live & (p >= used), ~live & (p < used)
    of, to = torch.nonzero(fill)[:, 0], torch.nonzero(hole)[:, 0]
    goes = p.clone()
    goes[of] = to
    s["pool"][:, to] = s["pool"][:, of]
    ref = torch.where(p < used, s["ref"], 0)
    ref[to] = s["ref"][of]
    table = torch.where(s["table"] >= 0, goes[s["table"].clamp(min=0).long()], s["table"].long())
    return dict(pool=s["pool"], table=table.int(), ref=ref, used=used.view(1).int())


def _plain_beam(s):
    z, (R, W) = s["z"], s["parent"].shape
    v = z.shape[1]
    top = z.amax(1, keepdim=True)
    norm = top.double() + torch.log(torch.exp((z - top).double()).sum(1, keepdim=True))  # candidates lie close together
    total = (s["scores"].double().view(-1, 1) + z.double() - norm).view(R, W, v)
    eos = total[:, :, s["eos"]].clone()
    total[:, :, s["eos"]] = -math.inf
    order = torch.argsort(total.view(R, W * v), dim=1, descending=True, stable=True)[:, :W]
    score = total.view(R, W * v).gather(1, order)
    parent = order // v + W * torch.arange(R, device="cuda")[:, None]
    # an ending beam counts where fewer than W candidates, other endings among them, go before it
    at = torch.arange(W, device="cuda")
    before = (score[:, None] > eos[..., None]) | ((score[:, None] == eos[..., None]) &
                                                  (order[:, None] < (at * v + s["eos"])[None, :, None]))
    other = (eos[:, None] > eos[..., None]) | ((eos[:, None] == eos[..., None]) & (at[None, None] < at[None, :, None]))
    ended = torch.where(before.sum(2) + other.sum(2) < W, eos, -math.inf)
    return dict(parent=parent.int(), token=(order % v).int(), scores=score.float(), ended=ended.float())


def run(s):
    if own:
        return _run_own(s)
    return dict(rope=_plain_rope, attn=_plain_attn, update=_plain_update, compact=_plain_compact,
                beam=_plain_beam)[s["case"]["kind"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    k, c = case["kind"], SHAPES[case["shape"]]
    h, g, d = c["h"], c["g"], c["d"]
    if k == "rope":
        n = sum(_ints(case["new"]))
        return dict(bytes=4 * n * (h + 2 * g) * d + 4 * n * c["axes"], flops=3 * n * (h + g) * d)
    if k == "attn":
        new, old, prefix = _ints(case["new"]), _ints(case["old"]), _ints(case["prefix"])
        n, pairs = sum(new), 0
        for x, o, p in zip(new, old, prefix):
            whole = min(x, max(0, p - o))  # rows that see the prefix and no more
            pairs += whole * p + sum(range(o + whole + 1, o + x + 1))
        return dict(bytes=4 * g * d * sum(x + o for x, o in zip(new, old)) + 4 * n * h * d + 4 * n * h, flops=4 * h * d * pairs)
    if k == "beam":
        return dict(bytes=4 * case["requests"] * case["beams"] * c["vocab"], flops=0)
    page, row = case["page"], 4 * g * d * case["layers"]
    if k == "update":
        R, W = case["requests"], case["beams"]
        prompt = [max(1, case["prompt"] * (R + i) // (2 * R)) for i in range(R)]
        if case["fork"]:
            copied = sum((W - 1) * (p % page) for p in prompt)
            entries = sum(_pages_of(p, page) + W * _pages_of(p + 1, page) for p in prompt)
        else:  # of W parents drawn with replacement W (1 - (1 - 1 / W)^W) differ
            copied = sum((p + case["answer"]) % page * W * (1 - 1 / W) ** W for p in prompt)
            entries = 2 * W * sum(_pages_of(p + case["answer"], page) for p in prompt)
        return dict(bytes=int(2 * copied * row + 4 * entries), flops=0)
    R = case["requests"]
    pages = [int(_pages_of(max(1, case["rows"] * (R + i) // (2 * R)), page)) for i in range(R)]
    gone = case["ended"] / R  # on average this share of the pages is free, and as large a share of those in use has to move
    return dict(bytes=int(sum(pages) * (1 - gone) * gone * 2 * row * page + 8 * sum(pages)), flops=0)


# ---- the definitions in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c, k = s["c"], case["kind"]
    if k == "beam":
        return _exact_beam(s)
    h, g, d, page = c["h"], c["g"], c["d"], s["page"]
    table = s["table"].cpu().numpy()
    if k == "rope":
        n, half = s["q"].shape[0], d // 2
        pos = s["pos"].cpu().numpy().astype(np.float64)
        w = np.array([c["theta"] ** (-2.0 * j / d) for j in range(half)])
        turn = torch.from_numpy(np.exp(1j * pos[s["axis"].astype(int)].T * w)).cuda()  # e^(i angle), [token][pair]

        def rotate(x):
            y = torch.complex(x[..., :half], x[..., half:]) * turn[:, None]
            return torch.cat([y.real, y.imag], -1)

        q = rotate(s["q"].double().view(n, h, d)).reshape(n, h * d)
        kv = s["kv"].double()
        kv = torch.cat([rotate(kv[:, :g * d].view(n, g, d)).reshape(n, g * d), kv[:, g * d:]], 1)
        pool = s["pool"].double().view(-1, 2 * g * d)
        at = [table[b, x // page] * page + x % page
              for b, (m, ln) in enumerate(zip(s["new"], s["lens"])) for x in range(ln - m, ln)]
        pool[torch.tensor(at, device="cuda")] = kv
        return dict(q=q, pool=pool.view(s["pool"].shape))
    if k == "attn":
        o, lse = [], []
        for b, (m, ln) in enumerate(zip(s["new"].tolist(), s["lens"].tolist())):
            lo = int(s["q_cu"][b])
            rows = torch.cat([s["pool"][p] for p in table[b, :-(-ln // page)].tolist()])[:ln].double()
            seen = torch.ones((m, ln), dtype=torch.bool, device="cuda").tril(ln - m)
            if s["prefix"] is not None:
                seen[:, :int(s["prefix"][b])] = True
            rows_o, rows_l = [], []
            for head in range(h):
                at = head // (h // g) * d
                x = s["q"][lo:lo + m, head * d:(head + 1) * d].double() @ rows[:, at:at + d].T * d ** -0.5
                x[~seen] = -math.inf
                rows_l.append(torch.logsumexp(x, 1))
                rows_o.append(torch.exp(x - rows_l[-1][:, None]) @ rows[:, g * d + at:g * d + at + d])
            o.append(torch.cat(rows_o, 1))
            lse.append(torch.stack(rows_l, 1))
        return dict(o=torch.cat(o), lse=torch.cat(lse))
    ref = s["ref"].cpu().numpy().astype(int).tolist()
    if k == "compact":
        live = [p for p in range(len(ref)) if ref[p] > 0]
        used = len(live)
        moves = dict(zip([p for p in live if p >= used], [p for p in range(used) if ref[p] <= 0]))
        out_ref = [ref[p] if p < used else 0 for p in range(len(ref))]
        for of, to in moves.items():
            out_ref[to] = ref[of]
            s["pool"][:, to] = s["pool"][:, of].clone()
        out = [[moves.get(int(p), int(p)) for p in t] for t in table]
        return dict(pool=s["pool"], table=torch.tensor(out, dtype=torch.int32), ref=torch.tensor(out_ref, dtype=torch.int32),
                    used=torch.tensor([used], dtype=torch.int32))
    lens, parent, grow = (s[x].cpu().tolist() for x in ("lens", "parent", "grow"))
    mine = [[int(p) for p in table[q][:-(-lens[q] // page)]] for q in parent]
    for b, ln in enumerate(lens):
        for p in table[b][:-(-ln // page)]:
            ref[p] -= 1
    for t in mine:
        for p in t:
            ref[p] += 1
    by_tail = {}
    for b, q in enumerate(parent):
        if lens[q] % page:
            by_tail.setdefault(mine[b][-1], []).append((-(lens[q] % page), b))
    copies = set()
    for p, users in by_tail.items():
        keeps = min(users)[1] if ref[p] == len(users) else -1
        copies |= {b for _, b in users if b != keeps and grow[b] > 0}
    for b in copies:
        ref[mine[b][-1]] -= 1
    free = iter([p for p in range(len(ref)) if ref[p] <= 0])
    for b, q in enumerate(parent):
        if b in copies:
            of, to, m = mine[b][-1], next(free), lens[q] % page
            s["pool"][:, to, :m] = s["pool"][:, of, :m]
            mine[b][-1] = to
            ref[to] = 1
        while len(mine[b]) * page < lens[q] + grow[b]:
            mine[b].append(next(free))
            ref[mine[b][-1]] = 1
    out = torch.tensor([t + [-1] * (table.shape[1] - len(t)) for t in mine], dtype=torch.int32)
    return dict(pool=s["pool"], table=out, lens=torch.tensor([lens[q] + x for q, x in zip(parent, grow)], dtype=torch.int32),
                ref=torch.tensor(ref, dtype=torch.int32))


def _exact_beam(s):
    R, W = s["parent"].shape
    z, prior, eos = s["z"].double().cpu().numpy(), s["scores"].double().cpu().numpy(), s["eos"]
    z = z - z.max(1, keepdims=True)
    z = z - np.log(np.exp(z).sum(1, keepdims=True))
    parent, token, score, ended = np.zeros((R, W)), np.zeros((R, W)), np.zeros((R, W)), np.full((R, W), -np.inf)
    for i in range(R):
        best = []
        for w in range(W):
            row = prior[i, w] + z[i * W + w]
            some = np.argpartition(-row, min(2 * W, len(row) - 1))[:2 * W + 1]
            best += [(-row[t], w, int(t)) for t in some]
            if eos not in some:
                best.append((-row[eos], w, eos))
        best.sort()
        go = [x for x in best if x[2] != eos][:W]
        parent[i], token[i], score[i] = [i * W + x[1] for x in go], [x[2] for x in go], [-x[0] for x in go]
        for x in best[:W]:
            if x[2] == eos:
                ended[i, x[1]] = -x[0]
    return dict(parent=torch.from_numpy(parent).int(), token=torch.from_numpy(token).int(), scores=torch.from_numpy(score),
                ended=torch.from_numpy(ended))
