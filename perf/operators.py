"""Answering from a cache with drafted tokens, and keeping the cache within a budget: the operators, in plain torch and
as this library's calls, with the sizes that are measured.

    tree     attention of drafted tokens (a tree a sequence, one token at the least) over a layer of the KV cache
    weights  the attention weight that every cached row received, added to its running total (all layers)
    evict    the rows of least weight leave the cache, per layer, sequence and K/V head (all layers)
    logits   penalties for repeated tokens, biases and grammar masks on logits, and the best token left

Cache rows are [K of every K/V head | V of every K/V head], bf16, at [layer][sequence][slot]. The shapes are those of the
repository's LLaVA-1.5 (32 heads of 128, 32000 words) and Qwen2-style decoders (28 heads on 4 of 128, 152064 words),
and a small one with heads of 64.
"""
import math

import numpy as np
import torch

own = False

BF16 = torch.bfloat16
SHAPES = {  # heads, K/V heads, head width, vocabulary
    "llava": dict(h=32, g=32, d=128, vocab=32000),
    "qwen": dict(h=28, g=4, d=128, vocab=152064),
    "small": dict(h=16, g=8, d=64, vocab=32003),
}
IMAGE_TOKEN = -200  # what a LLaVA prompt holds in the places of the image's rows
COST = 6e9          # bytes that a drawn tree case may take for its scores and weights in fp32, three copies in all


def listed():
    return [
        # the next token of one request, after an eviction (rotary position and slot differ): latency
        dict(name="tree_token", kind="tree", shape="llava", ctx="321", nodes="1", form="tree"),
        # a small decoder's window: the last 64 prompt tokens of four requests, as a chain
        dict(name="tree_window", kind="tree", shape="small", ctx="700,1131,65,2048", nodes="64,64,64,64", form="chain"),
        # a serving batch at different depths of their contexts, trees of 1 to 16 drafts
        dict(name="tree_batch", kind="tree", shape="qwen", ctx=_join(300 + 53 * i for i in range(32)),
             nodes=_join(1 + i % 16 for i in range(32)), form="tree"),
        # eight LLaVA requests with wide trees: every head has K and V of its own
        dict(name="tree_wide", kind="tree", shape="llava", ctx=_join(640 + 111 * i for i in range(8)), nodes=_join([48] * 8),
             form="tree"),
        # one long context: few rows, many keys
        dict(name="tree_long", kind="tree", shape="qwen", ctx="65521", nodes="16", form="tree"),
        # after one generated token of each of four requests, all 28 layers
        dict(name="weights_token", kind="weights", shape="qwen", layers=28, lens="2311,1801,3977,1024", rows="1,1,1,1"),
        # after the prompt: the last 32 tokens vote for what stays (LLaVA-NeXT, unpruned)
        dict(name="weights_window", kind="weights", shape="llava", layers=8, lens="3008", rows="32"),
        # eight requests a few accepted tokens over their budget, all 28 layers
        dict(name="evict_step", kind="evict", shape="qwen", layers=28, lens="1029,1030,1025,1031,1024,1028,1029,1027", budget=1024),
        # the prompt's cache cut to a third after the prefill
        dict(name="evict_prompt", kind="evict", shape="llava", layers=8, lens="3008", budget=1024),
        # one request's next token
        dict(name="logits_token", kind="logits", shape="llava", seqs=1, nodes=1, hist=700, bias=16),
        # a serving batch of 64 requests, half of them under a grammar
        dict(name="logits_batch", kind="logits", shape="qwen", seqs=64, nodes=1, hist=4000, bias=64),
        # every node of eight trees, each with the drafts on its path as further history
        dict(name="logits_tree", kind="logits", shape="qwen", seqs=8, nodes=24, hist=2000, bias=300),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _join(v):
    return ",".join(str(int(x)) for x in v)


def _ints(s):
    return [int(v) for v in str(s).split(",")]


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "weights", "evict", "logits"])
    shape = rng.choice(["llava", "qwen", "qwen", "small"])
    if kind == "logits":
        seqs = _log(rng, 1, 64)
        return dict(kind=kind, shape=shape, seqs=seqs, nodes=_log(rng, 1, max(1, 192 // seqs)), hist=_log(rng, 1, 8000),
                    bias=_log(rng, 1, 300))
    c = SHAPES[shape]
    b = _log(rng, 1, 32)
    if kind == "tree":
        most = max(64, int(COST / 3 / (4 * b * c["h"] * 32)))  # keys a sequence that keep the scores within COST / 3
        ctx = [_log(rng, 1, min(65521, most, 180000 // b if shape == "qwen" else 24000 // b)) for _ in range(b)]
        top = rng.choice([1, 8, 24, 64])
        return dict(kind=kind, shape=shape, ctx=_join(ctx), nodes=_join(_log(rng, 1, top) for _ in range(b)),
                    form=rng.choice(["tree", "tree", "chain"]))
    b = min(b, 8)
    layers = _log(rng, 1, 28)
    slots = max(64, int((6e8 if kind == "evict" else 4e8) / (layers * b * 4 * c["g"] * c["d"])))  # a cache of 0.6 GB at most
    lens = [_log(rng, 40, min(slots, 16000)) for _ in range(b)]
    if kind == "weights":
        top = rng.choice([1, 4, 32])
        return dict(kind=kind, shape=shape, layers=layers, lens=_join(lens), rows=_join(_log(rng, 1, top) for _ in range(b)))
    return dict(kind=kind, shape=shape, layers=layers, lens=_join(lens), budget=_log(rng, 20, max(lens)))


# ---- inputs -----------------------------------------------------------------------------------
def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt) % (1 << 62))


def _randn(shape, g, std=1.0, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype).mul_(std)


def _cu(v):
    return np.concatenate([[0], np.cumsum(v)]).astype(np.int32)


def _tree(r, n, form):
    """Which drafts each of n nodes sees: itself and its ancestors; a later node hangs under any earlier one."""
    see = np.eye(n, dtype=bool)
    for i in range(1, n):
        see[i] |= see[i - 1 if form == "chain" else r.integers(0, i)]
    return see


def _bits(see, words):
    """Rows of booleans as int32 words, bit j of word w for entry 32 w + j."""
    full = np.zeros((see.shape[0], 32 * words), np.uint8)
    full[:, :see.shape[1]] = see
    return torch.from_numpy(np.packbits(full, axis=1, bitorder="little").view(np.int32).copy()).cuda()


def _cache(c, seed, layers, seqs, slots):
    """Recycled cache memory: every slot holds finite rows, those past a sequence's length of somebody else."""
    return _randn((layers, seqs, slots, 2 * c["g"] * c["d"]), _gen(seed, 1), 1.0, BF16)


def prepare(case, seed):
    k, c = case["kind"], SHAPES[case["shape"]]
    g, r = _gen(seed, 2), np.random.default_rng(seed)
    e = lambda shape, dt: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
    s = dict(case=case, c=c)
    if k == "tree":
        ctx, nodes = _ints(case["ctx"]), _ints(case["nodes"])
        b, n, words = len(ctx), sum(nodes), (max(nodes) + 31) // 32
        slots = max(x + y for x, y in zip(ctx, nodes)) + 5
        return dict(s, ctx=np.array(ctx, np.int32), q_cu=_cu(nodes), slots=slots,
                    mask=torch.cat([_bits(_tree(r, m, case["form"]), words) for m in nodes]),
                    q=_randn((n, c["h"] * c["d"]), g, 2.5, BF16), kv=_cache(c, seed, 1, b, slots)[0],
                    o=e((n, c["h"] * c["d"]), BF16), lse=e((n, c["h"]), torch.float32), ws=e(64 << 20, torch.uint8))
    if k == "weights":
        lens, rows = _ints(case["lens"]), _ints(case["rows"])
        b, n, slots, L = len(lens), sum(rows), max(lens) + 3, case["layers"]
        kv = _cache(c, seed, L, b, slots)
        q = _randn((L, n + 2, c["h"] * c["d"]), g, 2.5, BF16)
        pick = torch.from_numpy(np.sort(r.permutation(n + 2)[:n]).astype(np.int32)).cuda()  # two drafts were not accepted
        s.update(lens=np.array(lens, np.int32), rows_cu=_cu(rows), slots=slots, q=q, kv=kv, pick=pick)
        lse = 1.0 + math.log(max(lens)) + 2.0 * torch.rand((L, n + 2, c["h"]), generator=g, device="cuda")
        acc = torch.rand((L, b, c["g"], slots), generator=g, device="cuda")
        return dict(s, lse=lse, acc=acc, acc_out=torch.zeros_like(acc), decay=0.98)
    if k == "evict":
        lens, L = _ints(case["lens"]), case["layers"]
        b, slots, bud = len(lens), max(_ints(case["lens"])) + 9, case["budget"]
        n = (L, b, c["g"], slots)
        pos = torch.argsort(torch.rand(n, generator=g, device="cuda"), -1).int()  # earlier evictions left no order
        return dict(s, lens=np.array(lens, np.int32), slots=slots, kv=_cache(c, seed, L, b, slots), sink=min(4, bud // 4),
                    recent=bud // 4, next_pos=np.full(b, slots, np.int32), acc=torch.exp(2.0 * _randn(n, g)), pos=pos,
                    acc_out=e(n, torch.float32), pos_out=e(n, torch.int32), src=e((L, b, c["g"], bud), torch.int32),
                    ws=e(4 * L * b * c["g"] * (2 * bud + 64) + 4096, torch.uint8))
    seqs, nodes, v = case["seqs"], case["nodes"], c["vocab"]
    n, words = seqs * nodes, (v + 31) // 32
    lens = [max(1, case["hist"] * (i + 1) // seqs) for i in range(seqs)]
    hist = (v * r.random(sum(lens)) ** 3).astype(np.int32)  # few words make up most of a text
    h_cu = _cu(lens)
    gen = h_cu[:-1] + np.array([x // 2 for x in lens], np.int32)
    for i in range(seqs):  # a fifth of the history is the image
        hist[h_cu[i]:h_cu[i] + lens[i] // 5] = IMAGE_TOKEN
    path = [r.integers(0, v, i % 6 if nodes > 1 else 0) for i in range(n)]
    ids = [np.sort(r.choice(v, case["bias"], replace=False)) for _ in range(seqs)]
    allow = r.random((4, v)) < np.array([0.002, 0.05, 0.5, 0.9])[:, None]
    allow[:, v // 3] = True
    t = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).cuda()  # noqa: E731
    return dict(s, z=_randn((n, v), g, 3.0), seq_of=t(np.arange(n) // nodes, np.int32), hist=t(hist, np.int32),
                hist_cu=t(h_cu, np.int32), gen=t(gen, np.int32), path=t(np.concatenate(path), np.int32),
                path_cu=t(_cu([len(p) for p in path]), np.int32), rep=t(r.uniform(1.0, 1.4, seqs), np.float32),
                freq=t(r.uniform(0.0, 0.4, seqs), np.float32), pres=t(r.uniform(0.0, 0.6, seqs), np.float32),
                bias_cu=t(_cu([len(x) for x in ids]), np.int32), bias_id=t(np.concatenate(ids), np.int32),
                bias=t(3.0 * r.standard_normal(seqs * case["bias"]), np.float32), allow=_bits(allow, words),
                rule=t(np.where(np.arange(n) % 2 == 1, np.arange(n) // 2 % 4, -1), np.int32),
                out=e((n, v), torch.float32), best=e(n, torch.int32))


# ---- the library's calls ----------------------------------------------------------------------
def _run_own(s):
    from paper_2609_34977_gb300 import _native as N
    k, c = s["case"]["kind"], s["c"]
    if k == "tree":
        N.spd_tree_attention(s["q"], s["q_cu"], s["ctx"], s["mask"], s["kv"], s["slots"], c["h"], c["g"], c["d"], s["o"],
                             s["lse"], s["ws"])
        return dict(o=s["o"], lse=s["lse"])
    if k == "weights":
        N.spd_cache_weights(s["q"], s["lse"], s["pick"], s["rows_cu"], s["kv"], s["lens"], s["slots"], c["h"], c["g"], c["d"],
                            s["decay"], s["acc"], s["acc_out"])
        return s["acc_out"]
    if k == "evict":
        N.spd_cache_evict(s["kv"], s["lens"], s["slots"], c["g"], c["d"], s["case"]["budget"], s["sink"], s["recent"],
                          s["next_pos"], s["acc"], s["pos"], s["acc_out"], s["pos_out"], s["src"], s["ws"])
        return dict(kv=s["kv"], acc=s["acc_out"], pos=s["pos_out"], src=s["src"])
    N.spd_logits_process(s["z"], s["out"], s["best"], seq_of=s["seq_of"], hist=s["hist"], hist_cu=s["hist_cu"],
                         gen_start=s["gen"], path=s["path"], path_cu=s["path_cu"], repetition=s["rep"], frequency=s["freq"],
                         presence=s["pres"], bias_cu=s["bias_cu"], bias_id=s["bias_id"], bias=s["bias"], allow=s["allow"],
                         rule=s["rule"])
    return dict(logits=s["out"], best=s["best"])


# ---- the plain forms --------------------------------------------------------------------------
def _dev(a):
    return torch.as_tensor(np.asarray(a, np.int64), device="cuda")


def _unpack(words, n):
    """int32 words -> booleans [.., n]."""
    bits = (words[..., None] >> torch.arange(32, device="cuda", dtype=torch.int32)) & 1
    return bits.flatten(-2)[..., :n].bool()


def _padded(cu):
    """Row index [seq][row] of packed rows and which entries are real."""
    cu = _dev(cu)
    i = torch.arange(int((cu[1:] - cu[:-1]).max()), device="cuda")
    real = i[None] < (cu[1:] - cu[:-1])[:, None]
    return torch.where(real, cu[:-1, None] + i[None], 0), real


def _plain_tree(s):
    c = s["c"]
    h, g, d = c["h"], c["g"], c["d"]
    rows, real = _padded(s["q_cu"])
    b, n = rows.shape
    ctx = _dev(s["ctx"])
    keys = min(s["slots"], int(s["ctx"].max()) + n)
    kv = s["kv"][:, :keys].float().view(b, keys, 2, g, d)
    q = s["q"].float().view(-1, g, h // g, d)[rows]                            # [b][n][g][m][d]
    score = torch.einsum("bngmd,bkgd->bgmnk", q, kv[:, :, 0]) / math.sqrt(d)
    draft = torch.arange(keys, device="cuda")[None] - ctx[:, None]             # [b][k]: which draft a slot holds
    seen = torch.gather(_unpack(s["mask"], 32 * s["mask"].shape[1])[rows], 2,
                        draft.clamp(0, 32 * s["mask"].shape[1] - 1)[:, None].expand(b, n, keys))
    nodes = real.sum(1)
    seen = (draft < 0)[:, None] | (seen & (draft >= 0)[:, None] & (draft[:, None] < nodes[:, None, None]))
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    w = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    o = torch.einsum("bgmnk,bkgd->bngmd", w / torch.where(total == 0, 1.0, total), kv[:, :, 1])
    lse = (torch.log(total) + top)[..., 0].permute(0, 3, 1, 2)
    return dict(o=o[real].reshape(-1, h * d).to(BF16), lse=lse[real].reshape(-1, h))


def _plain_weights(s):
    c = s["c"]
    h, g, d = c["h"], c["g"], c["d"]
    rows, real = _padded(s["rows_cu"])
    lens = _dev(s["lens"])
    L, b, n = s["q"].shape[0], *rows.shape
    at = s["pick"].long()[rows]
    q = s["q"].float().view(L, -1, g, h // g, d)[:, at]                        # [L][b][n][g][m][d]
    lse = s["lse"].view(L, -1, g, h // g)[:, at]
    key = s["kv"][..., :g * d].float().view(L, b, s["slots"], g, d)
    score = torch.einsum("lbngmd,lbkgd->lbgmnk", q, key) / math.sqrt(d)
    slot = torch.arange(s["slots"], device="cuda")
    see = (lens - real.sum(1))[:, None] + torch.arange(n, device="cuda")[None] + 1
    seen = (slot[None, None] < see[:, :, None]) & real[:, :, None]             # [b][n][k]
    w = torch.exp(score - lse.permute(0, 1, 3, 4, 2)[..., None]).masked_fill(~seen[None, :, None, None], 0.0)
    new = s["decay"] * s["acc"] + w.sum((3, 4))
    return new.masked_fill(slot[None] >= lens[:, None, None], 0.0)


def _plain_evict(s):
    c, bud = s["c"], s["case"]["budget"]
    L, b, g, slots = s["acc"].shape
    lens, slot = _dev(s["lens"]), torch.arange(slots, device="cuda")
    live = (slot[None] < lens[:, None])[None, :, None]                         # [1][b][1][slots]
    keep = torch.minimum(lens, torch.full_like(lens, bud))[None, :, None, None]
    held = (s["pos"] < s["sink"]) | (s["pos"] >= (_dev(s["next_pos"]) - s["recent"])[None, :, None, None])
    rank = torch.where(torch.isnan(s["acc"]), -math.inf, s["acc"])
    order = torch.argsort(rank, dim=-1, descending=True, stable=True)              # by weight, then by slot
    cls = torch.where(live, torch.where(held, 0, 1), 2).expand_as(rank)
    byslot = torch.where(torch.gather(cls, -1, order) == 1, 1, 2)              # the unprotected by weight, others after
    order = torch.gather(order, -1, torch.argsort(byslot, dim=-1, stable=True))
    place = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order).contiguous())
    n_held = ((cls == 0) * 1).sum(-1, keepdim=True)
    place = torch.where(cls == 0, torch.cumsum((cls == 0) * 1, -1) - 1, place + n_held)
    kept = (place < keep) & live
    hole, fill = ~kept & (slot < keep), kept & (slot >= keep)
    spare = torch.where(fill, torch.cumsum(fill * 1, -1) - 1, slots)           # j-th kept row past the budget
    fills = torch.zeros((L, b, g, slots + 1), dtype=torch.int64, device="cuda").scatter_(-1, spare, slot.expand_as(spare).contiguous())
    src = torch.where(hole, torch.gather(fills, -1, (torch.cumsum(hole * 1, -1) - 1).clamp(min=0)), slot)
    src = torch.where(slot < keep, src, slot)
    acc = torch.where(slot < keep, torch.gather(s["acc"], -1, src), 0.0)
    pos = torch.where(slot < keep, torch.gather(s["pos"], -1, src), torch.where(live, -1, 0).int())
    m = min(bud, slots)
    part = s["kv"].view(L, b, slots, 2, g, c["d"])
    at = src[..., :m].permute(0, 1, 3, 2)[:, :, :, None, :, None].expand(L, b, m, 2, g, c["d"])
    part[:, :, :m] = torch.gather(part, 2, at)
    whole = torch.zeros((L, b, g, bud), dtype=torch.int32, device="cuda")
    whole[..., :m] = torch.where(slot < keep, src, 0)[..., :m].int()
    return dict(kv=s["kv"], acc=acc, pos=pos.int(), src=whole)


def _plain_logits(s):
    z = s["z"]
    n, v = z.shape
    seqs = len(s["rep"])
    seq = s["seq_of"].long()
    i = torch.arange(len(s["hist"]), device="cuda")
    of = torch.searchsorted(s["hist_cu"][1:].contiguous(), i.int(), right=True)
    tok = s["hist"].long()
    fine = (tok >= 0) & (tok < v)
    new = i >= s["gen"].long()[of]
    seen = torch.zeros((seqs, v), device="cuda").index_put_((of, tok.clamp(0, v - 1)), fine * 1.0, accumulate=True)
    made = torch.zeros((seqs, v), device="cuda").index_put_((of, tok.clamp(0, v - 1)), (fine & new) * 1.0, accumulate=True)
    row = torch.searchsorted(s["path_cu"][1:].contiguous(), torch.arange(len(s["path"]), device="cuda").int(), right=True)
    on = torch.zeros((n, v), device="cuda").index_put_((row, s["path"].long()), torch.ones(len(s["path"]), device="cuda"),
                                                       accumulate=True)
    seen, made = seen[seq] + on, made[seq] + on
    rep, freq, pres = (s[k][seq][:, None] for k in ("rep", "freq", "pres"))
    x = torch.where(seen > 0, torch.where(z > 0, z / rep, z * rep), z)
    x = torch.where(made > 0, x - freq * made - pres, x)
    of = torch.searchsorted(s["bias_cu"][1:].contiguous(), torch.arange(len(s["bias"]), device="cuda").int(), right=True)
    add = torch.zeros((seqs, v), device="cuda").index_put_((of, s["bias_id"].long()), s["bias"], accumulate=True)
    x = x + add[seq]
    allowed = _unpack(s["allow"], v)[s["rule"].long().clamp(min=0)] | (s["rule"] < 0)[:, None]
    x = torch.where(allowed, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    first = torch.where(x == top, torch.arange(v, device="cuda"), v).amin(-1)
    return dict(logits=x, best=torch.where(top[:, 0] == -math.inf, -1, first).int())


def run(s):
    if own:
        return _run_own(s)
    return dict(tree=_plain_tree, weights=_plain_weights, evict=_plain_evict, logits=_plain_logits)[s["case"]["kind"]](s)


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    k, c = case["kind"], SHAPES[case["shape"]]
    h, g, d = c["h"], c["g"], c["d"]
    if k == "tree":
        ctx, nodes = _ints(case["ctx"]), _ints(case["nodes"])
        n, keys = sum(nodes), sum(ctx) + sum(nodes)
        return dict(bytes=4 * g * d * keys + 4 * n * h * d + 4 * n * h + n * ((max(nodes) + 31) // 32) * 4,
                    flops=4 * h * d * sum(x * y + y for x, y in zip(ctx, nodes)))
    if k == "weights":
        lens, rows, L = _ints(case["lens"]), _ints(case["rows"]), case["layers"]
        return dict(bytes=L * (sum(lens) * g * (2 * d + 8) + sum(rows) * h * (2 * d + 4)),
                    flops=L * 2 * h * d * sum(x * y for x, y in zip(lens, rows)))
    if k == "evict":
        # on average as many kept rows lie past the budget as its share of the length says
        lens, L, bud = _ints(case["lens"]), case["layers"], case["budget"]
        rows = sum(min(x, bud) for x in lens)
        moved = sum(max(0, x - bud) * bud / x for x in lens)
        return dict(bytes=L * g * (8 * sum(lens) + 8 * sum(lens) + 4 * rows + moved * 8 * d), flops=0)
    n, v = case["seqs"] * case["nodes"], c["vocab"]
    hist = sum(max(1, case["hist"] * (i + 1) // case["seqs"]) for i in range(case["seqs"]))
    return dict(bytes=8 * n * v + 4 * hist + 8 * case["seqs"] * case["bias"] + v // 2, flops=0)


# ---- the definitions in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    h, g, d = c["h"], c["g"], c["d"]
    m = h // g
    if case["kind"] == "tree":
        o, lse = [], []
        for b, n_ctx in enumerate(s["ctx"].tolist()):
            lo, hi = int(s["q_cu"][b]), int(s["q_cu"][b + 1])
            n = hi - lo
            sees = np.unpackbits(s["mask"][lo:hi].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)
            sees = torch.from_numpy(np.concatenate([np.ones((n, n_ctx), bool), sees], 1)).cuda()
            rows_o, rows_l = [], []
            for head in range(h):
                k = s["kv"][b, :n_ctx + n, (head // m) * d:(head // m + 1) * d].double()
                v = s["kv"][b, :n_ctx + n, (g + head // m) * d:(g + head // m + 1) * d].double()
                x = s["q"][lo:hi, head * d:(head + 1) * d].double() @ k.T * d ** -0.5
                x[~sees] = -math.inf
                rows_l.append(torch.logsumexp(x, 1))
                rows_o.append(torch.exp(x - rows_l[-1][:, None]) @ v)
            o.append(torch.cat(rows_o, 1))
            lse.append(torch.stack(rows_l, 1))
        return dict(o=torch.cat(o), lse=torch.cat(lse))
    if case["kind"] == "weights":
        out = torch.zeros(s["acc"].shape, dtype=torch.float64, device="cuda")
        for l in range(case["layers"]):
            for b, n in enumerate(s["lens"].tolist()):
                rows = s["pick"][int(s["rows_cu"][b]):int(s["rows_cu"][b + 1])].long()
                q, z = s["q"][l][rows].double(), s["lse"][l][rows].double()
                for head in range(h):
                    k = s["kv"][l, b, :n, (head // m) * d:(head // m + 1) * d].double()
                    w = torch.exp(q[:, head * d:(head + 1) * d] @ k.T * d ** -0.5 - z[:, head, None])
                    last = torch.arange(n - len(rows), n, device="cuda")[:, None]
                    out[l, b, head // m, :n] += torch.where(torch.arange(n, device="cuda")[None] <= last, w, 0.0).sum(0)
                out[l, b, :, :n] += s["decay"] * s["acc"][l, b, :, :n].double()
        return out
    if case["kind"] == "evict":
        kv = s["kv"].cpu().view(torch.int16).numpy().reshape(*s["kv"].shape[:3], 2, g, d)
        acc, pos = s["acc"].cpu().numpy(), s["pos"].cpu().numpy()
        acc_out, pos_out, src_out = np.zeros_like(acc), np.zeros_like(pos), np.zeros(s["src"].shape, np.int32)
        for l, b, u in np.ndindex(acc.shape[:3]):
            n = int(s["lens"][b])
            w, p = acc[l, b, u, :n].astype(np.float64), pos[l, b, u, :n]
            held = (p < s["sink"]) | (p >= s["next_pos"][b] - s["recent"])
            best = np.lexsort((np.arange(n), np.where(held, 0.0, -w), ~held))
            take = min(n, case["budget"])
            kept = np.sort(best[:take])
            src = np.arange(take)
            src[np.setdiff1d(src, kept)] = kept[kept >= take]
            kv[l, b, :take, :, u] = kv[l, b, src, :, u]
            acc_out[l, b, u, :take], pos_out[l, b, u, :take], pos_out[l, b, u, take:n] = acc[l, b, u, src], pos[l, b, u, src], -1
            src_out[l, b, u, :take] = src
        out = torch.from_numpy(kv.reshape(s["kv"].shape)).view(BF16)
        return dict(kv=out, acc=torch.from_numpy(acc_out).double(), pos=torch.from_numpy(pos_out), src=torch.from_numpy(src_out))
    z = s["z"].double().cpu().numpy()
    n, v = z.shape
    hist, h_cu, path, p_cu = (s[k].cpu().numpy() for k in ("hist", "hist_cu", "path", "path_cu"))
    b_cu, ids, bias, rule = (s[k].cpu().numpy() for k in ("bias_cu", "bias_id", "bias", "rule"))
    allow = np.unpackbits(s["allow"].cpu().numpy().view(np.uint8), axis=1, bitorder="little")[:, :v].astype(bool)
    best = np.full(n, -1, np.int32)
    for i in range(n):
        b = int(s["seq_of"][i])
        own_path = path[p_cu[i]:p_cu[i + 1]]
        text, new = hist[h_cu[b]:h_cu[b + 1]], hist[int(s["gen"][b]):h_cu[b + 1]]
        ok = lambda t: t[(t >= 0) & (t < v)]  # noqa: E731
        made = np.bincount(np.concatenate([ok(new), own_path]), minlength=v)
        seen = made + np.bincount(ok(text), minlength=v) > 0
        rep, freq, pres = (float(s[k][b]) for k in ("rep", "freq", "pres"))
        z[i] = np.where(seen, np.where(z[i] > 0, z[i] / rep, z[i] * rep), z[i]) - freq * made - pres * (made > 0)
        np.add.at(z[i], ids[b_cu[b]:b_cu[b + 1]], bias[b_cu[b]:b_cu[b + 1]])
        if rule[i] >= 0:
            z[i][~allow[rule[i]]] = -np.inf
        best[i] = np.argmax(z[i])
    return dict(logits=torch.from_numpy(z), best=torch.from_numpy(best))
