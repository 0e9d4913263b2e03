"""Answers from a KV cache with drafted tokens, rules on the logits and a cache kept within a budget.

    spd_prefill_kv       the prompt but for its last tokens (under its skip plan)
    spd_decode_tree      the window of last prompt tokens (a chain), then a tree of drafts a step
    spd_logits_process   penalties, biases and grammars on every node's logits; the best token left
    spd_tree_commit      the accepted drafts join the context
    spd_cache_weights    the attention weight that the accepted tokens gave to every cached row
    spd_cache_evict      back to the budget, per layer, sequence and K/V head

This module owns buffers and walks the trees on the host; every computation runs in the CUDA library. Drafts come from
the caller (a small model, the prompt's own n-grams). `python -m paper_2609_34977_gb300.answer` runs a small model.
"""
from __future__ import annotations

import itertools

import numpy as np
import torch

from . import _native as N


class TreeAnswer:
    """Cache, weights and host state of n_seqs answers.

    embed: bf16 [vocab][d_model]. At most max_nodes drafted tokens a sequence and step, the pending token among them. With a
    budget, a cache that has grown past it is cut back to `budget` rows after the prompt and after every step: the n_sink
    first and n_recent last positions stay, the others by the weight that they received (decay: what a step leaves of the
    total). rules: what spd_logits_process takes per sequence (repetition, frequency, presence: fp32 [n_seqs]; bias_cu,
    bias_id, bias; allow), and `rule`, a callable (sequence, generated tokens) -> row of allow or -1.

    Where a device-side wait ran out, start() and step() raise SpiderError before they take over any token, and so does every
    later call: what the cache holds is not to be relied on.
    """

    def __init__(self, model: N.SpdModel, embed, n_seqs: int, max_len: int, *, max_nodes: int = 32, budget: int | None = None,
                 n_sink: int = 4, n_recent: int = 32, decay: float = 1.0, rules: dict | None = None):
        c = self.cfg = model.cfg
        self.model, self.embed, self.B, self.max_len, self.max_nodes = model, embed, n_seqs, max_len, max_nodes
        self.budget, self.n_sink, self.n_recent, self.decay = budget, n_sink, n_recent, decay
        if budget is not None and not n_sink + n_recent <= budget <= max_len - max_nodes:
            raise ValueError("budget: needs room for sinks and recent tokens, and for a step's drafts up to max_len")
        if tuple(embed.shape) != (c["vocab"], c["d_model"]):
            raise ValueError(f"embed: {tuple(embed.shape)}, expected {(c['vocab'], c['d_model'])}")
        self.rules = dict(rules or {})
        self.rule = self.rules.pop("rule", None)
        L, G = c["n_layers"], c["n_kv_heads"]
        dev = dict(device="cuda")
        units = (L, n_seqs, G, max_len)
        self.kv = torch.zeros(L, n_seqs, max_len, 2 * G * c["head_dim"], dtype=torch.bfloat16, **dev)
        self.acc = torch.zeros(units, **dev)
        self.pos = torch.arange(max_len, dtype=torch.int32, **dev).expand(units).contiguous()
        self.lens = np.zeros(n_seqs, np.int32)
        self.next_pos = np.zeros(n_seqs, np.int32)
        self.hist = [[] for _ in range(n_seqs)]       # tokens of prompt and answer, as the penalties see them
        self.n_prompt = [0] * n_seqs
        self.pending = [None] * n_seqs                # the token that the next step begins with
        self.ws_evict = None
        if budget is not None:
            self.ws_evict = torch.zeros(N.spd_cache_evict_workspace_size(L, n_seqs, G, budget), dtype=torch.uint8, **dev)
        self._status = 0                              # the first failure of workspaces that are gone
        self._n, self.ws = 0, None
        self._room(n_seqs * max_nodes)

    def _room(self, n):
        """Buffers of a step of up to n nodes in all."""
        if n <= self._n:
            return
        self._note(self.ws)  # (it is replaced below)
        self._n = n
        c, dev = self.cfg, dict(device="cuda")
        self.logits = torch.empty(n, c["vocab"], **dev)
        self.best = torch.empty(n, dtype=torch.int32, **dev)
        self.ws = torch.zeros(N.spd_decode_tree_workspace_size(self.model, n), dtype=torch.uint8, **dev)
        self.ws_commit = torch.zeros(N.spd_tree_commit_workspace_size(self.B, n), dtype=torch.uint8, **dev)
        self.q = torch.empty(c["n_layers"] * n * c["n_heads"] * c["head_dim"], dtype=torch.bfloat16, **dev)
        self.lse = torch.empty(c["n_layers"] * n * c["n_heads"], **dev)

    def start(self, x, cu, tokens, skip_mask=None, window: int = 32):
        """The prompts: x bf16 [n][d_model] packed by cu, their tokens (ids outside the vocabulary for an image's rows) and
        skip mask [n_layers][n]. The last `window` tokens of each (text: they run every sub-layer) pass as a chain
        over the cache of the others and vote on what an eviction keeps."""
        c = self.cfg
        cu = np.asarray(cu, np.int64)
        n = np.diff(cu)
        if len(n) != self.B or n.min() < 2 or window < 1:
            raise ValueError("start: a prompt of two tokens at least for every sequence, and a window")
        self.acc.zero_()  # nothing of an earlier answer stays
        self.pos.copy_(torch.arange(self.max_len, dtype=torch.int32, device="cuda").expand(self.pos.shape))
        tail = np.minimum(window, n - 1)
        at = lambda lo, hi: np.concatenate([np.arange(a, b) for a, b in zip(lo, hi)])  # noqa: E731
        head = at(cu[:-1], cu[1:] - tail)
        hcu = np.concatenate([[0], np.cumsum(n - tail)]).astype(np.int32)
        ws = torch.zeros(N.spd_prefill_workspace_size(self.model, len(head), self.B), dtype=torch.uint8, device="cuda")
        h = torch.empty(len(head), c["d_model"], device="cuda")
        mask = None if skip_mask is None else np.ascontiguousarray(np.asarray(skip_mask)[:, head])
        xh = x.index_select(0, torch.from_numpy(head).to(x.device))
        N.spd_prefill_kv(self.model, xh, len(head), hcu, mask, h, None, self.kv, self.max_len, ws)
        self.lens[:] = n - tail
        self.next_pos[:] = n - tail
        for b in range(self.B):
            self.hist[b] = [int(t) for t in tokens[cu[b]:cu[b + 1]]]
            self.n_prompt[b] = len(self.hist[b])
        q_cu = np.concatenate([[0], np.cumsum(tail)]).astype(np.int32)
        self._room(int(q_cu[-1]))
        xt = x.index_select(0, torch.from_numpy(at(cu[1:] - tail, cu[1:])).to(x.device))
        depth = at(np.zeros_like(tail), tail)
        best = self._forward(xt, q_cu, None, depth, [[] for _ in range(len(depth))], ws)
        self._accept([list(range(k)) for k in tail], q_cu)
        self.pending = [int(best[q_cu[b + 1] - 1]) for b in range(self.B)]
        return list(self.pending)

    def step(self, drafts=None):
        """One step: the pending token of every sequence and the drafts behind it, drafts[b] = [(token, parent)] with parent 0
        the pending token and i the i-th draft. Returns the tokens that each sequence gained, at least one (a sequence whose
        rules leave no token gains -1 and ends: its next steps are empty)."""
        live = [p is not None and p >= 0 for p in self.pending]
        drafts = drafts or [[] for _ in range(self.B)]
        if any(not 0 <= t < self.cfg["vocab"] for d in drafts for t, _ in d):
            raise ValueError("drafts: a token outside the vocabulary")
        tok, parent = [], []
        for b in range(self.B):
            if not live[b]:
                tok.append([])
                parent.append([])
                continue
            if len(drafts[b]) + 1 > self.max_nodes:
                raise ValueError(f"sequence {b}: {len(drafts[b])} drafts, at most {self.max_nodes - 1}")
            tok.append([self.pending[b]] + [int(t) for t, _ in drafts[b]])
            parent.append([-1] + [int(p) for _, p in drafts[b]])
        q_cu = np.concatenate([[0], np.cumsum([len(t) for t in tok])]).astype(np.int32)
        if q_cu[-1] == 0:
            return [[] for _ in range(self.B)]
        mask, depth = N.spd_tree_mask(np.concatenate([np.asarray(p, np.int32) for p in parent]), q_cu)
        paths = []
        for t, p in zip(tok, parent):
            first = len(paths)
            for i in range(len(t)):
                paths.append((paths[first + p[i]] if p[i] >= 0 else []) + [t[i]])
        ids = torch.tensor([t for s in tok for t in s], device="cuda")
        best = self._forward(self.embed.index_select(0, ids), q_cu, torch.from_numpy(mask.view(np.int32)).cuda(), depth, paths)
        accepted, gained = [], []
        for b in range(self.B):
            path, new = [], []
            node = 0 if tok[b] else -1
            while node >= 0:  # the draft that says what the model says goes on
                path.append(node)
                self.hist[b].append(tok[b][node])
                new.append(int(best[q_cu[b] + node]))
                node = next((i for i in range(node + 1, len(tok[b])) if parent[b][i] == path[-1] and tok[b][i] == new[-1]), -1)
            accepted.append(path)
            gained.append(new)
            if new:
                self.pending[b] = new[-1]
        self._accept(accepted, q_cu)
        return gained

    def _forward(self, x, q_cu, mask, depth, paths, ws_prompt=None):
        """A pass over packed nodes; returns the best token of each after the rules (host), or raises what the device recorded."""
        c, n = self.cfg, int(q_cu[-1])
        per = np.repeat(self.next_pos, np.diff(q_cu))
        N.spd_decode_tree(self.model, x, q_cu, self.lens, per + depth, mask, self.kv, self.max_len, self.logits, self.ws,
                          q_out=self.q, lse_out=self.lse)
        seq = np.repeat(np.arange(self.B), np.diff(q_cu))
        up = lambda a: torch.tensor(np.asarray(a, np.int32), device="cuda")  # noqa: E731
        cu = lambda v: up(np.concatenate([[0], np.cumsum([len(t) for t in v])]))  # noqa: E731
        flat = lambda v: up([t for s in v for t in s])  # noqa: E731
        h_cu = np.concatenate([[0], np.cumsum([len(t) for t in self.hist])])
        kw = dict(self.rules)
        if any(k in kw for k in ("repetition", "frequency", "presence")):
            kw.update(hist=flat(self.hist), hist_cu=up(h_cu), gen_start=up(h_cu[:-1] + np.array(self.n_prompt)), path=flat(paths),
                      path_cu=cu(paths))
        if "allow" in kw:
            said = [self.hist[b][self.n_prompt[b]:] for b in range(self.B)]
            kw["rule"] = up([self.rule(int(b), said[b] + p) if self.rule else 0 for b, p in zip(seq, paths)])
        N.spd_logits_process(self.logits[:n], self.logits[:n], self.best, seq_of=up(seq), **kw)
        best = self.best[:n].cpu().numpy()
        self._note(ws_prompt)
        if self.status():
            raise N.SpiderError(self.status(), "a device-side wait of this answer ran out")
        return best

    def _accept(self, paths, q_cu):
        """Commits every sequence's accepted nodes, adds the weight they gave, and evicts back to the budget."""
        c, L = self.cfg, self.cfg["n_layers"]
        G, d, n = c["n_kv_heads"], c["head_dim"], int(q_cu[-1])
        cu = np.concatenate([[0], np.cumsum([len(p) for p in paths])]).astype(np.int32)
        N.spd_tree_commit(self.kv, L, [i for p in paths for i in p], cu, self.lens, self.max_len, G, d, self.ws_commit,
                          next_pos=self.next_pos, pos=self.pos, acc=self.acc)
        grown = np.diff(cu)
        self.lens += grown
        self.next_pos += grown
        if self.budget is None:
            return
        rows = torch.tensor([int(q_cu[b]) + i for b, p in enumerate(paths) for i in p], dtype=torch.int32, device="cuda")
        q = self.q[:L * n * c["n_heads"] * d].view(L, n, -1)
        lse = self.lse[:L * n * c["n_heads"]].view(L, n, -1)
        N.spd_cache_weights(q, lse, rows, cu, self.kv, self.lens, self.max_len, c["n_heads"], G, d, self.decay, self.acc,
                            self.acc, self.ws)
        if (self.lens > self.budget).any():
            self.lens = N.spd_cache_evict(self.kv, self.lens, self.max_len, G, d, self.budget, self.n_sink, self.n_recent,
                                          self.next_pos, self.acc, self.pos, self.acc, self.pos, None, self.ws_evict)

    def _note(self, ws):
        """Keeps a failure that a workspace holds, unless there is an earlier one."""
        if ws is not None and not self._status:
            self._status = N.spd_workspace_status(ws)

    def status(self) -> int:
        """First device-side failure recorded by prompts and steps (0 = OK; synchronises)."""
        self._note(self.ws)
        return self._status


def ngram_drafts(text, n: int, width: int = 2, vocab: int | None = None):
    """Drafts from the text so far: the continuations of the last `width` tokens' most recent earlier occurrence, as a chain
    of up to n tokens, up to the first outside the vocabulary (an image's placeholder)."""
    key = text[-width:]
    for i in range(len(text) - width - 1, -1, -1):
        if text[i:i + width] == key:
            return [(t, k) for k, t in enumerate(itertools.takewhile(lambda t: vocab is None or 0 <= t < vocab,
                                                                     text[i + width:i + width + n]))]
    return []


def main():
    from . import synth
    cfg = dict(synth.TINY_DECODER)
    w = synth.decoder_weights(1, cfg, std=0.05)
    wd = {k: v.cuda() for k, v in w.items() if k != "layers"}
    wd["layers"] = [{k: v.cuda() for k, v in lw.items()} for lw in w["layers"]]
    model = N.SpdModel(cfg, wd)
    g = torch.Generator().manual_seed(0)
    embed = torch.randn(cfg["vocab"], cfg["d_model"], generator=g).to(torch.bfloat16).cuda()
    lens = [180, 90]
    tokens = np.random.default_rng(0).integers(0, cfg["vocab"], sum(lens))
    run = TreeAnswer(model, embed, 2, 256, max_nodes=8, budget=96, n_recent=24,
                     rules=dict(frequency=torch.tensor([0.1, 0.0], device="cuda")))
    x = embed.index_select(0, torch.from_numpy(tokens).cuda())
    said = [[t] for t in run.start(x, [0, lens[0], sum(lens)], tokens)]
    steps = 0
    while min(len(s) for s in said) < 48:
        drafts = [ngram_drafts(run.hist[b] + [run.pending[b]], 5, vocab=cfg["vocab"]) for b in range(2)]
        for s, new in zip(said, run.step(drafts)):
            s.extend(new)
        steps += 1
    print(f"{[len(s) for s in said]} tokens in {steps} steps, {run.lens.tolist()} rows cached, status {run.status()}")


if __name__ == "__main__":
    main()
