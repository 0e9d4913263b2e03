"""Beam search over a paged cache.

    spd_pages_update   room for the next rows; the pages of the beams that go on, fork or end
    spd_decode_paged   chunks of the prompts, then a token of every beam, over the pages
    spd_beam_select    the best continuations of every request's beams, and the ends among them
    spd_pages_compact  the pages in use to the front of the pool (on demand)

This module owns buffers and keeps the texts; every computation runs in the CUDA library. A request's beams have the same
length, so the host keeps the lengths. A step ends with a look at what the device recorded, and waits for it.
`python -m paper_2609_34977_gb300.beams` runs a small model.
"""
from __future__ import annotations

import numpy as np
import torch

from . import _native as N


def select_workspace_size(n_seqs: int, n_beams: int, vocab: int) -> int:
    """Workspace bytes of both selections of a search: of the prompts, a row a request, and of the beams. (One row of a request may be
    cut into more slices than its beams have together.)"""
    return max(N.spd_beam_select_workspace_size(n_seqs, n_in, n_beams, vocab) for n_in in (1, n_beams))


class BeamAnswer:
    """Cache, tables and texts of n_seqs requests with n_beams beams each.

    embed: bf16 [vocab][d_model]. The pool has n_pages pages of page_size rows, a sequence at most max_pages of them. eos: the token
    that ends an answer (-1: none). axis: the axis of every rotary pair (host uint8 [head_dim / 2]) where positions have several.
    Prompts pass in chunks of up to `chunk` tokens a request.

    Where the pool is too small, or a device-side wait ran out, the call that meets it raises SpiderError before it takes over a token or
    an ended answer, and so does every later call but status(): what the cache holds is not to be relied on.
    """

    def __init__(self, model: N.SpdModel, embed, n_seqs: int, n_beams: int, *, n_pages: int, max_pages: int, page_size: int = 64,
                 eos: int = -1, axis=None, chunk: int = 512):
        c = self.cfg = model.cfg
        self.model, self.embed, self.R, self.W, self.eos, self.axis, self.chunk = model, embed, n_seqs, n_beams, eos, axis, chunk
        if tuple(embed.shape) != (c["vocab"], c["d_model"]):
            raise ValueError(f"embed: {tuple(embed.shape)}, expected {(c['vocab'], c['d_model'])}")
        if n_seqs < 1 or n_beams < 1 or chunk < 1:
            raise ValueError("a request, a beam and a token a chunk at least")
        dev = dict(device="cuda")
        i32 = dict(dtype=torch.int32, **dev)
        B = n_seqs * n_beams
        self.pool = torch.zeros(c["n_layers"], n_pages, page_size, 2 * c["n_kv_heads"] * c["head_dim"], dtype=torch.bfloat16, **dev)
        self.ref = torch.zeros(n_pages, **i32)
        # tables and lengths before and after an update take turns; the requests' own (one sequence each) until the beams fork
        self.tables = [torch.full((B, max_pages), -1, **i32) for _ in range(2)]
        self.rows = [torch.zeros(B, **i32) for _ in range(2)]
        self.now, self.B = 0, n_seqs
        self.room = max_pages * page_size  # rows that a table holds
        self.used = torch.zeros(1, **i32)
        self.ws_pages = torch.zeros(N.spd_pages_workspace_size(n_pages, B), dtype=torch.uint8, **dev)
        self.ws_beam = torch.zeros(select_workspace_size(n_seqs, n_beams, c["vocab"]), dtype=torch.uint8, **dev)
        self.logits = torch.empty(B, c["vocab"], **dev)
        self.parent, self.token = torch.zeros(n_seqs, n_beams, **i32), torch.zeros(n_seqs, n_beams, **i32)
        self.scores = torch.zeros(n_seqs, n_beams, **dev)
        self.ended = torch.zeros(n_seqs, n_beams, **dev)
        self.first = (torch.arange(n_seqs, **i32) * n_beams)[:, None]
        self.ws, self._n, self._status = None, 0, 0
        self.lens = np.zeros(n_seqs, np.int32)
        self.texts = torch.zeros(B, 0, **i32)          # the tokens of every beam
        self.answers = [[] for _ in range(n_seqs)]     # ended ones: (score, tokens)

    def _update(self, parent, grow):
        """The sequences that go on, and room for grow[b] more rows each."""
        old, new = self.now, 1 - self.now
        n_in, n_out = self.B, len(grow)
        N.spd_pages_update(self.pool, self.cfg["n_kv_heads"], self.cfg["head_dim"], self.ref, self.tables[old][:n_in],
                           self.rows[old][:n_in], parent, torch.tensor(grow, dtype=torch.int32, device="cuda"), self.ref,
                           self.tables[new][:n_out], self.rows[new][:n_out], self.ws_pages)
        self.now, self.B = new, n_out

    def _pass(self, x, new, lens, pos, table, prefix=None):
        """A pass over new[b] more tokens of every sequence of the table; logits of their last ones."""
        n, B = int(np.sum(new)), len(new)
        if n > self._n or self.ws is None:
            self._note(self.ws)
            self._n = n
            size = N.spd_decode_paged_workspace_size(self.model, n, self.R * self.W)
            self.ws = torch.zeros(size, dtype=torch.uint8, device="cuda")
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        N.spd_decode_paged(self.model, x, cu, lens, pos, table, self.pool, self.logits[:B], self.ws,
                           axis=self.axis, prefix=prefix)

    def start(self, x, cu, pos=None, prefix=None):
        """The prompts: x bf16 [n][d_model] packed by cu; pos int32 [axes][n] (host or device; None: 0, 1, ... of every request);
        prefix: leading rows of every request that see one another (an image), or None. The first tokens are chosen."""
        self._raise()
        cu = np.asarray(cu, np.int64)
        n = np.diff(cu)
        if len(n) != self.R or n.min() < 1 or cu[0] != 0 or cu[-1] > len(x):
            raise ValueError(f"start: a prompt for every request, packed from 0, in {len(x)} rows")
        if n.max() >= self.room:
            raise ValueError(f"start: a prompt of {n.max()} tokens and the first one behind it, a table holds {self.room} rows")
        axes = 1 if pos is None else len(pos)
        host = np.concatenate([np.arange(k) for k in n])[None] if pos is None else np.asarray(torch.as_tensor(pos).cpu())
        if host.shape != (axes, cu[-1]):
            raise ValueError(f"pos: shape {host.shape}, expected {(axes, int(cu[-1]))}")
        if prefix is not None:
            prefix = np.asarray(prefix, np.int64)
            if prefix.shape != n.shape or (prefix < 0).any() or (prefix > n).any():
                raise ValueError("prefix: a number of a prompt's rows for every request")
        self.axes = axes
        self.next_pos = np.array([host[:, a:b].max() + 1 for a, b in zip(cu[:-1], cu[1:])])
        # (an image's rows must be there before they see one another: a prefix passes as one chunk)
        first = np.maximum(self.chunk, 0 if prefix is None else prefix)
        done = np.zeros(self.R, np.int64)
        self.B, self.lens[:] = self.R, 0
        self.ref.zero_()
        self.rows[self.now].zero_()
        self.answers = [[] for _ in range(self.R)]
        self.texts = torch.zeros(self.R, 0, dtype=torch.int32, device="cuda")
        logits = torch.empty(self.R, self.cfg["vocab"], device="cuda")
        while (done < n).any():
            step = np.minimum(np.where(done == 0, first, self.chunk), n - done)
            self._update(None, step.tolist())
            live = np.flatnonzero(step)
            at = np.concatenate([np.arange(cu[b] + done[b], cu[b] + done[b] + step[b]) for b in live])
            done += step
            idx = torch.from_numpy(at).cuda()
            table = self.tables[self.now][:self.R]
            if len(live) < self.R:  # (a pass takes at least one token of every sequence that it is given)
                table = table[torch.from_numpy(live).cuda()].contiguous()
            there = np.ascontiguousarray(host[:, at], dtype=np.int32)  # (columns picked by numpy lie one after the other)
            self._pass(x.index_select(0, idx.to(x.device)), step[live], done[live], torch.from_numpy(there).cuda(), table,
                       None if prefix is None else prefix[live])
            logits[torch.from_numpy(live).cuda()] = self.logits[:len(live)]
        self.lens[:] = n
        self._select(logits, torch.zeros(self.R, 1, device="cuda"), torch.arange(self.R, dtype=torch.int32, device="cuda")[:, None])

    def _select(self, logits, scores, spare):
        """The beams' next tokens, and the pages of those that go on; spare: what a beam without a candidate stands in for (its score
        is -inf, and stays so). Raises what the device recorded before anything is taken over."""
        n_in = scores.shape[1]
        ended = self.ended[:, :n_in].contiguous()
        new = torch.empty_like(self.scores)
        N.spd_beam_select(logits, scores, self.eos, self.parent, self.token, new, ended, self.ws_beam)
        none = self.parent < 0
        parent = torch.where(none, spare.expand_as(self.parent), self.parent).flatten()
        token = torch.where(none, 0, self.token).flatten()
        self._update(parent, [1] * (self.R * self.W))
        self._check()
        if self.eos >= 0:
            over = ended.cpu().numpy()
            if np.isfinite(over).any():
                texts = self.texts.cpu().numpy().reshape(self.R, n_in, -1)
                for b, w in zip(*np.nonzero(np.isfinite(over))):
                    self.answers[b].append((float(over[b, w]), texts[b, w].tolist()))
        self.texts = torch.cat([self.texts.index_select(0, parent), token[:, None]], 1)
        self.scores = new
        self.lens += 1

    def step(self):
        """One token of every beam. Refused where a table has no row for it; the answers so far stay."""
        self._begun()
        if self.lens.max() >= self.room:
            raise N.SpiderError(N.SPD_EINVAL, f"a table holds {self.room} rows")
        pos = np.repeat(self.next_pos, self.W).astype(np.int32)
        x = self.embed.index_select(0, self.texts[:, -1])
        self._pass(x, np.ones(self.R * self.W, np.int32), np.repeat(self.lens, self.W),
                   torch.from_numpy(np.tile(pos, (self.axes, 1))).cuda(), self.tables[self.now])
        self._select(self.logits, self.scores, self.first)
        self.next_pos += 1

    def compact(self) -> int:
        """Moves the pages in use to the front of the pool; returns their number (synchronises)."""
        self._raise()
        t = self.tables[self.now][:self.B]
        N.spd_pages_compact(self.pool, self.cfg["n_kv_heads"], self.cfg["head_dim"], self.ref, t, self.ref, t, self.used, self.ws_pages)
        self._check()
        return int(self.used)

    def best(self, penalty: float = 0.0):
        """Every request's answers, ended or not, best first: (score / length ** penalty, tokens)."""
        self._begun()
        scores, texts = self.scores.cpu().numpy(), self.texts.cpu().numpy().reshape(self.R, self.W, -1)
        out = []
        for b in range(self.R):
            all_ = self.answers[b] + [(float(s), t.tolist()) for s, t in zip(scores[b], texts[b]) if np.isfinite(s)]
            out.append(sorted(((s / max(1, len(t)) ** penalty, t) for s, t in all_), key=lambda a: -a[0]))
        return out

    def _note(self, ws):
        """Keeps a failure that a workspace holds, unless there is an earlier one."""
        if ws is not None and not self._status:
            self._status = N.spd_workspace_status(ws)

    def _raise(self):
        """Raises a failure that is known."""
        if self._status:
            raise N.SpiderError(self._status, "the pool has no page left" if self._status == N.SPD_ENOSPC
                                else "a device-side failure of this answer")

    def _begun(self):
        self._raise()
        if self.texts.shape[1] == 0:
            raise ValueError("the prompts have not passed: start() first")

    def _check(self):
        self.status()
        self._raise()

    def status(self) -> int:
        """First device-side failure recorded (0 = OK; synchronises)."""
        for ws in (self.ws_pages, self.ws, self.ws_beam):
            self._note(ws)
        return self._status


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
    tokens = torch.randint(0, cfg["vocab"], (sum(lens),), generator=g).cuda()
    run = BeamAnswer(model, embed, 2, 4, n_pages=96, max_pages=16, page_size=16, eos=3, chunk=64)
    run.start(embed.index_select(0, tokens), [0, lens[0], sum(lens)])
    for _ in range(31):
        run.step()
    pages = run.compact()
    print(f"{run.texts.shape[1]} tokens a beam, {pages} pages in use, {[len(a) for a in run.answers]} ended, "
          f"best {[round(b[0][0], 3) for b in run.best(1.0)]}, status {run.status()}")


if __name__ == "__main__":
    main()
