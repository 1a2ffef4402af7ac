"""Host models of what sequences over shared pages do: groups of a batch, forks, steps, beams."""
from __future__ import annotations

import math

import numpy as np
import torch

from pages_common import DEV, Cache


class GroupCache(Cache):
    """A Cache whose sequences come in groups: (shared tokens, [(new, own tokens behind them)]).

    Whole pages of the shared tokens are the same in the group's tables; the others are each
    sequence's own.  loose: (new, tokens) of sequences before the groups, which are in none;
    `wide`: entries that the device's table has at least (no pages)."""

    def __init__(self, cache, heads, page, groups, loose=(), seed=0, wide=0, missing=(), **kw):
        seqs = list(loose) + [(n, shared + own) for shared, members in groups for n, own in members]
        super().__init__(cache, heads, page, seqs, seed=seed, **kw)
        at = len(loose)
        first = [at]
        for shared, members in groups:
            for b in range(at, at + len(members)):
                self.table[b, : shared // page] = self.table[at, : shared // page]
            at += len(members)
            first.append(at)
        for i, (b, s) in enumerate(missing):
            self.table[b, s] = (-1, self.n_pages, -7, 2 ** 31 - 1)[i % 4]
        self.grp_off = np.array(first, np.int32)
        self.wide = max(wide, self.width)

    def shared(self):
        """(tokens and leader of each group, tokens of each sequence), by the definition."""
        of_group, leader, of_seq = [], [], np.zeros(len(self.seqs), int)
        for f, l in zip(self.grp_off, self.grp_off[1:]):
            active = [b for b in range(f, l) if self.new[b] > 0]
            e = 0
            if active:
                agree = np.ones(self.width, bool)
                for b in active:
                    agree &= self.table[b] == self.table[active[0]]
                common = self.width if agree.all() else int(np.argmin(agree))
                seen = min(int(self.lens[b] - self.new[b]) + 1 for b in active)
                e = max(min(common * self.page, seen), 0) // 32 * 32
            of_group.append(e)
            leader.append(active[0] if active else f)
            of_seq[f:l] = e
        return np.array(of_group, int), np.array(leader, int), of_seq

    def device(self, max_tokens=None, max_len=None, table_gap=0, rows_after=0):
        import paper_2601_13631_amd as ckv
        table = np.full((len(self.seqs), self.wide + table_gap), -1, np.int32)
        table[:, self.wide:] = 0
        table[:, :self.width] = self.table
        batch = ckv.PageBatch(torch.from_numpy(table).to(DEV)[:, :self.wide], torch.from_numpy(self.lens).to(DEV),
                              torch.from_numpy(self.off).to(DEV), self.tokens + rows_after,
                              max_tokens=int(self.new.max()) if max_tokens is None else max_tokens,
                              max_len=int(self.lens.max()) if max_len is None else max_len)
        return ckv.PagePool(*self.device_pages()), batch

    def device_groups(self, batch, max_tokens=None, max_shared=None):
        import paper_2601_13631_amd as ckv
        off, n = self.grp_off, len(self.grp_off) - 1
        most = max([int(self.new[f:l].sum()) for f, l in zip(off, off[1:])] + [0])
        shared = torch.full((ckv.page_share_ints(n, len(self.seqs)),), -99, dtype=torch.int32, device=DEV)
        groups = ckv.PageGroups(torch.from_numpy(off).to(DEV), shared,
                                max_tokens=most if max_tokens is None else max_tokens,
                                max_shared=int(self.shared()[0].max(initial=0)) if max_shared is None else max_shared)
        ckv.page_share(self.page, batch, groups)
        return groups


def attend_shared(pool, batch, groups, q, sm=0.0, rows_after=0, stream=None):
    import paper_2601_13631_amd as ckv
    if rows_after:
        q = torch.cat([q, torch.full((rows_after,) + q.shape[1:], float("nan"), dtype=q.dtype, device=q.device)])
    out = torch.full_like(q, 7.0)
    ws = torch.full((ckv.page_attn_shared_workspace_bytes(pool, batch, groups, q.shape[1]),), 0xFF,
                    dtype=torch.uint8, device=DEV)
    ckv.page_attn_shared(pool, batch, groups, q, out, ws, sm_scale=sm, stream=stream)
    return out


def fork_model(page, table, lens, refs, parents, states=()):
    """Sequence by sequence: (table, lens, refs, {row: source} of the states)."""
    n, width = table.shape
    out = np.full((len(parents), width), -1, np.int32)
    out_lens, out_refs = np.zeros(len(parents), np.int32), refs.astype(np.int64)

    def pages(b):
        return table[b, : -(-min(max(int(lens[b]), 0), width * page) // page)]
    for b in range(n):
        for p in pages(b):
            if 0 <= p < refs.size:
                out_refs[p] -= 1
    for i, b in enumerate(parents):
        if not 0 <= b < n:
            continue
        held = pages(b)
        out[i, : held.size] = held
        out_lens[i] = min(max(int(lens[b]), 0), width * page)
        for p in held:
            if 0 <= p < refs.size:
                out_refs[p] += 1
    return out, out_lens, out_refs.astype(np.int32)


def extend_model(page, table, lens, refs, n_new, n_tokens):
    """Sequence by sequence, page by page."""
    n, width = table.shape
    table, before = table.copy(), refs
    refs, free = refs.copy(), [p for p in range(refs.size) if refs[p] <= 0]
    taken = asked = asked_tokens = refused = 0
    off, rows, src, dst, out_lens = [0], [], [], [], []
    for b in range(n):
        length, add = min(max(int(lens[b]), 0), width * page), max(int(n_new[b]), 0)
        src.append(-1)
        dst.append(-1)
        fill = []
        if -(-(length + add) // page) > width:
            refused, add = refused + 1, 0
        elif add:
            fill = list(range(-(-length // page), -(-(length + add) // page)))
            if length % page:
                tail = int(table[b, length // page])
                if 0 <= tail < refs.size and before[tail] > 1:
                    fill.insert(0, length // page)
            asked, asked_tokens = asked + len(fill), asked_tokens + add
            if (fill and asked > len(free)) or asked_tokens > n_tokens:
                refused, add, fill = refused + 1, 0, []
        for s in fill:
            if s * page < length:
                src[-1], dst[-1] = int(table[b, s]), free[taken]
                refs[src[-1]] -= 1
            table[b, s] = free[taken]
            refs[free[taken]] = 1
            taken += 1
        for pos in range(length, length + add):
            p = int(table[b, pos // page])
            rows.append((p * page + pos % page if 0 <= p < refs.size else -1, pos, b))
        off.append(off[-1] + add)
        out_lens.append(length + add)
    rows += [(-1, -1, -1)] * (n_tokens - len(rows))
    cols = np.array(rows, np.int64).reshape(n_tokens, 3)
    return {"table": table, "refs": refs, "lens": out_lens, "tok_off": off, "copy_src": src, "copy_dst": dst,
            "slots": cols[:, 0], "positions": cols[:, 1], "seqs": cols[:, 2],
            "counts": [off[-1], taken, len(free) - taken, refused]}


def select_model(logits, scores, done, keep, eos):
    """Request by request, every offer sorted: (parent, token, score in 64 bits, done)."""
    reqs, beams, vocab = logits.shape
    x = logits.astype(np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    largest = 3.3895313892515355e38 if logits.dtype == np.float64 else float(np.finfo(np.float32).max)
    x = np.where(x == np.inf, largest, x)
    parent, token = np.full((reqs, keep), -1), np.full((reqs, keep), -1)
    score, ended = np.full((reqs, keep), -np.inf), np.zeros((reqs, keep), int)
    for r in range(reqs):
        offers = []
        for b in range(beams):
            c = float(scores[r, b])
            if not c > -math.inf:
                continue
            if done is not None and done[r, b]:
                offers.append((-c, b, 0.0, eos, 1))
                continue
            row = x[r, b]
            m = row.max()
            if m == -np.inf:
                continue
            rest = math.log(math.fsum(np.exp(row - m)))
            # (more than are kept of one beam are of no use)
            best = np.lexsort((np.arange(vocab), -row))[:keep]
            offers += [(-math.fsum((row[v], -m, -rest, c)), b, -row[v], int(v), int(v == eos)) for v in best
                       if row[v] > -np.inf]
        for i, (s, b, _, v, d) in enumerate(sorted(offers)[:keep]):
            parent[r, i], token[r, i], score[r, i], ended[r, i] = r * beams + b, v, -s, d
    return parent, token, score, ended
