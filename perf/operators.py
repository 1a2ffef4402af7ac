"""The operators of a paged KV cache, as they are measured.

A cache of one layer is a pool of pages: a page holds the K and V rows of
``page`` consecutive tokens of one sequence (a ContiguousChunk of it), and a
table names the pages of each sequence in order.  The operators:

attn     attention of a ragged batch of sequences over their pages, one new token
         each (decoding) or many (prefill), over the whole sequence or over a
         sliding window and the sequence's first tokens; a cache in fp32, bf16, or
         8 bits (e4m3 codes, a power of two per page and KV head)
append   the new tokens' K and V rows into their pages, quantised for an 8-bit cache
copy     whole pages from one place of the pools to another, in every layer
         (what a forked sequence needs of the page it goes on writing)
compact  the pages still in use moved to the front of the pools, in every layer,
         with the tables and use counts that go with them

``own`` chooses between the plain form (elementary torch operations, 32 bits) and
the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"

# (query heads, KV heads, head_dim): Qwen2.5-0.5B, 7B and 14B/32B attention layers,
# then two generic ones
HEADS = ((14, 2, 64), (28, 4, 128), (40, 8, 128), (32, 8, 128), (12, 4, 64))
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}


def _attn(name, cache, seqs, new, length, heads, page, window=0, sinks=0, evict=False, mix=1):
    return {"name": name, "kind": "attn", "cache": cache, "seqs": seqs, "new": new, "len": length,
            "hq": heads[0], "hkv": heads[1], "d": heads[2], "page": page, "window": window,
            "sinks": sinks, "evict": evict, "mix": mix}


def _append(name, cache, seqs, new, length, heads, page, mix=1):
    return {"name": name, "kind": "append", "cache": cache, "seqs": seqs, "new": new, "len": length,
            "hkv": heads[1], "d": heads[2], "page": page, "mix": mix}


def _move(name, kind, cache, layers, pages, count, heads, page, mix=1):
    return {"name": name, "kind": kind, "cache": cache, "layers": layers, "pages": pages,
            "count": count, "hkv": heads[1], "d": heads[2], "page": page, "mix": mix}


def listed():
    return [
        # one token of one short chat on the smallest model: launches and latency count
        _attn("decode_1", "bf16", 1, 1, 1000, (14, 2, 64), 16, window=256, sinks=4),
        # a serving step: 48 requests of every age, a window of 4,096 tokens, and the
        # pages that left the window given back
        _attn("decode_window_48", "bf16", 48, 1, 30011, (28, 4, 128), 32, window=4096, sinks=32,
              evict=True, mix=2),
        # new turns of five chats of ragged lengths, all in one call
        _attn("prefill_window_5", "bf16", 5, 2048, 8192, (28, 4, 128), 64, window=1000, sinks=4, mix=3),
        # the fp32 configuration
        _attn("prefill_f32", "f32", 3, 96, 1024, (4, 1, 64), 16, window=128, sinks=4, mix=4),
        # the first answer token after a Re-Prefill of a 32K prefix, cache in 8 bits
        _attn("decode_8bit_1", "e4m3", 1, 1, 32801, (28, 4, 128), 32),
        # a full serving step over an 8-bit cache: the largest
        _attn("decode_8bit_64", "e4m3", 64, 1, 16384, (40, 8, 128), 16, mix=5),
        # a question of 512 tokens on a 32K prefix in 8 bits
        _attn("prefill_8bit_32k", "e4m3", 1, 512, 33280, (28, 4, 128), 32),
        # four draft tokens of 16 requests checked at once, fine pages, a window
        _attn("draft_8bit_16", "e4m3", 16, 4, 8000, (14, 2, 64), 8, window=2000, sinks=8, mix=6),
        # the rows of one serving step into the 8-bit cache
        _append("append_step_8bit", "e4m3", 64, 1, 16384, (40, 8, 128), 16, mix=5),
        # the rows of four prompts into the 8-bit cache
        _append("append_prompts_8bit", "e4m3", 4, 8000, 16000, (28, 4, 128), 32, mix=7),
        # eight chats forked: their last pages copied in all 28 layers
        _move("fork_8", "copy", "bf16", 28, 512, 8, (28, 4, 128), 16),
        # a pool of 4,000 pages of which 1,200 have been given back, all 28 layers
        _move("compact_4000", "compact", "e4m3", 28, 4000, 1200, (28, 4, 128), 16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "decode", "decode", "prefill", "prefill", "f32", "append", "append",
                       "copy", "compact"))
    heads = rng.choice(HEADS)
    page, mix = rng.choice((8, 16, 32, 64, 96)), rng.randint(10, 1 << 20)
    cache = rng.choice(("bf16", "e4m3"))
    if kind in ("decode", "prefill", "f32"):
        windowed = rng.random() < 0.5
        window, sinks = (_log_int(rng, 30, 5000), rng.choice((0, 1, 4, 8, 40))) if windowed else (0, 0)
        evict = windowed and rng.random() < 0.5
        if kind == "decode":
            seqs, new = _log_int(rng, 1, 64), rng.choice((1, 1, 1, 1, 2, 5))
            length = _log_int(rng, 60, min(131072, 1000000 // seqs))
        elif kind == "prefill":
            seqs, new = rng.randint(1, 6), _log_int(rng, 16, 2000)
            length = _log_int(rng, new, min(40000, 40000000 // (seqs * new)))
        else:
            cache, heads = "f32", (4, rng.choice((1, 2)), 64)
            seqs, new = rng.randint(1, 4), _log_int(rng, 1, 128)
            length = _log_int(rng, max(new, 100), 4096)
        return {k: v for k, v in _attn("", cache, seqs, new, max(length, new), heads, page, window,
                                       sinks, evict, mix).items() if k != "name"}
    if kind == "append":
        seqs = _log_int(rng, 1, 64)
        new = rng.choice((1, _log_int(rng, 1, 32000 // seqs)))
        got = _append("", rng.choice(("bf16", "e4m3", "e4m3")), seqs, new, _log_int(rng, new, 16000) + new,
                      heads, page, mix)
    else:
        layers, pages = rng.randint(1, 28), _log_int(rng, 64, 64000 // page)
        count = _log_int(rng, 1, 60) if kind == "copy" else rng.randint(1, pages // 2)
        got = _move("", kind, cache, layers, pages, min(count, pages // 2), heads, page, mix)
    return {k: v for k, v in got.items() if k != "name"}


# ---- shapes -------------------------------------------------------------------

def _lengths(case):
    """(new tokens, length with them) of each sequence, by the case alone: one sequence has
    the most of both, the others are spread below."""
    r, seqs = np.random.RandomState(case["mix"]), case["seqs"]
    new = r.randint(max(1, case["new"] // 8), case["new"] + 1, seqs)
    length = np.exp(r.uniform(math.log(max(1, case["len"] / 16)), math.log(case["len"]), seqs)).astype(np.int64)
    new[0], length[0] = case["new"], case["len"]
    return new, np.maximum(length, new)


def _seen(case, new, length):
    """(keys seen by one query or more, (query, key) pairs) of one sequence."""
    pos = np.arange(length - new, length)
    if not case["window"]:
        return length, int((pos + 1).sum())
    lo = np.maximum(pos - case["window"] + 1, 0)
    first = np.minimum(case["sinks"], lo)
    return int(length - lo[0] + first[0]), int((pos + 1 - lo + first).sum())


def _row(case):
    return case["hkv"] * case["d"] * BYTES[case["cache"]]


def work(case):
    kind, row = case["kind"], _row(case)
    scale = 2 * case["hkv"] if case["cache"] == "e4m3" else 0  # bytes of a page's scales
    if kind == "attn":
        new, length = _lengths(case)
        seen = [_seen(case, int(n), int(m)) for n, m in zip(new, length)]
        keys, pairs = sum(s[0] for s in seen), sum(s[1] for s in seen)
        q = int(new.sum()) * case["hq"] * case["d"] * (4 if case["cache"] == "f32" else 2)
        return {"bytes": 2 * keys * row + keys / case["page"] * (scale + 4) + 2 * q,
                "flops": 4.0 * case["d"] * case["hq"] * pairs}
    if kind == "append":
        new, length = _lengths(case)
        tokens = int(new.sum())
        old = int(((length - new) % case["page"]).sum()) if scale else 0  # may have to be scaled anew
        wide = case["hkv"] * case["d"] * (4 if case["cache"] == "f32" else 2)
        return {"bytes": 2 * tokens * (wide + row) + 2 * old * row + tokens / case["page"] * scale,
                "flops": 4.0 * tokens * case["hkv"] * case["d"]}
    moved = case["count"] if kind == "copy" else _moves(case)[0].size
    return {"bytes": 2.0 * case["layers"] * moved * (2 * case["page"] * row + scale) + 8 * case["pages"],
            "flops": 0.0}


# ---- inputs -------------------------------------------------------------------

def _generator(seed, salt):
    return torch.Generator(DEV).manual_seed(int(seed) * 1009 + salt)


def _scale_byte(amax):
    """The exponent of the least power of two s with amax <= 448 s, plus 127, at least 10."""
    f, x = torch.frexp(amax)
    return torch.where(amax > 0, torch.clamp(x - 9 + (f > 0.875).to(x.dtype) + 127, min=10), 10).to(torch.uint8)


def _power(byte):
    return torch.ldexp(torch.ones_like(byte, dtype=torch.float32), byte.to(torch.int32) - 127)


def _quantise(x):
    """Whole pages [P, page, Hkv, d] (fp32) as codes and scale bytes [P, Hkv]."""
    byte = _scale_byte(x.abs().amax(dim=(1, 3)))
    return (x / _power(byte)[:, None, :, None]).to(torch.float8_e4m3fn), byte


def _cache_rows(g, pages, page, hkv, d, cache, spread):
    """Page contents: unit normal rows, heads of different size, and a direction per head that
    5% of the pages share with the queries."""
    x = torch.randn(pages, page, hkv, d, generator=g, device=DEV)
    heavy = (torch.rand(pages, generator=g, device=DEV) < 0.05).float()
    x += 1.5 * heavy[:, None, None, None] * spread
    if cache != "e4m3":
        return x.to(TYPES[cache]), None
    return _quantise(x.to(torch.bfloat16).float())


def prepare(case, seed):
    kind, hkv, d, page = case["kind"], case["hkv"], case["d"], case["page"]
    g = _generator(seed, 1)
    st = {"case": dict(case)}
    size = torch.exp2(torch.rand(hkv, 1, generator=g, device=DEV) * 2 - 1)
    if kind in ("copy", "compact"):
        return _prepare_move(case, seed, st, g)
    new, length = _lengths(case)
    n_pages = -(-length // page)
    width = int(n_pages.max())
    table = np.full((case["seqs"], width), -1, np.int32)
    for b in range(case["seqs"]):
        first = 0
        if case.get("evict"):  # pages that no later query sees have been given back
            first = max(0, int(length[b] - new[b]) - case["window"] + 1) // page
        kept = [j for j in range(n_pages[b]) if j >= first or j * page < case.get("sinks", 0)]
        table[b, kept] = 0
    used = int((table == 0).sum())
    total = used + 3
    table[table == 0] = np.random.RandomState(seed % (1 << 31)).permutation(total)[:used]
    direction = torch.randn(hkv, d, generator=g, device=DEV)
    st["k"], st["k_scale"] = _cache_rows(g, total, page, hkv, d, case["cache"], direction)
    st["v"], st["v_scale"] = _cache_rows(g, total, page, hkv, d, case["cache"], size)
    st["table"] = torch.from_numpy(table).to(DEV)
    st["lens"] = torch.from_numpy(length.astype(np.int32)).to(DEV)
    st["tok_off"] = torch.from_numpy(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).to(DEV)
    st["tokens"], st["most_new"], st["most_len"] = int(new.sum()), int(new.max()), int(length.max())
    wide = torch.float32 if case["cache"] == "f32" else torch.bfloat16
    if kind == "append":
        st["k_new"] = (torch.randn(st["tokens"], hkv, d, generator=g, device=DEV) * size * 1.5).to(wide)
        st["v_new"] = (torch.randn(st["tokens"], hkv, d, generator=g, device=DEV) * size).to(wide)
    else:
        q = torch.randn(st["tokens"], hkv, case["hq"] // hkv, d, generator=g, device=DEV)
        st["q"] = (q + direction[:, None]).reshape(st["tokens"], case["hq"], d).to(wide)
    return st


def _in_use(case):
    """Use count of each page: `count` of them given back, a tenth shared by two sequences."""
    r = np.random.RandomState(case["mix"])
    refs = np.where(r.rand(case["pages"]) < 0.1, 2, 1).astype(np.int32)
    refs[r.permutation(case["pages"])[: case["count"]]] = 0
    return refs


def _moves(case):
    """(from, to) of a compaction."""
    refs = _in_use(case)
    n = int((refs > 0).sum())
    return np.nonzero(refs[n:] > 0)[0] + n, np.nonzero(refs[:n] <= 0)[0]


def _prepare_move(case, seed, st, g):
    layers, pages, page, hkv, d = (case[k] for k in ("layers", "pages", "page", "hkv", "d"))
    r = np.random.RandomState((seed * 7 + case["mix"]) % (1 << 31))
    for name in ("k", "v"):
        if case["cache"] == "e4m3":
            code = torch.randint(0, 127, (layers, pages, page, hkv, d), generator=g, device=DEV, dtype=torch.uint8)
            st[name] = code.view(torch.float8_e4m3fn)
            st[name + "_scale"] = torch.randint(110, 130, (layers, pages, hkv), generator=g, device=DEV,
                                                dtype=torch.uint8)
        else:
            st[name] = torch.randn(layers, pages, page, hkv, d, generator=g, device=DEV,
                                   dtype=torch.bfloat16).to(TYPES[case["cache"]])
            st[name + "_scale"] = None
    if case["kind"] == "copy":
        pick = r.permutation(pages)[: 2 * case["count"]].astype(np.int32)
        st["src"], st["dst"] = (torch.from_numpy(x.copy()).to(DEV) for x in np.split(pick, 2))
        return st
    refs = _in_use(case)
    held = np.nonzero(refs > 0)[0]
    entries = r.permutation(np.concatenate([held, held[refs[held] > 1]])).astype(np.int32)
    width = 64  # table rows of 64 pages, the last one short: the rest names no page
    table = np.full((-(-entries.size // width), width), -1, np.int32)
    table.reshape(-1)[: entries.size] = entries
    st["table"], st["refs"] = torch.from_numpy(table).to(DEV), torch.from_numpy(refs).to(DEV)
    return st


# ---- one pass -----------------------------------------------------------------

def run(st):
    if own:
        return _own(st)
    return {"attn": _plain_attn, "append": _plain_append, "copy": _plain_copy,
            "compact": _plain_compact}[st["case"]["kind"]](st)


def _states(st, names):
    return {n: st[n] for n in names if st[n] is not None}


POOL = ("k", "v", "k_scale", "v_scale")


def _own(st):
    import paper_2601_13631_amd as ckv
    case = st["case"]
    kind = case["kind"]
    if "own" not in st:  # the handles and the workspace that a serving program keeps
        if kind in ("copy", "compact"):
            part = lambda n, i: None if st[n] is None else st[n][i]  # noqa: E731
            pools = ckv.PageLayers([ckv.PagePool(*(part(n, i) for n in POOL)) for i in range(case["layers"])])
            ws = None
            if kind == "compact":
                ws = torch.empty(ckv.page_compact_workspace_bytes(case["pages"]), dtype=torch.uint8, device=DEV)
            st["own"] = (pools, ws)
        else:
            pool = ckv.PagePool(*(st[n] for n in POOL))
            batch = ckv.PageBatch(st["table"], st["lens"], st["tok_off"], st["tokens"],
                                  max_tokens=st["most_new"], max_len=st["most_len"])
            ws = None
            if kind == "attn":
                ws = torch.empty(ckv.page_attn_workspace_bytes(pool, batch, case["hq"], window=case["window"],
                                                               n_sinks=case["sinks"]),
                                 dtype=torch.uint8, device=DEV)
            st["own"] = (pool, batch, ws)
    if kind == "attn":
        pool, batch, ws = st["own"]
        out = torch.empty_like(st["q"])
        ckv.page_attn(pool, batch, st["q"], out, ws, window=case["window"], n_sinks=case["sinks"])
        return out
    if kind == "append":
        pool, batch, _ = st["own"]
        ckv.page_append(pool, batch, st["k_new"], st["v_new"])
        return _states(st, POOL)
    pools, ws = st["own"]
    if kind == "copy":
        ckv.page_copy(pools, st["src"], st["dst"])
        return _states(st, POOL)
    refs, table = torch.empty_like(st["refs"]), torch.empty_like(st["table"])
    n_live = torch.empty(1, dtype=torch.int32, device=DEV)
    ckv.page_compact(pools, st["refs"], refs, st["table"], table, n_live, ws)
    return dict(_states(st, POOL), refs=refs, table=table, n_live=n_live)


def _plain_attn(st):
    case = st["case"]
    hq, hkv, d, page = case["hq"], case["hkv"], case["d"], case["page"]
    table, lens, off, q = st["table"], st["lens"].long(), st["tok_off"].long(), st["q"]
    seqs, width = table.shape
    named = (table >= 0) & (table < st["k"].shape[0])
    pages = torch.where(named, table, 0).long()

    def rows(name):
        x, scale = st[name], st[name + "_scale"]
        x = (x[pages] if scale is None else x.view(torch.uint8)[pages].view(x.dtype)).float()
        if scale is not None:
            x *= _power(scale[pages])[:, :, None, :, None]
        return x.view(seqs, width * page, hkv, d).transpose(1, 2)

    most = st["most_new"]
    i = torch.arange(most, device=DEV)
    new = off[1:] - off[:-1]
    tok = (off[:-1, None] + i).clamp(max=q.shape[0] - 1)
    qp = q[tok].float().view(seqs, most, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4).reshape(seqs, hkv, -1, d)
    s = (qp @ rows("k").transpose(-1, -2)) / math.sqrt(d)
    s = s.view(seqs, hkv, hq // hkv, most, width * page)
    pos = ((lens - new)[:, None] + i)[:, :, None]
    j = torch.arange(width * page, device=DEV)
    see = (j <= pos) & (j < lens[:, None, None]) & named.repeat_interleave(page, 1)[:, None]
    if case["window"]:
        see &= (j > pos - case["window"]) | (j < case["sinks"])
    s.masked_fill_(~see[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = (s - torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(seqs, hkv, -1, width * page) @ rows("v")).view(seqs, hkv, hq // hkv, most, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(seqs, most, hq, d)
    t = torch.arange(q.shape[0], device=DEV)
    seq = torch.searchsorted(off[1:], t, right=True)
    return o[seq, t - off[seq]].to(q.dtype)


def _plain_append(st):
    page, table, off = st["case"]["page"], st["table"], st["tok_off"].long()
    lens = st["lens"].long()
    start = lens - (off[1:] - off[:-1])
    t = torch.arange(st["tokens"], device=DEV)
    seq = torch.searchsorted(off[1:], t, right=True)
    pos = start[seq] + t - off[seq]
    at, row = table[seq, pos // page].long(), pos % page
    for x, new, scale in ((st["k"], st["k_new"], st["k_scale"]), (st["v"], st["v_new"], st["v_scale"])):
        if scale is None:
            x[at, row] = new
            continue
        # the new rows' largest value in each page and head, over the scale of the rows that
        # the page held before (the first new token's page, if it starts inside one)
        w = new.float()
        amax = torch.zeros(scale.shape, device=DEV)
        amax.index_reduce_(0, at, w.abs().amax(-1), "amax")
        touched = torch.zeros(scale.shape[0], dtype=torch.bool, device=DEV)
        touched[at] = True
        held = torch.zeros_like(touched, dtype=torch.int64)
        first = table.gather(1, (start // page).clamp(max=table.shape[1] - 1)[:, None])[:, 0].long()
        held.index_reduce_(0, first.clamp(min=0), torch.where(first >= 0, start % page, 0), "amax")
        to = _scale_byte(amax)
        to = torch.where(touched[:, None], torch.where((held > 0)[:, None], torch.maximum(to, scale), to), scale)
        rise = torch.ldexp(torch.ones_like(amax), scale.to(torch.int32) - to.to(torch.int32))
        part = first.clamp(min=0)
        old = x.view(torch.uint8)[part].view(x.dtype).float()
        again = (old * rise[part][:, None, :, None]).to(x.dtype).view(torch.uint8)
        kept = torch.arange(page, device=DEV) < torch.where(first >= 0, start % page, 0)[:, None]
        b, r = torch.nonzero(kept, as_tuple=True)
        x.view(torch.uint8)[part[b], r] = again[b, r]
        x.view(torch.uint8)[at, row] = (w / _power(to)[at][:, :, None]).to(x.dtype).view(torch.uint8)
        scale.copy_(to)
    return _states(st, POOL)


def _plain_copy(st):
    src, dst = st["src"].long(), st["dst"].long()
    for name in POOL:
        if st[name] is not None:
            x = st[name].view(torch.uint8) if st["k_scale"] is not None else st[name]
            x[:, dst] = x[:, src]
    return _states(st, POOL)


def _plain_compact(st):
    refs, table = st["refs"], st["table"]
    live = refs > 0
    n_live = live.sum()
    at = torch.arange(refs.numel(), device=DEV)
    src, dst = torch.nonzero(live & (at >= n_live))[:, 0], torch.nonzero(~live & (at < n_live))[:, 0]
    for name in POOL:
        if st[name] is not None:
            x = st[name].view(torch.uint8) if st["k_scale"] is not None else st[name]
            x[:, dst] = x[:, src]
    to = torch.where(live, at, -1).to(torch.int32)
    to[src] = dst.to(torch.int32)
    counts = torch.where(live & (at < n_live), refs, 0)
    counts[dst] = refs[src]
    inside = (table >= 0) & (table < refs.numel())
    moved = torch.where(inside, to[torch.where(inside, table, 0).long()], table)
    return dict(_states(st, POOL), refs=counts, table=moved, n_live=n_live.to(torch.int32)[None])


# ---- the definition, in 64 bits --------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"attn": _exact_attn, "append": _exact_append, "copy": _exact_move,
            "compact": _exact_move}[case["kind"]](st)


def _exact_attn(st):
    """Sequence by sequence and KV head by KV head, over the tokens of its pages alone."""
    case, group = st["case"], st["case"]["hq"] // st["case"]["hkv"]
    table, lens, off = st["table"].cpu().numpy(), st["lens"].tolist(), st["tok_off"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    for b, (n0, n1) in enumerate(zip(off, off[1:])):
        where, have = [], []  # positions that have a page, and (page, row) of each
        for pos in range(0, lens[b], case["page"]):
            if 0 <= table[b, pos // case["page"]] < st["k"].shape[0]:
                rows = min(case["page"], lens[b] - pos)
                where.append(np.arange(pos, pos + rows))
                have.append(table[b, pos // case["page"]] * case["page"] + np.arange(rows))
        if not where:
            continue
        key = torch.from_numpy(np.concatenate(where)).to(DEV)
        have = torch.from_numpy(np.concatenate(have)).to(DEV)
        at = torch.arange(lens[b] - (n1 - n0), lens[b], device=DEV)[:, None]
        hide = key > at
        if case["window"]:
            hide = hide | ((at - key >= case["window"]) & (key >= case["sinks"]))
        for h in range(case["hkv"]):
            def tokens(name):
                x, s = st[name][:, :, h], st[name + "_scale"]
                x = x.double()
                if s is not None:
                    x = x * 2.0 ** (s[:, h].double() - 127)[:, None, None]
                return x.reshape(-1, case["d"])[have]
            k, v = tokens("k"), tokens("v")
            for i in range(group):
                s = st["q"][n0:n1, h * group + i].double() @ k.T / math.sqrt(case["d"])
                w = torch.softmax(s.masked_fill(hide, -1e300), -1).masked_fill(hide, 0.0)
                out[n0:n1, h * group + i] = w @ v
    return out


def _exact_append(st):
    """Page by page on the host, values and powers of two in 64 bits."""
    case, page = st["case"], st["case"]["page"]
    table, lens, off = st["table"].cpu().numpy(), st["lens"].tolist(), st["tok_off"].tolist()
    grid = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    values = np.unique(grid[np.isfinite(grid)])  # every code's value, ascending
    even = np.zeros(values.size, bool)  # those whose code is even, -0 and 0 as one
    for i in range(0, 256, 2):
        even[values == grid[i]] = True

    def nearest(x):
        hi = np.clip(np.searchsorted(values, x), 1, values.size - 1)
        up, down = values[hi] - x, x - values[hi - 1]
        return np.where((up < down) | ((up == down) & even[hi]), values[hi], values[hi - 1])

    got = {}
    for name in ("k", "v"):
        x, new = st[name].double().cpu().numpy(), st[name + "_new"].double().cpu().numpy()
        scale = None if st[name + "_scale"] is None else st[name + "_scale"].cpu().numpy().astype(np.int64)
        for b, (n0, n1) in enumerate(zip(off, off[1:])):
            start = lens[b] - (n1 - n0)
            for j in range(start // page, -(-lens[b] // page)):
                lo, hi, at = max(start, j * page), min(lens[b], j * page + page), table[b, j]
                rows = new[n0 + lo - start: n0 + hi - start]
                if scale is None:
                    x[at, lo - j * page: hi - j * page] = rows
                    continue
                most = np.abs(rows).max(axis=(0, 2))
                least = np.ceil(np.log2(np.maximum(most, 1e-300) / 448)).astype(np.int64)
                least -= (most <= 448 * 2.0 ** (least - 1)).astype(np.int64)
                least = np.maximum(least + 127, 10)
                if lo > j * page:
                    old = scale[at].copy()
                    least = np.maximum(least, old)
                    x[at, : lo - j * page] = nearest(x[at, : lo - j * page] * 2.0 ** (old - least)[None, :, None])
                scale[at] = least
                x[at, lo - j * page: hi - j * page] = nearest(rows / 2.0 ** (least - 127)[None, :, None])
        got[name] = torch.from_numpy(x)
        if scale is not None:
            got[name + "_scale"] = torch.from_numpy(scale)
    return got


def _exact_move(st):
    """The pages' numbers after the moves, then every pool read by them."""
    case = st["case"]
    got, come = {}, np.arange(case["pages"])  # come[p]: the page whose contents end at p
    if case["kind"] == "copy":
        for a, b in zip(st["src"].tolist(), st["dst"].tolist()):
            come[b] = a
    else:
        refs = st["refs"].cpu().numpy().copy()
        live, name = int((refs > 0).sum()), {int(p): int(p) for p in np.nonzero(refs > 0)[0]}
        free = [p for p in range(live) if refs[p] <= 0]
        for p, hole in zip([p for p in range(live, case["pages"]) if refs[p] > 0], free):
            come[hole], name[p] = p, hole
            refs[hole], refs[p] = refs[p], 0
        table = [[name.get(e, -1) if 0 <= e < case["pages"] else e for e in row] for row in st["table"].tolist()]
        got = {"refs": None, "table": torch.tensor(table), "n_live": torch.tensor([live])}
        got["refs"] = torch.from_numpy(np.maximum(refs, 0))
    index = torch.from_numpy(come).to(DEV)
    for n in POOL:
        if st[n] is not None:
            x = st[n].view(torch.uint8) if st["k_scale"] is not None else st[n]
            got[n] = x.index_select(1, index).view(st[n].dtype)
            got[n] = got[n].double() if got[n].numel() < 1 << 27 and n in ("k", "v") else got[n]
    return got
