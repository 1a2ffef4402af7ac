"""The operators of a decoding step over shared prefixes, as they are measured.

Sequences of a paged cache that begin with the same pages (beams of one request, chats
on one document) go through this loop: the continuations are chosen, the sequences
follow their parents, the step's pages and slots are found, and every layer attends.
The operators:

attn     attention of a batch in groups: the pages that all sequences of a group begin
         with are read once for all of them, the rest by each; the groups' shared lengths
         are found once for all layers of the step, which is part of the pass
select   the K best continuations of each request over its beams and the vocabulary, with
         their scores; done beams go on as they are, dead ones not at all
fork     tables, lengths, use counts and per-sequence rows after the parents of a step
extend   the pages of each sequence's new tokens, from the free ones; slots, positions and
         sequences of the call's token rows; the pages to copy because others hold them

``own`` chooses between the plain form (elementary torch operations; 32 bits, scores in
64) and the library's calls.
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
EOS = 2


def _attn(name, cache, layers, groups, seqs, new, shared, rest, heads, page, mix=1):
    return {"name": name, "kind": "attn", "cache": cache, "layers": layers, "groups": groups, "seqs": seqs,
            "new": new, "shared": shared, "rest": rest, "hq": heads[0], "hkv": heads[1], "d": heads[2],
            "page": page, "mix": mix}


def _select(name, type_, reqs, beams, keep, vocab, done=0.0, dead=0.0):
    return {"name": name, "kind": "select", "type": type_, "reqs": reqs, "beams": beams, "keep": keep,
            "vocab": vocab, "done": done, "dead": dead}


def _tables(name, kind, groups, seqs, new, shared, rest, page, pages, mix=1):
    return {"name": name, "kind": kind, "groups": groups, "seqs": seqs, "new": new, "shared": shared,
            "rest": rest, "page": page, "pages": pages, "mix": mix}


def listed():
    return [
        # four beams of one short request on the smallest model: launches and latency count
        _attn("attn_beams_4", "bf16", 1, 1, 4, 1, 1000, 40, (14, 2, 64), 16),
        # one decoding step of 48 chats on one document of 30K tokens, two of its layers
        _attn("attn_document_48", "bf16", 2, 1, 48, 1, 30011, 1500, (28, 4, 128), 32, mix=2),
        # eight requests of eight beams each over an 8-bit cache, two layers: the most bytes
        _attn("attn_8bit_8x8", "e4m3", 2, 8, 8, 1, 16384, 700, (40, 8, 128), 16, mix=3),
        # 24 questions of up to 48 tokens on a document of 32K in 8 bits: the most products
        _attn("attn_questions_24", "e4m3", 1, 1, 24, 48, 32768, 60, (28, 4, 128), 32, mix=4),
        # the fp32 configuration: three documents of different lengths
        _attn("attn_f32", "f32", 1, 3, 5, 1, 1024, 128, (4, 1, 64), 16, mix=5),
        # four beams of one request, a small vocabulary
        _select("select_4", "bf16", 1, 4, 4, 32000),
        # 64 requests of four beams; twice as many kept, so that done ones leave enough
        _select("select_64x4", "bf16", 64, 4, 8, 131072, done=0.1),
        # fp32 logits, an odd vocabulary, beams that ended and beams that are empty
        _select("select_f32_odd", "f32", 24, 6, 6, 100003, done=0.2, dead=0.1),
        # the beams of one request follow their parents
        _tables("fork_4", "fork", 1, 4, 1, 2000, 60, 16, 4096),
        # 64 requests of four beams on documents of 8K tokens
        _tables("fork_64x4", "fork", 64, 4, 1, 8192, 300, 16, 65536, mix=7),
        # a decoding step of 256 sequences, one of four just forked
        _tables("extend_step_256", "extend", 64, 4, 1, 8192, 300, 16, 65536, mix=7),
        # 40 prompts of up to 6,000 tokens get their pages
        _tables("extend_prompts_40", "extend", 40, 1, 6000, 500, 300, 32, 16384, mix=9),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("decode", "decode", "prompts", "f32", "select", "select", "fork", "extend", "extend"))
    mix = rng.randint(20, 1 << 20)
    if kind in ("decode", "prompts", "f32"):
        heads, page, cache = rng.choice(HEADS), rng.choice((8, 16, 32, 64, 96)), rng.choice(("bf16", "e4m3"))
        groups = _log_int(rng, 1, 8)
        if kind == "decode":
            seqs, new = _log_int(rng, 1, 64 // groups), rng.choice((1, 1, 1, 2, 4))
            shared, rest = _log_int(rng, 20, 49152 // groups), _log_int(rng, 4, 1000)
        elif kind == "prompts":
            seqs, new = _log_int(rng, 2, 20), _log_int(rng, 5, 60)
            shared, rest = _log_int(rng, 100, 25000000 // (groups * seqs * new)), _log_int(rng, new, 300)
        else:
            cache, heads, seqs, new = "f32", (4, rng.choice((1, 2)), 64), rng.randint(1, 8), rng.choice((1, 1, 3))
            shared, rest = _log_int(rng, 20, 4096), _log_int(rng, 4, 300)
        layers = 1 if kind == "prompts" else rng.choice((1, 1, 2))
        got = _attn("", cache, layers, groups, seqs, new, min(shared, 32768), max(rest, new), heads,
                    page, mix)
    elif kind == "select":
        beams = _log_int(rng, 1, 16)
        reqs = _log_int(rng, 1, 256 // beams)
        got = _select("", rng.choice(("bf16", "bf16", "f32")), reqs, beams, rng.randint(1, 2 * beams),
                      _log_int(rng, 1000, 60000), rng.choice((0.0, 0.1, 0.3)), rng.choice((0.0, 0.0, 0.2)))
    else:
        groups, seqs, page = _log_int(rng, 1, 64), rng.randint(1, 8), rng.choice((8, 16, 32, 64, 96))
        new = 1 if kind == "fork" else rng.choice((1, 1, 4, _log_int(rng, 2, 64000 // (groups * seqs))))
        shared, rest = _log_int(rng, 1, 8000), _log_int(rng, 1, 400)
        least = groups * (-(-shared // page) + seqs * (2 + (rest + new) // page))
        got = _tables("", kind, groups, seqs, new, shared, rest, page, max(64, int(least * rng.uniform(0.95, 3))), mix)
    return {k: v for k, v in got.items() if k != "name"}


# ---- shapes -------------------------------------------------------------------

def _spread(r, most, n):
    """n whole numbers up to `most`, spread over their logarithm, the first of them `most`."""
    x = np.exp(r.uniform(math.log(max(1, most / 16)), math.log(most + 1), n)).astype(np.int64)
    x[0] = most
    return np.clip(x, 1, most)


def _sizes(case):
    """(shared tokens of each group, own tokens of each sequence behind the shared pages, new ones
    among them), by the case alone."""
    r = np.random.RandomState(case["mix"])
    n = case["groups"] * case["seqs"]
    shared = _spread(r, case["shared"], case["groups"])
    shared[1:] = np.maximum(shared[1:], case["shared"] // 2)
    new = r.randint(max(1, case["new"] // 4), case["new"] + 1, n)
    new[0] = case["new"]
    rest = _spread(r, case["rest"], n)
    return shared, (np.maximum(rest, new) if case["kind"] == "attn" else rest), new


def _lengths(case):
    """Whole shared pages of each group, length of each sequence, new tokens of each. The shared
    tokens behind a group's last whole page are each sequence's own (a fork's copy)."""
    shared, rest, new = _sizes(case)
    pages = shared // case["page"]
    return pages, np.repeat(shared, case["seqs"]) + rest, new


def work(case):
    if case["kind"] == "select":
        rows = case["reqs"] * case["beams"]
        live = rows * (1 - case["done"]) * (1 - case["dead"])
        return {"bytes": live * case["vocab"] * (2 if case["type"] == "bf16" else 4) + 12.0 * case["reqs"] * case["keep"],
                "flops": 4.0 * live * case["vocab"]}
    pages, length, new = _lengths(case)
    c, n = case["page"], case["groups"] * case["seqs"]
    entries = int((-(-length // c)).sum())
    if case["kind"] == "attn":
        scale = 2 * case["hkv"] if case["cache"] == "e4m3" else 0  # bytes of a page's scales
        row = case["hkv"] * case["d"] * BYTES[case["cache"]]
        own_keys = length - np.repeat(pages, case["seqs"]) * c
        keys = int(pages.sum() * c + own_keys.sum())
        pairs = int((new * (length - new) + new * (new + 1) // 2).sum())
        q = int(new.sum()) * case["hq"] * case["d"] * (4 if case["cache"] == "f32" else 2)
        return {"bytes": case["layers"] * (2 * keys * row + keys / c * (scale + 4) + 2 * q) + 4 * entries,
                "flops": 4.0 * case["layers"] * case["d"] * case["hq"] * pairs}
    if case["kind"] == "fork":
        return {"bytes": 8.0 * entries + 8 * case["pages"] + 8 * n + 8 * n * 512, "flops": 0.0}
    return {"bytes": 8.0 * entries + 8 * case["pages"] + 12 * n + 16 * int(new.sum()), "flops": 0.0}


# ---- inputs -------------------------------------------------------------------

def _generator(seed, salt):
    return torch.Generator(DEV).manual_seed(int(seed) * 1009 + salt)


def prepare(case, seed):
    st = {"case": dict(case)}
    return {"attn": _prepare_attn, "select": _prepare_select, "fork": _prepare_tables,
            "extend": _prepare_tables}[case["kind"]](case, seed, st)


def _int32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)


def _table(case, pages, length, order):
    """The sequences' tables over pages taken from `order`, and the use count of each page."""
    c, seqs = case["page"], case["seqs"]
    width = int((-(-(length + case["new"]) // c)).max())
    table = np.full((length.size, width), -1, np.int32)
    refs, at = np.zeros(order.size, np.int32), 0
    for g in range(case["groups"]):
        common = order[at: at + pages[g]]
        at += pages[g]
        for b in range(g * seqs, (g + 1) * seqs):
            mine = -(-length[b] // c) - pages[g]
            table[b, : pages[g]] = common
            table[b, pages[g]: pages[g] + mine] = order[at: at + mine]
            at += mine
    held = table[table >= 0]
    np.add.at(refs, held, 1)
    return table, refs


def _pages_taken(case, pages, length):
    return int(pages.sum() + (-(-length // case["page"]) - np.repeat(pages, case["seqs"])).sum())


def _prepare_attn(case, seed, st):
    hkv, d, page, layers = case["hkv"], case["d"], case["page"], case["layers"]
    g = _generator(seed, 1)
    pages, length, new = _lengths(case)
    total = _pages_taken(case, pages, length) + 3
    table, _ = _table(case, pages, length, np.random.RandomState(seed % (1 << 31)).permutation(total))
    st["table"], st["lens"] = _int32(table), _int32(length)
    st["tok_off"] = _int32(np.concatenate([[0], np.cumsum(new)]))
    st["grp_off"] = _int32(np.arange(case["groups"] + 1) * case["seqs"])
    st["common"] = _int32(pages)  # whole pages that a group's sequences share
    st["tokens"], st["most_new"], st["most_len"] = int(new.sum()), int(new.max()), int(length.max())
    st["most_common"] = int(pages.max()) * page
    st["most_group"] = int(new.reshape(case["groups"], -1).sum(1).max())
    # rows of unit size with a direction per head that 5% of the pages share with the queries
    wide = torch.float32 if case["cache"] == "f32" else torch.bfloat16
    direction = torch.randn(hkv, d, generator=g, device=DEV)
    st["pools"], st["q"] = [], []
    for _ in range(layers):
        pool = {}
        for name, spread in (("k", direction), ("v", torch.rand(hkv, 1, generator=g, device=DEV) + 0.5)):
            x = torch.randn(total, page, hkv, d, generator=g, device=DEV)
            heavy = (torch.rand(total, generator=g, device=DEV) < 0.05).float()
            x += 1.5 * heavy[:, None, None, None] * spread
            pool[name + "_scale"] = None
            if case["cache"] == "e4m3":  # scales of about the pages' size, a power of two each
                byte = torch.randint(118, 121, (total, hkv), generator=g, device=DEV)
                x = (x / _power(byte)[:, None, :, None]).clamp(-448, 448)
                pool[name + "_scale"] = byte.to(torch.uint8)
            pool[name] = x.to(TYPES[case["cache"]])
        st["pools"].append(pool)
        q = torch.randn(st["tokens"], hkv, case["hq"] // hkv, d, generator=g, device=DEV)
        st["q"].append((q + direction[:, None]).reshape(st["tokens"], case["hq"], d).to(wide))
    return st


def _power(byte):
    return torch.ldexp(torch.ones_like(byte, dtype=torch.float32), byte.to(torch.int32) - 127)


def _prepare_select(case, seed, st):
    g = _generator(seed, 2)
    shape = (case["reqs"], case["beams"])
    # peaked as a language model's: a wide normal, some tokens far ahead
    x = torch.randn(*shape, case["vocab"], generator=g, device=DEV) * 2.5
    ahead = torch.randint(0, case["vocab"], (*shape, 6), generator=g, device=DEV)
    x.scatter_add_(2, ahead, torch.rand(*shape, 6, generator=g, device=DEV) * 12)
    st["logits"] = x.to(TYPES[case["type"]])
    scores = -30 * torch.rand(*shape, generator=g, device=DEV)
    r = np.random.RandomState((seed * 3 + 5) % (1 << 31))
    dead = r.rand(*shape) < case["dead"]
    dead[:, 0] = False
    st["scores"] = torch.where(torch.from_numpy(dead).to(DEV), -math.inf, scores)
    st["done"] = torch.from_numpy(((r.rand(*shape) < case["done"]) & ~dead).astype(np.uint8)).to(DEV)
    return st


def _prepare_tables(case, seed, st):
    pages, length, new = _lengths(case)
    taken, n = _pages_taken(case, pages, length), length.size
    r = np.random.RandomState(seed % (1 << 31))
    # where a pool is too small for all, sequences hold fewer tokens (the last ones none)
    total = max(case["pages"], taken)
    table, refs = _table(case, pages, length, r.permutation(total))
    if case["kind"] == "extend":
        # every fourth group has just been forked: its sequences hold the first one's last page too
        for g in range(0, case["groups"], 4):
            first = g * case["seqs"]
            slot = (length[first] - 1) // case["page"]
            for b in range(first + 1, first + case["seqs"]):
                held = table[b, pages[g]: -(-length[b] // case["page"])].copy()
                refs[held] -= 1
                table[b] = table[first]
                refs[table[b, pages[g]: slot + 1]] += 1
                length[b] = length[first]
        # some pages are held by a prefix store beside the tables
        refs[r.permutation(total)[: total // 50]] += 1
        st["n_new"], st["tokens"] = _int32(new), int(new.sum())
    else:
        # a request's beams after a step: each the child of any of its beams, the better ones more
        # often; a request in 20 has ended
        pick = np.minimum(r.exponential(case["seqs"] / 3, (case["groups"], case["seqs"])).astype(np.int64),
                          case["seqs"] - 1)
        parents = pick + np.arange(case["groups"])[:, None] * case["seqs"]
        parents[1:][r.rand(case["groups"] - 1) < 0.05] = -1
        st["parents"] = _int32(parents.reshape(-1))
        g = _generator(seed, 3)
        st["history"] = torch.randint(0, 32000, (n, 512), generator=g, device=DEV, dtype=torch.int32)
    st["table"], st["refs"], st["lens"] = _int32(table), _int32(refs), _int32(length)
    return st


# ---- one pass -----------------------------------------------------------------

def run(st):
    if own:
        return {"attn": _own_attn, "select": _own_select, "fork": _own_fork,
                "extend": _own_extend}[st["case"]["kind"]](st)
    return {"attn": _plain_attn, "select": _plain_select, "fork": _plain_fork,
            "extend": _plain_extend}[st["case"]["kind"]](st)


def _empty(n, dtype=torch.int32):
    return torch.empty(n, dtype=dtype, device=DEV)


def _own_attn(st):
    import paper_2601_13631_amd as ckv
    case = st["case"]
    if "own" not in st:  # the handles and the workspace that a serving program keeps
        batch = ckv.PageBatch(st["table"], st["lens"], st["tok_off"], st["tokens"], max_tokens=st["most_new"],
                              max_len=st["most_len"])
        groups = ckv.PageGroups(st["grp_off"], _empty(ckv.page_share_ints(case["groups"], batch.n_seqs)),
                                max_tokens=st["most_group"], max_shared=st["most_common"])
        pools = [ckv.PagePool(p["k"], p["v"], p["k_scale"], p["v_scale"]) for p in st["pools"]]
        ws = _empty(ckv.page_attn_shared_workspace_bytes(pools[0], batch, groups, case["hq"]), torch.uint8)
        st["own"] = (pools, batch, groups, ws)
    pools, batch, groups, ws = st["own"]
    ckv.page_share(case["page"], batch, groups)
    outs = []
    for pool, q in zip(pools, st["q"]):
        out = torch.empty_like(q)
        ckv.page_attn_shared(pool, batch, groups, q, out, ws)
        outs.append(out)
    return outs


def _own_select(st):
    import paper_2601_13631_amd as ckv
    case = st["case"]
    if "own" not in st:
        st["own"] = _empty(ckv.beam_select_workspace_bytes(st["logits"], case["keep"]), torch.uint8)
    shape = (case["reqs"], case["keep"])
    parent, token = _empty(shape), _empty(shape)
    scores, done = _empty(shape, torch.float32), _empty(shape, torch.uint8)
    ckv.beam_select(st["logits"], st["scores"], parent, token, scores, st["own"], done=st["done"], done_out=done,
                    eos=EOS)
    return {"parent": parent, "token": token, "scores": scores, "done": done}


def _own_fork(st):
    import paper_2601_13631_amd as ckv
    if "own" not in st:
        out = {n: torch.empty_like(st[n]) for n in ("table", "lens", "refs", "history")}
        st["own"] = (out, ckv.PageFork(st["case"]["page"], st["table"], out["table"], st["lens"], out["lens"],
                                       st["refs"], out["refs"], states=[(st["history"], out["history"])]))
        out["history"].zero_()  # rows of no parent are left as they were
    out, fork = st["own"]
    ckv.page_fork(fork, st["parents"])
    return out


def _own_extend(st):
    import paper_2601_13631_amd as ckv
    if "own" not in st:
        n, tokens = st["lens"].numel(), st["tokens"]
        out = {n: torch.empty_like(st[n]) for n in ("table", "lens", "refs")}
        out |= {"tok_off": _empty(n + 1), "slots": _empty(tokens, torch.int64), "positions": _empty(tokens),
                "seqs": _empty(tokens), "copy_src": _empty(n), "copy_dst": _empty(n), "counts": _empty(4)}
        step = ckv.PageStep(st["case"]["page"], st["table"], out["table"], st["lens"], out["lens"], st["refs"],
                            out["refs"], st["n_new"],
                            **{k: out[k] for k in ("tok_off", "slots", "positions", "seqs", "copy_src",
                                                   "copy_dst", "counts")})
        st["own"] = (out, step, _empty(ckv.page_extend_workspace_bytes(st["refs"].numel(), n), torch.uint8))
    out, step, ws = st["own"]
    ckv.page_extend(step, ws)
    return out


def _plain_attn(st):
    """Logits of the shared keys for a group's rows at once, of a sequence's own keys for its rows,
    and one softmax over both."""
    case = st["case"]
    hq, hkv, d, c = case["hq"], case["hkv"], case["d"], case["page"]
    G, n_groups, seqs = hq // hkv, case["groups"], case["seqs"]
    table, lens, off, common = st["table"], st["lens"].long(), st["tok_off"].long(), st["common"].long()
    B, width = table.shape
    n_tok, first = st["tokens"], torch.arange(n_groups, device=DEV) * seqs
    # token rows in a square for each group and for each sequence, and the way back
    tok = torch.arange(n_tok, device=DEV)
    seq = torch.searchsorted(off[1:], tok, right=True)
    grp = seq // seqs
    most_g = st["most_group"]
    row_g, row_s = tok - off[first][grp], tok - off[seq]
    square_g = torch.zeros(n_groups, most_g, dtype=torch.long, device=DEV).index_put_((grp, row_g), tok)
    square_s = torch.zeros(B, st["most_new"], dtype=torch.long, device=DEV).index_put_((seq, row_s), tok)
    pages_g = table[first][:, : int(st["most_common"]) // c].clamp(min=0).long()
    mine = -(-lens // c) - common.repeat_interleave(seqs)
    own_slots = common.repeat_interleave(seqs)[:, None] + torch.arange(
        st["most_len"] // c + 2 - case["shared"] // 2 // c, device=DEV)
    own_there = (own_slots < width)
    pages_s = table.gather(1, own_slots.clamp(max=width - 1)).clamp(min=0).long()
    pos = lens[seq] - (off[1:] - off[:-1])[seq] + row_s
    key_g = torch.arange(pages_g.shape[1] * c, device=DEV)
    see_g = key_g < (common * c)[:, None]
    key_s = (own_slots[:, :, None] * c + torch.arange(c, device=DEV)).view(B, -1)
    see_s = own_there.repeat_interleave(c, 1) & (key_s < lens[:, None])

    def rows(pool, name, pages):
        x, scale = pool[name], pool[name + "_scale"]
        x = (x[pages] if scale is None else x.view(torch.uint8)[pages].view(x.dtype)).float()
        if scale is not None:
            x *= _power(scale[pages])[:, :, None, :, None]
        return x.view(pages.shape[0], -1, hkv, d).transpose(1, 2).contiguous()

    outs = []
    for pool, q in zip(st["pools"], st["q"]):
        def part(square, pages, see):
            n, most = square.shape
            x = q.float()[square].view(n, most, hkv, G, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, G * most, d)
            k = rows(pool, "k", pages).transpose(-1, -2).contiguous()
            s = (x @ k).view(n, hkv, G, most, -1) / math.sqrt(d)
            s.masked_fill_(~see, -math.inf)
            top = s.amax(-1) if s.shape[-1] else s.new_full(s.shape[:-1], -math.inf)
            p = (s - torch.where(torch.isinf(top), 0.0, top)[..., None]).exp_()
            o = (p.view(n, hkv, G * most, -1) @ rows(pool, "v", pages)).view(n, hkv, G, most, d)
            return top, p.sum(-1), o
        parts = []
        for square, pages, see, at in ((square_g, pages_g, see_g[:, None, None, None], (grp, row_g)),
                                       (square_s, pages_s, None, (seq, row_s))):
            if see is None:
                at_s = torch.full(square.shape, -1, device=DEV).index_put_((seq, row_s), pos)
                see = (see_s[:, None] & (key_s[:, None] <= at_s[:, :, None]))[:, None, None]
            top, total, o = part(square, pages, see)
            parts.append([x.movedim(3, 1)[at].reshape(n_tok, hq, -1) for x in (top, total, o)])
        top = torch.maximum(parts[0][0], parts[1][0])
        w = [torch.where(torch.isinf(p[0]), 0.0, (p[0] - top).exp()) for p in parts]
        total = w[0] * parts[0][1] + w[1] * parts[1][1]
        outs.append(((w[0] * parts[0][2] + w[1] * parts[1][2]) / total).to(q.dtype))
    return outs


def _plain_select(st):
    case, live = st["case"], st["scores"] > -math.inf
    x = st["logits"].double()
    score = x - _lse(x) + st["scores"].double()[..., None]
    done = (st["done"] > 0) & live
    score = torch.where((live & ~done)[..., None], score, -math.inf)
    score[..., EOS] = torch.where(done, st["scores"].double(), score[..., EOS])
    flat = score.view(case["reqs"], -1)
    # some more than are kept, then by score and place
    value, at = flat.topk(min(case["keep"] + 64, flat.shape[1]), dim=1)
    at, order = at.sort(dim=1)
    value = value.gather(1, order)
    value, order = value.sort(dim=1, descending=True, stable=True)
    value, at = value[:, : case["keep"]], at.gather(1, order)[:, : case["keep"]]
    there = value > -math.inf
    beam = at // case["vocab"]
    token = torch.where(there, at % case["vocab"], -1).to(torch.int32)
    parent = torch.where(there, beam + torch.arange(case["reqs"], device=DEV)[:, None] * case["beams"], -1)
    ended = there & ((st["done"].gather(1, beam) > 0) | (token == EOS))
    return {"parent": parent.to(torch.int32), "token": token, "scores": value.float(), "done": ended.to(torch.uint8)}


def _lse(x):
    top = x.amax(-1, keepdim=True)
    return top + (x - top).exp().sum(-1, keepdim=True).log()


def _plain_fork(st):
    c, table, lens, refs, parents = st["case"]["page"], st["table"], st["lens"], st["refs"], st["parents"].long()
    held = (lens.long() + c - 1) // c
    slot = torch.arange(table.shape[1], device=DEV)
    there, p = parents >= 0, parents.clamp(min=0)
    used = there[:, None] & (slot < held[p][:, None])
    children = torch.zeros(lens.numel(), dtype=torch.int32, device=DEV).index_add_(0, p, there.to(torch.int32))
    mine = slot < held[:, None]
    seq = torch.nonzero(mine)[:, 0]
    counts = refs.index_add(0, table[mine].long(), children[seq] - 1)
    return {"table": torch.where(used, table[p], -1), "lens": torch.where(there, lens[p], 0), "refs": counts,
            "history": torch.where(there[:, None], st["history"][p], 0)}


def _plain_extend(st):
    c, table, refs = st["case"]["page"], st["table"].clone(), st["refs"].clone()
    lens, new, tokens = st["lens"].long(), st["n_new"].long(), st["tokens"]
    n, width = table.shape
    held, want = (lens + c - 1) // c, (lens + new + c - 1) // c
    tail = table.gather(1, (held - 1).clamp(min=0)[:, None])[:, 0].long()
    copied = (lens % c > 0) & (new > 0) & (refs[tail.clamp(min=0)] > 1)
    need = want - held + copied
    free = torch.nonzero(refs <= 0)[:, 0]
    upto = need.cumsum(0)
    fits = (need == 0) | (upto <= free.numel())
    need, new, copied = need * fits, new * fits, copied & fits
    first = upto - need  # (those that do not fit are behind all that need pages)
    off = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    off[1:] = new.cumsum(0)
    src, dst = torch.where(copied, tail, -1), torch.full_like(tail, -1)
    dst[copied] = free[first[copied]]
    refs.index_add_(0, tail[copied], refs.new_full((int(copied.sum()),), -1))
    take = torch.repeat_interleave(torch.arange(n, device=DEV), need)
    i = torch.arange(take.numel(), device=DEV) - (need.cumsum(0) - need)[take]
    page = free[first[take] + i]
    table[take, held[take] + i - copied[take].long()] = page.to(torch.int32)
    refs[page] = 1
    t = torch.arange(tokens, device=DEV)
    seq = torch.searchsorted(off[1:], t, right=True)
    there, s = seq < n, seq.clamp(max=n - 1)
    pos = lens[s] + t - off[s]
    at = table[s, torch.where(there, pos // c, 0)].long()
    neg = lambda x: torch.where(there, x, -1)  # noqa: E731
    got = {"table": table, "refs": refs, "lens": (lens + new).to(torch.int32), "tok_off": off.to(torch.int32),
           "slots": neg(at * c + pos % c), "positions": neg(pos).to(torch.int32), "seqs": neg(seq).to(torch.int32),
           "copy_src": src.to(torch.int32), "copy_dst": dst.to(torch.int32)}
    got["counts"] = torch.stack([off[-1], need.sum(), free.numel() - need.sum(), (~fits).sum()]).to(torch.int32)
    return got


# ---- the definition, in 64 bits --------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"attn": _exact_attn, "select": _exact_select, "fork": _exact_fork,
            "extend": _exact_extend}[case["kind"]](st)


def _exact_attn(st):
    """Sequence by sequence and KV head by KV head, over all tokens of its own table's pages."""
    case, group = st["case"], st["case"]["hq"] // st["case"]["hkv"]
    table, lens, off = st["table"].cpu().numpy(), st["lens"].tolist(), st["tok_off"].tolist()
    outs = []
    for pool, q in zip(st["pools"], st["q"]):
        out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
        for b, (n0, n1) in enumerate(zip(off, off[1:])):
            entries = torch.from_numpy(table[b, : -(-lens[b] // case["page"])].astype(np.int64)).to(DEV)
            key = torch.arange(lens[b], device=DEV)
            hide = key > torch.arange(lens[b] - (n1 - n0), lens[b], device=DEV)[:, None]
            for h in range(case["hkv"]):
                def tokens(name):
                    x, s = pool[name].view(torch.uint8) if case["cache"] == "e4m3" else pool[name], pool[name + "_scale"]
                    x = x[:, :, h][entries].view(pool[name].dtype).double()
                    if s is not None:
                        x = x * 2.0 ** (s[:, h][entries].double() - 127)[:, None, None]
                    return x.reshape(-1, case["d"])[: lens[b]]
                k, v = tokens("k"), tokens("v")
                for i in range(group):
                    s = q[n0:n1, h * group + i].double() @ k.T / math.sqrt(case["d"])
                    out[n0:n1, h * group + i] = torch.softmax(s.masked_fill(hide, -1e300), -1) @ v
        outs.append(out)
    return outs


def _exact_select(st):
    """Beam by beam its best tokens, request by request the best of those; the scores alone."""
    case = st["case"]
    value = np.full((case["reqs"], case["keep"]), -np.inf)
    for r in range(case["reqs"]):
        found = []
        for b in range(case["beams"]):
            cum = float(st["scores"][r, b])
            if cum == -math.inf:
                continue
            if int(st["done"][r, b]):
                found.append(cum)
                continue
            p = torch.log_softmax(st["logits"][r, b].double(), 0)
            found += (p.topk(min(case["keep"], case["vocab"])).values + cum).tolist()
        found = sorted(found, reverse=True)[: case["keep"]]
        value[r, : len(found)] = found
    return {"parent": None, "token": None, "scores": torch.from_numpy(value), "done": None}


def _exact_fork(st):
    """Sequence by sequence on the host."""
    c, table, lens = st["case"]["page"], st["table"].cpu().numpy(), st["lens"].tolist()
    refs, old = st["refs"].cpu().numpy().astype(np.int64), st["history"].cpu().numpy()
    got = np.full_like(table, -1)
    length, history = np.zeros(len(lens), np.int64), np.zeros_like(old)
    for b, n in enumerate(lens):
        np.subtract.at(refs, table[b, : -(-n // c)], 1)
    for i, p in enumerate(st["parents"].tolist()):
        if p >= 0:
            k = -(-lens[p] // c)
            got[i, :k], length[i], history[i] = table[p, :k], lens[p], old[p]
            np.add.at(refs, got[i, :k], 1)
    return {"table": torch.from_numpy(got), "lens": torch.from_numpy(length), "refs": torch.from_numpy(refs),
            "history": torch.from_numpy(history)}


def _exact_extend(st):
    """Sequence by sequence on the host, page by page from a list of the free ones."""
    c, table, lens, new = st["case"]["page"], st["table"].cpu().numpy().copy(), st["lens"].tolist(), st["n_new"].tolist()
    before = st["refs"].tolist()
    refs, free = list(before), [p for p, r in enumerate(before) if r <= 0]
    at, asked, refused, slots, where, who, off, src, dst, out = 0, 0, 0, [], [], [], [0], [], [], []
    for b, n in enumerate(lens):
        fill = [j for j in range(-(-n // c), -(-(n + new[b]) // c))]
        if n % c and new[b] and before[table[b, n // c]] > 1:
            fill.insert(0, n // c)
        asked += len(fill)
        src.append(-1)
        dst.append(-1)
        count = new[b]
        if fill and asked > len(free):
            refused, count = refused + 1, 0
        else:
            for j in fill:
                if j == n // c and n % c:
                    src[-1], dst[-1] = int(table[b, j]), free[at]
                    refs[src[-1]] -= 1
                table[b, j] = free[at]
                refs[free[at]] = 1
                at += 1
        for pos in range(n, n + count):
            slots.append(int(table[b, pos // c]) * c + pos % c)
            where.append(pos)
            who.append(b)
        off.append(off[-1] + count)
        out.append(n + count)
    rest = [-1] * (st["tokens"] - off[-1])
    got = {"table": table, "refs": refs, "lens": out, "tok_off": off, "slots": slots + rest,
           "positions": where + rest, "seqs": who + rest, "copy_src": src, "copy_dst": dst,
           "counts": [off[-1], at, len(free) - at, refused]}
    return {k: torch.as_tensor(np.asarray(v)) for k, v in got.items()}
