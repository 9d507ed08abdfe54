"""The operators around a paged key-value cache that a serving program's step is made of, as cases to be timed and compared.

For every step such a program decides which pages of the pool each sequence holds and where each new token's rows go
("plan"); each layer turns the new queries and keys by their positions and puts keys and values where the cache takes them
("rope"); beam search picks the step's best continuations from the logits ("beam") and lets every beam go on from its
parent: tails, page tables and counts change places, and pages that several beams would now write get copies ("fork").

Positions.  Channel pair i of rot / 2 turns by w_i radians a position, w_i = base^(-2 i / rot) or a scaled form of it
(`_speeds`); a pair is channels (i, i + rot / 2) ("halves") or (2 i, 2 i + 1) ("pairs").  Channels from rot on stay.

Token map.  A record of four int32 per token of a packed batch: sequence, position, row among the cache's rows, row among
the queries' rows (-1: none).  Records behind the last token are (-1, 0, -1, -1).

Pages.  refs counts a page's users; a page without any is free, and the lowest free pages are given out first, to sequences
in order, entries in order.  A sequence that grows inside a page that others use as well gets a page of its own, to which
the rows it has are copied; where all users of a page grow, the first of them keeps it.
"""
import math
import random

import torch

own = False

D = 128
TILE = 64


def _rope(name, **kw):
    """B sequences with `new` tokens at most (ragged: down to a quarter), from position `first` (far: up to 2^20) on.

    cap      rows of a sequence in the cache's buffers;  row0: the first that is written, at most
    q_rows   rows of a sequence in the queries' buffer; 0: the queries stay token by token
    pad      tokens of the packed batch that belong to no sequence
    """
    c = dict(name=name, kind="rope", dtype="bf16", B=1, N_q=32, N_kv=8, new=1, ragged=False, far=False, cap=128, row0=0, q_rows=1,
             pad=0, layout="halves", rot=128, base=10000.0, scaling="plain", factor=1.0, trained=8192)
    c.update(kw)
    return c


def _plan(name, **kw):
    """B sequences of S rows at most, most of which get one row more, while some end and others begin.

    room     pages of the pool, in percent of what the sequences hold or ask for at most
    shared   every second sequence has its first pages in common with its neighbour;  pinned: percent of pages others use
    """
    c = dict(name=name, kind="plan", B=4, S=1000, page_rows=64, room=150, shared=False, pinned=5, cap=128, q_rows=1, pad=0)
    c.update(kw)
    return c


def _beam(name, **kw):
    """B prompts of W beams, a vocabulary of V; the K best continuations.  ld: elements from row to row of the logits.

    masked   share of the vocabulary, in percent, that may not follow (-inf);  done: beams that have ended already, percent
    """
    c = dict(name=name, kind="beam", dtype="bf16", B=1, W=4, K=8, V=32768, ld=0, masked=0, done=0)
    c.update(kw)
    return c


def _fork(name, **kw):
    """B prompts of W beams, S rows at most in pages (ragged) and `tail` in a tail buffer of cap rows, L layers."""
    c = dict(name=name, kind="fork", dtype="bf16", bits=4, L=1, B=1, W=4, N_q=32, N_kv=8, S=1024, T=64, ragged=False, page_rows=128,
             cap=128, tail=64)
    c.update(kw)
    return c


def listed():
    return [
        # One token of one conversation: latency.
        _rope("rope_b1", row0=38),
        # A decode step of a batch in fp32, neighbouring channels turned, half of each head, far positions at a raised base.
        _rope("rope_f32_pairs_b64_far", dtype="f32", B=64, N_q=8, far=True, row0=99, layout="pairs", rot=64, scaling="base", factor=8.0),
        # Ragged prompts packed side by side, an odd part of each head, ramped speeds; the observation window's queries kept.
        _rope("rope_ragged_rot44", B=7, new=333, ragged=True, cap=512, q_rows=32, pad=9, rot=44, scaling="ramp", factor=16.0),
        # Two long prompts of a model with eight query heads per KV head: the largest.
        _rope("rope_prefill_8192", B=2, N_q=64, new=8192, cap=8192, q_rows=0, base=500000.0, scaling="bands", factor=8.0),
        # A step of a small server: latency.
        _plan("plan_b4"),
        # A batch with shared prompts, some requests ending and some beginning, in a pool that runs out.
        _plan("plan_b200_short", B=200, S=16384, page_rows=128, room=90, shared=True, pinned=10, pad=100),
        # A large batch of long sequences over a pool of some 300000 small pages.
        _plan("plan_b1024_s32768", B=1024, S=32768, shared=True, q_rows=32, cap=32768),
        # Four beams of one prompt: latency.
        _beam("beam_b1_w4_v32768"),
        # Five beams each, an odd vocabulary in fp32, a third of it masked, rows padded, some beams at their end.
        _beam("beam_f32_b7_w5_v100003", dtype="f32", B=7, W=5, K=10, V=100003, ld=100032, masked=33, done=20),
        # A full batch of eight beams.
        _beam("beam_b64_w8_v131072", B=64, W=8, K=16, V=131072),
        # The beams of two short prompts change places, a layer's cache.
        _fork("fork_b2_w4", B=2),
        # A larger batch, eight layers in one call, ragged prompts, pages of 256 rows.
        _fork("fork_l8_b8_w8", L=8, B=8, W=8, S=4096, ragged=True, page_rows=256, tail=100),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """A case of the listed ones' ranges: tokens, pages, vocabularies and batches over their logarithm, any even part of a
    head, one to 32 beams."""
    while True:
        kind = rng.choice(["rope", "rope", "plan", "beam", "beam", "fork"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        if kind == "rope":
            group, heads = rng.choice([1, 2, 4, 7, 8]), rng.choice([1, 4, 8, 8, 40])
            new = rng.choice([1, 1, _log_int(rng, 2, 8192)])
            rot = rng.choice([128, 128, 64, 32, 2 * rng.randint(2, 64)])
            scaling = rng.choice(["plain", "linear", "base", "ramp", "bands"])
            c = _rope("", dtype=dtype, B=_log_int(rng, 1, 256), N_kv=heads, N_q=group * heads, new=new, ragged=rng.random() < 0.6,
                      far=rng.random() < 0.3, row0=rng.randint(0, 60), q_rows=rng.choice([0, 1 if new == 1 else 32]),
                      pad=rng.choice([0, 0, rng.randint(1, 60)]), layout=rng.choice(["halves", "halves", "pairs"]), rot=rot,
                      base=rng.choice([10000.0, 500000.0]), scaling=scaling, factor=1.0 if scaling == "plain" else rng.choice([2.0, 8.0, 40.0]),
                      trained=rng.choice([2048, 8192]))
            c["cap"] = c["row0"] + new - (rng.random() < 0.2 and new > 1)
        elif kind == "plan":
            c = _plan("", B=_log_int(rng, 1, 1024), S=_log_int(rng, 64, 32768), page_rows=rng.choice([64, 128, 256]),
                      room=rng.choice([80, 120, 300]), shared=rng.random() < 0.5, pinned=rng.choice([0, 5, 30]),
                      cap=rng.choice([64, 128, 4096]), q_rows=rng.choice([1, 32]), pad=rng.choice([0, rng.randint(1, 300)]))
        elif kind == "beam":
            beams = rng.choice([1, 2, 4, 5, 8, rng.randint(1, 32)])
            c = _beam("", dtype=dtype, B=_log_int(rng, 1, 64), W=beams, K=min(64, rng.choice([beams, 2 * beams])), V=_log_int(rng, 1000, 250000),
                      masked=rng.choice([0, 0, 33, 95]), done=rng.choice([0, 0, 30]))
            c["ld"] = rng.choice([0, 0, -(-c["V"] // 64) * 64])
        else:
            c = _fork("", dtype=dtype, bits=rng.choice([0, 4, 8]), L=rng.choice([1, 1, 4, 8]), B=_log_int(rng, 1, 16), W=rng.choice([2, 4, 5, 8, 16]),
                      N_kv=rng.choice([1, 4, 8]), S=_log_int(rng, 64, 8192), T=rng.randint(32, 128), ragged=rng.random() < 0.6,
                      page_rows=rng.choice([64, 128, 256]), cap=rng.choice([0, 64, 128]))
            c["N_q"] = c["N_kv"] * 4
            c["tail"] = rng.randint(0, c["cap"])
        del c["name"]
        w = work(c)["bytes"]
        if w < (700e6 if kind == "rope" else 400e6):
            return c


# ------------------------------------------------------------------------------- sizes

def _esize(c):
    return 4 if c["dtype"] == "f32" else 2


def _tdtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _shorter(n, b, c):
    return n - (n * 3 * b) // (4 * c["B"]) if c["ragged"] else n


def _news(c):
    return [_shorter(c["new"], b, c) for b in range(c["B"])]


def _plan_rows(c):
    """(rows held before, rows asked for, new tokens) of every sequence: one in ten ends, one in ten begins."""
    before, after, new = [], [], []
    for b in range(c["B"]):
        n = max(1, round(c["S"] * (((b + 1) * 7919) % 101 + 1) / 102))
        what = (b * 37 + 3) % 10
        before.append(0 if what == 1 else n)
        after.append(0 if what == 0 else n if what == 1 else min(n + (1, 1, 1, TILE)[b % 4], c["S"]))
        new.append(0 if what == 0 else max(1, n // 16) if what == 1 else 1)
    return before, after, new


def _pages(rows, page_rows):
    return -(-rows // page_rows)


def _plan_pool(c):
    before, after, _ = _plan_rows(c)
    return max(1, sum(max(_pages(a, c["page_rows"]), _pages(b, c["page_rows"])) for a, b in zip(before, after)) * c["room"] // 100)


def _tile_bytes(c):
    """Bytes that 64 rows of a KV head have in a page."""
    chunks, unit = (c["T"] + 7) // 8, c["bits"] if c["bits"] else 8 * _esize(c)
    return (chunks + 16) * 64 * unit + ((chunks * 8 + 2 * TILE) * 2 * _esize(c) if c["bits"] else 0)


def _fork_rows(c):
    """Rows in pages of each prompt's beams: whole tiles, and mostly no whole page."""
    return [max(1, _shorter(c["S"], b, c) // TILE) * TILE - (TILE if b % 3 == 0 and c["S"] > 2 * TILE else 0) for b in range(c["B"])]


def _fork_tails(c):
    return [_shorter(c["tail"], b, c) for b in range(c["B"])]


def work(case):
    """Each input read once, each output written once."""
    c = case
    if c["kind"] == "rope":
        n, kept = sum(_news(c)), sum(min(x, max(0, c["cap"] - c["row0"])) for x in _news(c))
        rows_q = sum(min(x, c["q_rows"] or x) for x in _news(c)) * c["N_q"]
        rows = kept * 2 * c["N_kv"] + rows_q
        return {"bytes": 2 * rows * D * _esize(c) + 16 * (n + c["pad"]), "flops": 3 * c["rot"] * (kept * c["N_kv"] + rows_q)}
    if c["kind"] == "plan":
        before, after, new = _plan_rows(c)
        changed = sum(abs(_pages(a, c["page_rows"]) - _pages(b, c["page_rows"])) for a, b in zip(before, after))
        return {"bytes": 4 * _plan_pool(c) + 12 * changed + 32 * c["B"] + 16 * (sum(new) + c["pad"]), "flops": 0}
    if c["kind"] == "beam":
        rows = c["B"] * c["W"] * (100 - c["done"]) / 100
        return {"bytes": rows * c["V"] * _esize(c) + 8 * c["B"] * (c["W"] + 2 * c["K"]), "flops": 4 * rows * c["V"]}
    # about two thirds of the beams change, and nearly every beam's last page is copied where it is not full
    units, moved = c["L"] * c["N_kv"], 0
    for s, t in zip(_fork_rows(c), _fork_tails(c)):
        moved += c["W"] * 2 / 3 * 2 * units * 2 * D * _esize(c) * t
        moved += (c["W"] - 1) * 2 * units * _tile_bytes(c) * (s % c["page_rows"] // TILE)
        moved += c["W"] * 12 * _pages(s, c["page_rows"])
    return {"bytes": moved + 1, "flops": 0}


# ------------------------------------------------------------------------------- inputs

def _generator(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _prepare_rope(c, seed):
    g, r, dt = _generator(c, seed), random.Random(seed), _tdtype(c)
    news = _news(c)
    n, width = sum(news) + c["pad"], (c["N_q"] + 2 * c["N_kv"]) * D
    first = [r.randint(1 << 18, 1 << 20) if c["far"] else r.randint(0, 5000) if c["new"] == 1 else 0 for _ in news]
    row0 = [r.randint(c["row0"] // 2, c["row0"]) for _ in news]
    # the map, which a program has from the step's plan
    seq = torch.repeat_interleave(torch.arange(c["B"]), torch.tensor(news))
    i = torch.arange(seq.numel()) - (torch.tensor(news).cumsum(0) - torch.tensor(news))[seq]
    row = torch.tensor(row0)[seq] + i
    q_row = i - (torch.tensor(news) - c["q_rows"])[seq]
    rec = torch.stack([seq, torch.tensor(first)[seq] + i, torch.where(row < c["cap"], row, -1), torch.where(q_row >= 0, q_row, -1)], dim=1)
    rec = torch.cat([rec, torch.tensor([[-1, 0, -1, -1]]).expand(c["pad"], 4)])
    st = {"c": c, "n": n, "map": rec.to(torch.int32).cuda().contiguous()}
    qkv = _randn(g, n, width).to(dt)          # a projection's output: queries, keys and values of a token side by side
    st["q"], st["k"], st["v"] = qkv.split([c["N_q"] * D, c["N_kv"] * D, c["N_kv"] * D], dim=1)
    st["q_out"] = _randn(g, *((n, c["N_q"], D) if c["q_rows"] == 0 else (c["B"], c["N_q"], c["q_rows"], D))).to(dt)
    st["k_out"], st["v_out"] = (_randn(g, c["B"], c["N_kv"], c["cap"], D).to(dt) for _ in range(2))
    return st


def _prepare_plan(c, seed):
    r = random.Random(seed)
    before, after, new = _plan_rows(c)
    pr, total, most = c["page_rows"], _plan_pool(c), _pages(c["S"], c["page_rows"])
    order = list(range(total))
    r.shuffle(order)
    refs, table, held, at = [0] * total, [], [], 0
    for b, n in enumerate(before):
        want, row = _pages(n, pr), []
        if c["shared"] and b % 2 and want:
            row = table[b - 1][:min(held[b - 1], want) // 2]
        take = order[at:at + want - len(row)]
        at += len(take)
        row = row + take
        for p in row:
            refs[p] += 1
        held.append(len(row))
        table.append(row + [-1] * (most - len(row)))
    for p in order[at:at + total * c["pinned"] // 100]:
        refs[p] = r.randint(1, 3)
    st = {"c": c, "pass": 0, "rows": [_ints(after), _ints(before)], "n_pages": total, "n": sum(new) + c["pad"]}
    st["table"], st["held"], st["refs"] = _ints(table), _ints(held), _ints(refs)
    st["room"] = torch.zeros(c["B"], dtype=torch.int32, device="cuda")
    st["new"], st["first"] = _ints(new), _ints([r.randint(0, 3) + x for x in before])
    st["row0"] = _ints([r.randint(0, TILE - 1) for _ in before])
    st["map"] = torch.zeros(st["n"], 4, dtype=torch.int32, device="cuda")
    st["starts"] = torch.zeros(c["B"] + 1, dtype=torch.int32, device="cuda")
    return st


def _prepare_beam(c, seed):
    g = _generator(c, seed)
    rows, ld = c["B"] * c["W"], c["ld"] or c["V"]
    x = _randn(g, rows, ld) * 2
    x += 6 * (torch.rand(rows, ld, generator=g, device="cuda") < 20.0 / ld)      # a few continuations that are likely
    if c["masked"]:
        x = x.masked_fill(torch.rand(rows, ld, generator=g, device="cuda") < c["masked"] / 100, float("-inf"))
    st = {"c": c, "logits": x.to(_tdtype(c)).reshape(c["B"], c["W"], ld)}
    st["scores"] = -20 * torch.rand(c["B"], c["W"], generator=g, device="cuda")
    st["done"] = (torch.rand(c["B"], c["W"], generator=g, device="cuda") < c["done"] / 100).to(torch.int32)
    st["parent"], st["token"], st["done_out"] = (torch.zeros(c["B"], c["K"], dtype=torch.int32, device="cuda") for _ in range(3))
    st["score_out"] = torch.zeros(c["B"], c["K"], device="cuda")
    return st


def _prepare_fork(c, seed):
    g, r, dt = _generator(c, seed), random.Random(seed), _tdtype(c)
    pr, W, seqs = c["page_rows"], c["W"], c["B"] * c["W"]
    rows, tails = ([x for x in v for _ in range(W)] for v in (_fork_rows(c), _fork_tails(c)))
    most = _pages(max(rows) + TILE, pr)
    total = sum(_pages(s, pr) for s in _fork_rows(c)) + 2 * seqs + 3
    order = list(range(total))
    r.shuffle(order)
    refs, table, held, at = [0] * total, [], [], 0
    for b, n in enumerate(rows):      # a prompt's full pages belong to all its beams, the last one to each beam alone
        full = n // pr
        if b % W == 0:
            common, at = order[at:at + full], at + full
        row = list(common)
        if n % pr:
            row, at = row + [order[at]], at + 1
        for p in row:
            refs[p] += 1
        held.append(len(row))
        table.append(row + [-1] * (most - len(row)))
    st = {"c": c, "n_pages": total, "table": _ints(table), "held": _ints(held), "refs": _ints(refs)}
    st["s_pages"], st["s_tail"] = _ints(rows), _ints(tails)
    st["grown"] = _ints([n + TILE for n in rows])       # each beam's next tile is about to be stored
    st["room"] = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    st["moves"] = torch.zeros(seqs, 4, dtype=torch.int32, device="cuda")
    # two beams in three go on from another one; 2 W candidates, of which the first W are taken
    st["parent"] = _ints([[j if r.random() < 1 / 3 else r.randrange(W) for j in range(W)] + [0] * W for _ in range(c["B"])])
    tile = (c["L"], total, c["N_kv"], pr // TILE, _tile_bytes(c))
    st["pool"] = torch.randint(0, 256, tile, generator=g, device="cuda", dtype=torch.uint8)
    if c["cap"]:
        st["k_tail"], st["v_tail"] = (_randn(g, c["L"], seqs, c["N_kv"], c["cap"], D).to(dt) for _ in range(2))
    return st


def prepare(case, seed):
    return {"rope": _prepare_rope, "plan": _prepare_plan, "beam": _prepare_beam, "fork": _prepare_fork}[case["kind"]](case, seed)


# ------------------------------------------------------------------------------- the calls

def _setup(st):
    """What a program makes once: descriptions, the table of speeds, workspaces."""
    import paper_2407_21018_amd as thk
    c = st["c"]
    st["thk"] = thk
    bytes_ = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")  # noqa: E731
    if c["kind"] == "beam":
        st["beams"] = thk.make_beams(c["B"], c["W"], c["K"], c["V"], c["ld"], thk.THK_F32 if c["dtype"] == "f32" else thk.THK_BF16, 2)
        st["ws"] = bytes_(thk.thk_beam_workspace_bytes(st["beams"]))
        return
    dtype = thk.THK_F32 if c.get("dtype") == "f32" else thk.THK_BF16
    seqs = c["B"] * c.get("W", 1)
    st["shape"] = thk.make_shape(c.get("L", 1), seqs, c.get("N_q", 1), c.get("N_kv", 1), D, c.get("S", 1) + TILE, 1, c.get("T", D), 0, dtype)
    if c["kind"] == "rope":
        layout = {"halves": thk.THK_ROPE_HALVES, "pairs": thk.THK_ROPE_PAIRS}[c["layout"]]
        scaling = {"plain": thk.THK_ROPE_PLAIN, "linear": thk.THK_ROPE_LINEAR, "base": thk.THK_ROPE_BASE, "ramp": thk.THK_ROPE_RAMP,
                   "bands": thk.THK_ROPE_BANDS}[c["scaling"]]
        st["rope"] = thk.make_rope(layout, c["rot"], scaling, c["trained"], c["base"], c["factor"], *_TURNS[c["scaling"]])
        st["turns"] = torch.tensor(thk.thk_rope_turns(st["rope"]), dtype=torch.int64, device="cuda")
        return
    st["pages"] = thk.make_pages(c.get("bits", 4), c["page_rows"], st["table"].shape[1], st["n_pages"])
    st["ws"] = bytes_(thk.thk_workspace_bytes(st["shape"], thk.THK_OP_PAGED_RESERVE))


def _own_rope(st):
    c, ld = st["c"], st["q"].stride(0)
    st["thk"].thk_rope_qkv(st["shape"], st["rope"], st["turns"], st["q"], ld, st["k"], ld, st["v"], ld, st["map"], st["n"], st["q_out"],
                           c["q_rows"], st["k_out"], st["v_out"], c["cap"])
    return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}


def _own_plan(st):
    c, thk = st["c"], st["thk"]
    rows = st["rows"][st["pass"]]
    st["pass"] ^= 1
    thk.thk_paged_reserve(st["shape"], st["pages"], rows, None, st["held"], st["table"], st["refs"], st["room"], None, st["ws"])
    thk.thk_token_map(st["shape"], st["new"], st["first"], st["row0"], c["cap"], c["q_rows"], st["map"], st["n"], st["starts"])
    return {n: st[n] for n in ("table", "held", "refs", "room", "map", "starts")}


def _own_beam(st):
    st["thk"].thk_beam_select(st["beams"], st["logits"], st["scores"], st["done"], st["parent"], st["token"], st["score_out"], st["done_out"], st["ws"])
    return {n: st[n] for n in ("parent", "token", "score_out", "done_out")}


def _own_fork(st):
    c, thk = st["c"], st["thk"]
    thk.thk_beam_reorder(st["shape"], st["pages"], c["W"], st["parent"], 2 * c["W"], st.get("k_tail"), st.get("v_tail"), st["s_tail"], c["cap"],
                         st["s_pages"], st["held"], st["table"], st["refs"])
    thk.thk_paged_reserve(st["shape"], st["pages"], st["grown"], st["s_pages"], st["held"], st["table"], st["refs"], st["room"], st["moves"], st["ws"])
    thk.thk_paged_copy(st["shape"], st["pages"], st["moves"], st["moves"].shape[0], st["pool"])
    return {n: st[n] for n in _FORKED if n in st}


_FORKED = ("k_tail", "v_tail", "s_tail", "s_pages", "held", "table", "refs", "room", "moves", "pool")


# ------------------------------------------------------------------------------- the plain forms

_TURNS = {"plain": (0.0, 0.0), "linear": (0.0, 0.0), "base": (0.0, 0.0), "ramp": (1.0, 32.0), "bands": (1.0, 4.0)}


def _speeds(c):
    """Radians a position of every pair, in 64 bits, and what turned channels are multiplied by.

    linear   all slower by the factor
    base     the base raised to base factor^(rot / (rot - 2))
    ramp     r = turns of a pair over the trained length; pairs below the index where r is `high` keep their speed, those above
             the index where it is `low` are slower by the factor, a line over the indexes between; times 0.1 ln(factor) + 1
    bands    pairs with r above `high` keep their speed, below `low` are slower by the factor, a line over r between
    """
    half, base, f = c["rot"] // 2, c["base"], c["factor"]
    low, high = _TURNS[c["scaling"]]
    if c["scaling"] == "base":
        base = base * f ** (c["rot"] / (c["rot"] - 2))
    i = torch.arange(half, dtype=torch.float64, device="cuda")
    w = torch.exp(i * (-2.0 / c["rot"] * math.log(base)))
    if c["scaling"] == "linear":
        return w / f, 1.0
    if c["scaling"] == "ramp":
        at = lambda turns: c["rot"] * math.log(c["trained"] / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), c["rot"] - 1)
        slow = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        return w / f * slow + w * (1 - slow), 0.1 * math.log(f) + 1
    if c["scaling"] == "bands":
        r = c["trained"] * w / (2 * math.pi)
        keep = ((r - low) / (high - low)).clamp(0, 1)
        return w / f * (1 - keep) + w * keep, 1.0
    return w, 1.0


def _turn(x, cos, sin, c):
    """x [n, heads, D] in 32 bits, cos and sin [n, 1, rot / 2]."""
    half, rot = c["rot"] // 2, c["rot"]
    a, b = (x[..., :half], x[..., half:rot]) if c["layout"] == "halves" else (x[..., 0:rot:2], x[..., 1:rot:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([a, b], dim=-1) if c["layout"] == "halves" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _place(buffer, x, seq, row):
    """Rows x [n, heads, D] to buffer [B, heads, rows, D]; tokens with seq or row < 0 go nowhere (to a row behind the last)."""
    B, heads, rows, _ = buffer.shape
    live = (seq >= 0) & (row >= 0)
    flat = torch.cat([buffer.transpose(1, 2).reshape(B * rows, heads, D), buffer.new_zeros(1, heads, D)])
    flat[torch.where(live, seq * rows + row, B * rows)] = x
    buffer.copy_(flat[:-1].reshape(B, rows, heads, D).transpose(1, 2))


def _plain_rope(st):
    c, dt, n = st["c"], _tdtype(st["c"]), st["n"]
    seq, pos, row, q_row = st["map"].long().unbind(1)
    w, gain = _speeds(c)
    angle = (pos.double()[:, None] * w)[:, None]
    cos, sin = (gain * torch.cos(angle)).float(), (gain * torch.sin(angle)).float()
    q, k, v = (st[x].reshape(n, -1, D) for x in "qkv")
    q = _turn(q.float(), cos, sin, c).to(dt)
    if c["q_rows"] == 0:
        st["q_out"].copy_(torch.where((seq >= 0)[:, None, None], q, st["q_out"]))
    else:
        _place(st["q_out"], q, seq, q_row)
    _place(st["k_out"], _turn(k.float(), cos, sin, c).to(dt), seq, row)
    _place(st["v_out"], v, seq, row)
    return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}


def _reserve(st, rows, now, page_rows):
    """rows [B]: what each sequence has to have pages for; now: rows that it has written, or None."""
    table, refs, n_pages = st["table"].long(), st["refs"].long(), st["refs"].numel()
    most = table.shape[1]
    held, e = st["held"].long(), torch.arange(most, device="cuda")
    need = ((rows.long() + page_rows - 1) // page_rows).clamp(max=most)
    gone = (e >= need[:, None]) & (e < held[:, None])
    refs = refs.index_add(0, torch.where(gone, table, 0).flatten(), -gone.long().flatten())
    table = torch.where(gone, -1, table)
    have = torch.minimum(held, need)
    moves = torch.zeros_like(have, dtype=torch.bool)
    if now is not None:
        at = now.long() // page_rows
        grows = (now > 0) & (rows > now) & (now % page_rows != 0) & (at < have)
        page = table.gather(1, at.clamp(max=most - 1)[:, None])[:, 0].clamp(min=0)
        growers = torch.zeros_like(refs).index_add(0, page, grows.long())
        b = torch.arange(have.numel(), device="cuda")
        first = torch.full_like(refs, have.numel()).scatter_reduce(0, page, torch.where(grows, b, have.numel()), "amin")
        moves = grows & ~((growers[page] >= refs[page]) & (first[page] == b))
    want = moves.long() + (need - have).clamp(min=0)
    ends = want.cumsum(0)
    free = refs <= 0
    rank = free.long().cumsum(0)
    n_free = rank[-1]
    find = lambda k: torch.searchsorted(rank, k + 1).clamp(max=n_pages - 1)  # noqa: E731
    k = (ends - want + moves.long() - have)[:, None] + e
    got = (e >= have[:, None]) & (e < need[:, None]) & (k < n_free)
    table = torch.where(got, find(k.clamp(min=0).contiguous()), table)
    refs = torch.where(free, torch.where(rank <= ends[-1], 1, 0), refs)
    room = (have + got.sum(1)) * page_rows
    if now is not None:
        k = ends - want
        moved = moves & (k < n_free)
        dst = find(k)
        refs = refs.index_add(0, page, -moved.long())
        table = torch.where((e == at[:, None]) & moved[:, None], dst[:, None], table)
        room = torch.where(moves & ~moved, now.long(), room)
        st["moves"].copy_(torch.stack([torch.where(moved, page, -1), torch.where(moved, dst, -1),
                                       torch.where(moved, (now % page_rows + TILE - 1) // TILE, 0), torch.zeros_like(page)], dim=1))
    st["table"].copy_(table)
    st["refs"].copy_(refs)
    st["held"].copy_(have + got.sum(1))
    st["room"].copy_(room)


def _plain_plan(st):
    c = st["c"]
    _reserve(st, st["rows"][st["pass"]], None, c["page_rows"])
    st["pass"] ^= 1
    new, t = st["new"].long(), torch.arange(st["n"], device="cuda")
    ends = new.cumsum(0)
    st["starts"].copy_(torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=st["n"]))
    seq = torch.searchsorted(ends, t, right=True)
    live = seq < c["B"]
    s = seq.clamp(max=c["B"] - 1)
    i = t - (ends - new)[s]
    row, q_row = st["row0"].long()[s] + i, i - (new[s] - c["q_rows"])
    record = torch.stack([s, st["first"].long()[s] + i, torch.where(row < c["cap"], row, -1), torch.where(q_row >= 0, q_row, -1)], dim=1)
    st["map"].copy_(torch.where(live[:, None], record, _ints([-1, 0, -1, -1]).long()))
    return {n: st[n] for n in ("table", "held", "refs", "room", "map", "starts")}


def _plain_beam(st):
    c = st["c"]
    B, W, V, K, eos = c["B"], c["W"], c["V"], c["K"], 2
    x = st["logits"][..., :V].reshape(B * W, V).float()
    top = x.amax(1, keepdim=True)
    total = torch.exp(x.double() - top.double()).sum(1)
    # a beam's best continuations, by logit and then by the lower token: a key that has both
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long()
    key = (bits << 24) | (0xffffff - torch.arange(V, device="cuda"))
    token = 0xffffff - (torch.topk(key, min(K, V), dim=1).values & 0xffffff)
    score = st["scores"].reshape(-1, 1).double() + ((x.gather(1, token).double() - top.double()) - torch.log(total)[:, None])
    # one that has ended goes on as it is
    done = st["done"].reshape(-1, 1) != 0
    first = torch.arange(token.shape[1], device="cuda") == 0
    token = torch.where(done, eos, token)
    score = torch.where(done, torch.where(first, st["scores"].reshape(-1, 1).double(), float("-inf")), score)
    score = torch.where(score.isfinite(), score, float("-inf")).reshape(B, -1)
    at = (torch.arange(W, device="cuda")[:, None] * V + token.reshape(B, W, -1)).reshape(B, -1)
    # the best of all beams, equal scores by beam and token
    at, by = at.sort(dim=1)
    score, by = score.gather(1, by).sort(dim=1, descending=True, stable=True)
    at = at.gather(1, by)
    if at.shape[1] < K:
        at, score = (torch.nn.functional.pad(y, (0, K - y.shape[1]), value=z) for y, z in ((at, 0), (score, float("-inf"))))
    at, score = at[:, :K], score[:, :K]
    some = score > float("-inf")
    parent, token = at // V, at % V
    st["done_out"].copy_(some & ((token == eos) | (st["done"].gather(1, parent) != 0)))
    st["parent"].copy_(torch.where(some, parent, -1))
    st["token"].copy_(torch.where(some, token, -1))
    st["score_out"].copy_(score)
    return {n: st[n] for n in ("parent", "token", "score_out", "done_out")}


def _plain_fork(st):
    c, pr = st["c"], st["c"]["page_rows"]
    W, seqs = c["W"], c["B"] * c["W"]
    j = torch.arange(seqs, device="cuda")
    parent = (torch.arange(c["B"], device="cuda")[:, None] * W + st["parent"][:, :W]).reshape(-1)
    other = parent != j
    if c["cap"]:
        taken = (torch.arange(c["cap"], device="cuda") < st["s_tail"][parent][:, None]) & other[:, None]
        for tail in (st["k_tail"], st["v_tail"]):
            tail.copy_(torch.where(taken[None, :, None, :, None], tail[:, parent], tail))
    # pages: a beam that changes gives up its own and uses those of its parent that hold rows
    table, held, refs = st["table"].long(), st["held"].long(), st["refs"].long()
    e = torch.arange(table.shape[1], device="cuda")
    rows = st["s_pages"].long()
    keep = torch.where(other, torch.minimum(held, (rows + pr - 1) // pr)[parent], held)
    mine, theirs = other[:, None] & (e < held[:, None]), other[:, None] & (e < keep[:, None])
    refs = refs.index_add(0, torch.where(mine, table, 0).flatten(), -mine.long().flatten())
    new = torch.where(other[:, None], torch.where(e < keep[:, None], table[parent], -1), table)
    st["refs"].copy_(refs.index_add(0, torch.where(theirs, new, 0).flatten(), theirs.long().flatten()))
    st["table"].copy_(new)
    st["held"].copy_(keep)
    st["s_pages"].copy_(rows[parent])
    st["s_tail"].copy_(st["s_tail"][parent])
    _reserve(st, st["grown"], st["s_pages"], pr)
    # each page that has to be a beam's own: the tiles that hold rows
    src, dst, tiles, _ = st["moves"].long().unbind(1)
    pool, none = st["pool"], st["pool"].shape[1]
    copied = (torch.arange(pool.shape[3], device="cuda") < tiles[:, None])[None, :, None, :, None]
    pages = torch.where(copied, pool[:, src.clamp(min=0)], pool[:, dst.clamp(min=0)])
    more = torch.cat([pool, pool[:, :1]], dim=1)
    more[:, torch.where(dst >= 0, dst, none)] = pages
    pool.copy_(more[:, :none])
    return {n: st[n] for n in _FORKED if n in st}


def run(state):
    kind = state["c"]["kind"]
    if own:
        if "thk" not in state:
            _setup(state)
        return {"rope": _own_rope, "plan": _own_plan, "beam": _own_beam, "fork": _own_fork}[kind](state)
    return {"rope": _plain_rope, "plan": _plain_plan, "beam": _plain_beam, "fork": _plain_fork}[kind](state)


# ------------------------------------------------------------------------------- in 64 bits

def _exact_rope(c, seed):
    st = prepare(c, seed)
    rot, f = c["rot"], c["factor"]
    speeds, gain = [], 1.0
    for i in range(rot // 2):
        w = c["base"] ** (-2.0 * i / rot)
        turns = c["trained"] * w / (2 * math.pi)
        if c["scaling"] == "linear":
            w /= f
        elif c["scaling"] == "base":
            w = (c["base"] * f ** (rot / (rot - 2.0))) ** (-2.0 * i / rot)
        elif c["scaling"] == "bands":
            part = 0.0 if turns < 1 else 1.0 if turns > 4 else (turns - 1) / 3
            w = (1 - part) * w / f + part * w
        elif c["scaling"] == "ramp":
            index = [rot * math.log(c["trained"] / (2 * math.pi * t)) / (2 * math.log(c["base"])) for t in (32.0, 1.0)]
            lo, hi = max(0, math.floor(index[0])), min(rot - 1, math.ceil(index[1]))
            part = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            w = part * w / f + (1 - part) * w
            gain = 1 + math.log(f) / 10
        speeds.append(w)
    seq, pos, row, q_row = (x.cpu() for x in st["map"].long().unbind(1))
    angle = pos.cuda().double()[:, None] * torch.tensor(speeds, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, gain), angle)[:, None]                # complex, [n, 1, pairs]
    out = {n: st[n + "_out"].double() for n in "qkv"}
    for name in "qkv":
        x = st[name].double().reshape(st["n"], -1, D)
        if name != "v":
            part = x[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2) if c["layout"] == "halves" else x[..., :rot].unflatten(-1, (-1, 2))
            part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn)
            x[..., :rot] = (part.transpose(-1, -2) if c["layout"] == "halves" else part).flatten(-2)
        if name == "q" and c["q_rows"] == 0:
            live = (seq >= 0).nonzero()[:, 0].cuda()
            out["q"][live] = x[live]
            continue
        to = q_row if name == "q" else row
        live = ((seq >= 0) & (to >= 0)).nonzero()[:, 0]
        out[name][seq[live].cuda(), :, to[live].cuda()] = x[live.cuda()]
    return out


def _exact_reserve(table, held, refs, rows, now, pr, most):
    """The bookkeeping, step by step on lists, in place; (room, moves)."""
    B = len(rows)
    need = [min(-(-r // pr), most) for r in rows]
    for b in range(B):
        while held[b] > need[b]:
            held[b] -= 1
            refs[table[b][held[b]]] -= 1
            table[b][held[b]] = -1
    growers = {}
    for b in range(B if now is not None else 0):
        if 0 < now[b] < rows[b] and now[b] % pr and now[b] // pr < held[b]:
            growers.setdefault(table[b][now[b] // pr], []).append(b)
    moving = {b for p, users in growers.items() for b in (users[1:] if len(users) >= refs[p] else users)}
    free = [p for p, r in enumerate(refs) if r <= 0]
    for p in free:
        refs[p] = 0
    free.reverse()
    room, moves = [], []
    for b in range(B):
        move, stuck = [-1, -1, 0, 0], False
        if b in moving:
            if free:
                e = now[b] // pr
                move = [table[b][e], free.pop(), -(-(now[b] % pr) // TILE), 0]
                refs[move[0]] -= 1
                refs[move[1]] = 1
                table[b][e] = move[1]
            else:
                stuck = True
        while held[b] < need[b] and free:
            table[b][held[b]] = free.pop()
            refs[table[b][held[b]]] = 1
            held[b] += 1
        room.append(now[b] if stuck else held[b] * pr)
        moves.append(move)
    return room, moves


def _exact_plan(c, seed):
    st = prepare(c, seed)
    table, held, refs = (st[n].tolist() for n in ("table", "held", "refs"))
    room, _ = _exact_reserve(table, held, refs, st["rows"][0].tolist(), None, c["page_rows"], st["table"].shape[1])
    starts, records = [0], []
    for b, (n, first, row0) in enumerate(zip(st["new"].tolist(), st["first"].tolist(), st["row0"].tolist())):
        for i in range(n):
            records.append([b, first + i, row0 + i if row0 + i < c["cap"] else -1, max(-1, i - n + c["q_rows"])])
        starts.append(len(records))
    records += [[-1, 0, -1, -1]] * (st["n"] - len(records))
    return {n: _ints(v) for n, v in (("table", table), ("held", held), ("refs", refs), ("room", room), ("map", records), ("starts", starts))}


def _exact_beam(c, seed):
    st = prepare(c, seed)
    V, K, out = c["V"], c["K"], {"parent": [], "token": [], "score_out": [], "done_out": []}
    for b in range(c["B"]):
        x = torch.log_softmax(st["logits"][b, :, :V].double(), dim=1) + st["scores"][b].double()[:, None]
        ended = st["done"][b].bool()
        x[ended] = float("-inf")
        x[ended, 2] = st["scores"][b][ended].double()
        score, at = torch.sort(x.flatten(), descending=True, stable=True)
        score, at = (torch.nn.functional.pad(y[:K], (0, max(0, K - y.numel())), value=z) for y, z in ((score, float("-inf")), (at, 0)))
        none = ~score.isfinite()
        parent, token = at // V, at % V
        out["done_out"].append(((token == 2) | ended[parent]) & ~none)
        out["parent"].append(parent.masked_fill(none, -1))
        out["token"].append(token.masked_fill(none, -1))
        out["score_out"].append(score.masked_fill(none, float("-inf")))
    return {n: torch.stack(v).to(torch.float64 if n == "score_out" else torch.int32) for n, v in out.items()}


def _exact_fork(c, seed):
    st = prepare(c, seed)
    W, pr = c["W"], c["page_rows"]
    table, held, refs, rows, tails = (st[n].tolist() for n in ("table", "held", "refs", "s_pages", "s_tail"))
    old_table, old_held, old_rows, old_tails = [list(t) for t in table], list(held), list(rows), list(tails)
    out = {}
    for n in ("k_tail", "v_tail"):
        if n in st:
            out[n] = st[n].double()
    for b, parents in enumerate(st["parent"].tolist()):
        for j in range(W):
            me, from_ = b * W + j, b * W + parents[j]
            if me == from_:
                continue
            for n in out:
                out[n][:, me, :, :old_tails[from_]] = st[n][:, from_, :, :old_tails[from_]].double()
            for p in old_table[me][:old_held[me]]:
                refs[p] -= 1
            rows[me], tails[me] = old_rows[from_], old_tails[from_]
            held[me] = min(old_held[from_], -(-rows[me] // pr))
            table[me] = old_table[from_][:held[me]] + [-1] * (len(table[me]) - held[me])
            for p in table[me][:held[me]]:
                refs[p] += 1
    room, moves = _exact_reserve(table, held, refs, st["grown"].tolist(), rows, pr, len(table[0]))
    pool = st["pool"].clone()
    for src, dst, tiles, _ in moves:
        if dst >= 0:
            pool[:, dst, :, :tiles] = st["pool"][:, src, :, :tiles]
    out |= {n: _ints(v) for n, v in (("s_tail", tails), ("s_pages", rows), ("held", held), ("table", table), ("refs", refs), ("room", room), ("moves", moves))}
    return {n: out[n] for n in _FORKED if n in out} | {"pool": pool}


def exact(case, seed):
    """The results in 64 bits, whole numbers among them."""
    return {"rope": _exact_rope, "plan": _exact_plan, "beam": _exact_beam, "fork": _exact_fork}[case["kind"]](case, seed)
