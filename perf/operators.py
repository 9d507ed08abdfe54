"""The operators of a paged, channel-pruned, optionally quantised key-value cache, as cases to be timed and compared.

A serving program whose sequences differ in length keeps its caches in pages: a pool of equal pages, a table of page
numbers per sequence, a row count per sequence.  It stores a prompt's keys (kept channels only) and values there, in the
element type or as 4-bit or 8-bit codes, and reads them back when a prompt is continued; for every new token it appends
the token's key and value to the sequence's full-width tail and attends over both.  The cases are those calls: "store"
(written, then read back), "append", and "decode".

Codes.  A tile is 64 rows of one KV head.  A group is a kept key channel over a tile's rows, or one half (64 channels) of
one value row.  With N = 2^bits - 1 codes above zero, m = min x, the scale s = (max x - m) / N, held in the element type, and
the code of x is (x - m) / s rounded to the nearest integer (ties to even), at most N, 0 where s is 0.  The difference,
the quotient and the range are rounded to 32 bits before they are used.  A code stands for m + c s.

A tile's bytes: key codes, value codes, key parameters, value parameters.  Codes lie in units of eight (8 kept channels of a
row; 8 rows of a value channel) and units in groups of 64; `_pack` is the arrangement.
"""
import torch

own = False

D = 128
TILE = 64


def _case(name, kind, **kw):
    """A case with every field present.

    kind          "store", "append" or "decode"
    bits          0: pages in the element type; 4 or 8: codes
    L, B          layers of the call and sequences;  N_q, N_kv: query and key heads;  T: kept key channels
    S             rows of the longest sequence;  ragged: the others are shorter, down to a quarter
    page_rows     rows of a page
    cap, tail     rows of a tail buffer, and those in use by the fullest sequence (ragged: the others hold fewer)
    new           "append": rows that come from the source (1: a token; more: what of a prompt fills no tile)
    """
    c = dict(name=name, kind=kind, dtype="bf16", bits=4, L=1, B=1, N_q=32, N_kv=8, S=4096, T=64, ragged=False,
             page_rows=64, cap=0, tail=0, new=1)
    c.update(kw)
    return c


def listed():
    return [
        # The end of one short prompt, a layer at a time: latency.  1000 rows end inside a tile.
        _case("store_i4_b1_s1000", "store", S=1000, page_rows=128),
        # A batch of ragged prompts in fp32, 8-bit codes, at the smallest workload's heads and length.
        _case("store_i8_f32_b4_s2048", "store", dtype="f32", bits=8, B=4, N_q=8, S=2048, ragged=True),
        # Pages in the element type with rows of an odd width (lambda = 0.6), one length short of a power of two.
        _case("store_16_b8_s8191", "store", bits=0, B=8, S=8191, T=51, page_rows=256),
        # The end of prefill of a multi-head model, all its layers in one call (lambda = 0.4).
        _case("store_i4_l32_mha_s4096", "store", L=32, N_kv=32, S=4096, T=76),
        # One token of one sequence.
        _case("append_b1", "append", cap=128, tail=38),
        # What the prompts of a large ragged batch leave over when their whole tiles are in pages.
        _case("append_rest_l8_b64", "append", L=8, B=64, cap=128, tail=0, new=63, ragged=True),
        # One token of one short conversation over element-type pages: latency.
        _case("decode_16_b1_s1000", "decode", bits=0, S=1000, page_rows=128, cap=128, tail=38),
        # One layer's attention at the smallest workload, fp32 with 8-bit codes.
        _case("decode_i8_f32_s2048", "decode", dtype="f32", bits=8, N_q=8, S=2048),
        # A ragged multi-head batch, lambda = 0.6 (51 channels), a full tail.
        _case("decode_i4_mha_b16_s8192", "decode", B=16, N_q=40, N_kv=40, S=8192, T=51, ragged=True, cap=64, tail=64),
        # Eight query heads per KV head as in a 70B model, 8-bit codes, ragged.
        _case("decode_i8_gqa8_s8191", "decode", bits=8, B=8, N_q=64, S=8191, T=76, ragged=True, page_rows=256, cap=64, tail=33),
        # One very long prompt in element-type pages: the work is split over the length.
        _case("decode_16_gqa4_s131072", "decode", bits=0, S=131072, page_rows=256, cap=128, tail=17),
        # A full batch of long prompts, 4-bit codes: the largest.
        _case("decode_i4_gqa4_b32_s32768", "decode", B=32, S=32768, page_rows=128, cap=128, tail=100),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """A case of the listed ones' ranges: lengths from one row on and batch sizes over their logarithm, any count of kept
    channels from 32 to 128, one to eight query heads per KV head."""
    while True:
        kind = rng.choice(["store", "store", "append", "decode", "decode", "decode"])
        group = rng.choice([1, 1, 2, 4, 4, 5, 7, 8])
        heads = rng.choice([8, 8, 32, 40] if group == 1 else [4, 8, 8])
        c = _case("", kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), bits=rng.choice([0, 4, 4, 8]), N_kv=heads,
                  N_q=group * heads, B=_log_int(rng, 1, 64), S=_log_int(rng, 1 if rng.random() < 0.2 else 200, 131072),
                  ragged=rng.random() < 0.6, page_rows=rng.choice([64, 128, 256]), T=rng.choice([51, 64, 76, rng.randint(32, 128)]))
        del c["name"]
        c["cap"] = rng.choice([64, 64, 128]) if kind == "append" or rng.random() < 0.7 else 0
        if kind == "append":
            c["L"], c["new"] = rng.choice([1, 1, 8, 32]), rng.choice([1, 1, rng.randint(2, 63)])
            c["tail"] = rng.randint(0, c["cap"] - c["new"])
            c["S"] = TILE
        elif c["cap"]:
            c["tail"] = rng.randint(1, c["cap"])
        if kind == "store":
            c["L"] = rng.choice([1, 1, 4, 32])
            c["cap"] = c["tail"] = 0
        rows = c["L"] * c["B"] * c["N_kv"] * c["S"]
        if rows * (c["dtype"] == "f32" and 2 or 1) > (4 << 20 if kind == "store" else 8 << 20):
            continue
        return c


# ------------------------------------------------------------------------------- sizes

def _esize(c):
    return 4 if c["dtype"] == "f32" else 2


def _tdtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _shorter(n, b, c):
    """Row count of sequence b where the first has n: down to a quarter of it when ragged."""
    return n - (n * 3 * b) // (4 * c["B"]) if c["ragged"] else n


def _lengths(c):
    return [_shorter(c["S"], b, c) for b in range(c["B"])]


def _tails(c):
    return [_shorter(c["tail"], b, c) for b in range(c["B"])]


def _news(c):
    return [_shorter(c["new"], b, c) for b in range(c["B"])]


def _row_bytes(c):
    """Bytes of a row in a page, its share of the parameters included."""
    if c["bits"] == 0:
        return (c["T"] + D) * _esize(c)
    return (c["T"] + D) * c["bits"] / 8 + 2 * _esize(c) * (c["T"] / TILE + 2)


def work(case):
    """Each input read once, each output written once; a multiply-add is two operations."""
    c, e = case, _esize(case)
    units = c["L"] * c["N_kv"]
    rows = units * sum(_lengths(c))
    idx = c["L"] * c["B"] * c["N_kv"] * c["T"] * 2
    if c["kind"] == "append":
        return {"bytes": units * sum(_news(c)) * 4 * D * e, "flops": 0}
    if c["kind"] == "store":    # rows in, codes out and in again, values out; about five operations for a code
        io = rows * (2 * D * e + 2 * _row_bytes(c) + (c["T"] + D) * e) + idx
        return {"bytes": io, "flops": rows * (c["T"] + D) * (5 if c["bits"] else 0)}
    heads = c["N_q"] // c["N_kv"]
    tails = units * sum(_tails(c))
    io = rows * _row_bytes(c) + tails * 2 * D * e + 2 * c["L"] * c["B"] * c["N_q"] * D * e + idx
    return {"bytes": io, "flops": 2 * heads * (rows * (c["T"] + D) + tails * 2 * D)}


# ------------------------------------------------------------------------------- the format

def _unit_bytes(c):
    return c["bits"] if c["bits"] else 8 * _esize(c)


def _chunks(c):
    return (c["T"] + 7) // 8


def _tile_bytes(c):
    ch, ub = _chunks(c), _unit_bytes(c)
    params = (ch * 8 + 2 * TILE) * 2 * _esize(c) if c["bits"] else 0
    return (ch + 16) * 64 * ub + params


def _arrange(u):
    """[..., 4 (j), 16 (m), bytes of a unit] -> the bytes of a group: 16-byte cells, those of equal m side by side."""
    lead, ub = u.shape[:-3], u.shape[-1]
    if ub < 16:
        p = 16 // ub
        u = u.reshape(*lead, 4 // p, p, 16, ub).transpose(-3, -2)
    elif ub > 16:
        u = u.reshape(*lead, 4, 16, ub // 16, 16).transpose(-3, -2)
    return u.reshape(*lead, 64 * ub)


def _unarrange(b, ub):
    """The inverse of _arrange."""
    lead = b.shape[:-1]
    if ub < 16:
        p = 16 // ub
        return b.reshape(*lead, 4 // p, 16, p, ub).transpose(-3, -2).reshape(*lead, 4, 16, ub)
    if ub > 16:
        return b.reshape(*lead, 4, ub // 16, 16, 16).transpose(-3, -2).reshape(*lead, 4, 16, ub)
    return b.reshape(*lead, 4, 16, ub)


def _unit(x, bits):
    """[..., 8] elements or codes -> [..., bytes]: 4-bit code 2p at bits 4p of a word, code 2p + 1 at bits 16 + 4p."""
    if bits == 0:
        return x.contiguous().view(torch.uint8)
    if bits == 8:
        return x.to(torch.uint8)
    x = x.to(torch.uint8)
    low, high = x[..., 0::2], x[..., 1::2]
    return torch.cat([low[..., 0::2] | (low[..., 1::2] << 4), high[..., 0::2] | (high[..., 1::2] << 4)], dim=-1)


def _ununit(b, bits, dtype):
    """The inverse of _unit."""
    if bits == 0:
        return b.contiguous().view(dtype)
    if bits == 8:
        return b
    nibbles = torch.stack([b & 15, b >> 4], dim=-1)                    # [..., byte, 2]
    low, high = nibbles[..., :2, :].flatten(-2), nibbles[..., 2:, :].flatten(-2)
    return torch.stack([low, high], dim=-1).flatten(-2)


def _pack(c, kc, kp, vc, vp):
    """Tiles' bytes [N, tile bytes] from codes (or elements) kc [N, 64, T], vc [N, 64, 128] and parameters kp [N, T, 2],
    vp [N, 64, 2 (half), 2]."""
    n, ch, bits = kc.shape[0], _chunks(c), c["bits"]
    k = torch.nn.functional.pad(kc, (0, ch * 8 - c["T"])).reshape(n, 4, 16, ch, 8).permute(0, 3, 1, 2, 4)   # row 16 j + m
    k = _arrange(_unit(k, bits)).reshape(n, -1)
    v = vc.reshape(n, 2, 2, 4, 4, 2, 16, 4)                                 # row 32 g + 16 x + 4 h + r, channel 64 half + 4 m + j
    v = v.permute(0, 1, 3, 5, 7, 6, 2, 4).reshape(n, 16, 4, 16, 8)          # group (g, h, half), j, m, element (x, r)
    v = _arrange(_unit(v, bits)).reshape(n, -1)
    if bits == 0:
        return torch.cat([k, v], dim=1)
    kp = torch.nn.functional.pad(kp, (0, 0, 0, ch * 8 - c["T"])).contiguous().view(torch.uint8).reshape(n, -1)
    vp = vp.reshape(n, 2, 2, 4, 4, 2, 2).permute(0, 1, 3, 5, 2, 4, 6).contiguous().view(torch.uint8).reshape(n, -1)
    return torch.cat([k, v, kp, vp], dim=1)


def _unpack(c, tiles):
    """The values that tiles' bytes [..., tile bytes] stand for, in 32 bits: [..., 64, T] and [..., 64, 128]."""
    lead, ch, bits, ub, dt = tiles.shape[:-1], _chunks(c), c["bits"], _unit_bytes(c), _tdtype(c)
    cut = [ch * 64 * ub, 16 * 64 * ub] + ([ch * 8 * 2 * _esize(c), 2 * TILE * 2 * _esize(c)] if bits else [])
    parts = torch.split(tiles.reshape(-1, tiles.shape[-1]), cut, dim=1)
    n = parts[0].shape[0]
    k = _ununit(_unarrange(parts[0].reshape(n, ch, -1), ub), bits, dt).float()
    v = _ununit(_unarrange(parts[1].reshape(n, 16, -1), ub), bits, dt).float()
    if bits:
        kp = parts[2].contiguous().view(dt).float().reshape(n, ch, 1, 1, 8, 2)
        vp = parts[3].contiguous().view(dt).float().reshape(n, 16, 1, 1, 8, 2)
        k = kp[..., 1] + k * kp[..., 0]
        v = vp[..., 1] + v * vp[..., 0]
    k = k.permute(0, 2, 3, 1, 4).reshape(*lead, TILE, ch * 8)[..., :c["T"]]
    v = v.reshape(n, 2, 4, 2, 4, 16, 2, 4).permute(0, 1, 6, 2, 7, 3, 5, 4).reshape(*lead, TILE, D)
    return k, v


def _codes(x, low, high, bits, dt):
    """Codes of x whose group has the extremes low and high, scale and minimum (both values of the element type)."""
    top = float(2 ** bits - 1)
    scale = ((high - low).double() / top).float().to(dt).float()
    quotient = ((x - low).double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double()).float()
    code = torch.where(scale > 0, quotient.round().clamp(max=top), torch.zeros_like(quotient))
    return code, scale, low


# ------------------------------------------------------------------------------- inputs

class _Maker:
    """Seeded tensors on the GPU: key channels with a scale and an offset per (layer, head, channel), as key caches have."""

    def __init__(self, case, seed):
        self.c = case
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 7919 + 17)
        lead = (case["L"], 1, case["N_kv"], 1, D)
        self.scale = torch.exp(self.randn(*lead))
        self.offset = self.scale * self.randn(*lead)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def keys(self, B, rows):
        return (self.randn(self.c["L"], B, self.c["N_kv"], rows, D) * self.scale + self.offset).to(_tdtype(self.c))

    def values(self, B, rows):
        return self.randn(self.c["L"], B, self.c["N_kv"], rows, D).to(_tdtype(self.c))

    def kept(self):
        """Ascending kept channels, int16 [L, B, N_kv, T]."""
        c = self.c
        r = torch.rand(c["L"], c["B"], c["N_kv"], D, generator=self.g, device="cuda")
        return r.argsort(dim=-1)[..., :c["T"]].sort(dim=-1).values.to(torch.int16).contiguous()

    def table(self):
        """Page numbers int32 [B, most pages], pages in no order; -1 where a sequence has no page.  And the pool's pages."""
        c = self.c
        need = [-(-n // c["page_rows"]) for n in _lengths(c)]
        total = sum(need) + 3
        order = torch.randperm(total, generator=self.g, device="cuda").to(torch.int32)
        t = torch.full((c["B"], max(need)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(need):
            t[b, :n] = order[at:at + n]
            at += n
        return t, total


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _fill_pool(c, st, m, logical=None):
    """Writes every sequence's rows, quantised here in plain torch, into its pages.  `logical`: a list that receives each
    sequence's (codes or elements, parameters) as they are before they are packed, for the 64-bit result."""
    tpp = c["page_rows"] // TILE
    for b, n in enumerate(_lengths(c)):
        tiles = -(-n // TILE)
        pages = -(-n // c["page_rows"])
        k, v = m.keys(1, n), m.values(1, n)
        idx = st["idx"][:, b:b + 1, :, None, :].long().expand(-1, -1, -1, n, -1)
        k = k.gather(4, idx)
        pad = (0, 0, 0, pages * c["page_rows"] - n)
        k = torch.nn.functional.pad(k, pad).reshape(-1, TILE, c["T"])
        v = torch.nn.functional.pad(v, pad).reshape(-1, TILE, D)
        kp = vp = None
        if c["bits"]:
            inside = (torch.arange(pages * c["page_rows"], device="cuda") < n).reshape(1, -1, TILE, 1)
            inside = inside.expand(c["L"] * c["N_kv"], -1, -1, -1).reshape(-1, TILE, 1)
            kf, vf = k.float(), v.float().reshape(-1, TILE, 2, 64)
            low = kf.masked_fill(~inside, float("inf")).amin(1, keepdim=True)
            high = kf.masked_fill(~inside, float("-inf")).amax(1, keepdim=True)
            some = inside.any(1, keepdim=True)
            low, high = (torch.where(some, x, torch.zeros_like(x)) for x in (low, high))
            k, ks, km = _codes(kf, low, high, c["bits"], _tdtype(c))
            k = k.masked_fill(~inside, 0)
            kp = torch.stack([ks, km], dim=-1).reshape(-1, c["T"], 2).to(_tdtype(c))
            v, vs, vm = _codes(vf, vf.amin(3, keepdim=True), vf.amax(3, keepdim=True), c["bits"], _tdtype(c))
            v, vs, vm = (x.masked_fill(~inside[..., None], 0) for x in (v, vs, vm))
            v = v.reshape(-1, TILE, D)
            vp = torch.stack([vs, vm], dim=-1).reshape(-1, TILE, 2, 2).to(_tdtype(c))
        if logical is not None:
            logical.append((k, kp, v, vp))
        data = _pack(c, k, kp, v, vp).reshape(c["L"], c["N_kv"], pages, tpp, -1)
        if tiles:
            st["pool"][:, st["table"][b, :pages].long()] = data.permute(0, 2, 1, 3, 4)


def prepare(case, seed, logical=None):
    c, m = case, _Maker(case, seed)
    lead = (c["L"], c["B"], c["N_kv"])
    st = {"c": c, "idx": m.kept()}
    if c["kind"] == "append":
        st["k_new"], st["v_new"] = m.keys(c["B"], c["new"]), m.values(c["B"], c["new"])
        st["n_new"], st["s_tail"] = _ints(_news(c)), _ints(_tails(c))
        st["k_tail"], st["v_tail"] = m.keys(c["B"], c["cap"]), m.values(c["B"], c["cap"])
        return st
    st["table"], st["n_pages"] = m.table()
    st["pool"] = torch.zeros(c["L"], st["n_pages"], c["N_kv"], c["page_rows"] // TILE, _tile_bytes(c), dtype=torch.uint8, device="cuda")
    st["rows"] = _ints(_lengths(c))
    if c["kind"] == "store":
        st["k"], st["v"] = m.keys(c["B"], c["S"]), m.values(c["B"], c["S"])
        st["k_out"] = torch.zeros(*lead, c["S"], c["T"], dtype=_tdtype(c), device="cuda")
        st["v_out"] = torch.zeros(*lead, c["S"], D, dtype=_tdtype(c), device="cuda")
        return st
    st["q"] = (m.randn(c["L"], c["B"], c["N_q"], D) / m.scale.squeeze(3).repeat_interleave(c["N_q"] // c["N_kv"], 2)).to(_tdtype(c))
    st["out"] = torch.zeros_like(st["q"])
    st["s_tail"] = _ints(_tails(c))
    if c["cap"]:
        st["k_tail"], st["v_tail"] = m.keys(c["B"], c["cap"]), m.values(c["B"], c["cap"])
    _fill_pool(c, st, m, logical)
    return st


# ------------------------------------------------------------------------------- the calls

def _setup(st):
    """What a program makes once: the shape, the description of its pages, a workspace."""
    import paper_2407_21018_amd as thk
    c = st["c"]
    st["thk"] = thk
    st["shape"] = thk.make_shape(c["L"], c["B"], c["N_q"], c["N_kv"], D, c["S"], 1, c["T"], 0,
                                 thk.THK_F32 if c["dtype"] == "f32" else thk.THK_BF16)
    if c["kind"] != "append":
        st["pages"] = thk.make_pages(c["bits"], c["page_rows"], st["table"].shape[1], st["n_pages"])
    if c["kind"] == "decode":
        n = thk.thk_workspace_bytes(st["shape"], thk.THK_OP_DECODE_PAGED)
        st["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")


def _run_own(st):
    c = st["c"]
    if "thk" not in st:
        _setup(st)
    thk, shape = st["thk"], st["shape"]
    if c["kind"] == "append":
        thk.thk_tail_append_ragged(shape, st["k_new"], st["v_new"], c["new"], None, st["n_new"], st["k_tail"], st["v_tail"],
                                   st["s_tail"], c["cap"])
        return {"k_tail": st["k_tail"], "v_tail": st["v_tail"]}
    if c["kind"] == "store":
        thk.thk_paged_write(shape, st["pages"], st["k"], st["v"], c["S"], st["rows"], None, st["idx"], st["table"], st["pool"])
        thk.thk_paged_read(shape, st["pages"], st["pool"], st["table"], None, st["rows"], st["k_out"], st["v_out"], c["S"])
        return {"k": st["k_out"], "v": st["v_out"]}
    thk.thk_decode_attn_paged(shape, st["pages"], st["q"], st["pool"], st["table"], st["rows"], st["idx"], st.get("k_tail"),
                              st.get("v_tail"), st["s_tail"], c["cap"], st["out"], st["ws"])
    return {"out": st["out"]}


def _append(st):
    c = st["c"]
    step = torch.arange(c["new"], device="cuda")
    at = (st["s_tail"][:, None] + step).long()                                # [B, new]: tail row of each new row
    live = (step[None] < st["n_new"][:, None])
    at = torch.where(live, at, torch.full_like(at, c["cap"]))                 # dead rows go to a row that is cut off again
    out = {}
    for name in ("k", "v"):
        tail = torch.nn.functional.pad(st[name + "_tail"], (0, 0, 0, 1))
        where = at[None, :, None, :, None].expand_as(st[name + "_new"])
        st[name + "_tail"].copy_(tail.scatter_(3, where, st[name + "_new"])[..., :c["cap"], :])
        out[name + "_tail"] = st[name + "_tail"]
    return out


def _through_codes(x, inside, dim, bits, dt):
    """What x stands for once it has been coded, groups along `dim`; rows outside take no part."""
    low = x.masked_fill(~inside, float("inf")).amin(dim, keepdim=True)
    high = x.masked_fill(~inside, float("-inf")).amax(dim, keepdim=True)
    some = low <= high
    low, high = (torch.where(some, y, torch.zeros_like(y)) for y in (low, high))
    code, scale, low = _codes(x, low, high, bits, dt)
    return low + code * scale


def _store(st):
    c, dt = st["c"], _tdtype(st["c"])
    lead, s = (c["L"], c["B"], c["N_kv"]), c["S"]
    inside = (torch.arange(s, device="cuda") < st["rows"][:, None]).reshape(1, c["B"], 1, s, 1)
    k = st["k"].gather(4, st["idx"].long()[..., None, :].expand(*lead, s, c["T"]))
    v = st["v"]
    if c["bits"]:
        more = -s % TILE
        tiles = (s + more) // TILE
        full = torch.nn.functional.pad(inside, (0, 0, 0, more)).reshape(1, c["B"], 1, tiles, TILE, 1)
        kf = torch.nn.functional.pad(k.float(), (0, 0, 0, more)).reshape(*lead, tiles, TILE, c["T"])
        k = _through_codes(kf, full, 4, c["bits"], dt).reshape(*lead, s + more, c["T"])[..., :s, :].to(dt)
        vf = v.float().reshape(*lead, s, 2, 64)
        v = _through_codes(vf, inside[..., None], 5, c["bits"], dt).reshape(*lead, s, D).to(dt)
    zero = torch.zeros((), dtype=dt, device="cuda")
    st["k_out"].copy_(torch.where(inside, k, zero))
    st["v_out"].copy_(torch.where(inside, v, zero))
    return {"k": st["k_out"], "v": st["v_out"]}


def _decode(st):
    c = st["c"]
    L, B, N, G = c["L"], c["B"], c["N_kv"], c["N_q"] // c["N_kv"]
    pages = st["table"].clamp(min=0).long()
    tiles = st["pool"][:, pages]                                               # [L, B, pages, N, tiles of a page, bytes]
    k, v = _unpack(c, tiles.permute(0, 1, 3, 2, 4, 5))
    k, v = k.reshape(L * B * N, -1, c["T"]), v.reshape(L * B * N, -1, D)
    q = st["q"].float().reshape(L, B, N, G, D)
    qk = q.gather(4, st["idx"].long()[..., None, :].expand(L, B, N, G, c["T"])).reshape(L * B * N, G, c["T"])
    z = torch.bmm(qk, k.transpose(1, 2).contiguous()).reshape(L, B, N, G, -1)
    live = torch.arange(z.shape[-1], device="cuda") < st["rows"][:, None]
    if c["cap"]:
        kt, vt = (st[n].float().reshape(L * B * N, c["cap"], D) for n in ("k_tail", "v_tail"))
        zt = torch.bmm(q.reshape(L * B * N, G, D), kt.transpose(1, 2).contiguous()).reshape(L, B, N, G, -1)
        z, v = torch.cat([z, zt], dim=-1), torch.cat([v, vt], dim=1)
        live = torch.cat([live, torch.arange(c["cap"], device="cuda") < st["s_tail"][:, None]], dim=1)
    live = live[None, :, None, None, :]
    z = (z / D ** 0.5).masked_fill(~live, float("-inf"))
    p = torch.exp(z - z.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    v = v.reshape(L, B, N, -1, D) * live[:, :, :, 0, :, None]
    out = torch.bmm(p.reshape(L * B * N, G, -1), v.reshape(L * B * N, -1, D))
    st["out"].copy_(out.reshape(st["out"].shape))
    return {"out": st["out"]}


def run(state):
    if own:
        return _run_own(state)
    return {"append": _append, "store": _store, "decode": _decode}[state["c"]["kind"]](state)


# ------------------------------------------------------------------------------- in 64 bits

def _exact_group(x, bits, dt):
    """What the group x [.., n] (64 bits, values of the element type) stands for once coded, in 64 bits."""
    round32 = lambda y: y.to(torch.float32).to(torch.float64)  # noqa: E731
    top = 2 ** bits - 1
    low = x.min(dim=-1, keepdim=True).values
    scale = round32(round32(x.max(dim=-1, keepdim=True).values - low) / top).to(dt).to(torch.float64)
    code = torch.round(round32(round32(x - low) / scale))
    code = torch.where(scale == 0, torch.zeros_like(code), torch.minimum(code, torch.full_like(code, top)))
    return low + scale * code


def _exact_store(c, seed):
    st, dt = prepare(c, seed), _tdtype(c)
    k_out, v_out = st["k_out"].double(), st["v_out"].double()
    for b, n in enumerate(_lengths(c)):
        channels = st["idx"][:, b].long()[:, :, None, :].expand(-1, -1, n, -1)
        k, v = torch.gather(st["k"][:, b, :, :n].double(), 3, channels), st["v"][:, b, :, :n].double()
        if c["bits"]:
            for r in range(0, n, TILE):
                rows = k[:, :, r:r + TILE].transpose(2, 3)
                k[:, :, r:r + TILE] = _exact_group(rows, c["bits"], dt).transpose(2, 3)
            for half in (0, 64):
                v[..., half:half + 64] = _exact_group(v[..., half:half + 64], c["bits"], dt)
        k_out[:, b, :, :n], v_out[:, b, :, :n] = k, v
    return {"k": k_out, "v": v_out}


def _exact_append(c, seed):
    st = prepare(c, seed)
    k, v = st["k_tail"].double(), st["v_tail"].double()
    for b, (n, t) in enumerate(zip(_news(c), _tails(c))):
        k[:, b, :, t:t + n], v[:, b, :, t:t + n] = st["k_new"][:, b, :, :n].double(), st["v_new"][:, b, :, :n].double()
    return {"k_tail": k, "v_tail": v}


def _exact_decode(c, seed):
    logical = []
    st = prepare(c, seed, logical)
    L, N, G = c["L"], c["N_kv"], c["N_q"] // c["N_kv"]
    out = torch.zeros(L, c["B"], c["N_q"], D, dtype=torch.float64, device="cuda")
    for b, (n, t) in enumerate(zip(_lengths(c), _tails(c))):
        k, kp, v, vp = logical[b]
        k, v = k.double(), v.double()
        if c["bits"]:
            kp, vp = kp.double(), vp.double()
            k = k * kp[:, None, :, 0] + kp[:, None, :, 1]
            v = (v.reshape(-1, TILE, 2, 64) * vp[..., 0:1] + vp[..., 1:2])
        k, v = k.reshape(L * N, -1, c["T"])[:, :n], v.reshape(L * N, -1, D)[:, :n]
        for u in range(L * N):
            layer, h = divmod(u, N)
            q = st["q"][layer, b, h * G:(h + 1) * G].double()
            z, vals = [q[:, st["idx"][layer, b, h].long()] @ k[u].t().contiguous()], [v[u]]
            if t:
                z.append(q @ st["k_tail"][layer, b, h, :t].double().t().contiguous())
                vals.append(st["v_tail"][layer, b, h, :t].double())
            p = torch.softmax(torch.cat(z, dim=1) / 128.0 ** 0.5, dim=1)
            out[layer, b, h * G:(h + 1) * G] = p @ torch.cat(vals)
    return {"out": out}


def exact(case, seed):
    """The results in 64 bits."""
    return {"append": _exact_append, "store": _exact_store, "decode": _exact_decode}[case["kind"]](case, seed)
