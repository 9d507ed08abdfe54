"""Paged, ragged, quantised caches on the GPU against fp64 (oracle/paged.py): stored and read back, appended, attended over.

Everything a call must not use holds NaN: the pool before it is written, source rows past a sequence's count, tail rows
past theirs, outputs before the call.
"""
import os

import numpy as np
import pytest
import torch

import paper_2407_21018_amd as thk
from oracle import paged as P
from helpers import DT, TDT, ws_tensor

pytestmark = pytest.mark.gpu
D = 128
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}   # of the value, when it is rounded once


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _np(t):
    return t.detach().cpu().double().numpy()


class Cache:
    """A ragged batch: sources, index lists, pages in no order, tails; and the same on the host."""

    def __init__(self, dtype, bits, L, B, N_kv, G, T, rows, page_rows=64, tails=None, cap=0, seed=0, S=None, spare=2, n_split=0):
        g = torch.Generator(device="cuda"); g.manual_seed(9000 + seed)
        self.dtype, self.bits, self.L, self.B, self.N_kv, self.G, self.T = dtype, bits, L, B, N_kv, G, T
        self.rows, self.tails, self.cap, self.page_rows = list(rows), list(tails or [0] * B), cap, page_rows
        self.S = S or max(max(rows), 1)
        self.g, self.U = g, L * B * N_kv
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        scale, off = torch.exp(rnd(L, 1, N_kv, 1, D)), rnd(L, 1, N_kv, 1, D)
        self.k = (rnd(L, B, N_kv, self.S, D) * scale + off * scale).to(TDT[dtype])
        self.v = (rnd(L, B, N_kv, self.S, D) + 0.3 * rnd(L, 1, N_kv, 1, D)).to(TDT[dtype])
        for b, n in enumerate(self.rows):
            self.k[:, b, :, n:] = float("nan")
            self.v[:, b, :, n:] = float("inf")
        self.q = (rnd(L, B, N_kv * G, D) / scale[:, :, :, 0].repeat_interleave(G, 2)).to(TDT[dtype])
        self.idx = torch.rand(L, B, N_kv, D, generator=g, device="cuda").argsort(-1)[..., :T].sort(-1).values.to(torch.int16).contiguous()
        self.kt = (rnd(L, B, N_kv, max(cap, 1), D) * scale + off * scale).to(TDT[dtype])
        self.vt = rnd(L, B, N_kv, max(cap, 1), D).to(TDT[dtype])
        for b, n in enumerate(self.tails):
            self.kt[:, b, :, n:] = float("nan")
            self.vt[:, b, :, n:] = float("nan")
        need = [-(-n // page_rows) for n in self.rows]
        order = torch.randperm(sum(need) + spare, generator=g, device="cuda").cpu().numpy()
        self.max_pages = max(max(need), 1)
        table = np.full((B, self.max_pages), -1, np.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table = torch.from_numpy(table).cuda()
        self.shape = thk.make_shape(L, B, N_kv * G, N_kv, D, self.S, 1, T, 0, DT[dtype], n_split)
        self.pages = thk.make_pages(bits, page_rows, self.max_pages, sum(need) + spare)
        self.pool = torch.full((thk.thk_paged_pool_bytes(self.shape, self.pages),), 255, dtype=torch.uint8, device="cuda")
        self.s_pages, self.s_tail = _ints(self.rows), _ints(self.tails)

    def write(self, stream=None):
        thk.thk_paged_write(self.shape, self.pages, self.k, self.v, self.S, self.s_pages, None, self.idx, self.table, self.pool, stream)

    def decode(self, out=None, ws=None, stream=None, shape=None):
        shape = shape or self.shape
        if out is None:
            out = torch.full_like(self.q, float("nan"))
        if ws is None:
            ws = ws_tensor(thk.thk_workspace_bytes(shape, thk.THK_OP_DECODE_PAGED))
        tail = (self.kt, self.vt, self.s_tail, self.cap) if self.cap else (None, None, None, 0)
        thk.thk_decode_attn_paged(shape, self.pages, self.q, self.pool, self.table, self.s_pages, self.idx, *tail, out, ws, stream)
        return out

    def unit(self, l, b, h):
        """(kept rows, value rows) of a unit as stored, fp64; (tail rows); index list."""
        n, t, idx = self.rows[b], self.tails[b], _np(self.idx[l, b, h]).astype(int)
        k, v = P.stored(_np(self.k[l, b, h, :n])[:, idx], _np(self.v[l, b, h, :n]), self.bits, self.dtype)
        return k, v, _np(self.kt[l, b, h, :t]), _np(self.vt[l, b, h, :t]), idx


# (L, B, N_kv, G, T, rows, page_rows, S): lengths around a tile and a page, none, odd channel counts, several layers
STORE = [
    (1, 1, 1, 1, 64, [1], 64, None), (1, 1, 2, 1, 51, [64], 64, None), (1, 3, 2, 1, 76, [65, 0, 63], 64, None),
    (2, 2, 3, 1, 128, [200, 129], 128, None), (1, 4, 1, 2, 1, [500, 64, 1, 257], 256, None), (3, 2, 1, 1, 97, [130, 191], 64, None),
    (1, 1, 8, 4, 8, [1000], 512, None), (1, 2, 2, 1, 33, [70, 10], 64, 90),
]


@pytest.mark.parametrize("case", STORE, ids=[str(i) for i in range(len(STORE))])
@pytest.mark.parametrize("bits", [0, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_come_back_as_what_they_were_stored_as(dtype, bits, case):
    L, B, N_kv, G, T, rows, page_rows, S = case
    print("store", dtype, bits, case, flush=True)
    c = Cache(dtype, bits, L, B, N_kv, G, T, rows, page_rows, seed=T, S=S)
    c.write()
    for ld in (T, min(D, T + 5)):
        c.shape.ld_keep = ld
        out_rows = c.S + 3
        ko = torch.full((L, B, N_kv, out_rows, ld), 7.0, dtype=TDT[dtype], device="cuda")
        vo = torch.full((L, B, N_kv, out_rows, D), 7.0, dtype=TDT[dtype], device="cuda")
        thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, out_rows)
        torch.cuda.synchronize()
        for l in range(L):
            for b in range(B):
                for h in range(N_kv):
                    n = rows[b]
                    k, v, _, _, _ = c.unit(l, b, h)
                    for got, want in ((_np(ko[l, b, h])[:n, :T], k), (_np(vo[l, b, h])[:n], v)):
                        assert np.all(np.abs(got - want) <= (0 if bits == 0 else HALF_STEP[dtype]) * np.abs(want))
                    assert not _np(ko[l, b, h])[:n, T:].any()                      # the columns past T are zeros
        for b in range(B):
            assert torch.all(ko[:, b, :, rows[b]:] == 7) and torch.all(vo[:, b, :, rows[b]:] == 7)   # the rest as it was


# (B, N_kv, T, ld, rows): 1024 tiles of the grid (bf16; fp32: 512), up to which keys and values have blocks of their own, with the most
# rows of row0 = 0; a tile a unit more; and ragged ones well past it
LARGE = {"at": {"bf16": (4, 4, 51, 56, [4096, 4033, 1, 2048]), "f32": (2, 4, 51, 56, [4096, 100])},
         "past": {"bf16": (4, 4, 76, 76, [4097, 64, 0, 4096]), "f32": (2, 4, 76, 76, [4097, 4096])},
         "far": {"bf16": (3, 8, 33, 48, [6000, 5999, 17]), "f32": (2, 6, 128, 128, [5000, 4936])}}


@pytest.mark.parametrize("size", LARGE)
@pytest.mark.parametrize("bits", [0, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_writes_and_reads(dtype, bits, size):
    """One block for a tile's keys and values: all rows, any range of them, with both outputs and with one."""
    B, N_kv, T, ld, rows = LARGE[size][dtype]
    print("large", dtype, bits, size, flush=True)
    c = Cache(dtype, bits, 1, B, N_kv, 1, T, rows, 256, seed=300 + T)
    c.write()
    c.shape.ld_keep = ld
    units = [[c.unit(0, b, h)[:2] for h in range(N_kv)] for b in range(B)]
    inside = [min(37 + 64 * b, n) for b, n in enumerate(rows)]
    for row0, n in ((None, rows), (inside, [x - y for x, y in zip(rows, inside)]), (inside, [min(x - y, 65) for x, y in zip(rows, inside)])):
        for with_keys, with_values in ((True, True), (True, False), (False, True)):
            ko = torch.full((1, B, N_kv, c.S, ld), 7.0, dtype=TDT[dtype], device="cuda") if with_keys else None
            vo = torch.full((1, B, N_kv, c.S, D), 7.0, dtype=TDT[dtype], device="cuda") if with_values else None
            thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None if row0 is None else _ints(row0), _ints(n), ko, vo, c.S)
            torch.cuda.synchronize()
            for b in range(B):
                at = 0 if row0 is None else row0[b]
                for out, which, width in ((ko, 0, T), (vo, 1, D)):
                    if out is None:
                        continue
                    assert torch.all(out[0, b, :, n[b]:] == 7) and not out[0, b, :, :n[b], width:].any()
                    got = _np(out[0, b, :, :n[b], :width])
                    want = np.stack([units[b][h][which][at:at + n[b]] for h in range(N_kv)])
                    assert np.all(np.abs(got - want) <= (0 if bits == 0 else HALF_STEP[dtype]) * np.abs(want)), (b, row0, which)


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_range_of_rows_is_read(dtype, bits):
    c = Cache(dtype, bits, 1, 3, 2, 1, 51, [300, 129, 64], 128, seed=3)
    c.write()
    for row0, n in (([0, 0, 0], [300, 129, 64]), ([1, 63, 64], [299, 66, 0]), ([65, 128, 10], [64, 1, 1]), ([255, 100, 63], [45, 29, 1])):
        ko = torch.full((1, 3, 2, 300, 51), 7.0, dtype=TDT[dtype], device="cuda")
        vo = torch.full((1, 3, 2, 300, D), 7.0, dtype=TDT[dtype], device="cuda")
        thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, _ints(row0), _ints(n), ko, None, 300)
        thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, _ints(row0), _ints(n), None, vo, 300)
        torch.cuda.synchronize()
        for b in range(3):
            for h in range(2):
                k, v, _, _, _ = c.unit(0, b, h)
                for got, want in ((_np(ko[0, b, h]), k), (_np(vo[0, b, h]), v)):
                    want = want[row0[b]:row0[b] + n[b]]
                    assert np.all(np.abs(got[:n[b]] - want) <= (0 if bits == 0 else HALF_STEP[dtype]) * np.abs(want))
                    assert np.all(got[n[b]:] == 7)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_without_range_and_with_extreme_ones(dtype, bits):
    """Equal elements, scales that round to zero, the largest finite range, elements on the border between two codes."""
    c = Cache(dtype, bits, 1, 1, 1, 1, 128, [128], 64, seed=1)
    x = c.v[0, 0, 0]
    x[0] = -3.25
    x[1] = 0
    x[2, :64], x[2, 64:] = 0, 2.0 ** -133                          # subnormal in both types
    x[3] = 0
    x[3, 5] = 2.0 ** -133                                          # the scale is below half the least bf16 number
    x[4, ::2], x[4, 1::2] = 1.5e38, -1.5e38
    step = torch.arange(128, device="cuda") % 64
    x[5] = (step.float() * 0.5).clamp(max=15).to(x.dtype)            # with 4 bits: every second one half way between two codes
    x[6] = 1e-30 * torch.randn(128, generator=c.g, device="cuda").to(x.dtype)
    x[7] = 1e-38 * torch.randn(128, generator=c.g, device="cuda").to(x.dtype)    # subnormal scales
    c.k[0, 0, 0, :, :64] = x[:8].repeat(16, 1)[:, :64]
    c.write()
    ko, vo = (torch.empty(1, 1, 1, 128, D, dtype=TDT[dtype], device="cuda") for _ in range(2))
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, 128)
    torch.cuda.synchronize()
    k, v, _, _, _ = c.unit(0, 0, 0)
    least = 2.0 ** (-149 if dtype == "f32" else -133)   # half a step of a subnormal result is up to half of this
    for got, want in ((_np(ko[0, 0, 0]), k), (_np(vo[0, 0, 0]), v)):
        assert np.all(np.abs(got - want) <= HALF_STEP[dtype] * np.abs(want) + least / 2)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_below_the_normal_numbers_beside_ordinary_ones(dtype, bits):
    """Groups whose range is 8 to 300 of the type's least number: their scales have few bits, quotients go up to half as far again as
    the last code.  What an ordinary group beside them holds is its own."""
    c = Cache(dtype, bits, 1, 1, 4, 1, 128, [320], 64, seed=17)
    least = 2.0 ** (-149 if dtype == "f32" else -133)
    r = np.random.default_rng(170)

    def tiny(groups, n):
        """[groups, n]: whole multiples of the least number, from 0 (or from below it) over a range of 8 .. 300."""
        span = (8 + np.arange(groups) % 293)[:, None]
        x = r.integers(0, span + 1, (groups, n))
        x[:, 0], x[:, 1] = 0, span[:, 0]
        return (x - r.integers(0, 2, (groups, 1)) * 40) * least

    for h in range(4):
        k, v = _np(c.k[0, 0, h]), _np(c.v[0, 0, h])
        for t in range(5):
            some = r.random(D) < 0.5
            k[64 * t:64 * t + 64, some] = tiny(some.sum(), 64).T
        halves = v.reshape(-1, 64)
        some = r.random(len(halves)) < 0.5
        halves[some] = tiny(some.sum(), 64)
        c.k[0, 0, h], c.v[0, 0, h] = (torch.from_numpy(x).to(TDT[dtype]).cuda() for x in (k, v))
    c.write()
    ko, vo = (torch.empty(1, 1, 4, 320, D, dtype=TDT[dtype], device="cuda") for _ in range(2))
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, 320)
    torch.cuda.synchronize()
    for h in range(4):
        k, v, _, _, _ = c.unit(0, 0, h)
        for name, got, want in (("keys", _np(ko[0, 0, h]), k), ("values", _np(vo[0, 0, h]), v)):
            bad = np.abs(got - want) > HALF_STEP[dtype] * np.abs(want) + least / 2
            assert not bad.any(), (name, h, int(bad.sum()), np.abs(got - want).max())


@pytest.mark.parametrize("bits", [4, 8])
def test_bf16_rows_are_rounded_through_fp32(bits):
    """A minimum far below a step of fp32 decides a tie of m + c s between two bf16 numbers if that is rounded once; what is read is rounded
    to fp32 first."""
    c = Cache("bf16", bits, 1, 1, 2, 1, 128, [640], 128, seed=19)
    g = torch.Generator().manual_seed(190)
    x = (torch.rand(2, 640, 2, 64, generator=g) * 4 + 0.01) * torch.exp(torch.randn(2, 640, 2, 1, generator=g))
    x[..., 0] = 2.0 ** -40
    c.v[0, 0] = x.reshape(2, 640, D).to(torch.bfloat16).cuda()
    c.k[0, 0] = x.reshape(2, 10, D, 64).transpose(2, 3).reshape(2, 640, D).to(torch.bfloat16).cuda()
    c.write()
    ko, vo = (torch.empty(1, 1, 2, 640, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, 640)
    torch.cuda.synchronize()
    for h in range(2):
        k, v, _, _, _ = c.unit(0, 0, h)
        for got, want in ((_np(ko[0, 0, h]), k), (_np(vo[0, 0, h]), v)):
            step = 2.0 ** (np.floor(np.log2(want)) - 7)
            assert (np.rint(want / step) * step != P.round_to(want, "bf16")).sum() > 100   # round_to goes through fp32 too
            assert np.array_equal(got, P.round_to(want, "bf16"))


@pytest.mark.parametrize("dtype,bits", [("bf16", 4), ("bf16", 0), ("f32", 8)])
def test_a_chunk_after_a_chunk(dtype, bits):
    """A prompt stored in two calls is the prompt stored in one; sequences whose first row is not a tile's are left alone."""
    a = Cache(dtype, bits, 1, 3, 2, 1, 76, [320, 200, 128], 64, seed=11)
    a.write()
    want = a.pool.clone()
    a.pool.fill_(255)
    cut = [128, 64, 0]
    thk.thk_paged_write(a.shape, a.pages, a.k, a.v, a.S, _ints(cut), None, a.idx, a.table, a.pool)
    rest = a.S
    k2, v2 = torch.full_like(a.k, float("nan")), torch.full_like(a.v, float("nan"))
    for b, n in enumerate(cut):
        k2[:, b, :, :a.S - n], v2[:, b, :, :a.S - n] = a.k[:, b, :, n:], a.v[:, b, :, n:]
    n2 = [x - y for x, y in zip(a.rows, cut)]
    before = a.pool.clone()
    for bad in (1, 63, -64, 65):
        thk.thk_paged_write(a.shape, a.pages, k2, v2, rest, _ints(n2), _ints([bad] * 3), a.idx, a.table, a.pool)
    torch.cuda.synchronize()
    assert torch.equal(a.pool, before)
    thk.thk_paged_write(a.shape, a.pages, k2, v2, rest, _ints(n2), _ints(cut), a.idx, a.table, a.pool)
    torch.cuda.synchronize()
    assert torch.equal(a.pool, want)


def test_counts_and_tables_past_the_bounds_write_nothing_outside():
    """Counts above the bounds are clamped to them, negative ones to zero; tables with entries outside the pool."""
    c = Cache("bf16", 4, 1, 4, 1, 1, 64, [256, 256, 256, 256], 64, seed=2, spare=4)
    table = c.table.clone()
    table[0, 1], table[1, 2], table[2, 0], table[3, 3] = -1, c.pages.n_pages, 1 << 30, -(1 << 31)
    guard = torch.full((c.pool.numel() + 2048,), 255, dtype=torch.uint8, device="cuda")
    pool = guard[1024:-1024]
    thk.thk_paged_write(c.shape, c.pages, c.k, c.v, c.S, _ints([1 << 30, 256, 300, -5]), None, c.idx, table, pool)
    torch.cuda.synchronize()
    assert torch.all(guard[:1024] == 255) and torch.all(guard[-1024:] == 255)
    tile = c.pool.numel() // c.pages.n_pages
    written = {int(p) for p in range(c.pages.n_pages) if not torch.all(pool[p * tile:(p + 1) * tile] == 255)}
    assert written == {int(table[b, i]) for b in range(3) for i in range(4) if 0 <= table[b, i] < c.pages.n_pages}
    ko = torch.full((1, 4, 1, 256, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    thk.thk_paged_read(c.shape, c.pages, pool, table, None, _ints([1 << 30, 256, 256, -1]), ko, None, 256)
    thk.thk_paged_read(c.shape, c.pages, pool, table, _ints([-64, 1 << 30, (1 << 31) - 1, 256]), _ints([256] * 4), ko, None, 256)
    torch.cuda.synchronize()
    assert torch.all(ko[0, 0, 0, 64:128] == 7) and torch.all(ko[0, 1, 0, 128:192] == 7) and torch.all(ko[0, 2, 0, :64] == 7) and torch.all(ko[0, 3] == 7)
    assert not torch.all(ko[0, 0, 0, :64] == 7, dim=1).any()   # (single elements may well stand for 7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ragged_append(dtype):
    L, B, N_kv, cap, src = 2, 5, 3, 16, 9
    g = torch.Generator(device="cuda"); g.manual_seed(4)
    new = [torch.randn(L, B, N_kv, src, D, generator=g, device="cuda").to(TDT[dtype]) for _ in range(2)]
    tail = [torch.randn(L, B, N_kv, cap, D, generator=g, device="cuda").to(TDT[dtype]) for _ in range(2)]
    shape = thk.make_shape(L, B, N_kv, N_kv, D, 1, 1, 64, 0, DT[dtype])
    for row0, n, s in (([0, 0, 0, 0, 0], [1, 1, 1, 1, 1], [0, 3, 15, 16, 7]), ([0, 8, 2, 5, -1], [9, 4, 0, -3, 2], [0, 0, 5, 5, 5]),
                       ([3, 0, 0, 0, 0], [6, 9, 9, 9, 99], [10, 12, -2, 1 << 30, 0])):
        got = [t.clone() for t in tail]
        thk.thk_tail_append_ragged(shape, *new, src, _ints(row0), _ints(n), *got, _ints(s), cap)
        torch.cuda.synchronize()
        for x, y, z in zip(new, tail, got):
            want = y.clone()
            for b in range(B):
                for r in range(min(max(n[b], 0), src)):
                    if 0 <= row0[b] + r < src and 0 <= s[b] + r < cap:
                        want[:, b, :, s[b] + r] = x[:, b, :, row0[b] + r]
            assert torch.equal(z, want)
    got = [t.clone() for t in tail]
    one = [x[..., :1, :].contiguous() for x in new]
    thk.thk_tail_append_ragged(shape, *one, 1, None, None, *got, _ints([0, 1, 2, 15, 16]), cap)
    for x, y, z in zip(one, tail, got):
        want = y.clone()
        for b, s in enumerate([0, 1, 2, 15]):
            want[:, b, :, s] = x[:, b, :, 0]
        assert torch.equal(z, want)


def _check_attention(c, out):
    """Every output against fp64 attention over what is stored.  An output is rounded once; a logit is off by what the
    products' terms and their fp32 sums are -- c_z of the sum of the products' sizes, the sizes being at most those of
    q (|m| + 31 s), 31 s <= 31 / 15 (max k - min k) <= 4.2 max |k| -- and moves an output by at most twice that times the
    largest value; the values' products by c_z of at most 5.2 times the largest value."""
    c_z = {"bf16": 2.0 ** -16, "f32": 2.0 ** -20}[c.dtype]   # terms: 2^-17, 2^-25; sums of some 256 roundings of 2^-24, as random ones
    for l in range(c.L):
        for b in range(c.B):
            for h in range(c.N_kv):
                k, v, kt, vt, idx = c.unit(l, b, h)
                q = _np(c.q[l, b, h * c.G:(h + 1) * c.G])
                want = P.attend(q, idx, k, v, kt, vt)
                got = _np(out[l, b, h * c.G:(h + 1) * c.G])
                if len(k) + len(kt) == 0:
                    assert not got.any(), (l, b, h)
                    continue
                top = max(np.abs(v).max(initial=0), np.abs(vt).max(initial=0))
                size = 5.2 * np.abs(q[:, idx]) @ np.abs(k).max(0, initial=0) + np.abs(q) @ np.abs(kt).max(0, initial=0)
                tol = HALF_STEP[c.dtype] * np.abs(want) + c_z * top * (2 * size[:, None] / np.sqrt(D) + 5.2)
                bad = np.abs(got - want) > tol
                assert not bad.any(), (l, b, h, np.abs(got - want).max(), tol.min())


# (L, B, N_kv, G, T, rows, page_rows, tails, cap, n_split)
ATTEND = [
    (1, 1, 1, 1, 64, [1], 64, None, 0, 0), (1, 1, 1, 1, 1, [64], 64, [1], 1, 0), (1, 2, 2, 4, 51, [0, 65], 64, [0, 3], 16, 0),
    (1, 3, 2, 8, 76, [129, 0, 300], 128, [64, 65, 0], 128, 0), (2, 2, 3, 2, 128, [63, 512], 256, [0, 17], 64, 3),
    (1, 1, 2, 16, 97, [700], 64, [200], 200, 4), (1, 1, 1, 17, 96, [260], 64, [1], 64, 2), (1, 2, 1, 40, 65, [64, 130], 64, [5, 0], 8, 0),
    (1, 4, 2, 5, 33, [2000, 1, 640, 0], 128, [0, 0, 64, 2], 64, 0), (1, 1, 4, 4, 64, [5000], 512, None, 0, 100),
    (3, 1, 2, 3, 8, [257], 64, [33], 64, 1), (1, 2, 2, 1, 128, [0, 0], 64, [0, 64], 64, 0), (1, 2, 1, 7, 64, [4096, 30], 1024, [63, 1], 64, 7),
]


@pytest.mark.parametrize("case", ATTEND, ids=[str(i) for i in range(len(ATTEND))])
@pytest.mark.parametrize("bits", [0, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_over_pages_and_tail(dtype, bits, case):
    L, B, N_kv, G, T, rows, page_rows, tails, cap, n_split = case
    print("attend", dtype, bits, case, flush=True)
    c = Cache(dtype, bits, L, B, N_kv, G, T, rows, page_rows, tails, cap, seed=sum(rows) + G, n_split=n_split)
    c.write()
    out = c.decode()
    torch.cuda.synchronize()
    _check_attention(c, out)
    assert torch.equal(c.decode(), out)          # the same bits again


@pytest.mark.parametrize("dtype,bits", [("bf16", 0), ("bf16", 4), ("f32", 8)])
def test_rows_of_a_tile_past_the_count_do_not_matter(dtype, bits):
    """A sequence that was stored longer than it now is, as after rejected guesses of a draft model."""
    c = Cache(dtype, bits, 1, 2, 2, 4, 64, [300, 200], 64, seed=8)
    c.write()
    full = [c.unit(0, b, h) for b in range(2) for h in range(2)]
    for rows in ([299, 193], [257, 1], [64, 0]):
        c.s_pages, c.rows = _ints(rows), rows
        out = c.decode()
        torch.cuda.synchronize()
        for b in range(2):
            for h in range(2):
                k, v, kt, vt, idx = full[b * 2 + h]
                q = _np(c.q[0, b, h * 4:(h + 1) * 4])
                want = P.attend(q, idx, k[:rows[b]], v[:rows[b]], kt, vt)
                tol = {"bf16": 2.0 ** -8, "f32": 2e-5}[dtype] * max(np.abs(want).max(initial=0), 1e-30) + {"bf16": 1e-3, "f32": 1e-5}[dtype]
                assert np.abs(_np(out[0, b, h * 4:(h + 1) * 4]) - want).max() <= tol


@pytest.mark.parametrize("T", [128, 51])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_elements_of_any_bits_are_read_back(dtype, T):
    """Every bf16 number there is; fp32 numbers of random bits, NaN of both kinds, infinities and subnormal ones among them."""
    c = Cache(dtype, 0, 1, 1, 2, 1, T, [512], 128, seed=20)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    g = torch.Generator().manual_seed(200)
    if dtype == "bf16":
        x = torch.arange(1 << 16).to(torch.int16)
    else:
        x = torch.randint(-(1 << 31), 1 << 31, (1 << 16,), generator=g).to(torch.int32)
        x[::4] |= 0x7f800000                        # infinities and NaN
        x[1::8] &= -0x7f800001                      # subnormal numbers
        x[:4] = torch.tensor([0x7f800000, -0x800000, 0x7f800001, -1], dtype=torch.int32)
    c.k.view(bits)[0, 0] = torch.stack([x.view(512, D), x.flip(0).view(512, D)]).cuda()
    c.v.view(bits)[0, 0] = torch.stack([x.flip(0).view(512, D), x.view(512, D)]).cuda()
    c.write()
    ko, vo = (torch.empty(1, 1, 2, 512, n, dtype=TDT[dtype], device="cuda") for n in (T, D))
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, 512)
    torch.cuda.synchronize()
    assert torch.equal(vo.view(bits), c.v.view(bits))
    assert torch.equal(ko.view(bits), c.k.view(bits).gather(4, c.idx.long()[..., None, :].expand(1, 1, 2, 512, T)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_value_that_is_not_finite_spoils_its_channel_only(dtype):
    c = Cache(dtype, 0, 1, 3, 2, 3, 51, [300, 64, 20], 64, tails=[0, 9, 64], cap=64, seed=23)
    c.kt[:, 2], c.vt[:, 2] = c.k[:, 2, :, :64].nan_to_num(0, 0, 0), 1.0   # (finite in all rows)
    spots = [("v", 0, 0, 299, 5, float("inf")), ("v", 0, 1, 0, 127, float("nan")), ("v", 1, 0, 63, 64, -float("inf")),
             ("vt", 1, 1, 8, 63, float("inf")), ("vt", 2, 0, 63, 0, float("nan")), ("v", 2, 1, 19, 32, float("inf"))]
    outs = []
    for finite in (True, False):
        for name, b, h, r, ch, x in spots:
            getattr(c, name)[0, b, h, r, ch] = 0.0 if finite else x
        c.write()
        outs.append(c.decode().view(1, 3, 2, 3, D))
    torch.cuda.synchronize()
    assert torch.isfinite(outs[0]).all()
    hit = torch.zeros_like(outs[0], dtype=torch.bool)
    for _, b, h, _, ch, _ in spots:
        hit[0, b, h, :, ch] = True
    assert not torch.isfinite(outs[1][hit]).any() and torch.equal(outs[1][~hit], outs[0][~hit])


@pytest.mark.parametrize("T", [1, 33, 64, 72, 97, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_elements_past_the_count_may_be_anything(dtype, T):
    """Rows of element pages that a shorter count leaves out: infinities and NaN in keys and values, whose tile is still read."""
    c = Cache(dtype, 0, 1, 3, 2, 3, T, [300, 200, 64], 64, tails=[0, 3, 0], cap=8, seed=80 + T)
    rows = [295, 193, 1]
    full = [c.unit(0, b, h) for b in range(3) for h in range(2)]
    for b, n in enumerate(rows):
        for i, bad in enumerate((float("nan"), float("inf"), -float("inf"))):
            c.k[:, b, :, n + i:c.rows[b]:3], c.v[:, b, :, n + i:c.rows[b]:3] = bad, -bad
    c.write()
    c.s_pages, c.rows = _ints(rows), rows
    out = c.decode()
    torch.cuda.synchronize()
    for b in range(3):
        for h in range(2):
            k, v, kt, vt, idx = full[b * 2 + h]
            want = P.attend(_np(c.q[0, b, h * 3:(h + 1) * 3]), idx, k[:rows[b]], v[:rows[b]], kt, vt)
            tol = {"bf16": 2.0 ** -8, "f32": 2e-5}[dtype] * np.abs(want).max() + {"bf16": 1e-3, "f32": 1e-5}[dtype]
            assert np.abs(_np(out[0, b, h * 3:(h + 1) * 3]) - want).max() <= tol


@pytest.mark.parametrize("T", [1, 8, 33, 51, 64, 72, 97, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_keys_of_element_pages_have_no_weight(dtype, T):
    """Rows in use with an infinity in one kept channel, of the sign that makes the logit -inf, in each of the channels; likewise in the
    tail; a sequence that has no other rows."""
    c = Cache(dtype, 0, 1, 3, 2, 1, T, [300, 129, 70], 64, tails=[40, 64, 3], cap=64, seed=180 + T)
    live = {}
    for b in range(3):
        for h in range(2):
            idx, sign = c.idx[0, b, h].long(), torch.sign(c.q[0, b, h]).float()
            assert (sign != 0).all()
            for name, rows, channels in (("k", c.rows[b], idx), ("kt", c.tails[b], torch.arange(D, device="cuda"))):
                hit = np.arange(1, rows, 2) if b < 2 else np.arange(rows)
                at = channels[torch.from_numpy(hit).cuda() // 2 % len(channels)]
                getattr(c, name)[0, b, h, torch.from_numpy(hit).cuda(), at] = (-float("inf") * sign[at]).to(TDT[dtype])
                live[name, b, h] = np.setdiff1d(np.arange(rows), hit)
    c.write()
    out = c.decode()
    torch.cuda.synchronize()
    c_z = {"bf16": 2.0 ** -16, "f32": 2.0 ** -20}[dtype]   # as in _check_attention
    for b in range(3):
        for h in range(2):
            k, v, kt, vt, idx = c.unit(0, b, h)
            ks, ts = live["k", b, h], live["kt", b, h]
            q, got = _np(c.q[0, b, h:h + 1]), _np(out[0, b, h:h + 1])
            assert np.isfinite(k[ks]).all() and np.isfinite(kt[ts]).all() and (len(ks) > 0) == (b < 2)
            want = P.attend(q, idx, k[ks], v[ks], kt[ts], vt[ts])
            top = max(np.abs(v).max(), np.abs(vt).max())
            size = 5.2 * np.abs(q[:, idx]) @ np.abs(k[ks]).max(0, initial=0) + np.abs(q) @ np.abs(kt[ts]).max(0, initial=0)
            assert np.all(np.abs(got - want) <= HALF_STEP[dtype] * np.abs(want) + c_z * top * (2 * size[:, None] / np.sqrt(D) + 5.2)), (b, h)
            assert b < 2 or not got.any()


def test_pages_outside_the_pool_take_no_part():
    c = Cache("bf16", 4, 1, 2, 1, 4, 64, [256, 256], 64, tails=[3, 0], cap=64, seed=21)
    c.write()
    keep = c.table.clone()
    c.table = keep.clone()
    c.table[0, 1], c.table[1, 0], c.table[1, 1], c.table[1, 2], c.table[1, 3] = -1, c.pages.n_pages, 1 << 30, -7, -(1 << 31)
    out = c.decode()
    torch.cuda.synchronize()
    k, v, kt, vt, idx = c.unit(0, 0, 0)
    live = np.r_[0:64, 128:256]
    want = P.attend(_np(c.q[0, 0]), idx, k[live], v[live], kt, vt)
    assert np.abs(_np(out[0, 0]) - want).max() <= 2.0 ** -8 * np.abs(want).max() + 1e-3
    assert not out[0, 1].any()                   # all of its pages are missing


def test_counts_past_the_bounds_are_clamped():
    c = Cache("bf16", 8, 1, 3, 2, 2, 64, [128, 128, 128], 64, tails=[8, 8, 8], cap=8, seed=5)
    c.write()
    want = c.decode()
    c.s_pages, c.s_tail = _ints([1 << 30, 129, 128]), _ints([9, 1 << 30, 8])
    assert torch.equal(c.decode(), want)
    c.s_pages, c.s_tail = _ints([-1, 0, -(1 << 31)]), _ints([0, -1, -(1 << 31)])
    assert not c.decode().any()


@pytest.mark.parametrize("dtype,bits", [("bf16", 4), ("f32", 0)])
def test_every_split_gives_the_same_attention(dtype, bits):
    c = Cache(dtype, bits, 1, 2, 2, 4, 64, [1900, 700], 128, tails=[70, 3], cap=128, seed=31)
    c.write()
    for n in (1, 2, 5, 8, 30, 4096):
        c.shape.n_split = n
        _check_attention(c, c.decode())


# (L, B, N_kv, G, T, rows, page_rows, tails, cap, n_split, S): calls long enough to be cut into pieces by the lengths
_RAGGED = [int(x) for x in np.random.default_rng(77).integers(0, 700, 150)]
BY_LENGTHS = [
    (1, 150, 2, 4, 51, _RAGGED, 64, [b % 3 for b in range(150)], 4, 3, 2000), (1, 3, 4, 2, 64, [20000, 10, 0], 512, [0, 5, 0], 8, 2, 50000),
    (1, 1, 8, 1, 64, [5000], 256, [40], 64, 2, 70000), (1, 64, 1, 17, 33, [63 + b for b in range(64)], 64, None, 0, 2, 9000),
    (2, 2, 4, 8, 97, [2000, 1999], 128, [64, 1], 64, 7, 60000), (1, 65, 4, 4, 64, [0] * 64 + [3000], 64, [0] * 64 + [3], 4, 5, 3000),
]


@pytest.mark.parametrize("case", BY_LENGTHS, ids=[str(i) for i in range(len(BY_LENGTHS))])
@pytest.mark.parametrize("dtype,bits", [("bf16", 4), ("bf16", 0), ("bf16", 8), ("f32", 4)])
def test_pieces_by_the_lengths(dtype, bits, case):
    L, B, N_kv, G, T, rows, page_rows, tails, cap, n_split, S = case
    assert L * B * N_kv * -(-S // 64) >= 8192
    c = Cache(dtype, bits, L, B, N_kv, G, T, rows, page_rows, tails, cap, seed=len(rows) + G, n_split=n_split)
    c.write()
    c.shape.S = S                      # the host's bound; the lengths are what they are
    out = c.decode()
    torch.cuda.synchronize()
    _check_attention(c, out)
    assert torch.equal(c.decode(), out)
    c.shape.n_split = 0
    _check_attention(c, c.decode())


def test_many_sequences_in_pieces():
    """More sequences than are cut by their lengths."""
    rows = [int(x) for x in np.random.default_rng(78).integers(0, 300, 600)]
    c = Cache("bf16", 4, 1, 600, 1, 2, 64, rows, 64, [b % 5 for b in range(600)], 4, seed=90, n_split=3)
    c.write()
    c.shape.S = 2000
    _check_attention(c, c.decode())


def test_offsets_past_32_bits():
    """A pool of more than 4 GiB whose first and last pages are in use, and tails likewise."""
    c = Cache("bf16", 0, 1, 2, 8, 4, 128, [256, 130], 256, tails=[10, 64], cap=64, seed=6, spare=0)
    page = thk.thk_paged_pool_bytes(c.shape, c.pages) // c.pages.n_pages
    n_pages = (5 << 30) // page
    c.pages.n_pages = n_pages
    c.table = torch.tensor([[n_pages - 1], [n_pages // 2 + 7]], dtype=torch.int32, device="cuda")
    c.pool = torch.empty(n_pages * page, dtype=torch.uint8, device="cuda")
    c.write()
    out = c.decode()
    torch.cuda.synchronize()
    _check_attention(c, out)
    ko = torch.empty(1, 2, 8, 256, 128, dtype=torch.bfloat16, device="cuda")
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, None, 256)
    want = c.k.gather(4, c.idx.long()[..., None, :].expand(1, 2, 8, 256, 128))
    for b, n in enumerate(c.rows):
        assert torch.equal(ko[:, b, :, :n], want[:, b, :, :n])


@pytest.mark.parametrize("dtype,bits", [("f32", 0), ("bf16", 4)])
def test_the_largest_pages(dtype, bits):
    """Pages of 65536 rows, of the widest tiles among others; a sequence's last tile is the last of its page, and takes the weight."""
    T = 128
    c = Cache(dtype, bits, 1, 2, 2, 2, T, [65536 + 70, 65530], 65536, seed=6, spare=0)
    hot = [65530, 65500]
    for b, r in enumerate(hot):
        for h in range(2):
            c.k[0, b, h, r] = (40 * c.q[0, b, 2 * h].float() / c.q[0, b, 2 * h].float().norm()).to(c.k.dtype)
    c.write()
    ko, vo = (torch.empty(1, 2, 2, c.S, D, dtype=TDT[dtype], device="cuda") for _ in range(2))
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, c.S)
    out = c.decode()
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(2):
            k, v, kt, vt, idx = c.unit(0, b, h)
            for got, want in ((_np(ko[0, b, h, :c.rows[b]]), k), (_np(vo[0, b, h, :c.rows[b]]), v)):
                assert np.all(np.abs(got - want) <= (0 if bits == 0 else HALF_STEP[dtype]) * np.abs(want))
            q = _np(c.q[0, b, 2 * h:2 * h + 1])
            z = (q[:, idx] @ k.T / np.sqrt(D))[0]
            assert np.argmax(z) == hot[b] and z[hot[b]] - np.sort(z)[-2] > 2
    _check_attention(c, out)


@pytest.mark.parametrize("dtype,bits", [("bf16", 4), ("bf16", 0), ("f32", 8)])
def test_a_ragged_batch_grows(dtype, bits):
    """Prompts stored in whole tiles, their rests in the tails; tokens appended one by one; a full tail goes into pages.
    The whole step is captured once and replayed: lengths, and which sequences flush, change on the device."""
    L, B, N_kv, G, T, cap = 1, 3, 2, 4, 76, 64
    prompts, page_rows, steps = [130, 64, 20], 64, 110
    most = max(prompts) + steps
    c = Cache(dtype, bits, L, B, N_kv, G, T, [most] * B, page_rows, seed=40, S=most)
    idx = _np(c.idx).astype(int)
    # the host's account
    whole = [n // 64 * 64 for n in prompts]
    s_pages, s_tail = _ints([0] * B), _ints([0] * B)
    kt = torch.full((L, B, N_kv, cap, D), float("nan"), dtype=TDT[dtype], device="cuda")
    vt = kt.clone()
    n_prompt, n_whole = _ints(prompts), _ints(whole)
    thk.thk_paged_write(c.shape, c.pages, c.k, c.v, c.S, n_whole, None, c.idx, c.table, c.pool)
    thk.thk_tail_append_ragged(c.shape, c.k, c.v, c.S, n_whole, n_prompt - n_whole, kt, vt, s_tail, cap)
    s_pages += n_whole
    s_tail += n_prompt - n_whole
    k_new = torch.zeros(L, B, N_kv, D, dtype=TDT[dtype], device="cuda")
    v_new = torch.zeros_like(k_new)
    q, out = torch.zeros(L, B, N_kv * G, D, dtype=TDT[dtype], device="cuda"), torch.zeros(L, B, N_kv * G, D, dtype=TDT[dtype], device="cuda")
    ws = ws_tensor(thk.thk_workspace_bytes(c.shape, thk.THK_OP_DECODE_PAGED))

    def step():
        full = torch.where(s_tail == cap, s_tail, torch.zeros_like(s_tail))
        thk.thk_paged_write(c.shape, c.pages, kt, vt, cap, full, s_pages, c.idx, c.table, c.pool)
        s_pages.add_(full)
        s_tail.sub_(full)
        thk.thk_tail_append_ragged(c.shape, k_new, v_new, 1, None, None, kt, vt, s_tail, cap)
        s_tail.add_(1)
        thk.thk_decode_attn_paged(c.shape, c.pages, q, c.pool, c.table, s_pages, c.idx, kt, vt, s_tail, cap, out, ws)

    state = [t.clone() for t in (s_pages, s_tail, kt, vt, c.pool)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t, x in zip((s_pages, s_tail, kt, vt, c.pool), state):
        t.copy_(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for t, x in zip((s_pages, s_tail, kt, vt, c.pool), state):
        t.copy_(x)
    stored, tail = list(whole), [n - w for n, w in zip(prompts, whole)]
    for i in range(steps):
        at = [n + i for n in prompts]
        for b in range(B):
            k_new[:, b], v_new[:, b] = c.k[:, b, :, at[b]], c.v[:, b, :, at[b]]
            if tail[b] == cap:
                stored[b], tail[b] = stored[b] + cap, 0
            tail[b] += 1
        q.copy_(torch.randn(q.shape, generator=c.g, device="cuda"))
        if i % 2:
            step()
        else:
            graph.replay()
        torch.cuda.synchronize()
        assert s_pages.tolist() == stored and s_tail.tolist() == tail
        if i % 9 and tail != [1, 1, 1] and 1 not in tail:
            continue
        for b in range(B):
            for h in range(N_kv):
                kk, vv = _np(c.k[0, b, h, :stored[b] + tail[b]]), _np(c.v[0, b, h, :stored[b] + tail[b]])
                ks, vs = P.stored(kk[:stored[b]][:, idx[0, b, h]], vv[:stored[b]], bits, dtype)
                want = P.attend(_np(q[0, b, h * G:(h + 1) * G]), idx[0, b, h], ks, vs, kk[stored[b]:], vv[stored[b]:])
                tol = {"bf16": 2.0 ** -8, "f32": 2e-5}[dtype] * np.abs(want).max() + {"bf16": 4e-3, "f32": 5e-5}[dtype]
                assert np.abs(_np(out[0, b, h * G:(h + 1) * G]) - want).max() <= tol, (i, b, h)


def test_other_streams_and_refused_tensors():
    c = Cache("bf16", 4, 1, 2, 2, 4, 64, [500, 64], 64, tails=[3, 64], cap=64, seed=50)
    c.write()
    want = c.decode()
    torch.cuda.synchronize()
    c.pool.fill_(255)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.write(stream=side)
    got = torch.full_like(c.q, float("nan"))
    side.wait_stream(torch.cuda.current_stream())
    c.decode(out=got, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    for name, bad in (("q", c.q.float()), ("s_pages", c.s_pages.long()), ("idx", c.idx.int()), ("q", c.q[:, :1]), ("kt", c.kt.transpose(3, 4)),
                      ("table", c.table[:, :1].contiguous()), ("pool", c.pool[:-16]), ("s_tail", c.s_tail[:1]), ("vt", c.vt[..., :32, :].contiguous())):
        keep = getattr(c, name)
        setattr(c, name, bad)
        with pytest.raises(ValueError):
            c.decode(out=got, ws=ws_tensor(1 << 16))
        setattr(c, name, keep)


@pytest.mark.parametrize("bits", [0, 4, 8])
def test_shared_pages(bits):
    """Sequences whose first pages are the same ones, and a sequence that has one page twice."""
    c = Cache("bf16", bits, 1, 3, 2, 4, 64, [384, 384, 256], 128, tails=[5, 0, 64], cap=64, seed=60)
    c.idx[:] = c.idx[:, :1]                       # a shared page holds one choice of channels
    c.k[:, 1, :, :256], c.v[:, 1, :, :256] = c.k[:, 0, :, :256], c.v[:, 0, :, :256]
    c.k[:, 2, :, :128], c.v[:, 2, :, :128] = c.k[:, 0, :, 128:256], c.v[:, 0, :, 128:256]
    c.k[:, 2, :, 128:256], c.v[:, 2, :, 128:256] = c.k[:, 0, :, 128:256], c.v[:, 0, :, 128:256]
    c.write()
    want = c.decode()
    torch.cuda.synchronize()
    _check_attention(c, want)
    c.table[1, :2] = c.table[0, :2]
    c.table[2, :2] = c.table[0, 1]
    assert torch.equal(c.decode(), want)


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own, side by side."""
    cs = [Cache("bf16", 4, 1, 8, 8, 4, 64, [9000 - 900 * b for b in range(8)], 128, seed=70, S=9000),
          Cache("bf16", 8, 1, 2, 8, 4, 76, [9000, 3000], 128, tails=[9, 64], cap=64, seed=71)]
    wants, outs, streams = [], [], [torch.cuda.Stream() for _ in cs]
    for c in cs:
        c.write()
        wants.append(c.decode())
        outs.append(torch.zeros_like(wants[-1]))
    spaces = [ws_tensor(thk.thk_workspace_bytes(c.shape, thk.THK_OP_DECODE_PAGED)) for c in cs]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, out, ws, s in zip(cs, outs, spaces, streams):
            c.decode(out=out, ws=ws, stream=s)
    torch.cuda.synchronize()
    for out, want in zip(outs, wants):
        assert torch.equal(out, want)


@pytest.mark.parametrize("bits", [0, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pools_laid_out_by_others(dtype, bits, monkeypatch):
    """The pools of the measured cases are laid out there, from the description of a tile: rows in them are read as what they are."""
    monkeypatch.syspath_prepend(os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    from perf import operators as O
    for T, N_q, tail in ((51, 2, 20), (76, 16, 0)):
        case = O._case("x", "decode", dtype=dtype, bits=bits, B=3, N_q=N_q, N_kv=2, S=333, T=T, page_rows=64, cap=64, tail=tail, ragged=True)
        st = O.prepare(case, 5)
        O._setup(st)
        got = O._run_own(st)["out"].double()
        want = O.exact(case, 5)["out"]
        # outputs are rounded once; terms and sums as in _check_attention: twice c_z times the sizes of a logit's products, which are
        # below 16, and the largest value, which is below 8
        tol = {"bf16": 2.0 ** -8, "f32": 2.0 ** -23}[dtype] * want.abs() + {"bf16": 2.0 ** -16, "f32": 2.0 ** -20}[dtype] * 256
        assert ((got - want).abs() <= tol).all()
        ko = torch.zeros(1, 3, 2, 333, T, dtype=st["q"].dtype, device="cuda")
        thk.thk_paged_read(st["shape"], st["pages"], st["pool"], st["table"], None, st["rows"], ko, None, 333)
        again = torch.full_like(st["pool"], 255)
        v = torch.zeros(1, 3, 2, 333, D, dtype=st["q"].dtype, device="cuda")
        thk.thk_paged_read(st["shape"], st["pages"], st["pool"], st["table"], None, st["rows"], None, v, 333)
        k = torch.zeros_like(v).scatter_(4, st["idx"].long()[..., None, :].expand(1, 3, 2, 333, T), ko)
        if bits == 0:   # elements go back to where they came from
            thk.thk_paged_write(st["shape"], st["pages"], k, v, 333, st["rows"], None, st["idx"], st["table"], again)
            for b, n in enumerate(st["rows"].tolist()):
                pages = st["table"][b, :n // 64].long()
                assert torch.equal(again[:, pages], st["pool"][:, pages])


@pytest.mark.parametrize("seed", range(48))
def test_random_shapes(seed):
    """Shapes drawn from a seeded generator: stored, read back, attended over."""
    r = np.random.default_rng(4000 + seed)
    pick = lambda *x: x[r.integers(len(x))]   # noqa: E731
    dtype, bits = pick("bf16", "bf16", "f32"), pick(0, 4, 8)
    L, B, N_kv, G, T = int(r.integers(1, 3)), int(r.integers(1, 7)), int(r.integers(1, 4)), pick(1, 2, 3, 4, 5, 7, 8, 12, 16, 17), int(r.integers(1, 129))
    most = int(np.exp(r.uniform(0, np.log(3000))))
    rows = [int(x) for x in r.integers(0, most + 1, B)]
    cap = pick(0, 1, 37, 64, 100, 130)
    tails = [int(x) for x in r.integers(0, cap + 1, B)] if cap else None
    page_rows, n_split = pick(64, 128, 512), pick(0, 0, 1, 2, 3, 9)
    print("random", seed, dtype, bits, L, B, N_kv, G, T, rows, page_rows, tails, cap, n_split, flush=True)
    c = Cache(dtype, bits, L, B, N_kv, G, T, rows, page_rows, tails, cap, seed=100 + seed, n_split=n_split)
    c.write()
    out_rows = c.S + int(r.integers(0, 5))
    ko = torch.full((L, B, N_kv, out_rows, T), 7.0, dtype=TDT[dtype], device="cuda")
    vo = torch.full((L, B, N_kv, out_rows, D), 7.0, dtype=TDT[dtype], device="cuda")
    thk.thk_paged_read(c.shape, c.pages, c.pool, c.table, None, c.s_pages, ko, vo, out_rows)
    out = c.decode()
    torch.cuda.synchronize()
    for b, n in enumerate(rows):
        for l in range(L):
            for h in range(N_kv):
                k, v, _, _, _ = c.unit(l, b, h)
                for got, want in ((_np(ko[l, b, h]), k), (_np(vo[l, b, h]), v)):
                    assert np.all(np.abs(got[:n] - want) <= (0 if bits == 0 else HALF_STEP[dtype]) * np.abs(want))
                    assert np.all(got[n:] == 7)
    _check_attention(c, out)
    assert torch.equal(c.decode(), out)
