"""A serving step around the paged cache on the GPU, against the oracle in 64 bits: token map, rotary positions, pages, beam search,
each at the sizes and values where it can go wrong, and a run of them together, eager and captured."""
import math

import numpy as np
import pytest
import torch

import paper_2407_21018_amd as thk
from helpers import DT, TDT, ws_tensor
from oracle import step as O

pytestmark = pytest.mark.gpu
D = 128
ROUND = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}     # a rounding to the type is off by at most this, relative to the value


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def f64(x):
    return x.detach().cpu().to(torch.float64).numpy()


def bits_of(x):
    return x.contiguous().view(torch.uint8).cpu()


# ---- token map ----------------------------------------------------------------------------
def gpu_map(n_new, pos0, row0, cap, q_rows, n_tokens, starts=True):
    B = len(pos0)
    shape = thk.make_shape(1, B, 1, 1, D, 1, 1, 1)
    out = torch.full((n_tokens + 1, 4), -77, dtype=torch.int32, device="cuda")
    st = torch.full((B + 2,), -77, dtype=torch.int32, device="cuda") if starts else None
    thk.thk_token_map(shape, None if n_new is None else ints(n_new), ints(pos0), None if row0 is None else ints(row0), cap, q_rows, out, n_tokens, st)
    torch.cuda.synchronize()
    assert (out[n_tokens] == -77).all() and (st is None or st[B + 1] == -77)
    return out[:n_tokens].cpu().numpy(), None if st is None else st[:B + 1].tolist()


@pytest.mark.parametrize("B,longest,cap,q_rows,extra", [(1, 1, 1, 1, 0), (1, 700, 512, 32, 3), (3, 0, 8, 1, 5), (7, 333, 100, 32, 0), (64, 5, 64, 0, 1),
                                                        (255, 3, 64, 4, 0), (256, 2, 64, 1, 0), (257, 40, 30, 64, 70), (4096, 3, 2, 2, 10),
                                                        (4097, 3, 2, 2, 10), (9001, 2, 64, 1, 0)])
def test_token_map(B, longest, cap, q_rows, extra):
    rng = np.random.default_rng(B + longest)
    n_new = rng.integers(-1 if B > 2 else 0, longest + 1, B)
    if B == 1:
        n_new[0] = longest
    pos0, row0 = rng.integers(-5, 1 << 20, B), rng.integers(-3, cap + 3, B)
    n = int(np.maximum(n_new, 0).sum()) + extra
    want, starts = O.token_map(n_new, pos0, row0, cap, q_rows, n)
    got, got_starts = gpu_map(n_new, pos0, row0, cap, q_rows, n)
    assert np.array_equal(got, want) and got_starts == starts
    if B <= 4096:
        assert np.array_equal(gpu_map(n_new, pos0, row0, cap, q_rows, n, starts=False)[0], want)
    # fewer records than tokens: the rest is left out
    few = n // 2
    want, starts = O.token_map(n_new, pos0, row0, cap, q_rows, few)
    got, got_starts = gpu_map(n_new, pos0, row0, cap, q_rows, few)
    assert np.array_equal(got, want) and got_starts == starts


def test_token_map_defaults_and_no_tokens():
    want, starts = O.token_map([1] * 5, range(5), [0] * 5, 64, 1, 7)
    got, got_starts = gpu_map(None, list(range(5)), None, 64, 1, 7)
    assert np.array_equal(got, want) and got_starts == starts
    assert gpu_map([3, 4], [0, 0], None, 64, 1, 0)[1] == [0, 0, 0]
    assert gpu_map([0, 0], [0, 0], None, 64, 1, 0)[1] == [0, 0, 0]
    big = 2 ** 31 - 1      # sums past 32 bits: everything behind the first records is left out
    got, starts = gpu_map([5, big, big, big], [9, 0, 0, 0], None, 4, 0, 9)
    assert starts == [0, 5, 9, 9, 9] and got[:, 0].tolist() == [0] * 5 + [1] * 4 and got[:, 2].tolist() == [0, 1, 2, 3, -1, 0, 1, 2, 3]


# ---- rotary positions ---------------------------------------------------------------------
SCALE = {"plain": {}, "linear": dict(factor=8.0), "base": dict(factor=4.0), "ramp": dict(factor=16.0, trained=4096, low=1.0, high=32.0),
         "bands": dict(factor=8.0, trained=8192, low=1.0, high=4.0)}
SCALE_NO = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}


class Rope:
    def __init__(self, dtype, pairs, rot, scaling="plain", base=10000.0, gain=0.0):
        self.rope = thk.make_rope(int(pairs), rot, SCALE_NO[scaling], base=base, gain=gain, **SCALE[scaling])
        self.turns = torch.tensor(thk.thk_rope_turns(self.rope), dtype=torch.int64, device="cuda")
        self.w, own = O.speeds(rot, scaling, base, **SCALE[scaling])
        self.gain = gain or own
        self.dtype, self.pairs, self.rot = dtype, pairs, rot

    def exact(self, x, pos):
        return O.rope(f64(x), pos, self.w, self.gain, self.rot, self.pairs)

    def bound(self, x, want):
        """Sine and cosine within 2^-22; their product with the gain, the two products and the sum rounded to 32 bits: 2^-24 each of at
        most (|x| + |y|) gain; then the rounding to the type.  (Angles of the oracle: positions below 2^20 times 2^-52.)"""
        x = np.abs(f64(x))
        h = self.rot // 2
        i = np.arange(D)
        mate = np.where(i >= self.rot, i, i ^ 1 if self.pairs else np.where(i < h, i + h, i - h))
        e = (x + x[..., mate]) * abs(self.gain) * (2.0 ** -22 + 4 * 2.0 ** -24)
        return e + (np.abs(want) + e) * (ROUND[self.dtype] if self.dtype == "bf16" else 0) + 1e-37


def gpu_rope(r, L, B, N_q, N_kv, q, k, v, record, q_rows, cap, seed=0, out=None, ld=None):
    """(q_out, k_out, v_out, what they were before)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = record.shape[0]
    shape = thk.make_shape(L, B, N_q, N_kv, D, 1, 1, 1, 0, DT[r.dtype])
    make = lambda *s: torch.randn(*s, generator=g, device="cuda").to(TDT[r.dtype])  # noqa: E731
    before = [make(L, n, N_q, D) if q_rows == 0 else make(L, B, N_q, q_rows, D), make(L, B, N_kv, cap, D), make(L, B, N_kv, cap, D)]
    after = [x.clone() for x in before] if out is None else out
    lds = ld or [x.stride(-2) if x is not None else 0 for x in (q, k, v)]
    args = [x for pair in zip((q, k, v), lds) for x in pair]
    outs = [o if x is not None else None for o, x in zip(after, (q, k, v))]
    thk.thk_rope_qkv(shape, r.rope, r.turns, *args, record, n, outs[0], q_rows, outs[1], outs[2], cap)
    torch.cuda.synchronize()
    return after, before


def check_rope(r, L, B, N_q, N_kv, news, pos0, row0, q_rows, cap, pad=0, seed=1, joint=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(news) + pad
    rec, _ = O.token_map(news, pos0, row0, cap, q_rows, n)
    record = ints(rec).reshape(-1, 4)
    make = lambda w: torch.randn(L, n, w * D, generator=g, device="cuda").to(TDT[r.dtype])  # noqa: E731
    if joint:
        q, k, v = make(N_q + 2 * N_kv).split([N_q * D, N_kv * D, N_kv * D], dim=2)
    else:
        q, k, v = make(N_q), make(N_kv), make(N_kv)
    after, before = gpu_rope(r, L, B, N_q, N_kv, q, k, v, record, q_rows, cap)
    for l in range(L):
        for name, x, got, was, heads, col in (("q", q, after[0], before[0], N_q, 3), ("k", k, after[1], before[1], N_kv, 2),
                                              ("v", v, after[2], before[2], N_kv, 2)):
            x = x[l].reshape(n, heads, D)
            y = f64(x) if name == "v" else r.exact(x, rec[:, 1])
            e = np.zeros_like(y) if name == "v" else r.bound(x, y)
            e[..., r.rot:] = 0      # channels that stay keep their bits
            if name == "q" and q_rows == 0:
                live = rec[:, 0] >= 0
                want, tol = np.where(live[:, None, None], y, f64(was[l])), np.where(live[:, None, None], e, 0)
            else:
                want, tol = f64(was[l]), np.zeros(was[l].shape)
                O.place(want, y, rec[:, 0], rec[:, col])
                O.place(tol, e, rec[:, 0], rec[:, col])
            off = np.abs(f64(got[l]) - want)
            assert (off <= tol).all(), (name, l, float((off - tol).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("rot", [4, 6, 8, 16, 20, 24, 44, 64, 96, 126, 128])
def test_rope_parts_of_a_head(dtype, pairs, rot):
    print(f"rope {dtype} pairs={pairs} rot={rot}", flush=True)
    check_rope(Rope(dtype, pairs, rot), 1, 3, 4, 2, [5, 0, 9], [0, 3, 1000], [2, 0, 0], 4, 8, pad=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairs", [False, True])
def test_rope_rot_2(dtype, pairs):
    check_rope(Rope(dtype, pairs, 2), 1, 2, 3, 1, [3, 2], [10, 3], [0, 0], 1, 4)


@pytest.mark.parametrize("scaling", list(SCALE))
@pytest.mark.parametrize("gain", [0.0, 0.7])
def test_rope_scalings(scaling, gain):
    check_rope(Rope("f32", False, 128, scaling, 500000.0, gain), 1, 2, 2, 2, [7, 6], [100000, 1000], [0, 0], 0, 16)
    check_rope(Rope("bf16", True, 44, scaling, 10000.0, gain), 1, 2, 2, 2, [7, 6], [1 << 19, 0], [0, 0], 2, 16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,B,N_q,N_kv,news,q_rows,cap,pad,joint", [
    (1, 1, 1, 1, [1], 1, 1, 0, True), (1, 1, 32, 8, [1], 1, 128, 0, True), (3, 5, 6, 2, [1] * 5, 0, 7, 0, True), (2, 2, 8, 8, [40, 17], 32, 40, 3, False),
    (1, 9, 40, 40, [1] * 9, 1, 64, 1, False), (1, 2, 64, 8, [300, 211], 0, 256, 5, True), (1, 300, 4, 4, [2] * 300, 1, 3, 0, True),
    (1, 1, 7, 1, [2000], 32, 1990, 0, True), (4, 3, 1, 1, [129, 1, 64], 1, 130, 2, False)])
def test_rope_batches(dtype, L, B, N_q, N_kv, news, q_rows, cap, pad, joint):
    print(f"rope {dtype} L={L} B={B} heads={N_q}/{N_kv} q_rows={q_rows} cap={cap}", flush=True)
    rng = np.random.default_rng(B)
    pos0, row0 = rng.integers(0, 5000, B), rng.integers(0, 3, B)
    for pairs, rot in ((False, 128), (True, 128), (False, 44)):
        check_rope(Rope(dtype, pairs, rot), L, B, N_q, N_kv, news, pos0, row0, q_rows, cap, pad, joint=joint)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,B,N_q,N_kv,n,q_rows,share", [(1, 5, 6, 2, 900, 20, 1.0), (2, 3, 16, 4, 512, 7, 0.4), (1, 2, 1, 1, 4000, 3, 1.0), (3, 1, 40, 8, 200, 199, 1.0),
                                                         (1, 1, 8, 1, 3000, 1, 0.0), (1, 7, 40, 40, 640, 90, 1.0)])
def test_rope_queries_that_are_kept_lie_anywhere(dtype, L, B, N_q, N_kv, n, q_rows, share):
    """A map of the caller's: of many tokens few queries have a place, in no order; rows likewise; some records are no tokens."""
    print(f"rope {dtype} L={L} B={B} heads={N_q}/{N_kv} n={n} q_rows={q_rows}", flush=True)
    rng = np.random.default_rng(n + q_rows)
    cap = n // B + 5
    places = rng.permutation(B * cap)[:n]
    rec = np.stack([places // cap, rng.integers(0, 9000, n), places % cap, np.full(n, -1)], 1)
    for b in range(B):
        mine = rng.permutation(np.flatnonzero(rec[:, 0] == b))[:int(q_rows * share)]
        rec[mine, 3] = rng.permutation(q_rows)[:len(mine)]
    rec[rng.permutation(n)[:n // 20], 0] = rng.choice([-1, B, B + 7, -2 ** 31])
    rec[rng.permutation(n)[:n // 20], 2] = rng.choice([-1, cap, 2 ** 31 - 1])
    for pairs, rot in ((False, 128), (True, 96), (False, 44)):
        r = Rope(dtype, pairs, rot)
        g = torch.Generator(device="cuda").manual_seed(n)
        q, k, v = torch.randn(L, n, (N_q + 2 * N_kv) * D, generator=g, device="cuda").to(TDT[dtype]).split([N_q * D, N_kv * D, N_kv * D], dim=2)
        for parts in ((q, k, v), (q, None, v), (q, k, None), (q, None, None)):
            after, before = gpu_rope(r, L, B, N_q, N_kv, *parts, ints(rec), q_rows, cap, ld=[x.stride(-2) if x is not None else 0 for x in parts])
            for name, x, got, was, heads, col in zip("qkv", parts, after, before, (N_q, N_kv, N_kv), (3, 2, 2)):
                if x is None:
                    assert torch.equal(bits_of(got), bits_of(was))
                    continue
                for l in range(L):
                    y = f64(x[l].reshape(n, heads, D)) if name == "v" else r.exact(x[l].reshape(n, heads, D), rec[:, 1])
                    e = np.zeros_like(y) if name == "v" else r.bound(x[l].reshape(n, heads, D), y)
                    e[..., r.rot:] = 0
                    want, tol = f64(was[l]), np.zeros(was[l].shape)
                    O.place(want, y, rec[:, 0], rec[:, col])
                    O.place(tol, e, rec[:, 0], rec[:, col])
                    assert (np.abs(f64(got[l]) - want) <= tol).all(), (name, l, rot)


def test_rope_sines_of_far_positions():
    """(1, 0) turned is cosine and sine; positions over the whole range of 32 bits, the angle by whole numbers in the test too."""
    pos = np.concatenate([np.arange(-300, 300), [2 ** 31 - 1, -2 ** 31, 2 ** 30, 12345678, -87654321],
                          np.random.default_rng(3).integers(-2 ** 31, 2 ** 31, 3000)]).astype(np.int64)
    r = Rope("f32", False, 128)
    n = len(pos)
    rec = np.stack([np.zeros(n, np.int64), pos, np.full(n, -1), np.arange(n)], 1)
    q = torch.zeros(1, n, D, device="cuda")
    q[..., :64] = 1
    after, _ = gpu_rope(r, 1, 1, 1, 1, q, None, None, ints(rec), n, 1)
    got = f64(after[0]).reshape(n, D)
    turns = r.turns.tolist()
    at = np.array([[((int(p) * t) % 2 ** 64) / 2.0 ** 64 for t in turns] for p in pos]) * 2 * math.pi
    assert np.abs(got[:, :64] - np.cos(at)).max() <= 2.0 ** -22 and np.abs(got[:, 64:] - np.sin(at)).max() <= 2.0 ** -22


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_in_place_and_parts_of_the_call(dtype):
    for pairs, rot in ((False, 128), (True, 64), (False, 44)):
        r = Rope(dtype, pairs, rot)
        n, N_q = 37, 5
        rec, _ = O.token_map([n - 2], [11], [0], 64, 0, n)
        q = torch.randn(1, n, N_q * D, device="cuda").to(TDT[dtype])
        after, _ = gpu_rope(r, 1, 1, N_q, 1, q, None, None, ints(rec), 0, 1)
        same = q.clone()
        gpu_rope(r, 1, 1, N_q, 1, same, None, None, ints(rec), 0, 1, out=[same, None, None])
        assert torch.equal(bits_of(same.reshape(-1)[:(n - 2) * N_q * D]), bits_of(after[0].reshape(-1)[:(n - 2) * N_q * D]))
        assert torch.equal(same[:, n - 2:], q[:, n - 2:])      # the last two records are no tokens
        # keys alone, values alone: as with all three
        k, v = (torch.randn(1, n, 1 * D, device="cuda").to(TDT[dtype]) for _ in range(2))
        all3, _ = gpu_rope(r, 1, 1, N_q, 1, q, k, v, ints(rec), 0, 64, seed=4)
        only_k, was = gpu_rope(r, 1, 1, N_q, 1, None, k, None, ints(rec), 0, 64, seed=4)
        only_v, _ = gpu_rope(r, 1, 1, N_q, 1, None, None, v, ints(rec), 0, 64, seed=4)
        assert torch.equal(only_k[1], all3[1]) and torch.equal(only_v[2], all3[2])
        assert torch.equal(only_k[0], was[0]) and torch.equal(only_k[2], was[2]) and torch.equal(only_v[1], was[1])


def test_rope_records_that_name_nothing():
    """Sequences outside the batch, rows outside the buffers: nothing is written for them."""
    r = Rope("bf16", False, 128)
    rec = np.array([[0, 1, 0, 0], [2, 1, 0, 0], [-5, 1, 0, 0], [1, 1, 4, 0], [1, 1, -3, 1], [1, 7, 3, 2], [0, 1, 2, -1], [2 ** 31 - 1, 0, 0, 0]])
    q, k, v = (torch.randn(1, 8, 2 * D, device="cuda").bfloat16() for _ in range(3))
    after, before = gpu_rope(r, 1, 2, 2, 2, q, k, v, ints(rec), 2, 4)
    changed = [(a != b).any(-1).any(2)[0].cpu().numpy() for a, b in zip(after, before)]
    assert changed[0].tolist() == [[True, False], [True, True]]
    assert changed[1].tolist() == changed[2].tolist() == [[True, False, True, False], [False, False, False, True]]


def test_rope_values_that_are_not_finite_stay_in_their_pairs():
    for dtype in ("bf16", "f32"):
        for pairs, rot in ((False, 128), (True, 128), (False, 44), (True, 44)):
            r = Rope(dtype, pairs, rot)
            x = torch.randn(1, 3, D, device="cuda").to(TDT[dtype])
            clean, _ = gpu_rope(r, 1, 1, 1, 1, x, None, None, ints([[0, 5, 0, i] for i in range(3)]), 3, 1)
            y = x.clone()
            y[0, 0, 3], y[0, 1, 2], y[0, 2, 127] = float("nan"), float("inf"), float("nan")
            got, _ = gpu_rope(r, 1, 1, 1, 1, y, None, None, ints([[0, 5, 0, i] for i in range(3)]), 3, 1)
            mate = lambda c: c if c >= rot else c ^ 1 if pairs else c + rot // 2 if c < rot // 2 else c - rot // 2  # noqa: E731
            for i, c in enumerate((3, 2, 127)):
                spoilt = [c, mate(c)] if c < rot else [c]
                keep = [j for j in range(D) if j not in spoilt]
                assert torch.equal(got[0][0, 0, 0, i, keep], clean[0][0, 0, 0, i, keep]) and not torch.isfinite(got[0][0, 0, 0, i, spoilt]).any()


def test_rope_turned_back_is_the_gradient():
    """y = gain R x: the gradient of <c, y> with respect to x is gain R^T c, what the call gives for c at the negative position; against
    differences too, which for a linear function are exact but for rounding: 2 values of at most 8 each off by 2^-22 (|x| + |y|) gain."""
    r = Rope("f32", False, 64, "ramp")
    n = 6
    pos = np.array([0, 1, 17, 4000, 65535, 100000])
    x, c, step = (torch.randn(1, n, D, device="cuda") for _ in range(3))
    turn = lambda y, p: gpu_rope(r, 1, 1, 1, 1, y, None, None, ints(np.stack([0 * p, p, 0 * p, np.arange(n)], 1)), n, 1)[0][0].reshape(n, D)  # noqa: E731
    grad = turn(c, -pos)
    want = f64(c).reshape(n, 1, D).copy()
    a = -pos[:, None] * r.w
    co, si = (r.gain * f(a)[:, None] for f in (np.cos, np.sin))
    u, w = want[..., :32].copy(), want[..., 32:64].copy()
    want[..., :32], want[..., 32:64] = u * co - w * si, w * co + u * si
    assert (np.abs(f64(grad) - want[:, 0]) <= r.bound(c.reshape(n, 1, D), want)[:, 0]).all()
    difference = (f64(turn(x + step, pos)) - f64(turn(x, pos)) - 0) * f64(c)[0]
    assert abs(difference.sum() - (f64(grad) * f64((x + step)[0] - x[0])).sum()) <= n * D * 4 * 8 * 8 * 2.0 ** -21


# ---- pages --------------------------------------------------------------------------------
class Books:
    """The state of a page table on the device."""

    def __init__(self, B, page_rows, max_pages, n_pages, held=None, table=None, refs=None):
        self.shape = thk.make_shape(1, B, 1, 1, D, 64, 1, 1)
        self.pages = thk.make_pages(0, page_rows, max_pages, n_pages)
        self.pr, self.B = page_rows, B
        self.held = ints([0] * B if held is None else held)
        self.table = ints([[-1] * max_pages] * B if table is None else table)
        self.refs = ints([0] * n_pages if refs is None else refs)
        self.room = torch.full((B,), -9, dtype=torch.int32, device="cuda")
        self.moves = torch.full((B, 4), -9, dtype=torch.int32, device="cuda")
        self.ws = ws_tensor(thk.thk_workspace_bytes(self.shape, thk.THK_OP_PAGED_RESERVE))

    def reserve(self, rows, now=None):
        """The call, held against the oracle."""
        want = O.reserve(list(rows), None if now is None else list(now), self.held.tolist(), self.table.tolist(), self.refs.tolist(), self.pr)
        thk.thk_paged_reserve(self.shape, self.pages, ints(rows), None if now is None else ints(now), self.held, self.table, self.refs, self.room,
                              None if now is None else self.moves, self.ws)
        torch.cuda.synchronize()
        got = [self.held.tolist(), self.table.tolist(), self.refs.tolist(), self.room.tolist(), self.moves.tolist()]
        for name, g, w in zip(("held", "table", "refs", "room", "moves"), got, want):
            if name != "moves" or now is not None:
                assert g == w, (name, [(i, a, b) for i, (a, b) in enumerate(zip(g, w)) if a != b][:5])
        return want


@pytest.mark.parametrize("B,page_rows,max_pages,n_pages", [(1, 64, 1, 1), (1, 64, 5, 3), (4, 64, 16, 52), (3, 65536, 4, 9), (64, 128, 40, 1500), (64, 256, 40, 3000),
                                                           (5, 64, 4000, 8191), (5, 64, 4000, 8192), (5, 64, 4000, 8193), (1023, 64, 9, 5000), (1025, 64, 9, 5000),
                                                           (2500, 128, 6, 20000), (300, 64, 400, 70000), (4097, 64, 3, 9000), (40, 64, 3000, 131073),
                                                           (700, 64, 500, 300001)])
def test_reserve_step_by_step(B, page_rows, max_pages, n_pages):
    print(f"reserve B={B} page_rows={page_rows} max_pages={max_pages} n_pages={n_pages}", flush=True)
    rng = np.random.default_rng(B + n_pages)
    pinned = rng.random(n_pages) < 0.1
    books = Books(B, page_rows, max_pages, n_pages, refs=np.where(pinned, rng.integers(1, 4, n_pages), 0))
    top = max_pages * page_rows
    rows = rng.integers(0, top // 2 + 2, B)
    books.reserve(rows)
    for step in range(4):      # most grow a little, some end, some begin, some shrink
        what = rng.random(B)
        rows = np.where(what < 0.6, rows + 1, np.where(what < 0.7, 0, np.where(what < 0.8, rng.integers(0, top + 1, B), rows - rows // 3)))
        rows = np.minimum(rows, top)
        books.reserve(rows)
    books.reserve(rows)        # nothing to do
    books.reserve([0] * B)
    assert (books.refs.cpu().numpy()[~pinned] == 0).all() and (books.table == -1).all()


def test_reserve_clamps_what_is_out_of_range():
    books = Books(6, 64, 4, 30, held=[9, -2, 4, 2, 1, 0], table=[[0, 1, 2, 3], [-1] * 4, [4, 99, -3, 5], [6, 30, -1, -1], [7, -1, -1, -1], [-1] * 4],
                  refs=[1] * 8 + [0] * 8 + [-3] * 4 + [0] * 10)
    books.reserve([64, 65, -5, 0, 1 << 30, 0])
    books.reserve([2 ** 31 - 1, -2 ** 31, 256, 1, 0, 64])


def test_reserve_gives_each_page_to_its_first_user_and_others_copies():
    pr = 128
    # pages 0..3 full and shared by all; page 4 half full: 0, 1, 2 share it; 5: 3 and a user outside; 6: sequence 4 alone; 7: 5 and 6, of which 5 does not grow
    table = [[0, 4, -1], [0, 4, -1], [1, 4, -1], [1, 5, -1], [2, 6, -1], [2, 7, -1], [3, 7, -1], [3, -1, -1]]
    refs = [2, 2, 2, 2, 3, 2, 1, 2] + [0] * 8
    now = [192, 192, 192, 192, 192, 192, 192, 128]
    for rows in ([193, 193, 193, 193, 193, 192, 193, 129], [193, 192, 300, 300, 193, 300, 300, 300], [192] * 7 + [128], [0, 0, 300, 300, 0, 193, 100, 300]):
        for n in (16, 9, 8):      # pages enough, one to give, none
            Books(8, pr, 3, n, held=[2] * 7 + [1], table=table, refs=refs[:n]).reserve(rows, now)


@pytest.mark.parametrize("B,W,n_pages,max_pages", [(8, 4, 60, 6), (1200, 8, 9000, 5), (5000, 5, 20000, 3), (600, 6, 150000, 100)])
def test_reserve_after_sharing(B, W, n_pages, max_pages):
    """Groups of W sequences that share pages, the last one half full, and grow, each as it likes."""
    rng = np.random.default_rng(B)
    pr, held, table, now, at = 256, [], [], [], 0
    refs, order = [0] * n_pages, rng.permutation(n_pages).tolist()
    for g in range(B // W):
        n = int(rng.integers(1, max_pages)) * pr - int(rng.choice([0, 64, 128, 192]))
        pages = order[at:at + -(-n // pr)]
        at += len(pages)
        for j in range(W):
            mine = list(pages)
            if rng.random() < 0.3:
                mine[-1], at = order[at], at + 1
            for p in mine:
                refs[p] += 1
            held.append(len(mine))
            table.append(mine + [-1] * (max_pages - len(mine)))
            now.append(n)
    books = Books(B, pr, max_pages, n_pages, held, table, refs)
    rows = [n + int(rng.choice([0, 1, 64, 300])) for n in now]
    books.reserve(rows, now)
    books.reserve(rows, now)      # everybody has a page of their own now


@pytest.mark.parametrize("B,n_pages", [(64, 8192), (64, 8193), (65, 8192), (65, 500), (1024, 20000), (1025, 20000), (1024, 49152), (1024, 49153), (64, 49152), (64, 49153), (1500, 3000), (4096, 65536), (4097, 30000)])
def test_reserve_at_the_limits_of_its_forms(B, n_pages):
    """Each way in which the call is laid out, at its last size and one past it; runs of sequences share the page that they grow in."""
    print(f"reserve B={B} n_pages={n_pages}", flush=True)
    rng = np.random.default_rng(B + n_pages)
    pr, most = 128, max(2, min(40, n_pages // B - 2))
    refs, order, at = [0] * n_pages, rng.permutation(n_pages).tolist(), 0
    held, table, now = [], [], []
    for b in range(B):
        n = int(rng.integers(0, most * pr))
        pages, at = order[at:at + -(-n // pr)], at + -(-n // pr)
        if b and rng.random() < 0.4:
            n, pages, at = now[b - 1], table[b - 1][:held[b - 1]], at - len(pages)
        for p in pages:
            refs[p] += 1
        held.append(len(pages))
        now.append(n)
        table.append(pages + [-1] * (most + 1 - len(pages)))
    books = Books(B, pr, most + 1, n_pages, held, table, refs)
    rows = [max(0, n + int(rng.choice([0, 1, 1, 64, pr, -n, -pr]))) for n in now]
    books.reserve(rows, now)
    books.reserve(rows, None)
    room = books.room.tolist()
    books.reserve([n + int(rng.choice([0, 1, pr])) for n in rows], [min(n, r) for n, r in zip(rows, room)])


@pytest.mark.parametrize("dtype,bits,T,page_rows", [("bf16", 4, 64, 256), ("bf16", 0, 51, 128), ("f32", 8, 33, 64), ("f32", 0, 128, 1024), ("bf16", 8, 1, 4096)])
def test_paged_copy(dtype, bits, T, page_rows):
    L, N, n = 3, 2, 9
    shape = thk.make_shape(L, 4, N, N, D, 64, 1, T, 0, DT[dtype])
    pages = thk.make_pages(bits, page_rows, 4, n)
    size = thk.thk_paged_pool_bytes(shape, pages)
    pool = torch.randint(0, 256, (size,), dtype=torch.uint8, device="cuda")
    tpp = page_rows // 64
    for moves in ([[0, 8, tpp, 0], [3, 1, 1, 0], [-1, -1, 0, 0], [5, 9, 1, 0], [9, 2, 1, 0], [-1, 4, 1, 0], [3, 6, 0, 0], [2, 7, 1000000, 0]], [[8, 0, tpp - 1, 0]]):
        before = pool.clone().reshape(L, n, N, tpp, -1)
        thk.thk_paged_copy(shape, pages, ints(moves), len(moves), pool)
        torch.cuda.synchronize()
        want = before.clone()
        for src, dst, tiles, _ in moves:
            if 0 <= src < n and 0 <= dst < n:
                want[:, dst, :, :tiles] = before[:, src, :, :tiles]
        assert torch.equal(pool, want.reshape(-1))


# ---- beam search --------------------------------------------------------------------------
def gpu_select(x, scores, done, K, eos, ld=0, in_place=False):
    """x [B, W, ld or V] on the GPU."""
    B, W = scores.shape
    V = x.shape[2] if not ld else ld[1]
    beams = thk.make_beams(B, W, K, V, 0 if not ld else x.shape[2], thk.THK_F32 if x.dtype == torch.float32 else thk.THK_BF16, eos)
    ws = ws_tensor(thk.thk_beam_workspace_bytes(beams))
    ws.fill_(0xff)
    s = torch.tensor(scores, dtype=torch.float32, device="cuda")
    d = None if done is None else ints(done)
    out = [torch.full((B, K), -7, dtype=torch.int32, device="cuda") for _ in range(3)] + [torch.full((B, K), -7.0, device="cuda")]
    if in_place:
        out[3], out[2] = s, out[2] if d is None else d
    thk.thk_beam_select(beams, x, s, d, out[0], out[1], out[3], out[2], ws)
    torch.cuda.synchronize()
    return [o.cpu().numpy() for o in (out[0], out[1], out[3], out[2])]


# A row's sum is of terms 2^(x L - c), c at most 8 L below x L for the largest element of a lane: the exponent is rounded once, 2^-24 of itself
# at most, and L, log2 e in 32 bits, is off by 2^-26 (beyond 2^20 the difference x - r is rounded first, once more).  With |d| = |x - r|, a term is off by 2.25 2^-24 |d|
# of itself; the sum by that of the mean of |d| under its own weights, which is at most 8 + ln V (the largest element's distance to the mean
# is an entropy's part).  2^y is within 2^-23, and so is what makes c's own rounding good; three sums of 2^-24 lie between, before 64 bits.
def sum_error(V):
    return 2.25 * 2.0 ** -24 * (8 + math.log(V)) + 7 * 2.0 ** -24


def check_select(x, scores, done, K, eos, **kw):
    V = kw["ld"][1] if kw.get("ld") else x.shape[2]
    d = np.zeros(scores.shape, int) if done is None else np.asarray(done)
    scores = scores.astype(np.float32)
    parent, token, score, ended = O.beam_select(f64(x)[..., :V], scores.astype(np.float64), d, K + 1, eos)
    # the test's own inputs: neighbours are equal (of one beam, or of beams that are alike) or further apart than the sums' errors
    near = (parent[:, 1:] >= 0) & (np.diff(score) != 0) & (np.abs(np.diff(score)) < 2 * sum_error(V)) & (parent[:, 1:] != parent[:, :-1])
    assert not near.any(), "two beams' continuations are too near for a test"
    got = gpu_select(x, scores, done, K, eos, **kw)
    parent, token, score, ended = (y[:, :K] for y in (parent, token, score, ended))
    assert np.array_equal(got[0], parent) and np.array_equal(got[1], token) and np.array_equal(got[3], ended)
    fine = np.isfinite(score)
    assert np.array_equal(np.isneginf(got[2]), ~fine) or np.abs(score[fine]).max() > 3e38
    off = np.abs(got[2].astype(np.float64) - score)[fine & np.isfinite(got[2])]
    assert (off <= sum_error(V) + 2.0 ** -24 * np.abs(score[fine & np.isfinite(got[2])])).all(), off.max()


def logits(rng, B, W, V, dtype, scale=2.0):
    return torch.tensor(rng.standard_normal((B, W, V)) * scale, dtype=torch.float32).to(TDT[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,W,K,V", [(1, 1, 1, 1), (2, 1, 3, 2), (1, 4, 8, 7), (3, 2, 64, 9), (2, 32, 64, 3), (2, 5, 10, 63), (2, 5, 10, 64), (1, 3, 6, 513),
                                     (2, 4, 4, 1023), (1, 4, 8, 2047), (1, 4, 8, 2048), (1, 4, 64, 2049), (1, 32, 64, 4095), (3, 8, 16, 8191), (2, 8, 16, 8193),
                                     (1, 2, 4, 50001), (1, 1, 64, 131073), (5, 3, 5, 32768)])
def test_beam_select(dtype, B, W, K, V):
    print(f"beam {dtype} B={B} W={W} K={K} V={V}", flush=True)
    rng = np.random.default_rng(V * 37 + W)
    x, s = logits(rng, B, W, V, dtype), -10 * rng.random((B, W))
    check_select(x, s, None, K, -1)
    check_select(x, s, rng.random((B, W)) < 0.4, K, V // 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,W,K,V", [(64, 8, 16, 65001), (30, 8, 8, 131073), (64, 16, 16, 40000), (64, 4, 8, 32000), (23, 8, 8, 208660), (300, 32, 5, 7000), (1, 32, 64, 150001), (1, 9, 33, 70001)])
def test_beam_select_large_calls(dtype, B, W, K, V):
    """Rows in few pieces of many tiles, blocks in several rounds: two prompts against the oracle, the others are the same two."""
    print(f"beam {dtype} B={B} W={W} K={K} V={V}", flush=True)
    rng = np.random.default_rng(V + W)
    P = min(B, 2)
    x, s = logits(rng, P, W, V, dtype), (-10 * rng.random((P, W))).astype(np.float32)
    check_select(x, s, None, K, -1)
    want = gpu_select(x, s, None, K, -1)
    which = np.arange(B) % P
    got = gpu_select(x[torch.tensor(which).cuda()].contiguous(), s[which], None, K, -1)
    for name, g, w in zip(("parent", "token", "score", "done"), got, want):
        if name != "score":
            assert np.array_equal(g, w[which]), name
        else:      # another number of pieces, another order of the same sum
            assert (np.abs(g.astype(np.float64) - w[which]) <= 2 * sum_error(V) + 2.0 ** -23 * np.abs(w[which])).all()


def test_beam_select_many_rows():
    """Rows of the same quarters in other orders have the same sum, and scores in steps of 1/32 keep their continuations apart."""
    rng = np.random.default_rng(5)
    base = np.round(rng.standard_normal(3001) * 8) / 4
    x = torch.tensor(np.stack([rng.permutation(base) for _ in range(2400)]).reshape(300, 8, 3001), dtype=torch.float32).bfloat16().cuda()
    check_select(x, -rng.permuted(np.tile(np.arange(8) / 32, (300, 1)), axis=1), None, 16, 7)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_beam_select_rows_that_are_padded(dtype):
    rng = np.random.default_rng(6)
    for V, ld in ((1000, 1001), (1001, 1024), (5, 2050)):
        x = logits(rng, 2, 3, ld, dtype)
        x[..., V:] = float("nan")
        check_select(x, -5 * rng.random((2, 3)), None, 6, 1, ld=(ld, V))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_beam_select_masks(dtype):
    rng = np.random.default_rng(7)
    V = 4100
    x = logits(rng, 6, 3, V, dtype)
    inf = float("inf")
    x[0][:, torch.tensor(rng.random(V) < 0.95).cuda()] = -inf       # few are left
    x[1] = -inf                                                     # none
    x[2, 0], x[2, 1, 5:], x[2, 2, :] = -inf, -inf, -inf             # five, of one beam
    x[3, 0, 17], x[3, 1, 4099] = float("nan"), inf                  # these beams have none
    x[4] = torch.finfo(TDT[dtype]).min                              # the lowest value is a value: all alike
    x[5, 0, :4000], x[5, 1, 3:] = torch.finfo(TDT[dtype]).min, torch.finfo(TDT[dtype]).min
    s = -5 * rng.random((6, 3))
    check_select(x, s, None, 8, 3)
    x[5] = 0
    s[0, 0], s[1, 1], s[2, 2], s[5, 0], s[5, 2] = -inf, inf, float("nan"), -inf, 3e38
    check_select(x, s, None, 6, 3)
    check_select(x, s, np.ones((6, 3)), 6, 3)


def test_beam_select_far_values():
    """Logits of any size up to the end of the range, of either sign: what is small about them is their differences, and differences may
    have no place in 32 bits."""
    rng = np.random.default_rng(10)
    for shift in (1e3, -1e4, 2.0 ** 20, -2.0 ** 20 - 1, 3e7, -1e9):
        x = torch.tensor(np.round(rng.standard_normal((2, 3, 4100)) * 3) * max(1.0, abs(shift) * 2.0 ** -23) + shift, dtype=torch.float32, device="cuda")
        check_select(x, -np.arange(6).reshape(2, 3) / 7, None, 9, 1)
    for values in ([3.2e38, 3.1e38, -3.2e38], [-3.2e38, -3.3e38, -3.4e38], [1.5e38, -1.5e38, 9e37], [-9e37, -1.1e38, 0.0], [1e38, 1.0000001e38, 5.0]):
        x = torch.full((1, 2, 5000), values[2], device="cuda")
        x[0, 0, 4000], x[0, 0, 17], x[0, 1, 4999], x[0, 1, 4998] = values[0], values[1], values[0], values[0]
        check_select(x, np.array([[0.0, 0.25]]), None, 3, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_beam_select_equal_values(dtype):
    rng = np.random.default_rng(8)
    zero = np.zeros((2, 4))
    for V in (5, 300, 2050, 20000):
        x = torch.zeros(2, 4, V, device="cuda").to(TDT[dtype])
        check_select(x, zero, None, 9, 0)                           # all equal: the first tokens of the first beam
        x[:, :, 1::2] = -0.0                                        # which is the same number
        check_select(x, zero, None, 9, 0)
        few = torch.tensor(rng.integers(0, 3, (2, 1, V)), dtype=torch.float32).to(TDT[dtype]).cuda()
        check_select(few.expand(2, 4, V).contiguous(), zero, None, 33, 0)     # beams that are alike, three values
        if V > 8:
            x = torch.arange(V, device="cuda").float().neg().div(V)
            x = torch.where(torch.arange(V, device="cuda") % 7 == 3, 1.0, x).to(TDT[dtype]).expand(2, 4, V).contiguous()
            check_select(x, zero, None, 40, 3)


@pytest.mark.parametrize("K", [2, 3, 5, 8])
def test_beam_select_logits_that_64_bits_do_not_tell_apart(K):
    """Below 1e38 the scores of 5, 4 and 3 are one number: a beam's continuations are in the order of their logits all the same."""
    x = torch.full((1, 3, 5000), float("-inf"), device="cuda")
    for w in range(3):
        x[0, w, 4000], x[0, w, 100 + w], x[0, w, 7], x[0, w, 4999] = 1e38, 5.0, 4.0, 3.0
    x[0, 2, 8] = 4.0
    check_select(x, np.array([[0.0, 0.25, -0.5]]), None, K, 1)


def test_beam_select_orders_that_keep_the_list_busy():
    V = 70001
    up = torch.arange(V, dtype=torch.float32, device="cuda").div(1000).expand(1, 2, V).contiguous()
    s = np.array([[0.0, -0.5003]])
    for x in (up, up.flip(2).contiguous(), torch.cat([up[..., 35000:], up[..., :35000]], dim=2)):
        check_select(x, s, None, 64, 0)


def test_beam_select_sums_are_exact_where_beams_are_near():
    """Two beams whose best scores differ by 2^-19 through their sums alone, one logit far below the others."""
    V = 1000
    x = torch.zeros(1, 2, V, dtype=torch.float32, device="cuda")
    x[0, 0, 999], x[0, 1, 999] = -5.0, -5.5
    check_select(x, np.zeros((1, 2)), None, 3, -1)


def test_beam_select_in_place_on_another_stream_and_twice():
    rng = np.random.default_rng(9)
    x, s, d = logits(rng, 3, 4, 9000, "bf16"), -10 * rng.random((3, 4)).astype(np.float32), rng.random((3, 4)) < 0.3
    want = gpu_select(x, s, d, 4, 1)
    for _ in range(3):
        got = gpu_select(x, s, d, 4, 1, in_place=True)
        assert all(np.array_equal(g, w) for g, w in zip(got, want))
    with torch.cuda.stream(torch.cuda.Stream()):
        got = gpu_select(x, s, d, 4, 1)
    assert all(np.array_equal(g, w) for g, w in zip(got, want))


# ---- reordering ---------------------------------------------------------------------------
def reorder_case(dtype, L, prompts, W, N, cap, page_rows, max_pages, seed, paged=True, extra=0):
    rng = np.random.default_rng(seed)
    B = prompts * W
    g = torch.Generator(device="cuda").manual_seed(seed)
    kt, vt = (torch.randn(L, B, N, max(cap, 1), D, generator=g, device="cuda").to(TDT[dtype]) for _ in range(2))
    parent = rng.integers(-1, W + 1, (prompts, W + extra))
    s_tail = rng.integers(-1, cap + 2, B).tolist()
    s_pages = (rng.integers(0, max_pages * page_rows // 64 + 1, B) * 64).tolist()
    held = [min(max_pages, -(-n // page_rows) + int(rng.integers(0, 2))) for n in s_pages]
    n_pages = sum(held) + 5
    order, at, table, refs = rng.permutation(n_pages).tolist(), 0, [], [0] * n_pages
    for b, n in enumerate(held):
        row = order[at:at + n]
        at += n
        if b % W and n > 1 and held[b - 1] > 1:      # the first page in common with the neighbour
            row[0] = table[b - 1][0]
        for p in row:
            refs[p] += 1
        table.append(row + [-1] * (max_pages - n))
    return parent, kt, vt, s_tail, s_pages, held, table, refs, n_pages


@pytest.mark.parametrize("dtype,L,prompts,W,N,cap,page_rows,max_pages,extra", [
    ("bf16", 1, 1, 1, 1, 4, 64, 1, 0), ("bf16", 1, 2, 4, 8, 128, 128, 9, 4), ("f32", 2, 3, 5, 3, 33, 64, 20, 0), ("bf16", 2, 2, 8, 2, 65, 256, 5, 8),
    ("f32", 1, 2, 9, 1, 64, 64, 300, 1), ("bf16", 1, 1, 16, 1, 7, 64, 6, 16), ("bf16", 3, 2, 32, 2, 20, 128, 8, 0), ("f32", 1, 2, 17, 2, 5, 64, 3, 3),
    ("bf16", 1, 2, 2, 1, 0, 64, 700, 0), ("bf16", 4, 1, 3, 4, 200, 64, 2, 0)])
def test_reorder(dtype, L, prompts, W, N, cap, page_rows, max_pages, extra):
    print(f"reorder {dtype} L={L} prompts={prompts} W={W} cap={cap}", flush=True)
    for seed in range(4):
        parent, kt, vt, s_tail, s_pages, held, table, refs, n_pages = reorder_case(dtype, L, prompts, W, N, cap, page_rows, max_pages, seed, extra=extra)
        shape = thk.make_shape(L, prompts * W, N, N, D, 64, 1, 64, 0, DT[dtype])
        pages = thk.make_pages(0, page_rows, max_pages, n_pages)
        tails = [kt, vt] if cap else []
        want = O.reorder(parent.tolist(), W, [f64(t) for t in tails], s_tail, s_pages, held, table, refs, page_rows)
        dev = [ints(v) for v in (s_tail, s_pages, held, table, refs)]
        thk.thk_beam_reorder(shape, pages, W, ints(parent), W + extra, kt if cap else None, vt if cap else None, dev[0], cap, *dev[1:])
        torch.cuda.synchronize()
        for t, w in zip(tails, want[0]):
            assert np.array_equal(f64(t), w)
        for name, g, w in zip(("s_tail", "s_pages", "held", "table", "refs"), dev, want[1:]):
            assert g.tolist() == w, name


def test_reorder_without_pages():
    parent, kt, vt, s_tail, s_pages, *_ = reorder_case("bf16", 2, 2, 4, 2, 30, 64, 3, 11)
    shape = thk.make_shape(2, 8, 2, 2, D, 64, 1, 64, 0, thk.THK_BF16)
    want = O.reorder(parent.tolist(), 4, [f64(kt), f64(vt)], s_tail, s_pages, None, None, None, 64)
    st, sp = ints(s_tail), ints(s_pages)
    thk.thk_beam_reorder(shape, None, 4, ints(parent), 4, kt, vt, st, 30, sp, None, None, None)
    torch.cuda.synchronize()
    assert np.array_equal(f64(kt), want[0][0]) and np.array_equal(f64(vt), want[0][1]) and st.tolist() == want[1] and sp.tolist() == want[2]


# ---- together -----------------------------------------------------------------------------
class Server:
    """A decode loop with beam search over a paged cache: what each step's tokens, keys, values and logits are comes from seeded
    tables; everything between them is the library's."""

    def __init__(self, steps, prompts=2, W=3, N=2, G=2, T=40, page_rows=128, seed=0, bits=0):
        self.steps, self.P, self.W, self.N, self.G, self.T, self.V = steps, prompts, W, N, G, T, 500
        B = self.B = prompts * W
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.H = N * G
        self.qkv = rnd(steps, B, (self.H + 2 * N) * D)
        self.logits = rnd(steps, prompts, W, self.V) * 2
        one = torch.stack([torch.randperm(D, generator=g, device="cuda")[:T].sort().values for _ in range(prompts * N)]).reshape(prompts, 1, N, T)
        self.idx = one.expand(prompts, W, N, T).reshape(B, N, T).to(torch.int16).contiguous()
        self.cap = 64
        most = steps + 64
        self.shape = thk.make_shape(1, B, self.H, N, D, most, 1, T, 0, thk.THK_F32)
        self.mp = -(-most // page_rows) + 1
        n_pages = B * self.mp
        self.pages = thk.make_pages(bits, page_rows, self.mp, n_pages)
        self.r = Rope("f32", False, 128)
        z = lambda *s, t=torch.int32: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        self.s_tail, self.s_pages, self.held, self.refs, self.room = z(B), z(B), z(B), z(n_pages), z(B)
        self.table, self.moves, self.map = torch.full((B, self.mp), -1, dtype=torch.int32, device="cuda"), z(B, 4), z(B, 4)
        self.kt, self.vt = z(1, B, N, self.cap, D, t=torch.float32), z(1, B, N, self.cap, D, t=torch.float32)
        self.pool = z(thk.thk_paged_pool_bytes(self.shape, self.pages), t=torch.uint8)
        self.q_out, self.out = z(B, self.H, 1, D, t=torch.float32), z(B, self.H, D, t=torch.float32)
        self.scores = torch.zeros(prompts, W, device="cuda")
        self.scores[:, 1:] = float("-inf")            # the beams of a prompt begin as one
        self.done = z(prompts, W)
        self.parent, self.token = z(prompts, W), z(prompts, W)
        self.beams = thk.make_beams(prompts, W, W, self.V, 0, thk.THK_F32, 0)
        self.ws = [ws_tensor(n) for n in (thk.thk_workspace_bytes(self.shape, thk.THK_OP_PAGED_RESERVE),
                                          thk.thk_workspace_bytes(self.shape, thk.THK_OP_DECODE_PAGED), thk.thk_beam_workspace_bytes(self.beams))]
        self.in_qkv, self.in_logits = torch.zeros_like(self.qkv[0]), torch.zeros_like(self.logits[0])
        self.rows, self.full, self.pos = z(B), z(B), z(B)
        self.seen = []

    def step(self):
        """One token: everything is on the device."""
        # tails that are full go to pages of their beam's own
        self.full.copy_(torch.where(self.s_tail == self.cap, self.cap, 0))
        self.rows.copy_(self.s_pages + self.full)
        thk.thk_paged_reserve(self.shape, self.pages, self.rows, self.s_pages, self.held, self.table, self.refs, self.room, self.moves, self.ws[0])
        thk.thk_paged_copy(self.shape, self.pages, self.moves, self.B, self.pool)
        thk.thk_paged_write(self.shape, self.pages, self.kt, self.vt, self.cap, self.full, self.s_pages, self.idx, self.table, self.pool)
        self.s_pages.add_(self.full)
        self.s_tail.sub_(self.full)
        self.pos.copy_(self.s_pages + self.s_tail)
        thk.thk_token_map(self.shape, None, self.pos, self.s_tail, self.cap, 1, self.map, self.B)
        q, k, v = self.in_qkv.split([self.H * D, self.N * D, self.N * D], dim=1)
        ld = self.in_qkv.shape[1]
        thk.thk_rope_qkv(self.shape, self.r.rope, self.r.turns, q, ld, k, ld, v, ld, self.map, self.B, self.q_out, 1, self.kt, self.vt, self.cap)
        self.s_tail.add_(1)
        thk.thk_decode_attn_paged(self.shape, self.pages, self.q_out, self.pool, self.table, self.s_pages, self.idx, self.kt, self.vt, self.s_tail, self.cap,
                                  self.out, self.ws[1])
        thk.thk_beam_select(self.beams, self.in_logits, self.scores, self.done, self.parent, self.token, self.scores, self.done, self.ws[2])
        thk.thk_beam_reorder(self.shape, self.pages, self.W, self.parent, self.W, self.kt, self.vt, self.s_tail, self.cap, self.s_pages, self.held,
                             self.table, self.refs)

    def feed(self, t):
        self.in_qkv.copy_(self.qkv[t])
        self.in_logits.copy_(self.logits[t])

    def state(self):
        return [x.clone() for x in (self.out, self.parent, self.token, self.scores, self.s_tail, self.s_pages, self.held, self.table, self.refs, self.kt, self.vt)]


def test_beam_search_over_a_paged_cache():
    """150 steps against histories kept on the host: every beam's attention is over its own ancestors' keys and values."""
    s = Server(150)
    history = [[] for _ in range(s.B)]          # (step, beam it was then) of every token of a beam
    qkv = f64(s.qkv).reshape(s.steps, s.B, s.H + 2 * s.N, D)
    pos = np.arange(s.steps)
    turned = np.stack([O.rope(qkv[t], [t] * s.B, s.r.w, 1.0, 128, False) for t in pos])
    scores, done = f64(s.scores), np.zeros((s.P, s.W), int)
    idx = s.idx.cpu().numpy().astype(int)
    for t in range(s.steps):
        s.feed(t)
        s.step()
        torch.cuda.synchronize()
        for b in range(s.B):
            history[b].append((t, b))
        if t % 13 == 0 or t == s.steps - 1 or t in (63, 64, 65, 128, 129):
            for b in range(s.B):
                rows = len(history[b])
                in_pages = (rows - 1) // 64 * 64          # a full tail goes to pages in front of the next token
                k = np.stack([turned[u, c, s.H:s.H + s.N] for u, c in history[b]], 1)
                v = np.stack([qkv[u, c, s.H + s.N:] for u, c in history[b]], 1)
                for h in range(s.H):
                    kv = h // s.G
                    q, keys = turned[t, b, h], k[kv].copy()
                    kept = np.zeros(D)
                    kept[idx[b, kv]] = 1
                    keys[:in_pages] *= kept
                    z = keys @ q / math.sqrt(D)
                    p = np.exp(z - z.max())
                    want = p @ v[kv] / p.sum()
                    assert np.abs(f64(s.out[b, h]) - want).max() <= 1e-4 * np.abs(want).max(), (t, b, h)
        parent, token, score, ended = O.beam_select(f64(s.logits[t]), scores, done, s.W, 0)
        assert np.array_equal(s.parent.cpu().numpy(), parent) and np.array_equal(s.token.cpu().numpy(), token) and np.array_equal(s.done.cpu().numpy(), ended)
        scores, done = f64(s.scores), ended
        old = [list(h) for h in history]
        for p in range(s.P):
            for j in range(s.W):
                if parent[p, j] >= 0:
                    history[p * s.W + j] = list(old[p * s.W + parent[p, j]])
        table, held, refs = s.table.tolist(), s.held.tolist(), s.refs.tolist()
        users = [0] * len(refs)
        for row, n in zip(table, held):
            for q in row[:n]:
                users[q] += 1
        assert users == refs                     # the books are right after every step


def test_a_captured_step_is_the_eager_one():
    """The step as a graph, replayed while an eager server does the same beside it: identical bits after every replay."""
    eager, graphed = Server(140, W=4, seed=3, bits=8), Server(140, W=4, seed=3, bits=8)
    for s in (eager, graphed):      # the first steps, which load the kernels
        for t in range(3):
            s.feed(t)
            s.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed.step()
    for t in range(3, 140):
        for s in (eager, graphed):
            s.feed(t)
        eager.step()
        g.replay()
        if t % 10 == 0 or t > 125:
            torch.cuda.synchronize()
            for a, b in zip(eager.state(), graphed.state()):
                assert torch.equal(bits_of(a), bits_of(b)), t


def test_steps_on_other_streams_side_by_side():
    """Two servers, each on a stream of its own and not waiting for the other, and one on the current stream: identical bits."""
    servers = [Server(70, seed=5, bits=4) for _ in range(3)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.current_stream()]
    torch.cuda.synchronize()
    for t in range(70):
        for s, st in zip(servers, streams):
            with torch.cuda.stream(st):
                s.feed(t)
                s.step()
    torch.cuda.synchronize()
    for other in servers[:2]:
        for a, b in zip(other.state(), servers[2].state()):
            assert torch.equal(bits_of(a), bits_of(b))


@pytest.mark.parametrize("B,n_pages", [(40, 3000), (700, 20000), (1500, 9000), (300, 70000), (4200, 15000)])
def test_a_captured_plan(B, n_pages):
    """Pages and token map of every form as a graph, rows that change from replay to replay, against the eager calls."""
    print(f"captured plan B={B} n_pages={n_pages}", flush=True)
    rng = np.random.default_rng(B)
    eager, graphed = (Books(B, 64, 8, n_pages) for _ in range(2))
    rows, now, new = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    maps = [torch.zeros(3 * B, 4, dtype=torch.int32, device="cuda") for _ in range(2)]
    starts = [torch.zeros(B + 1, dtype=torch.int32, device="cuda") for _ in range(2)]

    def plan(b, m, st):
        thk.thk_paged_reserve(b.shape, b.pages, rows, now, b.held, b.table, b.refs, b.room, b.moves, b.ws)
        thk.thk_token_map(b.shape, new, now, None, 64, 1, m, 3 * B, st)

    for b, m, st in zip((eager, graphed), maps, starts):
        plan(b, m, st)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        plan(graphed, maps[1], starts[1])
    for _ in range(6):
        now.copy_(torch.minimum(rows, eager.room))
        rows.copy_(ints(rng.integers(0, 8 * 64 + 1, B)))
        new.copy_(ints(rng.integers(0, 4, B)))
        plan(eager, maps[0], starts[0])
        g.replay()
        torch.cuda.synchronize()
        for name in ("held", "table", "refs", "room", "moves"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), name
        assert torch.equal(*maps) and torch.equal(*starts)


def test_two_graphs_may_share_a_workspace_and_streams_need_one_each():
    rng = np.random.default_rng(12)
    a, b = logits(rng, 2, 4, 30000, "bf16"), logits(rng, 2, 4, 20001, "bf16")
    s = -5 * rng.random((2, 4))
    want = [gpu_select(x, s, None, 8, 1) for x in (a, b)]
    beams = [thk.make_beams(2, 4, 8, x.shape[2], 0, thk.THK_BF16, 1) for x in (a, b)]
    ws = ws_tensor(max(thk.thk_beam_workspace_bytes(x) for x in beams))
    sc = torch.tensor(s, dtype=torch.float32, device="cuda")
    outs, graphs = [], []
    for x, bm in zip((a, b), beams):
        o = [torch.zeros(2, 8, dtype=torch.int32, device="cuda") for _ in range(2)] + [torch.zeros(2, 8, device="cuda")]
        thk.thk_beam_select(bm, x, sc, None, o[0], o[1], o[2], None, ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            thk.thk_beam_select(bm, x, sc, None, o[0], o[1], o[2], None, ws)
        outs.append(o)
        graphs.append(g)
    for _ in range(3):
        for o in outs:
            for y in o:
                y.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(np.array_equal(y.cpu().numpy(), z) for y, z in zip(o, w))
    streams, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(ws) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, bm, o, st, w in zip((a, b), beams, outs, streams, spaces):
            thk.thk_beam_select(bm, x, sc, None, o[0], o[1], o[2], None, w, stream=st)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(np.array_equal(y.cpu().numpy(), z) for y, z in zip(o, w))


# ---- far offsets --------------------------------------------------------------------------
def test_rope_rows_past_4_gib():
    """Buffers of more than 2^32 bytes: rows at both ends of the last head of the last sequence."""
    cap, r = (1 << 23) + 5, Rope("bf16", False, 128)      # 2 x 2 x 2^23 rows of 256 bytes: 8 GiB
    rec = np.array([[1, 7, 0, -1], [1, 8, cap - 1, -1], [0, 9, 3, -1]])
    k, v = (torch.randn(1, 3, 2 * D, device="cuda").bfloat16() for _ in range(2))
    shape = thk.make_shape(1, 2, 2, 2, D, 1, 1, 1, 0, thk.THK_BF16)
    k_out = torch.empty(2, 2, cap, D, dtype=torch.bfloat16, device="cuda")
    v_out = torch.empty_like(k_out)
    thk.thk_rope_qkv(shape, r.rope, r.turns, None, 0, k, 2 * D, v, 2 * D, ints(rec), 3, None, 0, k_out, v_out, cap)
    torch.cuda.synchronize()
    want = r.exact(k.reshape(3, 2, D), rec[:, 1])
    tol = r.bound(k.reshape(3, 2, D), want)
    for t, (b, _, row, _) in enumerate(rec):
        assert torch.equal(v_out[b, :, row], v[0, t].reshape(2, D))
        assert (np.abs(f64(k_out[b, :, row]) - want[t]) <= tol[t]).all()


def test_reorder_and_copies_past_4_gib():
    cap = (1 << 23) + 3
    shape = thk.make_shape(1, 3, 1, 1, D, 64, 1, 1, 0, thk.THK_BF16)
    kt = torch.empty(1, 3, 1, cap, D, dtype=torch.bfloat16, device="cuda")      # 6 GiB
    vt = torch.empty_like(kt)
    rows = [0, 1 << 20, cap - 1]
    for x in (kt, vt):
        for b in range(3):
            x[0, b, 0, rows] = torch.randn(3, D, device="cuda").bfloat16()
    before = [x[0, :, 0, rows].clone() for x in (kt, vt)]
    thk.thk_beam_reorder(shape, None, 3, ints([[2, 0, 1]]), 3, kt, vt, ints([cap, cap, cap - 1]), cap, None, None, None, None)
    torch.cuda.synchronize()
    for x, was in zip((kt, vt), before):
        got = x[0, :, 0, rows]
        assert torch.equal(got[0, :2], was[2, :2]) and torch.equal(got[0, 2], was[0, 2])      # the parent's last row is not in use
        assert torch.equal(got[1], was[0]) and torch.equal(got[2], was[1])
    del kt, vt
    shape, pages = thk.make_shape(1, 1, 1, 1, D, 64, 1, 128, 0, thk.THK_F32), thk.make_pages(0, 65536, 1, 80)      # 80 pages of 64 MiB
    pool = torch.empty(thk.thk_paged_pool_bytes(shape, pages), dtype=torch.uint8, device="cuda").reshape(80, 1024, -1)
    pool[79] = torch.randint(0, 256, pool[79].shape, dtype=torch.uint8, device="cuda")
    pool[78] = 7
    thk.thk_paged_copy(shape, pages, ints([[79, 2, 1000, 0], [79, 78, 1, 0]]), 2, pool)
    torch.cuda.synchronize()
    assert torch.equal(pool[2, :1000], pool[79, :1000]) and torch.equal(pool[78, 0], pool[79, 0]) and (pool[78, 1:] == 7).all()


def test_beam_select_rows_past_4_gib():
    V, ld = 5000, (1 << 30) + 8
    x = torch.empty(3 * ld, dtype=torch.bfloat16, device="cuda")      # 6 GiB
    rng = np.random.default_rng(4)
    rows = logits(rng, 1, 3, V, "bf16")
    for w in range(3):
        x[w * ld:w * ld + V] = rows[0, w]
    s = -5 * rng.random((1, 3))
    want = gpu_select(rows, s, None, 6, 1)
    got = gpu_select(x.reshape(1, 3, ld), s, None, 6, 1, ld=(ld, V))
    assert all(np.array_equal(a, b) for a, b in zip(got, want))


def test_beam_select_largest_vocabulary():
    """2^24 tokens of one beam: a thousand pieces are joined."""
    V = 1 << 24
    x = torch.zeros(1, 1, V, device="cuda")
    at = torch.randperm(V, generator=torch.Generator().manual_seed(5))[:80]
    x[0, 0, at.cuda()] = torch.arange(80, device="cuda").float() / 8 + 1
    parent, token, score, ended = gpu_select(x, np.zeros((1, 1)), None, 64, 0)
    assert token[0].tolist() == at.flip(0)[:64].tolist() and not parent.any() and not ended[token != 0].any()
    e = np.arange(80)[::-1] / 8 + 1
    want = e[:64] - math.log(np.exp(e).sum() + V - 80)
    assert np.abs(score[0] - want).max() <= sum_error(V) + 2.0 ** -24 * 20
