"""A serving step around the paged cache, what needs no GPU: refusals of arguments, sizes, the speeds of rotary positions, and the
oracle's own properties."""
import math
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2407_21018_amd as thk
from oracle import step as O

A = 4096      # an aligned fake device address (never dereferenced on these paths)
BIG = 1 << 40


def _shape(**kw):
    d = dict(L=1, B=4, N_q=8, N_kv=2, D=128, S=1000, S_obs=32, T=64, ld_keep=0, dtype=thk.THK_BF16, n_split=0)
    d.update(kw)
    return thk.make_shape(**d)


def _pages(**kw):
    d = dict(bits=4, page_rows=128, max_pages=8, n_pages=20)
    d.update(kw)
    return thk.make_pages(**d)


def _status(fn, *a, **k):
    try:
        fn(*a, **k)
    except thk.ThkError as e:
        return e.status
    return 0


def _map(s, **kw):
    d = dict(n_new=A, pos0=A, row0=A, cap=64, q_rows=1, map=A, n_tokens=4, starts=A)
    d.update(kw)
    return _status(thk.thk_token_map, s, *d.values(), stream=0)


def _rope(s, r, **kw):
    d = dict(turns=A, q=A, ld_q=1024, k=A, ld_k=256, v=A, ld_v=256, map=A, n_tokens=4, q_out=A, q_rows=1, k_out=A, v_out=A, cap=64)
    d.update(kw)
    return _status(thk.thk_rope_qkv, s, r, *d.values(), stream=0)


def _reserve(s, p, **kw):
    d = dict(rows=A, now=A, held=A, table=A, refs=A, room=A, moves=A, ws=(A, BIG))
    d.update(kw)
    return _status(thk.thk_paged_reserve, s, p, *d.values(), stream=0)


def _copy(s, p, **kw):
    d = dict(moves=A, n_moves=4, pool=A)
    d.update(kw)
    return _status(thk.thk_paged_copy, s, p, *d.values(), stream=0)


def _select(b, **kw):
    d = dict(logits=A, scores=A, done=A, parent=A, token=A, score_out=A, done_out=A, ws=(A, BIG))
    d.update(kw)
    return _status(thk.thk_beam_select, b, *d.values(), stream=0)


def _reorder(s, p, **kw):
    d = dict(W=2, parent=A, ld_parent=4, k_tail=A, v_tail=A, s_tail=A, s_tail_cap=64, s_pages=A, held=A, table=A, refs=A)
    d.update(kw)
    return _status(thk.thk_beam_reorder, s, p, *d.values(), stream=0)


ROPE = thk.make_rope(thk.THK_ROPE_HALVES, 128)


@pytest.mark.parametrize("kw,want", [(dict(N_q=7), 2), (dict(T=0), 2), (dict(S=0), 2), (dict(D=64, T=32), 3), (dict(dtype=7), 3),
                                     (dict(B=0), 2), (dict(L=1 << 16, B=1 << 16), 2)])
def test_bad_shapes_are_refused(kw, want):
    s = _shape(**kw)
    assert (_map(s), _rope(s, ROPE), _reserve(s, _pages()), _copy(s, _pages()), _reorder(s, _pages())) == (want,) * 5
    assert thk.thk_workspace_bytes(s, thk.THK_OP_PAGED_RESERVE) == 0


@pytest.mark.parametrize("kw,want", [(dict(bits=2), 3), (dict(page_rows=96), 2), (dict(max_pages=0), 2), (dict(n_pages=0), 2)])
def test_bad_pages_are_refused(kw, want):
    s, p = _shape(), _pages(**kw)
    assert (_reserve(s, p), _copy(s, p), _reorder(s, p)) == (want,) * 3


def test_token_map_refusals():
    s = _shape()
    for name in ("pos0", "map"):
        assert _map(s, **{name: None}) == 1, name
    for name, off in (("n_new", 1), ("pos0", 2), ("row0", 1), ("map", 8), ("starts", 2)):
        assert _map(s, **{name: A + off}) == 4, name
    for kw in (dict(cap=-1), dict(q_rows=-1), dict(n_tokens=-1), dict(n_tokens=1 << 31)):
        assert _map(s, **kw) == 2, kw
    assert _map(_shape(B=4097, N_kv=1), starts=None) == 1


def test_rope_refusals():
    s = _shape()
    for kw, want in ((dict(layout=2), 3), (dict(layout=-1), 3), (dict(scaling=5), 3), (dict(scaling=-1), 3), (dict(rot=0), 2), (dict(rot=3), 2),
                     (dict(rot=130), 2), (dict(rot=-2), 2), (dict(base=1.0), 2), (dict(base=math.inf), 2), (dict(base=math.nan), 2),
                     (dict(gain=math.nan), 2), (dict(scaling=1, factor=0.0), 2), (dict(scaling=1, factor=-1.0), 2),
                     (dict(scaling=1, factor=math.inf), 2), (dict(scaling=2, rot=2), 2), (dict(scaling=3, low=1.0, high=32.0), 2),
                     (dict(scaling=3, trained=100, low=0.0, high=1.0), 2), (dict(scaling=4, trained=100, low=2.0, high=2.0), 2),
                     (dict(scaling=4, trained=100, low=2.0, high=math.inf), 2)):
        r = thk.make_rope(**{**dict(layout=0, rot=128), **kw})
        assert _rope(s, r) == want and _status(thk.thk_rope_turns, r) == want, kw
    for name in ("turns", "map", "q", "k", "v", "q_out", "k_out", "v_out"):
        assert _rope(s, ROPE, **{name: None}) == 1, name
    none = dict(q=None, k=None, v=None, q_out=None, k_out=None, v_out=None)
    assert _rope(s, ROPE, **none) == 1
    for name, off in (("turns", 4), ("map", 4), ("q", 8), ("k", 2), ("v", 8), ("q_out", 8), ("k_out", 4), ("v_out", 8)):
        assert _rope(s, ROPE, **{name: A + off}) == 4, name
    for kw, want in ((dict(ld_q=1023), 2), (dict(ld_k=255), 2), (dict(ld_v=0), 2), (dict(ld_q=1028), 4), (dict(ld_k=260), 4), (dict(ld_v=257), 4),
                     (dict(n_tokens=-1), 2), (dict(n_tokens=1 << 31), 2), (dict(cap=0), 2), (dict(cap=1 << 31), 2), (dict(q_rows=-1), 2),
                     (dict(n_tokens=(1 << 31) - 1), 2)):
        assert _rope(s, ROPE, **kw) == want, kw
    assert _rope(_shape(dtype=thk.THK_F32), ROPE, ld_q=1026) == 4


def test_rope_gains_that_32_bits_do_not_hold():
    for gain, want in ((1e39, 2), (-1e39, 2), (3e38, 0)):
        r = thk.make_rope(0, 128, gain=gain)
        assert _status(thk.thk_rope_turns, r) == want and _rope(_shape(), r, n_tokens=0) == want


def test_turns_of_a_whole_turn_less_a_little():
    """A factor that makes a speed as near to a whole turn as 64 bits tell: the table wraps or stays just below, never past its type."""
    for ulps in range(-3, 4):
        f = float(np.nextafter(1 / (2 * math.pi), 1)) * (1 + ulps * 2.0 ** -52)
        got = thk.thk_rope_turns(thk.make_rope(0, 4, thk.THK_ROPE_LINEAR, factor=f))[0] % 2 ** 64
        turn = Decimal(1) / Decimal(f) / (2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459")) * 2 ** 64
        assert abs((turn - got + 2 ** 63) % 2 ** 64 - 2 ** 63) <= 20


def test_no_tokens_and_no_moves_are_no_work():
    assert _rope(_shape(), ROPE, n_tokens=0, map=None) == 0
    assert _copy(_shape(), _pages(), n_moves=0, moves=None) == 0


def test_reserve_copy_and_reorder_refusals():
    s, p = _shape(), _pages()
    for name in ("rows", "held", "table", "refs", "room", "now", "moves"):
        assert _reserve(s, p, **{name: None}) == 1, name
    for name, off in (("rows", 2), ("held", 1), ("table", 2), ("refs", 2), ("room", 1), ("now", 2), ("moves", 8)):
        assert _reserve(s, p, **{name: A + off}) == 4, name
    n = thk.thk_workspace_bytes(s, thk.THK_OP_PAGED_RESERVE)
    assert n > 0 and _reserve(s, p, ws=None) == 5 and _reserve(s, p, ws=(A + 8, BIG)) == 5 and _reserve(s, p, ws=(A, n - 1)) == 5
    for name in ("moves", "pool"):
        assert _copy(s, p, **{name: None}) == 1, name
    assert _copy(s, p, moves=A + 4) == 4 and _copy(s, p, pool=A + 8) == 4 and _copy(s, p, n_moves=-1) == 2 and _copy(s, p, n_moves=1 << 30) == 2
    for name in ("parent", "k_tail", "v_tail", "s_tail", "s_pages", "held", "table", "refs"):
        assert _reorder(s, p, **{name: None}) == 1, name
    for name in ("held", "table", "refs"):      # without pages there are none of these
        assert _reorder(s, None, **{**dict(held=None, table=None, refs=None), name: A}) == 1, name
    for kw in (dict(W=0), dict(W=3), dict(W=33), dict(ld_parent=1), dict(s_tail_cap=-1)):
        assert _reorder(s, p, **kw) == 2, kw
    for name, off in (("parent", 2), ("k_tail", 8), ("v_tail", 4), ("s_tail", 1), ("s_pages", 2), ("held", 2), ("table", 1), ("refs", 2)):
        assert _reorder(s, p, **{name: A + off}) == 4, name
    assert _reorder(_shape(B=1 << 12, N_q=1 << 10, N_kv=1 << 10), p, s_tail_cap=1 << 20) == 2


def test_beam_select_refusals():
    def beams(**kw):
        return thk.make_beams(**{**dict(B=2, W=4, K=8, V=1000, eos=2), **kw})
    for kw, want in ((dict(B=0), 2), (dict(W=0), 2), (dict(W=33), 2), (dict(K=0), 2), (dict(K=65), 2), (dict(V=0), 2), (dict(V=(1 << 24) + 1), 2),
                     (dict(ld=999), 2), (dict(ld=-1), 2), (dict(eos=1000), 2), (dict(eos=-2), 2), (dict(dtype=2), 3), (dict(B=1 << 24), 2), (dict(B=1 << 23, W=1, V=8), 2)):
        b = beams(**kw)
        assert thk.thk_beam_workspace_bytes(b) == 0 and _select(b) == want, kw
    b = beams()
    for name in ("logits", "scores", "parent", "token", "score_out"):
        assert _select(b, **{name: None}) == 1, name
    for name, off in (("logits", 8), ("scores", 2), ("done", 1), ("parent", 2), ("token", 1), ("score_out", 2), ("done_out", 2)):
        assert _select(b, **{name: A + off}) == 4, name
    assert _select(beams(eos=-1)) == 2      # beams that have ended, and no token that ends them
    n = thk.thk_beam_workspace_bytes(b)
    assert n > 0 and _select(b, ws=None) == 5 and _select(b, ws=(A + 4, BIG)) == 5 and _select(b, ws=(A, n - 1)) == 5


def test_the_binding_refuses_tensors_on_the_host_and_short_ones():
    s, p = _shape(), _pages()
    i = torch.zeros(64, dtype=torch.int32)
    with pytest.raises(ValueError, match="n_new must be on the current GPU"):
        thk.thk_token_map(s, i, A, A, 64, 1, A, 4, stream=0)
    with pytest.raises(ValueError, match="q does not hold"):
        thk.thk_rope_qkv(s, ROPE, A, torch.zeros(4, 1023), 1024, A, 256, A, 256, A, 4, A, 1, A, A, 64, stream=0)
    with pytest.raises(ValueError, match="q does not hold"):
        thk.thk_rope_qkv(s, ROPE, A, torch.zeros(1024, 4).t(), 1024, A, 256, A, 256, A, 4, A, 1, A, A, 64, stream=0)
    with pytest.raises(ValueError, match="refs must be on"):
        thk.thk_paged_reserve(s, p, A, None, A, A, i, A, None, (A, BIG), stream=0)
    with pytest.raises(ValueError, match="moves must be on"):
        thk.thk_paged_copy(s, p, i, 4, A, stream=0)
    with pytest.raises(ValueError, match="logits must be on"):
        thk.thk_beam_select(thk.make_beams(1, 1, 1, 4), torch.zeros(4), A, None, A, A, A, None, (A, BIG), stream=0)
    with pytest.raises(ValueError, match="parent must be on"):
        thk.thk_beam_reorder(s, p, 2, i, 2, A, A, A, 64, A, A, A, A, stream=0)


# ---- speeds -------------------------------------------------------------------------------
SCALINGS = [("plain", {}), ("linear", dict(factor=8.0)), ("linear", dict(factor=0.3)), ("base", dict(factor=4.0)),
            ("ramp", dict(factor=16.0, trained=4096, low=1.0, high=32.0)), ("ramp", dict(factor=2.0, trained=1, low=1.0, high=2.0)),
            ("bands", dict(factor=8.0, trained=8192, low=1.0, high=4.0))]
NUMBER = {"plain": 0, "linear": 1, "base": 2, "ramp": 3, "bands": 4}


def test_numbers_of_the_scalings():
    assert [thk.THK_ROPE_PLAIN, thk.THK_ROPE_LINEAR, thk.THK_ROPE_BASE, thk.THK_ROPE_RAMP, thk.THK_ROPE_BANDS] == [0, 1, 2, 3, 4]


@pytest.mark.parametrize("rot", [4, 20, 44, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.5])
@pytest.mark.parametrize("scaling,kw", SCALINGS)
def test_speeds_are_rounded_once(scaling, kw, base, rot):
    """Against 60 digits: what the 64 bits of the host's arithmetic leave, a few 2^64ths of a turn.  A power with an exponent e ln(base)
    of up to 2^4.2 is off by 2^-63 + |e ln base| 2^-64 of itself or so: 20 units of 2^-64 for the fastest pair, w <= 1."""
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459")
    r = thk.make_rope(0, rot, NUMBER[scaling], base=base, **kw)
    f, b = Decimal(kw.get("factor", 1.0)), Decimal(base)
    if scaling == "base":
        b = b * (f.ln() * rot / (rot - 2)).exp()
    got = thk.thk_rope_turns(r)
    assert len(got) == rot // 2
    for i, g in enumerate(got):
        w = (b.ln() * -2 * i / rot).exp()
        if scaling == "linear":
            w /= f
        if scaling == "ramp":
            at = [rot * (kw["trained"] / (Decimal(t) * 2 * pi)).ln() / (2 * b.ln()) for t in (kw["high"], kw["low"])]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
            part = min(max((i - lo) / max(Decimal(hi - lo), Decimal("0.001")), Decimal(0)), Decimal(1))
            w = w / f * part + w * (1 - part)
        if scaling == "bands":
            part = min(max((kw["trained"] * w / (2 * pi) - Decimal(kw["low"])) / (Decimal(kw["high"]) - Decimal(kw["low"])), Decimal(0)), Decimal(1))
            w = w / f * (1 - part) + w * part
        turns = w / (2 * pi) * 2 ** 64
        assert abs((turns - g + 2 ** 63) % 2 ** 64 - 2 ** 63) <= 20 * max(1, w * kw.get("trained", 1)), (i, g)
    # ... and the oracle's, in 64-bit floats
    want, _ = O.speeds(rot, scaling, base, **kw)
    off = [abs(((g / 2.0 ** 64 - x / (2 * math.pi)) + 0.5) % 1 - 0.5) for g, x in zip(got, want)]
    assert max(off) < 1e-13


# ---- the oracle's own properties ----------------------------------------------------------
def test_oracle_rope_turns_by_angles():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 2, 128))
    w, gain = O.speeds(64, "plain", 10000.0)
    pos = [0, 1, 7, 1000, -3]
    for pairs in (False, True):
        y = O.rope(x, pos, w, gain, 64, pairs)
        assert np.array_equal(y[..., 64:], x[..., 64:]) and np.array_equal(y[0], x[0])
        z = (x[..., 0:64:2] + 1j * x[..., 1:64:2]) if pairs else (x[..., :32] + 1j * x[..., 32:64])
        z = z * np.exp(1j * np.asarray(pos)[:, None, None] * w)
        got = (y[..., 0:64:2] + 1j * y[..., 1:64:2]) if pairs else (y[..., :32] + 1j * y[..., 32:64])
        assert np.allclose(got, z, atol=1e-12)


def test_oracle_reserve_keeps_the_books():
    """Every held page is counted by its holders, free ones by none, whatever is asked for."""
    rng = np.random.default_rng(2)
    B, most, pr, n = 6, 5, 128, 17
    held, table, refs = [0] * B, [[-1] * most for _ in range(B)], [0] * n
    for _ in range(200):
        held, table, refs, room, _ = O.reserve(rng.integers(0, most * pr + 1, B).tolist(), None, held, table, refs, pr)
        users = [sum(row.count(p) for row in table) for p in range(n)]
        assert users == refs and all(h * pr == r for h, r in zip(held, room))
        assert all(-1 not in row[:h] and set(row[h:]) <= {-1} for row, h in zip(table, held))


def test_oracle_beam_is_a_full_sort():
    rng = np.random.default_rng(3)
    x, s = rng.standard_normal((2, 3, 50)), rng.standard_normal((2, 3))
    parent, token, score, done = O.beam_select(x, s, np.zeros((2, 3), int), 7, 4)
    for b in range(2):
        full = s[b][:, None] + x[b] - np.log(np.exp(x[b]).sum(1, keepdims=True))
        order = np.argsort(-full.ravel(), kind="stable")[:7]
        assert (parent[b] * 50 + token[b]).tolist() == order.tolist()
        assert np.allclose(score[b], full.ravel()[order]) and done[b].tolist() == [int(o % 50 == 4) for o in order]
