"""Paged caches, what needs no GPU: sizes, refusals of arguments in the library and in the binding, and the oracle's own
properties."""
import numpy as np
import pytest
import torch

import paper_2407_21018_amd as thk
from oracle import paged as P

A = 4096      # an aligned fake device address (never dereferenced on these paths)
BIG = 1 << 40


def _shape(**kw):
    d = dict(L=1, B=2, N_q=8, N_kv=2, D=128, S=1000, S_obs=32, T=64, ld_keep=0, dtype=thk.THK_BF16, n_split=0)
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


def _write(s, p, **kw):
    d = dict(k=A, v=A, src_rows=1000, n_rows=A, row0=None, idx=A, table=A, pool=A)
    d.update(kw)
    return _status(thk.thk_paged_write, s, p, *d.values(), stream=0)


def _read(s, p, **kw):
    d = dict(pool=A, table=A, row0=None, n_rows=A, k_out=A, v_out=A, out_rows=1000)
    d.update(kw)
    return _status(thk.thk_paged_read, s, p, *d.values(), stream=0)


def _append(s, **kw):
    d = dict(k_new=A, v_new=A, src_rows=1, src_row0=None, n_new=None, k_tail=A, v_tail=A, s_tail=A, s_tail_cap=64)
    d.update(kw)
    return _status(thk.thk_tail_append_ragged, s, *d.values(), stream=0)


def _decode(s, p, **kw):
    d = dict(q=A, pool=A, table=A, s_pages=A, idx=A, k_tail=A, v_tail=A, s_tail=A, s_tail_cap=64, out=A, ws=(A, BIG))
    d.update(kw)
    return _status(thk.thk_decode_attn_paged, s, p, *d.values(), stream=0)


@pytest.mark.parametrize("kw,want", [
    (dict(bits=2), 3), (dict(bits=16), 3), (dict(bits=-4), 3), (dict(page_rows=32), 2), (dict(page_rows=96), 2),
    (dict(page_rows=0), 2), (dict(page_rows=-64), 2), (dict(page_rows=131072), 2), (dict(max_pages=0), 2),
    (dict(max_pages=1 << 24), 2), (dict(n_pages=0), 2), (dict(n_pages=1 << 31), 2), (dict(n_pages=-1), 2)])
def test_bad_pages_are_refused(kw, want):
    s, p = _shape(), _pages(**kw)
    assert thk.thk_paged_pool_bytes(s, p) == 0
    assert (_write(s, p), _read(s, p), _decode(s, p)) == (want,) * 3


@pytest.mark.parametrize("kw,want", [
    (dict(N_q=7), 2), (dict(T=0), 2), (dict(T=129), 2), (dict(S=0), 2), (dict(S=1 << 31), 2), (dict(D=64, T=32), 3),
    (dict(dtype=7), 3), (dict(ld_keep=63), 2), (dict(n_split=-1), 2), (dict(n_split=5000), 2)])
def test_bad_shapes_are_refused(kw, want):
    s, p = _shape(**kw), _pages()
    assert thk.thk_paged_pool_bytes(s, p) == 0
    assert thk.thk_workspace_bytes(s, thk.THK_OP_DECODE_PAGED) == 0 and thk.thk_default_split(s, thk.THK_OP_DECODE_PAGED) == 0 or "n_split" in kw
    assert (_write(s, p), _read(s, p), _decode(s, p)) == (want,) * 3
    if kw.get("S") != 1 << 31:
        assert _append(s) == want


def test_null_alignment_sizes_and_workspace():
    s, p = _shape(), _pages()
    for name in ("k", "v", "n_rows", "idx", "table", "pool"):
        assert _write(s, p, **{name: None}) == 1, name
    for name, off in (("k", 8), ("v", 8), ("idx", 2), ("pool", 4), ("n_rows", 2), ("row0", 1), ("table", 2)):
        assert _write(s, p, **{name: A + off}) == 4, name
    for rows in (0, -1, 1 << 31):
        assert _write(s, p, src_rows=rows) == 2 and _read(s, p, out_rows=rows) == 2
    for name in ("pool", "table", "n_rows"):
        assert _read(s, p, **{name: None}) == 1, name
    assert _read(s, p, k_out=None, v_out=None) == 1
    for name, off in (("pool", 8), ("k_out", 8), ("v_out", 2), ("n_rows", 1), ("row0", 2), ("table", 3)):
        assert _read(s, p, **{name: A + off}) == 4, name
    for name in ("k_new", "v_new", "k_tail", "v_tail", "s_tail"):
        assert _append(s, **{name: None}) == 1, name
    for name, off in (("k_new", 8), ("v_tail", 8), ("s_tail", 2), ("src_row0", 2), ("n_new", 1)):
        assert _append(s, **{name: A + off}) == 4, name
    assert _append(s, src_rows=0) == 2 and _append(s, s_tail_cap=0) == 2
    for name in ("q", "pool", "table", "s_pages", "idx", "out", "k_tail", "v_tail", "s_tail"):
        assert _decode(s, p, **{name: None}) == 1, name
    for name, off in (("q", 8), ("pool", 8), ("idx", 2), ("out", 4), ("k_tail", 8), ("v_tail", 8), ("s_tail", 2), ("s_pages", 1), ("table", 2)):
        assert _decode(s, p, **{name: A + off}) == 4, name
    assert _decode(s, p, s_tail_cap=-1) == 2
    s.n_split = 3
    assert _decode(s, p, ws=None) == 5 and _decode(s, p, ws=(A + 8, BIG)) == 5
    assert _decode(s, p, ws=(A, thk.thk_workspace_bytes(s, thk.THK_OP_DECODE_PAGED) - 1)) == 5


def test_launches_too_large_for_one_grid_are_refused():
    p = _pages(page_rows=65536, max_pages=32767, n_pages=1)
    s = _shape(B=64, N_q=64, N_kv=64, S=(1 << 31) - 1)
    assert _write(s, p, src_rows=(1 << 31) - 1) == 2 and _read(s, p, out_rows=(1 << 31) - 1) == 2
    assert _append(_shape(B=1 << 14, N_q=1 << 13, N_kv=1 << 13)) == 2
    s.n_split = 4096
    assert _decode(s, p) == 2


@pytest.mark.parametrize("kw", [dict(L=1 << 30, B=1 << 30, N_kv=16, N_q=16), dict(L=1 << 30, B=1 << 30, N_kv=1 << 4, N_q=1 << 8),
                                dict(L=(1 << 31) - 1, B=(1 << 31) - 1, N_kv=(1 << 31) - 1, N_q=(1 << 31) - 1), dict(L=1 << 16, B=1 << 16)])
def test_units_past_the_number_range_are_refused(kw):
    """L * B * N_kv past 64 bits must not pass for a small number, nor for none."""
    s, p = _shape(**kw), _pages()
    assert _write(s, p) == 2 and _read(s, p) == 2 and _append(s) == 2 and _decode(s, p) == 2
    assert thk.thk_paged_pool_bytes(s, p) == 0
    assert thk.thk_workspace_bytes(s, thk.THK_OP_DECODE_PAGED) == 0 and thk.thk_default_split(s, thk.THK_OP_DECODE_PAGED) == 0


def test_pools_past_the_number_range_are_refused():
    s = _shape(L=64, N_q=64, N_kv=64)
    for n_pages, want in (((1 << 31) - 1, 2), (1 << 30, 2), (1 << 20, 0)):
        p = _pages(page_rows=65536, max_pages=1, n_pages=n_pages)
        assert (thk.thk_paged_pool_bytes(s, p) == 0) == (want == 2)
        if want:
            assert _write(s, p) == 2 and _read(s, p) == 2 and _decode(s, p) == 2


def test_sizes():
    for dtype, e in ((thk.THK_BF16, 2), (thk.THK_F32, 4)):
        for T in (1, 8, 51, 64, 76, 128):
            ch = -(-T // 8)
            for bits in (0, 4, 8):
                unit = bits or 8 * e
                tile = (ch + 16) * 64 * unit + ((ch * 8 + 128) * 2 * e if bits else 0)
                s, p = _shape(L=3, T=T, dtype=dtype), _pages(bits=bits, page_rows=256, n_pages=7)
                assert thk.thk_paged_pool_bytes(s, p) == 3 * 7 * 2 * 4 * tile
                assert tile % 16 == 0
    assert thk.thk_paged_pool_bytes(_shape(L=64, N_q=64, N_kv=64), _pages(n_pages=1 << 24)) > 1 << 45   # no 32-bit arithmetic


@pytest.mark.parametrize("S", [1, 63, 64, 65, 255, 256, 257, 4095, 4096, 131072, 10_000_000])
@pytest.mark.parametrize("units", [(1, 1, 1), (1, 8, 4), (64, 8, 8), (1, 8, 40), (4, 3, 17)])
def test_the_workspace_holds_every_piece(S, units):
    B, N_kv, G = units
    for n in (0, 1, 2, 7, 64, 4096):
        s = _shape(B=B, N_q=N_kv * G, N_kv=N_kv, S=S, S_obs=1, n_split=n)
        tiles = -(-S // 64)
        pieces = thk.thk_default_split(s, thk.THK_OP_DECODE_PAGED)
        assert 1 <= pieces <= tiles
        ws = thk.thk_workspace_bytes(s, thk.THK_OP_DECODE_PAGED)
        if n == 0:
            assert ws >= (pieces > 1) * B * N_kv * G * pieces * 130 * 4
        elif n > 1 and tiles > 1:
            per = -(-tiles // n)
            assert ws >= B * N_kv * G * -(-tiles // per) * 130 * 4 or tiles <= per


def test_tensors_are_checked_before_the_library_sees_them():
    s, p = _shape(), _pages()
    t = torch.zeros(4 * 1000 * 128, dtype=torch.bfloat16)   # on the host
    with pytest.raises(ValueError, match="k must be on the current GPU"):
        thk.thk_paged_write(s, p, t, A, 1000, A, None, A, A, A, stream=0)
    with pytest.raises(ValueError, match="s_pages must be on the current GPU"):
        thk.thk_decode_attn_paged(s, p, A, A, A, torch.zeros(2, dtype=torch.int32), A, A, A, A, 64, A, (A, BIG), stream=0)
    with pytest.raises(ValueError, match="v_tail must be on the current GPU"):
        thk.thk_tail_append_ragged(s, A, A, 1, None, None, A, t, A, 64, stream=0)
    with pytest.raises(ValueError, match="pool must be on the current GPU"):
        thk.thk_paged_read(s, p, torch.zeros(16, dtype=torch.uint8), A, None, A, A, A, 1000, stream=0)


@pytest.mark.parametrize("ws", [torch.empty(1 << 20, dtype=torch.uint8), (torch.empty(1 << 20, dtype=torch.uint8), 1 << 20), torch.empty(4).expand(1 << 18, 4)])
def test_a_workspace_on_the_host_is_refused(ws):
    """... and so is one whose elements are fewer than they look."""
    s, p = _shape(n_split=3), _pages()
    with pytest.raises(ValueError, match="ws must be"):
        thk.thk_decode_attn_paged(s, p, A, A, A, A, A, A, A, A, 64, A, ws, stream=0)


# ---- the oracle ------------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_oracle_s_codes_are_near_their_elements(bits, dtype):
    """|x - (m + c s)| <= s / 2 and what rounding s moves: s is off by half a step of its type at most, times the last code."""
    rng = np.random.default_rng(5)
    x = P.round_to(rng.standard_normal((200, 64)) * np.exp(2 * rng.standard_normal((200, 1))) + 3 * rng.standard_normal((200, 1)), dtype)
    c, s, m = P.codes(x, bits, dtype)
    assert c.min() == 0 and c.max() <= 2 ** bits - 1 and np.array_equal(m[:, 0], x.min(1))
    slack = (2 ** bits - 1) * s * {"f32": 2.0 ** -23, "bf16": 2.0 ** -8}[dtype]   # of s, and of the quotient in front of its rounding
    assert np.all(np.abs(x - (m + c * s)) <= s / 2 + slack)


def test_the_oracle_s_groups_at_their_edges():
    c, s, m = P.codes(np.full((1, 64), -2.5), 4, "bf16")          # no range
    assert not c.any() and s[0, 0] == 0 and m[0, 0] == -2.5
    c, s, m = P.codes(np.array([[0.0, 15.0, 0.5, 1.5, 2.5]]), 4, "f32")   # ties go to even
    assert s[0, 0] == 1 and c.tolist() == [[0, 15, 0, 2, 2]]
    tiny = 2.0 ** -133                                                # the smallest bf16 number: the scale rounds to zero
    c, s, m = P.codes(np.array([[0.0, tiny]]), 4, "bf16")
    assert s[0, 0] == 0 and not c.any()


def test_the_oracle_s_attention_is_the_formula():
    rng = np.random.default_rng(9)
    k, v, kt, vt, q = (rng.standard_normal(x) for x in ((5, 3), (5, 128), (2, 128), (2, 128), (4, 128)))
    idx = np.array([3, 50, 127])
    out = P.attend(q, idx, k, v, kt, vt)
    for n in range(4):
        z = np.concatenate([k @ q[n, idx], kt @ q[n]]) / np.sqrt(128)
        w = np.exp(z) / np.exp(z).sum()
        assert np.allclose(out[n], w @ np.concatenate([v, vt]), rtol=1e-12, atol=1e-12)
    assert not P.attend(q, idx, k[:0], v[:0], kt[:0], vt[:0]).any()
