"""Attention over long paged sequences in which every tile can be seen: a tile left out, or taken twice, moves some output by more than
the bound, which is shown on the host for every tile of every case.

Tile t has values near MARK in one channel, 37 t mod 128, and near zero in the others; so an output of n rows is some MARK * 64 / n for
each of the few tiles that share its channel.  Logits differ from tile to tile by up to 2 (one kept channel carries that), so that
pieces have maxima of their own, and by little inside a tile."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from helpers import TDT
from test_gpu_paged import HALF_STEP, Cache, _np

D, MARK = 128, 8.0

# (B, N_kv, G, T, rows, page_rows, tails, cap, n_split, host's bound)
CASES = {
    "by_lengths": (3, 4, 2, 64, [20000, 10, 0], 512, [0, 5, 0], 8, 2, 50000),
    "by_lengths_wide": (2, 3, 8, 97, [2000, 1999], 128, [64, 1], 64, 7, 120000),
    "by_bound": (1, 1, 8, 76, [5000], 64, None, 0, 100, 5000),
    "chosen_ragged": (4, 2, 5, 51, [3000, 64, 2000, 1], 128, [0, 3, 64, 0], 64, 0, 3000),
    "chosen_long": (1, 4, 1, 64, [20000], 256, None, 0, 0, 20000),
    "whole": (1, 2, 17, 128, [9000], 64, [40], 64, 1, 9000),
}
FORMATS = [("bf16", 4), ("bf16", 8), ("bf16", 0), ("f32", 4), ("f32", 8), ("f32", 0)]


def _inputs(name, dtype):
    """Per sequence keys and values [N_kv][rows][128] and tails, queries [N_kv][G][128], index lists, all of the element type."""
    B, N_kv, G, T, rows, _, tails, cap, _, _ = CASES[name]
    r = np.random.default_rng(sum(map(ord, name)))
    rnd = lambda x: P.round_to(x, dtype)   # noqa: E731
    seqs = []
    for b in range(B):
        n, t = rows[b], (tails or [0] * B)[b]
        idx = np.stack([np.sort(r.permutation(D)[:T]) for _ in range(N_kv)])
        k, v = 0.5 * r.standard_normal((N_kv, n, D)), 0.25 * r.standard_normal((N_kv, n, D))
        q = 0.02 * r.standard_normal((N_kv, G, D))
        tile = np.arange(n) // 64
        v[:, np.arange(n), 37 * tile % D] += MARK
        for h in range(N_kv):
            c = idx[h, T // 2]
            k[h, :, c] = 2.8 * np.sin(0.7 * tile + h) + 0.05 * r.standard_normal(n)
            q[h, :, c] = 4.0
        seqs.append(dict(k=rnd(k), v=rnd(v), q=rnd(q), idx=idx, kt=rnd(0.5 * r.standard_normal((N_kv, t, D))), vt=rnd(r.standard_normal((N_kv, t, D)))))
    return seqs


def _expected(seq, h, bits, dtype):
    """(outputs [G, 128], bounds, and per tile the sums of its weights and of its weighted values, and all of these): fp64.

    The bound: an output is rounded once.  A logit is off by c_z of the sizes of its products, which are at most |q| (|m| + 31 s) of the
    channel's group, or |q k|; that moves an output by at most twice as much of sum p |v|.  The values' products, of at most 5.2 R for the
    largest value R of the row, are off by c_z of it.  c_z: terms 2^-17 (bf16) and 2^-25 (fp32), sums of some 256 roundings of 2^-24, as
    random ones."""
    k, v = P.stored(seq["k"][h][:, seq["idx"][h]], seq["v"][h], bits, dtype)
    q, kt, vt = seq["q"][h], seq["kt"][h], seq["vt"][h]
    z = np.concatenate([q[:, seq["idx"][h]] @ k.T, q @ kt.T], axis=1) / np.sqrt(float(D))
    p = np.exp(z - z.max(1, keepdims=True))
    vals = np.concatenate([v, vt])
    total, sums = p.sum(1), p @ vals
    want = sums / total[:, None]
    c_z = {"bf16": 2.0 ** -16, "f32": 2.0 ** -20}[dtype]
    size = np.abs(q) @ np.abs(kt).max(0, initial=0)
    for a in range(0, len(k), 64):
        rows = seq["k"][h][a:a + 64][:, seq["idx"][h]]
        if bits:
            _, s, m = P.codes(rows.T, bits, dtype)
            rows = (np.abs(m) + 31 * s).T
        size = np.maximum(size, (np.abs(q[:, seq["idx"][h]]) @ np.abs(rows).T).max(1))
    spread = p @ np.abs(vals).max(1) / total
    tol = HALF_STEP[dtype] * np.abs(want) + (c_z * spread * (2 * size / np.sqrt(D) + 5.2))[:, None]
    cuts = range(0, len(k), 64)
    tiles = [(p[:, a:a + 64][:, :len(k) - a].sum(1), p[:, a:min(a + 64, len(k))] @ v[a:a + 64]) for a in cuts]
    return want, tol, tiles, total, sums


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("dtype,bits", FORMATS)
def test_a_tile_left_out_or_taken_twice_is_past_the_bound(dtype, bits, name):
    N_kv = CASES[name][1]
    for seq in _inputs(name, dtype):
        if seq["k"].shape[1] + seq["kt"].shape[1] == 0:
            continue
        for h in range(N_kv):
            want, tol, tiles, total, sums = _expected(seq, h, bits, dtype)
            assert np.allclose(want, P.attend(seq["q"][h], seq["idx"][h], *P.stored(seq["k"][h][:, seq["idx"][h]], seq["v"][h], bits, dtype),
                                              seq["kt"][h], seq["vt"][h]), rtol=1e-9, atol=1e-12)
            for weight, part in tiles:
                for times in (-1, 1):   # left out; taken twice
                    rest = total + times * weight
                    if np.all(rest > 1e-9 * total):   # (a tile that is all there is: without it there is no output; twice it is the same)
                        other = (sums + times * part) / rest[:, None]
                        assert len(tiles) == 1 or np.all((np.abs(other - want) > 2 * tol).any(1))


@pytest.mark.gpu
@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("dtype,bits", FORMATS)
def test_every_tile_is_in_the_result_once(dtype, bits, name):
    B, N_kv, G, T, rows, page_rows, tails, cap, n_split, bound = CASES[name]
    print("tiles", dtype, bits, name, flush=True)
    seqs = _inputs(name, dtype)
    c = Cache(dtype, bits, 1, B, N_kv, G, T, rows, page_rows, tails, cap, seed=len(name), n_split=n_split)
    put = lambda to, x: to.copy_(torch.from_numpy(x).to(TDT[dtype]))   # noqa: E731
    for b, seq in enumerate(seqs):
        put(c.k[0, b, :, :rows[b]], seq["k"])
        put(c.v[0, b, :, :rows[b]], seq["v"])
        put(c.q[0, b], seq["q"].reshape(N_kv * G, D))
        put(c.kt[0, b, :, :seq["kt"].shape[1]], seq["kt"])
        put(c.vt[0, b, :, :seq["vt"].shape[1]], seq["vt"])
        c.idx[0, b] = torch.from_numpy(seq["idx"].astype(np.int16))
    c.write()
    c.shape.S = bound
    out = c.decode()
    torch.cuda.synchronize()
    got = _np(out).reshape(B, N_kv, G, D)
    for b, seq in enumerate(seqs):
        for h in range(N_kv):
            if seq["k"].shape[1] + seq["kt"].shape[1] == 0:
                assert not got[b, h].any()
                continue
            want, tol, *_ = _expected(seq, h, bits, dtype)
            bad = np.abs(got[b, h] - want) > tol
            assert not bad.any(), (b, h, np.abs(got[b, h] - want).max(), tol.min())
    assert torch.equal(c.decode(), out)
