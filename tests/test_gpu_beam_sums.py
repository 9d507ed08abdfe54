"""Sums of beam selection where a lane's reference changes on the way over a row: several tiles a wave, at offsets of any size.  The softmax is
the same for logits that are all larger by the same amount, and so must the scores be."""
import math

import numpy as np
import pytest
import torch

from helpers import TDT
from oracle import step as O
from test_gpu_step import f64, gpu_select, sum_error

pytestmark = pytest.mark.gpu
TILE, TILES = 2048, 32          # of a row; a row is one block's, whose waves have eight tiles each
ROWS = 512                      # (as many as fill the card: with fewer a row is cut into pieces of fewer tiles)


def levels(dtype, offset):
    """(low, the largest value at most 8 above it, the next one at least 0.5 above that, one 8.25 above the last) in the type."""
    t = lambda x: float(torch.tensor(x, dtype=torch.float64).to(TDT[dtype]))  # noqa: E731
    low = t(offset)
    step = 2.0 ** (math.floor(math.log2(max(abs(low), abs(low + 24), 1.0))) - (7 if dtype == "bf16" else 23))
    low = t(math.floor(low / step) * step)
    below = t(low + math.floor(7.9 / step) * step if step <= 7.9 else low)
    above = t(low + math.ceil(8.01 / step) * step + math.ceil(0.45 / step) * step)
    last = t(above + math.ceil(8.25 / step) * step)
    assert below <= low + 8 < above and above + 8 < last
    return low, below, above, last


def rows_of(dtype, offset, rng):
    """Eight rows: the tiles of every wave in an order of their own."""
    low, below, above, last = levels(dtype, offset)
    orders = [[low] + [below] * 6 + [above], [low, above] + [below] * 6, [low] * 3 + [below] * 4 + [above], [low, below, above] + [low] * 4 + [last],
              [low, above, below, below, last, above, below, low]]
    orders += [rng.permutation([low, below, below, above, above, last, low, below]).tolist() for _ in range(3)]
    x = np.array([np.concatenate([rng.permutation(o) if i > 4 else o for _ in range(TILES // 8)]) for i, o in enumerate(orders)])
    x = np.repeat(x, TILE, axis=1)
    part = rng.random(x.shape) < 0.5      # in half of the places the lowest level or nothing
    x[part] = np.where(rng.random(int(part.sum())) < 0.5, low, -math.inf)
    return x


def check_offset(dtype, offset, bound):
    rng = np.random.default_rng(int(abs(offset)) + 1)
    x = torch.tensor(rows_of(dtype, offset, rng), dtype=torch.float64).to(TDT[dtype]).cuda()
    R, V = x.shape
    s = (-rng.random((R, 1)) * 3).astype(np.float32)
    parent, token, score, _ = O.beam_select(f64(x)[:, None], s.astype(np.float64), np.zeros((R, 1), int), 4, -1)
    which = np.arange(ROWS) % R
    got = gpu_select(x[torch.tensor(which).cuda()].reshape(ROWS, 1, V), s[which], None, 4, -1)
    assert np.array_equal(got[0], parent[which]) and np.array_equal(got[1], token[which])
    off = np.abs(got[2].astype(np.float64) - score[which])
    assert (off <= bound(V) + 2.0 ** -24 * np.abs(score[which])).all(), (offset, off.max(), bound(V))


OFFSETS = {"bf16": [0.0, 3.0, 60.0, 100.0, -100.0, 240.0, -1000.0, 5000.0, -70000.0, 1e6],
           "f32": [0.0, 3.0, 100.0, -100.0, 1e3, -1e3, 3e4, -3e4, 2.0 ** 20 - 40, 2.0 ** 20 - 4, -(2.0 ** 20) + 40, -(2.0 ** 20) - 4, 1e6, 3e7]}


@pytest.mark.parametrize("dtype,offset", [(d, o) for d in OFFSETS for o in OFFSETS[d]])
def test_the_reference_of_a_sum_changes(dtype, offset):
    print(f"beam sums {dtype} offset={offset}", flush=True)
    check_offset(dtype, offset, sum_error)


# A term's exponent is rounded once: 2^-24 (|x - r| + 0.35) of the term, r at most 2 below the lane's largest element; log2 e in 32 bits is off by 0.23
# 2^-24 of itself; 2^y is within 2^-23; three sums of 2^-24 lie before 64 bits.  Under the terms' own weights |x - r| is on average at most 2 and the
# logarithm of the 512 elements that a lane has at most.
SUM = (1.23 * (2 + math.log(512)) + 5.4) * 2.0 ** -24


@pytest.mark.parametrize("dtype,offset", [(d, o) for d in OFFSETS for o in OFFSETS[d]])
def test_a_sum_is_as_near_whatever_its_length_and_offset(dtype, offset):
    print(f"beam sums {dtype} offset={offset}", flush=True)
    check_offset(dtype, offset, lambda V: SUM)


def check_scores(x, s, K):
    """Every score within the bound; and the continuations themselves, for neighbours that are further apart than two of them can be off."""
    parent, token, score, _ = O.beam_select(f64(x), s.astype(np.float64), np.zeros(s.shape, int), K + 1, -1)
    near = (np.diff(score) != 0) & (np.abs(np.diff(score)) < 2 * SUM) & (parent[:, 1:] != parent[:, :-1])
    assert not near.any(), "two beams' continuations are too near for a test"
    got = gpu_select(x, s, None, K, -1)
    assert np.array_equal(got[0], parent[:, :K]) and np.array_equal(got[1], token[:, :K])
    assert (np.abs(got[2].astype(np.float64) - score[:, :K]) <= SUM + 2.0 ** -24 * np.abs(score[:, :K])).all()


def test_random_scores_of_many_rows():
    rng = np.random.default_rng(5)
    x = torch.tensor(rng.standard_normal((300, 8, 3001)) * 2, dtype=torch.float32).bfloat16().cuda()
    check_scores(x, (-10 * rng.random((300, 8))).astype(np.float32), 16)


@pytest.mark.parametrize("V", [262144, 1 << 20, (1 << 22) + 3])
def test_long_rows_whose_weight_lies_far_below_their_largest(V):
    """One large element a lane and tile, the others so far below that both halves of the sum count: the sum's size is that of the scores' places."""
    rng = np.random.default_rng(V)
    x = torch.full((1, 2, V), -5.25, device="cuda") + torch.tensor(rng.random((1, 2, V)) / 8, dtype=torch.float32).cuda()
    x[..., ::512] = 0.375
    x[0, 1, ::7] -= 40
    check_scores(x, np.array([[12.5, 12.0]], np.float32), 5)
