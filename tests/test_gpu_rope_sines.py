"""What a turn is made of: the gain of a scaling, and sines and cosines as near as their type holds them."""
import math

import numpy as np
import pytest
import torch

import paper_2407_21018_amd as thk
from oracle import step as O
from test_gpu_step import D, f64, gpu_rope, ints

pytestmark = pytest.mark.gpu


class Turn:
    """A description, its speeds on the device, and the type, as gpu_rope takes them."""

    def __init__(self, rot=D, pairs=False, **kw):
        self.rope = thk.make_rope(int(pairs), rot, **kw)
        self.turns = torch.tensor(thk.thk_rope_turns(self.rope), dtype=torch.int64, device="cuda")
        self.dtype, self.rot = "f32", rot


def turned_ones(r, pos):
    """(1, 0) of every pair of halves at positions pos: cosines and sines, times the gain."""
    n = len(pos)
    q = torch.zeros(1, n, D, device="cuda")
    q[..., :r.rot // 2] = 1
    rec = np.stack([np.zeros(n, np.int64), pos, np.full(n, -1), np.arange(n)], 1)
    got = f64(gpu_rope(r, 1, 1, 1, 1, q, None, None, ints(rec), n, 1)[0][0]).reshape(n, D)
    return got[:, :r.rot // 2], got[:, r.rot // 2:r.rot]


@pytest.mark.parametrize("factor,want", [(0.5, 1.0), (math.exp(-10), 1.0), (1e-3, 1.0), (1.0, 1.0), (1.5, 0.1 * math.log(1.5) + 1), (16.0, 0.1 * math.log(16) + 1)])
def test_the_ramp_has_a_gain_of_its_own_from_factor_1_on(factor, want):
    for given in (0.0, 0.75):
        r = Turn(scaling=thk.THK_ROPE_RAMP, trained=4096, factor=factor, low=1.0, high=32.0, gain=given)
        cos, sin = turned_ones(r, np.zeros(3, np.int64))
        assert (cos == np.float32(given or want)).all() and (sin == 0).all()
    assert O.speeds(D, "ramp", 10000.0, factor, 4096, 1.0, 32.0)[1] == want


@pytest.mark.parametrize("gain", [0.0, 1.75])
def test_sines_and_cosines_are_rounded_once(gain):
    """Half a step of the type below 1 is 2^-25; the angle is known to 2^-33 of a turn, 2^-30.3 radians, and the series to 2^-33: together less than
    2^-30.  Positions over the whole range of 32 bits, the test's angles from whole numbers."""
    pos = np.concatenate([np.arange(-200, 4000), [2 ** 31 - 1, -2 ** 31, 2 ** 30, -2 ** 30], np.random.default_rng(7).integers(-2 ** 31, 2 ** 31, 4000)]).astype(np.int64)
    r = Turn(base=500000.0, gain=gain)
    cos, sin = turned_ones(r, pos)
    at = np.array([[((int(p) * t) % 2 ** 64) / 2.0 ** 64 for t in r.turns.tolist()] for p in pos]) * 2 * math.pi
    g = gain or 1.0
    for got, want in ((cos, g * np.cos(at)), (sin, g * np.sin(at))):
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -20))) - 24)      # half a step at the value
        assert (np.abs(got - want) <= step * (1 + 2.0 ** -6) + g * 2.0 ** -30).all()
