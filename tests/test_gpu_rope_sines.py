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
