"""tkv_norm_rope at the ends of what its arguments may be: far positions, and more rows than a dimension of the grid takes."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2605_17170_amd import tkv

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
POS = [0, 1, -1, 7, -1000003, 2 ** 30, 2 ** 31 - 1, -2 ** 31]
TWO_PI = Fraction("6.283185307179586476925286766559005768394")


def turned(rope, pos, adjacent):
    """(1, 0) of every pair of a head: cosines and sines [tokens, pairs]."""
    n, half = len(pos), rope.rotary_dim // 2
    x = torch.zeros((n, 1, 128), dtype=torch.bfloat16, device=DEV)
    x[..., slice(0, 2 * half, 2) if adjacent else slice(0, half)] = 1.0
    out = torch.empty_like(x)
    axes = torch.tensor([pos] * rope.n_axes, dtype=torch.int32, device=DEV)
    tkv.tkv_norm_rope(rope, x, None, None, axes, None, None, 0.0, out, None)
    torch.cuda.synchronize()
    out = out[:, 0, :2 * half].double().cpu().numpy()
    return (out[:, 0::2], out[:, 1::2]) if adjacent else (out[:, :half], out[:, half:])


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("sections", [None, [16, 24, 24], [16, 16, 16, 16]])
def test_pairs_of_frequency_zero_do_not_turn(sections, adjacent):
    rope = tkv.tkv_rope_make(128, sections=sections, adjacent=adjacent, inv_freq=np.zeros(64), device=DEV)
    c, s = turned(rope, POS, adjacent)
    assert np.all(c == 1.0) and np.all(s == 0.0), np.abs(s).max()


@pytest.mark.parametrize("sections,interleaved", [(None, False), ([24, 20, 20], True), ([16, 16, 16, 16], False)])
def test_sines_of_angles_near_whole_turns(sections, interleaved):
    """Positions that bring a pair within 2^-20 of whole turns, where bf16 shows the angle to 2^-32 turns.  Tolerance: 2^-63 turns a
    position by the table, 2^-33 by its rounding to 32 bits, times 2 pi; 2^-21 of the sine (conversion and evaluation in 32 bits,
    a few half steps) and 2^-8 of it by the rounding to bf16."""
    rng = np.random.default_rng(5)
    pos, freq = [], []
    for k in range(64):                          # frequency p/q + a little turns a position, times q * m
        q = int(rng.integers(3, 60000))
        m = int(rng.integers(1, (2 ** 31 - 1) // q)) * int(rng.choice([-1, 1]))
        freq.append(float(Fraction(int(rng.integers(0, q)), q) * TWO_PI) + float(rng.choice([-1, 1])) * 2.0 ** -22 / abs(q * m) * float(rng.random()))
        pos.append(q * m)
    rope = tkv.tkv_rope_make(128, sections=sections, interleaved=interleaved, inv_freq=np.array(freq), device=DEV)
    _, s = turned(rope, pos, False)
    for k in range(64):
        turns = Fraction(freq[k]) / TWO_PI * pos[k]
        turns -= round(turns)
        assert abs(turns) < Fraction(1, 2 ** 20)
        want = math.sin(2 * math.pi * float(turns))
        tol = 2 * math.pi * (abs(pos[k]) * 2.0 ** -63 + 2.0 ** -33) + (2.0 ** -21 + 2.0 ** -8) * abs(want)
        # (the host's division and remainder in 64 bits: half a unit of 2^-64 a position besides)
        tol += 2 * math.pi * abs(pos[k]) * 2.0 ** -64
        assert abs(s[k, k] - want) <= tol, (k, pos[k], s[k, k], want, tol)


def test_more_rows_than_a_dimension_of_the_grid():
    """2^29 + 192 rows, in place; the first and last tokens and those around 2^28 and 2^29 rows, against calls of their own."""
    heads, tokens = 64, (1 << 23) + 3
    if torch.cuda.mem_get_info()[0] + torch.cuda.memory_reserved() - torch.cuda.memory_allocated() < tokens * heads * 256 + (8 << 30):
        pytest.skip("needs 146 GB of device memory")
    x = torch.empty((tokens, heads, 128), dtype=torch.bfloat16, device=DEV)
    x.fill_(0.5)
    at = [0, 1, (1 << 22) - 1, 1 << 22, (1 << 23) - 2, (1 << 23) - 1, 1 << 23, tokens - 1]
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    rows = torch.randn((len(at), heads, 128), device=DEV, generator=g).to(torch.bfloat16)
    for i, t in enumerate(at):
        x[t] = rows[i]
    weight = (1.0 + 0.3 * torch.randn((128,), device=DEV, generator=g)).to(torch.bfloat16)
    pos = torch.arange(tokens, dtype=torch.int32, device=DEV)[None]
    rope = tkv.tkv_rope_make(128, 1e6, device=DEV)
    want = torch.empty_like(rows)
    tkv.tkv_norm_rope(rope, rows, None, None, pos[:, at].contiguous(), weight, None, 1e-6, want, None)
    tkv.tkv_norm_rope(rope, x, None, None, pos, weight, None, 1e-6, x, None)
    torch.cuda.synchronize()
    for i, t in enumerate(at):
        assert torch.equal(x[t], want[i]), t
    # every token was normed: no row still holds what it did
    left = sum(int((x[t:t + (1 << 18)] == 0.5).all(-1).any(-1).sum()) for t in range(0, tokens, 1 << 18))
    del x
    torch.cuda.empty_cache()
    assert left == 0
