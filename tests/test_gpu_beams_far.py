"""lessdec_beam_select on logits that lie far from 0 beside masked ones, whole tiles of them: -inf, the type's lowest value, -1e4.  Adding a number to all
logits of a row changes nothing, so the oracle of tests/beams_oracle.py gets every row less its largest logit (exact in fp64 for what decides), and the
scores are held to half a step of fp32 (2^-24 of the value) and to 1e-11 for the sums, as in tests/test_gpu_beams.py."""
import numpy as np
import pytest

from tests import beams_oracle as bo
from tests.test_gpu_beams import types

pytestmark = pytest.mark.gpu


def check(x, score, groups, beams, picks, dtype):
    import torch
    from paper_2402_09398_amd import BeamSearch
    rows, vocab = x.shape
    own = BeamSearch(groups, beams, vocab, dtype, picks=picks)
    score = torch.tensor(score, dtype=torch.float32).cuda()
    n = groups * picks
    parent, token = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    best = torch.full((n,), 7.0, device="cuda")
    own.select(x, score, None, parent, token, best)
    y = x.double().cpu().numpy()
    top = y.max(1, keepdims=True)
    want = bo.select(np.where(np.isfinite(top), y - np.where(np.isfinite(top), top, 0), y), score.double().cpu().numpy(), None, groups, beams, picks, -1)
    got = [t.cpu().numpy().reshape(groups, picks) for t in (parent, token, best.double())]
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])
    there = want[0] >= 0
    assert (got[2][~there] == -np.inf).all()
    assert (np.abs(got[2][there] - want[2][there]) <= np.abs(want[2][there]) * 2.0 ** -24 + 1e-11).all()


# A wave takes a tile of 512 logits in every four: tiles of -inf before, between and behind the others, in the same wave and in other waves and parts.
MASKS = {
    "first 512": lambda v, n: v < 512, "first 2048": lambda v, n: v < 2048, "first two of a wave": lambda v, n: v % 2048 // 512 == 1,
    "every other tile": lambda v, n: v // 512 % 2 == 0, "all but the last three": lambda v, n: v < n - 3, "all but two in the middle": lambda v, n: abs(2 * v - n) > 2,
    "all but the first three": lambda v, n: v > 2, "behind 2048": lambda v, n: v >= 2048, "two thirds": lambda v, n: v % 3 != 1,
}
# rows, beams, logits: a part a row, three tiles a wave; 35 parts of two tiles a wave; one tile a wave
SIZES = [(1300, 2, 6001), (8, 8, 140001), (6, 3, 8192)]
SHIFTS = {"f32": [0, -240, -251, -300, -340, -400, -1000, -1e4, 260, 340, 1e4], "f16": [0, -251, -340, -400, -1000, -1e4, 340, 1e4],
          "bf16": [0, -251, -340, -400, -1000, -1e4, 340, 1e4]}


def rows_of(rows, vocab, dtype, seed, mask, value):
    """Rows shifted one after the other by all of SHIFTS, masked with value; scores near enough for all of them to be chosen from."""
    import torch
    g = torch.Generator().manual_seed(seed)
    t, shifts = types()[dtype], SHIFTS[dtype]
    x = torch.randn(rows, vocab, generator=g) * 2.5 + torch.tensor([shifts[r % len(shifts)] for r in range(rows)], dtype=torch.float32)[:, None]
    x = x.to(t)
    where = torch.tensor(mask(np.arange(vocab), vocab))
    x[:, where] = value
    return x.cuda(), np.random.default_rng(seed).uniform(-8, 0, rows)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("rows,beams,vocab", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masked_with_infinity(dtype, rows, beams, vocab, mask):
    x, score = rows_of(rows, vocab, dtype, len(mask), MASKS[mask], -np.inf)
    check(x, score, rows // beams, beams, 2 * beams, dtype)


@pytest.mark.parametrize("mask", ["first 512", "first 2048", "every other tile", "all but the last three", "all but the first three"])
@pytest.mark.parametrize("rows,beams,vocab", SIZES[1:])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_masked_with_finite_values(dtype, rows, beams, vocab, mask):
    """The type's lowest value, and one that is below most rows and above others (whose unmasked logits then weigh nothing)."""
    import torch
    for value in (torch.finfo(types()[dtype]).min, -5e3):
        x, score = rows_of(rows, vocab, dtype, len(mask), MASKS[mask], value)
        check(x, score, rows // beams, beams, 2 * beams, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_rows_of_extremes(dtype):
    """Rows of nothing but the type's lowest or largest value (every token has the same share, the lowest tokens come first), rows that step down from
    it, and rows of one value in one tile; masked and not."""
    import torch
    t, vocab = types()[dtype], 6001
    low, high = torch.finfo(t).min, torch.finfo(t).max
    x = torch.full((8, vocab), low, dtype=t)
    x[1] = high
    x[2, 4000:] = high
    x[3, :700] = -np.inf
    x[4, ::2] = -np.inf
    x[5, 5999] = low / 2
    x[6] = -np.inf
    x[6, 1030:1050] = low
    x[7, 3000] = 0
    for picks in (1, 8, 64):
        check(x.cuda(), np.linspace(-3, 0, 8), 1, 8, picks, dtype)
        check(x.cuda(), np.linspace(0, -3, 8), 8, 1, picks, dtype)


def test_logits_that_change_scale_within_a_row():
    """Largest logits that come early, late and in steps up and down through the range that a sum's exponents are relative to."""
    import torch
    vocab = 40000
    for dtype in ("f32", "bf16", "f16"):
        rng = np.random.default_rng(3)
        x = rng.standard_normal((8, vocab)) * 2.5
        at = np.arange(vocab) // 2048
        x[0] += np.linspace(-3000, 200, 20)[at]
        x[1] += np.linspace(200, -3000, 20)[at]
        x[2] += np.linspace(-600, -260, 20)[at]
        x[3] += np.linspace(-260, -240, 20)[at]
        x[4] += np.where(at % 2 == 0, -249.0, -500.0)
        x[5] += np.linspace(240, 1200, 20)[at]
        x[6] += np.where(at < 19, -1e4, -300)
        x[7] += np.linspace(-20000, 20000, 20)[at]
        x[:, rng.random(vocab) < 0.3] = -np.inf
        check(torch.tensor(x).to(types()[dtype]).cuda(), np.zeros(8) - np.arange(8) / 8, 2, 4, 16, dtype)
