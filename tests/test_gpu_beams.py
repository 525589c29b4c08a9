"""lessdec_beam_select on the GPU, through BeamSearch, against tests/beams_oracle.py: parents and tokens exactly, scores to half a step of
fp32 (2^-24 of the value) and what the sums allow: exponentials to 1e-14, at most 2^17 additions of 2^-53 one behind the other: 1e-11 covers both."""
import numpy as np
import pytest

from tests import beams_oracle as bo

pytestmark = pytest.mark.gpu


def types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def check(x, score, ended, groups, beams, picks, dtype, end_token=-1, own=None, in_place=False, stream=None):
    """x: a tensor on the GPU, rows may lie apart."""
    import torch
    from paper_2402_09398_amd import BeamSearch
    own = own or BeamSearch(groups, beams, x.shape[1], dtype, picks=picks, end_token=end_token)
    score = torch.tensor(score, dtype=torch.float32).cuda()
    flags = None if ended is None else torch.tensor(ended).cuda().to(torch.uint8 if groups % 2 else torch.bool)
    want = bo.select(x.double().cpu().numpy(), score.double().cpu().numpy(), ended, groups, beams, picks, end_token)
    n = groups * picks
    parent, token = (torch.full((n,), -7, dtype=torch.int32, device="cuda") for _ in range(2))
    best = score if in_place else torch.full((n,), 7.0, device="cuda")
    done = flags if in_place else torch.full((n,), 7, dtype=torch.uint8, device="cuda")
    own.select(x, score, flags, parent, token, best, done, stream=stream)
    torch.cuda.synchronize()
    got = [t.cpu().numpy().reshape(groups, picks) for t in (parent, token, best.double())]
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])
    there = want[0] >= 0
    assert (got[2][~there] == -np.inf).all()
    assert (np.abs(got[2][there] - want[2][there]) <= np.abs(want[2][there]) * 2.0 ** -24 + 1e-11).all()
    if done is not None:
        np.testing.assert_array_equal(done.cpu().numpy().reshape(groups, picks).astype(np.uint8), want[3].astype(np.uint8))
    return own


def logits(rows, vocab, dtype, seed=0, pad=0, scale=2.5, grid=None):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab + pad, generator=g, dtype=torch.float64) * scale
    if grid:
        x = (x / grid).round() * grid
    return x.to(types()[dtype]).cuda()[:, :vocab]


SHAPES = [(1, 1, 1, 1), (1, 1, 1, 64), (2, 3, 2, 5), (1, 64, 1, 64), (3, 2, 63, 4), (1, 5, 64, 5), (2, 4, 511, 8), (1, 4, 512, 4), (1, 3, 513, 3), (2, 2, 2048, 64),
          (1, 4, 2049, 1), (5, 7, 4097, 14), (1, 1, 100003, 64), (33, 1, 1000, 2), (700, 3, 77, 3), (1, 64, 3000, 64), (2, 17, 5000, 34)]


@pytest.mark.parametrize("groups,beams,vocab,picks", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_shapes(groups, beams, vocab, picks, dtype):
    """Odd sizes, rows at odd addresses, ties (logits on a grid; different rows differ in c by their scores)."""
    rng = np.random.default_rng(vocab)
    rows = groups * beams
    score = -20 * rng.random(rows)
    for pad, grid in ((0, None), (3, None), (1, 0.5)):
        check(logits(rows, vocab, dtype, picks, pad, grid=grid), score, None, groups, beams, picks, dtype)
    check(logits(rows, vocab, dtype, picks + 1, 5), score, rng.random(rows) < 0.4, groups, beams, picks, dtype, end_token=vocab - 1)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_orders_that_fill_every_list(dtype):
    """Rising, falling, constant and blocked logits; equal rows, whose pairs tie in c; zeros of both signs."""
    import torch
    vocab, picks, t = 6000, 48, types()[dtype]
    up = torch.arange(vocab, dtype=torch.float64) / 16 - 100
    x = torch.stack([up, up.flip(0), torch.zeros(vocab, dtype=torch.float64), (up / 40).round(), up, torch.where(torch.arange(vocab) % 2 == 0, -0.0, 0.0)])
    score = [-1.0, -1.0, -2.0, -3.0, -1.0, -2.0]
    for first in (x, x.flip(1), x[[2, 2, 5, 5, 2, 5]], x[[0, 0, 0, 0, 4, 4]]):
        check(first.to(t).cuda(), score, None, 1, 6, picks, dtype)
        check(first.to(t).cuda(), [-1.0] * 6, None, 2, 3, 3, dtype)


def test_what_is_none():
    """-inf, NaN and +inf among logits and scores; fewer pairs than are wanted."""
    import torch
    inf, nan = float("inf"), float("nan")
    for dtype in ("f32", "f16", "bf16"):
        x = logits(8, 5001, dtype, 5)
        x = x.clone()
        x[0, 5:] = -inf
        x[1] = -inf
        x[2, 4999] = nan
        x[3, 17] = inf
        x[4, :4990] = -inf
        x[5, 2::3] = -inf
        check(x, [-1.0, 0, 0, 0, -2, -30, -inf, nan], None, 1, 8, 64, dtype)
        check(x, [-1.0, 0, 0, 0, -2, -30, -inf, nan], None, 4, 2, 20, dtype)
        check(x, [-1.0, -3, -inf, nan, -2, -30, -5, -inf], np.array([0, 1, 1, 1, 0, 1, 0, 0], bool), 2, 4, 9, dtype, end_token=4)
        check(x[1:4].clone(), [0.0, -1.0, -2.0], None, 1, 3, 3, dtype)                # none at all
    # what a mask of the type's lowest value leaves
    for dtype, t in types().items():
        x = logits(2, 3001, dtype, 6).clone()
        x[:, 10:] = torch.finfo(t).min
        check(x, [-1.0, -1.5], None, 1, 2, 12, dtype)


def test_logits_far_from_zero_and_far_apart():
    """What exponents are relative to moves along a row; sums of one large and many small."""
    import torch
    for scale, shift in ((1e30, 0), (1.0, 1e6), (300.0, 0), (1e3, -1e4)):
        x = (logits(4, 30000, "f32", 7).double() * scale + shift).float()
        x[0] = x[0].sort()[0]
        x[1] = x[1].sort(descending=True)[0]
        check(x, [-1.0, -1.25, -1.5, -1.75], None, 2, 2, 8, "f32")
    x = torch.full((3, 20000), -60000.0, dtype=torch.float16, device="cuda")
    x[0, 19999], x[1, 3], x[2, 10000:] = 60000.0, 60000.0, -59000.0
    check(x, [-1.0, -2.0, -3.0], None, 1, 3, 6, "f16")


def test_in_place_over_steps_and_one_workspace():
    """Beams that go on from one another, scores and flags in place, until most have ended; one handle, other logits every time."""
    import torch
    from paper_2402_09398_amd import BeamSearch
    groups, beams, vocab = 5, 4, 700
    own = BeamSearch(groups, beams, vocab, "bf16", end_token=3)
    score = torch.tensor([0.0, -np.inf, -np.inf, -np.inf] * groups).cuda()
    ended = torch.zeros(groups * beams, dtype=torch.bool, device="cuda")
    parent, token = (torch.empty(groups * beams, dtype=torch.int32, device="cuda") for _ in range(2))
    for step in range(12):
        x = logits(groups * beams, vocab, "bf16", 100 + step).clone()
        x[:, 3] += 6
        want = bo.select(x.double().cpu().numpy(), score.double().cpu().numpy(), ended.cpu().numpy(), groups, beams, beams, 3)
        own.select(x, score, ended, parent, token, score, ended)
        np.testing.assert_array_equal(parent.cpu().numpy().reshape(groups, beams), want[0])
        np.testing.assert_array_equal(token.cpu().numpy().reshape(groups, beams), want[1])
        np.testing.assert_array_equal(ended.cpu().numpy().reshape(groups, beams), want[3])
        np.testing.assert_allclose(score.double().cpu().numpy().reshape(groups, beams), want[2], rtol=2.0 ** -24, atol=1e-11)
    assert ended.all()


def test_captured_and_on_another_stream():
    import torch
    from paper_2402_09398_amd import BeamSearch
    groups, beams, vocab, picks = 3, 4, 9001, 8
    own = BeamSearch(groups, beams, vocab, "f16", picks=picks, end_token=1)
    x = logits(12, vocab, "f16", 1, pad=3)
    ended = np.arange(12) % 5 == 4
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    check(x, -np.arange(12) / 3, ended, groups, beams, picks, "f16", end_token=1, own=own, stream=side)
    score, flags = torch.zeros(12, device="cuda"), torch.tensor(ended).cuda()
    parent, token = (torch.empty(groups * picks, dtype=torch.int32, device="cuda") for _ in range(2))
    best, done = torch.empty(groups * picks, device="cuda"), torch.empty(groups * picks, dtype=torch.bool, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        own.select(x, score, flags, parent, token, best, done)
    for seed in range(5):
        x.copy_(logits(12, vocab, "f16", 50 + seed))
        score.copy_(torch.tensor(-np.random.default_rng(seed).random(12)))
        graph.replay()
        torch.cuda.synchronize()
        want = bo.select(x.double().cpu().numpy(), score.double().cpu().numpy(), ended, groups, beams, picks, 1)
        np.testing.assert_array_equal(parent.cpu().numpy().reshape(groups, picks), want[0])
        np.testing.assert_array_equal(token.cpu().numpy().reshape(groups, picks), want[1])
        check(x, -np.arange(12) / 7, None, groups, beams, picks, "f16", end_token=1, own=own)


def test_offsets_past_31_bits():
    import torch
    rows, stride = 41, 1 << 26
    x = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").view(rows, stride)[:, :3001]
    x.copy_(logits(rows, 3001, "bf16", 9))
    check(x, -np.arange(rows) / 9, None, 1, rows, 50, "bf16")


def test_the_same_row_has_the_same_sum_wherever_it_lies():
    """Rows of equal logits at addresses of every alignment: their pairs tie, and go to the lower beam."""
    import torch
    for dtype in ("f32", "f16", "bf16"):
        row = logits(1, 20011, dtype, 3)[0]
        x = torch.empty(16, 20011 + 4 + (1 if dtype == "f32" else 0), dtype=row.dtype, device="cuda")[:, :20011]
        x.copy_(row.expand(16, -1))
        check(x, [-2.0] * 16, None, 1, 16, 48, dtype)


def test_wrong_tensors_are_refused():
    import torch
    from paper_2402_09398_amd import BeamSearch, LessdecError
    own = BeamSearch(2, 2, 100, "f16", end_token=1)
    i32 = lambda n=4: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    f32 = lambda n=4: torch.zeros(n, device="cuda")  # noqa: E731
    x = torch.zeros(4, 100, dtype=torch.float16, device="cuda")
    good = [x, f32(), None, i32(), i32(), f32(), None]
    for at, bad in ((0, x.float()), (0, x[:3]), (0, x.t().contiguous().t()), (0, x[:, :1].expand(4, 100)), (0, x[:1].expand(4, 100)), (0, x.cpu()),
                    (1, f32(5)), (1, f32().half()), (2, f32()), (3, i32().long()), (3, i32(8)[::2]), (4, i32(3)), (5, i32()), (6, i32())):
        args = list(good)
        args[at] = bad
        with pytest.raises(LessdecError):
            own.select(*args)
    for more in (dict(dtype="f64"), dict(picks=65), dict(end_token=100), dict(beams=0)):
        with pytest.raises(LessdecError):
            BeamSearch(**{**dict(groups=2, beams=2, vocab=100, dtype="f16"), **more})
