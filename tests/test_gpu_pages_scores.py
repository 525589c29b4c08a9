"""Attention of the paged cache where scores are far from 0.  Keys and queries are whole numbers, so that every score is one too before the scale
and equal scores are equal in any arithmetic; what differs, differs by far more than fp32 can lose."""
import numpy as np
import pytest

from tests.test_gpu_pages import HALF_STEP, Pair

pytestmark = pytest.mark.gpu


def check(p, counts, q):
    """out and lse of rows whose scores are exact, but for the scale.

    Scores that are equal give equal weights but for their values' exponents, others are powers of two apart, or count for nothing.  So out is
    off by half a step of its type, the rounding of a weight to fp16 (2^-11), that of its exponent where fp32 holds score and value
    exponent in one (|S| <= 1024: 2^-14), 2^-13 for it and the exponential, fp32 sums over the tokens, and fp16's smallest steps; lse by a few
    roundings of its own size, one each of the scale, the score, the sum and the logarithm's base."""
    start = np.concatenate([[0], np.cumsum(counts)])
    hq = p.ref.heads * p.ref.group
    out = p.t.full(q.shape, 3.5, dtype=p.own.tdtype, device="cuda")
    lse = p.t.full(q.shape[:2], 3.5, device="cuda")
    p.own.attend(0, q.cuda(), out, p.ints(start), int(max(counts)), lse)
    out, lse, u = out.double().cpu().numpy(), lse.double().cpu().numpy(), 2.0 ** -24
    for s in range(p.ref.slots):
        x, there = p.ref.tokens(0, s)
        assert there.all()
        for i in range(counts[s]):
            pos = p.ref.length[s] - counts[s] + i
            j = np.arange(p.ref.length[s])
            seen = (j <= pos) & ((j > pos - p.ref.window) | (j < p.ref.sinks) if p.ref.window else True)
            for h in range(hq):
                r, row = start[s] + i, q[start[s] + i, h].double().cpu().numpy()
                k, v = x[0, h // p.ref.group, seen], x[1, h // p.ref.group, seen]
                whole = k @ row
                assert (whole == np.round(whole)).all() and np.abs(whole).max() < 2 ** 24 * np.abs(row).max()
                w = np.exp((whole - whole.max()) * p.ref.scale)
                total, n = w.sum(), seen.sum()
                w /= total
                want, spread = (w[:, None] * v).sum(0), (w[:, None] * np.abs(v)).sum(0)
                tol = HALF_STEP[p.dtype] * np.abs(want) + spread * (2.0 ** -11 + 2.0 ** -13 + (2 * n + 64) * u) + 448 * 2.0 ** -31 * np.abs(v).max()
                off = np.abs(out[r, h] - want) - tol
                assert np.isfinite(out[r, h]).all() and (off <= 0).all(), (s, i, h, out[r, h][:4], want[:4], off.max())
                want = whole.max() * p.ref.scale + np.log(total)
                assert abs(lse[r, h] - want) <= 8 * u * abs(want) + (n + 64) * u, (s, i, h, lse[r, h], want)


def make(lengths, keys, scale, dim=64, dtype="bf16", group=2, page=16, **more):
    """A cache whose keys are whole numbers, keys(slot, tokens) [tokens, dim], and whose values lie many powers of two apart."""
    p = Pair(len(lengths), sum(-(-n // page) for n in lengths) + 1, page, -(-max(lengths) // page), 1, dim, dtype, q_per_kv=group, scale=scale, **more)
    p.reserve(lengths)

    def spoil(k, v, start):
        for s, n in enumerate(lengths):
            k[start[s]:start[s + 1], 0] = p.t.tensor(keys(s, n)).to(k.dtype)
        for b in range(0, v.shape[0], 16):
            v[b:b + 16] *= 2.0 ** (b // 16 * 5 % 13 - 8)
    p.append(lengths, spoil=spoil)
    return p


ROWS = [[1, 1], [4, 8], [40, 70]]                             # of one matrix tile, and of a workgroup's
FAR = [1.0, 2.0 ** 13, 2.0 ** 26, 2.0 ** 28, 2.0 ** 33, 2.0 ** 40]


@pytest.mark.parametrize("scale", FAR)
@pytest.mark.parametrize("dim,dtype,lengths", [(64, "bf16", [150, 90]), (128, "f16", [97, 200]), (64, "f16", [3000, 70])])
def test_the_largest_score_takes_all(scale, dim, dtype, lengths):
    """One token of largest score, or several that share it, in blocks whose values differ by many powers of two.  Scores are multiples of 32 (times
    the scale), so that e^-32 is the most that another token weighs."""
    r = np.random.default_rng(dim)
    p = make(lengths, lambda s, n: r.integers(-2, 3, (n, dim)), scale, dim, dtype)
    for rows in ROWS:
        check(p, rows, p.t.tensor(r.integers(-3, 4, (sum(rows), 2, dim)) * 32).to(p.own.tdtype))


@pytest.mark.parametrize("scale", FAR)
@pytest.mark.parametrize("window", [0, 50])
def test_equal_scores_share_alike(scale, window):
    """All keys are the same: the mean of the values that a row sees, however large the score and whatever the blocks' exponents."""
    p = make([140, 100], lambda s, n: np.tile(np.arange(64) % 5 - 1, (n, 1)), scale, sinks=3, window=window)
    for rows in ROWS:
        q = p.t.tensor(p.rng.integers(-3, 4, (sum(rows), 2, 64))).to(p.own.tdtype)
        check(p, rows, q)
        check(p, rows, q * 2.0 ** 20)


def test_scores_that_rise_block_by_block():
    """From 2^21 to 2^26, each block's scores eight (in powers of two) above the last one's: M moves again and again, by just what it need not move for."""
    step = np.float32(8 / 1.4426950408889634)                  # 8, times log2 e and rounded
    assert np.float32(float(step) * 1.4426950408889634) == 8
    keys = lambda s, n: np.concatenate([np.full((n, 1), 4), (np.arange(n) // 16 % 8)[:, None], np.zeros((n, 62))], 1)  # noqa: E731
    p = make([120, 100], keys, float(step), window=0)
    for rows in ROWS:
        for far in (2 ** 16, 2 ** 18, 2 ** 19, 2 ** 20, 2 ** 21):
            q = p.t.zeros(sum(rows), 2, 64)
            q[:, 0, 0], q[:, 1, 0], q[..., 1] = far, -far, 1
            check(p, rows, q.to(p.own.tdtype))


def test_one_long_sequence_over_many_workgroups():
    """Shares whose maxima are far from 0 are joined: one row of 20000 tokens, and 24 columns of them."""
    for scale in (2.0 ** 26, 2.0 ** 40):
        r = np.random.default_rng(5)
        p = make([20000, 30], lambda s, n: r.integers(-2, 3, (n, 64)), scale)
        for rows in ([1, 1], [12, 0]):
            check(p, rows, p.t.tensor(r.integers(-3, 4, (sum(rows), 2, 64)) * 32).to(p.own.tdtype))
        p = make([20000, 30], lambda s, n: np.tile(np.arange(64) % 5 - 1, (n, 1)), scale)
        for rows in ([1, 1], [12, 0]):
            check(p, rows, p.t.tensor(r.integers(-3, 4, (sum(rows), 2, 64))).to(p.own.tdtype))
