"""The paged cache in calls that its description allows and that come up less often: rows that begin behind row 0, more rows than tokens, pages that
no one has written yet, tokens counted from a slot's end, values in lengths and starts that are out of range."""
import numpy as np
import pytest

from tests.test_gpu_pages import HALF_STEP, Pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [-128, -127, 127])
@pytest.mark.parametrize("rows", [1, 20, 70])
@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (128, "bf16")])
def test_a_pool_that_is_not_written_yet(exponent, rows, dim, dtype):
    """The first page belongs to a slot that has its room and no tokens yet, and holds whatever the memory held: what lies behind another slot's
    end, or on a page that is not there, is read from it and must not count."""
    p = Pair(3, 60, 16, 30, 2, dim, dtype, q_per_kv=2)
    p.own.exps.fill_(exponent)
    p.reserve([16, 71, 400])
    p.append([0, 71, 400])
    p.attend([0, rows, rows])
    p.own.table[2, 3] = p.ref.table[2, 3] = -1
    p.own.table[2, 20] = p.ref.table[2, 20] = -1
    p.attend([0, rows, rows])


def test_a_slot_whose_last_page_is_missing():
    """Room for a slot whose partly filled page its table does not name: no page in its place (it would show what an earlier sequence left there);
    its new tokens on that page are passed over, those behind it have theirs."""
    for counts in ([1, 1, 1], [40, 3, 30]):
        p = Pair(3, 20, 16, 8, 1, 64)
        n = [21, 40, 16]
        p.reserve(n)
        p.append(n)
        p.own.table[0, 1] = p.ref.table[0, 1] = -1
        p.own.table[1, 2] = p.ref.table[1, 2] = -1
        p.own.refs[:] = p.ints([1, 0, 1, 1, 0, 1] + [0] * 14)
        p.ref.refs[:] = [1, 0, 1, 1, 0, 1] + [0] * 14
        p.reserve(counts)
        p.append(counts)
        p.held()
        p.attend(counts)


@pytest.mark.parametrize("rows,length", [(1, 70), (4, 70), (70, 80), (12, 9000)])
def test_scores_of_minus_infinity_over_values_that_are_no_numbers(rows, length):
    """A row whose every score is -inf gives zeros whatever the values hold, NaN among them; a row with one other score sees them."""
    p = Pair(1, length // 16 + 2, 16, length // 16 + 2, 1, 64, "bf16", q_per_kv=2)

    def spoil(k, v, start):
        k[:, 0, 0] = 1 + k[:, 0, 0].abs()
        v[3, 0, 5], v[20, 0, 7], v[length - 1, 0, 9] = float("nan"), float("inf"), float("nan")
    p.reserve([length])
    p.append([length], spoil=spoil)
    q = p.t.tensor(p.rng.standard_normal((rows + 2, 2, 64))).to(p.own.tdtype)
    q[:, 0] = 0
    q[:, 0, 0] = -float("inf")
    p.attend([rows], queries=q)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 16, 2 ** 30, 0, 5])
@pytest.mark.parametrize("counts", [[3, 8, 2], [8, 0, 5], [40, 90, 3], [130, 33, 1]])
def test_more_rows_than_tokens(window, counts):
    """Rows whose position would be below 0 are not stored and see nothing; the others are as ever, with a window as large as the type allows, too."""
    for sinks in (0, 2, 2 ** 31 - 1):
        p = Pair(3, 12, 16, 4, 2, 64, "f16", q_per_kv=1 + len(set(counts)) % 2, window=window, sinks=sinks)
        p.reserve([1, 33, 2])
        p.append([1, 33, 2])
        p.append(counts)
        p.attend(counts)
        p.held()
        p.reserve([min(20, counts[0]), min(1, counts[1]), 0])
        p.append(counts)
        p.attend(counts)
        p.held()


@pytest.mark.parametrize("slots,first", [(3, 1), (3, 100), (3, 1000), (70, 777), (300, 40)])
def test_rows_that_begin_behind_the_first(slots, first):
    """start[0] > 0: rows before it belong to no slot and blocks before the new tokens are left as they are, byte for byte."""
    p = Pair(slots, 12 * slots, 16, 16, 1, 64, "bf16", q_per_kv=3)
    n = [120 + s % 50 for s in range(slots)]
    p.reserve(n)
    p.append(n)
    for counts in ([1 + s % 3 for s in range(slots)], [20 + s % 60 if slots < 100 else 3 + s % 20 for s in range(slots)]):
        p.reserve(counts)
        start = first + np.concatenate([[0], np.cumsum(counts)])
        block = p.own.table.view(slots, -1).long()
        begin = p.own.length.long() - p.ints(counts).long()
        behind = p.t.arange(16, device="cuda") < (begin // 16)[:, None]          # pages of a block each that hold older tokens alone
        older = block[behind & (block >= 0)]
        saved = p.own.exps.clone()
        p.own.exps[:, older] = 77                             # (which no append has written)
        k, v = (p.t.tensor(p.rng.standard_normal((start[-1] + 2, 1, 64))).to(p.own.tdtype) for _ in range(2))
        codes = [x.clone() for x in (p.own.k_codes, p.own.v_codes)]
        p.own.append(0, k.cuda(), v.cuda(), p.ints(start))
        assert (p.own.exps[:, older] == 77).all()
        p.own.exps[:, older] = saved[:, older]
        for now, was in zip((p.own.k_codes, p.own.v_codes), codes):
            assert p.t.equal(now.view(p.ref.pages, -1)[older], was.view(p.ref.pages, -1)[older])
        p.ref.append(0, k.double().numpy(), v.double().numpy(), start)
        p.held()
        q = p.t.tensor(p.rng.standard_normal((start[-1] + 2, 3, 64))).to(p.own.tdtype)
        out = p.t.full(q.shape, 3.5, dtype=p.own.tdtype, device="cuda")
        p.own.attend(0, q.cuda(), out, p.ints(start), max(counts))
        want, _, tol, _ = p.ref.attend(0, q.double().numpy(), start, HALF_STEP["bf16"])
        got = out.double().cpu().numpy()
        assert (got[:first] == 3.5).all() and (got[start[-1]:] == 3.5).all()
        assert (np.abs(got - want) <= tol)[first:start[-1]].all()


@pytest.mark.parametrize("heads,dim,page,dtype", [(2, 64, 16, "f16"), (1, 128, 48, "bf16")])
def test_tokens_counted_from_a_slots_end(heads, dim, page, dtype):
    """read with negative `first` (before the slot's beginning, too), in the middle of a block, past the end; the same slot twice; slots that do not exist."""
    p = Pair(4, 40, page, 8, heads, dim, dtype)
    n = [50, 0, 17, 100]
    p.reserve(n)
    p.append(n, size=30.0)
    slots = [3, 0, -1, 2, 3, 4, 1, 2 ** 31 - 1, -2 ** 31]
    for first, count in ((-1, 1), (-17, 17), (-33, 20), (-100, 100), (-120, 70), (-2 ** 31, 5), (1, 15), (19, 40), (48, 3), (99, 33), (100, 2), (2 ** 31 - 1, 4)):
        K, V = (p.t.full((len(slots), heads, count, dim), 7.0, dtype=p.own.tdtype, device="cuda") for _ in range(2))
        p.own.read(0, p.ints(slots), first, K, V)
        want = p.ref.read(0, slots, first, count, float(p.t.finfo(p.own.tdtype).max))
        for got, w in zip((K, V), want):
            np.testing.assert_array_equal(got.double().cpu().numpy(), p.t.tensor(w).to(p.own.tdtype).double().numpy())


@pytest.mark.parametrize("slots,group", [(4, 1), (4, 5), (70, 5)])
def test_lengths_and_starts_out_of_range(slots, group):
    """Lengths and entries of start beyond their range count as the nearer end, to the bit; rows out of order touch nothing but the arrays."""
    low, high = -2 ** 31, 2 ** 31 - 1
    bad, near = [-5, high, 40, low] * (slots // 4 + 1), [0, 8 * 16, 40, 0] * (slots // 4 + 1)
    pairs = [Pair(slots, slots * 8, 16, 8, 2, 64, "f16", seed=3, q_per_kv=group) for _ in range(2)]
    rows = 400
    for p, length in zip(pairs, (bad, near)):
        fill = [100 if s % 4 == 1 else 40 if s % 4 == 2 else 20 for s in range(slots)]
        p.reserve(fill)
        p.append(fill)
        p.own.length.copy_(p.ints(length[:slots]))
    t, ints = pairs[0].t, pairs[0].ints
    k, v = (t.tensor(pairs[0].rng.standard_normal((rows, 2, 64))).half().cuda() for _ in range(2))
    q = t.tensor(pairs[0].rng.standard_normal((rows, 2 * group, 64))).half().cuda()
    tail = [390] * (slots - 3)
    starts = [([-7, 3, 90] + tail[:-1] + [rows, high], [0, 3, 90] + tail[:-1] + [rows, rows]), ([low, 0, 200] + tail + [high], [0, 0, 200] + tail + [rows])]
    for start, nearest in starts:
        assert len(start) == len(nearest) == slots + 1
        for most in (3, rows):
            got = []
            for p, at in zip(pairs, (start, nearest)):
                p.own.append(0, k, v, ints(at))
                out = t.full((rows + 64, 2 * group, 64), 3.5, dtype=t.float16, device="cuda")
                p.own.attend(0, q, out[32:-32], ints(at), most)
                assert (out[:32] == 3.5).all() and (out[-32:] == 3.5).all()
                K, V = (t.full((slots, 2, 33, 64), 7.0, dtype=t.float16, device="cuda") for _ in range(2))
                p.own.read(0, ints(range(slots)), -33, K, V)
                got.append([out, K, V] + [getattr(p.own, n) for n in ("k_codes", "v_codes", "exps", "table", "refs")])
            for a, b in zip(*got):
                assert t.equal(a.view(t.uint8) if a.is_floating_point() else a, b.view(t.uint8) if b.is_floating_point() else b)
    p = pairs[0]
    r = np.random.default_rng(slots)
    for _ in range(6):
        at = r.integers(-50, rows + 50, slots + 1)
        at[::5] = r.choice([low, high, 0, rows], len(at[::5]))
        p.own.length.copy_(ints(r.choice([low, high, -1, 0, 1, 40, 128, 129], slots)))
        for most in (1, 3, rows):
            out = t.full((rows + 64, 2 * group, 64), 3.5, dtype=t.float16, device="cuda")
            p.own.append(0, k, v, ints(at))
            p.own.attend(0, q, out[32:-32], ints(at), most)
            assert (out[:32] == 3.5).all() and (out[-32:] == 3.5).all()
    t.cuda.synchronize()


def test_plans_and_requests_out_of_range():
    """copy passes over pairs outside the pool and carries out no more than it is told; requests of the ends of the type; counts that are no counts."""
    low, high = -2 ** 31, 2 ** 31 - 1
    p = Pair(4, 24, 32, 5, 2, 64, "f16", layers=2)
    n = [100, 31, 0, 64]
    p.reserve(n)
    p.append(n)
    pairs = [(0, 20), (24, 21), (1, -1), (low, 22), (2, high), (high, low), (3, 23)]
    plan = p.ints([len(pairs)] + [x for pair in pairs for x in pair] + [7] * 32)
    before = [x.clone() for x in (p.own.k_codes, p.own.v_codes, p.own.exps)]
    for count, most in ((len(pairs), len(pairs)), (high, len(pairs)), (low, len(pairs)), (-1, 3), (len(pairs), 1)):
        plan[0] = count
        for x, was in zip((p.own.k_codes, p.own.v_codes, p.own.exps), before):
            x.copy_(was)
        p.own.copy(plan, most)
        moved = pairs[:max(0, min(count, most))]
        for x, was in zip((p.own.k_codes, p.own.v_codes, p.own.exps), before):
            now, want = x.view(2, 24, -1), was.view(2, 24, -1).clone()
            for a, b in moved:
                if 0 <= a < 24 and 0 <= b < 24:
                    want[:, b] = was.view(2, 24, -1)[:, a]
            assert p.t.equal(now, want), (count, most)
    p.reserve([high, low, 161, high - 31])
    p.reserve([1, 129, high, low])
    granted = p.ints([-9] * 4)
    r = np.random.default_rng(4)
    for _ in range(6):                                        # (nothing to compare: what is read stays in range, and the calls end)
        p.own.refs.copy_(p.ints(r.choice([low, -1, 0, 1, 2, high], 24)))
        p.own.table.copy_(p.ints(r.choice([low, -1, 0, 5, 23, 24, high], (4, 5))))
        p.own.length.copy_(p.ints(r.choice([low, 0, 7, 32, 150, 160, 161, high], 4)))
        p.own.reserve(p.ints(r.choice([low, 0, 1, 40, 160, high], 4)), granted, p.plan)
        p.own.select(p.ints(r.choice([low, -1, 0, 1, 3, 4, high], 4)))
        p.own.compact(p.plan)
        p.own.copy(p.plan, 12)
    p.t.cuda.synchronize()
