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
