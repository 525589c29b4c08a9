"""Attention that reads what slots share once, on the GPU, through PagedCache, against tests/pages_oracle.py, within the bounds that lessdec_pages_attend
is held to; and the plan: every node's slots name its pages, and a slot's nodes and its own part are all that it sees."""
import numpy as np
import pytest

from tests import pages_oracle as po
from tests.test_gpu_pages import HALF_STEP, Pair

pytestmark = pytest.mark.gpu


class Shared(Pair):
    def __init__(self, *args, **more):
        super().__init__(*args, **more)
        from paper_2402_09398_amd import lessdec_pages_shared_workspace_bytes
        own = self.own
        own.shared = True
        need = lessdec_pages_shared_workspace_bytes(own.desc, own.max_rows)
        own.workspace = self.t.zeros(need, dtype=self.t.uint8, device="cuda")
        own.desc.workspace, own.desc.workspace_bytes = own.workspace.data_ptr(), need
        self.sharing = own.share_plan()

    def nodes(self):
        """Every slot's own part (-1: it shares nothing), and (row, rows, first block, last, node before, tiles, shares) of every node."""
        slots, plan = self.ref.slots, self.sharing.cpu().numpy()
        node = plan[8:8 + 36 * slots].reshape(-1, 12)[:plan[0]]
        chain = plan[8 + 36 * slots:][:16 * slots].reshape(-1, 4, 4)
        slot = [-1] * slots
        for i, f in enumerate(node):
            if f[6] == 1 << 30:
                slot[f[0]] = i
        for s in range(slots):                                # first columns, columns and shares of its nodes
            at = slot[s]
            if at < 0:
                assert chain[s, 0, 0] == -1
                continue
            row = node[at][1]
            for x in chain[s]:
                want = (node[at][10] + (row - node[at][1]) * self.ref.group, node[at][2] * self.ref.group, node[at][11]) if at >= 0 else (0, 0, 0)
                assert tuple(x[:3]) == want
                at = node[at][7] if at >= 0 else -1
        return slot, [tuple(int(x) for x in (f[1], f[2], f[5], f[6], f[7], f[9], f[11])) for f in node]

    def share(self, counts, behind=2, least=0):
        """The plan for these rows, looked over; the nodes of several slots."""
        r, start = self.ref, np.concatenate([[0], np.cumsum(counts)])
        self.sharing.fill_(-5)
        self.own.share(self.ints(start), int(start[-1]) + behind, self.sharing, least_bytes=least)
        slot, nodes = self.nodes()
        per, several = r.page // 16, [n for n in nodes if n[3] < 1 << 30]
        assert nodes[:len(several)] == several
        for row, rows, first, last, before, tiles, shares in several:
            there = [s for s in range(r.slots) if counts[s] and row <= start[s] and start[s + 1] <= row + rows]
            assert len(there) > 1 and sum(counts[s] for s in there) == rows and first % per == last % per == 0 and shares > 0
            assert all(slot[s] >= 0 for s in there) and (before == -1 if first == 0 else several[before][3] == first)
            for j in range(first // per, last // per):
                named = set()
                for s in there:
                    p = r.length[s] - counts[s]
                    seen = np.arange(j * r.page, (j + 1) * r.page)
                    if (((seen > p - r.window) | (seen < r.sinks)) if r.window else seen >= 0).any():
                        named.add(r.table[s, j])
                assert len(named) <= 1
        own = set()
        for s in range(r.slots):
            if counts[s] == 0 or slot[s] < 0:
                assert slot[s] == -1 and not 16 < counts[s] * r.group < 128
                continue
            row, rows, first, last, at, *_ = nodes[slot[s]]
            assert slot[s] >= len(several) and slot[s] not in own and (row, rows, last) == (start[s], counts[s], 1 << 30) and (at >= 0 or first == 0)
            own.add(slot[s])
            while at >= 0:
                assert nodes[at][3] == first
                row, rows, first, last, at, *_ = nodes[at]
                assert row <= start[s] and start[s + 1] <= row + rows
            assert first == 0
        assert len(own) == len(nodes) - len(several)
        return several

    def attend_shared(self, counts, layer=0, size=1.0, queries=None, lse=True, stride=0):
        start = np.concatenate([[0], np.cumsum(counts)])
        hq = self.ref.heads * self.ref.group
        q = self.t.tensor(self.rng.standard_normal((start[-1] + 2, hq, self.ref.dim)) * size).to(self.own.tdtype).cuda() if queries is None else queries
        if stride:
            q = self.t.cat([q, q], 1)[:, :hq]
        out = self.t.full(q.shape, 3.5, dtype=self.own.tdtype, device="cuda")
        stat = self.t.full(q.shape[:2], 3.5, device="cuda") if lse else None
        self.own.attend_shared(layer, q, out, self.ints(start), int(max(counts)), self.sharing, stat)
        want, want_lse, tol, lse_tol = self.ref.attend(layer, q.double().cpu().numpy(), start, HALF_STEP[self.dtype])
        got, n = out.double().cpu().numpy(), start[-1]
        assert (got[n:] == 3.5).all(), "rows behind the last slot"
        np.testing.assert_array_equal(np.isnan(got[:n]), np.isnan(want[:n]))
        fine = ~np.isnan(want[:n])
        off = np.abs(got[:n] - want[:n])[fine] - tol[:n][fine]
        assert off.size == 0 or off.max() <= 0, off.max()
        if lse:
            got = stat.double().cpu().numpy()
            assert (got[n:] == 3.5).all()
            np.testing.assert_array_equal(np.isneginf(got[:n]), np.isneginf(want_lse[:n]))
            fine = np.isfinite(want_lse[:n])
            assert (np.abs(got[:n] - want_lse[:n])[fine] <= lse_tol[:n][fine]).all()
        return out

    def room(self, n):
        got = self.reserve(n)
        assert list(got) == list(n)
        self.append(n)


def prompt(p, n, slots):
    """A prompt of n tokens in slot 0, that slots become copies of."""
    p.room([n] + [0] * (p.ref.slots - 1))
    p.select([0 if s in slots else -1 for s in range(p.ref.slots)])


SHAPES = [                                                    # slots, heads, group, dim, page, dtype, prompt, own tokens, rows a slot, sinks, window
    (4, 2, 1, 64, 16, "f16", 200, [5, 1, 17, 40], [1, 1, 1, 1], 0, 0),
    (4, 2, 4, 128, 16, "bf16", 130, [5, 1, 17, 40], [1, 1, 1, 1], 0, 0),
    (5, 3, 5, 128, 32, "f16", 333, [1, 1, 1, 1, 1], [1, 1, 1, 1, 1], 0, 0),
    (9, 1, 16, 64, 64, "bf16", 500, [3, 70, 9, 1, 1, 20, 33, 2, 8], [1] * 9, 0, 0),
    (6, 2, 3, 64, 16, "f16", 401, [30, 2, 4, 16, 50, 9], [7, 2, 4, 5, 30, 1], 0, 0),
    (3, 1, 71, 64, 32, "f16", 300, [4, 40, 1], [1, 1, 1], 0, 0),
    (40, 1, 8, 128, 16, "bf16", 90, [1 + i % 5 for i in range(40)], [1] * 40, 0, 0),
    (3, 2, 1, 128, 16, "f16", 150, [60, 200, 33], [60, 140, 33], 0, 0),
    (6, 1, 2, 64, 16, "f16", 500, [30, 2, 4, 16, 50, 9], [3, 2, 4, 1, 8, 1], 0, 100),
    (6, 2, 4, 128, 32, "bf16", 500, [30, 2, 4, 16, 50, 9], [1] * 6, 4, 200),
    (5, 1, 30, 64, 16, "f16", 420, [3, 60, 1, 9, 33], [1, 3, 1, 2, 4], 40, 64),
    (4, 1, 1, 128, 16, "f16", 300, [20, 1, 3, 8], [20, 1, 3, 8], 70, 1),
]


@pytest.mark.parametrize("slots,heads,group,dim,page,dtype,n,own,rows,sinks,window", SHAPES)
def test_one_prompt(slots, heads, group, dim, page, dtype, n, own, rows, sinks, window):
    pages = -(-n // page) + sum(2 + -(-x // page) for x in own) + 4
    p = Shared(slots, pages, page, -(-(n + max(own)) // page) + 1, heads, dim, dtype, seed=slots + n, q_per_kv=group, sinks=sinks, window=window)
    prompt(p, n, range(slots))
    p.room(own)
    nodes = p.share(rows)
    assert nodes or window or max(rows) * group >= 128, "nothing is shared"      # (a slot of that many columns stands between the others)
    p.attend_shared(rows)
    p.attend_shared(rows, size=4.0, lse=False, stride=1)
    order = [(3 * s + 1) % slots for s in range(slots)]
    p.select(order)                                           # beams that go on from others
    rows = [rows[s] for s in order]
    p.share(rows)
    p.attend_shared(rows, size=2.0)


def test_all_is_shared():
    """Forks that have no token of their own yet, a partly filled page among what they share; then one of them gets some."""
    for group, rows in ((1, 1), (4, 3), (33, 1)):
        p = Shared(6, 60, 16, 20, 2, 64, "f16", q_per_kv=group)
        prompt(p, 203, range(6))
        assert len(p.share([rows] * 6)) == 1
        p.attend_shared([rows] * 6)
        p.room([0, 0, 4, 0, 0, 1])
        p.share([rows, 1, 3, 0, 0, 1])
        p.attend_shared([rows, 1, 3, 0, 0, 1])


def test_nested_prompts_and_slots_that_share_nothing():
    """Instructions for all, prompts of their own behind them, samples of each; a slot without rows in between, one of another prompt, one with
    many columns, one that is empty."""
    p = Shared(14, 200, 16, 40, 2, 64, "bf16", q_per_kv=2)
    p.room([150] + [0] * 13)
    p.select([0] * 12 + [-1, -1])
    p.room([100, 0, 0, 0, 64, 0, 0, 0, 33, 0, 0, 0, 90, 0])
    p.select([0, 0, 0, 0, 4, 4, 4, 4, 8, 8, 8, 8, 12, -1])
    p.room([3, 1, 20, 5, 1, 70, 2, 2, 1, 1, 1, 1, 2, 0])
    for rows in ([1] * 13 + [0], [1, 1, 0, 2, 1, 70, 1, 2, 1, 1, 1, 1, 2, 0], [0, 1, 0, 0, 0, 1, 0, 0, 0, 0, 0, 1, 0, 0], [3, 1, 9, 4, 1, 5, 2, 2, 1, 1, 1, 1, 2, 0]):
        nodes = p.share(rows)
        assert len(nodes) >= 1
        p.attend_shared(rows)
    assert any(node[4] >= 0 for node in p.share([1] * 13 + [0])), "no node within another"


def test_sharing_that_deepens_slot_by_slot():
    """Every slot goes on from the one before it: nodes within nodes, more than are kept."""
    p = Shared(8, 200, 16, 40, 1, 64, "f16")
    p.room([300] + [0] * 7)
    for s in range(1, 8):
        p.select([i if i < s else s - 1 if i == s else -1 for i in range(8)])
        p.room([0] * s + [48] + [0] * (7 - s))
    nodes = p.share([1] * 8)
    assert len(nodes) > 1
    p.attend_shared([1] * 8)
    p.select([7, 6, 5, 4, 3, 2, 1, 0])
    p.share([1] * 8)
    p.attend_shared([1] * 8)


def test_what_pays():
    """Nothing is shared if that saves too little: slots of few columns are attended to as they are, others as nodes without one around them."""
    for group in (2, 5, 40):
        p = Shared(5, 60, 16, 20, 2, 64, "f16", q_per_kv=group)
        prompt(p, 160, range(5))
        p.room([1, 20, 3, 40, 5])
        saved = 160 * 4 * 2 * 2 * 64
        for rows in ([1] * 5, [1, 3, 0, 9, 2]):
            for least in (-1, saved + 1):
                assert not p.share(rows, least=least)
                p.attend_shared(rows)
        assert p.share([1] * 5, least=saved)
        p.attend_shared([1] * 5)


def test_many_slots():
    for slots, group in ((70, 1), (300, 2), (1100, 1)):
        p = Shared(slots, slots * 2 + 60, 16, 14, 1, 64, "f16", q_per_kv=group)
        prompt(p, 100, range(slots))
        p.room([1 + s % 3 for s in range(slots)])
        assert len(p.share([1] * slots)) == 1
        p.attend_shared([1] * slots)
        p.select([s // 5 * 5 for s in range(slots)])
        p.room([s % 2 for s in range(slots)])
        rows = [s % 7 != 3 for s in range(slots)]
        p.share(rows)
        p.attend_shared(rows)


def test_a_long_prefix_over_many_workgroups():
    p = Shared(5, 1500, 16, 1400, 2, 64, "bf16", q_per_kv=3)
    prompt(p, 20000, range(5))
    p.room([1, 30, 7, 2, 500])
    for rows in ([1] * 5, [1, 9, 7, 2, 30]):
        nodes = p.share(rows)
        assert nodes[0][5] > 300 or rows == [1] * 5
        p.attend_shared(rows)


def test_what_a_row_does_not_see_does_not_reach_it():
    """NaN and infinities among shared tokens, seen by some of the slots' rows; scores far apart."""
    p = Shared(4, 60, 16, 20, 1, 64, "f16", q_per_kv=5, sinks=2, window=120)

    def spoil(k, v, start):
        nan, inf = float("nan"), float("inf")
        v[75, 0, 3], v[40, 0, 5], v[130, 0, 9], v[1, 0, 60] = nan, inf, nan, nan
        k[71, 0, 1] = nan
        k[150] *= 50
    p.reserve([200, 0, 0, 0])
    p.append([200, 0, 0, 0], spoil=spoil)
    p.select([0, 0, 0, 0])
    p.room([1, 40, 9, 20])
    for rows in ([1] * 4, [1, 3, 2, 12]):
        p.share(rows)
        p.attend_shared(rows)
        p.attend_shared(rows, size=30.0)


def test_plans_of_other_rows_and_other_contents():
    """With a plan for another number of rows, or an empty one, nothing is written."""
    p = Shared(6, 80, 16, 20, 2, 64, "f16", q_per_kv=4)
    prompt(p, 200, range(6))
    p.room([1, 2, 3, 4, 5, 6])
    p.share([1] * 6)
    q = p.t.zeros(11, 8, 64, dtype=p.t.float16, device="cuda")
    out = p.t.full_like(q, 3.5)
    p.own.attend_shared(0, q, out, p.ints([0, 1, 3, 6, 7, 8, 9]), 3, p.sharing)
    p.sharing.zero_()
    p.own.attend_shared(0, q, out, p.ints([0, 1, 3, 6, 7, 8, 9]), 3, p.sharing)
    assert (out == 3.5).all()
    p.share([1] * 6)
    p.attend_shared([1] * 6)


def test_a_captured_step():
    """Forks, then steps of one graph: room, copies, the plan, append and attention in two layers; eager calls in between."""
    import torch
    slots = 6
    p = Shared(slots, 120, 16, 24, 2, 64, "bf16", q_per_kv=2, layers=2)
    prompt(p, 180, range(slots))
    p.room([9, 1, 30, 4, 2, 16])
    one, start = p.ints([1] * slots), p.ints(np.arange(slots + 1))
    k, v = (torch.empty(slots, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.empty(slots, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    outs = [torch.empty_like(out) for _ in range(2)]
    plan = p.ints(np.zeros(1 + 2 * slots))

    def step():
        p.own.reserve(one, None, plan)
        p.own.copy(plan, slots)
        p.own.share(start, slots, p.sharing, least_bytes=0)
        for layer in range(2):
            p.own.append(layer, k, v, start)
            p.own.attend_shared(layer, q, outs[layer], start, 1, p.sharing)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(6):
        for x in (k, v, q):
            x.copy_(torch.tensor(p.rng.standard_normal(tuple(x.shape))))
        (step if i == 3 else graph.replay)()
        torch.cuda.synchronize()
        _, pairs = p.ref.reserve([1] * slots)
        p.ref.copy(pairs)
        p.state()
        for layer in range(2):
            p.ref.append(layer, k.double().cpu().numpy(), v.double().cpu().numpy(), np.arange(slots + 1))
            want, _, tol, _ = p.ref.attend(layer, q.double().cpu().numpy(), np.arange(slots + 1), HALF_STEP["bf16"])
            assert (np.abs(outs[layer].double().cpu().numpy() - want) <= tol).all()
        p.share([1] * slots, behind=0)
        p.attend([1] * slots)
        if i == 1:
            p.select([2, 2, 0, 3, 3, 1])


def test_rows_of_another_stream_and_wrong_tensors():
    import torch
    from paper_2402_09398_amd import LessdecError, PagedCache
    p = Shared(4, 60, 16, 16, 1, 128, "f16", q_per_kv=2)
    prompt(p, 150, range(4))
    p.room([1, 2, 3, 4])
    side = torch.cuda.Stream()
    q = torch.tensor(p.rng.standard_normal((4, 2, 128))).half().cuda()
    out, out2 = torch.empty_like(q), torch.empty_like(q)
    start = p.ints(np.arange(5))
    side.wait_stream(torch.cuda.current_stream())
    p.own.share(start, 4, p.sharing, least_bytes=0, stream=side)
    p.own.attend_shared(0, q, out, start, 1, p.sharing, stream=side)
    side.synchronize()
    p.own.share(start, 4, p.sharing, least_bytes=0)
    p.own.attend_shared(0, q, out2, start, 1, p.sharing)
    assert torch.equal(out, out2)
    bare = PagedCache(4, 60, 16, 16, 1, 128, "f16", q_per_kv=2, max_rows=4)
    for call in (lambda: bare.attend_shared(0, q, out, start, 1, bare.share_plan()), lambda: p.own.attend_shared(0, q, out, start, 1, p.sharing[:100]),
                 lambda: p.own.share(start[:4], 4, p.sharing), lambda: p.own.share(start, 4097, p.sharing), lambda: p.own.share(start, 4, p.sharing.float()),
                 lambda: p.own.share(start, 4, p.sharing[1:])):
        with pytest.raises(LessdecError):
            call()


@pytest.mark.parametrize("slots", [1900, 4096])
def test_as_many_slots_as_there_can_be(slots):
    p = Shared(slots, slots * 2 + 8, 16, 6, 1, 64, "bf16")
    prompt(p, 60, range(slots))
    p.room([1 + s % 3 for s in range(slots)])
    rows = [0, 0] + [1] * (slots - 2)
    assert len(p.share(rows)) == 1
    p.attend_shared(rows)
    rows = [s % 5 != 3 for s in range(slots)]
    p.select([s - s % 2 for s in range(slots)])
    p.share(rows)
    p.attend_shared(rows)


def test_many_columns_beside_few():
    """Slots of more columns than a tile has, that share nothing, before, between and behind those that do; head sizes and types."""
    for dim, dtype, group, window in ((64, "bf16", 2, 0), (128, "bf16", 5, 0), (64, "f16", 40, 100), (128, "f16", 1, 90)):
        p = Shared(7, 220, 16, 40, 2, dim, dtype, q_per_kv=group, window=window, sinks=3 if window else 0)
        prompt(p, 170, range(7))
        p.room([300, 1, 9, 300, 2, 30, 290])
        for rows in ([200, 1, 2, 130, 1, 3, 257], [0, 1, 9, 300, 2, 30, 0], [300, 1, 1, 0, 1, 1, 290]):
            p.share(rows)
            p.attend_shared(rows)


def test_offsets_past_31_bits():
    """A pool of 2.5 GiB a tensor: what is shared and what is not at its end, in the last layer."""
    import torch
    from paper_2402_09398_amd import PagedCache
    pages, heads, dim = 40960, 8, 128
    own = PagedCache(3, pages, 16, 16, heads, dim, "f16", layers=4, max_rows=64, shared=True)
    ref = po.Cache(3, 32, 16, 16, heads, dim)
    g = torch.Generator().manual_seed(5)
    far = [pages - 1, pages - 7, 33000, 5, pages - 2, pages - 100, 39999, pages - 50]
    at = iter(list(range(pages - 300, pages - 285)))
    tail = {s: [next(at) for _ in range(2)] for s in range(3)}
    names = {x: i for i, x in enumerate(far + sum(tail.values(), []))}
    ref.table[:] = -1
    for s in range(3):
        row = far + tail[s]
        own.table[s, :10] = torch.tensor(row, dtype=torch.int32)
        ref.table[s, :10] = [names[x] for x in row]
        ref.length[s] = 128 + 13 + s
    k, v, q = (torch.randn(192, heads, dim, generator=g).half() for _ in range(3))
    for counts, base in (([128, 0, 0], 0), ([13, 14, 15], 128)):
        lengths = [128, 128, 128] if base == 0 else [141, 142, 143]
        own.length[:] = torch.tensor(lengths, dtype=torch.int32)
        ref.length[:] = lengths
        start = np.concatenate([[0], np.cumsum(counts)])
        dev = torch.tensor(start, dtype=torch.int32).cuda()
        rows = slice(base, base + int(start[-1]))
        for layer in (0, 3):
            own.append(layer, k[rows].cuda(), v[rows].cuda(), dev)
        ref.append(0, k[rows].double().numpy(), v[rows].double().numpy(), start)
    plan = own.share_plan()
    for counts in ([1, 1, 1], [13, 14, 15]):
        start = np.concatenate([[0], np.cumsum(counts)])
        n, dev = int(start[-1]), torch.tensor(start, dtype=torch.int32).cuda()
        want, _, tol, _ = ref.attend(0, q[:n].double().numpy(), start, 2.0 ** -11)
        own.share(dev, n, plan, least_bytes=0)
        assert int(plan[0]) > 3 or counts == [1, 1, 1]
        for layer in (0, 3):
            out = torch.empty_like(q[:n]).cuda()
            own.attend_shared(layer, q[:n].cuda(), out, dev, max(counts), plan)
            assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


def test_rows_before_a_slots_first_token():
    """More rows than a slot has tokens, and slots that have none: what sees nothing is written as attend() writes it."""
    for group, rows in ((1, [3, 1, 9, 2, 4, 1]), (4, [6, 1, 30, 3, 9, 4]), (9, [2, 1, 14, 4, 2, 3]), (40, [5, 4, 1, 2, 2, 3])):
        p = Shared(6, 60, 16, 8, 2, 64, "f16", q_per_kv=group)
        p.room([2, 0, 2, 40, 40, 0])
        p.select([0, -1, 0, 3, 3, -1])
        p.room([0, 0, 1, 0, 1, 0])
        p.share(rows)
        out = p.attend_shared(rows)
        start = np.concatenate([[0], np.cumsum(rows)])
        for s in range(6):
            unseen = max(rows[s] - int(p.ref.length[s]), 0)
            assert (out[start[s]:start[s] + unseen] == 0).all() and (unseen > 0) == (s < 3 and rows[s] > p.ref.length[s] or s in (1, 5))


def test_plans_of_other_caches():
    """A plan that was made for as many rows of a cache with other slots writes nothing."""
    p, other = (Shared(n, 80, 16, 20, 2, 64, "f16", q_per_kv=4) for n in (6, 3))
    for x, rows in ((p, [1] * 6), (other, [2] * 3)):
        prompt(x, 200, range(len(rows)))
        x.room(rows)
        x.share(rows, behind=0)
    q = p.t.zeros(6, 8, 64, dtype=p.t.float16, device="cuda")
    out = p.t.full_like(q, 3.5)
    plan = p.own.share_plan()
    plan[:other.sharing.numel()] = other.sharing[:plan.numel()]
    p.own.attend_shared(0, q, out, p.ints(np.arange(7)), 1, plan)
    assert (out == 3.5).all()
