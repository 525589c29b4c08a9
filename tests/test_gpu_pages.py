"""The paged cache on the GPU, through PagedCache, against tests/pages_oracle.py: tables, lengths, counts, plans and stored values to
the bit, attention within tolerances that the oracle derives row by row."""
import numpy as np
import pytest

from tests import pages_oracle as po

pytestmark = pytest.mark.gpu
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


class Pair:
    """The cache and its oracle, driven together."""

    def __init__(self, slots, pages, page, wide, heads, dim, dtype="f16", seed=0, **more):
        import torch
        from paper_2402_09398_amd import PagedCache
        self.t, self.dtype = torch, dtype
        names = {"q_per_kv": "group"}
        self.own = PagedCache(slots, pages, page, wide, heads, dim, dtype, max_rows=4096, **more)
        self.ref = po.Cache(slots, pages, page, wide, heads, dim, **{names.get(k, k): v for k, v in more.items()})
        g = torch.Generator(device="cuda").manual_seed(seed)
        for name in ("k_codes", "v_codes"):                   # what an earlier program left there, NaN codes among it
            getattr(self.own, name).random_(0, 256, generator=g)
        self.own.exps.random_(-40, 41, generator=g)
        self.rng = np.random.default_rng(seed)
        self.plan = self.ints(np.full(1 + 2 * max(slots, pages // 2), -7))

    def ints(self, x):
        return self.t.tensor(np.asarray(x), dtype=self.t.int32).cuda()

    def state(self):
        assert np.array_equal(self.own.table.view(self.ref.slots, -1).cpu().numpy(), self.ref.table)
        assert np.array_equal(self.own.length.cpu().numpy(), self.ref.length)
        assert np.array_equal(self.own.refs.cpu().numpy(), self.ref.refs)

    def carry_out(self, plan):
        got = self.plan.cpu().numpy()
        assert got[0] == len(plan) and got[1:1 + 2 * len(plan)].reshape(-1, 2).tolist() == [list(p) for p in plan]
        self.ref.copy(plan)
        self.own.copy(self.plan, (self.plan.numel() - 1) // 2)
        self.state()

    def reserve(self, n_new):
        granted = self.ints(np.full(self.ref.slots, -9))
        self.own.reserve(self.ints(n_new), granted, self.plan)
        want, plan = self.ref.reserve(list(n_new))
        assert np.array_equal(granted.cpu().numpy(), want)
        self.carry_out(plan)
        return want

    def select(self, source):
        self.own.select(self.ints(source))
        self.ref.select(source)
        self.state()

    def compact(self):
        self.own.compact(self.plan)
        self.carry_out(self.ref.compact())

    def values(self, rows, heads, size):
        x = self.t.tensor(self.rng.standard_normal((rows, heads, self.ref.dim)) * size, dtype=self.own.tdtype)
        return x, x.double().numpy()

    def append(self, counts, size=1.0, spoil=None, layers=None):
        """Rows for the slots' last counts[s] tokens into every layer."""
        start = np.concatenate([[0], np.cumsum(counts)])
        for layer in range(self.ref.layers) if layers is None else layers:
            k, v = (self.t.tensor(self.rng.standard_normal((start[-1] + 2, self.ref.heads, self.ref.dim)) *
                                  np.exp2(self.rng.integers(-3, 4, (start[-1] + 2, 1, 1))) * size).to(self.own.tdtype) for _ in range(2))
            if spoil is not None:
                spoil(k, v, start)
            self.own.append(layer, k.cuda(), v.cuda(), self.ints(start))
            self.ref.append(layer, k.double().numpy(), v.double().numpy(), start)
        return start

    def held(self):
        for layer in range(self.ref.layers):
            count = max(1, int(self.ref.length.max()))
            slots = list(range(self.ref.slots))
            K, V = (self.t.full((len(slots), self.ref.heads, count, self.ref.dim), 7.0, dtype=self.own.tdtype, device="cuda") for _ in range(2))
            self.own.read(layer, self.ints(slots), 0, K, V)
            want = self.ref.read(layer, slots, 0, count, float(self.t.finfo(self.own.tdtype).max))
            for got, w in zip((K, V), want):
                np.testing.assert_array_equal(got.double().cpu().numpy(), self.t.tensor(w).to(self.own.tdtype).double().numpy())

    def attend(self, counts, layer=0, size=1.0, queries=None, lse=True):
        start = np.concatenate([[0], np.cumsum(counts)])
        hq = self.ref.heads * self.ref.group
        q = self.t.tensor(self.rng.standard_normal((start[-1] + 2, hq, self.ref.dim)) * size).to(self.own.tdtype) if queries is None else queries
        out = self.t.full(q.shape, 3.5, dtype=self.own.tdtype, device="cuda")
        stat = self.t.full(q.shape[:2], 3.5, device="cuda") if lse else None
        self.own.attend(layer, q.cuda(), out, self.ints(start), int(max(counts)), stat)
        want, want_lse, tol, lse_tol = self.ref.attend(layer, q.double().cpu().numpy(), start, HALF_STEP[self.dtype])
        got = out.double().cpu().numpy()
        assert (got[start[-1]:] == 3.5).all(), "rows behind the last slot"
        got, want, tol = got[:start[-1]], want[:start[-1]], tol[:start[-1]]
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        fine = ~np.isnan(want)
        off = np.abs(got - want)[fine] - tol[fine]
        assert (off <= 0).all(), f"off by up to {off.max():.3g} more than derived"
        if lse:
            got, want, lse_tol = stat.double().cpu().numpy(), want_lse[:start[-1]], lse_tol[:start[-1]]
            assert (got[start[-1]:] == 3.5).all()
            got = got[:start[-1]]
            np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
            np.testing.assert_array_equal(got == -np.inf, want == -np.inf)
            fine = np.isfinite(want)
            assert (np.abs(got[fine] - want[fine]) <= lse_tol[fine]).all()
        return out


STORE = [                                                     # heads, dim, page, dtype
    (1, 64, 16, "f16"), (3, 128, 32, "bf16"), (2, 128, 48, "f16"), (2, 64, 256, "bf16")]


@pytest.mark.parametrize("heads,dim,page,dtype", STORE)
def test_stored_values(heads, dim, page, dtype):
    """Prompts, single tokens into a block that goes on being filled, larger tokens that raise its exponent, blocks and pages that end."""
    p = Pair(5, 64, page, 8, heads, dim, dtype, layers=2)
    for n, size in (([5, 0, 33, 16, 1], 1.0), ([1, 1, 1, 1, 1], 1.0), ([1, 2, 0, 31, 14], 1e3), ([1, 1, 1, 1, 1], 1e-2), ([17, 40, 1, 0, 3], 30.0)):
        p.reserve(n)
        p.append(n, size)
        p.held()


def test_values_at_the_ends_of_the_types():
    """Infinities and NaN, zeros, the largest and smallest values, blocks of zeros, exponents at their limits; ties of the rounding."""
    p = Pair(3, 16, 16, 4, 2, 64, "bf16")

    def spoil(k, v, start):
        inf, nan = float("inf"), float("nan")
        k[0, 0, :6] = p.t.tensor([inf, -inf, nan, 0.0, -0.0, 1e-38])
        k[1] = 0
        v[0, :, 0], v[1, 1] = 1e38, 3e-30
        v[2, 0, :4] = p.t.tensor([448.0, 432.0, 416.0, 3.3e38])
        k[3, 0, :] = p.t.arange(64) * 0.0625 + 16
        k[4:, 1] = 0
    for n in ([3, 2, 16], [1, 1, 1], [13, 0, 2]):
        p.reserve(n)
        p.append(n, spoil=spoil if sum(n) > 5 else None)
        p.held()
    h = Pair(1, 4, 16, 2, 1, 64, "f16")
    h.reserve([3])
    h.append([3], spoil=lambda k, v, start: (k[0].fill_(65504.0), v[1].fill_(6e-8), v[0].zero_(), v[2].zero_()))
    h.held()


def test_rows_of_a_fused_projection():
    """q, k and v as views of one [rows, (Hq + 2 H) D] tensor."""
    p = Pair(2, 16, 16, 8, 2, 64, "f16", q_per_kv=3)
    n = [19, 4]
    p.reserve(n)
    both = p.t.tensor(p.rng.standard_normal((25, 10, 64))).half().cuda()
    q, k, v = both[:, :6], both[:, 6:8], both[:, 8:]
    start = np.array([0, 19, 23])
    p.own.append(0, k, v, p.ints(start))
    p.ref.append(0, k.double().cpu().numpy(), v.double().cpu().numpy(), start)
    p.held()
    packed = p.attend(n, queries=q.contiguous())
    out = p.t.full(q.shape, 3.5, dtype=p.t.float16, device="cuda")
    p.own.attend(0, q, out, p.ints(start), 19)
    assert p.t.equal(out, packed)


def test_room_is_made_in_order():
    """Free pages by index, slots by index; a slot that outgrows its table is passed over, one that does not fit ends the call; nothing wanted."""
    p = Pair(6, 10, 16, 5, 1, 64)
    p.reserve([16, 0, 40, 81, -3, 1])
    p.reserve([1, 80, 1, 1, 0, 0])
    p.reserve([48, 16, 40, 16, 16, 300])
    p.reserve([0] * 6)
    p.select([2, 2, -1, 0, 9, -5])
    p.reserve([3, 3, 3, 3, 3, 3])


@pytest.mark.parametrize("slots,page,wide", [(7, 16, 9), (70, 32, 6), (1030, 16, 3), (2500, 16, 2)])
def test_forks_share_until_they_write(slots, page, wide):
    p = Pair(slots, slots * wide // 2 + 5, page, wide, 1, 64)
    rng = np.random.default_rng(slots)
    n = np.zeros(slots, int)
    n[:5] = [20, 16, 33, 1, 17]
    p.reserve(n)
    p.append(n)
    p.select([int(x) if i > 4 else i for i, x in enumerate(rng.integers(0, 5, slots))])
    for _ in range(3):
        n = rng.integers(0, 3, slots)
        got = p.reserve(n)
        if slots < 100:
            p.append(got)
            p.held()
        source = rng.integers(-1, slots, slots)
        source[::3] = np.arange(slots)[::3]
        p.select(source.tolist())
        p.compact()
        if slots < 100:
            p.held()


def test_many_pages_of_one_slot():
    """A prompt of thousands of pages: the lists of free pages go over several turns of the workgroup."""
    p = Pair(3, 40000, 16, 30000, 1, 64)
    p.reserve([100, 300000, 7])
    p.select([0, -1, 2])
    p.reserve([1, 20000, 170000])
    p.select([-1, 1, 1])
    p.compact()


def test_pages_behind_the_window_are_let_go():
    p = Pair(4, 40, 16, 40, 1, 64, sinks=20, window=37)
    for n in ([50, 3, 200, 36], [1, 1, 1, 1], [16, 100, 1, 1], [1, 0, 90, 1], [1, 1, 1, 1]):
        got = p.reserve(n)
        p.append(got)
        p.held()
        p.attend(np.minimum(got, 3))
    p.select([2, 1, 2, 0])
    p.reserve([1, 1, 1, 1])


FEW = [                                                       # slots, heads, group, dim, page, dtype, lengths, rows a slot, sinks, window
    (1, 1, 1, 64, 16, "f16", [1], [1], 0, 0),
    (3, 2, 1, 128, 16, "f16", [1, 16, 17], [1, 1, 1], 0, 0),
    (5, 3, 4, 128, 32, "bf16", [129, 0, 31, 2000, 64], [1, 0, 1, 1, 1], 0, 0),
    (4, 2, 5, 64, 64, "f16", [300, 5, 127, 128], [3, 3, 1, 2], 0, 0),
    (2, 1, 16, 128, 16, "bf16", [777, 40], [1, 1], 0, 0),
    (4, 2, 2, 64, 16, "bf16", [900, 33, 3, 16], [1, 4, 2, 8], 0, 20),
    (4, 2, 2, 128, 32, "f16", [900, 33, 3, 500], [1, 4, 2, 8], 4, 100),
    (3, 1, 3, 64, 16, "f16", [400, 50, 17], [1, 5, 1], 70, 1),
    (300, 1, 1, 64, 16, "f16", [1 + 7 * i % 60 for i in range(300)], [i % 3 for i in range(300)], 0, 0),
]
WIDE = [
    (1, 2, 1, 128, 16, "f16", [17], [17], 0, 0),
    (2, 1, 1, 64, 32, "bf16", [200, 64], [200, 64], 0, 0),
    (3, 2, 4, 128, 16, "bf16", [300, 40, 1], [70, 33, 1], 0, 0),
    (3, 1, 71, 64, 32, "f16", [130, 64, 1], [1, 2, 1], 0, 0),
    (4, 2, 3, 64, 16, "f16", [500, 0, 77, 129], [129, 0, 77, 1], 0, 0),
    (2, 2, 2, 128, 64, "f16", [300, 150], [150, 20], 4, 64),
    (2, 1, 1, 64, 16, "bf16", [400, 90], [400, 90], 0, 33),
    (2, 1, 8, 128, 16, "f16", [600, 31], [20, 31], 40, 1),
    (1, 1, 20, 64, 16, "bf16", [2100], [1], 0, 0),
]


@pytest.mark.parametrize("slots,heads,group,dim,page,dtype,lengths,rows,sinks,window", FEW + WIDE)
def test_attention(slots, heads, group, dim, page, dtype, lengths, rows, sinks, window):
    wide = -(-max(lengths) // page) + 1
    p = Pair(slots, sum(-(-n // page) for n in lengths) + 3, page, wide, heads, dim, dtype, seed=slots + dim, q_per_kv=group, sinks=sinks, window=window)
    first = [n - r for n, r in zip(lengths, rows)]
    if any(first):
        p.reserve(first)
        p.append(first)
    p.reserve(rows)
    p.append(rows)
    p.attend(rows, size=1.0)
    p.attend(rows, size=4.0, lse=False)
    p.select([(i * 3 + 1) % slots for i in range(slots)])
    p.attend([rows[(i * 3 + 1) % slots] for i in range(slots)])


@pytest.mark.parametrize("group,rows", [(1, 1), (2, 6), (3, 40)])
def test_what_a_row_does_not_see_does_not_reach_it(group, rows):
    """NaN and infinite keys and values: rows that see them are NaN, the others are as without; codes behind a slot's end are left as an
    earlier program wrote them."""
    p = Pair(2, 40, 16, 20, 1, 64, "f16", q_per_kv=group, sinks=2, window=30)
    n = [100, 41]
    p.reserve(n)

    def spoil(k, v, start):
        nan, inf = float("nan"), float("inf")
        v[75, 0, 3], v[40, 0, 5], v[start[1] - 2, 0, 9], v[start[2] - 1, 0, 60] = nan, inf, nan, nan
        k[71, 0, 1] = nan
    p.append(n, spoil=spoil)
    p.held()
    p.attend([rows, min(rows, 41)])
    p.attend([1, 1])


def test_scores_and_exponents_far_apart():
    """Blocks whose values differ by many powers of two, keys that dominate, scores of +-1e4: weights relative to the contributions."""
    for dtype in ("f16", "bf16"):
        p = Pair(2, 40, 16, 20, 2, 64, dtype, q_per_kv=2)
        n = [200, 130]
        p.reserve(n)

        def spoil(k, v, start):
            for b in range(0, 330, 16):
                v[b:b + 16] *= 2.0 ** (b // 16 % 13 - 8)
            k[::37] *= 20
        p.append(n, spoil=spoil)
        for rows in ([1, 1], [3, 3], [90, 130]):
            p.attend(rows, size=1.0)
            p.attend(rows, size=30.0)
            p.attend(rows, size=0.0)


def test_a_long_sequence_over_many_workgroups():
    p = Pair(2, 1400, 16, 1300, 1, 64, "bf16", q_per_kv=2)
    n = [20000, 200]
    p.reserve(n)
    p.append(n)
    p.attend([1, 1])
    p.attend([9, 9])
    p.attend([3, 150])


def test_offsets_past_31_bits():
    """A pool of 2.5 GiB a tensor: pages at its end, in the last layer."""
    import torch
    from paper_2402_09398_amd import PagedCache
    pages, heads, dim = 40960, 8, 128
    own = PagedCache(2, pages, 16, 8, heads, dim, "f16", layers=4, max_rows=64)
    ref = po.Cache(2, 16, 16, 8, heads, dim)
    ref.table[:] = -1
    own.table[0, :4] = torch.tensor([pages - 1, pages - 7, 33000, 5], dtype=torch.int32)
    own.length[0] = 57
    ref.table[0, :4], ref.length[0] = [0, 1, 2, 3], 57
    g = torch.Generator().manual_seed(3)
    k, v, q = (torch.randn(57, heads, dim, generator=g).half() for _ in range(3))
    start = np.array([0, 57, 57])
    dev = torch.tensor(start, dtype=torch.int32).cuda()
    for layer in (0, 3):
        own.append(layer, k.cuda(), v.cuda(), dev)
    ref.append(0, k.double().numpy(), v.double().numpy(), start)
    want, _, tol, _ = ref.attend(0, q.double().numpy(), start, 2.0 ** -11)
    for layer in (0, 3):
        out = torch.empty_like(q).cuda()
        own.attend(layer, q.cuda(), out, dev, 57)
        assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


def test_serving_loop_replayed_from_a_graph():
    """Room, copies, append and attention of two layers as one captured step, replayed between eager work, against the oracle; forks and
    a compaction between replays."""
    import torch
    p = Pair(4, 60, 16, 12, 2, 64, "bf16", layers=2, q_per_kv=2)
    n = [30, 5, 0, 17]
    p.reserve(n)
    p.append(n)
    ones, start = p.ints([1] * 4), p.ints(range(5))
    k, v = (torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, out = (torch.zeros(2, 4, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step():
        p.own.reserve(ones, None, p.plan)
        p.own.copy(p.plan, 4)
        for layer in range(2):
            p.own.append(layer, k[layer], v[layer], start)
            p.own.attend(layer, q[layer], out[layer], start, 1)
    saved = [getattr(p.own, x).clone() for x in p.own.STATE]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x, y in zip(p.own.STATE, saved):
        getattr(p.own, x).copy_(y)
    for turn in range(5):
        for x in (k, v, q):
            x.copy_(torch.tensor(p.rng.standard_normal(x.shape)))
        if turn == 2:
            p.select([0, 0, 3, 3])
        if turn == 4:
            p.select([-1, 1, 2, 3])
            p.compact()
        graph.replay()
        torch.cuda.synchronize()
        _, plan = p.ref.reserve([1] * 4)
        p.ref.copy(plan)
        for layer in range(2):
            p.ref.append(layer, k[layer].double().cpu().numpy(), v[layer].double().cpu().numpy(), np.arange(5))
            want, _, tol, _ = p.ref.attend(layer, q[layer].double().cpu().numpy(), np.arange(5), HALF_STEP["bf16"])
            assert (np.abs(out[layer].double().cpu().numpy() - want) <= tol).all(), (turn, layer)
        p.state()
        p.held()


def test_a_sequence_goes_over_to_the_compressed_cache():
    """read() hands the tokens of paged slots to lessdec_prefill as [B, Hh, P, D]: its attention of the last token is the paged one's."""
    import torch
    from paper_2402_09398_amd import workloads as wl
    from tests import harness as hz
    w = wl.WORKLOADS[2].scaled(name="from-pages", batch=2, heads=3, prompt=50, steps=1, n_heavy=8, n_recent=8, hidden=64)
    p = Pair(3, 20, 16, 4, 3, w.head_dim)
    n = [50, 0, 50]
    p.reserve(n)
    p.append(n)
    K, V, Q = (torch.empty(2, 3, 50, w.head_dim, dtype=torch.float16, device="cuda") for _ in range(3))
    p.own.read(0, p.ints([0, 2]), 0, K, V)
    Q.copy_(torch.tensor(p.rng.standard_normal(Q.shape)))
    layer = hz.make_gpu(w)
    out = torch.empty_like(Q)
    layer.prefill(Q, K, V, out)
    start = np.array([0, 50, 50, 100])
    rows = Q.transpose(1, 2).reshape(100, 3, w.head_dim).contiguous()
    want, _, tol, _ = p.ref.attend(0, rows.double().cpu().numpy(), start, 2.0 ** -11)
    got = out.transpose(1, 2).reshape(100, 3, w.head_dim).double().cpu().numpy()
    assert (np.abs(got - want) <= tol).all()
    paged = torch.empty_like(rows)
    p.own.attend(0, rows, paged, p.ints(start), 50)
    assert (np.abs(paged.double().cpu().numpy() - want) <= tol).all()


def test_calls_on_another_stream():
    import torch
    p = Pair(2, 20, 16, 8, 2, 64)
    side = torch.cuda.Stream()
    ints = [p.ints(x) for x in ([40, 3], [0, 40, 43])]
    g = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(43, 2, 64, generator=g).half().cuda() for _ in range(3))
    out = torch.empty_like(q)
    side.wait_stream(torch.cuda.current_stream())
    p.own.reserve(ints[0], None, p.plan, stream=side)
    p.own.copy(p.plan, 2, stream=side)
    p.own.append(0, k, v, ints[1], stream=side)
    p.own.attend(0, q, out, ints[1], 40, stream=side)
    side.synchronize()
    p.ref.reserve([40, 3])
    start = np.array([0, 40, 43])
    p.ref.append(0, k.double().cpu().numpy(), v.double().cpu().numpy(), start)
    want, _, tol, _ = p.ref.attend(0, q.double().cpu().numpy(), start, 2.0 ** -11)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
