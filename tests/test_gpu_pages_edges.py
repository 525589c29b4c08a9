"""The paged cache where its kernels go round: look-ups that reach their next chunk, tiles over many workgroups, slots in and out of order,
tables with holes, calls that share a workspace or run beside one another."""
import numpy as np
import pytest

from tests.test_gpu_pages import HALF_STEP, Pair

pytestmark = pytest.mark.gpu


def holes(p, entries):
    """Entries of the table that name no page of the pool, in the cache and in the oracle."""
    for i, (slot, entry) in enumerate(entries):
        bad = [-1, p.ref.pages, 2 ** 31 - 1, -2 ** 31][i % 4]
        p.own.table[slot, entry] = bad
        p.ref.table[slot, entry] = bad


def fill(p, n, spoil=None):
    p.reserve(n)
    p.append(n, spoil=spoil)


@pytest.mark.parametrize("page,sinks,window", [(48, 0, 0), (16, 5, 39000), (1024, 70, 21000)])
def test_splits_of_many_tiles(page, sinks, window):
    """16 slots, one of 40000 tokens: a workgroup has 20 tiles and looks up its pages more than once; NaN and missing pages on the way."""
    n = [0] * 16
    n[3], n[7] = 40000, 18
    p = Pair(16, 40000 // page + 8, page, 40000 // page + 2, 1, 64, "bf16", q_per_kv=71, sinks=sinks, window=window)
    fill(p, n)
    rows = [0] * 16
    rows[3], rows[7] = 2, 1
    p.attend(rows)
    holes(p, [(3, 40000 // page - 2), (3, 0), (3, 25000 // page), (3, 25000 // page + 1)])
    p.attend(rows)
    q = p.t.tensor(p.rng.standard_normal((5, 71, 64))).to(p.own.tdtype)
    p.attend(rows, queries=q)


@pytest.mark.parametrize("slots,heads,window", [(64, 8, 0), (65, 8, 0), (64, 8, 700)])
def test_tiles_without_splits(slots, heads, window):
    """Enough workgroups without splits; up to 64 slots the longest come first, behind that they are in order.  24 tiles to a workgroup, a
    page missing in the second chunk, a NaN that only some rows see, slots without rows and with few."""
    n, rows = [0] * slots, [0] * slots
    for s, length, count in ((0, 40, 1), (1, 1500, 140), (2, 90, 90), (30, 1500, 20), (61, 17, 17), (slots - 1, 600, 33)):
        n[s], rows[s] = length, count
    p = Pair(slots, 260, 16, 100, heads, 64, "f16", sinks=3 if window else 0, window=window)

    def spoil(k, v, start):
        v[start[2] - 70, 1, 7] = v[start[slots] - 3, 0, 1] = float("nan")
    fill(p, n, spoil)
    p.attend(rows)
    holes(p, [(1, 70), (30, 92), (30, 93), (slots - 1, 2)])
    p.attend(rows)


@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (128, "bf16")])
def test_shares_of_many_steps(dim, dtype):
    """24 sequences of 140800 tokens, one new token each: more steps to a workgroup than it looks up at a time.  Their tables name the same
    64 pages again and again."""
    slots, wide = 24, 8800
    p = Pair(slots, 64, 16, wide, 1, dim, dtype)
    n = [0] * slots
    n[0] = 1024
    fill(p, n)
    table = p.rng.integers(0, 64, (slots, wide))
    table[5, 8000:8003] = [-1, 64, -9]
    length = np.full(slots, wide * 16)
    length[9], length[23] = 0, wide * 16 - 5
    p.own.table.copy_(p.ints(table))
    p.own.length.copy_(p.ints(length))
    p.ref.table, p.ref.length = table, length
    q = p.t.tensor(p.rng.standard_normal((slots, 1, dim))).to(p.own.tdtype)
    out, start = p.t.full(q.shape, 3.5, dtype=p.own.tdtype, device="cuda"), p.ints(range(slots + 1))
    p.own.attend(0, q.cuda(), out, start, 1)
    got = out.double().cpu().numpy()
    for s in (0, 5, 9, 23):
        one = np.array([0] * (s + 1) + [1] * (slots - s))
        want, _, tol, _ = p.ref.attend(0, q[s:s + 1].double().numpy(), one, HALF_STEP[dtype])
        assert (np.abs(got[s:s + 1] - want) <= tol).all(), s
    again = p.t.zeros_like(out)
    for _ in range(3):                                        # shares are joined in their order, whoever comes last
        p.own.attend(0, q.cuda(), again, start, 1)
        assert p.t.equal(again, out)


@pytest.mark.parametrize("group", [1, 40])
def test_the_most_slots(group):
    slots = 4096
    n, rows = [0] * slots, [0] * slots
    for s in (0, 1, 63, 64, 1000, 2047, 2048, 4030, 4095):
        n[s], rows[s] = 1 + s % 50, 1
    p = Pair(slots, 64, 16, 5, 1, 64, q_per_kv=group)
    fill(p, n)
    p.attend(rows)
    for s in (0, 4095):
        K, V = (p.t.full((1, 1, n[s], 64), 7.0, dtype=p.own.tdtype, device="cuda") for _ in range(2))
        p.own.read(0, p.ints([s]), 0, K, V)
        want = p.ref.read(0, [s], 0, n[s], 65504.0)
        np.testing.assert_array_equal(K.double().cpu().numpy(), want[0])
        np.testing.assert_array_equal(V.double().cpu().numpy(), want[1])


@pytest.mark.parametrize("group,rows", [(2, 3), (4, 50)])
def test_queries_that_are_no_numbers(group, rows):
    """Infinite and NaN queries spoil their own row; the largest finite ones dominate without overflow of a weight."""
    p = Pair(2, 30, 16, 10, 2, 128, "bf16", q_per_kv=group)
    n = [100, rows]
    fill(p, n)
    q = p.t.tensor(p.rng.standard_normal((2 * rows + 2, 2 * group, 128))).to(p.own.tdtype)
    q[0, 0, 3], q[1, 1, 5], q[2, 2, 7] = float("nan"), float("inf"), float("-inf")
    q[rows, 0], q[rows + 1, 1] = 0, 300
    p.attend([rows, rows], queries=q)


def test_rows_further_apart():
    """Rows eight elements further apart than packed, q, k and v each with a stride of its own."""
    p = Pair(2, 16, 16, 8, 3, 64, "bf16", q_per_kv=2)
    n = [21, 2]
    p.reserve(n)

    def apart(heads):
        x = p.t.tensor(p.rng.standard_normal((23, heads * 64 + 8 * heads))).to(p.own.tdtype).cuda()
        return x[:, :heads * 64].unflatten(1, (heads, 64))
    k, v, q, start = apart(3), apart(3), apart(6), np.array([0, 21, 23])
    p.own.append(0, k, v, p.ints(start))
    p.ref.append(0, k.double().cpu().numpy(), v.double().cpu().numpy(), start)
    p.held()
    out = p.t.empty(23, 6, 64, dtype=p.own.tdtype, device="cuda")
    p.own.attend(0, q, out, p.ints(start), 21)
    want, _, tol, _ = p.ref.attend(0, q.double().cpu().numpy(), start, HALF_STEP["bf16"])
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


def test_tables_with_holes():
    """append, attend and read pass over what is not there."""
    p = Pair(3, 30, 32, 9, 2, 64, "f16")
    n = [200, 70, 33]
    fill(p, n)
    holes(p, [(0, 1), (0, 6), (1, 2), (2, 0)])
    p.held()
    p.append([40, 7, 33])
    p.held()
    for rows in ([1, 1, 1], [40, 7, 33]):
        p.attend(rows)
    p.ref.table[2, 1] = -1                                    # nothing of a slot is there: its rows are 0, their lse is -inf
    p.own.table[2, 1] = -1
    p.attend([1, 0, 33])


def test_two_graphs_and_eager_calls_share_a_workspace():
    """A decode step's graph and a prompt's, replayed in turn on one stream, with eager calls of other shapes between them."""
    import torch
    p = Pair(3, 200, 16, 160, 2, 64, "f16", q_per_kv=2)
    n = [2300, 40, 700]
    fill(p, n)
    shapes = ([1, 1, 1], [30, 0, 200])
    calls = []
    for rows in shapes:
        start = p.ints(np.concatenate([[0], np.cumsum(rows)]))
        q = torch.zeros(sum(rows), 4, 64, dtype=torch.float16, device="cuda")
        calls.append((q, torch.zeros_like(q), start, max(rows)))
    graphs = []
    for q, out, start, most in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.own.attend(0, q, out, start, most)
        graphs.append(graph)
    for turn in range(4):
        for which in (0, 1) if turn % 2 else (1, 0):
            q, out, start, most = calls[which]
            q.copy_(torch.tensor(p.rng.standard_normal(q.shape)))
            out.fill_(3.5)
            graphs[which].replay()
            eager = torch.empty_like(out)
            p.own.attend(0, q, eager, start, most)
            assert torch.equal(eager, out)
            want, _, tol, _ = p.ref.attend(0, q.double().cpu().numpy(), start.cpu().numpy(), HALF_STEP["f16"])
            assert (np.abs(out.double().cpu().numpy() - want) <= tol).all(), (turn, which)
        p.attend([2, 7, 1])


def test_caches_beside_one_another():
    """Two caches, each on a stream of its own, at once."""
    import torch
    pairs = [Pair(4, 800, 16, 200, 2, 64, "f16", seed=i, q_per_kv=2) for i in range(2)]
    n = [3000, 10, 500, 2900]
    for p in pairs:
        fill(p, n)
    streams = [torch.cuda.Stream() for _ in pairs]
    for rows in ([1, 1, 1, 1], [3, 0, 90, 200]):
        start = np.concatenate([[0], np.cumsum(rows)])
        dev = pairs[0].ints(start)
        q = torch.randn(int(start[-1]), 4, 64, generator=torch.Generator().manual_seed(7)).half().cuda()
        alone, beside = [], [[torch.empty_like(q) for _ in range(6)] for _ in pairs]
        for p in pairs:
            alone.append(torch.empty_like(q))
            p.own.attend(0, q, alone[-1], dev, max(rows))
        torch.cuda.synchronize()
        for i in range(6):
            for p, s, out in zip(pairs, streams, beside):
                p.own.attend(0, q, out[i], dev, max(rows), stream=s)
        torch.cuda.synchronize()
        for want, outs in zip(alone, beside):
            assert all(torch.equal(want, out) for out in outs)


def test_no_rows():
    p = Pair(2, 8, 16, 4, 2, 64, q_per_kv=2)
    fill(p, [5, 0])
    none = p.t.empty(0, 2, 64, dtype=p.own.tdtype, device="cuda")
    start = p.ints([0, 0, 0])
    p.own.append(0, none, none, start)
    p.own.attend(0, none.expand(0, 2, 64).repeat(1, 2, 1), p.t.empty(0, 4, 64, dtype=p.own.tdtype, device="cuda"), start, 0)
    K = p.t.empty(0, 2, 3, 64, dtype=p.own.tdtype, device="cuda")
    p.own.read(0, p.ints([]), 0, K, K.clone())
    K = p.t.empty(1, 2, 0, 64, dtype=p.own.tdtype, device="cuda")
    p.own.read(0, p.ints([0]), 0, K, K.clone())
    p.reserve([0, 0])
    p.own.copy(p.plan, 0)
    p.held()


@pytest.mark.parametrize("group,dim,rows", [(17, 64, [1, 0, 2]), (128, 128, [1, 2, 0]), (3, 64, [5, 6, 1])])
def test_groups_at_the_edges_of_a_tile(group, dim, rows):
    """Columns just past one matrix tile, exactly one workgroup's, 15 and 18."""
    p = Pair(3, 40, 16, 12, 2, dim, "f16", q_per_kv=group)
    fill(p, [150, 40, 7])
    p.attend(rows)


@pytest.mark.parametrize("scale", [0.3, 2.0 ** -40, 3.0])
def test_scales(scale):
    p = Pair(2, 30, 32, 8, 1, 64, "bf16", q_per_kv=2, scale=scale)
    fill(p, [200, 50])
    for rows in ([1, 1], [40, 50]):
        p.attend(rows)


def test_the_functions_of_the_library_by_name():
    """The front end without PagedCache: its own descriptor, one call of each."""
    from paper_2402_09398_amd import pages as lib
    p = Pair(2, 12, 16, 4, 1, 64, "f16")
    d, t = p.own.desc, p.t
    assert lib.lessdec_pages_workspace_bytes(d, 4096) == d.workspace_bytes
    lib.lessdec_pages_reset(d)
    granted = p.ints([-1, -1])
    lib.lessdec_pages_reserve(d, p.ints([20, 3]), granted, p.plan)
    lib.lessdec_pages_copy(d, p.plan, 2)
    p.ref.reserve([20, 3])
    p.state()
    start = np.array([0, 20, 23])
    x = t.tensor(p.rng.standard_normal((3, 23, 1, 64))).half().cuda()
    lib.lessdec_pages_append(d, 0, x[0], x[1], 0, p.ints(start), 23)
    p.ref.append(0, x[0].double().cpu().numpy(), x[1].double().cpu().numpy(), start)
    p.held()
    out, lse = t.empty_like(x[2]), t.empty(23, 1, device="cuda")
    lib.lessdec_pages_attend(d, 0, x[2], 0, out, lse, p.ints(start), 23, 20)
    want, want_lse, tol, lse_tol = p.ref.attend(0, x[2].double().cpu().numpy(), start, HALF_STEP["f16"])
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all() and (np.abs(lse.double().cpu().numpy() - want_lse) <= lse_tol).all()
    lib.lessdec_pages_select(d, p.ints([-1, 0]))
    p.ref.select([-1, 0])
    lib.lessdec_pages_compact(d, p.plan)
    lib.lessdec_pages_copy(d, p.plan, 6)
    p.ref.copy(p.ref.compact())
    p.state()
    K, V = (t.empty(1, 1, 20, 64, dtype=t.float16, device="cuda") for _ in range(2))
    lib.lessdec_pages_read(d, 0, p.ints([1]), 1, 0, 20, K, V)
    assert np.array_equal(V.double().cpu().numpy(), p.ref.read(0, [1], 0, 20, 65504.0)[1])


def test_refusals():
    import torch
    from paper_2402_09398_amd import LessdecError, PagedCache
    c = PagedCache(2, 8, 16, 4, 2, 64, "f16", q_per_kv=2, max_rows=8)
    start, k, q = (torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda"),
                   torch.zeros(4, 4, 64, dtype=torch.float16, device="cuda"))
    ints = torch.zeros(64, dtype=torch.int32, device="cuda")
    wide = torch.zeros(4, 2, 128, dtype=torch.float16, device="cuda")
    bad = [
        lambda: PagedCache(2, 8, 16, 4, 2, 64, "f32"), lambda: PagedCache(2, 8, 20, 4, 2, 64, "f16"), lambda: PagedCache(2, 8, 16, 4, 2, 96, "f16"),
        lambda: PagedCache(2, 8, 16, 4, 2, 64, "f16", buffers={n: getattr(c, n)[:1] for n in c.STATE}),
        lambda: c.append(0, k.float(), k, start), lambda: c.append(0, k, k.cpu(), start), lambda: c.append(0, k, k[:3], start),
        lambda: c.append(1, k, k, start), lambda: c.append(-1, k, k, start), lambda: c.append(0, wide, wide, start),
        lambda: c.append(0, wide[..., ::2], wide[..., ::2], start), lambda: c.append(0, k.transpose(0, 1), k.transpose(0, 1), start),
        lambda: c.append(0, k[:1].expand(4, 2, 64), k[:1].expand(4, 2, 64), start),
        lambda: c.append(0, k.view(-1)[4:260].view(2, 2, 64), k[:2], start), lambda: c.append(0, k, k, start[:2]),
        lambda: c.append(0, k, k, start.long()), lambda: c.append(0, k, k, start.cpu()),
        lambda: c.attend(0, k, k, start, 1), lambda: c.attend(0, q, q[:3], start, 1), lambda: c.attend(0, q, q.bfloat16(), start, 1),
        lambda: c.attend(0, q, torch.zeros(4, 8, 64, dtype=torch.float16, device="cuda")[:, ::2], start, 1),
        lambda: c.attend(0, q, torch.empty_like(q), start, 1, lse=torch.zeros(4, 2, device="cuda")), lambda: c.attend(0, q, torch.empty_like(q), start, -1),
        lambda: c.attend(0, q.repeat(3, 1, 1), q.repeat(3, 1, 1), start, 1),
        lambda: c.reserve(ints[:1], None, ints), lambda: c.reserve(ints[:2], None, ints[:4]), lambda: c.reserve(ints, ints, ints),
        lambda: c.select(ints[:1]), lambda: c.select(c.length), lambda: c.compact(ints[:8]), lambda: c.copy(ints[:4], 2), lambda: c.copy(ints, -1),
        lambda: c.read(0, ints[:1], 0, torch.zeros(1, 2, 4, 64, device="cuda"), torch.zeros(1, 2, 4, 64, device="cuda")),
        lambda: c.read(0, ints[:1], 0, torch.zeros(2, 2, 4, 64, dtype=torch.float16, device="cuda"), torch.zeros(2, 2, 4, 64, dtype=torch.float16, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(LessdecError):
            call()
            pytest.fail(f"call {i} was let through")
    torch.cuda.synchronize()


@pytest.mark.parametrize("slots,page,heads,dim,dtype,group,window,sinks", [
    (3, 16, 3, 64, "f16", 1, 0, 0), (9, 48, 2, 128, "bf16", 4, 40, 3), (5, 256, 8, 64, "bf16", 17, 0, 0), (40, 32, 2, 64, "f16", 5, 7, 20),
    (70, 16, 1, 128, "bf16", 20, 100, 3)])
def test_sequences_that_come_and_go(slots, page, heads, dim, dtype, group, window, sinks):
    """Twelve turns, chosen at random, of a program that adds tokens, attends, forks, ends sequences and compacts its pool."""
    r = np.random.default_rng(slots * page)
    wide = -(-150 // page) + 1
    p = Pair(slots, slots * wide * 2 // 3 + 2, page, wide, heads, dim, dtype, seed=slots, q_per_kv=group, window=window, sinks=sinks)
    for turn in range(12):
        if turn % 4 == 2:
            source = r.integers(-1, slots, slots)
            stay = r.random(slots) < 0.5
            source[stay] = np.arange(slots)[stay]
            p.select(source.tolist())
        elif turn % 4 == 3 and turn > 4:
            p.compact()
        else:
            got = p.reserve(r.integers(0, [2, 6, 75][turn % 3], slots))
            p.append(got, [1.0, 30.0][turn % 2])
            rows = [int(min(n, r.integers(1, 40))) if r.random() < 0.4 else 0 for n in got]
            p.attend(rows if any(rows) else [1] + [0] * (slots - 1), size=[1.0, 5.0][turn % 2])
    p.held()
