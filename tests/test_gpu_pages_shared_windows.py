"""Attention over shared pages with a window, slots of several prompts side by side: what a slot no longer sees, it may still name, and what it sees, the
slot before it may have let go, or name and not see.  Against tests/pages_oracle.py; plans looked over node by node by Shared.share."""
import numpy as np
import pytest

from tests.test_gpu_pages_shared import Shared

pytestmark = pytest.mark.gpu


def forks(p, prompts, of):
    """Prompts of so many tokens in the first slots that are to have them; every slot a fork of one (-1: empty)."""
    slots = p.ref.slots
    first = [of.index(i) for i in range(len(prompts))]
    p.room([prompts[first.index(s)] if s in first else 0 for s in range(slots)])
    p.select([first[i] if i >= 0 else -1 for i in of])


def both(p, rows):
    nodes = p.share(rows)
    p.attend_shared(rows)
    return nodes


@pytest.mark.parametrize("dim,dtype,group", [(64, "f16", 1), (128, "bf16", 4), (64, "bf16", 20)])
def test_a_slot_that_names_what_it_does_not_see(dim, dtype, group):
    """Slots 1 and 2 are forks of one prompt and name its pages 25 to 27, of which only slot 2 sees a token; slot 0, of another prompt, lies as far back
    as slot 2 and names others there."""
    p = Shared(3, 140, 16, 40, 2, dim, dtype, q_per_kv=group, window=100)
    forks(p, [500, 500], [0, 1, 1])
    p.room([1, 50, 1])
    assert p.ref.table[1, 27] == p.ref.table[2, 27] != p.ref.table[0, 27]
    nodes = both(p, [1, 1, 1])
    assert any((row, rows) == (1, 2) and last == 31 for row, rows, _, last, *_ in nodes), "what slots 1 and 2 share"
    both(p, [1, 3, 1])
    both(p, [1, 50, 1])


def test_a_slot_that_has_let_go():
    """As above, but slot 1 names nothing there any more; and slots without rows, or with many columns, between the two prompts."""
    for group, between in ((1, 0), (4, 1), (16, 20)):
        p = Shared(5, 300, 16, 60, 2, 64, "f16", q_per_kv=group, window=100, sinks=5)
        forks(p, [500, 500], [0, 1, 1, 1, 1])
        p.room([1, 50, 1, 90, 1])
        p.room([0, 50, 1, 30, 1])
        for rows in ([1, 1, 1, 1, 1], [1, between, 1, 1, 1], [1, 1, 2, between, 2], [1, 0, 1, 0, 1]):
            both(p, rows)


@pytest.mark.parametrize("seed", range(24))
def test_prompts_side_by_side(seed):
    """Several prompts behind the same beginning or none, forks in any number, uneven reservations, fewer rows than were reserved for some."""
    rng = np.random.default_rng(seed)
    page, window, sinks = int(rng.choice([16, 16, 32, 48])), int(rng.choice([1, 17, 60, 100, 200, 350])), int(rng.choice([0, 0, 3, 40]))
    group, dim, dtype = int(rng.choice([1, 2, 5, 16, 40])), int(rng.choice([64, 128])), str(rng.choice(["f16", "bf16"]))
    slots, prompts = int(rng.integers(3, 14)), int(rng.integers(2, 4))
    of = sorted([*range(prompts), *rng.integers(0, prompts, slots - prompts).tolist()])
    p = Shared(slots, 500, page, 48, 1, dim, dtype, seed=seed, q_per_kv=group, window=window, sinks=sinks)
    if seed % 3 == 0:
        system = int(rng.integers(1, 200))
        p.room([system] + [0] * (slots - 1))
        p.select([0] * slots)
    first = [of.index(i) for i in range(prompts)]
    p.room([int(rng.integers(20, 300)) if s in first else 0 for s in range(slots)])
    p.select([first[i] for i in of])
    for step in range(3):
        new = [int(rng.choice([0, 1, 1, 5, rng.integers(1, 70)])) for _ in range(slots)]
        p.room(new)
        for rows in ([1] * slots, [int(rng.integers(0, min(n, 9) + 1)) for n in new], [max(n, 1) if rng.random() < 0.5 else 1 for n in new]):
            if any(rows):
                both(p, rows)
        p.select([s if rng.random() < 0.7 else int(rng.choice([t for t in range(slots) if of[t] == of[s]])) for s in range(slots)])


@pytest.mark.parametrize("window,sinks,n", [(100, 0, 130), (300, 4, 290), (260, 40, 400), (64, 200, 420)])
def test_windows_that_reach_into_the_prompt(window, sinks, n):
    """Slots of one prompt whose windows, or first tokens, reach into it share it: there are nodes."""
    for group, dim, dtype in ((1, 64, "f16"), (6, 128, "bf16"), (30, 64, "f16")):
        p = Shared(6, 200, 16, 40, 2, dim, dtype, q_per_kv=group, window=window, sinks=sinks)
        forks(p, [n], [0] * 6)
        p.room([30, 2, 4, 16, 50, 9])
        for rows in ([1] * 6, [3, 2, 4, 1, 4, 1]):
            assert both(p, rows)
        p.select([4, 4, 0, 1, 2, 2])
        assert both(p, [1] * 6)


def test_many_slots_of_many_prompts():
    """More slots than a wave has lanes, lengths that rise, fall and repeat."""
    slots, prompts = 150, 12
    of = [s * prompts // slots for s in range(slots)]
    p = Shared(slots, 1500, 16, 40, 1, 64, "f16", q_per_kv=2, window=150, sinks=4)
    forks(p, [100 + 23 * (i % 5) for i in range(prompts)], of)
    p.room([1 + 13 * s % 61 for s in range(slots)])
    for rows in ([1] * slots, [s % 3 for s in range(slots)]):
        assert both(p, rows)


def test_the_same_call_gives_the_same_bits():
    p = Shared(12, 300, 16, 60, 2, 128, "bf16", q_per_kv=4, window=300, sinks=4)
    forks(p, [600, 500, 400], [0] * 4 + [1] * 5 + [2] * 3)
    p.room([1, 30, 2, 9, 1, 1, 20, 4, 2, 17, 3, 1])
    q = p.t.randn(12, 8, 128, device="cuda").bfloat16()
    start, outs, plans = p.ints(np.arange(13)), [], []
    for turn in range(8):
        p.sharing.fill_(-turn)
        p.own.share(start, 12, p.sharing, least_bytes=0)
        outs.append(p.t.full_like(q, 3.5))
        p.own.attend_shared(0, q, outs[-1], start, 1, p.sharing)
        plans.append(p.nodes()[1])
    assert all(p.t.equal(x, outs[0]) for x in outs) and all(x == plans[0] for x in plans)
