"""Beam search over both kinds of cache as a program runs it, each step's calls one behind the other: the choice of beams, the pages and the
eviction states that follow the parents, a page of their own where beams part, the step itself with what beams share read once."""
import numpy as np
import pytest

from tests import beams_oracle as bo
from tests.test_gpu_pages import HALF_STEP
from tests.test_gpu_pages_shared import Shared
from tests.test_gpu_states import layer

pytestmark = pytest.mark.gpu


class Decoder:
    """A layer of paged attention and one with eviction, side by side; the attention's output, and a table by token, are the next logits."""

    def __init__(self, groups, beams, heads, group, page, prompts, steps, seed=0):
        import torch
        from paper_2402_09398_amd import BeamSearch
        self.torch, self.groups, self.beams, self.heads, self.group = torch, groups, beams, heads, group
        slots = self.slots = groups * beams
        vocab = self.vocab = heads * group * 64
        room = max(prompts) + steps + 1
        self.pages = Shared(slots, slots * (2 + -(-steps // page)) + sum(-(-n // page) + 1 for n in prompts), page, -(-room // page), heads, 64, "f16", seed=seed,
                            q_per_kv=group)
        n = [0] * slots
        n[::beams] = prompts
        self.pages.room(n)
        self.pages.select([s // beams * beams for s in range(slots)])
        self.lines, g = layer(slots, heads, 64, 3, 4, 5, seed=seed, group=group)
        self.lines.state_reset()
        self.search = BeamSearch(groups, beams, vocab, "f16", end_token=7)
        table = lambda *shape: torch.randn(vocab, *shape, generator=g, device="cuda").half()  # noqa: E731
        self.q_of, self.k_of, self.v_of, self.logits_of = table(heads * group, 64), table(heads, 64), table(heads, 64), table(vocab)
        ints = lambda *shape: torch.zeros(*shape, dtype=torch.int32, device="cuda")  # noqa: E731
        self.parent, self.token, self.plan = ints(slots), ints(slots), ints(1 + 2 * slots)
        self.one, self.start = self.pages.ints([1] * slots), self.pages.ints(np.arange(slots + 1))
        self.score = torch.full((slots,), -float("inf"), device="cuda")
        self.score[::beams] = 0
        self.ended = torch.zeros(slots, dtype=torch.uint8, device="cuda")
        self.out = torch.zeros(slots, heads * group, 64, dtype=torch.float16, device="cuda")
        self.evicted = torch.zeros(slots * heads, group, 64, dtype=torch.float16, device="cuda")
        self.logits = self.logits_of[torch.arange(slots, device="cuda") % vocab].contiguous()

    def choose(self):
        self.search.select(self.logits, self.score, self.ended, self.parent, self.token, self.score, self.ended)
        own = self.pages.own
        own.select(self.parent)
        own.reserve(self.one, None, self.plan)
        own.copy(self.plan, self.slots)
        self.lines.state_select(self.parent)

    def step(self):
        torch, own = self.torch, self.pages.own
        token = self.token.clamp_min(0).long()
        self.q, self.k, self.v = (x.index_select(0, token) for x in (self.q_of, self.k_of, self.v_of))
        own.share(self.start, self.slots, self.pages.sharing, least_bytes=0)
        own.append(0, self.k, self.v, self.start)
        own.attend_shared(0, self.q, self.out, self.start, 1, self.pages.sharing)
        units = self.slots * self.heads
        self.lines.step(self.q.view(units, self.group, 64), self.k.view(units, 64), self.v.view(units, 64), self.evicted)
        torch.add(self.out.view(self.slots, self.vocab) * 2, self.logits_of.index_select(0, token), out=self.logits)

    def buffers(self):
        return [getattr(self, n) for n in ("score", "ended", "parent", "token", "out", "evicted", "logits")] + \
               [getattr(self.lines, n) for n in self.lines.STATE] + [getattr(self.pages.own, n) for n in self.pages.own.STATE]


SHAPES = [(3, 4, 2, 2, 16, [70, 33, 5]), (2, 5, 1, 8, 32, [150, 1]), (5, 2, 2, 1, 16, [16, 17, 64, 3, 100]), (1, 30, 1, 3, 16, [200])]


@pytest.mark.parametrize("groups,beams,heads,group,page,prompts", SHAPES)
def test_against_the_oracles(groups, beams, heads, group, page, prompts):
    """Every step's choice, tables and outputs; at the end, the eviction states give what decoders give that had each beam's tokens alone.  One
    group's rows turn into NaN on the way: its beams come to nothing."""
    import torch
    steps = 14
    d = Decoder(groups, beams, heads, group, page, prompts, steps)
    ref, slots = d.pages.ref, d.slots
    history = [[] for _ in range(slots)]
    start = np.arange(slots + 1)
    lost = range((groups - 1) * beams, slots) if groups > 1 else range(0)
    for i in range(steps):
        if i == 9:
            d.logits[list(lost)] = float("nan")
        x, score, ended = d.logits.double().cpu().numpy(), d.score.double().cpu().numpy(), d.ended.cpu().numpy()
        want = bo.select(x, score, ended, groups, beams, beams, 7)
        d.choose()
        parent, token, best = (t.cpu().numpy() for t in (d.parent, d.token, d.score.double()))
        np.testing.assert_array_equal(parent, want[0].ravel())
        np.testing.assert_array_equal(token, want[1].ravel())
        there = parent >= 0
        assert (best[~there] == -np.inf).all() and there.any() and (i < 9 or not there[list(lost)].any())
        assert (np.abs(best[there] - want[2].ravel()[there]) <= np.abs(want[2].ravel()[there]) * 2.0 ** -24 + 1e-11).all()
        np.testing.assert_array_equal(d.ended.cpu().numpy(), want[3].ravel())
        history = [(history[p] if p >= 0 else []) + [max(int(t), 0)] for p, t in zip(parent, token)]
        ref.select(parent.tolist())
        granted, pairs = ref.reserve([1] * slots)
        assert (granted == 1).all()
        ref.copy(pairs)
        d.pages.state()
        d.step()
        ref.append(0, d.k.double().cpu().numpy(), d.v.double().cpu().numpy(), start)
        want, _, tol, _ = ref.attend(0, d.q.double().cpu().numpy(), start, HALF_STEP["f16"])
        assert (np.abs(d.out.double().cpu().numpy() - want) <= tol).all()
        d.pages.share([1] * slots, behind=0)
    lengths = {len(h) for h in history}
    assert steps in lengths and lengths <= {1, steps}
    for n in lengths:
        alone, _ = layer(slots, heads, 64, 3, 4, 5, group=group)
        alone.state_reset()
        units, out = slots * heads, torch.empty_like(d.evicted)
        rows = [b for b in range(slots) if len(history[b]) == n]
        for j in range(n):
            token = torch.tensor([h[j] if len(h) == n else 0 for h in history]).cuda()
            alone.step(d.q_of[token].view(units, group, 64), d.k_of[token].view(units, 64), d.v_of[token].view(units, 64), out)
        assert torch.equal(out.view(slots, -1)[rows], d.evicted.view(slots, -1)[rows])


def test_a_captured_step():
    """A graph of the choice and the step, replayed, an eager step among the replays, gives to the bit what eager steps give."""
    import torch
    for shape in ((3, 4, 2, 2, 16, [70, 33, 5]), (2, 8, 1, 5, 16, [300, 40])):
        d = Decoder(*shape, steps=20)

        def step():
            d.choose()
            d.step()
        step()                                                # (what a first call sets up)
        torch.cuda.synchronize()
        was = [x.clone() for x in d.buffers()]
        eager = []
        for _ in range(8):
            step()
            eager.append([x.clone() for x in d.buffers()])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for _ in range(2):
            for x, y in zip(d.buffers(), was):
                x.copy_(y)
            for i, want in enumerate(eager):
                (step if i == 3 else graph.replay)()
                torch.cuda.synchronize()
                for x, y in zip(d.buffers(), want):
                    assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i
