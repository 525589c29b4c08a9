"""How the plan of shared pages deals out its work, run on the CPU: the structures' text as it stands in the sources, compiled for the host.  Every tile
of every node goes to one worker, once; what is written has a place, and no two pieces have the same."""
import ctypes as C
import re
import subprocess

import numpy as np
import pytest

from tests.header_on_host import CSRC
from tests.test_pages_header_host import text

SHIMS = """#include <algorithm>
#define __device__
#define __host__
using std::min; using std::max;
constexpr int kBlock = 16;
struct Pages { int page_tokens, table_len, heads, pages, sinks, window; };
"""
GLUE = """
extern "C" {
int chunk_of(unsigned tiles, int part, int workers) { return Trunk::chunk_of(tiles, part, workers); }
long columns_of(int slots, int heads, int group, long rows) { return plan_columns(slots, heads, group, rows); }
int begin() { return kBegin; }
long units(int n, int columns, int chunk) { return Trunk{0, 1, chunk}.units(n, columns); }
// the workers' pieces, as (worker, unit of all, node, column, from, to, piece, only); nodes: first unit, tiles, columns
int deal(unsigned total, int workers, int chunk, int of_head, const int *nodes, int n, int *to) {
  const Trunk t{total, workers, chunk};
  int pieces = 0;
  for (int w = 0; w < workers; ++w)
    for (unsigned at = t.first(w), end = t.first(w + 1); at < end;) {
      const int head = at / of_head, in_head = at - head * of_head;
      int i = n - 1;
      while (nodes[3 * i] > in_head) --i;
      const Trunk::Dealt x = t.dealt(nodes[3 * i + 1], nodes[3 * i + 2], in_head - nodes[3 * i], end - at);
      const int row[9] = {w, head, i, x.column, x.from, x.to, x.piece, x.only, x.units};
      for (int k = 0; k < 9; ++k) to[9 * pieces + k] = row[k];
      ++pieces;
      if (x.units <= 0) return -1;
      at += x.units;
    }
  return pieces;
}
void cut(int sinks, int window, int lo, int hi, int first, int last, int *to, int *blocks) {
  const Pages c{16, 1 << 26, 1, 1, sinks, window};
  const Cut s(span_of(c, lo, hi), first, last);
  to[0] = s.count; to[1] = inner_first(c, s, hi); to[2] = inner_last(s, lo);
  for (int i = 0; i < s.count; ++i) blocks[i] = s.block(i);
}
int sees_it(int sinks, int window, int p, int token) { return sees(Pages{16, 1 << 26, 1, 1, sinks, window}, p, token); }
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    header = (CSRC / "lessdec_pages.h").read_text()
    constants = "".join(re.findall(r"^constexpr int (?:kFewColumns|kTrunkDepth|kTrunkTile|kSharedWorkers|kBegin) [^\n]*\n", header, re.M))
    parts = [text("lessdec_pages.h", "struct Trunk {"), text("lessdec_pages.h", "inline long plan_columns")]
    parts += [text("lessdec_pages_attend.hip", s) for s in ("struct Span", "struct Cut", "__device__ inline Span span_of", "__device__ inline bool sees")]
    attend = (CSRC / "lessdec_pages_attend.hip").read_text()
    for start in ("__device__ inline int inner_first(const Pages &c, const Cut", "__device__ inline int inner_last(const Cut"):
        parts.append(text("lessdec_pages_attend.hip", start))
    assert "struct Cut" in attend
    d = tmp_path_factory.mktemp("host")
    (d / "f.cpp").write_text(SHIMS + constants + "".join(parts) + GLUE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-o", str(d / "f.so"), str(d / "f.cpp")], check=True)
    lib = C.CDLL(str(d / "f.so"))
    lib.columns_of.restype = lib.units.restype = C.c_long
    return lib


def pointer(x):
    return x.ctypes.data_as(C.c_void_p)


def test_every_tile_goes_to_one_worker(host):
    rng = np.random.default_rng(1)
    for turn in range(400):
        heads, workers = int(rng.choice([1, 2, 5, 8, 32, 71])), int(rng.choice([8, 16, 64, 384, 480, 512]))
        n = int(rng.integers(1, 60))
        tiles = np.exp(rng.uniform(0, np.log(rng.choice([2, 9, 300, 4000])), n)).astype(int)
        tiles[rng.random(n) < 0.2] = 0
        columns = rng.integers(17, rng.choice([40, 127, 3000]), n)
        wide = -(-columns // 128)
        if not (tiles * wide).any():
            continue
        total = int((tiles * wide).sum()) * heads
        begun = total + int((wide * (tiles > 0)).sum()) * heads * host.begin()
        chunk = host.chunk_of(total, begun // workers, workers)
        assert chunk >= 1 and sum(-(-t // chunk) * w for t, w in zip(tiles, wide)) * heads <= 2 * workers + int((wide * (tiles > 0)).sum()) * heads
        first, at = [], 0
        for t, c in zip(tiles, columns):
            first.append(at)
            at += host.units(int(t), int(c), chunk)
        nodes = np.ascontiguousarray(np.stack([first, tiles, columns], 1), np.int32)
        out = np.zeros((200000, 9), np.int32)
        pieces = host.deal(C.c_uint(at * heads), workers, chunk, at, pointer(nodes), n, pointer(out))
        assert 0 < pieces < len(out)
        seen = [np.zeros((heads, w, t), int) for w, t in zip(wide, tiles)]
        places = {}
        for w, head, node, column, a, b, piece, only, units in out[:pieces].tolist():
            assert 0 <= head < heads and column % 128 == 0 and column < columns[node] and 0 <= a <= b <= tiles[node]
            if a == b:
                continue
            k = a // chunk
            assert (b - 1) // chunk == k and piece // 2 == k and piece % 2 == (a % chunk > 0) and (head, node, column, piece) not in places
            places[head, node, column, piece] = only
            assert only == (a == k * chunk and b == min((k + 1) * chunk, tiles[node]))
            seen[node][head, column // 128, a:b] += 1
        assert all((s == 1).all() for s in seen)
        for head, node, column, piece in places:              # a chunk is one piece that says so, or two
            other = (head, node, column, piece ^ 1)
            assert (other in places) != bool(places[head, node, column, piece])


def test_there_is_room_for_all_columns(host):
    """Rows in four nodes each, the most that there are; chunks as where workers have no whole ones."""
    rng = np.random.default_rng(2)
    for turn in range(400):
        heads, workers, slots = int(rng.choice([1, 2, 8, 32, 71])), int(rng.choice([8, 64, 480, 512])), int(rng.integers(2, 200))
        each = int(rng.integers(17, 128))
        nodes = []                                            # columns, tiles
        for level in range(4):
            cuts = [0, slots] if level == 0 else sorted({0, slots, *rng.integers(0, slots, rng.integers(0, slots)).tolist()}) if level < 3 else range(slots + 1)
            cuts = list(cuts)
            nodes += [((b - a) * each, int(np.exp(rng.uniform(0, np.log(rng.choice([2, 20, 2000])))))) for a, b in zip(cuts, cuts[1:])]
        wide = [-(-c // 128) for c, _ in nodes]
        total = sum(w * t for w, (_, t) in zip(wide, nodes)) * heads
        begun = total + sum(wide) * heads * host.begin()
        if begun >= 2 ** 31:
            continue
        chunk = host.chunk_of(total, begun // workers, workers)
        need = sum(2 * -(-t // chunk) * c for c, t in nodes)
        assert need <= host.columns_of(slots, heads, 1, C.c_long(slots * each))


def test_parts_of_a_list_of_blocks(host):
    rng = np.random.default_rng(3)
    got, blocks = np.zeros(3, np.int32), np.zeros(4096, np.int32)
    for turn in range(3000):
        window = int(rng.choice([0, 1, 15, 16, 100, 500]))
        sinks = int(rng.choice([0, 1, 16, 40, 200])) if window else 0
        hi = int(rng.integers(0, 1500))
        lo = max(hi - int(rng.integers(0, 200)), 0)
        first = int(rng.integers(0, 60))
        last = int(rng.choice([first + 4 * int(rng.integers(0, 20)), 1 << 30]))
        host.cut(sinks, window, lo, hi, first, last, pointer(got), pointer(blocks))
        there = blocks[:got[0]].tolist()
        assert there == sorted(set(there)) and all(first <= b < last for b in there)
        needed = [b for b in range(first, min(last, hi // 16 + 1)) if any(host.sees_it(sinks, window, p, t) for p in (lo, hi) for t in (16 * b, 16 * b + 15) if t <= p)
                  or 16 * b <= hi < 16 * b + 16]
        assert set(needed) <= set(there)
        for tile in range(got[1], got[2]):                    # what all rows see in full
            assert 4 * tile + 3 < len(there)
            for b in there[4 * tile:4 * tile + 4]:
                assert all(host.sees_it(sinks, window, p, t) for p in (lo, hi) for t in (16 * b, 16 * b + 15))
