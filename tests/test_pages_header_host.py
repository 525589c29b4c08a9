"""The index arithmetic of the paged cache's kernels, run on the CPU: the functions' text as it stands in the sources, compiled for the host."""
import ctypes as C
import re
import subprocess

import numpy as np
import pytest

from tests.header_on_host import CSRC

SHIMS = """#include <algorithm>
#include <cstddef>
#define __device__
using std::min; using std::max;
static inline unsigned __umulhi(unsigned a, unsigned b) { return (unsigned)((unsigned long long)a * b >> 32); }
constexpr int kBlock = 16;
"""
GLUE = """
extern "C" {
Pages make(int page_tokens, int table_len, int heads, int pages, int sinks, int window, int *length) {
  Pages c = {};
  c.page_tokens = page_tokens; c.table_len = table_len; c.heads = heads; c.pages = pages; c.sinks = sinks; c.window = window; c.length = length;
  const unsigned per = (unsigned)(page_tokens / kBlock);
  c.inverse = per == 1 ? 0 : (unsigned)(((1ull << 32) + per - 1) / per);
  return c;
}
long wrong_entries(int page_tokens, const int *blocks, long n) {
  const Pages c = make(page_tokens, 0, 1, 1, 0, 0, nullptr);
  long wrong = 0;
  for (long i = 0; i < n; ++i) wrong += entry_of(c, blocks[i]) != blocks[i] / (page_tokens / kBlock);
  return wrong;
}
int length_of(int page_tokens, int table_len, int n) { return slot_length(make(page_tokens, table_len, 1, 1, 0, 0, &n), 0); }
void rows_of(const int *start, int s, int rows, int *to) { const Rows r = slot_rows(start, s, rows); to[0] = r.first; to[1] = r.count; }
int block_of(int page_tokens, int heads, int pages, int page, int head, int block) { return block_in(make(page_tokens, 0, heads, pages, 0, 0, nullptr), page, head, block); }
void span(int sinks, int window, int lo, int hi, int *to) {
  const Pages c = make(16, 1 << 26, 1, 1, sinks, window, nullptr);
  const Span s = span_of(c, lo, hi);
  to[0] = s.sinks; to[1] = s.window; to[2] = s.count; to[3] = inner_first(c, s, hi); to[4] = inner_last(s, lo);
}
int sees_it(int sinks, int window, int p, int token) { return sees(make(16, 1 << 26, 1, 1, sinks, window, nullptr), p, token); }
int all_see_it(int sinks, int window, int lo, int hi, int t0) { return all_see(make(16, 1 << 26, 1, 1, sinks, window, nullptr), lo, hi, t0); }
}
"""


def text(file, start):
    """From a line that begins so to the closing brace (or, of one line, its end)."""
    src = (CSRC / file).read_text()
    at = src.index("\n" + start) + 1
    line = src[at:src.index("\n", at)]
    if line.count("{") and line.count("{") == line.count("}"):
        return line + "\n"
    end = re.compile(r"\n};?\n").search(src, at)
    return src[at:end.end()]


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    parts = [("lessdec_pages.h", s) for s in ("struct Pages", "__device__ inline int page_blocks", "__device__ inline int slot_length", "struct Rows",
                                              "__device__ inline Rows slot_rows", "__device__ inline int entry_of", "__device__ inline int block_in")]
    parts += [("lessdec_pages_attend.hip", s) for s in ("struct Span", "__device__ inline Span span_of", "__device__ inline bool sees",
                                                       "__device__ inline bool all_see", "__device__ inline int inner_first",
                                                       "__device__ inline int inner_last")]
    d = tmp_path_factory.mktemp("host")
    (d / "f.cpp").write_text(SHIMS + "".join(text(*p) for p in parts) + GLUE)
    subprocess.run(["g++", "-std=c++17", "-O2", "-fPIC", "-shared", "-Wno-return-type-c-linkage", "-o", str(d / "f.so"), str(d / "f.cpp")], check=True)
    return C.CDLL(str(d / "f.so"))


def ints(x):
    return np.ascontiguousarray(x, np.int32)


def pointer(x):
    return x.ctypes.data_as(C.c_void_p)


@pytest.mark.parametrize("page_tokens", range(16, 1025, 16))
def test_the_table_entry_of_a_block(host, page_tokens):
    """Exact for the 2^26 blocks that a slot can have: around every multiple where it could go wrong, and at random."""
    per, r = page_tokens // 16, np.random.default_rng(page_tokens)
    edges = r.integers(0, 2 ** 26 // per, 20000) * per
    blocks = ints(np.clip(np.concatenate([edges, edges + per - 1, edges - 1, r.integers(0, 2 ** 26, 20000), np.arange(2000), 2 ** 26 - 1 - np.arange(2000)]), 0, 2 ** 26 - 1))
    host.wrong_entries.restype = C.c_long
    assert host.wrong_entries(page_tokens, pointer(blocks), C.c_long(len(blocks))) == 0


def test_lengths_rows_and_pages_stay_in_range(host):
    low, high = -2 ** 31, 2 ** 31 - 1
    for page, wide in ((16, 1), (48, 7), (1024, 2 ** 20), (16, 2 ** 26)):
        for n in (low, -1, 0, 1, page * wide - 1, page * wide, min(page * wide + 1, high), high):
            assert host.length_of(page, wide, n) == min(max(n, 0), page * wide)
    r, got = np.random.default_rng(1), ints([0, 0])
    values = [low, low + 1, -5, -1, 0, 1, 2, 17, 399, 400, 401, high - 1, high]
    for rows in (0, 1, 17, 400, high):
        for a in values:
            for b in values:
                host.rows_of(pointer(ints([a, b])), 0, rows, pointer(got))
                first, count = int(got[0]), int(got[1])
                assert 0 <= first <= rows and 0 <= count <= rows - first
                x, y = (min(max(v, 0), rows) for v in (a, b))
                assert (first, count) == (x, max(y - x, 0))
    for _ in range(3000):
        page, heads, pages = 16 * int(r.integers(1, 65)), int(r.integers(1, 41)), int(r.integers(1, 1000))
        for which in (low, -1, 0, int(r.integers(0, pages)), pages - 1, pages, high):
            head, block = int(r.integers(0, heads)), int(r.integers(0, 2 ** 26))
            at = host.block_of(page, heads, pages, which, head, block)
            assert at == ((which * heads + head) * (page // 16) + block % (page // 16) if 0 <= which < pages else -1)


def test_what_rows_see(host):
    """The list of blocks of rows lo .. hi holds every token that one of them sees, in order and once; which blocks, and which tiles of four, all of
    them see."""
    r, got = np.random.default_rng(2), ints([0] * 5)
    for turn in range(1500):
        hi = int(r.integers(-3, 400))
        lo = hi - int(r.integers(0, 60))
        window = int(r.choice([0, 1, 2, 15, 16, 17, 33, 100, 399, 2 ** 30]))
        sinks = int(r.choice([0, 1, 15, 16, 17, 40, 300, 2 ** 31 - 1]))
        host.span(sinks, window, lo, hi, pointer(got))
        first, at, count, inner, last = (int(x) for x in got)
        blocks = [i if i < first else i - first + at for i in range(count)]
        assert blocks == sorted(set(blocks)) and (not blocks or 0 <= blocks[0] and blocks[-1] <= hi // 16)
        for block in range(max(hi, 0) // 16 + 2):
            seen = [[token <= p and (window == 0 or token > p - window or token < sinks) for p in range(lo, hi + 1)] for token in range(16 * block, 16 * block + 16)]
            assert [[bool(host.sees_it(sinks, window, p, 16 * block + i)) for p in range(lo, hi + 1)] for i in range(16)] == seen
            assert block in blocks or not np.any(seen)
            if hi >= 0 and block in blocks:
                assert not host.all_see_it(sinks, window, lo, hi, 16 * block) or np.all(seen)
                tile = blocks.index(block) // 4
                assert not inner <= tile < last or np.all(seen)
