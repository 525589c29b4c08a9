"""Host side of the paged cache: the descriptor's layout, sizes of the workspace, and what is refused before anything is launched.  No GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2402_09398_amd import binding
from paper_2402_09398_amd.binding import PagesDesc
from tests import pages_oracle as po

A, B = 0x10000, 0x20000                                       # stand for device pointers: no call below gets as far as reading them


def desc(**more):
    d = PagesDesc()
    d.slots, d.pages, d.page_tokens, d.table_len, d.heads, d.head_dim, d.q_per_kv, d.layers, d.dtype = 4, 64, 32, 16, 8, 128, 4, 2, binding.DTYPE_F16
    for name in ("k_codes", "v_codes", "exps", "table", "length", "refs", "workspace"):
        setattr(d, name, A)
    d.workspace_bytes = 1 << 40
    for k, v in more.items():
        setattr(d, k, v)
    return d


def calls(d, layer=0, stride=0, rows=8, pointer=A, most=1):
    L, p = binding.lib(), C.byref(d)
    return {
        "reset": lambda: L.lessdec_pages_reset(p, None),
        "reserve": lambda: L.lessdec_pages_reserve(p, pointer, B, B + 0x1000, None),
        "select": lambda: L.lessdec_pages_select(p, pointer and pointer + 0x5000, None),
        "compact": lambda: L.lessdec_pages_compact(p, pointer, None),
        "copy": lambda: L.lessdec_pages_copy(p, pointer, most, None),
        "append": lambda: L.lessdec_pages_append(p, layer, pointer, B, stride, B, rows, None),
        "attend": lambda: L.lessdec_pages_attend(p, layer, pointer, stride, B, None, B, rows, most, None),
        "read": lambda: L.lessdec_pages_read(p, layer, pointer, most, 0, rows, B, B, None),
    }


def test_descriptor_layout():
    assert C.sizeof(PagesDesc) == 12 * 4 + 7 * 8 + 8 and PagesDesc.k_codes.offset == 48


SHAPES = [dict(slots=0), dict(slots=4097), dict(pages=0), dict(pages=1 << 28), dict(page_tokens=0), dict(page_tokens=24), dict(page_tokens=1040),
          dict(table_len=0), dict(table_len=1 << 26), dict(heads=0), dict(heads=1025), dict(head_dim=96), dict(head_dim=256), dict(q_per_kv=-1),
          dict(q_per_kv=129), dict(layers=0), dict(layers=1025), dict(dtype=binding.DTYPE_F32), dict(dtype=3), dict(sinks=-1), dict(window=-1),
          dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))]


@pytest.mark.parametrize("bad", SHAPES, ids=lambda b: "-".join(f"{k}={v}" for k, v in b.items()))
def test_shapes_are_refused(bad):
    d = desc(**bad)
    assert binding.lib().lessdec_pages_workspace_bytes(C.byref(d), 8) == 0
    for name, call in calls(d).items():
        assert call() == binding.EINVAL, name


def test_pointers_are_refused():
    for field, needs in (("table", "reset reserve select compact append attend read"), ("length", "reset reserve select compact append attend read"),
                         ("refs", "reset reserve select compact"), ("k_codes", "copy append attend read"), ("v_codes", "copy append attend read"),
                         ("exps", "copy append attend read")):
        for value in (None, A + 1):
            got = calls(desc(**{field: value}))
            for name in needs.split():
                assert got[name]() == binding.EINVAL, (field, value, name)
    for value in (None, A + 2):
        for name, call in calls(desc(), pointer=value).items():
            if name != "reset":
                assert call() == binding.EINVAL, (name, value)
    for more in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=64)):
        got = calls(desc(**more))
        for name in ("reserve", "compact", "attend"):
            assert got[name]() == binding.EWORKSPACE, (more, name)
    L, d = binding.lib(), desc()
    assert L.lessdec_pages_reserve(C.byref(d), A, A, B, None) == binding.EINVAL            # granted is n_new
    assert L.lessdec_pages_reserve(C.byref(d), A, B, B, None) == binding.EINVAL
    assert L.lessdec_pages_select(C.byref(d), d.length, None) == binding.EINVAL
    assert binding.lib().lessdec_pages_reset(None, None) == binding.EINVAL


def test_sizes_are_refused():
    for more in (dict(layer=-1), dict(layer=2), dict(rows=-1), dict(stride=512), dict(stride=8 * 128 + 4), dict(stride=-8)):
        got = calls(desc(q_per_kv=1), **more)
        for name in ("append", "attend") + (("read",) if "stride" not in more else ()):
            assert got[name]() == binding.EINVAL, (more, name)
    assert calls(desc(), most=-1)["copy"]() == binding.EINVAL and calls(desc(), most=-1)["attend"]() == binding.EINVAL
    assert calls(desc(), most=65536)["read"]() == binding.EINVAL
    # nothing to do: nothing is launched (there is no GPU here)
    assert calls(desc(), rows=0)["append"]() == calls(desc(), rows=0)["attend"]() == calls(desc(), most=0)["attend"]() == binding.OK
    assert calls(desc(), most=0)["copy"]() == calls(desc(), most=0)["read"]() == calls(desc(), rows=0)["read"]() == binding.OK


@pytest.mark.parametrize("shape", [dict(), dict(heads=1, q_per_kv=71, head_dim=64), dict(slots=600), dict(table_len=1), dict(heads=40, q_per_kv=1),
                                   dict(pages=1 << 22)])
def test_the_workspace_never_falls(shape):
    d, f = desc(**shape), binding.lib().lessdec_pages_workspace_bytes
    sizes = [f(C.byref(d), n) for n in list(range(0, 3000, 7)) + [1 << 14, 1 << 18, 1 << 24]]
    assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] >= 4 * d.pages and sizes[-1] < 1 << 28
    assert all(x % 256 == 0 for x in sizes)
    d.workspace_bytes = sizes[-1] - 256
    assert binding.lib().lessdec_pages_attend(C.byref(d), 0, A, 0, B, None, B, 1 << 24 if d.heads == 1 else 1 << 18, 1, None) in \
        (binding.EWORKSPACE, binding.EINVAL)


def test_the_oracle_rounds_to_the_nearest_code():
    """Against torch's conversion where that is defined (up to 448), and the ends."""
    import torch
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.standard_normal(20000) * 60, rng.standard_normal(20000) * 0.01, po._HALVES, -po._HALVES, po._POSITIVE])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.tensor(x).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(po.nearest(x.astype(np.float64), 0), want)
    assert np.isnan(po.nearest(np.array([np.inf, -np.inf, np.nan]), 3)).all()
    assert po.nearest(np.array([1e30]), 40) == 448 * 2.0 ** 40
    assert [po.exponent(np.array([v])) for v in (0.0, 448.0, 448.1, 1.75, 1e-30, 1e30, np.inf)] == [-40, 0, 1, -8, -40, 40, -40]


def test_the_oracles_bookkeeping():
    """A fork shares its pages; of two that write into a shared page the first gets a copy; compacting fills the holes from behind."""
    c = po.Cache(4, 8, 16, 4, 1, 64)
    assert c.reserve([20, 0, 0, 3])[1] == []
    assert c.table[0].tolist() == [0, 1, -1, -1] and c.table[3].tolist() == [2, -1, -1, -1]
    c.select([0, 0, 0, -1])
    assert c.refs.tolist() == [3, 3, 0, 0, 0, 0, 0, 0]
    granted, plan = c.reserve([1, 1, 0, 0])
    assert granted.tolist() == [1, 1, 0, 0] and plan == [(1, 2), (1, 3)] and c.refs.tolist() == [3, 1, 1, 1, 0, 0, 0, 0]
    c.select([-1, 1, -1, -1])
    assert c.refs.tolist() == [1, 0, 0, 1, 0, 0, 0, 0] and c.compact() == [(3, 1)] and c.table[1].tolist() == [0, 1, -1, -1]
    assert c.reserve([16 * 5, 1, 0, 0])[0].tolist() == [0, 1, 0, 0]     # five pages: more than a table row holds
    assert c.reserve([16 * 4, 16, 64, 1])[0].tolist() == [64, 16, 0, 0] # two pages are left: the third gets none, nor does the last


def test_nothing_to_do_needs_no_pointers():
    """An empty tensor has no address."""
    L, p = binding.lib(), C.byref(desc())
    assert L.lessdec_pages_append(p, 0, None, None, 0, None, 0, None) == binding.OK
    assert L.lessdec_pages_attend(p, 0, None, 0, None, None, None, 0, 1, None) == binding.OK
    assert L.lessdec_pages_read(p, 0, None, 0, 0, 5, None, None, None) == L.lessdec_pages_read(p, 0, A, 1, 0, 0, None, None, None) == binding.OK
    for layer, stride, rows in ((2, 0, 0), (0, 12, 0), (0, 0, -1)):
        assert L.lessdec_pages_append(p, layer, None, None, stride, None, rows, None) == binding.EINVAL
        assert L.lessdec_pages_attend(p, layer, None, stride, None, None, None, rows, 1, None) == binding.EINVAL
    assert L.lessdec_pages_attend(p, 0, A, 0, B, None, B, 1 << 29, 1, None) == binding.EINVAL           # 2^31 query columns
