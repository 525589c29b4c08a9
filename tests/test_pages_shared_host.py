"""Host side of attention over shared pages: sizes and what is refused before anything is launched.  No GPU."""
import ctypes as C

import pytest

from paper_2402_09398_amd import binding
from tests.test_pages_host import A, B, SHAPES, desc


def calls(d, layer=0, stride=0, rows=8, q=A, start=B, plan=A, out=B, most=1):
    L, p = binding.lib(), C.byref(d)
    return (lambda: L.lessdec_pages_share(p, start, rows, -1, plan, None),
            lambda: L.lessdec_pages_attend_shared(p, layer, q, stride, out, None, start, rows, most, plan, None))


@pytest.mark.parametrize("bad", SHAPES, ids=lambda b: "-".join(f"{k}={v}" for k, v in b.items()))
def test_shapes_are_refused(bad):
    L, d = binding.lib(), desc(**bad)
    assert L.lessdec_pages_share_ints(C.byref(d), 8) == L.lessdec_pages_shared_workspace_bytes(C.byref(d), 8) == 0
    assert all(call() == binding.EINVAL for call in calls(d))


def test_arguments_are_refused():
    share, attend = range(2)
    for which, more in ((share, dict(start=None)), (share, dict(start=B + 1)), (share, dict(plan=None)), (share, dict(plan=A + 8)), (share, dict(plan=B)),
                        (share, dict(rows=-1)), (share, dict(rows=1 << 29)), (attend, dict(q=None)), (attend, dict(q=A + 8)), (attend, dict(out=None)),
                        (attend, dict(out=B + 4)), (attend, dict(start=None)), (attend, dict(plan=None)), (attend, dict(plan=A + 4)), (attend, dict(rows=-1)),
                        (attend, dict(rows=1 << 29)), (attend, dict(most=-1)), (attend, dict(layer=-1)), (attend, dict(layer=2)), (attend, dict(stride=12)),
                        (attend, dict(stride=8))):
        assert calls(desc(), **more)[which]() == binding.EINVAL, more
    for field in ("table", "length"):
        for value in (None, A + 1):
            assert all(call() == binding.EINVAL for call in calls(desc(**{field: value}), plan=B + 64))
    for field in ("k_codes", "v_codes", "exps"):
        assert calls(desc(**{field: None}))[1]() == binding.EINVAL
    big = dict(slots=4096, heads=1024, pages=1 << 20, table_len=1 << 25, page_tokens=16)      # 2^31 tiles
    assert all(call() == binding.EINVAL for call in calls(desc(**big), rows=4096, plan=B + 64))
    d = desc()
    less = binding.lib().lessdec_pages_shared_workspace_bytes(C.byref(d), 8) - 1
    for more in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=less)):
        assert calls(desc(**more))[1]() == binding.EWORKSPACE, more


def test_nothing_to_do_needs_no_pointers():
    L, p = binding.lib(), C.byref(desc(workspace=None))
    assert L.lessdec_pages_share(p, None, 0, 0, None, None) == binding.OK
    assert L.lessdec_pages_attend_shared(p, 0, None, 0, None, None, None, 0, 1, None, None) == binding.OK
    assert L.lessdec_pages_attend_shared(p, 0, None, 0, None, None, None, 8, 0, None, None) == binding.OK


@pytest.mark.parametrize("shape", [dict(), dict(heads=1, q_per_kv=71, head_dim=64), dict(slots=4096), dict(table_len=1), dict(heads=40, q_per_kv=1),
                                   dict(heads=1024, pages=512), dict(slots=1), dict(pages=1 << 22)])
def test_sizes_never_fall(shape):
    L, d = binding.lib(), desc(**shape)
    rows = [0, 1, 2, 3, 7, 8, 64, 65, 500, 4096, 5000, 1 << 16, 1 << 20, 1 << 24]
    ints = [L.lessdec_pages_share_ints(C.byref(d), n) for n in rows]
    work = [L.lessdec_pages_shared_workspace_bytes(C.byref(d), n) for n in rows]
    assert all(a <= b for a, b in zip(ints, ints[1:])) and all(a <= b for a, b in zip(work, work[1:]))
    assert all(w >= L.lessdec_pages_workspace_bytes(C.byref(d), n) and w % 256 == 0 for w, n in zip(work, rows))
    assert all(x >= n for x, n in zip(ints, rows)) and L.lessdec_pages_share_ints(C.byref(d), -1) == 0
