"""Host side of the paged cache: calls that have nothing to do.  No GPU."""
import ctypes as C

from paper_2402_09398_amd import binding
from tests.test_pages_host import A, desc


def test_nothing_to_attend_to_needs_no_workspace():
    L = binding.lib()
    for more in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=0)):
        p = C.byref(desc(**more))
        assert L.lessdec_pages_attend(p, 0, None, 0, None, None, None, 0, 1, None) == binding.OK
        assert L.lessdec_pages_attend(p, 0, None, 0, None, None, None, 8, 0, None) == binding.OK
        assert L.lessdec_pages_attend(p, 0, A, 0, A, None, A, 8, 1, None) == binding.EWORKSPACE
        assert L.lessdec_pages_append(p, 0, None, None, 0, None, 0, None) == binding.OK
        for layer, stride, rows in ((2, 0, 0), (0, 12, 0), (0, 0, -1)):
            assert L.lessdec_pages_attend(p, layer, None, stride, None, None, None, rows, 1, None) == binding.EINVAL
