"""Host side of the choice of beams: the descriptor's layout, sizes, refusals, and the oracle's own order.  No GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2402_09398_amd import binding
from paper_2402_09398_amd.binding import BeamDesc
from tests import beams_oracle as bo

A, B = 0x10000, 0x20000                                       # stand for device pointers: no call below gets as far as reading them


def desc(**more):
    d = BeamDesc()
    d.groups, d.beams, d.vocab, d.picks, d.dtype, d.end_token = 3, 4, 1000, 4, binding.DTYPE_F16, 2
    d.workspace, d.workspace_bytes = A, 1 << 40
    for k, v in more.items():
        setattr(d, k, v)
    return d


def call(d, logits=A, stride=0, score=A, ended=A, parent=A, token=B, next_score=B, next_ended=B):
    return binding.lib().lessdec_beam_select(C.byref(d), logits, stride, score, ended, parent, token, next_score, next_ended, None)


def test_descriptor_layout():
    assert C.sizeof(BeamDesc) == 6 * 4 + 2 * 8 and BeamDesc.workspace.offset == 24


@pytest.mark.parametrize("bad", [dict(groups=0), dict(beams=0), dict(beams=65), dict(groups=1 << 18, beams=5), dict(vocab=0), dict(vocab=(1 << 28) + 1), dict(picks=0),
                                 dict(picks=65), dict(dtype=3), dict(dtype=-1), dict(end_token=-2), dict(end_token=1000)],
                         ids=lambda b: "-".join(f"{k}={v}" for k, v in b.items()))
def test_shapes_are_refused(bad):
    assert binding.lib().lessdec_beam_workspace_bytes(C.byref(desc(**bad))) == 0
    assert call(desc(**bad)) == binding.EINVAL


def test_arguments_are_refused():
    assert binding.lib().lessdec_beam_select(None, A, 0, A, A, A, B, B, B, None) == binding.EINVAL
    for more in (dict(logits=None), dict(logits=A + 1), dict(score=None), dict(score=A + 2), dict(parent=None), dict(parent=A + 1), dict(token=None),
                 dict(token=A), dict(token=B + 2), dict(next_score=None), dict(next_score=B + 1), dict(stride=999), dict(stride=-1), dict(stride=1 << 41)):
        assert call(desc(), **more) == binding.EINVAL, more
    assert call(desc(dtype=binding.DTYPE_F32), logits=A + 2) == binding.EINVAL
    assert call(desc(end_token=-1)) == binding.EINVAL                                  # ended beams without a token
    assert call(desc(picks=5), next_score=A) == call(desc(picks=5), next_ended=A) == binding.EINVAL
    for more in (dict(workspace=None), dict(workspace=A + 128), dict(workspace_bytes=binding.lib().lessdec_beam_workspace_bytes(C.byref(desc())) - 1)):
        assert call(desc(**more)) == binding.EWORKSPACE, more


@pytest.mark.parametrize("groups,beams,vocab,picks", [(1, 1, 1, 1), (1, 4, 32000, 4), (64, 4, 128256, 8), (16384, 64, 50257, 64), (1, 1, 1 << 28, 64)])
def test_sizes(groups, beams, vocab, picks):
    rows = groups * beams
    n = binding.lib().lessdec_beam_workspace_bytes(C.byref(desc(groups=groups, beams=beams, vocab=vocab, picks=picks, end_token=-1)))
    assert rows * (4 + 16 + 8 * picks + 12 * picks) <= n <= rows * 64 * (28 + 24 * picks) + 1280


def test_the_oracles_order():
    x = np.array([[1.0, 3, 3, -np.inf], [0, 0, 0, 0], [9, 9, 9, np.nan], [1, 3, 3, -np.inf]])
    parent, token, c, ended = bo.select(x, np.array([-1.0, -5, 0, -1]), None, 1, 4, 6, 1)
    assert parent.tolist() == [[0, 0, 3, 3, 0, 3]] and token.tolist() == [[1, 2, 1, 2, 0, 0]] and ended.tolist() == [[True, False, True, False, False, False]]
    parent, token, c, ended = bo.select(x[1:3], np.array([-np.inf, -2.0]), np.array([0, 1]), 1, 2, 3, 1)
    assert parent.tolist() == [[1, -1, -1]] and token.tolist() == [[1, -1, -1]] and c.tolist() == [[-2.0, -np.inf, -np.inf]]
