"""ctypes front end of the choice of beams (include/lessdec.h, "Beams"): argument marshalling only.

Everything runs in the HIP kernels; torch is used for device memory and streams.
"""
from __future__ import annotations

import ctypes as C

from .binding import DTYPE_BF16, DTYPE_F16, DTYPE_F32, BeamDesc, LessdecError, _check, _p, _stream, lib


def lessdec_beam_workspace_bytes(desc: BeamDesc) -> int:
    return int(lib().lessdec_beam_workspace_bytes(C.byref(desc)))


def lessdec_beam_select(desc: BeamDesc, logits, row_stride: int, score, ended, parent, token, next_score, next_ended, stream=None):
    _check(lib().lessdec_beam_select(C.byref(desc), _p(logits), row_stride, _p(score), _p(ended), _p(parent), _p(token), _p(next_score),
                                     _p(next_ended), _stream(stream)), "lessdec_beam_select")


class BeamSearch:
    """Owns the scratch of the choice of beams for `groups` prompts of `beams` beams each, and its descriptor.

    Plumbing only: allocation with torch, checks of tensors, pointer marshalling, no arithmetic.  dtype: "f32", "f16" or "bf16", of the
    logits.  picks: how many are chosen for each prompt (beams if none is given).  Calls run on its device, on the current stream if
    none is given, one at a time.
    """

    def __init__(self, groups, beams, vocab, dtype, picks=None, end_token=-1, device="cuda:0"):
        import torch
        if not torch.cuda.is_available():
            raise LessdecError("no GPU visible: lessdec has no CPU path")
        types = {"f32": (torch.float32, DTYPE_F32), "f16": (torch.float16, DTYPE_F16), "bf16": (torch.bfloat16, DTYPE_BF16)}
        if dtype not in types:
            raise LessdecError("BeamSearch: dtype is 'f32', 'f16' or 'bf16'")
        lib()
        self.torch = torch
        self.device = torch.device(device)
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.groups, self.beams, self.vocab, self.picks = groups, beams, vocab, beams if picks is None else picks
        self.tdtype = types[dtype][0]
        d = BeamDesc()
        d.groups, d.beams, d.vocab, d.picks, d.dtype, d.end_token = groups, beams, vocab, self.picks, types[dtype][1], end_token
        need = lessdec_beam_workspace_bytes(d)
        if need == 0:
            raise LessdecError("lessdec_beam_workspace_bytes: invalid shape")
        self.workspace = torch.zeros(need, dtype=torch.uint8, device=self.device)   # (zeros: lessdec.h)
        d.workspace, d.workspace_bytes = self.workspace.data_ptr(), need
        self.desc = d
        self._bools = (torch.uint8, torch.bool)
        self._pointer, self._lib, self._current = C.pointer(d), lib(), (torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice)

    def _flat(self, t, count, types, what):
        if t.dtype not in types or t.numel() != count or not t.is_contiguous() or t.device != self.device:
            raise LessdecError(f"select: {what} must be {count} contiguous {types[0]} on {self.device}")
        return t.data_ptr()

    def select(self, logits, score, ended, parent, token, next_score, next_ended=None, stream=None):
        """logits [groups * beams, vocab], rows may lie apart; score fp32 and ended (uint8 or bool, or None) [groups * beams]; parent and token
        int32, next_score fp32 and next_ended (uint8 or bool, or None) [groups * picks].  With picks = beams, next_score may be score and
        next_ended may be ended."""
        rows, n, torch = self.groups * self.beams, self.groups * self.picks, self.torch
        if logits.dtype != self.tdtype or logits.device != self.device or tuple(logits.shape) != (rows, self.vocab) or \
                (logits.stride(1) != 1 and self.vocab > 1) or (rows > 1 and logits.stride(0) < self.vocab):
            raise LessdecError(f"select: logits must be [{rows}, {self.vocab}] {self.tdtype} on {self.device}, rows that do not overlap")
        args = (logits.data_ptr(), logits.stride(0) if rows > 1 else 0, self._flat(score, rows, (torch.float32,), "score"),
                None if ended is None else self._flat(ended, rows, self._bools, "ended"),
                self._flat(parent, n, (torch.int32,), "parent"), self._flat(token, n, (torch.int32,), "token"),
                self._flat(next_score, n, (torch.float32,), "next_score"),
                None if next_ended is None else self._flat(next_ended, n, self._bools, "next_ended"))
        raw_stream, device = self._current
        s = raw_stream(self.device.index) if stream is None else stream.cuda_stream
        if device() == self.device.index:
            rc = self._lib.lessdec_beam_select(self._pointer, *args, s)
        else:
            with torch.cuda.device(self.device):
                rc = self._lib.lessdec_beam_select(self._pointer, *args, s)
        if rc:
            _check(rc, "lessdec_beam_select")
