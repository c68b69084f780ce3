"""Thin PyTorch binding of the beam search's selection (ewsjf_beam_select in
include/ewsjf.h).  A step of a search whose beams hold their tokens in a paged
cache, `slot` their slots, [groups * beams]:

    parent, token, score = beam.beam_select(logits, score, beams, done=done, end=end)  # [groups][beams]
    granted = cache.reorder(slot, parent.flatten())  # each slot takes over its parent's tokens
    granted = cache.extend(slot, ones)               # room for `token`, which the next step appends

Nothing here synchronizes the host.
"""
from __future__ import annotations

import functools

import torch

from . import _lib as L
from .ewsjf import Workspace, _need, _stream
from .kv import _addr, _new, _scratch

_DTYPES = {torch.bfloat16: L.BF16, torch.float16: L.F16, torch.float32: L.F32}
_TYPES = (("parent", torch.int32), ("token", torch.int32), ("score", torch.float32))


@functools.lru_cache(maxsize=64)
def _sizes(*sizes):
    """The struct of a selection of these sizes, and its workspace's bytes."""
    b = L.Beams(*sizes)
    return b, int(L.lib().ewsjf_beam_workspace_bytes(_addr(b)))


def beam_select(logits: torch.Tensor, score: torch.Tensor, beams: int, picks: int | None = None, *,
                done: torch.Tensor | None = None, end: int = 0, out=None, ws: Workspace | None = None, stream=None):
    """The `picks` (default: beams) best next tokens of each group of `beams`
    rows: (parent, token, score), int32, int32 and float32 [groups][picks].

    logits: bfloat16, float16 or float32 [groups * beams][vocab], rows any
    stride apart.  score: float32 [groups * beams], the sums of log
    probabilities so far, -inf for a beam that is not there.  done: int32
    [groups * beams], a beam that is not 0 goes on by the token `end` alone, at no
    cost.  parent is the row that a pick continues, as PagedCache.reorder takes
    it; -1, token -1 and score -inf where there are no more candidates.  out: the
    three tensors to write."""
    if not isinstance(logits, torch.Tensor) or logits.dtype not in _DTYPES or not logits.is_cuda or logits.dim() != 2 \
            or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise TypeError("logits must be a CUDA tensor [groups * beams][vocab] of bfloat16, float16 or float32 with "
                        "contiguous rows")
    rows, vocab = logits.shape
    if beams < 1 or rows % beams:
        raise ValueError("logits has groups * beams rows")
    groups, picks = rows // beams, beams if picks is None else int(picks)
    if _need(score, torch.float32, "score").numel() != rows or score.device != logits.device:
        raise ValueError("score has one entry per row, on the logits' device")
    if done is not None and (_need(done, torch.int32, "done").numel() != rows or done.device != logits.device):
        raise ValueError("done has one entry per row, on the logits' device")
    b, nbytes = _sizes(groups, beams, picks, vocab, _DTYPES[logits.dtype], int(end),
                       logits.stride(0) if rows > 1 else vocab)
    if nbytes == 0:
        raise ValueError("a selection of these sizes or strides is not supported (see ewsjf_beam_select)")
    if out is None:
        parent, token, bits = _new(stream, (3, groups, picks), dtype=torch.int32, device=logits.device).unbind(0)
        out = parent, token, bits.view(torch.float32)
    else:
        for t, (name, kind) in zip(out, _TYPES):
            if _need(t, kind, name).shape != (groups, picks) or t.device != logits.device:
                raise ValueError(f"{name} is [groups][picks] on the logits' device")
    parent, token, best = out
    raw = _stream(stream)
    if (torch._C._cuda_getDevice() if stream is None else stream.device.index) != logits.device.index:
        raise ValueError("the logits are on another device than the call's stream")
    buf = _scratch(ws, nbytes, logits.device, raw, stream)
    L.check(L.lib().ewsjf_beam_select(_addr(b), logits.data_ptr(), score.data_ptr(),
                                      None if done is None else done.data_ptr(), parent.data_ptr(), token.data_ptr(),
                                      best.data_ptr(), buf.data_ptr(), buf.numel(), raw), "ewsjf_beam_select")
    return out
