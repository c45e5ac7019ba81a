"""Rotary positions of queries and keys, before they are scored, compacted or decoded: one dkv_rotate call, prompts and single tokens.

    rotary = Rotary(128, base=500000.0, scaling=dict(kind="bands", factor=8.0, original=8192, low=1.0, high=4.0))
    rotary.rotate(positions, q, k)          # in place; positions int32 [n_seqs][n_tokens], q [n_seqs][n_tokens][Hq][d], k [..][Hkv][d]

q and k are views of any strides: a prompt's keys kept by head, [n_seqs][Hkv][n_tokens][d], go in as k.transpose(1, 2).
"""
from __future__ import annotations

import numpy as np
import torch

from . import dkv

_KINDS = {"linear": dkv.DKV_ROTARY_LINEAR, "bands": dkv.DKV_ROTARY_BANDS, "ramp": dkv.DKV_ROTARY_RAMP}
_DTYPES = {dkv.DKV_BF16: torch.bfloat16, dkv.DKV_F32: torch.float32}
_current_device = getattr(torch._C, "_cuda_getDevice", None)        # what torch.cuda.current_device() asks, without its start-up


class Rotary:
    """head_dim: elements of a head; the first rot_dim of them (all, if None) are rotated, as pairs (i, i + rot_dim / 2) or, if
    interleaved, (2 i, 2 i + 1). scaling: None, or a dict with "kind" ("linear", "bands", "ramp") and that kind's numbers ("factor",
    "original", "low", "high"), as include/dkv.h defines them."""

    def __init__(self, head_dim, rot_dim=None, base=10000.0, interleaved=False, scaling=None, dtype=dkv.DKV_BF16, device="cuda"):
        rot_dim = head_dim if rot_dim is None else rot_dim
        given = dict(scaling or {})
        kind = given.pop("kind", None)
        if kind is None and not given:
            given["scaling"] = dkv.DKV_ROTARY_PLAIN
        elif kind in _KINDS:
            given["scaling"] = _KINDS[kind]
        else:
            raise ValueError("scaling is None or a dict with a kind of %s: got %r" % (", ".join(sorted(_KINDS)), scaling))
        if not 1 <= head_dim <= 1024 or not 0 <= rot_dim <= head_dim:
            raise ValueError("head_dim is 1 to 1024 and rot_dim at most head_dim: got %r, %r" % (head_dim, rot_dim))
        turns, factor = dkv.dkv_rotary_turns(rot_dim, base, **given)
        self.tdtype = _DTYPES[dtype]
        self.turns = torch.from_numpy(np.array(turns, dtype=np.uint64).view(np.int64)).to(device)
        self.device = self.turns.device
        self._index = -1 if self.device.type != "cuda" else self.device.index
        self._head = head_dim
        self.desc = dkv.dkv_rotary(head_dim, rot_dim, int(bool(interleaved)), dtype, factor, self.turns.data_ptr() if rot_dim else None)

    def _refuse(self, x, n_seqs, n_tokens, name):
        if x.requires_grad and torch.is_grad_enabled():
            raise ValueError("%s requires a gradient, which autograd does not record here: rotate under torch.no_grad(), the gradient with -positions"
                             % name)
        if x.dtype is not self.tdtype or x.get_device() != self._index:
            raise ValueError("%s: %s on %s is required, got %s on %s" % (name, self.tdtype, self.device, x.dtype, x.device))
        if len(x.shape) != 4 or x.shape[:2] != (n_seqs, n_tokens) or x.shape[3] != self._head:
            raise ValueError("%s: [%d][%d][heads][%d] is required, got %s" % (name, n_seqs, n_tokens, self._head, list(x.shape)))
        raise ValueError("%s: the elements of a head lie side by side" % name)

    def _pair(self, x, out, n_seqs, n_tokens, name):
        """(heads, x, out, their strides) of tensors that fit."""
        shape, strides = x.shape, x.stride()
        if len(shape) != 4:
            self._refuse(x, n_seqs, n_tokens, name)
        a, b, heads, d = shape
        seq, token, head, element = strides
        if a != n_seqs or b != n_tokens or d != self._head or (element != 1 and d > 1) or x.dtype is not self.tdtype or \
                x.get_device() != self._index or (x.requires_grad and torch.is_grad_enabled()):
            self._refuse(x, n_seqs, n_tokens, name)
        if out is None or out is x:
            return heads, x, x, (seq, token, head), (seq, token, head)
        if out.shape != shape:
            raise ValueError("%s_out has the shape of %s" % (name, name))
        out_seq, out_token, out_head, element = out.stride()
        if (element != 1 and d > 1) or out.dtype is not self.tdtype or out.get_device() != self._index or \
                (out.requires_grad and torch.is_grad_enabled()):
            self._refuse(out, n_seqs, n_tokens, name + "_out")
        return heads, x, out, (seq, token, head), (out_seq, out_token, out_head)

    def _on(self, call, args, stream):
        if self._index < 0:
            raise ValueError("the frequencies are on %s: rotations run on a GPU" % self.device)
        if stream is None and _current_device() != self._index:
            with torch.cuda.device(self.device):         # a stream belongs to a device
                call(*args)
        else:
            call(*args, stream=stream)

    def rotate(self, positions, q, k=None, q_out=None, k_out=None, stream=None):
        """q (and k) rotated by positions, into q_out and k_out or in place. Negative positions undo positive ones. What is written for
        the one overlaps neither tensor of the other, and its own input only in place. Nothing is recorded for autograd: tensors that require
        a gradient are refused unless grad mode is off. The gradient of a rotation is the rotation of the outputs' gradient by -positions."""
        if positions.dim() != 2 or positions.dtype is not torch.int32 or positions.get_device() != self._index or not positions.is_contiguous():
            raise ValueError("positions: contiguous int32 [n_seqs][n_tokens] on %s is required" % self.device)
        n_seqs, n_tokens = positions.shape
        args = (self.desc, n_seqs, n_tokens, positions) + self._pair(q, q_out, n_seqs, n_tokens, "q")
        if k is not None:
            args += self._pair(k, k_out, n_seqs, n_tokens, "k")
        elif k_out is not None:
            raise ValueError("k_out without k")
        self._on(dkv.dkv_rotate, args, stream)
        q_out = q if q_out is None else q_out
        return q_out if k is None else (q_out, k if k_out is None else k_out)
