"""A cache in pages of 8-bit rows: what the prefill leaves of each layer, the new tokens behind it, and the attention over both.

Where Compressor's padded blocks keep window + layer_max row slots for every layer, a PagedCache keeps pages for the rows that are
there, one byte an element. Every call is one dkv_pages_* call; the row counts stay on the device.

    cache = PagedCache(comp.desc, n_pages=4096, max_rows=8192)
    cache.resize(comp.counts, cu_seqlens=comp.cu)                       # room for the window rows and the retained rows
    cache.store_layers(0, ks, vs, comp.cu, comp.idx, comp.counts)       # (or Compressor(cfg, pages=cache), which does both)
    per token:  cache.fork(parents)                                     # beams: before the growth, which copies what they share
                cache.resize(cache.rows, 1)
                per layer:  cache.append(l, k_new, v_new);  cache.attention(l, q_new, out, expected_rows=about_as_many)
    now and then:  cache.missing                                        # not 0: the pool was too small, nothing was written since
"""
from __future__ import annotations

import torch

from . import dkv

_DTYPES = {dkv.DKV_BF16: torch.bfloat16, dkv.DKV_F32: torch.float32}
_current_device = getattr(torch._C, "_cuda_getDevice", None)        # what torch.cuda.current_device() asks, without its start-up


NEW_ROWS = 1024                     # room for new tokens behind a prompt's rows where max_rows is not given


class PagedCache:
    """desc: the dkv_desc of the sequences that share the pool. max_rows: rows that one (sequence, layer) can hold (rounded up to pages);
    by default all that a prompt can leave, window + layer_max, and NEW_ROWS, or as many as a table that is handed over has entries for.
    The tensors (k, v as torch.float8_e4m3fn, k_scale, v_scale, table, rows, refs, missing; shapes as in include/dkv.h) are allocated
    and cleared, unless the caller hands over its own."""

    def __init__(self, desc, n_pages, page_rows=64, max_rows=None, device="cuda", **tensors):
        self.desc, self.tdtype = desc, _DTYPES[desc.dtype]
        L, Hkv, d, n_seqs = desc.n_layers, desc.n_kv_heads, desc.head_dim, desc.n_seqs
        if page_rows not in (16, 32, 64, 128) or n_pages < 1:
            raise ValueError("page_rows is 16, 32, 64 or 128 and n_pages at least 1: got %r, %r" % (page_rows, n_pages))
        by_default, table, prompt = max_rows is None, tensors.get("table"), desc.window + desc.layer_max
        table_len = max(-(-(prompt + NEW_ROWS if by_default else max_rows) // page_rows), 1)
        if by_default and table is not None and table.dim() == 3:
            table_len = max(table.shape[2], 1)
        self.max_rows = table_len * page_rows
        # attention's hint where the caller has none: that the tables have room for new tokens does not make the prompt's rows more
        self._expected = -(-prompt // page_rows) * page_rows if by_default and table is None else 0
        shapes = {"k": ((n_pages, Hkv, page_rows, d), torch.float8_e4m3fn), "v": ((n_pages, Hkv, d, page_rows), torch.float8_e4m3fn),
                  "k_scale": ((n_pages, Hkv), torch.float32), "v_scale": ((n_pages, Hkv), torch.float32),
                  "table": ((n_seqs, L, table_len), torch.int32), "rows": ((n_seqs, L), torch.int32),
                  "refs": ((n_pages,), torch.int32), "missing": ((1,), torch.int32)}
        unknown = set(tensors) - set(shapes)
        if unknown or (tensors and set(tensors) != set(shapes)):
            raise ValueError("all of %s or none are handed over: got %s" % (", ".join(shapes), ", ".join(sorted(tensors))))
        self.device = torch.device(device if not tensors else tensors["k"].device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        for name, (shape, dtype) in shapes.items():
            t = tensors.get(name)
            if t is None:
                # pages start as zeros: codes that nothing has written are numbers
                t = torch.zeros(shape, dtype=torch.uint8, device=self.device).view(dtype) if name in "kv" else \
                    torch.ones(shape, dtype=dtype, device=self.device) if "scale" in name else \
                    torch.zeros(shape, dtype=dtype, device=self.device)
            elif tuple(t.shape) != shape or t.dtype != dtype or t.device != self.device or not t.is_contiguous():
                raise ValueError("%s: contiguous %s %s on %s is required" % (name, dtype, list(shape), self.device))
            setattr(self, name, t)
        self.pages = dkv.dkv_pages(n_pages, page_rows, table_len, *(getattr(self, name).data_ptr() for name in shapes))
        n = dkv.dkv_pages_workspace_bytes(desc, self.pages)
        if n == 0:
            raise dkv.DkvError(dkv.DKV_ERR_INVALID_ARG, "dkv_pages_workspace_bytes")
        self.ws = torch.empty(n, dtype=torch.uint8, device=self.device)
        self._index = -1 if self.device.type != "cuda" else self.device.index
        self._of_pairs, self._of_seqs, self._of_bounds = torch.Size((n_seqs, L)), torch.Size((n_seqs,)), torch.Size((n_seqs + 1,))
        self._of_rows, self._of_row = torch.Size((n_seqs, Hkv, d)), torch.Size((Hkv, d))
        self._of_idx, self._of_layer_idx = torch.Size((L, n_seqs, Hkv, desc.layer_max)), torch.Size((n_seqs, Hkv, desc.layer_max))
        self._of_q, self._of_lse = torch.Size((n_seqs, desc.n_q_heads, d)), torch.Size((n_seqs, desc.n_q_heads))
        if not tensors:
            self.clear()

    def _on(self, call, *args):
        if self._index < 0:
            raise ValueError("the cache's tensors are on %s: its calls run on a GPU" % self.device)
        # a stream belongs to a device: the last argument, None, is the current stream of the cache's
        if args[-1] is None and _current_device() != self._index:
            with torch.cuda.device(self.device):
                return call(*args)
        return call(*args)

    def _whole(self, t, shape, dtype, name):
        if t.shape != shape or t.dtype is not dtype or t.get_device() != self._index or not t.is_contiguous():
            raise ValueError("%s: contiguous %s %s on %s is required, got %s %s on %s"
                             % (name, dtype, list(shape), self.device, t.dtype, list(t.shape), t.device))

    def _ints(self, t, shape, name):
        if t is not None and t is not self.rows:
            self._whole(t, shape, torch.int32, name)
        return t

    def clear(self, stream=None):
        """No rows, all pages free."""
        self._on(dkv.dkv_pages_clear, self.desc, self.pages, stream)

    def resize(self, base=None, extra=0, cu_seqlens=None, active=None, layer_begin=0, n_layers=None, stream=None):
        """Every (sequence, layer) of the call gets base + extra rows (and, with cu_seqlens, its window rows: base is then `counts`).
        Growth is all or nothing: cache.missing becomes the number of pages that lacked, and while it is not 0 nothing grows and no
        row is written. The caller looks at it when it likes, ends or shortens sequences and sets it to 0 (missing.zero_())."""
        self._on(dkv.dkv_pages_resize, self.desc, layer_begin, self._of_pairs[1] - layer_begin if n_layers is None else n_layers, self.pages,
                 self._ints(base, self._of_pairs, "base"), self._ints(cu_seqlens, self._of_bounds, "cu_seqlens"), extra,
                 self._ints(active, self._of_seqs, "active"), self.ws, stream)

    def fork(self, parents, stream=None):
        """Sequence q goes on from what sequence parents[q] holds, for all q at once; parents[q] outside the batch: it is emptied. Before
        the resize that makes room for new rows: that copies a last page that is shared, and append writes to no page that is."""
        self._on(dkv.dkv_pages_fork, self.desc, self.pages, self._ints(parents, self._of_seqs, "parents"), self.ws, stream)

    def _prompt_strides(self, ks, vs, stride_token, stride_head):
        """As given, else those of the tensors, [Hkv][tokens][d]; the call has one pair of strides for all of them."""
        if stride_token is None or stride_head is None:
            Hkv, d = self._of_row
            shape, strides = ks[0].shape, ks[0].stride()
            alike = len(shape) == 3 and shape[0] == Hkv and shape[2] == d and strides[2] == 1
            for xs in (ks, vs):
                for x in xs:
                    if x.shape != shape or (x.stride() != strides and self._lies_apart(x, strides)):
                        alike = False
            if not alike:
                raise ValueError("k, v: [%d][tokens][%d] with the same tokens and strides, or stride_token and stride_head, are required" % (Hkv, d))
            stride_token = strides[1] if stride_token is None else stride_token
            stride_head = strides[0] if stride_head is None else stride_head
        return stride_token, stride_head

    @staticmethod
    def _lies_apart(x, strides):
        """Whether x has other strides, along dimensions of more than one element."""
        return any(n > 1 and a != b for n, a, b in zip(x.shape, x.stride(), strides))

    def _prompt(self, ks, vs, cu_seqlens, idx, of_idx, counts):
        dtype, index, i32 = self.tdtype, self._index, torch.int32
        for xs in (ks, vs):
            for x in xs:
                if x.dtype is not dtype or x.get_device() != index:
                    raise ValueError("k, v: %s on %s is required, got %s on %s" % (dtype, self.device, x.dtype, x.device))
        if not (cu_seqlens.dtype is idx.dtype is counts.dtype is i32 and cu_seqlens.get_device() == idx.get_device() == counts.get_device() == index and
                cu_seqlens.shape == self._of_bounds and idx.shape == of_idx and counts.shape == self._of_pairs and
                cu_seqlens.is_contiguous() and idx.is_contiguous() and counts.is_contiguous()):
            self._whole(cu_seqlens, self._of_bounds, i32, "cu_seqlens")
            self._whole(idx, of_idx, i32, "idx")
            self._whole(counts, self._of_pairs, i32, "counts")

    def store(self, layer, k, v, cu_seqlens, idx, counts, stride_token=None, stride_head=None, stream=None):
        """The window rows and the retained rows of a layer (idx [n_seqs][Hkv][layer_max], as the selection writes it). k, v: [Hkv][tokens]
        [d], or any order whose strides (in elements) are given."""
        self._prompt((k,), (v,), cu_seqlens, idx, self._of_layer_idx, counts)
        self._on(dkv.dkv_pages_store, self.desc, layer, self.pages, k, v, *self._prompt_strides((k,), (v,), stride_token, stride_head),
                 cu_seqlens, idx, counts, stream)

    def store_layers(self, layer_begin, ks, vs, cu_seqlens, idx_all, counts, stride_token=None, stride_head=None, stream=None):
        """The same for consecutive layers in one call (idx_all [L][n_seqs][Hkv][layer_max]; all ks and vs have the same strides: they are compared
        unless both strides are given, which then are those of all)."""
        ks, vs = ks if type(ks) is list else list(ks), vs if type(vs) is list else list(vs)
        if not ks or len(ks) != len(vs):
            raise ValueError("as many of v as of k, and one at least: got %d and %d" % (len(vs), len(ks)))
        self._prompt(ks, vs, cu_seqlens, idx_all, self._of_idx, counts)
        self._on(dkv.dkv_pages_store_layers, self.desc, layer_begin, self.pages, ks, vs,
                 *self._prompt_strides(ks, vs, stride_token, stride_head), cu_seqlens, idx_all, counts, stream)

    def append(self, layer, k_new, v_new, active=None, stream=None):
        """The last rows of every sequence become the new tokens' [n_seqs][n_new][Hkv][d] (or [n_seqs][Hkv][d]: one token); k_new and v_new
        have the same strides. Rows in a page that several sequences share, and all rows while cache.missing is not 0, are left out."""
        shape, strides = k_new.shape, k_new.stride()
        if v_new.shape != shape or v_new.stride() != strides or strides[-1] != 1:
            raise ValueError("k_new and v_new have the same shape and strides, with the elements of a row side by side")
        if shape == self._of_rows:
            n_new, strides = 1, (strides[0], 0, strides[1])
        elif len(shape) == 4 and shape[0] == self._of_rows[0] and shape[2:] == self._of_row:
            n_new, strides = shape[1], strides[:3]
        else:
            n_new = 0
        if n_new == 0 or not (k_new.dtype is v_new.dtype is self.tdtype and k_new.get_device() == v_new.get_device() == self._index):
            raise ValueError("k_new, v_new: %s [%d](n_new)%s on %s is required, got %s, %s %s on %s"
                             % (self.tdtype, self._of_rows[0], list(self._of_row), self.device, k_new.dtype, v_new.dtype, list(shape), k_new.device))
        self._on(dkv.dkv_pages_append, self.desc, layer, self.pages, n_new, k_new, v_new, *strides,
                 self._ints(active, self._of_seqs, "active"), stream)

    def attention(self, layer, q_new, out, lse_out=None, expected_rows=0, stream=None):
        """Attention of one new token per sequence (q_new [n_seqs][Hq][d]) over layer `layer`; out fp32 like q_new, lse_out [n_seqs][Hq].
        expected_rows: how many rows there are, about; it decides the time, and the split over workgroups that pays for long rows costs
        short ones a launch. 0: as many as max_rows, or, where that is the default, as a prompt leaves at most."""
        self._whole(q_new, self._of_q, self.tdtype, "q_new")
        self._whole(out, self._of_q, torch.float32, "out")
        if lse_out is not None:
            self._whole(lse_out, self._of_lse, torch.float32, "lse_out")
        self._on(dkv.dkv_pages_attention, self.desc, layer, self.pages, expected_rows or self._expected, q_new, out, lse_out, self.ws, stream)

    def attention_layers(self, layer_begin, n_layers, q_new_all, out_all, lse_all=None, expected_rows=0, stream=None):
        """The same for n_layers consecutive layers in one call: q_new_all, out_all [n_layers][n_seqs][Hq][d]."""
        self._whole(q_new_all, (n_layers,) + self._of_q, self.tdtype, "q_new_all")
        self._whole(out_all, (n_layers,) + self._of_q, torch.float32, "out_all")
        if lse_all is not None:
            self._whole(lse_all, (n_layers,) + self._of_lse, torch.float32, "lse_all")
        self._on(dkv.dkv_pages_attention_layers, self.desc, layer_begin, n_layers, self.pages, expected_rows or self._expected, q_new_all, out_all,
                 lse_all, self.ws, stream)
