"""The fp16 paged KV cache with several new tokens of a sequence at once (include/okv_chunk.h) over torch-owned memory.

    cache = Cache16(n_layers=32, n_q_heads=32, n_kv_heads=8, head_dim=128, page_tokens=64, n_pages=4096, max_seqs=64, max_pages_per_seq=64)
    rope = Rope.of(128, base=10000.0, device="cuda:0")
    cache.pages.extend(seqs, n_new)                                              # lengths grow, pages are taken            (pages.py)
    cache.append(layer, k, v, starts, cache.lens, seqs, q=q, q_out=q, rope=rope) # rows [rows][G][d], turned by their positions
    cache.attend(layer, q, out, starts, cache.lens, seqs)                        # every row over its sequence, up to itself
    cache.pages.shrink(seqs, rejected)                                           # drafted tokens that were rejected go again

Pools are laid out as okv.h says: okv_decode_attn_static reads them too.  Every call runs the library's kernels on the current stream, allocates nothing and does
not wait: it may be captured in a graph.  Calls of one Cache16 follow one another on one stream, and come from one thread at a time: they share its workspace.  Calls that
may run at the same time need caches of their own (over the same pool and table, if they only attend).
"""
import ctypes
import math
import operator

import torch

from . import binding
from .cache8 import _address, need
from .pages import PageArray, Pages


class Rope:
    """How heads are turned by positions: pair j of the first 2 len(inv_freq) elements by position * inv_freq[j] (radians, float64).  Pairs are elements j and
    j + len(inv_freq), or with `interleaved` elements 2 j and 2 j + 1."""

    def __init__(self, inv_freq, interleaved=False):
        if inv_freq.dtype != torch.float64 or inv_freq.dim() != 1 or inv_freq.numel() % 8:
            raise ValueError("inv_freq must be a float64 vector of a multiple of 8 numbers")
        self.turns = (inv_freq / (2 * math.pi)).contiguous()
        self.rotated, self.interleaved, self.device = 2 * inv_freq.numel(), bool(interleaved), inv_freq.device

    @classmethod
    def of(cls, rotated, base=10000.0, interleaved=False, device="cuda:0"):
        """inv_freq[j] = base ** (-2 j / rotated)."""
        return cls(base ** (-torch.arange(0, rotated, 2, dtype=torch.float64, device=device) / rotated), interleaved)


class Cache16:
    """Buffers of the cache: pool [layers][n_pages][elements of a page], `table` [max_seqs][max_pages_per_seq] and `lens` [max_seqs], int32."""

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_pages_per_seq, pool=None, table=None, device="cuda:0"):
        self.device = torch.empty(0, device=device).device      # "cuda" is the current device's "cuda:n", as its tensors say
        self._index = self.device.index
        self.L, self.H, self.G, self.d, self.T, self.max_seqs = n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, max_seqs
        if n_layers < 1 or page_tokens < 16:
            raise ValueError("a cache has at least one layer, and pages of at least 16 tokens")
        c = binding.OkvLayerPool(n_q_heads, n_kv_heads, head_dim, page_tokens, max_pages_per_seq, 0, max_seqs, n_pages)
        self._workspace_bytes = int(binding.lib().okv_chunk_workspace_bytes(ctypes.byref(c)))
        binding._check(min(self._workspace_bytes, 0))
        shape = (n_layers, n_pages, 2 * n_kv_heads * page_tokens * head_dim)
        if pool is None:
            pool = torch.zeros(shape, dtype=torch.float16, device=self.device)
        if table is None:
            table = torch.full((max_seqs, max_pages_per_seq), -1, dtype=torch.int32, device=self.device)
        need("pool", pool, torch.float16, shape, self.device)
        need("table", table, torch.int32, (max_seqs, max_pages_per_seq), self.device)
        self.pool, self.table = pool, table
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=self.device)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=self.device)
        unit = 16 * binding.okv_slab_tiles(n_kv_heads, head_dim, page_tokens)
        self.pages = Pages(table=self.table, lens=self.lens, refs=self.refs, page_tokens=page_tokens, arrays=[PageArray(pool, unit)])
        c.block_table, c.refused = self.table.data_ptr(), self.pages.status.data_ptr() + 12      # after an extend() that could not take its pages nothing is
        self._layers = []                                                                        # written until check()
        for l in range(n_layers):
            x = binding.OkvLayerPool.from_buffer_copy(c)
            x.pool = pool[l].data_ptr()
            self._layers.append((x, ctypes.byref(x)))
        self.workspace = torch.empty(self._workspace_bytes, dtype=torch.uint8, device=self.device)
        self._rows = binding.OkvRows()
        self._rows_ref = ctypes.byref(self._rows)
        self._rope, self._chunk = binding.OkvRope(), binding.OkvChunk(workspace=self.workspace.data_ptr() or None, workspace_bytes=self._workspace_bytes)
        self._rope_ref, self._chunk_ref = ctypes.byref(self._rope), ctypes.byref(self._chunk)
        self._append, self._attend = binding.lib().okv_rope_append, binding.lib().okv_chunk_attn

    # (A small call is as short on the GPU as on the host: checks are written so that tensors as they should be pass in a few tests.)
    def _whose(self, layer, rows, starts, lens, seqs):
        device, int32 = self.device, torch.int32
        if not 0 <= layer < self.L:
            raise ValueError(f"layer must be in [0, {self.L})")
        batch = starts.shape[0] - 1 if starts.dim() == 1 else -1
        if starts.dtype is not int32 or batch < 0 or not starts.is_contiguous() or starts.get_device() != self._index:
            raise ValueError(f"starts must be an int32 vector of an entry more than there are sequences, on {device}")
        if lens.dtype is not int32 or lens.dim() != 1 or not lens.is_contiguous() or lens.get_device() != self._index or lens.shape[0] < (batch if seqs is None else self.max_seqs):
            raise ValueError(f"lens must be an int32 vector on {device} with an entry per row of the table (per sequence where seqs is None)")
        if seqs is not None and (seqs.dtype is not int32 or seqs.shape != (batch,) or not seqs.is_contiguous() or seqs.get_device() != self._index):
            need("seqs", seqs, int32, (batch,), device)
        r = self._rows
        r.batch, r.n_rows, r.seqs, r.starts, r.lens = batch, rows, _address(seqs), starts.data_ptr(), lens.data_ptr()
        return self._layers[layer][1]

    def _heads(self, name, t, rows, heads):
        """The stride of rows of heads, which are contiguous in a row."""
        d = self.d
        if t.dtype is torch.float16 and t.shape == (rows, heads, d) and t.get_device() == self._index:
            if t.is_contiguous():
                return heads * d
            if t.stride(2) == 1 and (heads == 1 or t.stride(1) == d):
                return t.stride(0) if rows > 1 else heads * d
        raise ValueError(f"{name} must be fp16 [{rows}][{heads}][{d}] on {self.device}, the heads of a row contiguous; it is {t.dtype} {list(t.shape)} on {t.device}")

    def append(self, layer, k, v, starts, lens, seqs=None, q=None, q_out=None, rope=None, positions=None):
        """Rows starts[b] .. starts[b + 1] - 1 of k and v (fp16 [rows][G][d], rows strided alike) become the last tokens of sequence b, which has lens[...] of them with
        these: lens is indexed by row of the table, seqs says which row each sequence is (None: b).  With a Rope the keys are turned by their place in
        the sequence, or by `positions` (int32 [rows]); so are the queries q [rows][H][d], into q_out (which may be q)."""
        rows = k.shape[0]
        kv_stride = self._heads("k", k, rows, self.G)
        if self._heads("v", v, rows, self.G) != kv_stride:
            raise ValueError("the rows of k and v must be strided alike")
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out come together")
        q_stride, out_stride = (0, 0) if q is None else (self._heads("q", q, rows, self.H), self._heads("q_out", q_out, rows, self.H))
        at = self._whose(layer, rows, starts, lens, seqs)
        turned = None
        if rope is not None:
            if rope.device != self.device:
                raise ValueError(f"the rope must be on {self.device}")
            if positions is not None and (positions.dtype is not torch.int32 or positions.shape != (rows,) or not positions.is_contiguous() or positions.device != self.device):
                need("positions", positions, torch.int32, (rows,), self.device)
            p = self._rope
            p.turns, p.rotated, p.interleaved, p.positions = rope.turns.data_ptr(), rope.rotated, rope.interleaved, _address(positions)
            turned = self._rope_ref
        elif positions is not None:
            raise ValueError("positions are a rope's")
        rc = self._append(at, self._rows_ref, turned, k.data_ptr(), v.data_ptr(), kv_stride, _address(q), q_stride, _address(q_out), out_stride,
                          binding.current_stream(self.device))
        if rc:
            binding._check(rc)

    def attend(self, layer, q, out, starts, lens, seqs=None, scale=0.0, cap=0.0, window=0, slopes=None, prefix=None):
        """Rows starts[b] .. starts[b + 1] - 1 of q (fp16 [rows][H][d], rows may be strided) are the last of sequence b's tokens and attend over it up to themselves;
        out fp16 or fp32 [rows][H][d], contiguous.  scale 0: 1 / sqrt(d).  cap: scores become cap tanh(score / cap).  window: a row sees that many tokens, its own among
        them.  slopes (fp32 [H]): scores fall by slopes[h] times the distance.  prefix (int32, by row of the table): that many tokens are seen by all."""
        rows, device = q.shape[0], self.device
        if window >= 1 << 31:
            raise ValueError("window must be below 2^31")
        q_stride = self._heads("q", q, rows, self.H)
        if out.dtype not in (torch.float16, torch.float32) or out.shape != q.shape or not out.is_contiguous() or out.get_device() != self._index:
            raise ValueError(f"out must be a contiguous fp16 or fp32 tensor {list(q.shape)} on {device}")
        at = self._whose(layer, rows, starts, lens, seqs)
        a = self._chunk
        if slopes is not None or prefix is not None:
            self._vectors(slopes, prefix, self._rows.batch if seqs is None else self.max_seqs)
        a.scale, a.cap, a.window, a.slopes, a.prefix, a.out_dtype = scale, cap, window, _address(slopes), _address(prefix), out.dtype is torch.float32
        rc = self._attend(at, self._rows_ref, self._chunk_ref, q.data_ptr(), q_stride, out.data_ptr(), binding.current_stream(device))
        if rc:
            binding._check(rc)

    def _vectors(self, slopes, prefix, entries):
        if slopes is not None:
            need("slopes", slopes, torch.float32, (self.H,), self.device)
        if prefix is not None and (prefix.dtype is not torch.int32 or prefix.dim() != 1 or not prefix.is_contiguous() or prefix.device != self.device or prefix.shape[0] < entries):
            raise ValueError(f"prefix must be an int32 vector on {self.device} with an entry per row of the table (per sequence where seqs is None)")

    def check_how(self, scale=0.0, cap=0.0, window=0, slopes=None, prefix=None):
        """Raises unless attend() takes these, with sequences by their rows of the table."""
        try:
            good = all(x == 0 or 1e-30 <= x <= 1e30 for x in (scale, cap)) and 0 <= operator.index(window) < 1 << 31
        except TypeError:
            good = False
        if not good:
            raise ValueError("scale and cap must be 0 or in [1e-30, 1e30], window a whole number in [0, 2^31)")
        self._vectors(slopes, prefix, self.max_seqs)
