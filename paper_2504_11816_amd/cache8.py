"""The 8-bit paged KV cache (include/okv_cache8.h) over torch-owned memory.

    cache = Cache8(n_layers=32, n_q_heads=32, n_kv_heads=8, head_dim=128, page_tokens=64, n_pages=4096, max_seqs=64, max_pages_per_seq=64)
    cache.pages.extend(seqs, n_new)                     # lengths grow, pages are taken            (pages.py)
    cache.store(k, v, starts, cache.lens, seqs)         # prompts: [layers][rows][G][d], quantised
    cache.pages.extend(seqs, ones)
    cache.step(q, k_new, v_new, out, cache.lens, seqs)  # a token per sequence in every layer
    cache.pages.fork(src, dst)                          # dst[i] becomes a copy of src[i] that shares its full pages
    cache.pages.free(seqs)

Every call runs the library's kernels on the current stream, allocates nothing and does not wait: it may be captured in a graph.
"""
import ctypes

import torch

from . import binding
from .pages import PageArray, Pages, RowArray

FORMATS = {"int8": 0, "e4m3": 1}
TILE = 32


def _address(t):
    return 0 if t is None else t.data_ptr()


def need(name, t, dtype, device, shape=None, dims=None):
    """Raises unless t is a contiguous tensor of this type, on this device, of this shape."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a {dtype} tensor on {device}")
    if (shape is not None and tuple(t.shape) != tuple(shape)) or (dims is not None and t.dim() != dims):
        raise ValueError(f"{name} has shape {tuple(t.shape)}" + (f", {tuple(shape)} is wanted" if shape is not None else ""))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


class Cache8:
    """Buffers of the cache: codes, scales, tails (see the header), `table` [max_seqs][max_pages_per_seq] and `lens` [max_seqs], int32.  The
    fp16 tails of all layers are [layers][max_seqs][2][G][32][d]."""

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_pages_per_seq, format="int8",
                 out_dtype=torch.float16, table=None, device="cuda:0"):
        if format not in FORMATS:
            raise ValueError(f"format must be one of {sorted(FORMATS)}")
        if out_dtype not in (torch.float16, torch.float32):
            raise ValueError("out_dtype must be torch.float16 or torch.float32")
        self.device = torch.device(device)
        self.L, self.H, self.G, self.d, self.T = n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens
        self.max_seqs, self.out_dtype = max_seqs, out_dtype
        c = self.c = binding.Okv8Cache(n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, FORMATS[format], int(out_dtype == torch.float32),
                                       max_seqs, max_pages_per_seq, n_pages)
        self.ref = ctypes.byref(c)

        def bytes_of(fn, *more):
            n = getattr(binding.lib(), fn)(self.ref, *more)
            return int(n) if n >= 0 else binding._check(int(n))

        tpp = page_tokens // TILE
        self.codes = torch.zeros(bytes_of("okv8_codes_bytes"), dtype=torch.uint8, device=self.device).view(n_layers, n_pages, tpp, -1)
        self.scales = torch.zeros(bytes_of("okv8_scales_bytes") // 4, dtype=torch.float32, device=self.device).view(n_layers, n_pages, tpp, -1)
        self.tails = torch.zeros(bytes_of("okv8_tails_bytes") // 2, dtype=torch.float16, device=self.device).view(
            n_layers, max_seqs, 2, n_kv_heads, TILE, head_dim)
        if table is None:
            table = torch.full((max_seqs, max_pages_per_seq), -1, dtype=torch.int32, device=self.device)
        need("table", table, torch.int32, self.device, (max_seqs, max_pages_per_seq))
        self.table = table
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=self.device)
        c.codes, c.scales, c.tails, c.page_table = (x.data_ptr() for x in (self.codes, self.scales, self.tails, self.table))
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=self.device)
        self.pages = Pages(table=self.table, lens=self.lens, refs=self.refs, page_tokens=page_tokens,
                           arrays=[PageArray(self.codes, TILE, whole_units=True), PageArray(self.scales, TILE, whole_units=True)],
                           rows=[RowArray(self.tails, 2 * n_kv_heads, TILE)])
        # the workspace of a whole batch; steps of one cache follow one another on one stream
        n = min(max_seqs, 4096)
        self.workspace = torch.empty(bytes_of("okv8_workspace_bytes", n), dtype=torch.uint8, device=self.device)
        self._step = binding.Okv8Step(workspace=self.workspace.data_ptr(), workspace_bytes=self.workspace.numel())
        self._step_ref = ctypes.byref(self._step)
        self._decode_step = binding.lib().okv8_decode_step

    # ---- prompts ----------------------------------------------------------------------------------

    def _rows(self, fn, k, v, starts, lens, seqs, layer):
        n_layers = k.shape[0] if k.dim() == 4 else 1
        batch = starts.numel() - 1
        shape = (*k.shape[:-2], self.G, self.d)
        for name, t in (("k", k), ("v", v)):
            if t.dtype != torch.float16 or t.device != self.device or tuple(t.shape) != shape or t.dim() not in (3, 4):
                raise ValueError(f"{name} must be fp16 [layers][rows][{self.G}][{self.d}] (or one layer's) on {self.device}")
            if t.numel() and (t[..., 0, :, :].stride()[-2:] != (self.d, 1) or any(a != b for a, b, n in zip(t.stride(), k.stride(), k.shape) if n > 1)):
                raise ValueError("the heads of a row must be contiguous, k and v laid out alike")
        self._seqs(seqs, batch)
        need("starts", starts, torch.int32, self.device, dims=1)
        need("lens", lens, torch.int32, self.device, dims=1)
        if lens.numel() < (self.max_seqs if seqs is not None else batch):
            raise ValueError("lens has an entry per row of the table (per sequence where seqs is None)")
        binding._check(fn(self.ref, layer, n_layers, batch, _address(seqs), starts.data_ptr(), lens.data_ptr(), k.shape[-3], k.data_ptr(), v.data_ptr(),
                          k.stride(-3) if k.shape[-3] > 1 else self.G * self.d, k.stride(0) if n_layers > 1 else 0, binding.current_stream(self.device)))

    def _seqs(self, seqs, batch):
        if seqs is not None:
            need("seqs", seqs, torch.int32, self.device, (batch,))

    def store(self, k, v, starts, lens, seqs=None, layer=0):
        """Stores rows starts[b] .. starts[b + 1] - 1 of k, v (fp16 [layers][rows][G][d], from `layer` on; or one layer's [rows][G][d]) as the last tokens of
        sequence b, which then has lens[...] of them: lens is indexed by row of the table, seqs says which row each sequence is (None: b)."""
        self._rows(binding.lib().okv8_store, k, v, starts, lens, seqs, layer)

    def load(self, k, v, starts, lens, seqs=None, layer=0):
        """The reverse: the values that the cache holds, into k and v."""
        self._rows(binding.lib().okv8_load, k, v, starts, lens, seqs, layer)

    # ---- decode steps -----------------------------------------------------------------------------

    def _describe(self, batch, appends, lens, seqs):
        if lens.dtype != torch.int32 or lens.device != self.device or lens.numel() < (self.max_seqs if seqs is not None else batch) or not lens.is_contiguous():
            raise ValueError("lens must be int32 with an entry per row of the table (per sequence where seqs is None)")
        self._seqs(seqs, batch)
        s = self._step
        s.batch, s.appends, s.seqs, s.lens, s.stream = batch, appends, _address(seqs), lens.data_ptr(), binding.current_stream(self.device)

    def begin(self, batch, lens, seqs=None, appends=True):
        """Describes a step whose layers come one by one (attend)."""
        self._describe(batch, int(appends), lens, seqs)
        binding._check(binding.lib().okv8_step_begin(self.ref, self._step_ref))

    def attend(self, layer, q, k_new, v_new, out):
        """One layer of the step that begin() described: q [batch][H][d], k_new / v_new [batch][G][d] (rows may be strided, k_new and v_new alike)
        or None, out [batch][H][d]."""
        batch = self._step.batch
        if q.dtype != torch.float16 or tuple(q.shape) != (batch, self.H, self.d) or q.stride(2) != 1 or q.stride(1) != self.d:
            raise ValueError(f"q must be fp16 [{batch}][{self.H}][{self.d}], rows may be strided")
        need("out", out, self.out_dtype, self.device, (batch, self.H, self.d))
        kv_stride = 0
        if k_new is not None:
            for t in (k_new, v_new):
                if t.dtype != torch.float16 or tuple(t.shape) != (batch, self.G, self.d) or t.stride(2) != 1 or t.stride(1) != self.d or t.stride(0) != k_new.stride(0):
                    raise ValueError(f"k_new and v_new must be fp16 [{batch}][{self.G}][{self.d}], rows strided alike")
            kv_stride = k_new.stride(0) if batch > 1 else self.G * self.d
        binding._check(binding.lib().okv8_decode_attn(self.ref, self._step_ref, layer, q.data_ptr(), q.stride(0) if batch > 1 else self.H * self.d,
                                                      _address(k_new), _address(v_new), kv_stride, out.data_ptr()))

    def step(self, q, k_new, v_new, out, lens, seqs=None):
        """One step of all layers whose inputs are there: q [L][batch][H][d], k_new / v_new [L][batch][G][d] or None (nothing is appended),
        out [L][batch][H][d].  lens: keys attended, an appended one included."""
        batch = q.shape[1]
        need("q", q, torch.float16, self.device, (self.L, batch, self.H, self.d))
        need("out", out, self.out_dtype, self.device, (self.L, batch, self.H, self.d))
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new come together")
        if k_new is not None:
            need("k_new", k_new, torch.float16, self.device, (self.L, batch, self.G, self.d))
            need("v_new", v_new, torch.float16, self.device, (self.L, batch, self.G, self.d))
        self._describe(batch, int(k_new is not None), lens, seqs)
        binding._check(self._decode_step(self.ref, self._step_ref, q.data_ptr(), _address(k_new), _address(v_new), out.data_ptr()))
