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
    return None if t is None else t.data_ptr()


def _fits(t, dtype, shape, device):
    return t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.device == device


def need(name, t, dtype, shape, device):
    """Raises unless t is a contiguous tensor of this type and shape on this device."""
    if not isinstance(t, torch.Tensor) or not _fits(t, dtype, shape, device):
        what = f"{t.dtype} {list(t.shape)} on {t.device}" if isinstance(t, torch.Tensor) else type(t).__name__
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on {device}, it is {what}")


class Cache8:
    """Buffers of the cache: codes, scales, tails (see the header), `table` [max_seqs][max_pages_per_seq] and `lens` [max_seqs], int32.  The
    fp16 tails of all layers are [layers][max_seqs][2][G][32][d]."""

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs, max_pages_per_seq, format="int8",
                 out_dtype=torch.float16, table=None, device="cuda:0"):
        if format not in FORMATS:
            raise ValueError(f"format must be one of {sorted(FORMATS)}")
        if out_dtype not in (torch.float16, torch.float32):
            raise ValueError("out_dtype must be torch.float16 or torch.float32")
        self.device = torch.empty(0, device=device).device      # "cuda" is the current device's "cuda:n", as its tensors say
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
        need("table", table, torch.int32, (max_seqs, max_pages_per_seq), self.device)
        self.table = table
        self.lens = torch.zeros(max_seqs, dtype=torch.int32, device=self.device)
        c.codes, c.scales, c.tails, c.page_table = (x.data_ptr() for x in (self.codes, self.scales, self.tails, self.table))
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=self.device)
        self.pages = Pages(table=self.table, lens=self.lens, refs=self.refs, page_tokens=page_tokens,
                           arrays=[PageArray(self.codes, TILE, whole_units=True), PageArray(self.scales, TILE, whole_units=True)],
                           rows=[RowArray(self.tails, 2 * n_kv_heads, TILE)])
        c.refused = self.pages.status.data_ptr() + 12        # after an extend() that could not take its pages nothing is written until check()
        # the workspace of a whole batch; steps of one cache follow one another on one stream
        n = min(max_seqs, 4096)
        self.workspace = torch.empty(bytes_of("okv8_workspace_bytes", n), dtype=torch.uint8, device=self.device)
        self._step = binding.Okv8Step(workspace=self.workspace.data_ptr(), workspace_bytes=self.workspace.numel())
        self._step_ref = ctypes.byref(self._step)
        # the step that begin() described, and the lens and seqs that its layers read; None: there is none
        self._layers = binding.Okv8Step(workspace=self.workspace.data_ptr(), workspace_bytes=self.workspace.numel())
        self._layers_ref, self._reads = ctypes.byref(self._layers), None
        lib = binding.lib()
        self._store, self._load, self._decode_step = lib.okv8_store, lib.okv8_load, lib.okv8_decode_step

    # ---- prompts ----------------------------------------------------------------------------------

    # (A small call is as short on the GPU as on the host: checks are written so that tensors as they should be pass in a few tests.)
    def _rows(self, call, k, v, starts, lens, seqs, layer):
        shape, half, G, d, device = k.shape, torch.float16, self.G, self.d, self.device
        if (k.dtype is not half or v.dtype is not half or v.shape != shape or len(shape) not in (3, 4) or shape[-1] != d or shape[-2] != G or k.device != device
                or v.device != device):
            raise ValueError(f"k and v must be fp16 [layers][rows][{G}][{d}] (or one layer's) on {device}, alike")
        n_layers, rows = shape[0] if len(shape) == 4 else 1, shape[-3]
        if k.is_contiguous() and v.is_contiguous():
            row_stride, layer_stride = G * d, rows * G * d
        else:
            if rows and n_layers and (k[..., 0, :, :].stride()[-2:] != (d, 1) or any(x != y for x, y, n in zip(k.stride(), v.stride(), shape) if n > 1)):
                raise ValueError("the heads of a row must be contiguous, k and v laid out alike")
            row_stride, layer_stride = k.stride(-3) if rows > 1 else G * d, k.stride(0) if n_layers > 1 else 0
        batch = self._batch(starts, lens, seqs)
        rc = call(self.ref, layer, n_layers, batch, _address(seqs), starts.data_ptr(), lens.data_ptr(), rows, k.data_ptr(), v.data_ptr(), row_stride, layer_stride,
                  binding.current_stream(device))
        if rc:
            binding._check(rc)

    def _batch(self, starts, lens, seqs):
        batch = starts.shape[0] - 1 if starts.dim() == 1 else -1
        if starts.dtype is not torch.int32 or batch < 0 or not starts.is_contiguous() or starts.device != self.device:
            raise ValueError(f"starts must be an int32 vector of an entry more than there are sequences, on {self.device}")
        self._lens(lens, seqs, batch)
        return batch

    def _lens(self, lens, seqs, batch):
        if lens.dtype is not torch.int32 or lens.dim() != 1 or not lens.is_contiguous() or lens.device != self.device or lens.shape[0] < (batch if seqs is None else self.max_seqs):
            raise ValueError(f"lens must be an int32 vector on {self.device} with an entry per row of the table (per sequence where seqs is None)")
        if seqs is not None:
            need("seqs", seqs, torch.int32, (batch,), self.device)

    def store(self, k, v, starts, lens, seqs=None, layer=0):
        """Stores rows starts[b] .. starts[b + 1] - 1 of k, v (fp16 [layers][rows][G][d], from `layer` on; or one layer's [rows][G][d]) as the last tokens of
        sequence b, which then has lens[...] of them: lens is indexed by row of the table, seqs says which row each sequence is (None: b)."""
        self._rows(self._store, k, v, starts, lens, seqs, layer)

    def load(self, k, v, starts, lens, seqs=None, layer=0):
        """The reverse: the values that the cache holds, into k and v."""
        self._rows(self._load, k, v, starts, lens, seqs, layer)

    # ---- decode steps -----------------------------------------------------------------------------

    def _describe(self, s, batch, appends, lens, seqs):
        self._reads = None                                   # (the workspace is this step's from here on)
        self._lens(lens, seqs, batch)
        s.batch, s.appends, s.seqs, s.lens, s.stream = batch, appends, _address(seqs), lens.data_ptr(), binding.current_stream(self.device)

    def begin(self, batch, lens, seqs=None, appends=True):
        """Describes a step whose layers come one by one (attend).  Every layer reads lens and seqs: they are kept until the next begin() or step(), and
        must not change before the last layer."""
        self._describe(self._layers, batch, int(appends), lens, seqs)
        binding._check(binding.lib().okv8_step_begin(self.ref, self._layers_ref))
        self._reads = lens, seqs

    def attend(self, layer, q, k_new, v_new, out):
        """One layer of the step that begin() described: q [batch][H][d], k_new / v_new [batch][G][d] (rows may be strided, k_new and v_new alike)
        or None, out [batch][H][d].  A step() of all layers, or a begin() that is refused, ends the step."""
        if self._reads is None:
            raise ValueError("begin() describes the step first (a step() of all layers in between ends it)")
        batch = self._layers.batch
        if q.dtype != torch.float16 or tuple(q.shape) != (batch, self.H, self.d) or q.stride(2) != 1 or q.stride(1) != self.d or q.device != self.device:
            raise ValueError(f"q must be fp16 [{batch}][{self.H}][{self.d}] on {self.device}, rows may be strided")
        need("out", out, self.out_dtype, (batch, self.H, self.d), self.device)
        kv_stride = 0
        if (k_new is None) != (v_new is None) or (k_new is None) != (self._layers.appends == 0):
            raise ValueError("k_new and v_new come together, if the step appends")
        if k_new is not None:
            for t in (k_new, v_new):
                if (t.dtype != torch.float16 or tuple(t.shape) != (batch, self.G, self.d) or t.stride(2) != 1 or t.stride(1) != self.d
                        or t.stride(0) != k_new.stride(0) or t.device != self.device):
                    raise ValueError(f"k_new and v_new must be fp16 [{batch}][{self.G}][{self.d}] on {self.device}, rows strided alike")
            kv_stride = k_new.stride(0) if batch > 1 else self.G * self.d
        self._layers.stream = binding.current_stream(self.device)
        binding._check(binding.lib().okv8_decode_attn(self.ref, self._layers_ref, layer, q.data_ptr(), q.stride(0) if batch > 1 else self.H * self.d,
                                                      _address(k_new), _address(v_new), kv_stride, out.data_ptr()))

    def step(self, q, k_new, v_new, out, lens, seqs=None):
        """One step of all layers whose inputs are there: q [L][batch][H][d], k_new / v_new [L][batch][G][d] or None (nothing is appended),
        out [L][batch][H][d].  lens: keys attended, an appended one included."""
        L, H, d, device = self.L, self.H, self.d, self.device
        batch = q.shape[1] if q.dim() == 4 else 0
        if not _fits(q, torch.float16, (L, batch, H, d), device) or not _fits(out, self.out_dtype, (L, batch, H, d), device):
            need("q", q, torch.float16, (L, batch, H, d), device)
            need("out", out, self.out_dtype, (L, batch, H, d), device)
        if (k_new is None) != (v_new is None):
            raise ValueError("k_new and v_new come together")
        if k_new is not None and not (_fits(k_new, torch.float16, (L, batch, self.G, d), device) and _fits(v_new, torch.float16, (L, batch, self.G, d), device)):
            need("k_new", k_new, torch.float16, (L, batch, self.G, d), device)
            need("v_new", v_new, torch.float16, (L, batch, self.G, d), device)
        self._describe(self._step, batch, 0 if k_new is None else 1, lens, seqs)
        rc = self._decode_step(self.ref, self._step_ref, q.data_ptr(), _address(k_new), _address(v_new), out.data_ptr())
        if rc:
            binding._check(rc)
