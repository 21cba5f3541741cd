"""Pages of a paged KV cache (include/okv_pages.h) over torch-owned memory.

    pages = Pages(table=table, lens=lens, refs=refs, page_tokens=T, arrays=[PageArray(pool, unit_tokens=16)])
    pages.extend(seqs, n_new); pages.fork(src, dst); pages.shrink(seqs, n_drop); pages.free(seqs); pages.compact(); pages.copy(src_ids, dst_ids, to=[PageArray(staging)])

The state is on the GPU and every call runs on the current stream without waiting; check() reads the status and raises.
"""
import ctypes

import torch

from . import binding


class PageArray:
    """What every page holds in every layer: tensor [layers][n_pages][...], contiguous in a page.  unit_tokens and whole_units: what a fork copies
    of a page that is not full (see the header)."""

    def __init__(self, tensor, unit_tokens=1, whole_units=False):
        if tensor.dim() < 2 or not tensor[0].is_contiguous():
            raise ValueError("a page array is [layers][n_pages][...], every layer contiguous")
        self.tensor = tensor
        self.layers, self.pages, self.device = tensor.shape[0], tensor.shape[1], tensor.device
        self.page_bytes = tensor[0, 0].numel() * tensor.element_size()
        self.c = binding.OkvPageArray(tensor.data_ptr(), self.page_bytes, tensor.stride(0) * tensor.element_size(), unit_tokens, int(whole_units))


class RowArray:
    """What every sequence holds beside its pages: tensor [layers][max_seqs][...] whose sequences are `groups` groups of `rows` rows."""

    def __init__(self, tensor, groups, rows):
        if tensor.dim() < 3 or not tensor[0].is_contiguous():
            raise ValueError("a row array is [layers][max_seqs][...], every layer contiguous")
        per_seq = tensor[0, 0].numel() * tensor.element_size()
        if groups < 1 or rows < 1 or per_seq % (groups * rows):
            raise ValueError("a sequence's rows do not come out even")
        self.tensor = tensor
        self.c = binding.OkvRowArray(tensor.data_ptr(), tensor.stride(0) * tensor.element_size(), groups, rows, per_seq // (groups * rows))


class Pages:
    """table [max_seqs][max_pages_per_seq], lens [max_seqs], refs [n_pages]: int32 tensors that the calls read and write (new ones: -1, 0, 0)."""

    def __init__(self, *, table, lens, refs, page_tokens, arrays=(), rows=()):
        self.device, self._lib = table.device, binding.lib()
        for name, t, dims in (("table", table, 2), ("lens", lens, 1), ("refs", refs, 1)):
            if t.dtype != torch.int32 or t.dim() != dims or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"{name} must be a contiguous int32 tensor of {dims} dimension(s) on {self.device}")
        if lens.numel() != table.shape[0]:
            raise ValueError("lens has an entry per row of the table")
        if len(arrays) > 4 or len(rows) > 2:
            raise ValueError("at most 4 page arrays and 2 row arrays")
        every = [*arrays, *rows]
        if len({a.tensor.shape[0] for a in every}) > 1 or any(a.tensor.device != self.device for a in every):
            raise ValueError("all arrays have the same layers, on the table's device")
        if any(a.tensor.shape[1] != refs.numel() for a in arrays) or any(r.tensor.shape[1] != table.shape[0] for r in rows):
            raise ValueError("page arrays have refs.numel() pages, row arrays a sequence per row of the table")
        self.table, self.lens, self.refs, self.arrays, self.rows = table, lens, refs, list(arrays), list(rows)
        self.status = torch.zeros(4, dtype=torch.int32, device=self.device)
        n = int(binding.lib().okv_pages_workspace_bytes(refs.numel()))
        binding._check(min(n, 0))
        self.workspace = torch.empty(n, dtype=torch.uint8, device=self.device)
        c = self.c = binding.OkvPages(n_layers=every[0].tensor.shape[0] if every else 1, page_tokens=page_tokens, max_seqs=table.shape[0],
                                      max_pages_per_seq=table.shape[1], n_pages=refs.numel(), n_arrays=len(arrays), n_rows=len(rows))
        for i, a in enumerate(arrays):
            c.arrays[i] = a.c
        for i, r in enumerate(rows):
            c.rows[i] = r.c
        c.table, c.lens, c.refs, c.status = (t.data_ptr() for t in (table, lens, refs, self.status))
        c.workspace, c.workspace_bytes = self.workspace.data_ptr(), n
        self.ref = ctypes.byref(c)

    def _ids(self, name, t, n=None):
        if t.dtype is not torch.int32 or t.dim() != 1 or not t.is_contiguous() or t.device != self.device:
            raise ValueError(f"{name} must be a contiguous int32 vector on {self.device}")
        if n is not None and t.shape[0] != n:
            raise ValueError(f"{name} has {t.shape[0]} entries, {n} are wanted")
        return t.data_ptr()

    def _done(self, rc):
        if rc:
            binding._check(rc)

    def extend(self, seqs, n_new=None):
        """Sequence seqs[i] grows by n_new[i] tokens (None: one each) and takes the pages that it lacks.  Changes nothing where there are too few, and
        nothing from then on until check() has raised."""
        at, n = self._ids("seqs", seqs), seqs.shape[0]
        self._done(self._lib.okv_pages_extend(self.ref, n, at, None if n_new is None else self._ids("n_new", n_new, n), binding.current_stream(self.device)))

    def fork(self, src, dst):
        """Sequence dst[i] (empty) becomes a fork of src[i]: shares its full pages, copies the rest."""
        at, n = self._ids("src", src), src.shape[0]
        self._done(self._lib.okv_pages_fork(self.ref, n, at, self._ids("dst", dst, n), binding.current_stream(self.device)))

    def free(self, seqs):
        """The sequences become empty; pages that belong to no other are free."""
        self._done(self._lib.okv_pages_free(self.ref, seqs.shape[0], self._ids("seqs", seqs), binding.current_stream(self.device)))

    def shrink(self, seqs, n_drop):
        """Sequence seqs[i] loses its last n_drop[i] tokens; pages that it needs no longer are free, if they belong to no other.  Changes nothing where
        that does not fit the state (see the header)."""
        at, n = self._ids("seqs", seqs), seqs.shape[0]
        self._done(self._lib.okv_pages_shrink(self.ref, n, at, self._ids("n_drop", n_drop, n), binding.current_stream(self.device)))

    def compact(self):
        """Pages in use become 0 .. n_used - 1 (status[1] says how many, status[2] how many were moved)."""
        self._done(self._lib.okv_pages_compact(self.ref, binding.current_stream(self.device)))

    def copy(self, src_ids, dst_ids, to=None):
        """Copies pages src_ids[i] to pages dst_ids[i] of the arrays `to` (PageArrays like this cache's; None: this cache's own)."""
        to = self.arrays if to is None else to
        if len(to) != len(self.arrays):
            raise ValueError("`to` has an array for each of the cache's")
        if not to:
            return
        pages, c = 0x7fffffff, (binding.OkvPageArray * len(to))()
        for i, (t, a) in enumerate(zip(to, self.arrays)):
            if t.page_bytes != a.page_bytes or t.layers != a.layers or t.device != self.device:
                raise ValueError("`to` has an array for each of the cache's, with the same layers and page sizes")
            c[i], pages = t.c, min(pages, t.pages)
        at, n = self._ids("src_ids", src_ids), src_ids.shape[0]
        self._done(self._lib.okv_pages_copy(self.ref, n, at, self._ids("dst_ids", dst_ids, n), c, pages, binding.current_stream(self.device)))

    def check(self):
        """Waits for the GPU; raises if a call could not be carried out since the last check.  After an extend() that could not be, no
        sequence grows and a Cache8 is not written to until check() has raised."""
        code = int(self.status[0])
        if code:
            self.status[::3] = 0
            raise binding.OkvError(code, "no room: too few free pages, or a row of the table is full" if code == binding.OKV_ENOSPC
                                   else "the sequences that were named do not fit the state of the cache")
