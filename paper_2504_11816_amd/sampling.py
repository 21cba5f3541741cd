"""From logits to tokens (include/okv_sample.h) over torch-owned memory.

    sampler = Sampler(max_batch=64, vocab=32000)
    sampler.probs(logits, probs, temperature)                                               # fp16 or fp32 [rows][vocab] -> fp32
    sampler.verify(probs, drafts, starts, uniforms, tokens, accepted, rejected, draft_probs=q)   # drafted tokens held against the target's probabilities
    cache.pages.shrink(seqs, rejected)

Every call runs the library's kernels on the current stream, allocates nothing and does not wait: it may be captured in a graph.
"""
import torch

from . import binding
from .cache8 import _address, need


class Sampler:
    """Workspace for calls of up to max_batch rows (probs) and sequences (verify); calls of one Sampler follow one another on one stream."""

    def __init__(self, *, max_batch, vocab, device="cuda:0"):
        self.device = torch.empty(0, device=device).device
        self.max_batch, self.vocab, self._index = max_batch, vocab, self.device.index
        lib = binding.lib()
        sizes = [int(lib.okv_token_probs_workspace_bytes(max_batch, vocab)), int(lib.okv_verify_workspace_bytes(min(max_batch, 4096), vocab))]
        binding._check(min(*sizes, 0))
        self.workspace = torch.empty(max(sizes), dtype=torch.uint8, device=self.device)
        self._at, self._bytes = self.workspace.data_ptr() or None, max(sizes)
        self._probs, self._verify = lib.okv_token_probs, lib.okv_verify

    def _table(self, name, t, dtypes, rows):
        """The stride of rows of vocab numbers."""
        if t.dtype in dtypes and t.shape == (rows, self.vocab) and t.get_device() == self._index:
            if t.is_contiguous():
                return self.vocab
            if self.vocab == 1 or t.stride(1) == 1:
                return t.stride(0) if rows > 1 else self.vocab
        raise ValueError(f"{name} must be {' or '.join(map(str, dtypes))} [{rows}][{self.vocab}] on {self.device}, rows contiguous; it is {t.dtype} {list(t.shape)} on {t.device}")

    def probs(self, logits, out, temperature=None):
        """out (fp32) = softmax of each row of logits (fp16 or fp32 [rows][vocab], rows may be strided) / temperature (fp32 [rows], or None: 1).  Temperature 0: 1 at the
        first of the largest."""
        rows = logits.shape[0]
        stride = self._table("logits", logits, (torch.float16, torch.float32), rows)
        out_stride = self._table("out", out, (torch.float32,), rows)
        if rows > self.max_batch:
            raise ValueError(f"the sampler has room for {self.max_batch} rows")
        if temperature is not None:
            need("temperature", temperature, torch.float32, (rows,), self.device)
        rc = self._probs(logits.data_ptr(), int(logits.dtype is torch.float32), stride, _address(temperature), out.data_ptr(), out_stride, rows, self.vocab,
                         self._at, self._bytes, binding.current_stream(self.device))
        if rc:
            binding._check(rc)

    def verify(self, target, drafts, starts, uniforms, tokens, accepted, rejected=None, draft_probs=None):
        """Sequence b's drafts are starts[b] .. starts[b + 1] - 1 of drafts (int32 [n]); draft_probs (fp32 [n][vocab], or None: the drafts were certain) is what they were drawn
        from.  target (fp32 [n + batch][vocab]) and uniforms (fp32 [n + batch]) have one row more per sequence, the first at starts[b] + b.  tokens (int32 [n + batch]) receives
        the accepted drafts, the next token and -1 behind it; accepted and rejected (int32 [batch]) how many they are.  (See the header.)"""
        n, batch, device = drafts.shape[0] if drafts.dim() == 1 else -1, starts.shape[0] - 1 if starts.dim() == 1 else -1, self.device
        if not 0 <= batch <= self.max_batch:
            raise ValueError(f"starts must have an entry more than there are sequences, of which there is room for {self.max_batch}")
        for name, t, size in (("drafts", drafts, n), ("starts", starts, batch + 1), ("tokens", tokens, n + batch), ("accepted", accepted, batch), ("rejected", rejected, batch)):
            if t is not None and (t.dtype is not torch.int32 or t.shape != (size,) or not t.is_contiguous() or t.get_device() != self._index):
                need(name, t, torch.int32, (size,), device)
        need("uniforms", uniforms, torch.float32, (n + batch,), device)
        stride = self._table("target", target, (torch.float32,), n + batch)
        draft_stride = self.vocab if draft_probs is None else self._table("draft_probs", draft_probs, (torch.float32,), n)
        at = None if draft_probs is None else draft_probs.data_ptr() or target.data_ptr()      # (of no rows: an address that is not read)
        rc = self._verify(target.data_ptr(), stride, at, draft_stride, drafts.data_ptr(), starts.data_ptr(), uniforms.data_ptr(), tokens.data_ptr(), accepted.data_ptr(),
                          _address(rejected), batch, n, self.vocab, self._at, self._bytes, binding.current_stream(device))
        if rc:
            binding._check(rc)
