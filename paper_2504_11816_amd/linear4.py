"""Linear layers with 4-bit weights and group scales (include/okv_linear4.h) over torch-owned memory.

    w = Linear4.quantize(weight, group=128)           # fp16 [n_out][n_in], as a framework's linear layer has it
    w = Linear4(codes, scales, zeros, bias)           # quantised elsewhere
    w(x, out, relu=True)                              # out = relu(x W^T + bias)
    qkv(x, [q, k, v])                                 # the output features in up to three tensors
    w(x, y, residual=y)                               # y += x W^T + bias

For a decode batch's rows: from 32 (4096 x 4096) to 128 rows on, by group size and matrix, fp16 weights are faster (figures in the header).
"""
import ctypes

import torch

from . import binding


_One = ctypes.c_void_p * 1


class Linear4:
    """W[n][k] = (codes[n][k] - zeros[n][k / group]) * scales[n][k / group], packed for the product kernels.

    codes uint8 [n_out][n_in] (0 .. 15 each) or [n_out][n_in / 2] (two a byte, the even input low), scales fp16 [n_out][n_in / group], zeros uint8 of
    that shape or None (8 everywhere), bias fp16 [n_out] or None.  n_in says which of the two codes are, group is taken from it and the scales."""

    def __init__(self, codes, scales, zeros=None, bias=None, n_in=None):
        n_out = codes.shape[0]
        self._shape(n_out, codes.shape[1] if n_in is None else n_in, None, zeros is not None, codes.device)
        if scales.dim() != 2 or scales.shape[0] != n_out or scales.shape[1] < 1 or self.n_in % scales.shape[1]:
            raise ValueError("scales must be [n_out][n_in / group]")
        self.group = self.n_in // scales.shape[1]
        if codes.shape[1] not in (self.n_in, self.n_in // 2):
            raise ValueError("codes must be [n_out][n_in], or [n_out][n_in / 2] with n_in given")
        for name, t, dtype in (("codes", codes, torch.uint8), ("scales", scales, torch.float16), ("zeros", zeros, torch.uint8)):
            if t is not None and (t.dtype != dtype or t.device != self.device or t.dim() != 2 or (name == "zeros" and t.shape != scales.shape)):
                raise ValueError(f"{name} must be a {dtype} matrix on {self.device}" + (" of the scales' shape" if name == "zeros" else ""))
        self._allocate(bias)
        with torch.cuda.device(self.device):
            codes, scales, zeros = (t.contiguous() if t is not None else None for t in (codes, scales, zeros))
            binding._check(binding.lib().okv_linear4_pack(self.packed.data_ptr(), codes.data_ptr(), self.n_in // codes.shape[1], scales.data_ptr(),
                                                          zeros.data_ptr() if zeros is not None else None, n_out, self.n_in, self.group, self._stream()))

    def _shape(self, n_out, n_in, group, zeros, device):
        self.n_out, self.n_in, self.group, self.zeros, self.device = n_out, n_in, group, int(zeros), device

    def _stream(self):
        return binding.current_stream(self.device)

    def _allocate(self, bias):
        n = int(binding.lib().okv_linear4_packed_bytes(self.n_out, self.n_in, self.group, self.zeros))
        binding._check(min(n, 0))
        if bias is not None and (bias.dtype != torch.float16 or tuple(bias.shape) != (self.n_out,) or bias.device != self.device or not bias.is_contiguous()):
            raise ValueError(f"bias must be a contiguous fp16 vector of {self.n_out} on {self.device}")
        self.bias = bias
        self.packed = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.workspace, self._workspace_bytes, self._wants, self._outgrown = None, 0, {}, []
        self._call, self._packed_at, self._bias_at = binding.lib().okv_linear4, self.packed.data_ptr(), bias.data_ptr() if bias is not None else None

    @classmethod
    def quantize(cls, weight, group=128, zeros=False, bias=None):
        """Quantises fp16 [n_out][n_in] weights, every group by itself (see the header).  A group with a weight that is infinite or NaN is
        NaN throughout."""
        if weight.dtype != torch.float16 or weight.dim() != 2:
            raise ValueError("weight must be an fp16 matrix")
        w = cls.__new__(cls)
        w._shape(weight.shape[0], weight.shape[1], group, zeros, weight.device)
        w._allocate(bias)
        weight = weight.contiguous()
        binding._check(binding.lib().okv_linear4_quantize(w.packed.data_ptr(), weight.data_ptr(), w.n_out, w.n_in, group, w.zeros, w._stream()))
        return w

    def _bad(self, what, t, m, width):
        raise ValueError(f"{what} must be a contiguous fp16 matrix [{m}][{width}] on {self.device}, it is {t.dtype} {list(t.shape)} on {t.device}")

    def __call__(self, x, out, relu=False, residual=None):
        """out = act(x W^T + bias) + residual: x fp16 [m][n_in], out fp16 [m][n_out] or a list of up to three tensors that share the
        output features, in order.  Products of one Linear4 that may run at the same time need copies of it (they share its workspace)."""
        # A call is 5 us of host time, with kernels of as little: checks are written out, and what depends on the shape alone is kept.
        m, half, device = x.shape[0], torch.float16, self.device
        if x.dtype is not half or x.shape != (m, self.n_in) or not x.is_contiguous() or x.device != device:
            self._bad("x", x, m, self.n_in)
        if type(out) in (list, tuple):
            n = len(out)
            if not 1 <= n <= 3:
                raise ValueError("one to three output tensors")
            for o in out:
                if o.dtype is not half or o.dim() != 2 or o.shape[0] != m or not o.is_contiguous() or o.device != device:
                    self._bad("out", o, m, "width")
            arr, cols = (ctypes.c_void_p * n)(*[o.data_ptr() for o in out]), (ctypes.c_int32 * n)(*[o.shape[1] for o in out])
        else:
            n, cols = 1, None
            if out.dtype is not half or out.shape != (m, self.n_out) or not out.is_contiguous() or out.device != device:
                self._bad("out", out, m, self.n_out)
            arr = _One(out.data_ptr())
        if residual is not None and (residual.dtype is not half or residual.shape != (m, self.n_out) or not residual.is_contiguous() or residual.device != device):
            self._bad("residual", residual, m, self.n_out)
        if m == 0:
            return out
        want = self._wants.get(m)
        if want is None:
            want = self._wants[m] = max(0, int(binding.lib().okv_linear4_workspace_bytes(m, self.n_out, self.n_in)))
        ws = self.workspace
        if want and (ws is None or self._workspace_bytes < want):
            if ws is not None:
                self._outgrown.append(ws)                    # captured graphs may write to it for as long as this matrix is there
            ws = self.workspace = torch.empty(want, dtype=torch.uint8, device=device)
            self._workspace_bytes = want
        rc = self._call(x.data_ptr(), self._packed_at, self._bias_at, None if residual is None else residual.data_ptr(), arr, cols, n, m, self.n_out, self.n_in,
                        self.group, self.zeros, 1 if relu else 0, None if ws is None else ws.data_ptr(), self._workspace_bytes, self._stream())
        if rc:
            binding._check(rc)
        return out
