"""Linear layers with 4-bit weights and group scales (include/okv_linear4.h) over torch-owned memory.

    w = Linear4.quantize(weight, group=128)           # fp16 [n_out][n_in], as a framework's linear layer has it
    w = Linear4(codes, scales, zeros, bias)           # quantised elsewhere
    w(x, out, relu=True)                              # out = relu(x W^T + bias)
    qkv(x, [q, k, v])                                 # the output features in up to three tensors
    w(x, y, residual=y)                               # y += x W^T + bias
"""
import ctypes

import torch

from . import binding


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

    @staticmethod
    def _stream():
        return torch.cuda.current_stream().cuda_stream

    def _allocate(self, bias):
        n = int(binding.lib().okv_linear4_packed_bytes(self.n_out, self.n_in, self.group, self.zeros))
        binding._check(min(n, 0))
        if bias is not None and (bias.dtype != torch.float16 or tuple(bias.shape) != (self.n_out,) or bias.device != self.device or not bias.is_contiguous()):
            raise ValueError(f"bias must be a contiguous fp16 vector of {self.n_out} on {self.device}")
        self.bias = bias
        self.packed = torch.empty(n, dtype=torch.uint8, device=self.device)
        self.workspace = None
        self._call = binding.lib().okv_linear4

    @classmethod
    def quantize(cls, weight, group=128, zeros=False, bias=None):
        """Quantises fp16 [n_out][n_in] weights, every group by itself (see the header)."""
        if weight.dtype != torch.float16 or weight.dim() != 2:
            raise ValueError("weight must be an fp16 matrix")
        w = cls.__new__(cls)
        w._shape(weight.shape[0], weight.shape[1], group, zeros, weight.device)
        w._allocate(bias)
        weight = weight.contiguous()
        binding._check(binding.lib().okv_linear4_quantize(w.packed.data_ptr(), weight.data_ptr(), w.n_out, w.n_in, group, w.zeros, w._stream()))
        return w

    def __call__(self, x, out, relu=False, residual=None):
        """out = act(x W^T + bias) + residual: x fp16 [m][n_in], out fp16 [m][n_out] or a list of up to three tensors that share the
        output features, in order.  Products of one Linear4 that may run at the same time need copies of it (they share its workspace)."""
        outs = out if isinstance(out, (list, tuple)) else (out,)
        m, n = x.shape[0], len(outs)
        if not 1 <= n <= 3:
            raise ValueError("one to three output tensors")
        for t, width in ((x, self.n_in), *((o, None) for o in outs), *(((residual, self.n_out),) if residual is not None else ())):
            if t.dtype != torch.float16 or t.dim() != 2 or t.shape[0] != m or (width is not None and t.shape[1] != width) or not t.is_contiguous() or t.device != self.device:
                raise ValueError(f"x, out and residual must be contiguous fp16 matrices of {m} rows on {self.device}, of the layer's widths")
        if m == 0:
            return out
        arr = (ctypes.c_void_p * n)(*[o.data_ptr() for o in outs])
        cols = (ctypes.c_int32 * n)(*[o.shape[1] for o in outs])
        want = binding.lib().okv_linear4_workspace_bytes(m, self.n_out, self.n_in)
        if want > 0 and (self.workspace is None or self.workspace.numel() < want):
            self.workspace = torch.empty(want, dtype=torch.uint8, device=self.device)
        ws = self.workspace
        binding._check(self._call(x.data_ptr(), self.packed.data_ptr(), self.bias.data_ptr() if self.bias is not None else None,
                                  residual.data_ptr() if residual is not None else None, arr, cols, n, m, self.n_out, self.n_in, self.group, self.zeros,
                                  int(relu), ws.data_ptr() if ws is not None else None, ws.numel() if ws is not None else 0, self._stream()))
        return out
