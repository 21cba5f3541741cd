"""Decoder layers whose weights are held in 4 bits over a KV cache held in 8: the same steps as harness.decode_step_with_layers, with a quarter
of the bytes of the weights and half of those of the keys and values.

    layers = [CompressedLayer(w, group=128) for w in weights]              # harness.LayerWeights, or anything with the same tensors in .t
    scratch = Scratch(max_batch, h1, h2, kv_cols, device)
    decoder_step(cache, layers, scratch, x, seqs)                          # x fp16 [batch][h1]: a token's embeddings in, the last layer's output out
"""
import torch

from . import binding
from .cache8 import need
from .linear4 import Linear4


class CompressedLayer:
    """One decoder layer: its six matrices quantised in groups (query, key and value stacked), norms and biases as they are."""

    def __init__(self, weights, group=128, zeros=False):
        t = self.t = weights.t
        h1, kv, h2 = self.h1, self.kv_cols, self.h2 = t["wq"].shape[1], t["wk"].shape[0], t["w1"].shape[0]
        for name, shape in (("wq", (h1, h1)), ("wk", (kv, h1)), ("wv", (kv, h1)), ("wo", (h1, h1)), ("w1", (h2, h1)), ("w2", (h1, h2))):
            if tuple(t[name].shape) != shape:
                raise ValueError(f"{name} must be {list(shape)}, it is {list(t[name].shape)}")
        for name in ("ln1_g", "ln1_b", "ln2_g", "ln2_b"):
            need(name, t[name], torch.float16, (h1,), t["wq"].device)
        self.qkv = Linear4.quantize(torch.cat([t["wq"], t["wk"], t["wv"]]), group, zeros, torch.cat([t["bq"], t["bk"], t["bv"]]))
        self.o = Linear4.quantize(t["wo"], group, zeros, t["bo"])
        self.ff1 = Linear4.quantize(t["w1"], group, zeros, t["b1"])
        self.ff2 = Linear4.quantize(t["w2"], group, zeros, t["b2"])

    def packed_bytes(self):
        return sum(w.packed.numel() for w in (self.qkv, self.o, self.ff1, self.ff2))


class Scratch:
    """Activations of a step of up to max_batch sequences (fp16), used by every layer in turn."""

    def __init__(self, max_batch, h1, h2, kv_cols, device):
        def buf(cols):
            return torch.empty((max_batch, cols), dtype=torch.float16, device=device)
        self.a, self.q, self.k, self.v = buf(h1), buf(h1), buf(kv_cols), buf(kv_cols)
        self.t, self.y, self.z, self.u = buf(h1), buf(h1), buf(h1), buf(h2)

    def rows(self, batch):
        if batch > self.a.shape[0]:
            raise ValueError(f"the scratch has room for {self.a.shape[0]} sequences")
        return (b[:batch] for b in (self.a, self.q, self.k, self.v, self.t, self.y, self.z, self.u))


def _check(cache, layers, scratch, x, seqs):
    """Raises before anything has changed: lengths that have grown, or layers that have appended, would stay so."""
    B, h1, kv = x.shape[0], cache.H * cache.d, cache.G * cache.d
    need("x", x, torch.float16, (B, h1), cache.device)
    need("seqs", seqs, torch.int32, (B,), cache.device)
    if cache.out_dtype is not torch.float16:
        raise ValueError("the cache's results go into products: out_dtype must be torch.float16")
    h2 = scratch.u.shape[1]
    if len(layers) != cache.L or any(w.h1 != h1 or w.kv_cols != kv or w.h2 != h2 for w in layers):
        raise ValueError(f"there must be {cache.L} layers of widths {h1}, {kv} and {h2}, as the cache and the scratch have them")
    if scratch.a.shape[1] != h1 or scratch.k.shape[1] != kv or scratch.a.device != cache.device:
        raise ValueError(f"the scratch must be for widths {h1} and {kv}, on {cache.device}")


def decoder_step(cache, layers, scratch, x, seqs, eps=1e-5):
    """One token for each of the sequences `seqs` (int32 rows of the cache's table): their lengths grow by one, and every layer appends its key and value
    and attends.  x fp16 [batch][h1], overwritten with the last layer's output.  Nothing waits or allocates on the GPU's side; a cache that is out of pages
    says so in cache.pages.check(): it is then as it was before the step, and x means nothing.  Arguments that do not fit raise a ValueError, and change
    nothing."""
    rows = scratch.rows(x.shape[0])
    _check(cache, layers, scratch, x, seqs)
    B, stream = x.shape[0], binding.current_stream(x.device)
    a, q, k, v, t, y, z, u = rows
    h1 = x.shape[1]
    cache.pages.extend(seqs)
    cache.begin(B, cache.lens, seqs)
    for l, w in enumerate(layers):
        binding.okv_layernorm(x, w.t["ln1_g"], w.t["ln1_b"], a, B, h1, eps, stream)
        w.qkv(a, [q, k, v])
        cache.attend(l, q.view(B, cache.H, cache.d), k.view(B, cache.G, cache.d), v.view(B, cache.G, cache.d), t.view(B, cache.H, cache.d))
        w.o(t, y, residual=x)
        binding.okv_layernorm(y, w.t["ln2_g"], w.t["ln2_b"], z, B, h1, eps, stream)
        w.ff1(z, u, relu=True)
        w.ff2(u, x, residual=y)
