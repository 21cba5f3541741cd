"""4-bit weights, written out from their definition (oracle side).

TEST INFRASTRUCTURE ONLY; shares no code with the HIP library.
"""
import numpy as np


def quantise(w, group, zeros):
    """fp16 [n_out][n_in] -> the fp64 values of the quantised weights.  Every group by itself, in fp32, the scale rounded to fp16;
    NaN where a weight is infinite or NaN."""
    n_out, n_in = w.shape
    t = w.astype(np.float32).reshape(n_out, -1, group)
    lo, hi = np.minimum(t.min(-1), 0), np.maximum(t.max(-1), 0)
    s = ((hi - lo) / np.float32(15) if zeros else np.maximum(hi, -lo) / np.float32(7)).astype(np.float16).astype(np.float32)
    s = np.where(np.isfinite(t).all(-1), s, np.float32(np.nan))
    safe = np.where(s > 0, s, np.float32(1))
    z = np.where(s > 0, np.minimum(np.rint(-lo / safe), 15), 8) if zeros else np.full_like(s, 8)
    code = np.clip(np.rint(np.where(s[..., None] > 0, t / safe[..., None], 0)) + z[..., None], 0, 15)
    return ((code - z[..., None]).astype(np.float64) * s[..., None]).reshape(n_out, n_in)
