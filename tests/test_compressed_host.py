"""The 8-bit cache, its pages and the 4-bit products without a GPU: what the headers declare is exported, every refusal of bad arguments, and the
oracles on closed forms.  No call here reaches a kernel."""
import ctypes
import math
import os
import re
from fractions import Fraction

import numpy as np
import pytest

from oracle import cache8 as oracle8
from oracle import pages as oracle_pages
from paper_2504_11816_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("header,prefix,names", [("okv_cache8.h", "okv8_", binding.CACHE8_EXPORTS), ("okv_pages.h", "okv_pages_", binding.PAGES_EXPORTS),
                                                 ("okv_linear4.h", "okv_linear4", binding.LINEAR4_EXPORTS)])
def test_headers_and_exports_agree(header, prefix, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    declared = {n for n in re.findall(r"\b([a-z_0-9]+)\s*\(", text) if n.startswith(prefix)}
    assert sorted(declared) == sorted(names)
    for n in names:
        assert hasattr(binding.lib(), n)


def cache(**kw):
    c = binding.Okv8Cache(n_layers=2, n_q_heads=8, n_kv_heads=4, head_dim=64, page_tokens=64, format=0, out_dtype=0, max_seqs=8, max_pages_per_seq=4,
                          n_pages=40, codes=1 << 20, scales=1 << 20, tails=1 << 20, page_table=1 << 20)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHE = [dict(n_layers=0), dict(n_q_heads=6), dict(n_q_heads=0), dict(n_q_heads=68), dict(n_kv_heads=0), dict(n_kv_heads=2000, n_q_heads=2000),
             dict(head_dim=96), dict(page_tokens=16), dict(page_tokens=48), dict(page_tokens=2048), dict(format=2), dict(format=-1), dict(out_dtype=2),
             dict(max_seqs=0), dict(max_pages_per_seq=0), dict(max_pages_per_seq=1 << 26), dict(n_pages=0), dict(n_pages=1 << 31)]


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_bad_caches_are_refused(bad):
    L, c = binding.lib(), cache(**bad)
    for fn in (L.okv8_codes_bytes, L.okv8_scales_bytes, L.okv8_tails_bytes):
        assert fn(ctypes.byref(c)) == binding.OKV_EINVAL
    assert L.okv8_workspace_bytes(ctypes.byref(c), 1) == binding.OKV_EINVAL
    assert L.okv8_store(ctypes.byref(c), 0, 1, 1, None, 16, 16, 4, 16, 16, 256, 0, None) == binding.OKV_EINVAL
    s = step(c)
    assert L.okv8_step_begin(ctypes.byref(c), ctypes.byref(s)) == binding.OKV_EINVAL


def step(c, **kw):
    s = binding.Okv8Step(batch=4, appends=1, lens=16, workspace=256, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def test_sizes_of_the_buffers():
    L, c = binding.lib(), cache()
    assert L.okv8_codes_bytes(ctypes.byref(c)) == 2 * 40 * 64 * 2 * 4 * 64
    assert L.okv8_scales_bytes(ctypes.byref(c)) == 2 * 40 * 2 * 4 * 2 * 4
    assert L.okv8_tails_bytes(ctypes.byref(c)) == 2 * 8 * 2 * 4 * 32 * 64 * 2
    assert L.okv8_workspace_bytes(ctypes.byref(c), 8) > L.okv8_workspace_bytes(ctypes.byref(c), 1) > 0
    assert L.okv8_workspace_bytes(ctypes.byref(c), 0) == L.okv8_workspace_bytes(ctypes.byref(c), 4097) == binding.OKV_EINVAL
    assert L.okv8_codes_bytes(None) == binding.OKV_EINVAL


@pytest.mark.parametrize("args", [dict(codes=0), dict(scales=0), dict(tails=0), dict(page_table=0), dict(codes=(1 << 20) + 8)], ids=str)
def test_null_and_misaligned_buffers_are_refused(args):
    L, c = binding.lib(), cache(**args)
    s = step(c)
    assert L.okv8_step_begin(ctypes.byref(c), ctypes.byref(s)) == binding.OKV_EINVAL
    assert L.okv8_load(ctypes.byref(c), 0, 1, 1, None, 16, 16, 4, 16, 16, 256, 0, None) == binding.OKV_EINVAL


@pytest.mark.parametrize("bad,code", [(dict(batch=0), -1), (dict(batch=9), -1), (dict(appends=2), -1), (dict(lens=0), -1), (dict(workspace=0), -1),
                                      (dict(workspace=16), -1), (dict(workspace_bytes=1000), -2)], ids=str)
def test_bad_steps_are_refused(bad, code):
    L, c = binding.lib(), cache()
    s = step(c, **bad)
    assert L.okv8_step_begin(ctypes.byref(c), ctypes.byref(s)) == code
    assert L.okv8_decode_attn(ctypes.byref(c), ctypes.byref(s), 0, 16, 512, 16, 16, 256, 16) == code
    assert L.okv8_decode_step(ctypes.byref(c), ctypes.byref(s), 16, 16, 16, 16) == code
    assert binding.lib().okv_last_error(None)


def test_a_step_beyond_32_bits_is_refused():
    L = binding.lib()
    c = cache(max_seqs=4096, max_pages_per_seq=1 << 20, page_tokens=1024, n_pages=1 << 22)
    s = step(c, batch=4096)
    assert L.okv8_step_begin(ctypes.byref(c), ctypes.byref(s)) == binding.OKV_EINVAL


@pytest.mark.parametrize("args", [dict(layer=2), dict(layer=-1), dict(q=0), dict(q=8), dict(q_stride=511), dict(q_stride=504), dict(k=0), dict(v=0), dict(k=24),
                                  dict(kv_stride=248), dict(kv_stride=260), dict(out=0), dict(out=4), dict(appends=0)], ids=str)
def test_bad_attention_calls_are_refused(args):
    a = dict(layer=0, q=16, q_stride=512, k=16, v=16, kv_stride=256, out=16, appends=1)
    a.update(args)
    c = cache()
    s = step(c, appends=a["appends"])
    assert binding.lib().okv8_decode_attn(ctypes.byref(c), ctypes.byref(s), a["layer"], a["q"], a["q_stride"], a["k"], a["v"], a["kv_stride"],
                                          a["out"]) == binding.OKV_EINVAL


@pytest.mark.parametrize("args", [dict(layer=-1), dict(layer=2), dict(n_layers=0), dict(n_layers=3), dict(batch=0), dict(batch=9), dict(starts=0), dict(lens=0),
                                  dict(n_rows=-1), dict(n_rows=1 << 31), dict(k=0), dict(v=8), dict(row=128), dict(row=260), dict(layer_stride=4)], ids=str)
def test_bad_row_calls_are_refused(args):
    a = dict(layer=0, n_layers=2, batch=2, starts=16, lens=16, n_rows=10, k=16, v=16, row=256, layer_stride=2560)
    a.update(args)
    for fn in (binding.lib().okv8_store, binding.lib().okv8_load):
        assert fn(ctypes.byref(cache()), a["layer"], a["n_layers"], a["batch"], None, a["starts"], a["lens"], a["n_rows"], a["k"], a["v"], a["row"],
                  a["layer_stride"], None) == binding.OKV_EINVAL


def pages(**kw):
    p = binding.OkvPages(n_layers=2, page_tokens=32, max_seqs=4, max_pages_per_seq=4, n_pages=10, n_arrays=1, n_rows=1, table=16, lens=16, refs=16, status=16,
                         workspace=16, workspace_bytes=1 << 30)
    p.arrays[0] = binding.OkvPageArray(1 << 20, 4096, 1 << 16, 32, 1)
    p.rows[0] = binding.OkvRowArray(1 << 20, 1 << 16, 4, 32, 128)
    for k, v in kw.items():
        target = p
        *path, last = k.split("__")
        for name in path:
            target = getattr(target, name)[0]
        setattr(target, last, v)
    return p


@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(page_tokens=24), dict(page_tokens=2048), dict(max_seqs=0), dict(max_pages_per_seq=0), dict(n_pages=0),
                                 dict(max_pages_per_seq=1 << 27), dict(n_arrays=5), dict(n_rows=3), dict(table=0), dict(lens=0), dict(refs=0), dict(status=0),
                                 dict(workspace=0), dict(workspace=8), dict(workspace_bytes=64), dict(arrays__base=0), dict(arrays__page_bytes=0),
                                 dict(arrays__page_bytes=4098), dict(arrays__unit_tokens=0), dict(arrays__unit_tokens=64), dict(arrays__unit_tokens=3),
                                 dict(arrays__layer_stride=2), dict(arrays__page_bytes=1 << 31), dict(rows__base=0), dict(rows__groups=0), dict(rows__rows=0),
                                 dict(rows__row_bytes=6), dict(rows__layer_stride=2)], ids=str)
def test_bad_pages_are_refused(bad):
    L, p = binding.lib(), pages(**bad)
    assert L.okv_pages_extend(ctypes.byref(p), 1, 16, 16, None) == binding.OKV_EINVAL
    assert L.okv_pages_fork(ctypes.byref(p), 1, 16, 16, None) == binding.OKV_EINVAL
    assert L.okv_pages_free(ctypes.byref(p), 1, 16, None) == binding.OKV_EINVAL
    assert L.okv_pages_compact(ctypes.byref(p), None) == binding.OKV_EINVAL
    assert L.okv_pages_copy(ctypes.byref(p), 1, 16, 16, p.arrays, 10, None) == binding.OKV_EINVAL


def test_bad_page_calls_are_refused():
    L, p = binding.lib(), pages()
    r = ctypes.byref(p)
    assert L.okv_pages_extend(r, -1, 16, 16, None) == L.okv_pages_extend(r, 4097, 16, 16, None) == L.okv_pages_extend(r, 5, None, None, None) == binding.OKV_EINVAL
    assert L.okv_pages_fork(r, 1, None, 16, None) == L.okv_pages_fork(r, 1, 16, None, None) == L.okv_pages_fork(r, 4097, 16, 16, None) == binding.OKV_EINVAL
    assert L.okv_pages_free(r, 1, None, None) == L.okv_pages_free(r, 4097, 16, None) == binding.OKV_EINVAL
    assert L.okv_pages_copy(r, 1, None, 16, p.arrays, 10, None) == L.okv_pages_copy(r, 1, 16, 16, p.arrays, 0, None) == binding.OKV_EINVAL
    other = (binding.OkvPageArray * 1)(binding.OkvPageArray(16, 8192, 0, 32, 1))
    assert L.okv_pages_copy(r, 1, 16, 16, other, 10, None) == binding.OKV_EINVAL
    assert L.okv_pages_workspace_bytes(0) == binding.OKV_EINVAL and L.okv_pages_workspace_bytes(100) > 0
    # nothing to do: no launch, no error
    assert L.okv_pages_extend(r, 0, 16, 16, None) == L.okv_pages_fork(r, 0, None, None, None) == L.okv_pages_free(r, 0, None, None) == 0


@pytest.mark.parametrize("bad", [dict(m=0), dict(m=4097), dict(n_out=24), dict(n_out=0), dict(n_in=48), dict(n_in=96, group=64), dict(group=16), dict(n_seg=0),
                                 dict(n_seg=4), dict(n_seg=2, residual=16), dict(x=0), dict(packed=8), dict(bias=8), dict(out=[0]), dict(out=[8]),
                                 dict(n_seg=2, cols=[48, 40]), dict(n_seg=2, cols=[32, 32]), dict(n_seg=2, cols=[-32, 128])], ids=str)
def test_bad_products_are_refused(bad):
    a = dict(x=16, packed=16, bias=None, residual=None, out=[16, 16, 16], cols=None, n_seg=1, m=4, n_out=96, n_in=128, group=32)
    a.update(bad)
    out = (ctypes.c_void_p * 4)(*a["out"])
    cols = None if a["cols"] is None else (ctypes.c_int32 * 3)(*a["cols"])
    assert binding.lib().okv_linear4(a["x"], a["packed"], a["bias"], a["residual"], out, cols, a["n_seg"], a["m"], a["n_out"], a["n_in"], a["group"], 0, 0, None, 0,
                                     None) == binding.OKV_EINVAL


def test_bad_weights_are_refused():
    L = binding.lib()
    assert L.okv_linear4_packed_bytes(96, 1056, 32, 1) == 6 * 9 * 1024 + 96 * 36 * 3
    for n_out, n_in, group in ((24, 128, 32), (96, 100, 32), (96, 96, 64), (96, 128, 48), (0, 128, 32), (96, 0, 32)):
        assert L.okv_linear4_packed_bytes(n_out, n_in, group, 0) == binding.OKV_EINVAL
        assert L.okv_linear4_pack(16, 16, 1, 16, None, n_out, n_in, group, None) == binding.OKV_EINVAL
        assert L.okv_linear4_quantize(16, 16, n_out, n_in, group, 0, None) == binding.OKV_EINVAL
    assert L.okv_linear4_pack(16, 16, 3, 16, None, 96, 128, 32, None) == L.okv_linear4_pack(8, 16, 1, 16, None, 96, 128, 32, None) == binding.OKV_EINVAL
    assert L.okv_linear4_pack(0, 16, 1, 16, None, 96, 128, 32, None) == L.okv_linear4_quantize(16, 8, 96, 128, 32, 0, None) == binding.OKV_EINVAL
    assert L.okv_linear4_workspace_bytes(0, 96, 128) == L.okv_linear4_workspace_bytes(4, 90, 128) == binding.OKV_EINVAL


# ---- the oracles ------------------------------------------------------------------------------------

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_codes_are_nearest_by_exact_arithmetic(fmt):
    """Against Fractions and the list of all codes: nearest, ties to the even code."""
    grid = sorted({oracle8.value(b, fmt) for b in range(256) if not (fmt == "e4m3" and b & 127 == 127)} - ({-128} if fmt == "int8" else set()))
    rng = np.random.default_rng(3)
    for case in range(6):
        x = (rng.standard_normal((32, 64)) * 10.0 ** rng.integers(-4, 4)).astype(np.float16)
        if case == 1:
            x[3, 5] = 65504
        if case == 2:
            x = (rng.integers(-3, 4, (32, 64)) * 2.0 ** -24).astype(np.float16)
        codes, s = oracle8.quantise_tile(x, fmt)
        assert np.abs(codes).max() <= oracle8.MOST[fmt]
        m, _ = math.frexp(s)
        assert m * 4096 == int(m * 4096)
        for v, c in list(zip(x.reshape(-1), codes.reshape(-1)))[::7]:
            y = Fraction(float(v)) / Fraction(s)
            d = min(abs(y - Fraction(g)) for g in grid)
            near = [g for g in grid if abs(y - Fraction(g)) == d]
            assert abs(y - Fraction(float(c))) == d
            if len(near) == 2 and fmt == "int8":
                assert c % 2 == 0


def test_attention_oracle_on_closed_forms():
    rng = np.random.default_rng(1)
    k = np.zeros((40, 1, 64))
    v = rng.integers(-5, 6, (40, 1, 64)).astype(np.float64)
    out = oracle8.attend(np.ones((2, 64)), k, v, 20, "int8", True)      # equal scores: the mean
    np.testing.assert_allclose(out, np.tile(v[:20, 0].mean(0), (2, 1)))
    assert (oracle8.attend(np.ones((2, 64)), k, v, 0, "int8", False) == 0).all()


def test_page_model_shares_and_returns_pages():
    m = oracle_pages.Model(10, 4, 4, 4)
    m.extend([0], [10])
    assert m.table[0] == [0, 1, 2, -1] and m.fork([0, 0], [1, 3]) == [(2, 3, 2), (2, 4, 2)]
    assert m.refs == [3, 3, 1, 1, 1, 0, 0, 0, 0, 0]
    m.free([0])
    assert m.refs == [2, 2, 0, 1, 1, 0, 0, 0, 0, 0] and m.compact() == [(4, 2)] and m.table[3] == [0, 1, 2, -1]
