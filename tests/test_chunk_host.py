"""Steps with several tokens a sequence without a GPU: what the headers declare is exported, and every refusal of bad arguments.  No call here reaches a kernel."""
import ctypes
import os
import re

import pytest

from paper_2504_11816_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("header,names", [("okv_chunk.h", binding.CHUNK_EXPORTS), ("okv_sample.h", binding.SAMPLE_EXPORTS)])
def test_headers_and_exports_agree(header, names):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(okv_[a-z_0-9]+)\s*\(", text))) == sorted(names)
    for n in names:
        assert hasattr(binding.lib(), n)


def pool(**kw):
    c = binding.OkvLayerPool(n_q_heads=8, n_kv_heads=4, head_dim=64, block_tokens=64, max_blocks_per_seq=4, max_ctx=0, max_seqs=8, n_blocks=40, pool=1 << 20, block_table=1 << 20)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows(**kw):
    r = binding.OkvRows(batch=4, n_rows=10, starts=16, lens=16)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def chunk(**kw):
    a = binding.OkvChunk(workspace=1 << 20, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def append(c=None, r=None, rope=None, k=16, v=16, kv=256, q=16, qs=512, out=16, os=512):
    return binding.lib().okv_rope_append(ctypes.byref(c or pool()), ctypes.byref(r or rows()), ctypes.byref(rope) if rope else None, k, v, kv, q, qs, out, os, None)


def attend(c=None, r=None, a=None, q=16, qs=512, out=1 << 20):
    return binding.lib().okv_chunk_attn(ctypes.byref(c or pool()), ctypes.byref(r or rows()), ctypes.byref(a or chunk()), q, qs, out, None)


BAD_SHAPE = [dict(n_q_heads=6), dict(n_q_heads=0), dict(n_q_heads=68), dict(n_kv_heads=0), dict(n_kv_heads=2000, n_q_heads=2000), dict(head_dim=96), dict(head_dim=0),
             dict(block_tokens=8), dict(block_tokens=48), dict(block_tokens=2048), dict(block_tokens=-16), dict(max_blocks_per_seq=0), dict(max_blocks_per_seq=1 << 25),
             dict(max_seqs=0), dict(n_blocks=0), dict(n_blocks=1 << 31), dict(block_tokens=0, max_ctx=0), dict(block_tokens=0, max_ctx=24)]


@pytest.mark.parametrize("bad", [*BAD_SHAPE, dict(pool=None), dict(pool=(1 << 20) + 8), dict(block_table=None)], ids=str)
def test_bad_pools_are_refused(bad):
    c = pool(**bad)
    assert append(c) == attend(c) == binding.OKV_EINVAL
    assert (binding.lib().okv_chunk_workspace_bytes(ctypes.byref(c)) == binding.OKV_EINVAL) == (bad in BAD_SHAPE)


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(batch=4097), dict(n_rows=-1), dict(starts=None), dict(lens=None), dict(batch=9)], ids=str)
def test_bad_rows_are_refused(bad):
    assert append(r=rows(**bad)) == attend(r=rows(**bad)) == binding.OKV_EINVAL


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(k=8), dict(v=24), dict(kv=255), dict(kv=248), dict(kv=260), dict(q=None), dict(out=None), dict(q=8), dict(out=8), dict(qs=504),
                                 dict(os=516), dict(os=520, out=16, q=16), dict(rope=binding.OkvRope(16, 24)), dict(rope=binding.OkvRope(16, 80)), dict(rope=binding.OkvRope(16, -16)),
                                 dict(rope=binding.OkvRope(None, 64))], ids=str)
def test_bad_appends_are_refused(bad):
    assert append(**bad) == binding.OKV_EINVAL


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(q=8), dict(out=24), dict(qs=504), dict(qs=516), *[dict(a=chunk(**{n: x})) for n in ("scale", "cap") for x in (-1.0, INF, NAN)],
                                 dict(a=chunk(window=-1)), dict(a=chunk(out_dtype=2)), dict(a=chunk(out_dtype=-1)), dict(r=rows(n_rows=1 << 30))], ids=str)
def test_bad_attentions_are_refused(bad):
    assert attend(**bad) == binding.OKV_EINVAL


def test_calls_over_nothing_do_nothing():
    for r in (rows(batch=0), rows(n_rows=0)):
        assert append(r=r, k=None, v=None, q=None, out=None) == attend(r=r, q=None, out=None) == 0
    assert binding.lib().okv_token_probs(None, 0, 100, None, None, 100, 0, 100, None, 0, None) == 0
    assert binding.lib().okv_verify(None, 100, None, 100, None, None, None, None, None, None, 0, 0, 100, None, 0, None) == 0


def probs(logits=16, dtype=0, stride=100, t=16, out=16, out_stride=100, n=3, vocab=100, ws=1 << 20, size=1 << 40):
    return binding.lib().okv_token_probs(logits, dtype, stride, t, out, out_stride, n, vocab, ws, size, None)


@pytest.mark.parametrize("bad", [dict(logits=None), dict(logits=17), dict(logits=18, dtype=1), dict(out=None), dict(out=18), dict(dtype=2), dict(stride=99), dict(out_stride=99), dict(n=-1),
                                 dict(n=(1 << 20) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(t=18)], ids=str)
def test_bad_probabilities_are_refused(bad):
    assert probs(**bad) == binding.OKV_EINVAL


def verify(target=16, ts=100, q=16, qs=100, drafts=16, starts=16, u=16, tokens=16, accepted=16, rejected=16, batch=3, n=4, vocab=100, ws=1 << 20, size=1 << 40):
    return binding.lib().okv_verify(target, ts, q, qs, drafts, starts, u, tokens, accepted, rejected, batch, n, vocab, ws, size, None)


@pytest.mark.parametrize("bad", [dict(target=None), dict(drafts=None), dict(starts=None), dict(u=None), dict(tokens=None), dict(accepted=None), dict(target=18), dict(q=18), dict(drafts=18),
                                 dict(starts=18), dict(u=18), dict(tokens=18), dict(accepted=18), dict(rejected=18), dict(ts=99), dict(qs=99), dict(batch=-1), dict(batch=4097), dict(n=-1),
                                 dict(vocab=0), dict(vocab=(1 << 24) + 1)], ids=str)
def test_bad_verifications_are_refused(bad):
    assert verify(**bad) == binding.OKV_EINVAL


def test_small_workspaces_are_refused():
    for vocab in (1, 100, 32000, 1 << 24):
        need = binding.lib().okv_verify_workspace_bytes(3, vocab)
        assert need > 0 and binding.lib().okv_verify_workspace_bytes(0, vocab) == 0
        for kw in (dict(size=need - 1), dict(ws=None), dict(ws=24)):
            assert verify(vocab=vocab, ts=vocab, qs=vocab, **kw) == binding.OKV_ENOSPC
    need = binding.lib().okv_chunk_workspace_bytes(ctypes.byref(pool()))
    if need:
        for kw in (dict(workspace_bytes=need - 1), dict(workspace=None), dict(workspace=128)):
            assert attend(a=chunk(**kw)) == binding.OKV_ENOSPC


def test_shrinking_without_its_numbers_is_refused():
    p = binding.OkvPages(n_layers=1, page_tokens=16, max_seqs=4, max_pages_per_seq=4, n_pages=16, table=16, lens=16, refs=16, status=16, workspace=16, workspace_bytes=1 << 30)
    assert binding.lib().okv_pages_shrink(ctypes.byref(p), 2, 16, None, None) == binding.lib().okv_pages_shrink(ctypes.byref(p), -1, 16, 16, None) == binding.OKV_EINVAL
    assert binding.lib().okv_pages_shrink(ctypes.byref(p), 5, None, 16, None) == binding.lib().okv_pages_shrink(ctypes.byref(p), 4097, 16, 16, None) == binding.OKV_EINVAL
    assert binding.lib().okv_pages_shrink(ctypes.byref(p), 0, None, None, None) == 0
