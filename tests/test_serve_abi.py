"""Refusals of the chunk calls and the sampler (include/nightjar_serve.h): bad
arguments are found on the host before anything is enqueued, and the reference
that the GPU tests use agrees with the format's definition."""
import ctypes
import os

import numpy as np
import pytest

import serve_ref as ref
from paper_2512_22420_amd import binding as nb
from paper_2512_22420_amd import workload as W
from paper_2512_22420_amd.device import model_desc

pytestmark = pytest.mark.skipif(not os.path.exists(nb.LIB_PATH), reason="libnightjar.so not built")

BF = model_desc(W.LLAMA8B_LAYER)
F32 = model_desc(W.TINY_F32)
BIG = 1 << 40


def _layer(dtype=nb.NJ_BF16, scale=256, blocks=4, k=256, v=256):
    return nb.KvLayer(k, v, scale, scale, blocks, dtype)


def _batch(starts=256, ctx=256, table=256, max_blocks=4, B=2, rows=8, max_chunk=8):
    return nb.ChunkBatch(starts, ctx, table, max_blocks, B, rows, max_chunk)


def _calls(desc, layer, batch, ws=256, n=BIG, row=256, row2=1 << 30, stride=6144):
    """Return code and message of each chunk call with these (unmapped) pointers."""
    L, c = nb.lib(), ctypes.byref
    d = c(desc) if desc is not None else None
    out = []
    for f, a in ((L.nightjar_chunk_store, (row, stride, row2)), (L.nightjar_chunk_load, (row, row2)),
                 (L.nightjar_chunk_attn, (row, row2))):
        out.append((f(d, c(layer) if layer else None, c(batch) if batch else None, *a, ws, n, 0), nb.last_error()))
    return out


@pytest.mark.parametrize("kw,word", [
    (dict(desc=None), "desc"), (dict(layer=None), "NULL"), (dict(batch=None), "NULL"),
    (dict(batch=_batch(B=0)), "B >= 1"), (dict(batch=_batch(rows=0, max_chunk=0)), "rows"),
    (dict(batch=_batch(max_chunk=0)), "max_chunk"), (dict(batch=_batch(max_chunk=9)), "max_chunk"),
    (dict(batch=_batch(rows=(1 << 24) + 1)), "2^24"), (dict(batch=_batch(max_blocks=0)), "max_blocks"),
    (dict(batch=_batch(starts=0)), "NULL"), (dict(batch=_batch(ctx=0)), "NULL"), (dict(batch=_batch(table=0)), "NULL"),
    (dict(layer=_layer(blocks=0)), "num_blocks"), (dict(layer=_layer(k=0)), "NULL"), (dict(layer=_layer(v=0)), "NULL"),
    (dict(layer=_layer(k=264)), "aligned"), (dict(layer=_layer(nb.NJ_F32)), "go with"),
    (dict(layer=_layer(7)), "go with"), (dict(desc=F32, layer=_layer(nb.NJ_BF16)), "go with"),
    (dict(layer=_layer(nb.NJ_E4M3, scale=0)), "k_scale"), (dict(layer=_layer(nb.NJ_E4M3, scale=8)), "aligned"),
    (dict(ws=0), "workspace"), (dict(n=255), "workspace"), (dict(ws=128), "aligned"), (dict(row=0), ""), (dict(row=8), "aligned"),
])
def test_chunk_calls_refuse(kw, word):
    args = {"desc": BF, "layer": _layer(), "batch": _batch()} | kw
    for rc, msg in _calls(**args):
        assert rc == nb.NJ_EINVAL and word in msg, (rc, msg)


def test_overlapping_rows_are_refused():
    c = ctypes.byref
    for f, a in ((nb.lib().nightjar_chunk_store, (4096, 6144, 4096 + 16)), (nb.lib().nightjar_chunk_load, (4096, 4096 + 16)),
                 (nb.lib().nightjar_chunk_attn, (4096, 4096 + 16))):
        assert f(c(BF), c(_layer()), c(_batch()), *a, 256, BIG, 0) == nb.NJ_EINVAL and "overlap" in nb.last_error()


def test_chunk_calls_refuse_descriptors():
    for field, value in (("n_kv_heads", 5), ("n_kv_heads", 0), ("block_size", 32), ("dtype", 2), ("head_dim", 64),
                         ("head_dim", 12), ("n_heads", 4096)):
        d = model_desc(W.LLAMA8B_LAYER)
        setattr(d, field, value)
        assert all(rc == nb.NJ_EINVAL for rc, _ in _calls(d, _layer(), _batch())), field
        assert nb.lib().nightjar_chunk_attn_workspace_bytes(ctypes.byref(d), 2, 8, 8) == 0


def test_single_call_refusals():
    L, c = nb.lib(), ctypes.byref
    k, b = _layer(), _batch()
    assert L.nightjar_chunk_store(c(BF), c(k), c(b), 256, 6140, 0, 256, BIG, 0) == nb.NJ_EINVAL and "qkv_stride" in nb.last_error()
    assert L.nightjar_chunk_store(c(BF), c(k), c(b), 256, 6146, 0, 256, BIG, 0) == nb.NJ_EINVAL and "qkv_stride" in nb.last_error()
    assert L.nightjar_chunk_store(c(BF), c(k), c(b), 256, 6144, 8, 256, BIG, 0) == nb.NJ_EINVAL and "aligned" in nb.last_error()
    d = model_desc(W.LLAMA8B_LAYER)
    d.rope_theta = 0.0
    assert L.nightjar_chunk_store(c(d), c(k), c(b), 256, 6144, 256, 256, BIG, 0) == nb.NJ_EINVAL and "rope" in nb.last_error()
    assert L.nightjar_chunk_attn(c(BF), c(k), c(b), 256, 1 << 30, 256, 255, 0) == nb.NJ_EINVAL and "workspace" in nb.last_error()
    assert L.nightjar_chunk_attn(c(BF), c(k), c(b), 256, 256 + 4096, 256, BIG, 0) == nb.NJ_EINVAL and "overlap" in nb.last_error()


def test_chunk_workspace_serves_every_smaller_batch():
    L = nb.lib()
    for desc in (BF, model_desc(W.QWEN7B), F32):
        top = L.nightjar_chunk_attn_workspace_bytes(ctypes.byref(desc), 64, 4096, 2048)
        assert top >= 256
        for B in (1, 2, 7, 33, 64):
            for rows in (1, 5, 64, 1000, 4096):
                for mc in (1, 3, 17, 500, 2048):
                    if mc <= rows:
                        n = L.nightjar_chunk_attn_workspace_bytes(ctypes.byref(desc), B, rows, mc)
                        assert 256 <= n <= top, (B, rows, mc, n, top)


def _sample(logits=256, ls=100, rows=2, V=100, u=256, tok=256, probs=0, ps=0, ws=256, n=BIG):
    return nb.lib().nightjar_sample(logits, ls, rows, V, 0, 0, 0, 0, u, tok, probs, ps, ws, n, 0), nb.last_error()


@pytest.mark.parametrize("kw,word", [
    (dict(logits=0), "NULL"), (dict(u=0), "NULL"), (dict(tok=0), "NULL"), (dict(ws=0), "NULL"), (dict(rows=0), "rows"),
    (dict(V=0), "vocab"), (dict(V=524289, ls=524289), "vocab"), (dict(ls=99), "stride"), (dict(probs=1 << 30, ps=99), "stride"),
    (dict(probs=256, ps=100), "overlap"), (dict(probs=256 + 400, ps=100), "overlap"), (dict(n=255), "workspace"),
    (dict(ws=128), "aligned")])
def test_sample_refuses(kw, word):
    rc, msg = _sample(**kw)
    assert rc == nb.NJ_EINVAL and word in msg, (rc, msg)
    assert nb.lib().nightjar_sample_workspace_bytes(0, 100) == 0
    assert nb.lib().nightjar_sample_workspace_bytes(4, 524289) == 0


def test_reference_format():
    """The reference's codes are the format's: every code's value is its own encoding, borders go to the even code,
    the scale is the smallest that holds the row."""
    assert len(ref.GRID) == 127 and ref.GRID[126] == 448.0 and ref.GRID[8] == 2.0 ** -6 and ref.GRID[1] == 2.0 ** -9
    x = np.concatenate([ref.GRID, -ref.GRID])[None].astype(np.float32)
    v, s, _ = ref.encode(x)
    assert s[0] == 127 and np.array_equal(v, x)
    v, s, _ = ref.encode(np.array([[448.0 * 2 ** -3, 0.0, np.nan, np.inf]], np.float32))
    assert s[0] == 124 and v[0, 0] == 56.0 and v[0, 1] == 0 and np.isnan(v[0, 2]) and np.isnan(v[0, 3])
    assert ref.encode(np.array([[449.0, 17.0 + 1.0]], np.float32))[1][0] == 128
    v, _, near = ref.encode(np.array([[448.0, 17.0, 19.0]], np.float32))  # codes 16, 18, 20: halfway, to the even code
    assert v[0, 1] == 16.0 and v[0, 2] == 20.0 and near[0, 1] == 0.0
    assert ref.encode(np.zeros((1, 4), np.float32))[1][0] == 15


def test_reference_sampler_against_enumeration():
    """On a grid of uniforms the reference draws each token as often as its truncated probability says."""
    rng = np.random.default_rng(3)
    l = rng.normal(size=12).astype(np.float32)
    l[4] = l[7]
    for T, k, p, m in ((1.0, 0, 1.0, 0.0), (0.7, 5, 1.0, 0.0), (1.3, 0, 0.6, 0.0), (0.9, 6, 0.8, 0.3), (0.0, 0, 1.0, 0.0)):
        n = 20000
        toks = [ref.sample(l, (i + 0.5) / n, T, k, p, m)[0] for i in range(0, n, 7)]
        _, probs = ref.sample(l, 0.1, T, k, p, m)
        freq = np.bincount(toks, minlength=12) / len(toks)
        assert abs(probs.sum() - 1) < 1e-12 and np.abs(freq - probs).max() < 2e-3  # one grid step in 2858
        assert (probs > 0).sum() == (1 if T == 0 else k if k and p == 1 else (probs > 0).sum())
