"""The norm + rotation + append, prefill and shared-prefix calls of the C ABI reject bad arguments on
the host, before anything is launched; their workspace sizes; and the host-side frequencies."""

import ctypes
import math
import os

import numpy as np
import pytest
import torch

import paper_2608_15473_amd as qf
from paper_2608_15473_amd.binding import DecodeDesc, Rope, load_library

needs_lib = pytest.mark.skipif(not os.path.exists(qf.LIB_PATH), reason="libqfattn.so not built")
A, OFF8, OFF2 = ctypes.c_void_p(4096), ctypes.c_void_p(4104), ctypes.c_void_p(4098)


def _desc(**kw):
    base = dict(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=128, page_size=16, max_pages_per_seq=8,
                num_pages=16, max_shards=1, softmax_scale=1 / math.sqrt(128))
    base.update(kw)
    return DecodeDesc(**base)


BAD_DESC = [(dict(batch=-1), qf.QF_EINVAL), (dict(n_q_heads=3), qf.QF_EINVAL),
            (dict(n_q_heads=32), qf.QF_EUNSUPPORTED), (dict(head_dim=64), qf.QF_EUNSUPPORTED),
            (dict(page_size=32), qf.QF_EUNSUPPORTED), (dict(max_pages_per_seq=0), qf.QF_EINVAL),
            (dict(num_pages=0), qf.QF_EINVAL), (dict(max_shards=0), qf.QF_EINVAL),
            (dict(softmax_scale=math.inf), qf.QF_EINVAL)]


def _rope(over=None, desc=None, n=6, rope=(128, 0, 4096, 1.0), strides=(512, 256, 256), eps=1e-6):
    a = dict(cu=A, ctx=A, q=A, k=A, v=A, qg=A, kg=A, qo=ctypes.c_void_p(8192), kc=A, vc=A, bt=A, st=None)
    a.update(over or {})
    d = _desc() if desc is None else desc
    r = None if rope is None else ctypes.byref(Rope(*rope))
    rc = load_library().qf_qkv_rope_append(
        ctypes.byref(d), n, a["cu"], a["ctx"], r, a["q"], strides[0], a["k"], strides[1], a["v"],
        strides[2], a["qg"], a["kg"], eps, a["qo"], a["kc"], a["vc"], a["bt"], a["st"], None)
    assert rc == qf.QF_OK or load_library().qf_last_error().decode() != ""
    return rc


@needs_lib
def test_rope_append_refusals():
    for kw, code in BAD_DESC:
        assert _rope(desc=_desc(**kw)) == code, kw
    assert load_library().qf_qkv_rope_append(None, 1, A, A, None, A, 512, A, 256, A, 256, None, None,
                                             0.0, A, A, A, A, None, None) == qf.QF_EINVAL
    assert _rope(n=-1) == qf.QF_EINVAL
    assert _rope(n=1 << 24) == qf.QF_EINVAL
    assert _rope(over=dict(cu=None), n=3) == qf.QF_EINVAL           # one token per request
    assert _rope(rope=(128, 2, 4096, 1.0)) == qf.QF_EINVAL
    assert _rope(rope=(-16, 0, 4096, 1.0)) == qf.QF_EINVAL
    assert _rope(rope=(144, 0, 4096, 1.0)) == qf.QF_EINVAL
    assert _rope(rope=(24, 0, 4096, 1.0)) == qf.QF_EUNSUPPORTED
    assert _rope(rope=(128, 0, None, 1.0)) == qf.QF_EINVAL
    assert _rope(rope=(128, 0, 4100, 1.0)) == qf.QF_EALIGN
    assert _rope(rope=(128, 0, 4096, math.nan)) == qf.QF_EINVAL
    assert _rope(eps=math.nan) == qf.QF_EINVAL and _rope(eps=-1.0) == qf.QF_EINVAL
    for name in ("k", "v"):
        assert _rope(over={name: None}) == qf.QF_EINVAL, name        # k and v go together
    assert _rope(over=dict(q=None, k=None, v=None)) == qf.QF_EINVAL
    for name in ("ctx", "qo", "kc", "vc"):
        assert _rope(over={name: None}) == qf.QF_EINVAL, name
    for strides in ((511, 256, 256), (504, 256, 256), (512, 248, 256), (512, 256, 260)):
        assert _rope(strides=strides) == qf.QF_EINVAL, strides
    assert _rope(over=dict(qo=A), strides=(520, 256, 256)) == qf.QF_EINVAL    # in place with gaps
    for name in ("q", "k", "v", "qg", "kg", "qo", "kc", "vc"):
        assert _rope(over={name: OFF8}) == qf.QF_EALIGN, name
    for name in ("cu", "ctx", "bt", "st"):
        assert _rope(over={name: OFF2}) == qf.QF_EALIGN, name
    assert _rope(over=dict(bt=None), desc=_desc(num_pages=15)) == qf.QF_EINVAL
    assert _rope(n=0) == qf.QF_OK
    assert _rope(desc=_desc(batch=0), n=0, over=dict(cu=None)) == qf.QF_OK


def _prefill(over=None, desc=None, n=6, ws=1 << 30):
    a = dict(q=A, k=A, v=A, bt=A, ctx=A, cu=A, out=A, lse=A, ws=A)
    a.update(over or {})
    d = _desc(max_pages_per_seq=4096, num_pages=8192) if desc is None else desc
    rc = load_library().qf_attn_prefill(ctypes.byref(d), n, a["q"], a["k"], a["v"], a["bt"], a["ctx"],
                                        a["cu"], a["out"], a["lse"], a["ws"], ws, None)
    assert rc == qf.QF_OK or load_library().qf_last_error().decode() != ""
    return rc


def _prefill_bytes(n, **kw):
    size = ctypes.c_size_t(1 << 60)
    rc = load_library().qf_attn_prefill_workspace_size(ctypes.byref(_desc(**kw)), n, ctypes.byref(size))
    return rc, size.value


@needs_lib
def test_prefill_refusals():
    for kw, code in BAD_DESC:
        assert _prefill(desc=_desc(**kw)) == code, kw
        assert _prefill_bytes(6, **kw)[0] == code, kw
    assert _prefill(n=-1) == qf.QF_EINVAL
    assert _prefill(n=(1 << 31) - 1) == qf.QF_EINVAL
    for name in ("q", "k", "v", "ctx", "cu", "out", "ws"):
        assert _prefill(over={name: None}) == qf.QF_EINVAL, name
    assert _prefill(ws=64) == qf.QF_EINVAL
    for name in ("q", "k", "v", "ws"):
        assert _prefill(over={name: OFF8}) == qf.QF_EALIGN, name
    assert _prefill(over=dict(out=ctypes.c_void_p(4100))) == qf.QF_EALIGN
    for name in ("lse", "ctx", "cu", "bt"):
        assert _prefill(over={name: OFF2}) == qf.QF_EALIGN, name
    assert _prefill(over=dict(bt=None), desc=_desc(num_pages=15)) == qf.QF_EINVAL
    assert _prefill(n=0) == qf.QF_OK
    assert _prefill(desc=_desc(batch=0)) == qf.QF_OK


@needs_lib
def test_prefill_workspace_only_for_few_rows():
    """The pairs of the key ranges: none where the row tiles fill the chip, or the table is short."""
    rc, n = _prefill_bytes(8192, batch=1, n_q_heads=16, n_kv_heads=8, max_pages_per_seq=1024)
    assert rc == 0 and n == 0
    assert _prefill_bytes(6, max_pages_per_seq=4) == (0, 0)
    rc, n = _prefill_bytes(6, max_pages_per_seq=4096)
    # whole sets of pairs, one word, and what rounds that up to 16 bytes
    assert rc == 0 and n > 0 and n % (6 * 4 * 129 * 4) <= 16
    assert _prefill_bytes(0)[1] == 0 and _prefill_bytes(6, batch=0)[1] == 0


def _shared(over=None, desc=None, groups=1, pages=64, pair=0, ws=1 << 30):
    a = dict(q=A, k=A, v=A, pt=A, pl=A, gr=A, bt=A, ctx=A, ns=A, out=A, lse=A, ws=A)
    a.update(over or {})
    d = _desc() if desc is None else desc
    rc = load_library().qf_attn_decode_shared(
        ctypes.byref(d), a["q"], a["k"], a["v"], groups, pages, a["pt"], a["pl"], a["gr"], a["bt"],
        a["ctx"], a["ns"], pair, a["out"], a["lse"], a["ws"], ws, None)
    assert rc == qf.QF_OK or load_library().qf_last_error().decode() != ""
    return rc


@needs_lib
def test_shared_refusals():
    size = ctypes.c_size_t(0)
    f = load_library().qf_attn_decode_shared_workspace_size
    for kw, code in BAD_DESC:
        assert _shared(desc=_desc(**kw)) == code, kw
        assert f(ctypes.byref(_desc(**kw)), 1, 64, ctypes.byref(size)) == code, kw
    assert f(ctypes.byref(_desc()), 1, 64, None) == qf.QF_EINVAL
    assert _shared(groups=-1) == qf.QF_EINVAL
    assert _shared(pages=0) == qf.QF_EINVAL and _shared(pages=1 << 28) == qf.QF_EINVAL
    for name in ("q", "k", "v", "pt", "pl", "gr", "ctx", "ns", "out", "ws"):
        assert _shared(over={name: None}) == qf.QF_EINVAL, name
    assert _shared(pair=1, over=dict(lse=None)) == qf.QF_EINVAL
    assert _shared(ws=64) == qf.QF_EINVAL
    for name in ("q", "k", "v", "ws"):
        assert _shared(over={name: OFF8}) == qf.QF_EALIGN, name
    assert _shared(over=dict(out=OFF2)) == qf.QF_EALIGN
    assert _shared(pair=1, over=dict(out=OFF8)) == qf.QF_EALIGN
    for name in ("pt", "pl", "gr", "bt", "ctx", "ns", "lse"):
        assert _shared(over={name: OFF2}) == qf.QF_EALIGN, name
    assert _shared(over=dict(bt=None), desc=_desc(num_pages=15)) == qf.QF_EINVAL
    assert _shared(desc=_desc(batch=0)) == qf.QF_OK


def test_plans_refuse_tensors_that_are_not_on_a_gpu():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)  # noqa: E731
    i = lambda *s: z(*s, dtype=torch.int32)  # noqa: E731
    cache = z(4, 2, 16, 128)
    with pytest.raises(qf.QFError):
        qf.qkv_rope_append(z(3, 4, 128), z(3, 2, 128), z(3, 2, 128), cache, cache, i(1, 4), i(1), i(2))
    with pytest.raises(qf.QFError):
        qf.qkv_rope_append(None, z(3, 2, 128), None, cache, cache, i(1, 4), i(1), i(2))
    with pytest.raises(qf.QFError):
        qf.attn_prefill(z(3, 4, 128), cache, cache, i(1, 4), i(1), i(2))
    with pytest.raises(qf.QFError):
        qf.attn_decode_shared(z(1, 4, 128), cache, cache, i(1, 4), i(1), i(2), i(1, 4), i(1), 1)


def test_rope_frequencies():
    f = qf.rope_frequencies(128, theta=1e6)
    assert f.dtype == torch.float64 and f.shape == (64,)
    assert np.allclose(f.numpy(), 1e6 ** (-np.arange(64) / 64), rtol=1e-14)
    assert torch.equal(qf.rope_frequencies(64, 1e4, stretch=4.0), qf.rope_frequencies(64, 1e4) / 4)
    g = qf.rope_frequencies(128, 1e6, stretch=4.0, trained=32768)
    turns = f * 32768 / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32])
    assert torch.allclose(g[turns <= 1], f[turns <= 1] / 4, rtol=1e-14)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and bool(((g < f) & (g > f / 4))[mid].all())
    assert qf.rope_frequencies(0).shape == (0,)
    for kw in (dict(rotary_dim=3), dict(rotary_dim=-2), dict(rotary_dim=8, theta=0.0),
               dict(rotary_dim=8, stretch=0.0)):
        with pytest.raises(qf.QFError):
            qf.rope_frequencies(**kw)
