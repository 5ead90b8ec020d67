"""The C entry points of the paged key-value cache refuse bad arguments before any device work (no GPU
needed: the pointers are fakes that must never be read)."""

import ctypes

import pytest
import torch

from paper_2609_38795_gb300 import alr, build_lib

A16, MIS = 0x10000, 0x10002
I, U = alr.ALR_ERR_INVALID_ARG, alr.ALR_ERR_UNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    build_lib.build()
    return alr.lib()


def test_struct_layouts():
    assert ctypes.sizeof(alr.AlrKvCache) == 64 and alr.AlrKvCache.n_pages.offset == 40
    assert ctypes.sizeof(alr.AlrKvPlanOutputs) == 7 * 8
    assert ctypes.sizeof(alr.AlrKvAttentionParams) == 48 and alr.AlrKvAttentionParams.scale.offset == 44


def _cache(**kw):
    d = dict(K=A16, V=A16, stride_page=16 * 256, stride_token=256, stride_head=128, n_pages=10, page=16,
             heads=2, dim=128, dtype=0)
    return alr.AlrKvCache(**{**d, **kw})


def _run(lib, cases):
    for n, (call, code, text) in enumerate(cases):
        rc = call()
        msg = lib.alr_last_error().decode()
        assert rc == code and text in msg, (n, rc, msg)


CACHES = [(dict(dtype=2), U, "dtype 2"), (dict(page=0), I, "page=0"), (dict(heads=0), I, "heads=0"), (dict(heads=1025), I, "heads=1025"),
          (dict(n_pages=-1), I, "n_pages=-1"), (dict(n_pages=1 << 27), I, "2^31"), (dict(page=65537), I, "page=65537"),
          (dict(dim=12), I, "dim = 12"), (dict(dim=264), I, "dim = 264"), (dict(dim=0), I, "dim = 0"),
          (dict(dim=6, dtype=1), I, "dim = 6"), (dict(stride_page=4), I, "strides"),
          (dict(stride_token=-8), I, "strides"), (dict(stride_head=(1 << 40) + 8), I, "strides"),
          (dict(K=None), I, "K and V"), (dict(V=MIS), I, "K and V")]


def test_plan_refusals(lib):
    def plan(S=4, page=16, cols=8, n_pool=30, T=8, len=A16, add=A16, pool=A16, used=A16, table=A16, **o):
        out = alr.AlrKvPlanOutputs(**{**{f: A16 for f in alr._KV_PLAN_FIELDS}, **o})
        return lib.alr_kv_plan(S, page, cols, n_pool, T, len, add, pool, used, table, ctypes.byref(out), None)

    _run(lib, [(lambda: plan(S=-1), I, "S = -1"), (lambda: plan(S=8193), I, "S = 8193"),
               (lambda: plan(page=0), I, "page=0"), (lambda: plan(page=65537), I, "page=65537"), (lambda: plan(cols=0), I, "cols=0"),
               (lambda: plan(page=1 << 16, cols=1 << 15), I, "2^31"), (lambda: plan(n_pool=-1), I, "n_pool=-1"),
               (lambda: plan(T=-5), I, "T=-5"), (lambda: plan(len=None), I, "len"),
               (lambda: plan(add=None), I, "add"), (lambda: plan(table=None), I, "table"),
               (lambda: plan(pool=None), I, "pool"), (lambda: plan(used=None), I, "pool_used"),
               (lambda: plan(pool_used=None), I, "pool_used"), (lambda: plan(slot=None), I, "slot"),
               (lambda: lib.alr_kv_plan(4, 16, 8, 30, 8, A16, A16, A16, A16, A16, None, None), I, "pool_used")])


def test_append_refusals(lib):
    def append(c=None, k=A16, v=A16, src=0, T=4, ld=256, slot=A16):
        return lib.alr_kv_append(ctypes.byref(c or _cache()), k, v, src, T, ld, slot, None)

    _run(lib, [(lambda kw=kw: append(_cache(**kw)), code, text) for kw, code, text in CACHES])
    _run(lib, [(lambda: lib.alr_kv_append(None, A16, A16, 0, 4, 256, A16, None), I, "cache is NULL"),
               (lambda: append(src=3), U, "src_dtype 3"), (lambda: append(T=-1), I, "T = -1"),
               (lambda: append(T=(1 << 26) + 1), I, "2^26"), (lambda: append(ld=248), I, "ld = 248"),
               (lambda: append(ld=260), I, "ld = 260"), (lambda: append(k=None), I, "K_new"),
               (lambda: append(v=MIS), I, "K_new"), (lambda: append(slot=None), I, "slot"),
               (lambda: append(_cache(dim=4, dtype=1, stride_page=64, stride_token=8, stride_head=4), ld=8), I,
                "16 bytes")])
    assert append(T=0, k=None, v=None, slot=None) == alr.ALR_OK


def test_attention_refusals(lib):
    def attend(c=None, Q=A16, table=A16, len=A16, seq=A16, pl=None, ps=None, out=A16, ws=A16, nb=1 << 40, **kw):
        p = alr.AlrKvAttentionParams(**{**dict(N=4, ldq=1024, ldo=1024, H=8, n_seq=4, cols=8, rows_per_seq=1,
                                               rows_per_prefix=1, scale=1.0), **kw})
        return lib.alr_kv_attention(ctypes.byref(c or _cache()), ctypes.byref(p), Q, table, len, seq, pl, ps, out,
                                    None, ws, nb, None)

    _run(lib, [(lambda kw=kw: attend(_cache(**kw)), code, text) for kw, code, text in CACHES])
    _run(lib, [(lambda: attend(N=-1), I, "N = -1"), (lambda: attend(N=(1 << 24) + 1), I, "2^24"),
               (lambda: attend(H=7), I, "H = 7"), (lambda: attend(H=0), I, "H = 0"),
               (lambda: attend(H=1026), I, "H = 1026"), (lambda: attend(n_seq=-1), I, "n_seq=-1"),
               (lambda: attend(cols=0), I, "cols=0"), (lambda: attend(cols=1 << 27), I, "2^31"),
               (lambda: attend(rows_per_seq=0), I, "rows_per_seq"),
               (lambda: attend(rows_per_prefix=-3), I, "rows_per_prefix"),
               (lambda: attend(scale=float("nan")), I, "scale"), (lambda: attend(scale=float("inf")), I, "scale"),
               (lambda: attend(ldq=1016), I, "ldq = 1016"), (lambda: attend(ldo=1028), I, "ldo = 1028"),
               (lambda: attend(Q=None), I, "Q and out"), (lambda: attend(out=MIS), I, "Q and out"),
               (lambda: attend(len=None), I, "len"), (lambda: attend(table=None), I, "table"),
               (lambda: attend(pl=A16), I, "go together"), (lambda: attend(ps=A16), I, "go together"),
               (lambda: attend(seq=None, n_seq=3), I, "without seq"),
               (lambda: attend(seq=None, n_seq=1, rows_per_seq=3), I, "without seq"),
               (lambda: attend(ws=None), I, "workspace"), (lambda: attend(ws=MIS), I, "workspace"),
               (lambda: attend(nb=8), I, "(got 8)"),
               (lambda: lib.alr_kv_attention(ctypes.byref(_cache()), None, *[A16] * 9, 1 << 40, None), I,
                "params is NULL")])
    assert attend(N=0, Q=None, out=None, len=None, ws=None) == alr.ALR_OK


def test_workspace_size(lib):
    size = lib.alr_kv_attention_workspace_size
    for bad in ((-1, 8, 128), ((1 << 24) + 1, 8, 128), (4, 0, 128), (4, 8, 0), (4, 8, 257), (4, 1025, 128)):
        assert size(*bad, 0) == 0, bad
    assert 0 < size(1, 1, 8, 0) <= size(768, 32, 128, 0) <= size(768, 32, 128, 1)


def test_binding_refuses_host_tensors():
    K, i = torch.zeros(2, 4, 1, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA device"):
        alr.alr_kv_append(K[0], K[0], K, K, i)
    with pytest.raises(ValueError, match="CUDA device"):
        alr.alr_kv_plan(i, i, i, i[:1], i[:, None], 4, dict(len=i, slot=i, pool_used=i[:1]))
    with pytest.raises(TypeError, match="torch.Tensor"):
        alr.alr_kv_attention(None, K.numpy(), K, None, i, None, None)


@pytest.mark.parametrize("scale,fits", [(2.35e38, True), (-2.35e38, True), (2.36e38, False), (-2.36e38, False), (3.4e38, False)])
def test_attention_refuses_a_scale_without_room_for_log2e(lib, scale, fits):
    """Scores are held times log2(e): a larger scale made every score infinite."""
    p = alr.AlrKvAttentionParams(N=0, ldq=1024, ldo=1024, H=8, n_seq=4, cols=8, rows_per_seq=1, rows_per_prefix=1,
                                 scale=scale)
    rc = lib.alr_kv_attention(ctypes.byref(_cache()), ctypes.byref(p), *[A16] * 7, None, A16, 1 << 40, None)
    assert rc == (alr.ALR_OK if fits else I)
    assert fits or "scale" in lib.alr_last_error().decode()
