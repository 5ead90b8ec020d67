"""The C entry points of the operators on logits in hand and of the embedding refuse bad arguments
before any device work (no GPU needed: the pointers are fakes that must never be read)."""

import ctypes

import pytest

from paper_2609_38795_gb300 import alr, build_lib


@pytest.fixture(scope="module")
def lib():
    build_lib.build()
    return alr.lib()


A16, MIS = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10002)


def test_struct_layouts():
    assert ctypes.sizeof(alr.AlrDistillParams) == 48           # 3 x 8, 3 x 4, 2 x 4, padded
    assert alr.AlrDistillParams.temperature.offset == 36 and alr.AlrDistillParams.lam.offset == 40
    assert ctypes.sizeof(alr.AlrDistillOutputs) == 8 * 8


def test_refusals(lib):
    def top(Z=A16, dt=1, N=4, V=100, ld=100, K=8, T=1.0, val=A16):
        return lib.alr_top_logits(Z, dt, N, V, ld, K, T, val, A16, None, None, None)

    def sample(Z=A16, dt=0, N=4, V=100, ld=100, u=A16, tok=A16):
        return lib.alr_sample_tokens(Z, dt, N, V, ld, u, None, None, None, None, tok, None, None, None)

    def params(**kw):
        return alr.AlrDistillParams(**dict(dict(N=4, ldz=100, ldg=100, V=100, K=8, dtype=0,
                                                temperature=1.0, lam=1.0), **kw))

    def outs(**kw):
        return alr.AlrDistillOutputs(**dict({f: 0x20000 for f in alr._DISTILL_FIELDS}, **kw))

    def fwd(p, o=None, Z=A16, val=A16, rest=None):
        o = outs() if o is None else o
        return lib.alr_distill_fwd(ctypes.byref(p), Z, val, A16, rest, None, ctypes.byref(o), None)

    def bwd(p, G=A16, lse=A16, rest=None, lse_rest=None, Z=A16):
        return lib.alr_distill_bwd(ctypes.byref(p), Z, A16, A16, rest, None, lse, lse_rest, A16, G, None)

    def both(p, G=A16, Z=A16):
        return lib.alr_distill_fwd_bwd(ctypes.byref(p), Z, A16, A16, None, None, None,
                                       ctypes.byref(outs()), G, None)

    def embed(E=A16, dt=0, V=10, d=8, tok=A16, N=4, out=A16):
        return lib.alr_embed(E, dt, V, d, tok, N, 1.0, out, None)

    def grad(dY=A16, dt=0, V=10, d=8, tok=A16, N=4, dE=A16, ws=A16, nb=1 << 40):
        return lib.alr_embed_grad(dY, dt, V, d, tok, N, 1.0, 0, dE, ws, nb, None)

    I, U = alr.ALR_ERR_INVALID_ARG, alr.ALR_ERR_UNSUPPORTED
    big = alr.ALR_LOGITS_MAX_V
    cases = [
        (lambda: top(dt=2), U, "dtype 2"), (lambda: top(N=-1), I, "N = -1"),
        (lambda: top(N=(1 << 26) + 1), I, "2^26"), (lambda: top(V=0), I, "V = 0"),
        (lambda: top(V=big + 1, ld=big + 1), I, "V = 262145"), (lambda: top(ld=99), I, "stride 99"),
        (lambda: top(ld=1 << 41), I, "stride"), (lambda: top(Z=None), I, "Z must be"),
        (lambda: top(Z=MIS), I, "aligned"), (lambda: top(K=0), I, "K = 0"),
        (lambda: top(K=257), I, "K = 257"), (lambda: top(val=None), I, "top_val"),
        (lambda: top(T=0.0), I, "temperature"), (lambda: top(T=-1.0), I, "temperature"),
        (lambda: top(T=float("nan")), I, "temperature"), (lambda: top(T=float("inf")), I, "temperature"),
        (lambda: top(T=1e-45), I, "temperature"),
        (lambda: sample(dt=-1), U, "dtype -1"), (lambda: sample(u=None), I, "u and token"),
        (lambda: sample(tok=None), I, "u and token"), (lambda: sample(ld=3), I, "stride 3"),
        (lambda: lib.alr_distill_fwd(None, *[A16] * 5, ctypes.byref(outs()), None), I, "params"),
        (lambda: fwd(params(dtype=9)), U, "dtype 9"), (lambda: fwd(params(K=300)), I, "K = 300"),
        (lambda: fwd(params(temperature=0.0)), I, "temperature"),
        (lambda: fwd(params(lam=float("nan"))), I, "lambda"), (lambda: fwd(params(ldz=50)), I, "stride 50"),
        (lambda: fwd(params(), val=None), I, "top_val"), (lambda: fwd(params(), outs(lse=None)), I, "lse"),
        (lambda: fwd(params(), outs(loss_row=None)), I, "loss_row"),
        (lambda: fwd(params(), outs(weight_sum=None)), I, "weight_sum"),
        (lambda: fwd(params(), outs(lse_rest=None), rest=A16), I, "lse_rest"),
        (lambda: lib.alr_distill_fwd(ctypes.byref(params()), A16, A16, A16, None, None, None, None), I,
         "loss_total"),
        (lambda: bwd(params(ldg=99)), I, "ldg = 99"), (lambda: bwd(params(), G=None), I, "G must be"),
        (lambda: bwd(params(), G=MIS), I, "aligned"), (lambda: bwd(params(), lse=None), I, "lse"),
        (lambda: bwd(params(), rest=A16), I, "lse_rest"),
        (lambda: lib.alr_distill_fwd_bwd(ctypes.byref(params()), A16, A16, A16, None, None,
                                         ctypes.c_void_p(0x20000), ctypes.byref(outs()), A16, None), I,
         "batch_weight_sum"),
        (lambda: both(params(ldz=120)), I, "ldg = ldz"), (lambda: both(params(), Z=MIS), I, "aligned"),
        (lambda: embed(dt=3), U, "dtype 3"), (lambda: embed(V=0), I, "V=0"), (lambda: embed(d=0), I, "d=0"),
        (lambda: embed(N=-2), I, "N = -2"), (lambda: embed(tok=None), I, "tokens"),
        (lambda: embed(E=MIS), I, "aligned"), (lambda: embed(out=None), I, "non-NULL"),
        (lambda: grad(N=(1 << 24) + 1), I, "N ="), (lambda: grad(dE=None), I, "dE"),
        (lambda: grad(dY=MIS), I, "dY"), (lambda: grad(ws=None), I, "workspace"),
        (lambda: grad(nb=8), I, "(got 8)"), (lambda: grad(ws=MIS), I, "workspace"),
    ]
    for n, (call, code, text) in enumerate(cases):
        rc = call()
        msg = lib.alr_last_error().decode()
        assert rc == code and text in msg, (n, rc, msg)


def test_no_rows_need_no_device_where_nothing_is_written(lib):
    """N = 0: nothing to do, so no pointer is looked at and no device is needed."""
    assert lib.alr_top_logits(None, 0, 0, 10, 10, 3, 1.0, *[None] * 5) == alr.ALR_OK
    assert lib.alr_sample_tokens(None, 1, 0, 10, 10, *[None] * 9) == alr.ALR_OK
    assert lib.alr_embed(None, 0, 10, 8, None, 0, 1.0, None, None) == alr.ALR_OK


def test_workspace_size(lib):
    size = lib.alr_embed_grad_workspace_size
    assert size(0, 8, 4) == 0 and size(10, 0, 4) == 0 and size(10, 8, -1) == 0
    assert size(10, 8, (1 << 24) + 1) == 0
    assert 0 < size(10, 8, 0) <= size(10, 8, 100) <= size(151936, 4096, 32768)


def test_binding_refuses_host_tensors():
    import torch
    Z = torch.zeros(4, 32)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA device"):
        alr.alr_sample_tokens(Z, i, dict(token=i))
    with pytest.raises(TypeError, match="torch.Tensor"):
        alr.alr_top_logits(Z.numpy(), 3, {})
    with pytest.raises(ValueError, match="CUDA device"):
        alr.alr_embed(Z, i, Z)


def test_temperatures_whose_scale_overflows_are_refused(lib):
    """1 / T is a float down to 2.94e-39, log2(e) / T, by which the kernels multiply, down to 4.24e-39."""
    p = lambda T: alr.AlrDistillParams(N=4, ldz=100, ldg=100, V=100, K=8, dtype=1, temperature=T,  # noqa: E731
                                       lam=1.0)
    o = alr.AlrDistillOutputs(**{f: 0x20000 for f in alr._DISTILL_FIELDS})
    for T in (3e-39, 4.2e-39):
        for call in (lambda: lib.alr_top_logits(A16, 1, 4, 100, 100, 8, T, A16, A16, None, None, None),
                     lambda: lib.alr_distill_fwd(ctypes.byref(p(T)), A16, A16, A16, None, None,
                                                 ctypes.byref(o), None),
                     lambda: lib.alr_distill_bwd(ctypes.byref(p(T)), A16, A16, A16, None, None, A16, None, A16,
                                                 A16, None)):
            assert call() == alr.ALR_ERR_INVALID_ARG and "temperature" in lib.alr_last_error().decode(), T
