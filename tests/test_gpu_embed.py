"""The embedding lookup and the gradient of its table on the GPU against the oracle.

The lookup is one fp32 product rounded once: bit for bit.  A gradient entry is a sum of n products in
fp32: within (n + 2) 2^-24 of the sum of their absolute values, whatever the order."""

import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo
from paper_2609_38795_gb300 import alr, build_lib
from tests import parity as P

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    build_lib.build()
    alr.lib()
    assert alr.alr_device_supported() == alr.ALR_OK, alr.alr_last_error()


def _tokens(N, V, kind, seed):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(0, V, (N,), generator=g)
    if kind == "one":                                        # every row the same token
        t[:] = V // 2
    elif kind == "mask":                                     # a block's mask token, mostly
        t[torch.rand(N, generator=g) < 0.9] = V - 1
    elif kind == "pad":
        t[torch.rand(N, generator=g) < 0.4] = -1
        t[torch.rand(N, generator=g) < 0.1] = V
        t[torch.rand(N, generator=g) < 0.05] = 2 ** 31 - 1
        t[torch.rand(N, generator=g) < 0.05] = -2 ** 31
    elif kind == "none":
        t[:] = -1
    return t.to(torch.int32).cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V,d", [(1, 1, 1), (5, 3, 7), (64, 100, 8), (33, 1000, 129), (300, 50, 320),
                                   (17, 20, 4096), (1000, 5000, 257)])
def test_embed(dtype, N, V, d):
    g = torch.Generator().manual_seed(N + d)
    E = torch.randn(V, d, generator=g).cuda().to(dtype)
    for kind in ("any", "pad"):
        tok = _tokens(N, V, kind, d)
        out = torch.full((N, d), 9.0, dtype=dtype, device="cuda")
        alr.alr_embed(E, tok, out, scale=11.3)
        ok = (tok >= 0) & (tok < V)
        want = (E.float()[torch.where(ok, tok, 0).long()] * 11.3 * ok[:, None]).to(dtype)
        assert torch.equal(out, want)


def _grad(dY, tok, V, scale, dE=None, accumulate=False):
    N, d = dY.shape
    if dE is None:
        dE = torch.full((V, d), 9.0, device="cuda")
    n = alr.alr_embed_grad_workspace_size(V, d, N)
    ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")   # whatever it held
    alr.alr_embed_grad(dY, tok, dE, ws, scale=scale, accumulate=accumulate)
    torch.cuda.synchronize()
    return dE


def _check_grad(dY, tok, V, scale):
    d = dY.shape[1]
    ref, size = lo.embed_grad(P.np64(dY), tok.cpu().numpy(), V, scale)
    t = tok.cpu().numpy()
    n = np.bincount(t[(t >= 0) & (t < V)], minlength=V)[:, None]
    tol = (n + 2) * EPS * size
    got = _grad(dY, tok, V, scale)
    assert (np.abs(P.np64(got) - ref) <= tol).all()          # zeros where nothing occurred
    assert torch.equal(got, _grad(dY, tok, V, scale))        # the same bits every time
    base = torch.randn(V, d, device="cuda")
    added = _grad(dY, tok, V, scale, dE=base.clone(), accumulate=True)
    assert (np.abs(P.np64(added) - (P.np64(base) + ref)) <= tol + 2 * EPS * np.abs(P.np64(base) + ref)).all()
    assert torch.equal(added[torch.tensor(n[:, 0] == 0).cuda()], base[torch.tensor(n[:, 0] == 0).cuda()])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kind", ["any", "one", "mask", "pad", "none"])
@pytest.mark.parametrize("N,V,d", [(1, 1, 1), (3, 5, 7), (31, 40, 8), (64, 7, 129), (500, 3, 64),
                                   (1200, 1000, 320), (3000, 200, 100)])
def test_embed_grad(dtype, kind, N, V, d):
    g = torch.Generator().manual_seed(N + V)
    _check_grad(torch.randn(N, d, generator=g).cuda().to(dtype), _tokens(N, V, kind, d), V, 3.3)


@pytest.mark.parametrize("N,V,d,kind", [(20000, 151936, 16, "mask"), (40000, 70000, 12, "any"),
                                        (70001, 300, 8, "pad"), (33000, 262145, 8, "mask")])
def test_embed_grad_many_tokens(N, V, d, kind):
    g = torch.Generator().manual_seed(N)
    _check_grad(torch.randn(N, d, generator=g).cuda().to(BF), _tokens(N, V, kind, 1), V, 0.5)


def test_embed_grad_against_differences():
    """The lookup is linear in the table: <dE, D> is the difference of <out, dY> along D."""
    N, V, d = 200, 30, 40
    g = torch.Generator().manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    E, D, dY, tok = r(V, d), r(V, d), r(N, d), _tokens(N, V, "pad", 4)
    def f(table):
        out = torch.empty(N, d, device="cuda")
        alr.alr_embed(table, tok, out, scale=1.7)
        return float((out.double() * dY.double()).sum())
    num = (f(E + 0.5 * D) - f(E - 0.5 * D))
    ana = float((_grad(dY, tok, V, 1.7).double() * D.double()).sum())
    # 8000 products of order 1 to 10, each off by 3 roundings
    assert abs(num - ana) <= 8000 * 10 * 3 * 2 * EPS


def test_no_rows():
    V, d = 12, 8
    dY, tok = torch.empty(0, d, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    assert not _grad(dY, tok, V, 1.0).any()
    base = torch.randn(V, d, device="cuda")
    assert torch.equal(_grad(dY, tok, V, 1.0, dE=base.clone(), accumulate=True), base)
    alr.alr_embed(base, tok, torch.empty(0, d, device="cuda"))


def test_binding_refuses_wrong_buffers():
    V, d, N = 10, 8, 6
    E, tok = torch.randn(V, d, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    out = torch.empty(N, d, device="cuda")
    with pytest.raises(ValueError, match="out must be"):
        alr.alr_embed(E, tok, out.bfloat16())
    with pytest.raises(ValueError, match="tokens must be"):
        alr.alr_embed(E, tok.long(), out)
    with pytest.raises(ValueError, match="fewer than"):
        alr.alr_embed(E, tok, out[:-1])
    with pytest.raises(alr.AlrError, match="workspace"):
        alr.alr_embed_grad(out, tok, E, torch.empty(0, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        alr.alr_embed_grad(out.t().contiguous().t(), tok, E, None)
    with pytest.raises(ValueError, match="dE must be"):
        alr.alr_embed_grad(out, tok, E.double(), None)
