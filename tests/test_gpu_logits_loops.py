"""The loops of the operators on logits in hand and of the embedding: clusters that take several rows each,
rows of weight 0 before, between and after live ones, every number of packs a thread, the wide search of
the gradient's join; and the distillation gradient alone, entry by entry.  Tolerances are those of
test_gpu_logits.py and test_gpu_embed.py unless a test derives its own."""

import numpy as np
import pytest
import torch

from paper_2609_38795_gb300 import alr
from tests import parity as P
from tests.test_gpu_embed import _check_grad, _tokens
from tests.test_gpu_logits import (BF, EPS, F32, _check_distill, _distill_out, _lib, _logits, _new,  # noqa: F401
                                   _rows)

pytestmark = pytest.mark.gpu


def _labels(N, V, K, T, seed):
    """A teacher's top K and rest, by torch (the rows are many), lists that end early among them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn(N, V, generator=g, device="cuda") * 3
    val, idx = torch.topk(t, K, dim=1)
    rest = torch.logsumexp(t.scatter(1, idx, float("-inf")) / T, 1)
    idx = idx.int()
    idx[::7, K - 1] = -1
    return val.contiguous(), idx.contiguous(), rest.contiguous()


def _weights(N, kind):
    g = torch.Generator().manual_seed(N)
    w = 0.1 + torch.rand(N, generator=g)
    if kind == "ends":                                       # nothing at the start and at the end
        w[: N // 3] = 0.0
        w[-N // 5:] = 0.0
    elif kind == "some":                                     # runs of them in between
        w[torch.rand(N, generator=g) < 0.4] = 0.0
    elif kind == "last":                                     # one row alone
        w[:-1] = 0.0
    return w.cuda()


# (clusters that fit 152 SMs at once): 304 blocks of one, 152 of two, 38 of eight; 19 of eight with 18 packs
@pytest.mark.parametrize("dtype,N,V,stride", [(BF, 700, 33001, 33003), (BF, 400, 60001, 0), (BF, 200, 152064, 0),
                                              (F32, 700, 17001, 0), (F32, 90, 140003, 140003),
                                              (F32, 50, 160001, 0), (BF, 3000, 5000, 5000)])
@pytest.mark.parametrize("kind", ["all", "some", "ends"])
def test_distill_of_more_rows_than_the_device_holds(dtype, N, V, stride, kind):
    val, idx, rest = _labels(N, V, 8, 1.3, V)
    Z = _rows(torch.randn(N, V, generator=torch.Generator().manual_seed(V)) * 3, dtype, stride)
    _check_distill(Z, val, idx, rest if kind != "ends" else None, _weights(N, kind) if kind != "all" else None,
                   1.3, 1.1, ldg=stride)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_of_one_live_row_among_many(dtype):
    N, V = 1500, 4001
    val, idx, rest = _labels(N, V, 5, 1.0, 1)
    _check_distill(_rows(_logits(N, V, 2), dtype, 4003), val, idx, rest, _weights(N, "last"), 1.0, 1.0, ldg=4002)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_repeats_bit_for_bit_while_clusters_take_rows_in_turn(dtype):
    """The same results from every call and from the call over Z itself, for rows of two to five turns."""
    N, V, K = 800, 24001, 8
    val, idx, rest = _labels(N, V, K, 1.0, 3)
    w = _weights(N, "some")
    g = torch.Generator(device="cuda").manual_seed(4)
    z = (torch.randn(N, V, generator=g, device="cuda") * 3).to(dtype)
    want, first = _distill_out(N), torch.empty_like(z)
    alr.alr_distill_fwd_bwd(z, val, idx, want, first, rest=rest, weight=w)
    for over in (False, True) * 4:
        Z, out = z.clone(), _distill_out(N)
        G = Z if over else torch.empty_like(z)
        alr.alr_distill_fwd_bwd(Z, val, idx, out, G, rest=rest, weight=w)
        assert torch.equal(G, first)
        for k, x in out.items():
            assert torch.equal(x.view(torch.int32), want[k].view(torch.int32)), k


@pytest.mark.parametrize("shift,T", [(0.0, 1.0), (300.0, 1.0), (-700.0, 0.3), (1e4, 2.7)])
@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient_alone_entry_by_entry(shift, T, tail):
    """G from given log-sum-exps, against fp64 on the very floats that the kernel gets, so that nothing of their own
    rounding enters.  An exponential of d = z / T - lse: the difference from T lse, its product with log2(e) / T
    (two factors, each rounded) and the rest of lse, |d| eps each and one more, the unit's 2^-22, the row's factors
    of half a dozen steps: eps (6 |d| + 24).  The label's probabilities: 8 eps (1 + |log p| + |t| / T), as in
    test_gpu_logits.py, |t| the spread of the list (differences are taken first)."""
    N, V, K, lam = 40, 3001, 8, 1.7
    val, idx, rest = _labels(N, V, K, T, 5)
    z = (_logits(N, V, 6) + shift).cuda()
    n = lambda x: x.double().cpu().numpy()  # noqa: E731
    t = float(np.float32(T))
    s = n(z) / t
    listed = np.zeros((N, V), dtype=bool)
    at = idx.cpu().numpy()
    for r in range(N):
        listed[r, at[r][at[r] >= 0]] = True
    sum_exp = lambda x: x.max(1) + np.log(np.exp(x - x.max(1, keepdims=True)).sum(1))  # noqa: E731
    f = lambda x: torch.tensor(x, dtype=F32, device="cuda")  # noqa: E731
    lse, lse_rest = f(sum_exp(s)), f(sum_exp(np.where(listed, -np.inf, s)))
    w = _weights(N, "all")
    ws = w.sum()[None]
    G = torch.empty_like(z)
    alr.alr_distill_bwd(z, val, idx, lse, lse_rest if tail else None, ws, G, rest=rest if tail else None, weight=w,
                        temperature=T, lam=lam)
    a = np.where(at >= 0, n(val) / t, -np.inf)
    a = np.concatenate([a, n(rest)[:, None] if tail else np.full((N, 1), -np.inf)], 1)
    p = np.exp(a - a.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        perr = np.where(p > 0, p * 8 * EPS * (1 + np.abs(np.log(p)) + np.ptp(n(val), axis=1)[:, None] / t), 0.0)
    d, dr = s - n(lse)[:, None], s - n(lse_rest)[:, None]
    q, share = np.exp(d), np.where(listed, 0.0, p[:, -1:] * np.exp(dr))
    want = q - share
    err = q * EPS * (6 * np.abs(d) + 24)
    if tail:   # (exp(lse_rest - lse) - p_0) exp(z / T - lse_rest)
        gap = np.abs(n(lse) - n(lse_rest))[:, None]
        err = np.where(listed, err, (q * EPS * (2 * gap + 8) + share * EPS * 8 + np.exp(dr) * perr[:, -1:])
                       + np.abs(want) * EPS * (6 * np.abs(dr) + 24))
    for r in range(N):
        for i, v in enumerate(at[r]):
            if v >= 0:
                want[r, v] -= p[r, i]
                err[r, v] += perr[r, i] + p[r, i] * 8 * EPS
    c = lam * n(w)[:, None] / (n(ws) * t)
    assert (np.abs(n(G) - want * c) <= err * c + 8 * EPS * np.abs(want * c) + 1e-36).all()


@pytest.mark.parametrize("N,V,d,kind", [(65536, 40, 3, "one"), (131072, 5, 4, "any"), (131073, 300, 2, "mask"),
                                        (300001, 70000, 3, "mask"), (262144, 9, 1, "pad")])
def test_embed_grad_of_runs_of_many_chunks(N, V, d, kind):
    """Runs of up to thousands of chunks: the join looks for their ends in ever smaller steps."""
    g = torch.Generator().manual_seed(N)
    _check_grad(torch.randn(N, d, generator=g).cuda().to(BF), _tokens(N, V, kind, 1), V, 0.5)
