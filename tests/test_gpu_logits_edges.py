"""Edges of the operators on logits in hand: calls repeated for the same bits, settings and temperatures at
the ends of their ranges, masks of the type's lowest value.  Tolerances are those of test_gpu_logits.py
unless a test derives its own."""

import pytest
import torch

from paper_2609_38795_gb300 import alr
from tests.test_gpu_logits import (BF, F32, _check_sample, _draws, _lib, _logits, _new,  # noqa: F401
                                   _rows)

pytestmark = pytest.mark.gpu


def _trained(N, V, seed, lift=24.0):
    """A few tokens far above a wide bulk: the largest logit is nowhere near 0."""
    z = _logits(N, V, seed, scale=2.5)
    n = min(40, V)
    g = torch.Generator().manual_seed(seed + 1)
    tok = torch.randint(0, V, (N, n), generator=g)
    return z.scatter(1, tok, lift - 0.5 * torch.arange(n).float().expand(N, n))


def _same_every_time(Z, u, T, repeats, **kw):
    """The oracle's draws, and the same bits in every one of many calls in a row."""
    want = _check_sample(Z, u, T, **kw)
    outs = [dict(token=_new(len(u), dtype=torch.int32), prob=_new(len(u)),
                 n_kept=_new(len(u), dtype=torch.int32)) for _ in range(repeats)]
    for out in outs:
        alr.alr_sample_tokens(Z, u, out, temperature=T, **kw)
    for out in outs:
        for key, x in out.items():
            assert torch.equal(x.view(torch.int32), want[key].view(torch.int32)), key


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V", [(330, 2048), (330, 5003), (24, 5003), (3, 40001)])
def test_nucleus_draws_are_the_same_in_every_call(dtype, N, V):
    """No top-k, or one past the few: the row's largest logit goes straight into a histogram.  Rows one block
    reads, several blocks to an SM, and rows of clusters; largest logits far above and far below 0."""
    for lift in (24.0, -50.0):
        Z = _rows(_trained(N, V, V, lift) + min(lift, 0.0), dtype)
        f = lambda x: torch.full((N,), x, device="cuda")  # noqa: E731
        _same_every_time(Z, _draws(N, 1), f(0.9), 40, top_p=f(0.95))
        _same_every_time(Z, _draws(N, 2), f(1.3), 10, min_p=f(0.01))
        _same_every_time(Z, _draws(N, 3), f(1.1), 10, top_p=f(0.9),
                         top_k=torch.full((N,), 700, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [2048, 9001])
def test_draws_among_many_equal_tokens_are_the_same_in_every_call(dtype, V):
    """Rows that one block reads, several blocks to an SM, whose candidates do not fit: constant rows, steps of
    equal logits, rows with fewer tokens left than the top-k, +inf in some."""
    N = 330
    z = torch.full((N, V), 1.5)
    up = torch.arange(V).float() / V
    z[0::5] = (up * 3).floor() - 40
    z[1::5, V // 70:] = float("-inf")
    z[2::5] = _trained(len(z[2::5]), V, V)
    z[3::40, 7] = float("inf")
    finite = z.clone()
    finite[3::40] = float("-inf")
    finite[3::40, 7] = 0.0                                   # all mass on the +inf
    i = lambda x: torch.full((N,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    T = torch.full((N,), 0.8, device="cuda")
    for k, p in ((50, 0.95), (190, 1.0), (230, 0.5), (1, 1.0)):
        kw = dict(top_k=i(k), top_p=torch.full((N,), p, device="cuda"))
        want = _check_sample(_rows(finite, dtype), _draws(N, k), T, **kw)
        for _ in range(30):
            out = dict(token=_new(N, dtype=torch.int32), prob=_new(N), n_kept=_new(N, dtype=torch.int32))
            alr.alr_sample_tokens(_rows(z, dtype), _draws(N, k), out, temperature=T, **kw)
            for key, x in out.items():
                assert torch.equal(x, want[key]), key
    _same_every_time(_rows(finite, dtype), _draws(N, 9), torch.zeros(N, device="cuda"), 30)


# Below log2(e) / the largest float a temperature's scale is infinite; 5e-39 is above.
TINY = 4e-39


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V", [(8, 5003), (330, 2048)])
def test_temperatures_too_small_for_a_scale_are_greedy(dtype, N, V):
    """T = 0 is their limit; every output is written, also where the neighbours draw."""
    z = _logits(N, V, 61)
    z[1] = 2.0                                               # the lowest id of equal tokens
    z[2] = float("-inf")
    Z = _rows(z, dtype)
    T = torch.where(torch.arange(N) % 3 == 0, 1.0, TINY).cuda()
    T[4], T[5], T[7] = 1e-45, 5e-39, float("nan")
    as_zero = torch.where(T >= 5e-39, T, 0.0)
    f = lambda x: torch.full((N,), x, device="cuda")  # noqa: E731
    i = lambda x: torch.full((N,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    for kw in (dict(), dict(top_k=i(5)), dict(top_p=f(0.9)), dict(min_p=f(0.1)), dict(top_k=i(700))):
        want = _check_sample(Z, _draws(N, 5), as_zero, **kw)
        got = dict(token=_new(N, dtype=torch.int32), prob=_new(N), n_kept=_new(N, dtype=torch.int32))
        alr.alr_sample_tokens(Z, _draws(N, 5), got, temperature=T, **kw)
        for key in got:
            assert torch.equal(got[key], want[key]), key


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V", [(6, 5003), (330, 2048)])
def test_settings_that_are_not_numbers_cut_nothing(dtype, N, V):
    """A NaN top_p or min_p is one that is not given, with a top-k and without."""
    Z = _rows(_logits(N, V, 71), dtype)
    u, T, nan = _draws(N, 6), torch.full((N,), 0.9, device="cuda"), torch.full((N,), float("nan"), device="cuda")
    for k in (0, 20, 600):
        kw = dict(top_k=torch.full((N,), k, dtype=torch.int32, device="cuda"))
        want = _check_sample(Z, u, T, **kw)
        for more in (dict(top_p=nan), dict(min_p=nan), dict(top_p=nan, min_p=nan)):
            got = dict(token=_new(N, dtype=torch.int32), prob=_new(N), n_kept=_new(N, dtype=torch.int32))
            alr.alr_sample_tokens(Z, u, got, temperature=T, **kw, **more)
            for key in got:
                assert torch.equal(got[key], want[key]), (k, more.keys(), key)
