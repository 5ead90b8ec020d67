"""Edges of the operators on logits in hand: calls repeated for the same bits, settings and temperatures at
the ends of their ranges, masks of the type's lowest value.  Tolerances are those of test_gpu_logits.py
unless a test derives its own."""

import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo
from paper_2609_38795_gb300 import alr
from tests import parity as P
from tests.test_gpu_logits import (BF, EPS, F32, LSE_TOL, _check_lse, _check_sample, _distill_out,  # noqa: F401
                                   _draws, _lib, _logits, _new, _rows)

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


def _masks(V, K, value):
    """A row's tokens masked to `value` in long stretches: none, the upper half, the lower third, all but
    three tokens (fewer than the list's), all but the K (+ 2) tokens of the list and two more."""
    m = torch.zeros(5, V, dtype=torch.bool)
    m[1, V // 2:] = True
    m[2, : V // 3] = True
    m[3], m[3, [5, V // 2, V - 1]] = True, False
    m[4], m[4, V // 7: V // 7 + K] = True, False
    return m, value


def _distil_masked(dtype, V, value, T):
    """(Z, val, idx, rest, live logits' size): student and teacher under the same masks."""
    K = 8
    value = torch.finfo(dtype).min if value is None else value
    m, _ = _masks(V, K, value)
    z = _logits(5, V, V).masked_fill(m, value)
    Z = _rows(z, dtype, V + 3)
    t = lo.top_logits(_logits(5, V, V + 1).to(dtype).double().masked_fill(m, float(Z.min())).numpy(), K, T)
    with np.errstate(over="ignore"):                         # past fp32's range: -inf
        f = lambda x: torch.tensor(x.astype(np.float32), device="cuda")  # noqa: E731
        val, rest = f(t["top_val"]), f(t["lse_rest"])
    return Z, val, torch.tensor(t["top_idx"], dtype=torch.int32, device="cuda"), rest, z[~m].abs().max().item() / T


def _check_masked(Z, val, idx, rest, T, big):
    """The bounds of test_gpu_logits.py with `big` the live logits' size (a masked logit is not rounded)."""
    N, V = Z.shape
    n = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    ref = lo.distill(Z.float().cpu().numpy(), n(val), n(idx), n(rest), None, T, 1.0)
    kw = dict(rest=rest, temperature=T)
    out, one, two, G = _distill_out(N), _distill_out(N), Z.clone(), Z.clone()
    alr.alr_distill_fwd(Z, val, idx, out, **kw)
    alr.alr_distill_fwd_bwd(Z, val, idx, one, G, **kw)
    alr.alr_distill_bwd(Z, val, idx, out["lse"], out["lse_rest"] if rest is not None else None, out["weight_sum"],
                        two, **kw)
    p_rel = 8 * EPS * (21 + big)
    for o in (out, one):
        with np.errstate(over="ignore"):
            _check_lse(o["lse"], ref["lse"].astype(np.float32).astype(np.float64))
            if rest is not None:
                _check_lse(o["lse_rest"], ref["lse_rest"].astype(np.float32).astype(np.float64))
        assert np.array_equal(P.npi(o["argmax"]), ref["argmax"])
        tol = 2 * LSE_TOL + p_rel * (np.abs(ref["loss_row"]) + big) + 8 * EPS * big
        assert (np.abs(P.np64(o["loss_row"]) - ref["loss_row"]) <= tol).all()
        assert (np.abs(P.np64(o["ent_row"]) - ref["ent_row"]) <= p_rel * (ref["ent_row"] + 4)).all()
    half = 2.0 ** -8 if Z.dtype == BF else 2 * EPS
    gtol = ref["size"] * (2 * LSE_TOL + p_rel + 8 * EPS * big) + half * np.abs(ref["G"]) + 1e-36
    for g in (G, two):
        assert (np.abs(P.np64(g) - ref["G"]) <= gtol).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("value", [-1e10, -1e30, None])
@pytest.mark.parametrize("V,T", [(5003, 1.0), (40001, 0.5), (40001, 2.0)])
def test_distill_with_tokens_masked_by_large_numbers(dtype, tail, value, V, T):
    """Masks by finite numbers up to the type's lowest value (None), over stretches longer than a warp's part
    of the row: next to nothing of the mass, no NaN anywhere."""
    Z, val, idx, rest, big = _distil_masked(dtype, V, value, T)
    _check_masked(Z, val, idx, rest if tail else None, T, big)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [1e-6, 1e-9, 1e-30])
def test_distill_at_tiny_temperatures(dtype, T):
    """Logits / T far past 2^24: losses in proportion, gradients of one-hot rows, nothing overflows on the way."""
    N, V, K = 4, 3001, 4
    g = torch.Generator().manual_seed(81)
    z = torch.stack([torch.randperm(V, generator=g) for _ in range(N)]).float() * 0.125 - 150   # distinct
    Z = _rows(z if dtype == F32 else (z / 32).round() * 4, dtype)
    t = lo.top_logits(Z.roll(1, 0).float().cpu().numpy(), K, T)
    val = torch.tensor(t["top_val"], dtype=F32, device="cuda")
    idx = torch.tensor(t["top_idx"], dtype=torch.int32, device="cuda")
    # the oracle from each row's largest on (loss and gradient are the same): logits / T themselves are past fp64
    below = lambda x: (x - x.max(1, keepdim=True).values).double().cpu().numpy()  # noqa: E731
    ref = lo.distill(below(Z.double()), below(val.double()), idx.cpu().numpy(), None, None, T, T)
    out, G = _distill_out(N), Z.clone()
    alr.alr_distill_fwd_bwd(Z, val, idx, out, G, temperature=T, lam=T)
    want = ref["loss_row"]
    assert (np.abs(P.np64(out["loss_row"]) - want) <= 16 * EPS * want + 1e-3).all() and (want > 1).all()
    # a probability is that of one of n equal tokens, or 0
    assert (np.abs(P.np64(G) - ref["G"]) <= 2.0 ** -8 * np.abs(ref["G"])).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [0.5, 1.0, 2.0])
def test_distill_rows_of_the_lowest_value(dtype, T):
    """Every token of student and teacher masked to the type's lowest value: all equal, so the label is even
    over its entries and q over the vocabulary, also where the logits / T leave fp32's range."""
    N, V, K, low = 3, 5003, 8, torch.finfo(dtype).min
    Z = _rows(torch.full((N, V), low), dtype)
    val = torch.full((N, K), low, device="cuda")
    idx = torch.arange(K, dtype=torch.int32, device="cuda").expand(N, K).contiguous()
    rest = torch.full((N,), low, device="cuda") / T          # T = 0.5: -inf, no bin
    out, G = _distill_out(N), Z.clone()
    alr.alr_distill_fwd_bwd(Z, val, idx, out, G, rest=rest, temperature=T)
    p0 = 0.0 if T < 1 else 1 / (K + 1)
    p = (1 - p0) / K
    loss = np.log(V) - (p0 * np.log(V - K) if p0 else 0.0)
    assert np.allclose(P.np64(out["loss_row"]), loss, rtol=0, atol=LSE_TOL)
    assert np.allclose(P.np64(out["ent_row"]), np.log(1 / p), rtol=0, atol=8 * EPS * 8)
    assert torch.equal(out["lse"], rest)                     # log V is below its rounding
    want = np.full((N, V), 1 / V)
    want[:, :K] -= p
    want[:, K:] -= p0 / (V - K)
    want /= N * T
    tol = (2.0 ** -8 if dtype == BF else 0) * np.abs(want) + 3 * LSE_TOL * (1 / V + p) / (N * T)
    assert (np.abs(P.np64(G) - want) <= tol).all() and out["argmax"].eq(0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("value", [-1e10, -1e30, None])
@pytest.mark.parametrize("T", [0.7, 1.0, 1.3])
def test_distill_gradient_alone_next_to_masks_of_large_numbers(dtype, value, T):
    """Log-sum-exps of masked tokens alone, of a size at which a float says nothing about differences of
    logits: the gradient from a forward's results is finite, 0 for the row or for the tokens that they are of."""
    Z, val, idx, rest, big = _distil_masked(dtype, 5003, value, T)
    _check_masked(Z, val, idx, rest, T, big)
    N, V = Z.shape
    Z[0] = Z.min()                                           # everything masked
    out, two = _distill_out(N), Z.clone()
    alr.alr_distill_fwd(Z, val, idx, out, rest=rest, temperature=T)
    alr.alr_distill_bwd(Z, val, idx, out["lse"], out["lse_rest"], out["weight_sum"], two, rest=rest, temperature=T)
    assert torch.isfinite(two).all() and not two[0].any() and two[1:].any(1).all()
    # up to there exp(z / T - lse) is that of the numbers given: z - T lse is exact enough
    z = torch.tensor([[2.0 ** 24 - 64, 0.0, -1.0]], device="cuda") * T
    lse, ws = torch.full((1,), 2.0 ** 24 - 64, device="cuda"), torch.ones(1, device="cuda")
    G, one = torch.empty_like(z), torch.zeros(1, 1, device="cuda")
    idx = torch.tensor([[1]], dtype=torch.int32, device="cuda")
    alr.alr_distill_bwd(z, one, idx, lse, None, ws, G, temperature=T)
    t = float(np.float32(T))
    q = np.exp(z[0, 0].item() / t - lse.item())
    assert abs(G[0, 0].item() * t - q) <= 32 * EPS * q and G[0, 2] == 0 and abs(G[0, 1].item() * t + 1) <= 8 * EPS


@pytest.mark.parametrize("N,V", [(6, 2056), (330, 2056)])
def test_rest_far_below_the_list(N, V):
    """The tokens not listed are all 0, 2048 of them, the list 38 to 42 above: log 2048 within a step of fp32's
    logarithm (2^-21 here), for both forms of a row: nothing is added to 0 and the sum is a whole number."""
    z = torch.zeros(N, V)
    z[:, 100:108] = 38 + 4 * torch.arange(N).float()[:, None] / N + 0.01 * torch.arange(8)
    for dtype in (BF, F32):
        out = dict(top_val=_new(N, 8), top_idx=_new(N, 8, dtype=torch.int32), lse=_new(N), lse_rest=_new(N))
        alr.alr_top_logits(_rows(z, dtype), 8, out)
        assert (np.abs(P.np64(out["lse_rest"]) - np.log(2048)) <= 2.0 ** -21).all()


@pytest.mark.parametrize("N", [40, 330])
def test_log_sum_exp_of_one_token_is_its_quotient(N):
    """lse = z / T where a token has all the mass, rounded once; the same for the rest."""
    V, T = 2100, 0.7
    g = torch.Generator().manual_seed(91)
    z = torch.full((N, V), float("-inf"))
    z[:, 9], z[:, 2001] = 300 + 100 * torch.rand(N, generator=g), 100 * torch.rand(N, generator=g)
    out = dict(top_val=_new(N, 1), top_idx=_new(N, 1, dtype=torch.int32), lse=_new(N), lse_rest=_new(N))
    alr.alr_top_logits(_rows(z, F32), 1, out, temperature=T)
    t = float(np.float32(T))
    for key, col in (("lse", 9), ("lse_rest", 2001)):
        want = z[:, col].double().numpy() / t
        assert (np.abs(P.np64(out[key]) - want) <= EPS * np.abs(want)).all(), key


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V", [(12, 9001), (330, 2500)])
def test_sampling_and_top_logits_under_masks_by_large_numbers(dtype, N, V):
    """Masks by finite numbers down to the type's lowest value, whole rows of it, few tokens left; temperatures
    from 1e-30 to infinity."""
    low = torch.finfo(dtype).min
    z = _logits(N, V, 101)
    z[1::6, V // 3:] = low
    z[2::6, 30:] = -1e10
    z[3::6] = low
    z[4::6] = z[4::6].masked_fill(torch.rand(z[4::6].shape, generator=torch.Generator().manual_seed(1)) < 0.99, low)
    z[5::6] += 1e30
    z[5::6, : V // 2] = -1e30
    Z = _rows(z, dtype, V + 1)
    f = lambda x: torch.full((N,), x, device="cuda")  # noqa: E731
    i = lambda x: torch.full((N,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    for T in (1e-30, 0.6, 1.0, 40.0, 1e30, float("inf")):
        for kw in (dict(top_p=f(0.9)), dict(top_k=i(60), top_p=f(0.95)), dict(top_k=i(500)), dict(min_p=f(0.05)), {}):
            _check_sample(Z, _draws(N, 8), f(T), **kw)
    for K in (1, 8, 64, 256):
        for T in (0.6, 1.0, 3.0):
            out = dict(top_val=_new(N, K), top_idx=_new(N, K, dtype=torch.int32), lse=_new(N), lse_rest=_new(N))
            alr.alr_top_logits(Z, K, out, temperature=T)
            ref = lo.top_logits(Z.float().cpu().numpy(), K, T)
            assert np.array_equal(P.npi(out["top_idx"]), ref["top_idx"])
            assert np.array_equal(P.np64(out["top_val"]), ref["top_val"])
            with np.errstate(over="ignore"):                 # past fp32's range: -inf
                _check_lse(out["lse"], ref["lse"].astype(np.float32).astype(np.float64))
                _check_lse(out["lse_rest"], ref["lse_rest"].astype(np.float32).astype(np.float64))
