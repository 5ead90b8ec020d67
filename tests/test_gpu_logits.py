"""Top logits, distillation and sampling on the GPU against the oracle: odd and tiny sizes, rows of
any stride, ties, masked tokens and rows, both element types, and the refusals of the binding.

Tolerances, from the arithmetic (eps = 2^-24, half an fp32 step):
  log-sum-exps  the exponentials of V terms: an argument rounded a few times (its error times a term
                x exp(-x) <= 1/e of the sum) and the special-function unit's 2^-22, < 5e-7 in all;
                sums of at most 600 terms per thread one after another, < 600 eps = 3.6e-5 at worst;
                the result's own rounding, 2 eps |lse|.
  probabilities 8 eps (1 + |log p| + |m| / T) relative: expf, the differences it takes, one sum.
  losses        a log-sum-exp's error, and a list's terms at a probability's relative error.
  gradients     a probability exp(s - lse) has the error of lse plus 4 eps |s|: relative to the sum of
                the absolute terms of the entry (q + p, q + tail share), then one rounding to the
                element type (2^-9 for bf16), and a flush to zero below the normal range.
"""

import numpy as np
import pytest
import torch

from oracle import logits_oracle as lo
from paper_2609_38795_gb300 import alr, build_lib
from tests import parity as P

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
LSE_TOL = 4e-5
NEG = float("-inf")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    build_lib.build()
    alr.lib()
    assert alr.alr_device_supported() == alr.ALR_OK, alr.alr_last_error()


def _rows(values, dtype, stride=0):
    """Rows `stride` elements apart; what lies between them must never be read as a logit."""
    N, V = values.shape
    buf = torch.full((N, max(stride, V)), 1e4, dtype=dtype, device="cuda")
    buf[:, :V] = values.to("cuda", dtype)
    return buf[:, :V]


def _logits(N, V, seed, scale=3.0, masked=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(N, V, generator=g) * scale
    z[:, V - masked:] = NEG if masked else z[:, V - masked:]
    return z


def _new(N, *more, dtype=F32, fill=-7):
    return torch.full((N, *more), fill, dtype=dtype, device="cuda")


# ------------------------------------------------------------------------ top logits ---
def _top(Z, K, T=1.0):
    N = Z.shape[0]
    out = dict(top_val=_new(N, K), top_idx=_new(N, K, dtype=torch.int32), lse=_new(N), lse_rest=_new(N))
    alr.alr_top_logits(Z, K, out, temperature=T)
    torch.cuda.synchronize()
    return out


def _check_lse(got, want):
    got, want = P.np64(got), np.asarray(want)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    ok = np.isfinite(want)
    assert (np.abs(got - want)[ok] <= LSE_TOL + 4 * EPS * np.abs(want[ok])).all()


def _check_top(Z, K, T=1.0):
    out = _top(Z, K, T)
    ref = lo.top_logits(Z.float().cpu().numpy(), K, T)
    assert np.array_equal(P.npi(out["top_idx"]), ref["top_idx"])
    assert np.array_equal(out["top_val"].cpu().numpy().astype(np.float64), ref["top_val"])
    _check_lse(out["lse"], ref["lse"])
    _check_lse(out["lse_rest"], ref["lse_rest"])
    return out, ref


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V,K,stride", [(1, 1, 1, 0), (3, 1, 4, 0), (2, 7, 256, 9), (5, 33, 8, 37),
                                          (4, 511, 20, 0), (3, 4097, 64, 4097), (2, 32001, 256, 0),
                                          (2, 152064, 8, 0), (1, 262144, 33, 0), (17, 1003, 5, 1008)])
def test_top_logits(dtype, N, V, K, stride):
    _check_top(_rows(_logits(N, V, V + K), dtype, stride), K, T=0.7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [40, 1000, 40001])
def test_top_logits_ties_masks_and_special_rows(dtype, V):
    """Equal values (everywhere; in two levels; at the threshold), rows sorted up and down, tokens
    masked by -inf and NaN, rows with none and with one left, signed zeros."""
    g = torch.Generator().manual_seed(V)
    z = torch.zeros(12, V)
    z[1] = (torch.rand(V, generator=g) < 0.5).float()
    z[2] = torch.randint(-3, 4, (V,), generator=g).float()
    z[3] = torch.arange(V).float() / V * 8 - 4
    z[4] = -z[3]
    z[5] = NEG
    z[6] = NEG
    z[6, V // 2] = -3.0
    z[7] = torch.where(torch.rand(V, generator=g) < 0.9, torch.tensor(float("nan")), z[2])
    z[8] = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0)
    z[9] = torch.finfo(torch.bfloat16).min
    z[9, 3] = -1e30
    z[10] = torch.randn(V, generator=g)
    z[10, : V // 3] = NEG
    z[11, V - 1] = 5.0
    for K in (1, 8, 39, 256):
        _check_top(_rows(z, dtype, V + 3), K)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,stride", [(2048, 0), (5003, 5007), (33001, 0), (140000, 140008)])
def test_top_logits_of_many_rows(dtype, V, stride):
    """As many rows as the device has SMs and more, each read by one block: logits in no order, rising and
    falling along the row (the largest last, or all first), masked to a stretch, all equal."""
    N = 330 if V < 10000 else 170
    z = _logits(N, V, V, masked=V // 50)
    up = torch.arange(V).float() / V
    z[3], z[4] = 9 * up, -9 * up
    z[5] += 30 * up
    z[6, V // 60:] = NEG
    z[7, : V - V // 60] = NEG
    z[8] = NEG
    z[9] = 1.5
    z[10] = (up * 20).floor()
    Z = _rows(z, dtype, stride)
    for K in (1, 8, 64, 199, 256) if V < 100000 else (8, 199):
        _check_top(Z, K, T=0.9)


# ------------------------------------------------------------------------ distillation ---
def _teacher(N, V, K, T, seed, dtype=F32):
    t = lo.top_logits(_logits(N, V, seed).numpy(), K, T)
    f = lambda x, dt=F32: torch.tensor(x, dtype=dt, device="cuda")  # noqa: E731
    return f(t["top_val"]), f(t["top_idx"], torch.int32), f(t["lse_rest"])


def _distill_out(N):
    return dict(loss_row=_new(N), ent_row=_new(N), lse=_new(N), lse_rest=_new(N),
                argmax=_new(N, dtype=torch.int32), loss_total=_new(1), weight_sum=_new(1),
                wl_sum=_new(1))


def _check_distill(Z, val, idx, rest, weight, T, lam, ldg=0):
    N, V = Z.shape
    kw = dict(rest=rest, weight=weight, temperature=T, lam=lam)
    out = _distill_out(N)
    alr.alr_distill_fwd(Z, val, idx, out, **kw)
    z = Z.float().cpu().numpy()
    n = lambda t: None if t is None else t.cpu().numpy()  # noqa: E731
    ref = lo.distill(z, n(val), n(idx), n(rest), n(weight), T, lam)
    big = np.where(np.isfinite(z), np.abs(z), 0).max(initial=0) / T
    p_rel = 8 * EPS * (1 + big + 20)
    live = np.ones(N, bool) if weight is None else n(weight) != 0
    _check_lse(out["lse"], ref["lse"])
    if rest is not None:
        _check_lse(out["lse_rest"], ref["lse_rest"])
    assert np.array_equal(P.npi(out["argmax"]), ref["argmax"])
    tol = 2 * LSE_TOL + p_rel * (np.abs(ref["loss_row"]) + big) + 8 * EPS * big
    got = P.np64(out["loss_row"])
    assert np.array_equal(np.isinf(got), np.isinf(ref["loss_row"]))
    fin = np.isfinite(ref["loss_row"])
    assert (np.abs(got - ref["loss_row"])[fin] <= np.broadcast_to(tol, N)[fin]).all()
    assert (got[~live] == 0).all()
    assert (np.abs(P.np64(out["ent_row"]) - ref["ent_row"]) <= p_rel * (ref["ent_row"] + 4)).all()
    w = np.ones(N) if weight is None else P.np64(weight)
    if np.isfinite(ref["loss_total"]):
        assert abs(out["loss_total"].item() - ref["loss_total"]) <= abs(lam) * (np.max(tol) + 2e-7 * 50)
        assert abs(out["wl_sum"].item() - ref["wl_sum"]) <= (w * tol).sum() + 4 * EPS * abs(ref["wl_sum"]) + 1e-30
    assert abs(out["weight_sum"].item() - ref["weight_sum"]) <= 2 * EPS * abs(ref["weight_sum"])
    # the gradient: from the forward's results, in one call, and over Z itself
    def grad_of(call):
        G = _rows(torch.full((N, V), 3.0), Z.dtype, ldg)
        call(G)
        torch.cuda.synchronize()
        return G
    two = grad_of(lambda G: alr.alr_distill_bwd(Z, val, idx, out["lse"],
                                                out["lse_rest"] if rest is not None else None,
                                                out["weight_sum"], G, **kw))
    out2 = _distill_out(N)
    one = grad_of(lambda G: alr.alr_distill_fwd_bwd(Z, val, idx, out2, G, **kw))
    half = 2.0 ** -8 if Z.dtype == BF else 2 * EPS
    gtol = ref["size"] * (2 * LSE_TOL + p_rel + 8 * EPS * big) + half * np.abs(ref["G"]) + 1e-36
    for G in (two, one):
        assert (np.abs(P.np64(G) - ref["G"]) <= gtol).all()
    for k in ("loss_row", "ent_row", "lse", "argmax", "loss_total", "weight_sum", "wl_sum"):
        assert torch.equal(out[k].view(torch.int32), out2[k].view(torch.int32)), k
    buf = torch.empty(N, max(Z.stride(0), V), dtype=Z.dtype, device="cuda")[:, :V]
    buf.copy_(Z)
    alr.alr_distill_fwd_bwd(buf, val, idx, _distill_out(N), buf, **kw)
    assert torch.equal(buf, one)
    return out, one, ref


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("N,V,K,stride", [(1, 1, 1, 0), (2, 3, 5, 0), (5, 33, 4, 40), (3, 1001, 8, 0),
                                          (16, 4096, 8, 0), (4, 9999, 256, 10007), (2, 60001, 20, 0),
                                          (2, 151936, 8, 0), (1, 262144, 64, 0)])
def test_distill(dtype, tail, N, V, K, stride):
    T, lam = 1.5, 1.013441
    val, idx, rest = _teacher(N, V, K, T, seed=V)
    g = torch.Generator().manual_seed(7)
    weight = torch.rand(N, generator=g).cuda()
    if N > 2:
        weight[1] = 0.0
    _check_distill(_rows(_logits(N, V, V + 1), dtype, stride), val, idx, rest if tail else None,
                   weight, T, lam, ldg=stride)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [5, 33, 1001, 9999, 60001])
@pytest.mark.parametrize("apart", [(0, 1), (3, 0), (5, 2), (8, 3)])
def test_distill_rows_of_two_alignments(dtype, V, apart):
    """Rows of Z and of G that start at different places of their 16-byte packs, every difference of them
    among the rows; nothing outside a row is written."""
    N, K = 17 if V < 10000 else 9, 4
    val, idx, rest = _teacher(N, V, K, 1.0, seed=V)
    Z = _rows(_logits(N, V, V + 2), dtype, V + apart[0])
    ldg = V + apart[1]
    _check_distill(Z, val, idx, rest, None, 1.0, 1.0, ldg=ldg)
    buf = torch.full((N, ldg + 3), 77.0, dtype=dtype, device="cuda")
    alr.alr_distill_fwd_bwd(Z, val, idx, _distill_out(N), buf[:, :V], rest=rest)
    assert (buf[:, V:] == 77).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_distill_masks_and_empty_rows(dtype):
    """Absent entries, rows without a label, without weight, without logits; a masked vocabulary; a
    student that gives no mass to a listed token; nothing outside the list; other temperatures."""
    N, V, K = 10, 517, 6
    val, idx, rest = _teacher(N, V, K, 1.0, seed=3)
    z = _logits(N, V, 4, scale=5.0, masked=17)
    idx[0, 3:] = -1
    idx[1] = -1
    rest[1] = NEG                                            # no label at all
    z[2] = NEG                                               # no logits
    idx[3] = -1                                              # only the tail bin
    val[4, 1:] = NEG                                         # listed tokens of probability 0
    z[5] = NEG
    z[5, idx[5].cpu().long()] = torch.arange(K).float()      # nothing outside the list
    rest[5] = NEG
    idx[6, 2] = V + 5                                        # outside the vocabulary: absent
    weight = torch.ones(N, device="cuda")
    weight[7] = 0.0
    z[8, int(idx[8, 0])] = NEG                               # q = 0 where p > 0: infinite loss
    Z = _rows(z, dtype, 520)
    out, G, ref = _check_distill(Z, val, idx, rest, weight, 1.0, 1.0)
    assert np.isinf(P.np64(out["loss_row"])[8]) and not G[1].any() and not G[2].any()
    for T in (0.05, 30.0):
        _check_distill(_rows(_logits(N, V, 5), dtype), val, idx, rest, weight, T, T * T)
    zero = torch.zeros(N, device="cuda")
    out, G, _ = _check_distill(Z, val, idx, rest, zero, 1.0, 1.0)
    assert out["loss_total"].item() == 0 and not G.any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("apart", [60.0, 120.0, 3000.0])
def test_distill_list_far_above_the_rest(dtype, apart):
    """The student gives the tokens outside the list next to nothing (below the exponentials' range),
    the label does not: a large finite loss and a gradient without overflow."""
    N, V, K = 3, 700, 4
    val, idx, rest = _teacher(N, V, K, 1.0, seed=41)
    z = _logits(N, V, 42)
    z.scatter_add_(1, idx.cpu().long(), torch.full((N, K), apart))
    out, G, ref = _check_distill(_rows(z, dtype), val, idx, rest, None, 1.0, 1.0)
    assert np.isfinite(P.np64(out["loss_row"])).all() and torch.isfinite(G).all()


def test_distill_normaliser_of_a_sharded_batch():
    """Two halves with the batch's sum of weights give the whole batch's gradient bit for bit."""
    N, V, K = 12, 2000, 8
    val, idx, rest = _teacher(N, V, K, 1.0, seed=11)
    Z = _rows(_logits(N, V, 12), BF)
    w = torch.rand(N, device="cuda")
    whole, G = _distill_out(N), _new(N, V, dtype=BF)
    alr.alr_distill_fwd_bwd(Z, val, idx, whole, G, rest=rest, weight=w)
    for a, b in ((0, 5), (5, 12)):
        part, Gp = _distill_out(b - a), _new(b - a, V, dtype=BF)
        alr.alr_distill_fwd_bwd(Z[a:b].contiguous(), val[a:b].contiguous(), idx[a:b].contiguous(), part,
                                Gp, rest=rest[a:b].clone(), weight=w[a:b].clone(),
                                batch_weight_sum=whole["weight_sum"])
        assert torch.equal(Gp, G[a:b])


def test_distill_gradient_against_differences():
    """Central differences of the forward's own loss along random directions, fp32 logits.  With a
    step of 0.02 the third-order term is below step^2, the loss's error (LSE_TOL at worst, common to
    both sides for the most part) over the step below 2e-3."""
    N, V, K, step = 6, 257, 8, 0.02
    val, idx, rest = _teacher(N, V, K, 1.0, seed=21)
    z = _logits(N, V, 22).cuda()
    G = torch.empty(N, V, device="cuda")
    alr.alr_distill_fwd_bwd(z, val, idx, _distill_out(N), G, rest=rest)

    def loss(x):
        o = _distill_out(N)
        alr.alr_distill_fwd(x.contiguous(), val, idx, o, rest=rest)
        return P.np64(o["loss_row"]).sum() / N

    g = torch.Generator().manual_seed(23)
    for _ in range(8):
        v = torch.randn(N, V, generator=g).cuda()
        num = (loss(z + step * v) - loss(z - step * v)) / (2 * step)
        assert abs(num - float((G.double() * v.double()).sum())) < 2e-3 + step ** 2


# ---------------------------------------------------------------------------- sampling ---
def _w32(Z, T):
    z = Z.float()
    m = z.max(1, keepdim=True).values
    c = torch.full_like(T, 1.4426950408889634) / torch.where(T > 0, T, 1.0)
    return torch.exp2((z - m) * c[:, None])


def _check_sample(Z, u, T, **kw):
    N = Z.shape[0]
    out = dict(token=_new(N, dtype=torch.int32), prob=_new(N), n_kept=_new(N, dtype=torch.int32))
    alr.alr_sample_tokens(Z, u, out, temperature=T, **kw)
    Tn = torch.ones(N, device="cuda") if T is None else T
    n = lambda t: t.cpu().numpy()  # noqa: E731
    clean = torch.where(torch.isnan(Z.float()), torch.tensor(NEG, device="cuda"), Z.float())
    ref = lo.sample(n(clean), n(_w32(clean, Tn)), n(u), None if T is None else n(T),
                    **{k: n(v) for k, v in kw.items()})
    assert np.array_equal(P.npi(out["token"]), ref["token"])
    assert np.array_equal(P.npi(out["n_kept"]), ref["n_kept"])
    assert np.array_equal(n(out["prob"]), ref["prob"].astype(np.float32))
    return out


def _draws(N, seed):
    g = torch.Generator().manual_seed(seed)
    u = torch.randint(-(1 << 31), 1 << 31, (N,), generator=g, dtype=torch.int64).to(torch.int32)
    u[0] = 0
    u[N - 1] = -1                                            # 2^32 - 1, the last of u
    return u.cuda()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("N,V,stride", [(1, 1, 0), (3, 2, 0), (9, 33, 35), (16, 1001, 0), (6, 4096, 0),
                                        (4, 32001, 32005), (2, 152064, 0), (1, 262144, 0)])
def test_sample(dtype, N, V, stride):
    Z = _rows(_logits(N, V, V), dtype, stride)
    f = lambda x: torch.full((N,), x, device="cuda")  # noqa: E731
    i = lambda x: torch.full((N,), x, dtype=torch.int32, device="cuda")  # noqa: E731
    _check_sample(Z, _draws(N, 1), None)
    for j, kw in enumerate((dict(), dict(top_k=i(5)), dict(top_p=f(0.9)), dict(min_p=f(0.02)),
                            dict(top_k=i(50), top_p=f(0.6)), dict(top_k=i(700)),
                            dict(top_k=i(V), top_p=f(0.999), min_p=f(1e-5)),
                            dict(top_k=i(3000), top_p=f(0.97)))):
        _check_sample(Z, _draws(N, 2 + j), f(0.8 + 0.3 * j), **kw)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sample_settings_differ_by_row(dtype):
    N, V = 96, 2003
    g = torch.Generator().manual_seed(5)
    r = lambda: torch.rand(N, generator=g).cuda()  # noqa: E731
    Z = _rows(_logits(N, V, 6, scale=2.0, masked=100), dtype, 2008)
    Z[3] = NEG                                               # nothing allowed
    Z[4, 1:] = NEG                                           # one token allowed
    Z[5] = float("nan")
    Z[6, ::2] = float("nan")
    Z[7] = 1.0                                               # everything equal
    Z[8, 17] = float("inf")
    T = torch.where(r() < 0.2, 0.0, 0.02 + 3 * r())
    T[0], T[7] = -1.0, 1.0
    k = torch.where(r() < 0.3, 0, 1 + (r() * 300).int()).int()
    p = torch.where(r() < 0.3, 1.0, r())
    p[10], p[11] = 0.0, 1e-9
    m = torch.where(r() < 0.5, 0.0, r() * 0.3)
    m[12], m[13] = 1.0, 1.5
    z = Z.clone()
    z[8] = NEG
    z[8, 17] = 0.0                                           # all mass on the +inf
    out = dict(token=_new(N, dtype=torch.int32), prob=_new(N), n_kept=_new(N, dtype=torch.int32))
    alr.alr_sample_tokens(Z, _draws(N, 7), out, temperature=T, top_k=k, top_p=p, min_p=m)
    same = _check_sample(z, _draws(N, 7), T, top_k=k, top_p=p, min_p=m)
    for key in out:
        assert torch.equal(out[key], same[key])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V,stride,scale", [(2048, 0, 3.0), (5003, 5007, 1.3), (33001, 0, 1.3),
                                            (120000, 120008, 4.0)])
def test_sample_of_many_rows(dtype, V, stride, scale):
    """As many rows as the device has SMs and more, each with settings of its own; among them masked
    stretches, constant rows, steps of equal logits and rows without a candidate."""
    N = 340 if V < 10000 else 160
    g = torch.Generator().manual_seed(V)
    r = lambda: torch.rand(N, generator=g).cuda()  # noqa: E731
    z = _logits(N, V, V + 1, scale=scale, masked=V // 50)
    up = torch.arange(V).float() / V
    z[3], z[4] = 9 * up, -9 * up
    z[5, V // 60:] = NEG
    z[6, : V - V // 60] = NEG
    z[7] = NEG
    z[8] = 1.5
    z[9] = (up * 20).floor()
    z[10] = float("nan")
    z[11, 1::3] = float("nan")
    Z = _rows(z, dtype, stride)
    T = torch.where(r() < 0.15, 0.0, 0.2 + 1.5 * r())
    T[3:12] = 1.0
    k = torch.where(r() < 0.4, 0, 1 + (r() * 300).int()).int()
    k[12], k[13] = 1500, V - 1
    p = torch.where(r() < 0.4, 1.0, r())
    m = torch.where(r() < 0.6, 0.0, r() * 0.3)
    _check_sample(Z, _draws(N, 3), T, top_k=k, top_p=p, min_p=m)
    if V > 100000:
        return
    k[:], p[:] = 0, 0.9
    _check_sample(Z, _draws(N, 4), T, top_p=p)
    _check_sample(Z, _draws(N, 5), T)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_sample_ties_at_the_cuts(dtype):
    """Few distinct values: every cut falls inside a run of equal tokens."""
    N, V = 24, 5003
    g = torch.Generator().manual_seed(8)
    Z = _rows(torch.randint(-2, 3, (N, V), generator=g).float(), dtype)
    f = lambda x: torch.full((N,), x, device="cuda")  # noqa: E731
    for k, p in ((1, 1.0), (40, 0.5), (0, 0.3), (0, 0.9), (2000, 0.77), (4999, 0.99)):
        kk = torch.full((N,), k, dtype=torch.int32, device="cuda")
        _check_sample(Z, _draws(N, k), f(1.0), top_k=kk, top_p=f(p))


def test_sample_frequencies():
    """65536 draws from one row against the fp64 probabilities: within 5 standard deviations."""
    N, V = 65536, 37
    z = _logits(1, V, 9, scale=1.5).expand(N, V)
    g = torch.Generator().manual_seed(10)
    u = torch.randint(-(1 << 31), 1 << 31, (N,), generator=g, dtype=torch.int64).to(torch.int32).cuda()
    out = dict(token=_new(N, dtype=torch.int32))
    alr.alr_sample_tokens(z.cuda().contiguous(), u, out, temperature=torch.full((N,), 0.9, device="cuda"))
    p = torch.softmax(z[0].double() / 0.9, 0).numpy()
    n = np.bincount(P.npi(out["token"]), minlength=V)
    assert (np.abs(n - N * p) <= 5 * np.sqrt(N * p) + 1).all()


# --------------------------------------------------------------- calls and their refusals ---
def test_no_rows():
    for dtype in (BF, F32):
        Z = torch.empty(0, 50, dtype=dtype, device="cuda")
        e, i = torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
        alr.alr_top_logits(Z, 3, dict(top_val=e, top_idx=i))
        alr.alr_sample_tokens(Z, i, dict(token=i))
        out = dict(loss_row=e, lse=e, loss_total=_new(1), weight_sum=_new(1))
        alr.alr_distill_fwd_bwd(Z, e.view(0, 3), i.view(0, 3), out, Z.clone())
        assert out["loss_total"].item() == 0 and out["weight_sum"].item() == 0


def test_binding_refuses_wrong_buffers():
    N, V, K = 4, 64, 3
    Z, u = torch.randn(N, V, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    val, idx = _new(N, K), _new(N, K, dtype=torch.int32)
    out = dict(top_val=val, top_idx=idx)
    for bad, what in ((Z.t(), "contiguous rows"), (Z[:1].expand(N, V), "contiguous rows"),
                      (Z.view(-1), "matrix"), (Z.cpu(), "CUDA device"), (Z.half(), "dtype")):
        with pytest.raises(ValueError, match=what):
            alr.alr_top_logits(bad, K, out)
    with pytest.raises(ValueError, match="fewer than"):
        alr.alr_top_logits(Z, K + 1, out)
    with pytest.raises(alr.AlrError, match="aligned"):
        alr.alr_top_logits(torch.randn(N * V + 1, device="cuda")[1:].view(N, V), K, out)
    with pytest.raises(alr.AlrError, match="temperature"):
        alr.alr_top_logits(Z, K, out, temperature=0.0)
    with pytest.raises(ValueError, match="token must be"):
        alr.alr_sample_tokens(Z, u, dict(token=_new(N)))
    with pytest.raises(ValueError, match="G must be"):
        alr.alr_distill_fwd_bwd(Z, val, idx, _distill_out(N), torch.empty(N, V + 1, device="cuda"))
    with pytest.raises(ValueError, match="G must be"):
        alr.alr_distill_fwd_bwd(Z, val, idx, _distill_out(N), Z.bfloat16())
    with pytest.raises(alr.AlrError, match="lse_rest"):
        o = _distill_out(N)
        del o["lse_rest"]
        alr.alr_distill_fwd(Z, val, idx, o, rest=_new(N))


def test_another_stream_and_a_graph():
    """Calls on a side stream and replayed from a CUDA graph give the eager results."""
    N, V, K = 8, 5000, 8
    val, idx, rest = _teacher(N, V, K, 1.0, seed=31)
    Z, u = _rows(_logits(N, V, 32), BF), _draws(N, 33)
    def all_ops(o, G, s):
        alr.alr_top_logits(Z, K, o["top"])
        alr.alr_sample_tokens(Z, u, o["sample"], top_p=s)
        alr.alr_distill_fwd_bwd(Z, val, idx, o["distill"], G, rest=rest)
    def new():
        return dict(top=dict(top_val=_new(N, K), top_idx=_new(N, K, dtype=torch.int32), lse=_new(N)),
                    sample=dict(token=_new(N, dtype=torch.int32), prob=_new(N)),
                    distill=_distill_out(N)), _new(N, V, dtype=BF)
    top_p = torch.full((N,), 0.8, device="cuda")
    (want, Gw), (got, G), (rep, Gr) = new(), new(), new()
    all_ops(want, Gw, top_p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_ops(got, G, top_p)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        all_ops(rep, Gr, top_p)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for o, g in ((got, G), (rep, Gr)):
        assert torch.equal(g, Gw)
        for k in want:
            for f in want[k]:
                assert torch.equal(o[k][f].view(torch.int32), want[k][f].view(torch.int32)), (k, f)
