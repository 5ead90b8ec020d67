"""Pins of the oracle of the operators on logits in hand: closed forms, brute force, differences."""

import itertools

import numpy as np
import pytest
import torch

from oracle import alr_oracle as orc
from oracle import logits_oracle as lo


def _rng(seed):
    return np.random.default_rng(seed)


def test_top_logits_order_ties_and_masks():
    z = np.array([[1.0, 3.0, -np.inf, 3.0, np.nan, 2.0], [-np.inf] * 6, [0.0, -0.0, 5.0, 5.0, 5.0, 1.0]])
    t = lo.top_logits(z, 4)
    assert t["top_idx"].tolist() == [[1, 3, 5, 0], [-1] * 4, [2, 3, 4, 5]]
    assert t["lse_rest"][0] == -np.inf and t["lse"][1] == -np.inf
    np.testing.assert_allclose(t["lse_rest"][2], np.log(2.0), rtol=1e-15)
    z = _rng(0).standard_normal((5, 30))
    t = lo.top_logits(z, 7, T=1.7)
    np.testing.assert_allclose(t["lse"], torch.logsumexp(torch.tensor(z) / 1.7, 1).numpy(), rtol=1e-14)
    both = np.logaddexp(t["lse_rest"], torch.logsumexp(torch.tensor(t["top_val"]) / 1.7, 1).numpy())
    np.testing.assert_allclose(both, t["lse"], rtol=1e-14)


def test_distill_with_the_whole_vocabulary_listed_is_soft_cross_entropy():
    r = _rng(1)
    zs, zt = r.standard_normal((6, 9)) * 2, r.standard_normal((6, 9)) * 2
    t = lo.top_logits(zt, 9, T=2.0)
    d = lo.distill(zs, t["top_val"], t["top_idx"], rest=t["lse_rest"], T=2.0)
    p = torch.softmax(torch.tensor(zt) / 2.0, 1)
    want = torch.nn.functional.cross_entropy(torch.tensor(zs) / 2.0, p, reduction="none").numpy()
    np.testing.assert_allclose(d["loss_row"], want, rtol=1e-13)
    np.testing.assert_allclose(d["loss_total"], want.mean(), rtol=1e-13)


def test_distill_at_temperature_one_is_the_compact_label_loss():
    """The framework's own top-8 + tail loss, from probabilities, at T = 1."""
    r = _rng(2)
    N, V, K = 5, 40, 8
    zs, zt = r.standard_normal((N, V)) * 3, r.standard_normal((N, V)) * 3
    t = lo.top_logits(zt, K)
    d = lo.distill(zs, t["top_val"], t["top_idx"], rest=t["lse_rest"])
    p = np.exp(t["top_val"] - t["lse"][:, None])
    tail = np.exp(t["lse_rest"] - t["lse"])
    q = orc.softmax(zs)
    qi = np.take_along_axis(q, t["top_idx"], 1)
    want = -(p * np.log(qi)).sum(1) - tail * np.log(1 - qi.sum(1))
    np.testing.assert_allclose(d["loss_row"], want, rtol=1e-11)
    assert (d["loss_row"] >= d["ent_row"] - 1e-12).all()       # Gibbs on the K + 1 bins


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T", [0.7, 2.0])
def test_distill_gradient_against_differences(tail, T):
    r = _rng(3)
    N, V, K = 4, 11, 3
    z = r.standard_normal((N, V)) * 2
    t = lo.top_logits(r.standard_normal((N, V)) * 2, K, T=T)
    t["top_idx"][1, 2] = -1                                    # an absent entry
    w = np.array([1.0, 0.5, 0.0, 2.0])
    kw = dict(rest=t["lse_rest"] if tail else None, weight=w, T=T, lam=1.3)
    G = lo.distill(z, t["top_val"], t["top_idx"], **kw)["G"]
    eps = 1e-5
    for i, v in itertools.product(range(N), range(V)):
        zp, zm = z.copy(), z.copy()
        zp[i, v] += eps
        zm[i, v] -= eps
        num = (lo.distill(zp, t["top_val"], t["top_idx"], **kw)["loss_total"]
               - lo.distill(zm, t["top_val"], t["top_idx"], **kw)["loss_total"]) / (2 * eps)
        assert abs(num - G[i, v]) < 1e-8                       # eps^2 and 1e-16 / eps
    np.testing.assert_allclose(G.sum(1), 0.0, atol=1e-15)      # shifting a row changes nothing


def test_distill_rows_without_a_label_or_logits():
    z = np.array([[0.0, 1.0], [-np.inf, -np.inf], [0.5, 0.0]])
    d = lo.distill(z, [[1.0], [1.0], [1.0]], np.array([[-1], [0], [0]]))
    assert d["loss_row"][0] == 0 and d["loss_row"][1] == 0 and d["weight_sum"] == 3
    assert not d["G"][:2].any() and d["G"][2].any()
    assert d["argmax"].tolist() == [1, -1, 0]


def _w32(z, T):
    z = np.asarray(z, dtype=np.float32)
    m = z.max(1, keepdims=True)
    c = (np.float32(1.4426950408889634) / np.asarray(T, dtype=np.float32))[:, None]
    return np.exp2((z - m) * c, dtype=np.float32)


def test_sample_frequencies_follow_the_truncated_softmax():
    """A fine grid of u against the probabilities of an independent fp64 truncation."""
    z = np.array([[2.0, -1.0, 0.5, 2.0, 1.0, -np.inf, 0.0, 1.5]], dtype=np.float32)
    n = 4096
    u = (np.arange(n, dtype=np.int64) * (1 << 32) // n + 12345)
    for kw, keep in (({}, [0, 1, 2, 3, 4, 6, 7]), (dict(top_k=3), [0, 3, 7]),
                     (dict(top_p=0.5), [0, 3]), (dict(min_p=0.3), [0, 3, 7]),
                     (dict(top_k=5, top_p=0.7, min_p=0.7), [0, 3])):
        args = {k: np.full(n, v) for k, v in kw.items()}
        T = np.full(n, 0.8)
        Z = np.repeat(z, n, 0)
        s = lo.sample(Z, _w32(Z, T), u, T, **args)
        p = np.exp(z[0, keep].astype(np.float64) / 0.8)
        p /= p.sum()
        assert set(s["n_kept"]) == {len(keep)}
        for v, pv in zip(keep, p):
            assert abs((s["token"] == v).mean() - pv) <= 2.0 / n
            assert np.allclose(s["prob"][s["token"] == v], pv, rtol=1e-6)


def test_sample_edges():
    z = np.array([[1.0, 3.0, 3.0], [-np.inf] * 3, [np.nan, -np.inf, 2.0]], dtype=np.float32)
    T = np.array([0.0, 1.0, 1.0])
    s = lo.sample(z, np.ones((3, 3)), np.array([-1, 5, 7]), T)
    assert s["token"].tolist() == [1, -1, 2] and s["n_kept"].tolist() == [1, 0, 1]
    z = np.zeros((2, 4), dtype=np.float32)
    s = lo.sample(z, np.ones((2, 4)), np.array([0, -1]))       # the first and the last of u
    assert s["token"].tolist() == [0, 3]
    s = lo.sample(z, np.ones((2, 4)), np.array([0, -1]), top_p=np.array([0.0, 0.5]))
    assert s["n_kept"].tolist() == [1, 2] and s["token"].tolist() == [0, 1]


def test_embed_and_its_gradient_are_adjoint():
    r = _rng(4)
    E, tok = r.standard_normal((7, 5)), np.array([3, 0, 3, -1, 7, 6, 3])
    y = lo.embed(E, tok, 2.5)
    assert not y[3].any() and not y[4].any()
    dY = r.standard_normal(y.shape)
    dE, size = lo.embed_grad(dY, tok, 7, 2.5)
    np.testing.assert_allclose((y * dY).sum(), (E * dE).sum(), rtol=1e-13)
    np.testing.assert_allclose(dE[3], 2.5 * dY[[0, 2, 6]].sum(0), rtol=1e-13)
    assert not dE[[1, 2, 4, 5]].any() and (size >= np.abs(dE)).all()
