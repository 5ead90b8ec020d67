"""The paged key-value cache on the GPU against the oracle.

Plans and appended rows are compared bit for bit.  Attention: with u = 2^-24 a score, a sum of `dim`
products in fp32 (on tensor cores truncated, so 2 u a step), is off by dx = 2 (dim + 4) u reach, reach the
largest sum of |q k| scale; a weight by 2 dx and its exponential's 2^-21, of a bf16 cache by half a step of
bf16 (2^-8) more; the sums over n tokens by 2 (n + 16) u; the output by its own rounding."""

import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from paper_2609_38795_gb300 import alr, build_lib
from tests import parity as P

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    build_lib.build()
    alr.lib()
    assert alr.alr_device_supported() == alr.ALR_OK, alr.alr_last_error()


def _i(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


# ------------------------------------------------------------------------------ plan ---
def _plan(length, add, pool, used, table, page, T, in_place=False):
    t = dict(len=_i(length), add=_i(add), pool=_i(pool), used=_i([used]), table=_i(table))
    S = len(length)
    e = lambda n: torch.full((n,), 77, dtype=torch.int32, device="cuda")  # noqa: E731
    out = dict(len=t["len"] if in_place else e(S), slot=e(T), pool_used=t["used"] if in_place else e(1),
               start=e(S + 1), tok_seq=e(T), tok_len=e(T), n_refused=e(1))
    alr.alr_kv_plan(t["len"], t["add"], t["pool"], t["used"], t["table"], page, out)
    got = {k: v.cpu().numpy() for k, v in dict(out, pool=t["pool"], table=t["table"]).items()}
    want = ko.plan(np.asarray(length), np.asarray(add), np.asarray(pool), used, np.asarray(table), page, T)
    for k, v in want.items():
        assert np.array_equal(got[k].reshape(-1), np.asarray(v).reshape(-1)), k
    return want


def _state(S, page, cols, n_pool, lengths, seed):
    rng = np.random.default_rng(seed)
    length = np.minimum(lengths(rng), cols * page)
    table, pool, used = np.full((S, cols), -1), rng.permutation(n_pool), 0
    for s in range(S):
        n = min(-(-length[s] // page), n_pool - used)
        length[s] = min(length[s], n * page)
        table[s, :n] = pool[used:used + n]
        used += n
    return length, table, pool, used, rng


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("S,page,cols,n_pool,most,T", [
    (1, 1, 1, 1, 1, 1), (1, 16, 4, 3, 70, 64), (5, 3, 7, 20, 9, 17), (33, 16, 9, 200, 1, 33),
    (257, 8, 40, 3000, 30, 2000), (1025, 16, 20, 9000, 2, 1500), (3000, 4, 6, 9000, 40, 30000),
    (8192, 16, 3, 9000, 1, 8192), (40, 48, 60, 900, 900, 20000)])
def test_plan(S, page, cols, n_pool, most, T, in_place):
    length, table, pool, used, rng = _state(S, page, cols, n_pool,
                                            lambda r: r.integers(0, cols * page // 2 + 2, S), S)
    for add in (rng.integers(0, most + 1, S), rng.integers(-1, most + 1, S), np.full(S, most), np.full(S, -1),
                np.zeros(S, int), np.where(rng.random(S) < 0.1, most, -1)):
        _plan(length, add, pool, used, table, page, T, in_place)


def test_plan_of_huge_requests():
    """Requests whose sum passes 32 bits, and one past the batch, are refused; later ones fit or not."""
    for add in ([2 ** 31 - 1] * 4, [3, 2 ** 31 - 1, 2], [0, 9, 1], [8, 1, 0], [2, 100, -1]):
        S = len(add)
        table = np.full((S, 4), -1)
        got = _i(add)
        e = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
        out = dict(len=e(S), slot=e(8), pool_used=e(1), start=e(S + 1), n_refused=e(1))
        alr.alr_kv_plan(_i([0] * S), got, _i(np.arange(10)), _i([0]), _i(table), 4, out)
        want = ko.plan(np.zeros(S, int), np.array(add), np.arange(10), 0, table, 4, 8)
        for k in ("len", "slot", "pool_used", "n_refused"):
            assert np.array_equal(out[k].cpu().numpy().reshape(-1), np.asarray(want[k]).reshape(-1)), (add, k)
        assert np.array_equal(out["start"].cpu().numpy(), np.minimum(want["start"], 2 ** 31 - 1))


def test_plan_of_nothing():
    z = torch.empty(0, dtype=torch.int32, device="cuda")
    out = dict(len=z, slot=torch.full((3,), 9, dtype=torch.int32, device="cuda"), pool_used=_i([5]), start=_i([7]))
    alr.alr_kv_plan(z, z, _i([1, 2]), _i([1]), z.view(0, 4), 16, out)
    assert out["pool_used"].tolist() == [1] and out["slot"].tolist() == [-1] * 3 and out["start"].tolist() == [0]


def test_plan_bounds_what_it_reads():
    """Lengths past the table, a pool_used past the pool, more pages back than were taken."""
    S, cols, page = 3, 2, 4
    table = _i(np.arange(6).reshape(3, 2))
    e = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
    out = dict(len=e(S), slot=e(4), pool_used=e(1), n_refused=e(1))
    pool = _i([50, 51, 52])
    alr.alr_kv_plan(_i([100, -7, 8]), _i([-1, 1, -1]), pool, _i([9]), table, page, out)
    assert out["len"].tolist() == [0, 1, 0] and out["slot"].tolist() == [0, -1, -1, -1]
    assert pool.tolist() == [1, 4, 5] and out["pool_used"].tolist() == [0] and out["n_refused"].tolist() == [0]
    assert table[1, 0] == 0


# ---------------------------------------------------------------------------- append ---
def _cache(n_pages, page, heads, dim, dtype, hnd, g, fill=None):
    shape = (n_pages, heads, page, dim) if hnd else (n_pages, page, heads, dim)
    kv = [torch.randn(*shape, generator=g).to(dtype).cuda() if fill is None else
          torch.full(shape, fill, dtype=dtype, device="cuda") for _ in "KV"]
    return [t.transpose(1, 2) if hnd else t for t in kv]


@pytest.mark.parametrize("src,dtype", [(BF, BF), (F32, BF), (F32, F32), (BF, F32)])
@pytest.mark.parametrize("T,heads,dim,page,n_pages,hnd,extra", [
    (1, 1, 8, 1, 2, False, 0), (7, 3, 16, 5, 4, True, 0), (33, 2, 128, 16, 5, False, 64), (200, 8, 80, 20, 14, True, 40),
    (1000, 5, 256, 48, 30, False, 0), (64, 16, 112, 7, 12, True, 200)])
def test_append(T, heads, dim, page, n_pages, hnd, extra, src, dtype):
    g = torch.Generator().manual_seed(T)
    K, V = _cache(n_pages, page, heads, dim, dtype, hnd, g)
    slot = torch.randperm(n_pages * page, generator=g)[:T].int()
    if T > 5:
        slot[::5] = torch.tensor([-1, n_pages * page, -2 ** 31, 2 ** 31 - 1])[torch.arange(len(slot[::5])) % 4].int()
    new = [torch.randn(T, heads * dim + extra, generator=g).to(src).cuda()[:, extra:].unflatten(1, (heads, dim))
           for _ in "KV"]
    want = [K.clone(), V.clone()]
    for i, s in enumerate(slot.tolist()):
        if 0 <= s < n_pages * page:
            for w, x in zip(want, new):
                w[s // page, s % page] = x[i].to(dtype)
    alr.alr_kv_append(*new, K, V, slot.cuda())
    assert torch.equal(K, want[0]) and torch.equal(V, want[1])


# ------------------------------------------------------------------------- attention ---
class Case:
    """Sequences of given lengths in a cache whose other slots hold NaN; `rows` of (seq, len) and
    maybe (prefix_seq, prefix_len)."""

    def __init__(self, lengths, rows, prefix=None, heads=2, group=2, dim=64, page=16, dtype=BF, hnd=False,
                 seed=0, spare=3, sharp=1.0, scale=None, size=1.0):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        held = [-(-n // page) for n in lengths]
        n_pages, cols = sum(held) + spare, max(held + [1])
        pages = rng.permutation(n_pages)
        self.table = np.full((len(lengths), cols), -1)
        self.K, self.V = _cache(n_pages, page, heads, dim, dtype, hnd, g, fill=NAN)
        at = 0
        for s, n in enumerate(lengths):
            self.table[s, :held[s]] = pages[at:at + held[s]]
            at += held[s]
            t = np.arange(n)
            pg, pos = self.table[s, t // page], t % page
            for c in (self.K, self.V):
                c[pg, pos] = (size * torch.randn(n, heads, dim, generator=g)).to(dtype).cuda()
        self.rows, self.prefix, self.page = np.asarray(rows).reshape(-1, 2), prefix, page
        N, H = len(self.rows), heads * group
        self.Q = (sharp * torch.randn(N, H, dim, generator=g)).to(dtype).cuda()
        self.scale = dim ** -0.5 if scale is None else scale

    def run(self, per=1, per_prefix=1, seq=True, lse=True, out=None, ws=None):
        N, H, dim = self.Q.shape
        out = torch.full_like(self.Q, 9.0) if out is None else out
        n = alr.alr_kv_attention_workspace_size(N, H, dim, prefix=self.prefix is not None)
        if ws is None:
            ws = torch.randint(0, 256, (n,), dtype=torch.uint8, device="cuda")   # whatever it held
        l = torch.full((N, H), 9.0, device="cuda") if lse else None  # noqa: E741
        kw = {}
        if self.prefix is not None:
            p = np.asarray(self.prefix).reshape(-1, 2)
            kw = dict(prefix_seq=_i(p[:, 0]), prefix_len=_i(p[:, 1]))
        alr.alr_kv_attention(self.Q, self.K, self.V, _i(self.table), _i(self.rows[:, 1]), out, ws,
                             seq=_i(self.rows[:, 0]) if seq else None, lse=l, scale=self.scale,
                             rows_per_seq=per, rows_per_prefix=per_prefix, **kw)
        torch.cuda.synchronize()
        assert alr.alr_device_status() == alr.ALR_OK
        return out, l

    def expected(self):
        if not hasattr(self, "_want"):
            parts = [self.rows.T] + ([] if self.prefix is None else [np.asarray(self.prefix).reshape(-1, 2).T])
            self._want = ko.attention(P.np64(self.Q), P.np64(self.K), P.np64(self.V), self.table, parts, self.scale)
        return self._want

    def check(self, **kw):
        out, lse = self.run(**kw)
        ref, ref_lse, size, reach, n = self.expected()
        u, dim = 2.0 ** -24, self.Q.shape[2]
        bf = self.Q.dtype == BF
        dx = 2 * (dim + 4) * u * reach
        rel = 2 * dx + 2.0 ** -21 + 2 * (n[:, None] + 16) * u + (2.0 ** -8 if bf else 0.0)
        tol = rel[:, :, None] * size + (2.0 ** -8 if bf else u) * np.abs(ref) + 1e-30
        err = np.abs(P.np64(out) - ref)
        assert (err <= tol).all(), (np.argwhere(~(err <= tol))[:5], np.nanmax(err / tol), np.isnan(err).sum())
        none = ref_lse == -np.inf
        got = P.np64(lse)
        assert (got[none] == -np.inf).all() and not P.np64(out)[none].any()
        some = ~none
        ltol = dx + 2.0 ** -21 + 2 * (n[:, None] + 16) * u + 4 * u * np.abs(ref_lse)
        assert (np.abs(got[some] - ref_lse[some]) <= ltol[some]).all()
        return out, lse


FORMS = [dict(heads=2, group=2, dim=64, page=16, dtype=BF), dict(heads=1, group=4, dim=128, page=16, dtype=BF),
         dict(heads=3, group=1, dim=16, page=5, dtype=BF, hnd=True), dict(heads=1, group=7, dim=80, page=48, dtype=BF),
         dict(heads=2, group=16, dim=128, page=1, dtype=BF, hnd=True), dict(heads=1, group=20, dim=256, page=64, dtype=BF),
         dict(heads=1, group=1, dim=8, page=3, dtype=BF), dict(heads=2, group=5, dim=112, page=128, dtype=BF, hnd=True),
         dict(heads=1, group=8, dim=32, page=8, dtype=BF), dict(heads=1, group=3, dim=200, page=20, dtype=BF),
         dict(heads=2, group=1, dim=80, page=20, dtype=F32), dict(heads=1, group=4, dim=128, page=16, dtype=F32, hnd=True),
         dict(heads=2, group=7, dim=36, page=7, dtype=F32), dict(heads=1, group=17, dim=256, page=32, dtype=F32),
         dict(heads=3, group=2, dim=4, page=1, dtype=F32)]


@pytest.mark.parametrize("form", FORMS + [dict(heads=1, group=71, dim=64, page=16, dtype=BF),
                                          dict(heads=2, group=32, dim=128, page=8, dtype=BF, hnd=True),
                                          dict(heads=1, group=150, dim=80, page=20, dtype=BF)])
def test_decode(form):
    """One row for each sequence: lengths from none on, either side of pages and of tiles."""
    p = form["page"]
    lengths = [0, 1, 2, p - 1, p, p + 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 300, 0, 511, 700]
    c = Case(lengths, list(enumerate(lengths)), **form)
    out, lse = c.check(seq=False)
    again, lse2 = c.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("per", [2, 5, 8, 16, 40])
def test_blocks(form, per):
    """Rows under a causal mask, blocks cut short, whole blocks of nothing."""
    rng = np.random.default_rng(per)
    lengths = [1, per, per + 3, 150, 64, 0, 290]
    rows = []
    for s, n in enumerate(lengths):
        cut = rng.integers(0, per + 1)
        rows += [(s, max(0, n - per + 1 + j) if j < cut or s == 3 else 0) for j in range(per)]
    c = Case(lengths, rows, seed=per, **form)
    c.check(per=per)
    if per == 8:
        c.check(per=per, seq=False)
        for other in (1, 3, 64):               # a hint that is wrong costs time, nothing else
            c.check(per=other)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("share", [2, 6, 33])
def test_prefixes(form, share):
    """Rollouts that share a prefix, each up to its own anchor, some without one or without own tokens."""
    rng = np.random.default_rng(share)
    n = 3 * share - 1
    lengths = [int(x) for x in rng.integers(0, 20, n)] + [200, 1, 77]
    rows = [(i, lengths[i]) for i in range(n)]
    prefix = [(n + i // share, int(rng.integers(0, lengths[n + i // share] + 1))) for i in range(n)]
    c = Case(lengths, rows, prefix=prefix, seed=share, **form)
    c.check(per_prefix=share)
    c.check(per_prefix=1)
    c.check(per_prefix=4 * share)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_in_any_order(dtype):
    """Sequences that come back, rows of other sequences between, sequences and pages outside."""
    rng = np.random.default_rng(3)
    lengths = [40, 100, 7, 260]
    seqs = rng.integers(-1, 6, 70)
    rows = [(int(s), int(rng.integers(-3, lengths[s] + 1)) if 0 <= s < 4 else 50) for s in seqs]
    prefix = [(int(s), int(rng.integers(-3, lengths[s] + 1)) if 0 <= s < 4 else 50) for s in rng.integers(-1, 6, 70)]
    for p in (None, prefix):
        c = Case(lengths, rows, prefix=p, page=16, dim=64, dtype=dtype)
        c.table[3, 5], c.table[1, 0] = -1, c.K.shape[0]     # holes
        for per in (1, 4, 16, 70):
            c.check(per=per, per_prefix=per)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("per", [1, 4, 32])
def test_poison_reaches_only_its_readers(dtype, per):
    """A NaN or infinity in a key or value that some rows of a tile read: the others are untouched."""
    lengths, page = [300, 260], 16
    rows = [(s, lengths[s] - 2 * (31 - j)) for s in range(2) for j in range(32)]
    for bad, where in ((NAN, "V"), (float("inf"), "V"), (NAN, "K")):
        clean = Case(lengths, rows, page=page, dim=64, dtype=dtype)
        clean.check(per=per)
        c = Case(lengths, rows, page=page, dim=64, dtype=dtype)
        cache = getattr(c, where)
        t = 270                                              # of sequence 0: rows with len > 270
        cache[c.table[0, t // page], t % page] = bad
        hit = torch.tensor([s == 0 and n > t for s, n in rows]).cuda()
        out, lse = c.run(per=per)
        ref, ref_lse = clean.run(per=per)
        assert torch.isnan(out[hit].float()).any(-1).all() or bad == float("inf")
        assert not torch.isfinite(out[hit].float()).any()
        diff = (out[~hit].float() - ref[~hit].float()).abs()
        assert bool((diff <= 2.0 ** -7 * ref[~hit].float().abs() + 2.0 ** -7).all())
        assert torch.allclose(lse[~hit], ref_lse[~hit], rtol=0, atol=1e-4)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-30, 3.0])
def test_scales(dtype, scale):
    rows = [(s, n) for s in range(3) for n in (0, 5, 200, 260)]
    for per in (1, 4):
        Case([270, 280, 261], rows, dim=64, dtype=dtype, group=8, scale=scale).check(per=per)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("per,group", [(1, 1), (16, 1), (16, 2), (16, 8)])
def test_extreme_scores(dtype, per, group):
    """Keys of -inf (tokens masked in the cache), scores of thousands, one token that has all the mass,
    rising and falling scores."""
    n = 400
    c = Case([n], [(0, n - 15 + j) for j in range(16)], dim=64, dtype=dtype, heads=1, group=group)
    flat_k, flat_v = c.K.clone(), c.V.clone()
    pg, pos = c.table[0, np.arange(n) // 16], np.arange(n) % 16
    q = c.Q.clone()
    for slope in (-200.0, 200.0, 0.02):
        c.K[pg, pos] = flat_k[pg, pos]
        c.Q.copy_(q)
        c.Q[..., 0] = 8.0
        c.K[pg, pos, :, 0] = (torch.arange(n, device="cuda")[:, None] * slope / 64).to(dtype)
        c.__dict__.pop("_want", None)
        c.check(per=per)
    for top in (1e9, -1e9, 1e30, -1e30):                     # large scores next to ordinary ones
        c.K[pg, pos] = flat_k[pg, pos]
        c.K[pg[::2], pos[::2], :, 0] = top
        c.__dict__.pop("_want", None)
        c.check(per=per)
        c.K[pg, pos, :, 0] = top                             # all alike but for what is below their rounding
        c.__dict__.pop("_want", None)
        out, lse = c.run(per=per)
        assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()
        assert bool((out.float().abs() <= flat_v[pg, pos].float().abs().max() * 1.01).all())
    c.K[pg, pos] = flat_k[pg, pos]
    c.K[pg[::3], pos[::3], :, 0] = -float("inf")             # a third of the tokens masked by their keys
    c.__dict__.pop("_want", None)
    c.check(per=per)
    c.K[pg, pos, :, 0] = -float("inf")                       # all of them
    c.__dict__.pop("_want", None)
    c.check(per=per)


def test_long_offsets():
    """A cache of more than 2^32 bytes and 2^31 elements a tensor."""
    page, heads, dim = 64, 8, 128
    n_pages = (1 << 31) // (page * heads * dim) + 40
    K = torch.empty(n_pages, page, heads, dim, dtype=BF, device="cuda")
    V = torch.empty_like(K)
    g = torch.Generator().manual_seed(0)
    pages = [n_pages - 1, 0, n_pages - 3, n_pages // 2]
    n = 4 * page - 5
    for i, p in enumerate(pages):
        K[p] = torch.randn(page, heads, dim, generator=g).cuda()
        V[p] = torch.randn(page, heads, dim, generator=g).cuda()
    c = Case([1], [(0, n)], heads=heads, group=2, dim=dim, page=page)
    small = torch.tensor(pages, device="cuda")
    c.K, c.V, c.table = K[small], V[small], np.arange(4)[None]
    want, _ = c.check()
    c.K, c.V, c.table = K, V, np.array([pages])
    got, _ = c.run()
    assert torch.equal(got, want)
    slot = _i([n_pages * page - 1])
    row = torch.randn(1, heads, dim, generator=g).cuda()
    alr.alr_kv_append(row, row, K, V, slot)
    assert torch.equal(K[-1, -1], row[0].to(BF)) and torch.equal(V[-1, -1], row[0].to(BF))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form", [dict(heads=4, group=2, dim=32, page=16), dict(heads=3, group=1, dim=128, page=32),
                                  dict(heads=2, group=12, dim=64, page=20), dict(heads=5, group=5, dim=48, page=8, hnd=True)])
def test_many_blocks(form, dtype):
    """More blocks than workers: stretches that end inside items, items over many workers and thread blocks."""
    rng = np.random.default_rng(5)
    lengths = [0, 1, 3000, 5, 40, 2047, 0, 900] + [int(x) for x in np.exp(rng.uniform(0, 7.5, 40))] + [6000]
    c = Case(lengths, list(enumerate(lengths)), dtype=dtype, **form)
    out, lse = c.check(seq=False)
    for _ in range(2):                         # whatever the workspace held
        again, lse2 = c.run()
        assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form", [dict(heads=2, group=4, dim=64, page=16), dict(heads=1, group=8, dim=128, page=32),
                                  dict(heads=2, group=3, dim=80, page=20, hnd=True),
                                  dict(heads=1, group=2, dim=24, page=64), dict(heads=1, group=4, dim=112, page=8)])
def test_many_block_rows(form, dtype):
    """Tiles of rows over long sequences, cut at stretches' ends, some rows ending tiles before others."""
    rng = np.random.default_rng(6)
    lengths, per = [3000, 16, 0, 1500, 129, 128, 127, 2500], 16
    rows = [(s, max(0, n - int(rng.integers(0, 2 * per)))) if rng.random() < 0.9 else (s, int(rng.integers(0, n + 1)))
            for s, n in enumerate(lengths) for _ in range(per)]
    c = Case(lengths, rows, dtype=dtype, **form)
    out, lse = c.check(per=per)
    again, lse2 = c.run(per=per)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("heads,group,dim,dtype", [(1, 1, 64, BF), (2, 8, 128, BF), (1, 16, 256, BF), (1, 4, 128, F32)])
def test_one_long_sequence(heads, group, dim, dtype):
    c = Case([20011], [(0, 20011)], heads=heads, group=group, dim=dim, dtype=dtype, page=64)
    c.check()


def test_lengths_past_the_table():
    """Lengths past what the table holds count as that; rows of a sequence that is not there are empty."""
    c = Case([64, 64], [(0, 10 ** 6), (1, 2 ** 31 - 1), (1, -2 ** 31), (2 ** 31 - 1, 5), (-2 ** 31, 5)], page=16)
    c.check()
    c = Case([64, 64], [(s, 10 ** 6) for s in range(2) for _ in range(16)], page=16, group=4)
    c.check(per=16)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strided_rows(dtype):
    """Queries out of a fused projection, results into wider rows, whose other elements stay."""
    rows = [(s, 50 * s + j) for s in range(4) for j in range(8)]
    for per, group in ((1, 2), (8, 2), (8, 4)):
        c = Case([10, 60, 110, 160], rows, dtype=dtype, group=group, dim=64)
        N, H, dim = c.Q.shape
        wide = torch.randn(N, 3 * H * dim, device="cuda").to(dtype)
        wide[:, H * dim:2 * H * dim] = c.Q.reshape(N, -1)
        want, _ = c.run(per=per)
        c.Q = wide[:, H * dim:2 * H * dim].unflatten(1, (H, dim))
        to = torch.full((N + 2, H * dim + 64), 3.0, dtype=dtype, device="cuda")
        got, _ = c.run(per=per, out=to[:N, 32:32 + H * dim].unflatten(1, (H, dim)))
        assert torch.equal(got, want)
        assert (to[N:] == 3).all() and (to[:, :32] == 3).all() and (to[:, 32 + H * dim:] == 3).all()


def test_two_calls_at_once():
    """Calls on two streams, each with a workspace of its own."""
    a = Case([4000] * 6, [(s, 4000 - s) for s in range(6)], heads=2, group=4, dim=128)
    b = Case([3000] * 4, [(s, 3000 - j) for s in range(4) for j in range(16)], heads=2, group=4, dim=128, seed=1)
    want = a.run()[0], b.run(per=16)[0]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    calls = []
    for c, per in ((a, 1), (b, 16)):
        N, H, dim = c.Q.shape
        n = alr.alr_kv_attention_workspace_size(N, H, dim)
        calls.append((c, per, torch.empty_like(c.Q), torch.empty(n, dtype=torch.uint8, device="cuda"), _i(c.table),
                      _i(c.rows[:, 1]), _i(c.rows[:, 0])))
    torch.cuda.synchronize()
    for _ in range(20):
        for s, (c, per, out, ws, table, length, seq) in zip(streams, calls):
            alr.alr_kv_attention(c.Q, c.K, c.V, table, length, out, ws, seq=seq, rows_per_seq=per, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(call[2], w) for call, w in zip(calls, want))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("most", [1, 5])
def test_steps_in_a_graph(dtype, most):
    """Plan, append and attention of a rollout's steps as one captured graph, replayed as sequences grow, end and
    begin again; rows of the batch beyond its tokens are empty."""
    S, page, cols, heads, group, dim, T = 9, 8, 6, 2, 2, 64, 24
    n_pool, H = 40, heads * group
    g = torch.Generator().manual_seed(most)
    rng = np.random.default_rng(most)
    K, V = _cache(n_pool, page, heads, dim, dtype, False, g, fill=NAN)
    length, add, pool, used = _i(np.zeros(S)), _i(np.zeros(S)), _i(rng.permutation(n_pool)), _i([0])
    table = torch.full((S, cols), -1, dtype=torch.int32, device="cuda")
    e = lambda *n: torch.empty(*n, dtype=torch.int32, device="cuda")  # noqa: E731
    plan = dict(len=length, slot=e(T), pool_used=used, start=e(S + 1), tok_seq=e(T), tok_len=e(T), n_refused=e(1))
    qkv = torch.zeros(T, (H + 2 * heads) * dim, device="cuda")
    cut = [H * dim, (H + heads) * dim]
    k_new, v_new = (qkv[:, cut[i]:cut[i] + heads * dim].unflatten(1, (heads, dim)) for i in range(2))
    q = torch.zeros(T, H, dim, dtype=dtype, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(T, H, device="cuda")
    ws = torch.empty(alr.alr_kv_attention_workspace_size(T, H, dim), dtype=torch.uint8, device="cuda")

    def step():
        alr.alr_kv_plan(length, add, pool, used, table, page, plan)
        alr.alr_kv_append(k_new, v_new, K, V, plan["slot"])
        q.copy_(qkv[:, :H * dim].unflatten(1, (H, dim)))
        alr.alr_kv_attention(q, K, V, table, plan["tok_len"], out, ws, seq=plan["tok_seq"], lse=lse, rows_per_seq=most)

    step()                                                   # nothing to do: loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    held = {s: [] for s in range(S)}                         # each sequence's (key, value) rows
    for n in range(25):
        a = rng.integers(0, most + 1, S) if n % 5 else rng.integers(-1, most + 1, S)
        add.copy_(_i(a))
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        before = [len(held[s]) for s in range(S)]
        graph.replay()
        torch.cuda.synchronize()
        start, slot = plan["start"].tolist(), plan["slot"].tolist()
        for s in range(S):
            if a[s] < 0:
                held[s] = []
            else:
                rows = range(start[s], start[s] + a[s])
                took = [r for r in rows if r < T and slot[r] >= 0]
                assert len(took) in (0, a[s])
                held[s] += [(k_new[r].to(dtype).clone(), v_new[r].to(dtype).clone()) for r in took]
        assert length.tolist() == [len(held[s]) for s in range(S)]
        seqs, lens = plan["tok_seq"].tolist(), plan["tok_len"].tolist()
        for r in range(T):
            if seqs[r] < 0:
                assert lens[r] == 0 and not out[r].any() and (lse[r] == -float("inf")).all()
                continue
            assert lens[r] == before[seqs[r]] + r - start[seqs[r]] + 1
            k, v = (torch.stack([x[i] for x in held[seqs[r]][:lens[r]]]).double().repeat_interleave(group, 1)
                    for i in range(2))
            x = (k * q[r].double()).sum(-1) * dim ** -0.5     # [tokens, H]
            want = (torch.softmax(x, 0)[..., None] * v).sum(0)
            # scores and values of order 3: two roundings of bf16, or the sums' of fp32
            assert (out[r].double() - want).abs().max() <= (2 * 2.0 ** -8 if dtype == BF else 1e-5) * v.abs().max()
            assert (lse[r].double() - torch.logsumexp(x, 0)).abs().max() <= 1e-5 * max(1.0, float(x.abs().max()))


def test_binding_refuses_wrong_buffers():
    c = Case([20], [(0, 20)])
    N, H, dim = c.Q.shape
    ws = torch.empty(alr.alr_kv_attention_workspace_size(N, H, dim), dtype=torch.uint8, device="cuda")
    table, length, out = _i(c.table), _i([20]), torch.empty_like(c.Q)
    call = lambda Q=c.Q, K=c.K, V=c.V, t=table, n=length, o=out, w=ws, **kw: (  # noqa: E731
        alr.alr_kv_attention(Q, K, V, t, n, o, w, **kw))
    call()
    for match, kw in (("laid out alike", dict(V=c.V[:-1])), ("must be torch.bfloat16", dict(V=c.V.float())),
                      ("4 dimensions", dict(K=c.K[0])), ("overlap", dict(K=c.K[:1].expand(5, -1, -1, -1), V=c.V)),
                      ("last dimension", dict(K=c.K.transpose(2, 3))), ("must be torch.bfloat16", dict(Q=c.Q.float())),
                      ("must be \\[N, H, 64\\]", dict(o=out[:, :1])), ("table must be", dict(t=table[0])),
                      ("table must be torch.int32", dict(t=table.long())), ("len holds", dict(n=length[:0])),
                      ("heads must be contiguous", dict(Q=torch.empty(1, H, 2 * dim, dtype=BF, device="cuda")[..., :dim])),
                      ("lse holds", dict(lse=torch.empty(1, device="cuda")))):
        with pytest.raises(ValueError, match=match):
            call(**kw)
    for match, kw in (("go together", dict(prefix_len=length)), ("workspace", dict(w=ws[:64])),
                      ("workspace", dict(w=None)), ("rows_per_seq", dict(rows_per_seq=0)), ("scale", dict(scale=NAN))):
        with pytest.raises(alr.AlrError, match=match):
            call(**kw)
    with pytest.raises(alr.AlrError, match="prefix|workspace"):
        call(prefix_len=length, prefix_seq=_i([0]), w=ws[:-1])
    new = torch.zeros(3, 2, 64, device="cuda")
    with pytest.raises(ValueError, match="rows of"):
        alr.alr_kv_append(new[:, :1], new[:, :1], c.K, c.V, _i([0, 1, 2]))
    with pytest.raises(ValueError, match="slot holds"):
        alr.alr_kv_append(new, new, c.K, c.V, _i([0, 1]))
    with pytest.raises(ValueError, match="laid out alike"):
        alr.alr_kv_append(new, new[:2], c.K, c.V, _i([0, 1, 2]))
    with pytest.raises(ValueError, match="table must be"):
        alr.alr_kv_plan(length, length, length, length, table[:0], 16, dict(len=length, slot=_i([0]), pool_used=_i([0])))
    with pytest.raises(KeyError):
        alr.alr_kv_plan(length, length, length, length, table, 16, dict(len=length))
