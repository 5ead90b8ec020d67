"""Calls of the paged key-value cache at the edges of what its documentation allows, on the GPU.

u = 2^-24; bounds as in test_gpu_kv.py, each derived where it is used."""

import time

import numpy as np
import pytest
import torch

from paper_2609_38795_gb300 import alr, build_lib
from tests.test_gpu_kv import Case

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")
U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    build_lib.build()
    alr.lib()
    assert alr.alr_device_supported() == alr.ALR_OK, alr.alr_last_error()


def _i(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _attend(Q, K, V, table, length, seq, per=1, **kw):
    N, H, dim = Q.shape
    ws = torch.empty(alr.alr_kv_attention_workspace_size(N, H, dim, "prefix_len" in kw), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(Q, 9.0), torch.full((N, H), 9.0, device="cuda")
    alr.alr_kv_attention(Q, K, V, table, length, out, ws, seq=seq, lse=lse, rows_per_seq=per, **kw)
    torch.cuda.synchronize()
    assert alr.alr_device_status(clear=True) == alr.ALR_OK, alr.alr_last_error()
    return out, lse


@pytest.mark.parametrize("dim", [64, 128])
def test_poison_at_the_end_of_long_sequences(dim):
    """Half of 64 sequences of a million tokens (pages used again and again) end with a value of NaN that the
    last row of each block alone reads: taking the other rows' 112 queries again over 400 thousand tokens of a
    thread block ends no wait, and no other item is touched."""
    S, per, group, page, cols, common = 64, 8, 16, 1024, 1024, 3
    g = torch.Generator(device="cuda").manual_seed(dim)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    K, V = rand(common + S, page, 1, dim).to(BF), (1 + 0.1 * rand(common + S, page, 1, dim)).to(BF)
    table = torch.arange(cols)[None].repeat(S, 1) % common
    table[:, -1] = common + torch.arange(S)
    lens = cols * page - per + 1 + torch.arange(per).repeat(S)
    seq = torch.arange(S).repeat_interleave(per)
    Q = rand(S * per, group, dim).to(BF)
    args = Q, K, V, _i(table), _i(lens), _i(seq)
    clean, clean_lse = _attend(*args, per=per)
    V[common::2, -1] = NAN
    out, lse = _attend(*args, per=per)
    hit = (seq % 2 == 0).cuda()
    last = torch.arange(S * per, device="cuda") % per == per - 1
    assert torch.equal(out[~hit], clean[~hit]) and torch.equal(lse[~hit], clean_lse[~hit])
    assert out[hit & last].isnan().all()
    # fp64, each page of the sequence as often as it is in it
    scale = dim ** -0.5
    V[common::2, -1] = 0                       # masked below
    times = torch.bincount(table[0, :-1], minlength=common).double().cuda()
    k = K[:common, :, 0].double().flatten(0, 1)
    x = scale * Q.double() @ k.T                                         # [N, group, tokens]
    own = scale * Q.double() @ K[common:, :, 0].double()[seq.cuda()].transpose(1, 2)
    own = own.masked_fill((torch.arange(page) >= (lens - (cols - 1) * page)[:, None]).cuda()[:, None], -INF)
    x = torch.cat([x + times.log().repeat_interleave(page), own], -1)
    w = torch.softmax(x, -1)
    n = common * page
    want = w[..., :n] @ V[:common, :, 0].double().flatten(0, 1) + w[..., n:] @ V[common:, :, 0].double()[seq.cuda()]
    # sums over a thread block's tokens (152 share them), products of bf16 weights, values of 1 +- 0.5
    reach = scale * (Q.double().abs().amax((0, 1)) * K.double().abs().amax((0, 1, 2))).sum().item()
    dx = 2 * (dim + 4) * U * reach
    rel = 2 * dx + 2.0 ** -21 + 2 * (S * cols * page / 152 + 400) * U
    some = ~(hit & last)
    for o, l in ((clean, clean_lse), (out, lse)):  # noqa: E741
        assert (o[some].double() - want[some]).abs().max().item() <= (rel + 2 * 2.0 ** -8) * 1.5
        assert (l[some].double() - torch.logsumexp(x, -1)[some]).abs().max().item() <= dx + rel + 4 * U * 32


@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("form", [dict(heads=3, group=1, dim=16), dict(heads=2, group=4, dim=64), dict(heads=2, group=12, dim=128),
                                  dict(heads=1, group=20, dim=64), dict(heads=1, group=20, dim=128),
                                  dict(heads=1, group=3, dim=256), dict(heads=1, group=16, dim=256)])
def test_values_of_tokens_masked_by_their_scores(form, dtype, bad):
    """A token whose score is -inf does not reach a row by its value either, be rows alone or in tiles, and in
    own tokens as in a prefix; a row of such tokens alone is empty."""
    n, per = 700, 5
    rows = [(s, n - per + 1 + j) for s in range(2) for j in range(per)]
    prefix = [(2 + s, 300 - j) for s in range(2) for j in range(per)]
    for pre in (None, prefix):
        c = Case([n, n, 300, 300], rows, prefix=pre, dtype=dtype, page=16, seed=4, **form)
        c.Q[..., 0] = 8.0
        t = np.arange(n)
        for s, these in ((0, t[::3]), (1, t), (2, t[5:300:7]), (3, t[:300])):
            pg, pos = c.table[s, these // 16], these % 16
            c.K[pg, pos, :, 0] = -INF
            c.V[pg, pos] = 0.0
        c.expected()                           # weights of 0, values of 0
        for s, these in ((0, t[::3]), (1, t), (2, t[5:300:7]), (3, t[:300])):
            c.V[c.table[s, these // 16], these % 16] = bad
        for p in (1, 2, per):
            out, lse = c.check(per=p, per_prefix=p)
        assert (lse[per:] == -INF).all() and not out[per:].any() and lse[:per].isfinite().all()
        # one of them with an ordinary score: its value arrives
        pg, pos = c.table[0, 0], 0
        c.K[pg, pos, :, 0] = 0.0
        for p in (1, 2, per):
            out, lse = c.run(per=p, per_prefix=p)
            assert not out[:per].isfinite().any() and lse[:per].isfinite().all() and not out[per:].any()


@pytest.mark.parametrize("T", [2 ** 31 - 1, 2 ** 31 - 31, 2 ** 31 - 32, 2 ** 31 - 4096, 2 ** 26 + 1])
def test_plan_of_the_largest_batches(T):
    """Batches of up to 2^31 - 1 rows: every row is written, with its slot if its sequence has a place."""
    a, page = T - 19, 16                       # refused: past the table
    length, table = _i([0, 1, 0]), _i([[-1] * 4, [3, -1, -1, -1], [-1] * 4])
    slot, n = torch.full((T,), 77, dtype=torch.int32, device="cuda"), _i([0] * 3)
    start, refused = _i([0] * 4), _i([0])
    alr.alr_kv_plan(length, _i([a, 7, 9]), _i([5, 6]), _i([0]), table, page,
                    dict(len=n, slot=slot, pool_used=_i([0]), start=start, n_refused=refused))
    assert n.tolist() == [0, 8, 9] and refused.tolist() == [1] and start.tolist() == [0, a, a + 7, a + 16]
    assert slot[a:].tolist() == [3 * page + 1 + i for i in range(7)] + [5 * page + i for i in range(9)] + [-1] * 3
    for part in slot[:a].split(1 << 28):
        assert bool((part == -1).all())
    del slot, part
    torch.cuda.empty_cache()


def test_heads_far_apart():
    """Heads 2^30 elements apart within a token's row: places of the last head's elements pass 31 bits."""
    page, heads, dim, group, far = 8, 3, 64, 4, 1 << 30
    g = torch.Generator(device="cuda").manual_seed(0)
    room = torch.empty(page * heads * far, dtype=BF, device="cuda")
    K, V = (room.as_strided((1, page, heads, dim), (page * heads * far, heads * far, far, 1), at) for at in (0, dim))
    near = [torch.randn(1, page, heads, dim, generator=g, device="cuda").to(BF) for _ in "KV"]
    K.copy_(near[0])
    V.copy_(near[1])
    Q = torch.randn(8, heads * group, dim, generator=g, device="cuda").to(BF)
    args = _i([[0] * 20] * 1), _i(np.arange(8) + 140), _i([0] * 8)
    for per in (8, 1):
        want, want_lse = _attend(Q, *near, *args, per=per)
        out, lse = _attend(Q, K, V, *args, per=per)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    row = torch.randn(1, heads, dim, generator=g, device="cuda").to(BF)
    alr.alr_kv_append(row, -row, K, V, _i([5]))
    assert torch.equal(K[0, 5], row[0]) and torch.equal(V[0, 5], -row[0])
    del room, K, V
    torch.cuda.empty_cache()


@pytest.mark.parametrize("form", [dict(heads=2, group=4, dim=64, page=16), dict(heads=1, group=8, dim=128, page=32),
                                  dict(heads=1, group=3, dim=80, page=20, hnd=True), dict(heads=2, group=1, dim=128, page=8),
                                  dict(heads=1, group=40, dim=128, page=16), dict(heads=1, group=4, dim=256, page=16),
                                  dict(heads=1, group=4, dim=64, page=16, dtype=F32)])
def test_prompts(form):
    """Hundreds of rows of each sequence, packed without gaps as a step's plan has them: many tiles of a sequence,
    tiles of several, rows of single tokens between; whatever the hint."""
    lengths, new = [700, 1, 33, 450, 64, 5], [650, 1, 33, 301, 1, 5]
    rows = [(s, n - k + 1 + j) for s, (n, k) in enumerate(zip(lengths, new)) for j in range(k)]
    c = Case(lengths, rows, seed=9, **form)
    for per in (1, 32, 650, 10 ** 6, 7):
        out, lse = c.check(per=per)
    # each sequence's rows begin a group of their own, the rows behind them empty
    c.rows = np.array([(s, lengths[s] - new[s] + 1 + j if j < new[s] else 0) for s in range(6) for j in range(650)])
    Q, at = torch.zeros(6 * 650, *c.Q.shape[1:], dtype=c.Q.dtype, device="cuda"), np.flatnonzero(c.rows[:, 1])
    Q[at] = c.Q
    c.Q = Q
    padded, padded_lse = c.run(per=650, seq=False)
    # values of up to 5, weights and output of bf16 each off by 2^-8 on either side, or fp32 sums of 700
    assert (padded[at].float() - out.float()).abs().max() <= 5 * (4 * 2.0 ** -8 if c.Q.dtype == BF else 1e-3)
    assert (padded_lse[at] - lse).abs().max() <= 1e-3
    empty = np.flatnonzero(c.rows[:, 1] == 0)
    assert not padded[empty].any() and (padded_lse[empty] == -INF).all()


@pytest.mark.parametrize("lengths,per,prefix,form", [
    ([3000, 0, 70, 1500], 1, 0, dict(heads=2, group=4, dim=128)), ([60, 1, 0, 17], 1, 0, dict(heads=2, group=4, dim=64)),
    ([3000, 0, 70, 1500], 1, 0, dict(heads=1, group=12, dim=64)), ([3000, 0, 70, 1500], 4, 0, dict(heads=2, group=4, dim=80, dtype=F32)),
    ([60, 1, 0, 17], 1, 0, dict(heads=1, group=1, dim=32, dtype=F32)),
    ([40000, 0, 70, 1500], 8, 0, dict(heads=4, group=8, dim=128)), ([40000, 0, 70, 1500], 8, 0, dict(heads=4, group=8, dim=64, page=20)),
    ([70, 300], 8, 0, dict(heads=2, group=4, dim=64)), ([9, 12, 5, 2], 1, 4, dict(heads=2, group=8, dim=128))])
def test_withheld_stage_times_out_and_context_survives(lengths, per, prefix, form):
    """The first stage of every warp's ring, or of a thread block's, is never filled: the waits give up after their
    limit, the kernels run to their end, the timeout is reported, and the next call is right."""
    rows = [(s, max(0, n - j)) for s, n in enumerate(lengths) for j in range(per)]
    pre = [(len(lengths), 900 - 50 * j) for j in range(len(rows))] if prefix else None
    c = Case(lengths + [900] * bool(prefix), rows, prefix=pre, **{"page": 16, **form})
    want, want_lse = c.check(per=per, per_prefix=max(prefix, 1))
    N, H, dim = c.Q.shape
    ws = torch.empty(alr.alr_kv_attention_workspace_size(N, H, dim, prefix > 0), dtype=torch.uint8, device="cuda")
    kw = dict(prefix_seq=_i([p[0] for p in pre]), prefix_len=_i([p[1] for p in pre]), rows_per_prefix=prefix) if prefix else {}
    args = c.Q, c.K, c.V, _i(c.table), _i(c.rows[:, 1]), torch.empty_like(c.Q), ws
    seq = _i(c.rows[:, 0])
    torch.cuda.synchronize()
    assert alr.alr_device_status(clear=True) == alr.ALR_OK
    alr.alr_debug_withhold_next_stage(True)
    t0 = time.monotonic()
    alr.alr_kv_attention(*args, seq=seq, rows_per_seq=per, **kw)
    rc = alr.alr_device_status(clear=True)
    waited = time.monotonic() - t0
    assert rc == alr.ALR_ERR_TIMEOUT, alr.alr_last_error()
    assert 1.0 < waited < 20.0
    out, lse = c.run(per=per, per_prefix=max(prefix, 1))
    assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("form", [dict(heads=2, group=1, dim=8), dict(heads=1, group=12, dim=72), dict(heads=1, group=20, dim=104),
                                  dict(heads=2, group=4, dim=128), dict(heads=2, group=3, dim=36, dtype=F32)])
def test_workspaces_aligned_to_16_bytes(form):
    """A workspace 16 bytes past a multiple of more, for items cut between workers, prefixes and queries taken
    again."""
    per = 4
    lengths = [5000, 3000, 2000]
    rows = [(s, n - per + 1 + j) for s, n in ((0, 5000), (1, 3000)) for j in range(per)]
    for pre in (None, [(2, 2000 - j // 2) for j in range(2 * per)]):
        c = Case(lengths, rows, prefix=pre, page=16, **form)
        for t, s in ((4999, 0), (1999, 2)):    # the last row of one sequence and some of the prefix read these
            c.V[c.table[s, t // 16], t % 16] = INF
        N, H, dim = c.Q.shape
        ws = torch.empty(alr.alr_kv_attention_workspace_size(N, H, dim, pre is not None) + 64, dtype=torch.uint8, device="cuda")
        assert ws.data_ptr() % 64 == 0
        want = c.run(per=per, per_prefix=2 * per, ws=ws)
        got = c.run(per=per, per_prefix=2 * per, ws=ws[16:])
        assert not want[0].isfinite().all() and want[0].isfinite().any()
        assert torch.equal(got[0].nan_to_num(7.0), want[0].nan_to_num(7.0)) and torch.equal(got[1], want[1])
