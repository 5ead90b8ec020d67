"""The operators around a rollout and a distillation step, as cases whose speed can be measured.

A case is a dict of plain values.  `prepare` makes what a program holds before the call (seeded
inputs and the output buffers), `run` makes one pass through one operator, in plain torch or, where
`own` is true, by the library's entry points, and `exact` computes the same outputs in fp64.

Kinds of case
  distill  the distillation loss of student logits against a teacher's top logits: the forward
           ("fwd"), the gradient from its results ("bwd"), or both in one call ("both");
  top      a teacher's top logits and its log-sum-exps, the labels that distillation reads;
  sample   one token for each row of logits: temperature, top-k, top-p, min-p, given random numbers;
  embed    the scaled lookup of a block's tokens ("fwd"), the gradient of the table ("bwd"), or the
           lookup and the gradient of one training step ("both").
"""

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LAM = 1.013441
NEG = float("-inf")


def _case(kind, **kw):
    base = {
        # pad: logits past V - pad are -inf (a vocabulary padded for the head); ld: row stride
        "distill": dict(N=256, V=4096, K=8, dtype="bf16", way="both", tail=True, T=1.0,
                        masked=False, pad=0, ld=0, sharp=True),
        "top": dict(N=64, V=4096, K=8, dtype="bf16", T=1.0, pad=0, ld=0, sharp=True),
        "sample": dict(N=64, V=4096, dtype="bf16", mode="k_p", pad=0, ld=0, sharp=True),
        "embed": dict(N=256, V=4096, d=512, dtype="bf16", way="both", mask=0.0),
    }[kind]
    return dict(base, kind=kind, **kw)


def listed():
    return [
        # one sample of 128 anchors x 16 slots at the 8B head: loss and gradient, the paper's top 8
        # and tail, slots past a rollout's end masked, a padded vocabulary
        _case("distill", name="distill_sample", N=2048, V=151936, masked=True, pad=293),
        # a longer list without the tail, softened labels, fp32 logits, loss alone (evaluation)
        _case("distill", name="distill_eval_f32", N=512, V=32000, K=64, dtype="f32", way="fwd",
              tail=False, T=2.0),
        # the gradient alone, from a forward's results: an odd vocabulary in rows of another stride
        _case("distill", name="distill_grad_ragged", N=2000, V=60001, K=20, way="bwd", T=1.5,
              ld=60016, masked=True),
        # the smallest training call: one anchor block
        _case("distill", name="distill_one_block", N=16, V=4096),
        # labels of one rollout step of 6 samples x 128 running rollouts
        _case("top", name="top_rollout_step", N=768, V=151936, K=64, pad=293),
        # labels of a few rows, fp32 logits of an odd vocabulary
        _case("top", name="top_few_f32", N=15, V=32001, K=20, dtype="f32", T=0.7),
        # the rollout step's next tokens: top-k and top-p
        _case("sample", name="sample_rollout_step", N=768, V=151936, pad=293),
        # nucleus sampling for a few running sequences: latency
        _case("sample", name="sample_few_p", N=4, V=152064, mode="p"),
        # every row with its own settings, greedy rows and truncations off among them
        _case("sample", name="sample_mixed_f32", N=512, V=32000, dtype="f32", mode="mixed",
              sharp=False),
        # the block inputs of a device batch: 2048 anchors x 16 slots, anchor token then mask tokens
        _case("embed", name="embed_blocks", N=32768, V=151936, d=4096, way="fwd", mask=0.9375),
        # the table's gradient for the same blocks of a 32000-token model
        _case("embed", name="embed_grad_blocks", N=32768, V=32000, d=2048, way="bwd", mask=0.9375),
        # the smallest training step: lookup and gradient of 12 anchors
        _case("embed", name="embed_smallest", N=192, V=1400, d=320),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["distill", "distill", "top", "sample", "sample", "embed"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "embed":
        V = _log_int(rng, 500, 151936)
        d = _log_int(rng, 64, 4096)
        way = rng.choice(["fwd", "bwd", "both"])
        d = d if rng.random() < 0.3 else max(8, d // 8 * 8)
        return _case("embed", N=_log_int(rng, 1, 32768), V=V, d=d, dtype=dtype, way=way,
                     mask=rng.choice([0.0, 0.5, 0.9375, 1.0]))
    V = _log_int(rng, 1000, 152064)
    most = {"distill": 2048, "top": 1024, "sample": 768}[kind]
    N = _log_int(rng, 1, most if dtype == "bf16" else most // 2)
    c = dict(N=N, V=V, dtype=dtype, pad=rng.choice([0, 0, V // 100]), sharp=rng.random() < 0.6,
             ld=V + rng.choice([0, 0, 5, 64]))
    if kind == "sample":
        return _case("sample", mode=rng.choice(["k_p", "p", "k", "min_p", "all", "mixed"]), **c)
    c.update(K=_log_int(rng, 1, 256), T=rng.choice([0.7, 1.0, 1.0, 2.0]))
    if kind == "top":
        return _case("top", **c)
    return _case("distill", way=rng.choice(["fwd", "bwd", "both", "both"]),
                 tail=rng.random() < 0.6, masked=rng.random() < 0.5, **c)


# ---------------------------------------------------------------------------- inputs ---
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _rows(c, values):
    """[N, V] view of rows `ld` apart in the case's element type, the padded tokens -inf."""
    N, V = values.shape
    buf = torch.zeros(N, c["ld"] or V, dtype=DTYPES[c["dtype"]], device="cuda")
    z = buf[:, :V]
    z.copy_(values)
    if c["pad"]:
        z[:, V - c["pad"]:] = NEG
    return z


def _logits(c, g):
    """fp32 logits: a trained head's (few tokens far above a wide bulk, |z| to about 30) or a random
    head's (one bulk, |z| below 7)."""
    N, V = c["N"], c["V"]
    if not c["sharp"]:
        return torch.randn(N, V, generator=g, device="cuda") * 1.3
    z = torch.randn(N, V, generator=g, device="cuda") * 2.5
    n = min(40, V)
    tok = torch.randint(0, V, (N, n), generator=g, device="cuda")
    lift = 24.0 - 3.0 * torch.arange(n, device="cuda", dtype=torch.float32).sqrt()
    lift = lift + torch.randn(N, n, generator=g, device="cuda")
    return z.scatter_reduce_(1, tok, lift, "amax")      # a token drawn twice takes the larger


def _distill_state(c, g):
    N, V, K, T = c["N"], c["V"], c["K"], c["T"]
    teacher = _rows(dict(c, ld=0), _logits(c, g)).float()
    student = teacher.masked_fill(teacher == NEG, 0.0)
    student += torch.randn(N, V, generator=g, device="cuda")
    k = min(K, V - c["pad"])
    val, idx = torch.topk(teacher, k, dim=1)
    top_val = torch.full((N, K), NEG, device="cuda")
    top_idx = torch.full((N, K), -1, dtype=torch.int32, device="cuda")
    top_val[:, :k], top_idx[:, :k] = val, idx.int()
    s = dict(Z=_rows(c, student), top_val=top_val, top_idx=top_idx, rest=None, weight=None)
    if c["tail"]:
        s["rest"] = torch.logsumexp(teacher.scatter(1, idx, NEG) / T, 1)
    if K > 2:                                   # some lists end early: a teacher that kept fewer
        short = torch.arange(N, device="cuda") % 7 == 3
        s["top_idx"][short, K - K // 3:] = -1
    if c["masked"]:
        slot = torch.arange(N, device="cuda") % 16
        end = torch.randint(4, 17, (N,), generator=g, device="cuda")[torch.arange(N, device="cuda")
                                                                     // 16 * 16]
        s["weight"] = torch.exp(-slot.float() / 2.0) * (slot < end)
    f = lambda *n: torch.empty(*n, device="cuda")  # noqa: E731
    s["out"] = dict(loss_row=f(N), ent_row=f(N), lse=f(N),
                    argmax=torch.empty(N, dtype=torch.int32, device="cuda"), loss_total=f(1),
                    weight_sum=f(1), wl_sum=f(1))
    if c["tail"]:
        s["out"]["lse_rest"] = f(N)
    if c["way"] != "fwd":
        s["G"] = torch.empty(N, V, dtype=DTYPES[c["dtype"]], device="cuda")
    if c["way"] == "bwd":                       # a forward's results, as the training step keeps them
        o = _plain_distill(dict(s, **dict(c, way="fwd")))
        s["lse"], s["lse_rest"] = o["lse"], o.get("lse_rest")
        s["weight_sum"] = o["weight_sum"]
    return s


def _top_state(c, g):
    N, K = c["N"], c["K"]
    return dict(Z=_rows(c, _logits(c, g)),
                out=dict(top_val=torch.empty(N, K, device="cuda"),
                         top_idx=torch.empty(N, K, dtype=torch.int32, device="cuda"),
                         lse=torch.empty(N, device="cuda"), lse_rest=torch.empty(N, device="cuda")))


def _sample_state(c, g):
    N, V, mode = c["N"], c["V"], c["mode"]
    z = _rows(c, _logits(c, g))
    if N > 2:                                   # a grammar allows few tokens here; nothing there
        z[N // 2, V // 50:] = NEG
        if mode == "mixed":
            z[N - 1] = NEG
    s = dict(Z=z, temperature=torch.full((N,), 0.8, device="cuda"), top_k=None, top_p=None,
             min_p=None)
    r = lambda: torch.rand(N, generator=g, device="cuda")  # noqa: E731
    if mode in ("k_p", "k"):
        s["top_k"] = torch.full((N,), 50, dtype=torch.int32, device="cuda")
    if mode in ("k_p", "p"):
        s["top_p"] = torch.full((N,), 0.95, device="cuda")
    if mode == "min_p":
        s["min_p"] = torch.full((N,), 0.05, device="cuda")
    if mode == "mixed":
        s["temperature"] = torch.where(r() < 0.2, 0.0, 0.3 + r())
        s["top_k"] = torch.where(r() < 0.4, 0, 1 + (r() * 200).int()).int()
        s["top_p"] = torch.where(r() < 0.4, 1.0, 0.2 + 0.8 * r())
        s["min_p"] = torch.where(r() < 0.6, 0.0, 0.2 * r())
    s["u"] = torch.randint(-(1 << 31), 1 << 31, (N,), generator=g, device="cuda",
                           dtype=torch.int64).to(torch.int32)      # the bits of uint32 draws
    s["out"] = dict(token=torch.empty(N, dtype=torch.int32, device="cuda"),
                    prob=torch.empty(N, device="cuda"),
                    n_kept=torch.empty(N, dtype=torch.int32, device="cuda"))
    return s


def _embed_state(c, g):
    N, V, d, dt = c["N"], c["V"], c["d"], DTYPES[c["dtype"]]
    tok = (V * torch.rand(N, generator=g, device="cuda") ** 4).int().clamp_(max=V - 1)
    tok = torch.where(torch.rand(N, generator=g, device="cuda") < c["mask"], V // 3, tok)
    tok[torch.rand(N, generator=g, device="cuda") < 0.01] = -1     # padding
    s = dict(tokens=tok.int(), scale=math.sqrt(d))
    if c["way"] != "bwd":
        s["E"] = (torch.randn(V, d, generator=g, device="cuda") * 0.02).to(dt)
        s["out"] = torch.empty(N, d, dtype=dt, device="cuda")
    if c["way"] != "fwd":
        s["dY"] = torch.randn(N, d, generator=g, device="cuda").to(dt)
        s["dE"] = torch.empty(V, d, device="cuda")
    return s


def prepare(case, seed):
    make = {"distill": _distill_state, "top": _top_state, "sample": _sample_state,
            "embed": _embed_state}[case["kind"]]
    return dict(make(case, _gen(seed)), **case)


# ----------------------------------------------------------------------- plain forms ---
def _plain_distill(s):
    z, T, way = s["Z"].float() / s["T"], s["T"], s["way"]
    N, V = z.shape
    w = torch.ones(N, device="cuda") if s["weight"] is None else s["weight"]
    live = w != 0
    idx = s["top_idx"].long()
    there = (idx >= 0) & (idx < V)
    a = torch.where(there, s["top_val"] / T, NEG)
    rest = torch.full((N,), NEG, device="cuda") if s["rest"] is None else s["rest"]
    a = torch.cat([a, rest[:, None]], 1)
    m = a.max(1, keepdim=True).values
    has = m[:, 0] > NEG
    e = torch.where(has[:, None], torch.exp(a - m), 0.0)
    p = e / e.sum(1, keepdim=True).clamp(min=1e-30)
    logp = torch.where(p > 0, a - m - torch.log(e.sum(1, keepdim=True).clamp(min=1e-30)), 0.0)
    # the list's student logits, and the row without them
    at = torch.where(there, idx, V)
    zx = torch.cat([z, torch.full((N, 1), NEG, device="cuda")], 1)
    zi = zx.gather(1, at)
    out = zx.scatter(1, at, NEG)[:, :V]
    if way != "bwd":
        mz = z.max(1, keepdim=True).values
        S = torch.exp(z - mz).sum(1)
        So = torch.exp(out - mz).sum(1)
        u = torch.cat([mz - zi, -torch.log(So)[:, None]], 1)       # max - s_i, max - R
        terms = torch.where(p > 0, p * (torch.log(S)[:, None] + u), 0.0)
        o = dict(loss_row=torch.where(live & has, terms.sum(1), 0.0),
                 ent_row=torch.where(live & has, -(p * logp).sum(1), 0.0),
                 lse=torch.where(live, mz[:, 0] + torch.log(S), 0.0),
                 argmax=torch.where(live, z.argmax(1), -1).int(),
                 weight_sum=w.sum()[None])
        o["wl_sum"] = (w * o["loss_row"]).sum()[None]
        o["loss_total"] = torch.where(o["weight_sum"] > 0, LAM * o["wl_sum"] / o["weight_sum"], 0.0)
        lse, lse_rest = o["lse"], torch.where(live, mz[:, 0] + torch.log(So), 0.0)
        if s["rest"] is not None:
            o["lse_rest"] = lse_rest
        if way == "fwd":
            return o
        ws = o["weight_sum"]
    else:
        o, lse, ws = {}, s["lse"], s["weight_sum"]
        lse_rest = s["lse_rest"]
    coef = torch.where(live & has & (ws > 0), LAM * w / (ws * T), 0.0)[:, None]
    q = torch.exp(z - lse[:, None])
    if s["rest"] is not None:
        r = torch.where(lse_rest > NEG, lse_rest, 0.0)[:, None]
        q = q - p[:, -1:] * torch.exp(out - r)
    q = torch.cat([q, torch.zeros(N, 1, device="cuda")], 1)
    q = q.scatter_add(1, at, -p[:, :-1])[:, :V]
    o["G"] = torch.where(coef != 0, coef * q, 0.0).to(s["Z"].dtype)
    return o


def _plain_top(s):
    z = s["Z"].float()
    N, V = z.shape
    K = s["K"]
    val, idx = torch.sort(z, dim=1, descending=True, stable=True)
    val, idx = val[:, :K], idx[:, :K]
    if K > V:
        val = torch.cat([val, torch.full((N, K - V), NEG, device="cuda")], 1)
        idx = torch.cat([idx, torch.zeros(N, K - V, dtype=idx.dtype, device="cuda")], 1)
    idx = torch.where(val > NEG, idx, V)
    x = z / s["T"]
    m = x.max(1, keepdim=True).values
    S = torch.exp(x - m).sum(1)
    So = torch.exp(torch.cat([x, m], 1).scatter(1, idx, NEG)[:, :V] - m).sum(1)
    return dict(top_val=val, top_idx=torch.where(idx < V, idx, -1).int(), lse=m[:, 0] + torch.log(S),
                lse_rest=m[:, 0] + torch.log(So))


def _plain_sample(s):
    z = s["Z"].float()
    N, V = z.shape
    m = z.max(1, keepdim=True).values
    some = m[:, 0] > NEG
    T = s["temperature"]
    greedy = T <= 0
    c = (torch.full((N,), 1.4426950408889634, device="cuda")
         / torch.where(greedy, 1.0, T))[:, None]
    w = torch.exp2((z - m) * c)
    w = torch.where((z > NEG) & some[:, None], w, 0.0)
    # integer weights: their sums are exact, so the draw depends on no order of summation
    a = (w * 2147483648.0).to(torch.int64)
    _, order = torch.sort(z, dim=1, descending=True, stable=True)
    ws, as_ = w.gather(1, order), a.gather(1, order)
    keep = as_ > 0
    rank = torch.arange(V, device="cuda")[None, :]
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], V)
        keep &= rank < k[:, None]
    if s["top_p"] is not None:
        kept = as_ * keep
        before = kept.cumsum(1) - kept
        lim = s["top_p"].double() * kept.sum(1).double()
        keep &= (before.double() < lim[:, None]) | (rank == 0) | (s["top_p"] >= 1)[:, None]
    if s["min_p"] is not None:
        keep &= (ws >= s["min_p"][:, None]) | (rank == 0)
    keep &= (rank == 0) | ~greedy[:, None]
    n_kept = keep.sum(1)
    a = a * torch.zeros_like(keep).scatter_(1, order, keep)
    cum = a.cumsum(1)
    S = cum[:, -1]
    u = s["u"].long() & 0xffffffff
    # floor(u S / 2^32) in 64 bits, S in pieces of 16 bits
    hi, mid, lo = S >> 32, (S >> 16) & 0xffff, S & 0xffff
    R = u * hi + ((u * mid + ((u * lo) >> 16)) >> 16)
    token = (cum <= R[:, None]).sum(1)
    got = a.gather(1, token.clamp(max=V - 1)[:, None])[:, 0]
    return dict(token=torch.where(some, token, -1).int(),
                prob=(got.double() / S.clamp(min=1).double()).float(), n_kept=n_kept.int())


def _plain_embed(s):
    tok, o = s["tokens"].long(), {}
    V = (s["E"] if "E" in s else s["dE"]).shape[0]
    ok = (tok >= 0) & (tok < V)
    t = torch.where(ok, tok, 0)
    if s["way"] != "bwd":
        o["out"] = torch.where(ok[:, None], s["E"][t].float() * s["scale"], 0.0).to(s["E"].dtype)
    if s["way"] != "fwd":
        dy = torch.where(ok[:, None], s["dY"].float(), 0.0)
        o["dE"] = torch.zeros(V, dy.shape[1], device="cuda").index_add_(0, t, dy) * s["scale"]
    return o


# ------------------------------------------------------------------- the library's calls ---
def _own(s):
    from paper_2609_38795_gb300 import alr
    if s["kind"] == "distill":
        kw = dict(rest=s["rest"], weight=s["weight"], temperature=s["T"], lam=LAM)
        lists = (s["Z"], s["top_val"], s["top_idx"])
        if s["way"] == "fwd":
            alr.alr_distill_fwd(*lists, s["out"], **kw)
            return s["out"]
        if s["way"] == "bwd":
            alr.alr_distill_bwd(*lists, s["lse"], s["lse_rest"], s["weight_sum"], s["G"], **kw)
            return dict(G=s["G"])
        alr.alr_distill_fwd_bwd(*lists, s["out"], s["G"], **kw)
        return dict(s["out"], G=s["G"])
    if s["kind"] == "top":
        alr.alr_top_logits(s["Z"], s["K"], s["out"], temperature=s["T"])
        return s["out"]
    if s["kind"] == "sample":
        alr.alr_sample_tokens(s["Z"], s["u"], s["out"], temperature=s["temperature"],
                              top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return s["out"]
    o = {}
    if s["way"] != "bwd":
        alr.alr_embed(s["E"], s["tokens"], s["out"], scale=s["scale"])
        o["out"] = s["out"]
    if s["way"] != "fwd":
        if "ws" not in s:
            n = alr.alr_embed_grad_workspace_size(*s["dE"].shape, s["tokens"].numel())
            s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
        alr.alr_embed_grad(s["dY"], s["tokens"], s["dE"], s["ws"], scale=s["scale"])
        o["dE"] = s["dE"]
    return o


def run(state):
    if own:
        return _own(state)
    return {"distill": _plain_distill, "top": _plain_top, "sample": _plain_sample,
            "embed": _plain_embed}[state["kind"]](state)


# ------------------------------------------------------------------------------ work ---
def work(case):
    N, V = case["N"], case["V"]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "embed":
        d, b, f = case["d"], 4 * N, 0
        if case["way"] != "bwd":
            distinct = min(V, math.ceil(N * (1 - case["mask"])) + 1)     # rows of the table
            b += distinct * d * e + N * d * e
            f += N * d
        if case["way"] != "fwd":
            b += N * d * e + V * d * 4
            f += N * d
        return {"bytes": b, "flops": f}
    if case["kind"] == "sample":
        return {"bytes": N * V * e + 32 * N, "flops": 4 * N * V}
    if case["kind"] == "top":
        return {"bytes": N * V * e + N * (8 * case["K"] + 8), "flops": 4 * N * V}
    live = 0.6 if case["masked"] else 1.0       # rows past a rollout's end are not read
    read = N * live * (V * e + 8 * case["K"])
    return {"bytes": read + 32 * N + (0 if case["way"] == "fwd" else N * V * e),
            "flops": (8 if case["way"] == "both" else 4) * live * N * V}


# ------------------------------------------------------------------ the definitions, fp64 ---
def _exact_distill(s):
    """Row by row over the list's tokens with the full softmax beside it, in fp64."""
    T, way = s["T"], s["way"]
    x = s["Z"].double().div_(T)
    N, V = x.shape
    w = torch.ones(N, device="cuda", dtype=torch.float64) if s["weight"] is None \
        else s["weight"].double()
    listed_ = torch.zeros(N, V + 1, dtype=torch.bool, device="cuda")
    at = s["top_idx"].long()
    at = torch.where(at < 0, V, at)
    listed_.scatter_(1, at, True)
    listed_ = listed_[:, :V]
    p = torch.zeros(N, V + 1, dtype=torch.float64, device="cuda")
    p.scatter_(1, at, torch.exp(s["top_val"].double() / T))
    p[:, V] = 0 if s["rest"] is None else torch.exp(s["rest"].double())
    mass = p.sum(1, keepdim=True)
    p = p / mass
    lse = torch.logsumexp(x, 1)
    lse_rest = torch.logsumexp(x.masked_fill(listed_, NEG), 1)
    o = {}
    if way != "bwd":
        ce = torch.where(p[:, :V] > 0, p[:, :V] * (lse[:, None] - x), 0.0).sum(1)
        ce += torch.where(p[:, V] > 0, p[:, V] * (lse - lse_rest), 0.0)
        on = w != 0
        o = dict(loss_row=torch.where(on, ce, 0.0),
                 ent_row=torch.where(on, torch.special.entr(p).sum(1), 0.0),
                 lse=torch.where(on, lse, 0.0), argmax=None, weight_sum=w.sum()[None])
        o["wl_sum"] = (w * o["loss_row"]).sum()[None]
        o["loss_total"] = LAM * o["wl_sum"] / o["weight_sum"]
        if s["rest"] is not None:
            o["lse_rest"] = torch.where(on, lse_rest, 0.0)
    if way != "fwd":
        g = torch.exp(x - lse[:, None]) - p[:, :V]
        if s["rest"] is not None:
            g -= p[:, V:] * torch.exp(x - lse_rest[:, None]).masked_fill_(listed_, 0.0)
        o["G"] = g * (LAM / T * w / w.sum())[:, None]
    return o


def _exact_top(s):
    z = s["Z"].double()
    N, V = z.shape
    k = min(s["K"], V)
    val = torch.full((N, s["K"]), NEG, dtype=torch.float64, device="cuda")
    val[:, :k] = torch.topk(z, k, dim=1).values
    keep = torch.sort(z / s["T"], dim=1, descending=True).values
    n = torch.clamp((val > NEG).sum(1), max=V)
    lse = torch.logsumexp(keep, 1)
    keep = keep.masked_fill(torch.arange(V, device="cuda")[None, :] < n[:, None], NEG)
    return dict(top_val=val, top_idx=None, lse=lse, lse_rest=torch.logsumexp(keep, 1))


def _exact_sample(s):
    """The probabilities of the drawn tokens.  A token's weight is defined as a whole number (a 32-bit
    exp2 times 2^31, rounded down); fp64 holds every sum of them exactly."""
    z = s["Z"].float()
    N, V = z.shape
    top = z.amax(1, keepdim=True)
    some = top[:, 0] > NEG
    T = s["temperature"]
    scale = torch.where(T > 0, torch.tensor(1.4426950408889634, device="cuda") / T, 0.0)
    x = torch.where(some[:, None], z - top, NEG) * torch.where(T > 0, scale, 1.0)[:, None]
    w32 = torch.exp2(x)
    wt = torch.floor(w32.double() * 2.0 ** 31)
    order = torch.argsort(-z, dim=1, stable=True)
    srt = wt.gather(1, order)
    place = torch.arange(V, device="cuda")[None, :]
    n = (srt > 0).sum(1)
    if s["top_k"] is not None:
        n = torch.where(s["top_k"] > 0, torch.minimum(n, s["top_k"].long()), n)
    if s["top_p"] is not None:
        run_ = torch.where(place < n[:, None], srt, 0.0).cumsum(1)
        need = 1 + (run_ < (s["top_p"].double() * run_[:, -1])[:, None]).sum(1)
        n = torch.where(s["top_p"] < 1, torch.minimum(n, need), n)
    if s["min_p"] is not None:
        n = torch.minimum(n, (w32 >= s["min_p"][:, None]).sum(1))
    n = torch.where(T > 0, n.clamp(min=1), 1)
    kept = torch.zeros_like(srt).scatter_(1, order, torch.where(place < n[:, None], srt, 0.0))
    run_ = kept.cumsum(1)
    total = run_[:, -1]
    u = (s["u"].long() & 0xffffffff).double()
    # floor(u total / 2^32) from fp64 may be one off where it lies at a token's end: rare, and such a
    # row's token is its neighbour
    R = torch.floor(u * (total / 2.0 ** 32))
    token = (run_ <= R[:, None]).sum(1).clamp(max=V - 1)
    prob = kept.gather(1, token[:, None])[:, 0] / total
    return dict(token=None, prob=torch.where(some, prob, 0.0), n_kept=None)


def _exact_embed(s):
    tok, o = s["tokens"].long(), {}
    V = (s["E"] if "E" in s else s["dE"]).shape[0]
    if s["way"] != "bwd":
        table = torch.cat([s["E"].double(), torch.zeros(1, s["d"], dtype=torch.float64,
                                                        device="cuda")])
        o["out"] = table[torch.where(tok < 0, V, tok)] * s["scale"]
    if s["way"] != "fwd":
        # rows sorted by token; a token's sum is the difference of the running sum at its ends
        t, order = torch.sort(torch.where(tok < 0, V, tok), stable=True)
        run_ = torch.cat([torch.zeros(1, s["d"], dtype=torch.float64, device="cuda"),
                          s["dY"][order].double().cumsum(0)])
        ends = torch.searchsorted(t, torch.arange(V + 1, device="cuda"))
        o["dE"] = (run_[ends[1:]] - run_[ends[:-1]]) * s["scale"]
    return o


def exact(case, seed):
    return {"distill": _exact_distill, "top": _exact_top, "sample": _exact_sample,
            "embed": _exact_embed}[case["kind"]](prepare(case, seed))
