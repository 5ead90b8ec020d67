"""The rollout's key-value cache, as cases whose speed can be measured.

A case is a dict of plain values.  `prepare` makes what a program holds before the call (seeded
inputs, the cache, the output buffers), `run` makes one pass through one operator, in plain torch or,
where `own` is true, by the library's entry points, and `exact` computes the same outputs in fp64.

Kinds of case
  plan    block tables and slot maps of the next step, from the sequences' lengths: pages taken from
          a pool for the tokens to come, pages of ended sequences returned to it;
  append  the new tokens' keys and values written to their slots of the paged cache;
  attend  attention of query rows over the paged cache: one new token for each sequence ("decode"),
          a block of tokens for each ("block"), or rollouts that share a sample's prefix ("prefix").
"""

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NEG = float("-inf")


def _case(kind, **kw):
    base = {
        # S sequences of `lo` to `hi` tokens (evenly, or by their logarithm); each asks for up to
        # `most` tokens; every `end`-th has ended; `spare`: pages of the pool for each new page
        "plan": dict(S=64, lo=1, hi=1024, log=False, most=1, page=16, end=10, spare=1.2),
        # T tokens, one in ten without a slot; src: type of the new rows, ld: elements between them
        "append": dict(T=256, heads=8, dim=128, page=16, dtype="bf16", src="bf16", ld=0, hnd=False),
        # S sequences of `lo` to `hi` tokens, `per` query rows each; with `prefix` > 0 every `share`
        # rows read one of the prefixes too, each row up to an anchor of its own in [1, prefix]
        "attend": dict(S=16, lo=0, hi=1024, log=False, per=1, heads=8, group=4, dim=128, page=16,
                       dtype="bf16", hnd=False, prefix=0, share=0),
    }[kind]
    return dict(base, kind=kind, **kw)


def listed():
    return [
        # one step of 6 samples x 128 rollouts: a token each, some rollouts at their end
        _case("plan", name="plan_rollout_step", S=768, hi=2048),
        # 96 prompts of up to 8192 tokens enter the cache at once
        _case("plan", name="plan_prompts", S=96, lo=0, hi=1, most=8192, page=32, end=0),
        # the new keys and values of that rollout step, fp32 rows out of one fused projection
        _case("append", name="append_rollout_step", T=768, src="f32", ld=6144),
        # the keys and values of a prompt batch, into a cache laid out by heads
        _case("append", name="append_prompts", T=32768, heads=4, page=64, hnd=True),
        # one step of 6 samples x 128 rollouts over their shared corpus prefixes and own 14 tokens
        _case("attend", name="attend_rollout_prefix", S=768, lo=1, hi=14, prefix=2032, share=128),
        # one token for each of 256 running sequences
        _case("attend", name="attend_decode_many", S=256, hi=8192),
        # lengths from none to 32768, 28 query heads on 4, a cache by heads, pages no power of two
        _case("attend", name="attend_decode_ragged", S=64, lo=0, hi=32768, log=True, heads=4,
              group=7, page=48, hnd=True),
        # one long sequence: latency
        _case("attend", name="attend_one_long", S=1, lo=131071, hi=131071, page=64),
        # verification: 16 drafted tokens for each of 128 sequences, some blocks cut short
        _case("attend", name="attend_verify_blocks", S=128, lo=1024, hi=3000, per=16, page=32),
        # fp32, a head for every query head, an odd head size and page
        _case("attend", name="attend_f32_heads", S=48, lo=1, hi=4001, heads=16, group=1, dim=80,
              page=20, dtype="f32"),
        # fp32 of a small model
        _case("attend", name="attend_f32_small", S=64, lo=0, hi=500, heads=2, dim=32, page=8,
              dtype="f32"),
        # the smallest step: 12 sequences of a few tokens
        _case("attend", name="attend_smallest", S=12, lo=1, hi=60, heads=5, group=1, dim=64),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "attend"])
    page = rng.choice([8, 16, 16, 20, 32, 48, 64, 128])
    if kind == "plan":
        S = _log_int(rng, 1, 2048)
        prompts = rng.random() < 0.4
        hi = _log_int(rng, 2, 8192)
        return _case("plan", S=S, lo=0 if prompts else 1, hi=1 if prompts else hi, page=page,
                     most=max(1, min(hi, 400000 // S)) if prompts else rng.choice([1, 1, 16]),
                     end=rng.choice([0, 3, 10]), spare=rng.choice([0.7, 1.2]))
    dtype = rng.choice(["bf16", "bf16", "f32"])
    dim = rng.choice([16, 32, 64, 80, 112, 128, 128, 256])
    heads = rng.choice([1, 2, 4, 5, 8, 8, 16])
    hnd = rng.random() < 0.4
    if kind == "append":
        src = dtype if rng.random() < 0.5 else "f32"
        return _case("append", T=_log_int(rng, 1, 32768 * 1024 // max(1024, heads * dim)), heads=heads,
                     dim=dim, page=page, dtype=dtype, src=src, hnd=hnd,
                     ld=heads * dim + rng.choice([0, 0, 64, 200]))
    group = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    c = dict(heads=heads, group=group, dim=dim, page=page, dtype=dtype, hnd=hnd)
    token = heads * dim * 2 * (2 if dtype == "bf16" else 4)          # bytes of a token's cache
    form = rng.choice(["decode", "decode", "block", "prefix"])
    if form == "prefix":
        share = _log_int(rng, 2, 128)
        n = max(1, min(6, 16384 // (heads * group * share)))
        return _case("attend", S=n * share, lo=1, hi=rng.choice([1, 14, 40]),
                     prefix=_log_int(rng, 16, 4096), share=share, **c)
    S = _log_int(rng, 1, 256)
    per = rng.choice([2, 5, 8, 16]) if form == "block" else 1
    tokens = 3.0e9 / token / S if per == 1 else min(3.0e9 / token, 2.0e8 / (heads * group * per)) / S
    hi = _log_int(rng, 16, max(17, min(65536, int(tokens))))
    return _case("attend", S=S, lo=0 if rng.random() < 0.6 else hi // 2, hi=hi, per=per,
                 log=rng.random() < 0.4, **c)


# ---------------------------------------------------------------------------- inputs ---
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _spread(n, lo, hi, log):
    """n whole numbers from lo to hi, evenly or by their logarithm: the same for every seed."""
    if n == 1:
        return [hi]
    if log:
        return [lo + round(math.exp(math.log1p(hi - lo) * i / (n - 1))) - 1 for i in range(n)]
    return [lo + round((hi - lo) * i / (n - 1)) for i in range(n)]


def _shuffled(values, g, dtype=torch.int32):
    t = torch.tensor(values, dtype=dtype, device="cuda")
    return t[torch.randperm(len(values), generator=g, device="cuda")]


def _pages(tokens, page):
    return (tokens + page - 1) // page


def _plan_state(c, g):
    S, page, most = c["S"], c["page"], c["most"]
    length = _shuffled(_spread(S, c["lo"], c["hi"], c["log"]), g)
    add = torch.full((S,), 1, dtype=torch.int32, device="cuda") if most == 1 else \
        _shuffled(_spread(S, 1, most, False), g)
    who = torch.arange(S, device="cuda")
    add = torch.where(who % 20 == 7, 0, add)                         # a slot of the batch left idle
    if c["end"]:
        add = torch.where(who % c["end"] == 1, -1, add)
    add = add.int()
    cols = _pages(c["hi"] + most, page)
    held = _pages(length, page)
    used = int(held.sum())
    tokens = sum(_spread(S, 1, most, False)) if most > 1 else S
    n_pool = used + max(1, int(c["spare"] * (tokens // page + (S // 4 if most > 1 else 0))))
    pool = torch.randperm(n_pool, generator=g, device="cuda").int()
    table = torch.full((S, cols), -1, dtype=torch.int32, device="cuda")
    col = torch.arange(cols, device="cuda")[None, :]
    first = held.cumsum(0) - held
    table = torch.where(col < held[:, None],
                        pool[(first[:, None] + col).clamp(max=n_pool - 1)], table).contiguous()
    T = -(-tokens // 64) * 64                                        # the batch's rows, padded
    e = lambda *n: torch.empty(*n, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(len=length, add=add, pool=pool, table=table, T=T,
                pool_used=torch.tensor([used], dtype=torch.int32, device="cuda"),
                out=dict(len=e(S), slot=e(T), pool_used=e(1), start=e(S + 1), tok_seq=e(T),
                         tok_len=e(T), n_refused=e(1)))


def _cache(c, n_pages, g):
    """(K, V), views [n_pages, page, heads, dim] of a cache laid out by tokens or by heads."""
    shape = (n_pages, c["heads"], c["page"], c["dim"]) if c["hnd"] else \
        (n_pages, c["page"], c["heads"], c["dim"])
    kv = [torch.randn(*shape, generator=g, device="cuda", dtype=DTYPES[c["dtype"]]) for _ in "KV"]
    return [t.transpose(1, 2) if c["hnd"] else t for t in kv]


def _append_state(c, g):
    T, heads, dim = c["T"], c["heads"], c["dim"]
    n_pages = _pages(T + T // 4, c["page"]) + 1
    K, V = _cache(c, n_pages, g)
    ld = max(c["ld"], heads * dim)
    new = [torch.randn(T, ld, generator=g, device="cuda").to(DTYPES[c["src"]])
           [:, ld - heads * dim:].unflatten(1, (heads, dim)) for _ in "KV"]
    slot = torch.randperm(n_pages * c["page"], generator=g, device="cuda")[:T].int()
    slot[torch.rand(T, generator=g, device="cuda") < 0.1] = -1
    return dict(K=K, V=V, K_new=new[0], V_new=new[1], slot=slot)


def _tables(c, longest, g):
    """Tables for sequences of the given lengths, their pages all over the cache, and the cache."""
    held = [_pages(n, c["page"]) for n in longest]
    n_pages = max(1, sum(held))
    pages = torch.randperm(n_pages, generator=g, device="cuda").int()
    h = torch.tensor(held, device="cuda")
    col = torch.arange(max(1, max(held)), device="cuda")[None, :]
    at = ((h.cumsum(0) - h)[:, None] + col).clamp(max=n_pages - 1)
    table = torch.where(col < h[:, None], pages[at], -1).int().contiguous()
    return table, _cache(c, n_pages, g)


def _attend_state(c, g):
    S, per, H = c["S"], c["per"], c["heads"] * c["group"]
    N = S * per
    length = _spread(S, c["lo"], c["hi"], c["log"])
    length = [length[i] for i in torch.randperm(S, generator=g, device="cuda").tolist()]
    s = dict(seq=None, prefix_seq=None, prefix_len=None)
    who = torch.arange(N, device="cuda")
    n = torch.tensor(length, device="cuda")[who // per]
    if per > 1:                     # row j reads the tokens before the block and its own up to j
        j = who % per
        cut = 1 + (torch.arange(S, device="cuda") * 7 % (4 * per)).clamp(max=per - 1)[who // per]
        n = torch.where(j < cut, (n - per + 1 + j).clamp(min=0), 0)   # no rows past a block's end
        s["seq"] = (who // per).int()
    s["len"] = n.int()
    if c["prefix"]:
        sp = -(-S // c["share"])
        length = length + [c["prefix"]] * sp
        s["prefix_seq"] = (S + who // c["share"]).int()
        s["prefix_len"] = _shuffled(_spread(N, 1, c["prefix"], False), g)
    s["table"], (s["K"], s["V"]) = _tables(c, length, g)
    dt = DTYPES[c["dtype"]]
    s["Q"] = (2.0 * torch.randn(N, H, c["dim"], generator=g, device="cuda")).to(dt)
    s["out"] = torch.empty(N, H, c["dim"], dtype=dt, device="cuda")
    s["lse"] = torch.empty(N, H, device="cuda")
    return s


def prepare(case, seed):
    make = {"plan": _plan_state, "append": _append_state, "attend": _attend_state}[case["kind"]]
    return dict(case, **make(case, _gen(seed)))


# ----------------------------------------------------------------------- plain forms ---
def _plain_plan(s):
    length, add, page, T = s["len"].long(), s["add"].long(), s["page"], s["T"]
    table, pool = s["table"].long(), s["pool"].long()
    (S, cols), n_pool = table.shape, pool.numel()
    used = s["pool_used"].long()
    ended = add < 0
    tokens = add.clamp(min=0)
    end = tokens.cumsum(0)
    start = end - tokens
    held = _pages(length, page)
    asks = ~ended & (length + tokens <= cols * page) & (end <= T)
    need = torch.where(asks, _pages(length + tokens, page) - held, 0)
    back = torch.where(ended, held, 0)
    n_back = back.sum()
    ok = asks & ((need == 0) | (need.cumsum(0) <= n_pool - used + n_back))
    # returned pages go below the used ones' end, in order; pages are taken from there on
    col = torch.arange(cols, device="cuda")[None, :]
    base = used - n_back
    at = torch.where(col < back[:, None], base + (back.cumsum(0) - back)[:, None] + col, n_pool)
    ext = torch.cat([pool, pool.new_zeros(1)]).scatter(0, at.reshape(-1), table.reshape(-1))
    pool = ext[:n_pool]
    taken = torch.where(ok, need, 0)
    k = (need.cumsum(0) - need)[:, None] + col - held[:, None]
    fresh = ok[:, None] & (col >= held[:, None]) & (col < (held + taken)[:, None])
    table = torch.where(fresh, ext[(base + k).clamp(min=0, max=n_pool)], table)
    t = torch.arange(T, device="cuda")
    q = torch.searchsorted(end, t, right=True).clamp(max=S - 1)
    pos = length[q] + t - start[q]
    live = (t < end[-1]) & ok[q]
    slot = table[q, (pos // page).clamp(0, cols - 1)] * page + pos % page
    i = lambda x: x.int()  # noqa: E731
    return dict(table=i(table), pool=i(pool),
                len=i(torch.where(ended, 0, torch.where(ok, length + tokens, length))),
                slot=i(torch.where(live, slot, -1)), pool_used=i(base + taken.sum()),
                start=i(torch.cat([start, end[-1:]])), tok_seq=i(torch.where(live, q, -1)),
                tok_len=i(torch.where(live, pos + 1, 0)), n_refused=i((~ended & ~ok).sum()[None]))


def _plain_append(s):
    slot = s["slot"].long()
    there = slot >= 0
    at = slot[there]
    for cache, new in ((s["K"], s["K_new"]), (s["V"], s["V_new"])):
        cache[at // s["page"], at % s["page"]] = new[there].to(cache.dtype)
    return dict(K=s["K"], V=s["V"])


def _read(cache, table, tokens):
    """[sequences, heads, tokens, dim] in fp32, through the table."""
    t = torch.arange(tokens, device="cuda")
    page = cache.shape[1]
    return cache[table[:, t // page].long().clamp(min=0), t % page].float().transpose(1, 2)


def _part(q, K, V, table, n):
    """Scores [rows, H, tokens] of one part, and its values; rows come in equal groups, one for
    each sequence of the table."""
    S, (N, H, D) = table.shape[0], q.shape
    heads, cols = K.shape[2], table.shape[1] * K.shape[1]
    tokens = min(cols, int(n.max()))
    k, v = _read(K, table, tokens), _read(V, table, tokens)
    qs = q.view(S, N // S, heads, H // heads, D).transpose(1, 2).reshape(S, heads, -1, D)
    x = (qs @ k.transpose(2, 3)).view(S, heads, N // S, H // heads, tokens)
    x = x.transpose(1, 2).reshape(N, H, tokens)
    beyond = torch.arange(tokens, device="cuda")[None, None, :] >= n[:, None, None]
    return x.masked_fill(beyond, NEG), v


def _weigh(p, v):
    S, heads, tokens, D = v.shape
    N, H, _ = p.shape
    ps = p.view(S, N // S, heads, H // heads, tokens).transpose(1, 2).reshape(S, heads, -1, tokens)
    o = (ps @ v).view(S, heads, N // S, H // heads, D)
    return o.transpose(1, 2).reshape(N, H, D)


def _plain_attend(s):
    q = s["Q"].float() * (1.0 / math.sqrt(s["dim"]))
    S = s["S"]
    parts = [_part(q, s["K"], s["V"], s["table"][:S], s["len"])]
    if s["prefix_len"] is not None:
        parts.append(_part(q, s["K"], s["V"], s["table"][S:], s["prefix_len"]))
    x = torch.cat([p[0] for p in parts], 2)
    if x.shape[2] == 0:
        return dict(out=torch.zeros_like(s["Q"]), lse=torch.full(x.shape[:2], NEG, device="cuda"))
    m = x.amax(2, keepdim=True)
    e = torch.exp(x - torch.where(m > NEG, m, 0.0))
    total = e.sum(2, keepdim=True)
    o = sum(_weigh(w, p[1]) for w, p in zip(e.split([p[0].shape[2] for p in parts], 2), parts))
    return dict(out=torch.where(total > 0, o / total.clamp(min=1e-30), 0.0).to(s["Q"].dtype),
                lse=(m + torch.log(total))[:, :, 0])


# ------------------------------------------------------------------- the library's calls ---
def _own(s):
    from paper_2609_38795_gb300 import alr
    if s["kind"] == "plan":
        alr.alr_kv_plan(s["len"], s["add"], s["pool"], s["pool_used"], s["table"], s["page"],
                        s["out"])
        return dict(s["out"], table=s["table"], pool=s["pool"])
    if s["kind"] == "append":
        alr.alr_kv_append(s["K_new"], s["V_new"], s["K"], s["V"], s["slot"])
        return dict(K=s["K"], V=s["V"])
    if "ws" not in s:
        n = alr.alr_kv_attention_workspace_size(*s["Q"].shape, prefix=s["prefix_len"] is not None)
        s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    alr.alr_kv_attention(s["Q"], s["K"], s["V"], s["table"], s["len"], s["out"], s["ws"],
                         seq=s["seq"], prefix_seq=s["prefix_seq"], prefix_len=s["prefix_len"],
                         lse=s["lse"], rows_per_seq=s["per"], rows_per_prefix=max(1, s["share"]))
    return dict(out=s["out"], lse=s["lse"])


def run(state):
    if own:
        return _own(state)
    return {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend}[state["kind"]](state)


# ------------------------------------------------------------------------------ work ---
def work(case):
    c = case
    if c["kind"] == "plan":
        add = _spread(c["S"], 1, c["most"], False) if c["most"] > 1 else [1] * c["S"]
        tokens = sum(add) * (1 - 1 / c["end"] if c["end"] else 1.0)
        # lengths and requests read, lengths and offsets written; a token's slot, sequence and length;
        # a new page out of the pool into its table
        return {"bytes": 16 * c["S"] + 12 * tokens + 8 * tokens / c["page"], "flops": 0}
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "append":
        row = 2 * c["heads"] * c["dim"]
        return {"bytes": 4 * c["T"] + 0.9 * c["T"] * row * (e + (2 if c["src"] == "bf16" else 4)),
                "flops": 0}
    S, N, H = c["S"], c["S"] * c["per"], c["heads"] * c["group"]
    tokens = sum(_spread(S, c["lo"], c["hi"], c["log"]))
    pairs = tokens * c["per"]
    if c["prefix"]:
        pairs += sum(_spread(N, 1, c["prefix"], False))
        tokens += c["prefix"] * -(-S // c["share"])
    return {"bytes": tokens * c["heads"] * c["dim"] * 2 * e + tokens / c["page"] * 4
            + N * H * (2 * c["dim"] * e + 4) + 4 * N, "flops": 4 * pairs * H * c["dim"]}


# ------------------------------------------------------------------ the definitions, fp64 ---
def _exact_attend(s):
    """Sequence by sequence, from the softmax's definition, in fp64."""
    N, H, D = s["Q"].shape
    heads = s["K"].shape[2]
    page = s["page"]
    q = s["Q"].double().view(N, heads, H // heads, D)
    out = torch.zeros(N, heads, H // heads, D, dtype=torch.float64, device="cuda")
    lse = torch.full((N, heads, H // heads), NEG, dtype=torch.float64, device="cuda")

    def tokens_of(cache, seq, n):                          # [heads, n, D]
        pages = s["table"][seq, :_pages(n, page)].long()
        return cache[pages].reshape(-1, heads, D)[:n].double().permute(1, 0, 2)

    per = s["share"] if s["prefix"] else s["per"]          # rows that read tokens in common
    own_len = s["len"].tolist()
    pre_len = s["prefix_len"].tolist() if s["prefix"] else [0] * N
    for first in range(0, N, per):
        rows = range(first, min(N, first + per))
        if s["prefix"]:
            n = max(pre_len[r] for r in rows)
            k0 = tokens_of(s["K"], s["S"] + first // per, n)
            v0 = tokens_of(s["V"], s["S"] + first // per, n)
        else:
            n = max(own_len[r] for r in rows)
            k0, v0 = tokens_of(s["K"], first // per, n), tokens_of(s["V"], first // per, n)
        for r in rows:
            m = pre_len[r] if s["prefix"] else own_len[r]
            k, v = k0[:, :m], v0[:, :m]
            if s["prefix"]:
                k = torch.cat([k, tokens_of(s["K"], r, own_len[r])], 1)
                v = torch.cat([v, tokens_of(s["V"], r, own_len[r])], 1)
            if k.shape[1] == 0:
                continue
            x = torch.matmul(q[r], k.transpose(1, 2)) / math.sqrt(D)
            out[r] = torch.matmul(torch.softmax(x, 2), v)
            lse[r] = torch.logsumexp(x, 2)
    return dict(out=out.view(N, H, D), lse=lse.view(N, H))


def exact(case, seed):
    """Tables, slots and lengths are whole numbers; an appended row is its input, rounded once."""
    s = prepare(case, seed)
    if case["kind"] == "plan":
        return None
    if case["kind"] == "attend":
        return _exact_attend(s)
    o = {}
    for name in "KV":
        cache = s[name].double()
        flat = cache.reshape(-1, case["heads"], case["dim"])
        slot = s["slot"].long()
        # the row that fills each slot, if any
        row = torch.full((flat.shape[0] + 1,), -1, dtype=torch.long, device="cuda")
        row[torch.where(slot < 0, flat.shape[0], slot)] = torch.arange(len(slot), device="cuda")
        row = row[:-1, None, None]
        new = s[name + "_new"].double()
        o[name] = torch.where(row >= 0, new[row[:, 0, 0].clamp(min=0)], flat).view(cache.shape)
    return o
