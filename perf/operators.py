"""Cases and plain forms of the cache operators of a speculative-decoding round.

A round appends the keys and values of every sequence's pending token and of its drafts to a paged cache
held in e4m3 (one power-of-two scale for each block of tokens and head), attends over it, and keeps what the
verification accepted.  Four operators: the block tables and slot maps of a round (plan), the quantising write
(append), the attention of a few new tokens per sequence, or of a piece of a prompt, over the cache (attend),
and the move of an accepted tree path to the front of its tree (keep).

A block holds `bt` consecutive tokens of one sequence; caches are [blocks, heads, bt, d], scales [blocks, heads].
"""
import torch

own = False
DEV = "cuda"
CAP_BITS = {"length": 64, "blocks": 128, "room": 256}          # status bits of the plan


# ---- cases -----------------------------------------------------------------------------------------------

def listed():
    return [
        # block tables and slots of one decoding round: 64 sequences, speculation lengths 2 to 8, 16-token blocks
        {"name": "plan_round", "op": "plan", "B": 64, "new": "3,5,7,9", "lo": 1, "hi": 8192, "bt": 16},
        # a wave of 256 prompts admitted at once
        {"name": "plan_admit", "op": "plan", "B": 256, "new": "2048,77,511,1500,9", "lo": 0, "hi": 0, "bt": 16},
        # one token of one sequence: the smallest write there is
        {"name": "append_one", "op": "append", "B": 1, "new": "1", "lo": 200, "hi": 200, "H": 8, "d": 128, "bt": 16, "dtype": "bf16"},
        # a round of a large batch, heads of 64, views of a fused projection
        {"name": "append_round", "op": "append", "B": 256, "new": "2,4,6,9", "lo": 1, "hi": 500, "H": 8, "d": 64, "bt": 16, "dtype": "bf16"},
        # prompts of ragged lengths entering the cache
        {"name": "append_prompts", "op": "append", "B": 16, "new": "2048,4095,1000,1", "lo": 0, "hi": 0, "H": 8, "d": 128, "bt": 64, "dtype": "bf16"},
        # one token of one short sequence: latency
        {"name": "attend_one", "op": "attend", "B": 1, "new": "1", "lo": 200, "hi": 200, "Hq": 32, "Hkv": 8, "d": 128, "bt": 16, "tree": 0},
        # trees of drafts, 5 to 14 nodes, on ordinary contexts
        {"name": "attend_tree", "op": "attend", "B": 64, "new": "6,15,13", "lo": 100, "hi": 4096, "Hq": 32, "Hkv": 8, "d": 128, "bt": 16, "tree": 5},
        # the large batch: 256 sequences, speculation lengths 1 to 8, seven query heads per key head
        {"name": "attend_wide", "op": "attend", "B": 256, "new": "2,4,6,9", "lo": 1, "hi": 8191, "Hq": 28, "Hkv": 4, "d": 128, "bt": 64, "tree": 0},
        # two long contexts: the work has to be split over the tokens
        {"name": "attend_long", "op": "attend", "B": 2, "new": "5", "lo": 100003, "hi": 131072, "Hq": 32, "Hkv": 8, "d": 128, "bt": 32, "tree": 0},
        # pieces of prompts behind what is cached already
        {"name": "attend_prompt", "op": "attend", "B": 4, "new": "512,333", "lo": 0, "hi": 4096, "Hq": 32, "Hkv": 8, "d": 128, "bt": 16, "tree": 0},
        # accepted paths of a few small trees
        {"name": "keep_small", "op": "keep", "B": 4, "new": "7", "lo": 5, "hi": 300, "H": 8, "d": 128, "bt": 16, "tree": 3},
        # accepted paths of a large batch of trees
        {"name": "keep_large", "op": "keep", "B": 256, "new": "32,15,13", "lo": 0, "hi": 600, "H": 8, "d": 128, "bt": 16, "tree": 7},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))

    def some(lo, hi, k):
        return ",".join(str(log(lo, hi)) for _ in range(k))

    op = rng.choice(["plan", "append", "attend", "attend", "attend", "keep"])
    bt = rng.choice([16, 32, 64, 128])
    if op == "plan":
        if rng.random() < 0.5:
            return {"op": op, "B": log(1, 1024), "new": some(1, 32, 3), "lo": 0, "hi": log(1, 8192), "bt": bt}
        return {"op": op, "B": log(1, 128), "new": some(1, 1800, 3), "lo": 0, "hi": log(1, 500), "bt": bt}
    if op == "append":
        c = {"op": op, "H": rng.choice([1, 2, 5, 8]), "d": rng.choice([64, 128]), "bt": bt, "dtype": rng.choice(["bf16", "f32"])}
        if rng.random() < 0.5:
            return {**c, "B": log(1, 256), "new": some(1, 32, 3), "lo": 0, "hi": log(1, 500)}
        return {**c, "B": log(1, 8), "new": some(16, 2048, 3), "lo": 0, "hi": log(1, 200)}
    if op == "keep":
        return {"op": op, "B": log(1, 200), "new": some(2, 32, 3), "lo": 0, "hi": log(1, 600), "H": rng.choice([1, 4, 8]),
                "d": rng.choice([64, 128]), "bt": bt, "tree": rng.randrange(1, 1000)}
    Hkv = rng.choice([1, 2, 4, 8])
    c = {"op": op, "Hq": Hkv * rng.choice([1, 2, 4, 7, 8]), "Hkv": Hkv, "d": rng.choice([64, 128]), "bt": bt}
    if rng.random() < 0.2:                                       # a piece of a prompt
        return {**c, "B": log(1, 4), "new": some(33, 512, 2), "lo": 0, "hi": log(1, 4096), "tree": 0}
    B = log(1, 256)
    hi = log(1, min(65536, 500000 // B))
    return {**c, "B": B, "new": some(1, 20, 3), "lo": rng.randrange(0, hi + 1), "hi": hi, "tree": rng.choice([0, rng.randrange(1, 1000)])}


def _new(case):
    n = [int(x) for x in case["new"].split(",")]
    return [n[b % len(n)] for b in range(case["B"])]


def _ctx(case):
    """Tokens in the cache before the call: spread over lo..hi, the same for every seed."""
    span = case["hi"] - case["lo"]
    return [case["lo"] + int(round(span * ((b * 0.6180339887498949 + 1.0) % 1.0 if case["B"] > 2 else 1.0 - b))) for b in range(case["B"])]


def _parents(case, n):
    """Parents of nodes 1..n-1 of a tree of n rows (row 0: the pending token)."""
    return [(k * k * case["tree"] + case["tree"]) % k for k in range(1, n)]


# ---- inputs ------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cache(shape, g):
    """A cache filled by earlier rounds: values of a size of their own for each block and head, as codes and scales."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    x *= torch.exp(0.5 * torch.randn(shape[:2] + (1, 1), generator=g, device=DEV)).to(torch.bfloat16)
    s = _scale_of(x.abs().amax((2, 3)).float())
    x /= s[:, :, None, None].to(torch.bfloat16)
    return x.to(torch.float8_e4m3fn), s


def _tables(ctx, new, bt, g, spare=5):
    """Blocks in a shuffled order for ctx + new tokens of every sequence."""
    held = [-(-(c + n) // bt) for c, n in zip(ctx, new)]
    n_blocks = sum(held) + spare
    perm = torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(ctx), max(held) + 1), -1, dtype=torch.int32, device=DEV)
    h = torch.tensor(held, device=DEV)
    at = torch.arange(table.shape[1], device=DEV)[None] < h[:, None]
    table[at] = perm[: sum(held)]
    return table, n_blocks


def _slots(table, ctx, new, bt):
    b = torch.repeat_interleave(torch.arange(len(new), device=DEV), torch.tensor(new, device=DEV))
    cu = torch.zeros(len(new) + 1, dtype=torch.int64, device=DEV)
    cu[1:] = torch.tensor(new, device=DEV).cumsum(0)
    pos = torch.arange(len(b), device=DEV) - cu[b] + torch.tensor(ctx, device=DEV)[b]
    return cu.to(torch.int32), (table[b, pos // bt] * bt + pos % bt).to(torch.int32)


def prepare(case, seed):
    g, op, B, bt = _gen(seed), case["op"], case["B"], case["bt"]
    ctx, new = _ctx(case), _new(case)
    s = {"case": dict(case), "ctx": _ints(ctx), "new": _ints(new), "nmax": max(new)}
    if op == "plan":
        held = [-(-c // bt) for c in ctx]
        want = [-(-(c + n) // bt) for c, n in zip(ctx, new)]
        n_blocks, T = sum(want) + 7, sum(new) + 13
        perm = torch.randperm(n_blocks, generator=g, device=DEV).to(torch.int32)
        table = torch.full((B, max(want) + 2), -1, dtype=torch.int32, device=DEV)
        at = torch.arange(table.shape[1], device=DEV)[None] < torch.tensor(held, device=DEV)[:, None]
        table[at] = perm[: sum(held)]
        free = torch.full((n_blocks,), -1, dtype=torch.int32, device=DEV)
        free[: n_blocks - sum(held)] = perm[sum(held):]
        e = lambda *n: torch.empty(*n, dtype=torch.int32, device=DEV)  # noqa: E731
        outs = lambda T: {"kv_len": e(B), "cu_new": e(B + 1), "slot_map": e(T), "positions": e(T), "status": e(B)}  # noqa: E731
        s.update(table=table, held=_ints(held), free=free, n_free=_ints([n_blocks - sum(held)]), seq_len=_ints(ctx),
                 none=_ints([0] * B), taken=outs(T), given=outs(1))
        return s
    table, n_blocks = _tables(ctx, new, bt, g)
    H = case["Hkv"] if op == "attend" else case["H"]
    s["table"] = table
    s["k_cache"], s["k_scale"] = _cache((n_blocks, H, bt, case["d"]), g)
    s["v_cache"], s["v_scale"] = _cache((n_blocks, H, bt, case["d"]), g)
    s["cu"], s["slots"] = _slots(table, ctx, new, bt)
    T = sum(new)
    if op == "append":                                           # keys and values as views of one fused projection
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        qkv = torch.randn(T, 4 * H, case["d"], generator=g, device=DEV, dtype=dt)
        qkv *= torch.exp(torch.randn(T, 1, 1, generator=g, device=DEV)).to(dt)
        s["k"], s["v"] = qkv[:, 2 * H : 3 * H], qkv[:, 3 * H :]
    elif op == "attend":
        s["q"] = (2.0 * torch.randn(T, case["Hq"], case["d"], generator=g, device=DEV)).to(torch.bfloat16)
        s["out"] = torch.zeros_like(s["q"])
        s["kv_len"] = s["ctx"] + s["new"]
        s["scale"] = case["d"] ** -0.5
        s["parent"] = None
        if case["tree"]:
            N = max(new) - 1
            s["parent"] = _ints([(_parents(case, n) + [0] * N)[:N] for n in new]) if N else None
    else:                                                        # accepted paths: root to a node drawn from the seed
        N = max(new) - 1
        pick = torch.randint(0, 1 << 30, (B,), generator=g, device=DEV).tolist()
        path, tau = [], []
        for b, n in enumerate(new):
            parent, node, p = _parents(case, n), pick[b] % n, []
            while node:
                p.insert(0, node)
                node = parent[node - 1]
            path.append((p + [-1] * N)[:N])
            tau.append(len(p))
        s["path"], s["tau"] = _ints(path), _ints(tau)
    return s


# ---- the operators ---------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"plan": _own_plan, "append": _own_append, "attend": _own_attend, "keep": _own_keep}[op](s)
    return {"plan": _plan, "append": _append, "attend": _attend, "keep": _keep}[op](s)


def _own_plan(s):
    """A round's blocks are taken, and given back as after a round that keeps nothing."""
    from paper_2505_15141_b200 import binding as bs
    for new, o in ((s["new"], s["taken"]), (s["none"], s["given"])):
        bs.bs_cache_plan(s["seq_len"], None, new, 0, None, s["case"]["bt"], s["table"], s["held"], s["free"], s["n_free"],
                         o["kv_len"], o["cu_new"], o["slot_map"], o["positions"], o["status"])
    return {"taken": s["taken"], "given": s["given"], "free": s["free"], "n_free": s["n_free"], "table": s["table"]}


def _own_append(s):
    from paper_2505_15141_b200 import binding as bs
    bs.bs_cache_append(s["k"], s["v"], s["slots"], s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"])
    return {n: s[n] for n in ("k_cache", "k_scale", "v_cache", "v_scale")}


def _own_attend(s):
    from paper_2505_15141_b200 import binding as bs
    c = s["case"]
    if "workspace" not in s:
        s["workspace"] = bs.new_cache_workspace(c["Hq"], c["Hkv"], c["d"], DEV)
    bs.bs_cache_attention(s["q"], s["cu"], s["kv_len"], s["table"], s["parent"], s["k_cache"], s["k_scale"], s["v_cache"],
                          s["v_scale"], s["nmax"], s["scale"], s["out"], None, s["workspace"])
    return s["out"]


def _own_keep(s):
    from paper_2505_15141_b200 import binding as bs
    bs.bs_cache_keep_path(s["path"], s["tau"], s["ctx"], s["table"], s["k_cache"], s["k_scale"], s["v_cache"], s["v_scale"], None)
    return {n: s[n] for n in ("k_cache", "k_scale", "v_cache", "v_scale")}


def _scale_of(amax):
    """The smallest power of two s with amax / s <= 448, at least 2^-64."""
    m, e = torch.frexp(amax)                                     # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    return torch.ldexp(torch.ones_like(amax), torch.where(amax > 0, e - 9 + (m > 0.875).int(), -64).clamp(min=-64))


def _codes(x):
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _plan_once(s, new, o):
    bt, T = s["case"]["bt"], o["slot_map"].numel()
    B, wide = s["table"].shape
    n_blocks = s["free"].numel()
    L, held, n = s["seq_len"].long(), s["held"].long(), new.long()
    n_free = s["n_free"].long()
    bad = (L < 0) | (n < 0) | (held < 0) | (held > wide) | (L > held * bt) | (L + n > wide * bt)
    n = torch.where(bad, 0, n)
    full = ~bad & (n > 0) & (n.cumsum(0) > T)
    delta = torch.where(bad | full, 0, (L + n + bt - 1) // bt - held)
    back, need = (-delta).clamp(min=0), delta.clamp(min=0)
    avail = n_free + back.sum()
    short = (need > 0) & (need.cumsum(0) > avail)
    got = torch.where(short, 0, need)
    n = torch.where(full | short, 0, n)
    L = torch.where(bad, 0, L)
    col = torch.arange(wide, device=DEV)[None]
    table = s["table"].long()
    gives = (col >= (held - back)[:, None]) & (col < held[:, None])
    takes = (col >= held[:, None]) & (col < (held + got)[:, None])
    gone = table[gives]                                          # in the order of the sequences, ascending within one
    stack = torch.cat([s["free"].long(), torch.zeros_like(gone)])
    top = n_free + len(gone)
    stack[top - 1 - torch.arange(len(gone), device=DEV)] = gone
    count = got.sum()
    table[gives] = -1
    table[takes] = stack[top - 1 - torch.arange(int(count), device=DEV)]
    s["table"].copy_(table)
    s["free"].copy_(stack[:n_blocks])
    s["held"].copy_(held - back + got)
    s["n_free"].copy_(top - count)
    cu = torch.zeros(B + 1, dtype=torch.int64, device=DEV)
    cu[1:] = n.cumsum(0)
    i = torch.arange(T, device=DEV)
    b = torch.searchsorted(cu[1:], i, right=True).clamp(max=B - 1)
    pos = i - cu[b] + L[b]
    live = i < cu[-1]
    pos = torch.where(live, pos, 0)
    o["slot_map"].copy_(torch.where(live, table[b, pos // bt] * bt + pos % bt, -1))
    o["positions"].copy_(torch.where(live, pos, -1))
    o["kv_len"].copy_(L + n)
    o["cu_new"].copy_(cu)
    o["status"].copy_(CAP_BITS["length"] * bad + CAP_BITS["room"] * full + CAP_BITS["blocks"] * short)


def _plan(s):
    _plan_once(s, s["new"], s["taken"])
    _plan_once(s, s["none"], s["given"])
    return {"taken": s["taken"], "given": s["given"], "free": s["free"], "n_free": s["n_free"], "table": s["table"]}


def _append_one(x, slots, cache, scale, bt):
    live = slots >= 0
    x, at = x[live].float(), slots[live].long()
    ub, inv = torch.unique(at // bt, return_inverse=True)
    off = at % bt
    first = torch.full((len(ub),), bt, device=DEV, dtype=torch.int64).scatter_reduce_(0, inv, off, "amin")
    big = torch.where(torch.isfinite(x), x.abs(), 0).amax(2)     # [T, H]
    amax = torch.zeros(len(ub), x.shape[1], device=DEV).scatter_reduce_(0, inv[:, None].expand_as(big), big, "amax")
    old, s_new = scale[ub], _scale_of(amax)
    s_new = torch.where(first[:, None] == 0, s_new, torch.maximum(old, s_new))
    codes = cache.view(torch.uint8)
    page = codes[ub]                                             # [blocks, H, bt, d]
    kept = (torch.arange(bt, device=DEV)[None] < first[:, None])[:, None, :, None] & (s_new > old)[:, :, None, None]
    again = _codes(page.view(torch.float8_e4m3fn).float() * (old / s_new)[:, :, None, None])
    page = torch.where(kept, again, page)
    page[inv, :, off] = _codes(x / s_new[inv][:, :, None])
    codes[ub] = page
    scale[ub] = s_new


def _append(s):
    _append_one(s["k"], s["slots"], s["k_cache"], s["k_scale"], s["case"]["bt"])
    _append_one(s["v"], s["slots"], s["v_cache"], s["v_scale"], s["case"]["bt"])
    return {n: s[n] for n in ("k_cache", "k_scale", "v_cache", "v_scale")}


def _seen(s, nmax, L):
    """[B, nmax, L]: which positions of its sequence a new token sees; the rows behind a sequence's last see nothing."""
    B = s["table"].shape[0]
    kv, n = s["kv_len"].long(), s["new"].long()
    base = (kv - n)[:, None, None]
    i = torch.arange(nmax, device=DEV)[None, :, None]
    p = torch.arange(L, device=DEV)[None, None]
    if s["parent"] is None:
        see = p <= base + i
    else:
        anc = torch.eye(nmax, dtype=torch.bool, device=DEV).repeat(B, 1, 1)
        anc[:, :, 0] = True
        parent = torch.nn.functional.pad(s["parent"].long(), (1, 0))[:, :nmax]
        up = torch.arange(nmax, device=DEV)[None].repeat(B, 1)
        for _ in range(nmax):                                    # one step towards the root for every node at once
            up = torch.where(up > 0, parent.gather(1, up), 0)
            anc.scatter_(2, up[:, :, None], True)
        j = (p - base).clamp(0, nmax - 1).expand(B, nmax, L)
        see = (p < base) | anc.gather(2, j)
    return see & (p < kv[:, None, None]) & (i < n[:, None, None])


def _attend(s):
    c = s["case"]
    B, wide = s["table"].shape
    Hkv, G, d, nmax = c["Hkv"], c["Hq"] // c["Hkv"], c["d"], s["nmax"]
    at = s["table"].long().clamp(min=0)
    L = wide * c["bt"]
    k, v = ((s[n + "_cache"][at].float() * s[n + "_scale"][at][..., None, None]).transpose(1, 2).reshape(B, Hkv, L, d)
            for n in ("k", "v"))
    i = s["cu"][:-1].long()[:, None] + torch.arange(nmax, device=DEV)[None]
    live = torch.arange(nmax, device=DEV)[None] < s["new"][:, None]
    q = s["q"][i.clamp(max=s["q"].shape[0] - 1)].float().view(B, nmax, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, nmax * G, d)
    see = _seen(s, nmax, L)[:, None, :, None].expand(B, 1, nmax, G, L).reshape(B, 1, nmax * G, L)
    t = (q @ k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~see, float("-inf"))
    t = t.sub_(t.amax(3, keepdim=True).clamp(min=-3e38)).exp_()
    o = (t @ v) / t.sum(3, keepdim=True).clamp(min=1e-30)
    o = o.view(B, Hkv, nmax, G, d).permute(0, 2, 1, 3, 4).reshape(B, nmax, Hkv * G, d)
    s["out"][i[live]] = o[live].to(torch.bfloat16)
    return s["out"]


def _keep_one(s, cache, scale, bt):
    B, N = s["path"].shape
    j = torch.arange(N, device=DEV)[None]
    live = j < s["tau"][:, None]
    base = s["ctx"].long()[:, None]
    b = torch.arange(B, device=DEV)[:, None].expand(B, N)[live]
    src, dst = (base + s["path"].long())[live], (base + 1 + j)[live]
    table = s["table"].long()
    sb, db = table[b, src // bt], table[b, dst // bt]
    ub, inv = torch.unique(db, return_inverse=True)
    codes = cache.view(torch.uint8)
    H = scale.shape[1]
    old, moved = scale[ub], scale[sb]                            # [blocks, H], [tokens, H]
    s_new = old.clone().scatter_reduce_(0, inv[:, None].expand(-1, H), moved, "amax")
    first = torch.full((len(ub),), bt, device=DEV, dtype=torch.int64).scatter_reduce_(0, inv, dst % bt, "amin")
    x = codes[sb, :, src % bt].view(torch.float8_e4m3fn).float() * (moved / s_new[inv])[:, :, None]
    page = codes[ub]
    stays = (torch.arange(bt, device=DEV)[None] < first[:, None])[:, None, :, None]
    again = _codes(page.view(torch.float8_e4m3fn).float() * (old / s_new)[:, :, None, None])
    page = torch.where(stays & (s_new > old)[:, :, None, None], again, page)
    page[inv, :, dst % bt] = _codes(x)
    codes[ub] = page
    scale[ub] = s_new


def _keep(s):
    _keep_one(s, s["k_cache"], s["k_scale"], s["case"]["bt"])
    _keep_one(s, s["v_cache"], s["v_scale"], s["case"]["bt"])
    return {n: s[n] for n in ("k_cache", "k_scale", "v_cache", "v_scale")}


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    B, bt, new, ctx = case["B"], case["bt"], _new(case), _ctx(case)
    T = sum(new)
    if case["op"] == "plan":
        taken = sum(-(-(c + n) // bt) - -(-c // bt) for c, n in zip(ctx, new))
        # lengths, counts and results of every sequence, slots and positions, blocks taken and given back
        return {"bytes": 2 * 4 * 7 * B + 8 * (T + 13) + 4 * 4 * taken, "flops": 0}
    d = case["d"]
    if case["op"] == "append":
        e = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * T * case["H"] * d * (e + 1) + 4 * T, "flops": 4 * T * case["H"] * d}
    if case["op"] == "keep":
        # about half of a tree's depth passes; a moved token is read and written once in each cache
        moved = sum(max(1, n.bit_length() // 2) for n in new)
        return {"bytes": 4 * moved * case["H"] * d + 8 * B, "flops": 2 * moved * case["H"] * d}
    Hq, Hkv = case["Hq"], case["Hkv"]
    kv = sum(c + n for c, n in zip(ctx, new))
    pairs = sum(n * c + n * (n + 1) // 2 for c, n in zip(ctx, new))
    return {"bytes": kv * Hkv * (2 * d + 8 / bt) + 4 * T * Hq * d + 4 * kv / bt, "flops": 4 * pairs * Hq * d}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _grid64(x):
    """x rounded to the nearest e4m3 value, ties to the even one, what is too large to the largest."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp(max=8) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _scale64(amax):
    """2^e with the smallest e >= -64 that brings amax to 448 or less."""
    e = torch.ceil(torch.log2(amax.clamp(min=1e-60) / 448.0)).clamp(min=-64)
    e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)
    e = torch.where((e > -64) & (amax <= 448.0 * torch.exp2(e - 1)), e - 1, e)
    return torch.exp2(e)


def _exact_plan(case, s):
    """Whole numbers, sequence by sequence: a stack of free blocks, popped and pushed."""
    return None                                                  # no computed numbers among its outputs


def _exact_append(case, s):
    bt, out = case["bt"], {}
    for n in ("k", "v"):
        codes, scale, x = s[n + "_cache"].double(), s[n + "_scale"].double(), s[n].double()
        start = 0
        for L, m in zip(_ctx(case), _new(case)):
            slots = s["slots"][start:start + m].tolist()
            i = 0
            while i < m:
                blk, off = divmod(slots[i], bt)
                r = min(m - i, bt - off)
                rows = x[start + i:start + i + r]                # [r, H, d]
                sc = _scale64(rows.abs().amax((0, 2)))
                if off:
                    sc = torch.maximum(sc, scale[blk])
                    codes[blk, :, :off] = _grid64(codes[blk, :, :off] * (scale[blk] / sc)[:, None, None])
                codes[blk, :, off:off + r] = _grid64(rows.transpose(0, 1) / sc[:, None, None])
                scale[blk] = sc
                i += r
            start += m
        out[n + "_cache"], out[n + "_scale"] = codes, scale
    return {n: out[n] for n in ("k_cache", "k_scale", "v_cache", "v_scale")}


def _exact_attend(case, s):
    bt, G = case["bt"], case["Hq"] // case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    start = 0
    for b, (c, n) in enumerate(zip(_ctx(case), _new(case))):
        L = c + n
        blocks = s["table"][b, : -(-L // bt)].long()
        see = torch.ones(n, L, dtype=torch.bool, device=DEV)
        if case["tree"]:
            parent, line = _parents(case, n), []
            for i in range(n):
                line.append({i} if i == 0 else {i} | line[parent[i - 1]])
            see[:, c:] = torch.tensor([[j in line[i] for j in range(n)] for i in range(n)], device=DEV)
        else:
            see[:, c:] = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
        for h in range(case["Hkv"]):
            k = (s["k_cache"][blocks, h].double() * s["k_scale"][blocks, h, None, None].double()).reshape(-1, case["d"])[:L]
            v = (s["v_cache"][blocks, h].double() * s["v_scale"][blocks, h, None, None].double()).reshape(-1, case["d"])[:L]
            q = s["q"][start:start + n, h * G:(h + 1) * G].double()
            t = torch.einsum("igd,ld->gil", q, k) * s["scale"]
            p = torch.softmax(t.masked_fill(~see, float("-inf")), 2)
            out[start:start + n, h * G:(h + 1) * G] = torch.einsum("gil,ld->igd", p, v)
        start += n
    return out


def _exact_keep(case, s):
    bt, out = case["bt"], {}
    paths, taus, tables = s["path"].tolist(), s["tau"].tolist(), s["table"].tolist()
    for n in ("k", "v"):
        was, sc0 = s[n + "_cache"].double(), s[n + "_scale"].double()
        codes, scale = was.clone(), sc0.clone()
        for b, base in enumerate(_ctx(case)):
            moves = [(divmod(base + 1 + i, bt), divmod(base + paths[b][i], bt)) for i in range(taus[b])]
            for page in sorted({m[0][0] for m in moves}):
                blk, here = tables[b][page], [m for m in moves if m[0][0] == page]
                sc = torch.stack([sc0[blk]] + [sc0[tables[b][m[1][0]]] for m in here]).amax(0)
                lead = here[0][0][1]
                codes[blk, :, :lead] = _grid64(was[blk, :, :lead] * (sc0[blk] / sc)[:, None, None])
                for (_, to), (sp, so) in here:
                    sb = tables[b][sp]
                    codes[blk, :, to] = _grid64(was[sb, :, so] * (sc0[sb] / sc)[:, None])
                scale[blk] = sc
        out[n + "_cache"], out[n + "_scale"] = codes, scale
    return {n: out[n] for n in ("k_cache", "k_scale", "v_cache", "v_scale")}


def exact(case, seed):
    s = prepare(case, seed)
    return {"plan": _exact_plan, "append": _exact_append, "attend": _exact_attend, "keep": _exact_keep}[case["op"]](case, s)
