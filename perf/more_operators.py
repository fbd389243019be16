"""Cases and plain forms of what a prompt and a round need around the key / value cache and the verification.

A prompt enters through four steps: its queries and keys are rotated to their positions (rotate), it attends to itself
(attend), its keys and values go into the cache, and its tokens are entered in the token history of its sequence
(history).  A round rotates at the positions of its chain or tree, attends over the cache, and before the verification the
logits of every drafted position are adjusted by penalties on the history and on the drafted tokens of its path, by
biases and by grammar masks (adjust); what was emitted is entered in the history again.

New tokens of all sequences are packed: those of sequence b are rows cu[b] .. cu[b + 1] - 1.  An entry of the history is
2 * (times the token was emitted, up to 16383) + (1 if it is in the prompt).
"""
import math

import torch

own = False
DEV = "cuda"
MOST = 16383                                                     # emitted tokens that an entry counts


# ---- cases -----------------------------------------------------------------------------------------------

def listed():
    return [
        # one short prompt: latency counts
        {"name": "attend_one", "op": "attend", "n": "130", "Hq": 32, "Hkv": 8, "d": 128},
        # a wave of ragged prompts admitted at once, one of them a single token
        {"name": "attend_wave", "op": "attend", "n": "2048,77,511,1500,9,3001,4096,128,1,1023,2500,640,3333,256,1800,901", "Hq": 32, "Hkv": 8, "d": 128},
        # a long document
        {"name": "attend_long", "op": "attend", "n": "16384", "Hq": 32, "Hkv": 8, "d": 128},
        # heads of 64, each with keys of its own
        {"name": "attend_narrow", "op": "attend", "n": "4095,2047,1000,3500", "Hq": 16, "Hkv": 16, "d": 64},
        # the pending token and four drafts of one sequence, far into its context
        {"name": "rotate_one", "op": "rotate", "n": "5", "lo": 100003, "hi": 100003, "Hq": 32, "Hkv": 8, "d": 128, "rot": 128,
         "pairs": "half", "scaling": "yarn", "dtype": "bf16", "tree": 0},
        # trees of drafts of a large batch, neighbours as pairs, a quarter of the head
        {"name": "rotate_trees", "op": "rotate", "n": ",".join(["6", "15", "13", "32"] * 64), "lo": 1, "hi": 8191, "Hq": 28, "Hkv": 4, "d": 128,
         "rot": 32, "pairs": "next", "scaling": "none", "dtype": "bf16", "tree": 5},
        # a wave of prompts, frequencies scaled by bands
        {"name": "rotate_prompts", "op": "rotate", "n": "2048,4095,1000,1,8192,600,5000,3001", "lo": 0, "hi": 0, "Hq": 32, "Hkv": 8, "d": 128,
         "rot": 128, "pairs": "half", "scaling": "bands", "dtype": "bf16", "tree": 0},
        # one sequence, four drafts, penalties and a few biases
        {"name": "adjust_one", "op": "adjust", "B": 1, "V": 128256, "gamma": "4", "R": 5, "dtype": "f32", "tree": 0, "pen": True, "bias": 20,
         "masks": 0, "inplace": False},
        # a batch of ragged rounds with penalties, biases and grammar masks
        {"name": "adjust_round", "op": "adjust", "B": 64, "V": 152064, "gamma": "2,4,6,8", "R": 9, "dtype": "bf16", "tree": 0, "pen": True,
         "bias": 300, "masks": 40, "inplace": False},
        # grammar masks alone on the logits where they lie, trees of drafts, an odd vocabulary
        {"name": "adjust_masks", "op": "adjust", "B": 64, "V": 32003, "gamma": "5,14,12", "R": 15, "dtype": "f32", "tree": 3, "pen": False,
         "bias": 0, "masks": 200, "inplace": True},
        # what a round of a large batch emitted
        {"name": "history_round", "op": "history", "B": 256, "V": 152064, "n": "", "W": 9},
        # a wave of prompts: histories begin anew
        {"name": "history_prompts", "op": "history", "B": 64, "V": 128256, "n": "2048,77,511,1500,9,8192,4096,1", "W": 0},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))

    op = rng.choice(["attend", "attend", "rotate", "adjust", "adjust", "history"])
    if op == "attend":
        Hkv = rng.choice([1, 2, 4, 8, 16])
        c = {"op": op, "Hq": Hkv * rng.choice([1, 2, 4, 7, 8]), "Hkv": Hkv, "d": rng.choice([64, 128])}
        n, room = [], 16384.0 ** 2 * 32 * 128
        for _ in range(log(1, 48)):                              # no more than a long document costs
            k = min(log(1, 16384), int(math.sqrt(room / c["Hq"] / c["d"])))
            if k < 1 or sum(n) + k > 40000:
                break
            n.append(k)
            room -= float(k) * k * c["Hq"] * c["d"]
        return {**c, "n": ",".join(map(str, n))}
    if op == "rotate":
        tree = rng.choice([0, 0, rng.randrange(1, 1000)])
        Hkv, d = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
        few = tree or rng.random() < 0.5
        n = [log(1, 32) for _ in range(log(1, 256))] if few else [log(1, 8192) for _ in range(log(1, 6))]
        hi = log(1, 200000) if few else 0
        return {"op": op, "n": ",".join(map(str, n)), "lo": rng.randrange(0, hi + 1), "hi": hi, "Hq": Hkv * rng.choice([1, 2, 4, 7]), "Hkv": Hkv,
                "d": d, "rot": rng.choice([d, d, d // 2, d // 4, 24]), "pairs": rng.choice(["half", "next"]),
                "scaling": rng.choice(["none", "linear", "bands", "yarn"]), "dtype": rng.choice(["bf16", "bf16", "f32"]), "tree": tree}
    if op == "adjust":
        R, V, dtype = rng.randrange(1, 17), log(1000, 152064), rng.choice(["bf16", "f32"])
        B = max(1, min(log(1, 256), 80000000 // (R * V)))
        masks = rng.choice([0, log(1, 200)])
        return {"op": op, "B": B, "V": V, "gamma": ",".join(str(rng.randrange(0, R)) for _ in range(3)), "R": R, "dtype": dtype,
                "tree": rng.choice([0, rng.randrange(1, 1000)]), "pen": masks == 0 or rng.random() < 0.7, "bias": rng.choice([0, log(1, 400)]),
                "masks": masks, "inplace": False}
    V = log(1000, 152064)
    if rng.random() < 0.5:
        return {"op": op, "B": log(1, 512), "V": V, "n": "", "W": rng.randrange(1, 33)}
    return {"op": op, "B": log(1, 64), "V": V, "n": ",".join(str(log(1, 8192)) for _ in range(3)), "W": rng.choice([0, 5])}


def _numbers(text):
    return [int(x) for x in text.split(",")] if text else []


def _per_sequence(case, key):
    v = _numbers(case[key])
    return [v[b % len(v)] for b in range(case["B"])]


def _ctx(case, B):
    """Tokens in the cache before the call: spread over lo..hi, the same for every seed."""
    span = case["hi"] - case["lo"]
    return [case["lo"] + int(round(span * ((b * 0.6180339887498949 + 1.0) % 1.0))) for b in range(B)]


def _parents(tree, n):
    """Parents of nodes 1..n-1 of a tree of n rows (row 0: the pending token)."""
    return [(tree * (k + 3) // 2) % k if tree else k - 1 for k in range(1, n)]


SCALINGS = {"none": {}, "linear": {"factor": 4.0}, "bands": {"factor": 8.0, "low": 1.0, "high": 4.0, "original": 8192},
            "yarn": {"factor": 32.0, "low": 1.0, "high": 32.0, "original": 4096}}
BASE = 500000.0


# ---- inputs ------------------------------------------------------------------------------------------------

def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cu(n):
    return torch.nn.functional.pad(torch.tensor(n, device=DEV).cumsum(0), (1, 0)).to(torch.int32)


def _tokens(shape, V, g):
    """Token ids, the low ones far more often, as in text."""
    return (V * torch.rand(shape, generator=g, device=DEV) ** 4).long().clamp(max=V - 1).to(torch.int32)


def prepare(case, seed):
    g, op = torch.Generator(device=DEV).manual_seed(int(seed)), case["op"]
    s = {"case": dict(case)}
    if op == "attend":                                           # views of a fused projection
        n, Hq, Hkv, d = _numbers(case["n"]), case["Hq"], case["Hkv"], case["d"]
        qkv = torch.randn(sum(n), Hq + 2 * Hkv, d, generator=g, device=DEV)
        qkv[:, :Hq] *= 2.0
        qkv = qkv.to(torch.bfloat16)
        s.update(n=n, cu=_cu(n), q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], v=qkv[:, Hq + Hkv:],
                 out=torch.zeros(sum(n), Hq, d, dtype=torch.bfloat16, device=DEV), scale=d ** -0.5)
    elif op == "rotate":
        n, Hq, Hkv, d = _numbers(case["n"]), case["Hq"], case["Hkv"], case["d"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        qkv = torch.randn(sum(n), Hq + 2 * Hkv, d, generator=g, device=DEV, dtype=dt)
        b = torch.repeat_interleave(torch.arange(len(n), device=DEV), torch.tensor(n, device=DEV))
        cu = _cu(n)
        s.update(cu=cu, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], seq=b,
                 positions=(torch.arange(sum(n), device=DEV) - cu[b] + _ints(_ctx(case, len(n)))[b]).to(torch.int32),
                 q_out=torch.zeros(sum(n), Hq, d, dtype=dt, device=DEV), k_out=torch.zeros(sum(n), Hkv, d, dtype=dt, device=DEV))
        s["parent"] = None
        if case["tree"]:
            N = max(max(n) - 1, 1)
            s["parent"] = _ints([(_parents(case["tree"], k) + [0] * N)[:N] for k in n])
    elif op == "adjust":
        B, V, R, gamma = case["B"], case["V"], case["R"], _per_sequence(case, "gamma")
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        N = max(R - 1, 1)
        s.update(logits=(3.0 * torch.randn(B, R, V, generator=g, device=DEV, dtype=dt)), gamma=_ints(gamma), drafted=_tokens((B, N), V, g))
        s["out"] = s["logits"] if case["inplace"] else torch.zeros_like(s["logits"])
        s["parent"] = _ints([(_parents(case["tree"], R) + [0] * N)[:N]] * B) if case["tree"] else None
        s["history"] = s["rep"] = s["pres"] = s["freq"] = s["begin"] = s["bias_tokens"] = s["bias"] = s["masks"] = s["mask_row"] = None
        if case["pen"]:
            s["history"] = torch.zeros(B, V, dtype=torch.int16, device=DEV)
            prompt, emitted = _tokens((B, 700), V, g).long(), _tokens((B, 300), V, g).long()
            s["history"].scatter_(1, prompt, 1)
            s["history"].scatter_add_(1, emitted, torch.full_like(emitted, 2, dtype=torch.int16))
            r = torch.rand(3, B, generator=g, device=DEV)
            s["rep"], s["pres"], s["freq"] = 1.0 + 0.5 * r[0], 2.0 * r[1] - 0.5, 1.5 * r[2] - 0.3
        if case["bias"]:
            count = [case["bias"] * (b % 3) // 2 if B > 1 else case["bias"] for b in range(B)]
            s["begin"] = _cu(count)
            s["bias_tokens"] = _tokens((sum(count),), V, g)
            s["bias"] = 5.0 * torch.randn(sum(count), generator=g, device=DEV)
        if case["masks"]:                                        # a handful of tokens, a third, nearly all
            share = torch.tensor([0.002, 0.3, 0.98], device=DEV)[torch.arange(case["masks"], device=DEV) % 3]
            words = -(-V // 32)
            s["masks"] = torch.empty(case["masks"], words, dtype=torch.int32, device=DEV)
            bit = torch.arange(32, device=DEV)
            for m in range(case["masks"]):
                allowed = torch.rand(words, 32, generator=g, device=DEV) < share[m]
                s["masks"][m] = (allowed.long() << bit).sum(1).to(torch.int32)
            s["mask_row"] = torch.randint(-1, case["masks"], (B, R), generator=g, device=DEV, dtype=torch.int32)
    else:
        B, V = case["B"], case["V"]
        s["history"] = 2 * torch.randint(0, 3, (B, V), generator=g, device=DEV, dtype=torch.int16) + (torch.rand(B, V, generator=g, device=DEV) < 0.01)
        s["history"] = s["history"].to(torch.int16)
        s["fresh"] = s["cu"] = s["prompt"] = s["tokens"] = s["len"] = None
        if case["n"]:
            n = _per_sequence(case, "n")
            s.update(fresh=torch.ones(B, dtype=torch.uint8, device=DEV), cu=_cu(n), prompt=_tokens((sum(n),), V, g))
        if case["W"]:
            s.update(tokens=_tokens((B, case["W"]), V, g), len=torch.randint(1, case["W"] + 1, (B,), generator=g, device=DEV, dtype=torch.int32))
    return s


# ---- the operators ---------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": _own_attend, "rotate": _own_rotate, "adjust": _own_adjust, "history": _own_history}[op](s)
    return {"attend": _attend, "rotate": _rotate, "adjust": _adjust, "history": _history}[op](s)


def _own_attend(s):
    from paper_2505_15141_b200 import binding as bs
    bs.bs_prompt_attention(s["q"], s["k"], s["v"], s["cu"], s["scale"], s["out"], None)
    return s["out"]


def _own_rotate(s):
    from paper_2505_15141_b200 import binding as bs
    c = s["case"]
    if "table" not in s:                                         # made once, when a program starts
        s["table"] = bs.new_rotary_table(c["rot"], BASE, c["scaling"], **SCALINGS[c["scaling"]], device=DEV)
    trees = {} if s["parent"] is None else {"cu_new": s["cu"], "node_parent": s["parent"]}
    bs.bs_rotary(s["q"], s["k"], s["positions"], s["table"], c["pairs"] == "next", s["q_out"], s["k_out"], **trees)
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_adjust(s):
    from paper_2505_15141_b200 import binding as bs
    bs.bs_logits_adjust(s["logits"], s["out"], s["gamma"], 1, draft_tokens=s["drafted"], node_parent=s["parent"], history=s["history"],
                        repetition=s["rep"], presence=s["pres"], frequency=s["freq"], bias_begin=s["begin"], bias_tokens=s["bias_tokens"],
                        bias_values=s["bias"], masks=s["masks"], mask_row=s["mask_row"])
    return s["out"]


def _own_history(s):
    from paper_2505_15141_b200 import binding as bs
    bs.bs_history_update(s["history"], fresh=s["fresh"], cu_prompt=s["cu"], prompt_tokens=s["prompt"], out_tokens=s["tokens"], out_len=s["len"])
    return s["history"]


def _attend(s):
    """Sequence by sequence, as many rows at a time as some gigabytes of scores allow."""
    c, start = s["case"], 0
    G = c["Hq"] // c["Hkv"]
    for n in s["n"]:
        q, k, v = (s[x][start:start + n].float().transpose(0, 1) for x in ("q", "k", "v"))
        q, out = q.reshape(c["Hkv"], G, n, c["d"]), s["out"][start:start + n]
        rows = max(64, min(n, (1 << 29) // (c["Hq"] * n)))
        for i in range(0, n, rows):
            end = min(n, i + rows)
            qi = q[:, :, i:end].reshape(c["Hkv"], G * (end - i), c["d"])
            t = (qi @ k[:, :end].transpose(1, 2)).mul_(s["scale"]).view(c["Hkv"], G, end - i, end)
            later = torch.arange(end, device=DEV)[None] > torch.arange(i, end, device=DEV)[:, None]
            t = t.masked_fill_(later, float("-inf"))
            t = t.sub_(t.amax(3, keepdim=True)).exp_()
            o = (t.view(c["Hkv"], G * (end - i), end) @ v[:, :end]).view(c["Hkv"], G, end - i, c["d"]) / t.sum(3, keepdim=True)
            out[i:end] = o.view(c["Hq"], end - i, c["d"]).transpose(0, 1).to(torch.bfloat16)
        start += n
    return s["out"]


def _frequencies(case):
    """Radians a position, [rot / 2] in 64 bits, and the amplitude."""
    rot, w = case["rot"], SCALINGS[case["scaling"]]
    i = torch.arange(rot // 2, dtype=torch.float64, device=DEV)
    f = BASE ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        return f / w["factor"], 1.0
    if case["scaling"] == "bands":
        keep = ((w["original"] * f / (2 * math.pi) - w["low"]) / (w["high"] - w["low"])).clamp(0, 1)
        return f * (keep + (1 - keep) / w["factor"]), 1.0
    if case["scaling"] == "yarn":
        at = [rot * math.log(w["original"] / (2 * math.pi * r)) / (2 * math.log(BASE)) for r in (w["high"], w["low"])]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        ramp = ((i - first) / max(last - first, 0.001)).clamp(0, 1)
        return f * (1 - ramp + ramp / w["factor"]), 0.1 * math.log(w["factor"]) + 1.0
    return f, 1.0


def _depths(s):
    """Positions of the tokens: a tree's node stands as far behind the root as it is deep."""
    if s["parent"] is None:
        return s["positions"]
    B, N = s["parent"].shape
    parent = torch.nn.functional.pad(s["parent"].long(), (1, 0))
    up, depth = torch.arange(N + 1, device=DEV).repeat(B, 1), torch.zeros(B, N + 1, dtype=torch.int64, device=DEV)
    for _ in range(N):                                           # one step towards the root for every node at once
        depth += up > 0
        up = parent.gather(1, up)
    row = torch.arange(len(s["seq"]), device=DEV) - s["cu"][s["seq"]]
    return s["positions"] - row + depth[s["seq"], row]


def _rotate(s):
    c = s["case"]
    f, amplitude = _frequencies(c)
    angle = _depths(s).double()[:, None] * f                     # far positions: 64 bits
    cos, sin = ((fn(angle) * amplitude).float()[:, None] for fn in (torch.cos, torch.sin))
    for x, y in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
        r, half = c["rot"], c["rot"] // 2
        a, b = (x[..., :half], x[..., half:r]) if c["pairs"] == "half" else (x[..., 0:r:2], x[..., 1:r:2])
        a, b = a.float(), b.float()
        a, b = a * cos - b * sin, b * cos + a * sin
        y[..., :r] = torch.cat([a, b], 2) if c["pairs"] == "half" else torch.stack([a, b], 3).flatten(2)
        y[..., r:] = x[..., r:]
    return {"q": s["q_out"], "k": s["k_out"]}


def _on_path(s):
    """[B, R, N]: whether drafted token j stands before row r: on its path from the root."""
    B, R, N = s["case"]["B"], s["case"]["R"], s["drafted"].shape[1]
    if s["parent"] is None:
        return (torch.arange(N, device=DEV)[None] < torch.arange(R, device=DEV)[:, None]).expand(B, R, N)
    on = torch.zeros(B, R, R + N + 1, dtype=torch.bool, device=DEV)
    parent = torch.nn.functional.pad(s["parent"].long(), (1, 0))
    up = torch.arange(R, device=DEV).repeat(B, 1)
    for _ in range(R):
        on.scatter_(2, up[:, :, None], True)
        up = torch.where(up > 0, parent.gather(1, up.clamp(max=N)), 0)
    return on[:, :, 1:N + 1]


def _adjust(s):
    c = s["case"]
    B, R, V = s["logits"].shape
    x = s["logits"].to(torch.float32, copy=True)
    if c["pen"]:
        h = s["history"].int()
        count = (h >> 1)[:, None].repeat(1, R, 1)
        at = s["drafted"].long()[:, None].expand(B, R, -1)
        count.scatter_add_(2, at, _on_path(s).int())
        seen = (count > 0) | (h & 1).bool()[:, None]
        rep, pres, freq = (s[n][:, None, None] for n in ("rep", "pres", "freq"))
        x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
        x -= freq * count + pres * (count > 0)
    if c["bias"]:
        b = torch.repeat_interleave(torch.arange(B, device=DEV), s["begin"].diff().long())
        add = torch.zeros(B, V, dtype=torch.float64, device=DEV)   # a token listed twice: both count
        add.index_put_((b, s["bias_tokens"].long()), s["bias"].double(), accumulate=True)
        x += add.float()[:, None]
    if c["masks"]:
        m = s["mask_row"].long()
        bit = (s["masks"][:, :, None] >> torch.arange(32, dtype=torch.int32, device=DEV)) & 1
        allowed = bit.bool().flatten(1)[:, :V]
        x = x.masked_fill_(~(allowed[m.clamp(min=0)] | (m < 0)[..., None]), float("-inf"))
    rows = torch.arange(R, device=DEV)[None] < s["gamma"][:, None] + 1
    s["out"].copy_(torch.where(rows[..., None], x.to(s["out"].dtype), s["out"]))
    return s["out"]


def _history(s):
    h = s["history"]
    B, V = h.shape
    if s["fresh"] is not None:
        h.masked_fill_(s["fresh"].bool()[:, None], 0)
    flat = h.view(-1)
    if s["prompt"] is not None:
        at = torch.repeat_interleave(torch.arange(B, device=DEV), s["cu"].diff().long()) * V + s["prompt"].long()
        flat[at] = flat[at] | 1
    if s["tokens"] is not None:
        live = torch.arange(s["tokens"].shape[1], device=DEV)[None] < s["len"][:, None]
        at, times = torch.unique((torch.arange(B, device=DEV)[:, None] * V + s["tokens"])[live], return_counts=True)
        old = flat[at].int()
        flat[at] = (2 * ((old >> 1) + times).clamp(max=MOST) + (old & 1)).to(torch.int16)
    return h


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "attend":
        n, Hq, Hkv, d = _numbers(case["n"]), case["Hq"], case["Hkv"], case["d"]
        pairs = sum(k * (k + 1) // 2 for k in n)
        return {"bytes": 2 * sum(n) * d * (2 * Hq + 2 * Hkv), "flops": 4 * pairs * Hq * d}
    if op == "rotate":
        T, e = sum(_numbers(case["n"])), 2 if case["dtype"] == "bf16" else 4
        H = case["Hq"] + case["Hkv"]
        return {"bytes": T * (2 * H * case["d"] * e + 4), "flops": 3 * T * H * case["rot"]}
    B, V = case["B"], case["V"]
    if op == "adjust":
        e = 2 if case["dtype"] == "bf16" else 4
        rows = sum(g + 1 for g in _per_sequence(case, "gamma"))
        # in place a grammar mask alone writes what it forbids; else every row is read and written
        moved = rows * V * e * (0.57 if case["inplace"] else 2.0)
        bias = sum(case["bias"] * (b % 3) // 2 if B > 1 else case["bias"] for b in range(B))
        masked = min(rows * case["masks"] / (case["masks"] + 1), case["masks"]) if case["masks"] else 0
        return {"bytes": moved + (2 * B * V if case["pen"] else 0) + 8 * bias + masked * V / 8, "flops": 4 * rows * V if case["pen"] else 0}
    if case["n"]:                                                # a history that begins anew is written, not read
        return {"bytes": 2 * B * V + 4 * sum(_per_sequence(case, "n")) + 4 * B * case["W"], "flops": 0}
    return {"bytes": B * (4 + 8 * (case["W"] + 1) / 2), "flops": 0}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _exact_attend(case, s):
    G, start = case["Hq"] // case["Hkv"], 0
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for n in s["n"]:
        for h in range(case["Hq"]):
            q, k, v = (s[x][start:start + n, h if x == "q" else h // G].double() for x in ("q", "k", "v"))
            for i in range(0, n, 4096):
                e = min(n, i + 4096)
                t = torch.ones(e - i, e, dtype=torch.bool, device=DEV).tril(i)
                t = torch.where(t, (q[i:e] @ k[:e].T) * s["scale"], float("-inf"))
                out[start + i:start + e, h] = torch.softmax(t, 1) @ v[:e]
        start += n
    return out


def _exact_rotate(case, s):
    rot, w, kind = case["rot"], SCALINGS[case["scaling"]], case["scaling"]
    freq, amplitude = [], 1.0
    for i in range(rot // 2):
        f = math.exp(-2.0 * i / rot * math.log(BASE))
        if kind == "linear":
            f /= w["factor"]
        elif kind == "bands":
            wave = 2 * math.pi / f
            if wave > w["original"] / w["low"]:
                f /= w["factor"]
            elif wave >= w["original"] / w["high"]:
                u = (w["original"] / wave - w["low"]) / (w["high"] - w["low"])
                f = (1 - u) * f / w["factor"] + u * f
        elif kind == "yarn":
            turns = lambda r: rot * math.log(w["original"] / (r * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
            a, b = max(math.floor(turns(w["high"])), 0), min(math.ceil(turns(w["low"])), rot - 1)
            u = min(max((i - a) / max(b - a, 0.001), 0.0), 1.0)
            f = f / w["factor"] * u + f * (1 - u)
            amplitude = 0.1 * math.log(w["factor"]) + 1.0
        freq.append(f)
    at = []
    for n, c in zip(_numbers(case["n"]), _ctx(case, len(_numbers(case["n"])))):
        depth = [0]
        for p in _parents(case["tree"], n):
            depth.append(depth[p] + 1)
        at += [c + x for x in depth]
    turn = torch.polar(torch.full((len(at), rot // 2), amplitude, dtype=torch.float64, device=DEV),
                       torch.outer(torch.tensor(at, dtype=torch.float64, device=DEV), torch.tensor(freq, dtype=torch.float64, device=DEV)))[:, None]
    out = {}
    for n in ("q", "k"):
        y = s[n].double().clone()
        one, two = (slice(0, rot // 2), slice(rot // 2, rot)) if case["pairs"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(y[..., one].contiguous(), y[..., two].contiguous()) * turn
        y[..., one], y[..., two] = z.real, z.imag
        out[n] = y
    return out


def _exact_adjust(case, s):
    V, begin = case["V"], s["begin"].tolist() if case["bias"] else None
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV) if not case["inplace"] else s["logits"].double()
    drafted = s["drafted"].tolist()
    shift = torch.arange(32, dtype=torch.int64, device=DEV)
    allowed = [None] * case["masks"]
    for m in range(case["masks"]):
        allowed[m] = ((s["masks"][m].long()[:, None] >> shift) % 2 == 1).flatten()[:V]
    chosen = s["mask_row"].tolist() if case["masks"] else None
    for b, g in enumerate(_per_sequence(case, "gamma")):
        parent = _parents(case["tree"], case["R"])
        for r in range(g + 1):
            x = s["logits"][b, r].double()
            if case["pen"]:
                count = (s["history"][b] // 2).double()
                node = r
                while node > 0:
                    count[drafted[b][node - 1]] += 1
                    node = parent[node - 1]
                known = (count > 0) | (s["history"][b] % 2 == 1)
                rep = s["rep"][b].double()
                x = torch.where(known, torch.where(x > 0, x / rep, x * rep), x)
                x = x - s["freq"][b].double() * count - s["pres"][b].double() * (count > 0).double()
            if case["bias"]:
                lo, hi = begin[b], begin[b + 1]
                x.index_add_(0, s["bias_tokens"][lo:hi].long(), s["bias"][lo:hi].double())
            if case["masks"] and chosen[b][r] >= 0:
                x = torch.where(allowed[chosen[b][r]], x, float("-inf"))
            out[b, r] = x
    return out


def exact(case, seed):
    if case["op"] == "history":
        return None                                              # no computed numbers among its outputs
    s = prepare(case, seed)
    return {"attend": _exact_attend, "rotate": _exact_rotate, "adjust": _exact_adjust}[case["op"]](case, s)
