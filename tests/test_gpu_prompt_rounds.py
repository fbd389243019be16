"""The calls together, as a serving loop makes them: prompts enter (plan, rotate, attend, cache, history), then rounds of chains and of
trees (plan, rotate, cache, attend; adjust, verify, keep, history) -- against the same model written out in 64 bits over whole
sequences, without a cache, and as one captured graph."""
import numpy as np
import pytest
import torch

from oracle import logits as ol
from oracle import prompt as op

pytestmark = pytest.mark.gpu
DEV = "cuda"
Hq, Hkv, d, V, bt, E = 8, 2, 64, 1000, 16, 96


def _ints(v):
    return torch.tensor(np.asarray(v).tolist(), dtype=torch.int32, device=DEV)


class Model:
    """One attention layer between an embedding and an output matrix: enough that every token looks back at all others."""

    def __init__(self, lib, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.lib = lib
        self.embed = torch.randn(V, E, generator=g, device=DEV)
        self.qkv = torch.randn(E, (Hq + 2 * Hkv) * d, generator=g, device=DEV) / E ** 0.5
        self.head = torch.randn(Hq * d, V, generator=g, device=DEV) / 2
        self.table = lib.new_rotary_table(d, 10000.0, "bands", factor=4.0, low=1.0, high=4.0, original=64, device=DEV)

    def project(self, tokens):
        x = (self.embed[tokens.long()] @ self.qkv).to(torch.bfloat16).view(-1, Hq + 2 * Hkv, d)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]

    def logits(self, att):
        return att.float().reshape(len(att), -1) @ self.head

    def exact(self, tokens, positions, see):
        """Logits in fp64 of every token of one sequence; see [n, n]: what a token looks at."""
        q, k, v = (x.double().cpu().numpy() for x in self.project(torch.tensor(tokens, device=DEV)))
        f, amp = op.frequencies(d, 10000.0, "bands", 4.0, 1.0, 4.0, 64)
        q, k = op.rotate(q, positions, f, amp, False), op.rotate(k, positions, f, amp, False)
        out = np.zeros(q.shape)
        for h in range(Hq):
            s = np.where(see, q[:, h] @ k[:, h // (Hq // Hkv)].T * d ** -0.5, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            out[:, h] = p / p.sum(1, keepdims=True) @ v[:, h // (Hq // Hkv)]
        return out.reshape(len(tokens), -1) @ self.head.double().cpu().numpy()


class Loop:
    """Buffers of a batch and the calls of a prompt and of a round."""

    def __init__(self, lib, model, prompts, N):
        B = len(prompts)
        self.lib, self.m, self.B, self.N = lib, model, B, N
        nb = 64
        (self.kc, self.ks), (self.vc, self.vs) = lib.new_cache(nb, Hkv, bt, d, DEV), lib.new_cache(nb, Hkv, bt, d, DEV)
        self.table, self.free, self.n_free = torch.full((B, 16), -1, dtype=torch.int32, device=DEV), torch.arange(nb, dtype=torch.int32, device=DEV), _ints([nb])
        self.seq, self.held, self.kv = _ints([0] * B), _ints([0] * B), _ints([0] * B)
        self.cu, self.status = _ints([0] * (B + 1)), _ints([0] * B)
        self.hist, self.ws = lib.new_history(B, V, DEV), lib.new_cache_workspace(Hq, Hkv, d, DEV)
        self.kept = None

    def plan(self, new, T):
        slots, pos = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(T, dtype=torch.int32, device=DEV)
        self.lib.bs_cache_plan(self.seq, self.kept, new, 0, None, bt, self.table, self.held, self.free, self.n_free, self.kv, self.cu, slots, pos, self.status,
                               last_cu=self.cu if self.kept is not None else None)
        return slots, pos

    def prompts(self, prompts):
        lens = [len(x) for x in prompts]
        flat = _ints(sum(prompts, []))
        slots, pos = self.plan(_ints(lens), sum(lens))
        q, k, v = self.m.project(flat)
        self.lib.bs_rotary(q, k, pos, self.m.table, False, q, k)             # in place, in the fused projection
        att = torch.zeros(len(flat), Hq, d, dtype=torch.bfloat16, device=DEV)
        self.lib.bs_prompt_attention(q, k, v, self.cu, d ** -0.5, att, self.status)
        self.lib.bs_cache_append(k, v, slots, self.kc, self.ks, self.vc, self.vs)
        self.lib.bs_history_update(self.hist, torch.ones(self.B, dtype=torch.uint8, device=DEV), self.cu, flat, status=self.status)
        self.kept = _ints(lens)
        return self.m.logits(att)

    def rows(self, tokens, new, parent):
        """Logits [B, N + 1, V] of the pending token and the drafts; tokens [B, N + 1]."""
        T = self.B * (self.N + 1)
        slots, pos = self.plan(new, T)
        q, k, v = self.m.project(tokens.reshape(-1))
        trees = {} if parent is None else {"cu_new": self.cu, "node_parent": parent}
        self.lib.bs_rotary(q, k, pos, self.m.table, False, q, k, **trees)
        self.lib.bs_cache_append(k, v, slots, self.kc, self.ks, self.vc, self.vs)
        att = torch.empty(T, Hq, d, dtype=torch.bfloat16, device=DEV)
        self.lib.bs_cache_attention(q, self.cu, self.kv, self.table, parent, self.kc, self.ks, self.vc, self.vs, self.N + 1, d ** -0.5, att, self.status, self.ws)
        return self.m.logits(att).view(self.B, self.N + 1, V)


def _prompts(rng):
    return [rng.integers(0, V, n).tolist() for n in (37, 130, 1)]


def _near(got, want, share):
    """The cache holds e4m3 codes (2^-4 relative each, of keys and values), so logits follow to a share of their spread."""
    assert np.abs(got - want).max() <= share * want.std() * 6, np.abs(got - want).max() / want.std()


def test_prompts_then_rounds_of_chains(lib):
    rng = np.random.default_rng(5)
    m, prompts, N = Model(lib), _prompts(rng), 3
    loop = Loop(lib, m, prompts, N)
    out = loop.prompts(prompts).double().cpu().numpy()
    at = 0
    for p in prompts:
        want = m.exact(p, range(len(p)), np.tril(np.ones((len(p), len(p)), bool)))
        _near(out[at:at + len(p)], want, 0.02)                # bf16 alone
        at += len(p)
    assert not loop.status.any()
    texts = [list(p) for p in prompts]                        # what is in the cache
    pending = rng.integers(0, V, 3)
    emitted = [[] for _ in prompts]
    rep, pres, freq = (torch.full((3,), x, device=DEV) for x in (1.3, 0.4, 0.2))
    vws = lib.new_workspace(3, N, V, DEV)
    for rnd in range(3):
        drafts = rng.integers(0, V, (3, N))
        drafts[0, 1] = drafts[0, 0]                           # drafted twice on the way
        gamma = _ints([3, 3, 3])
        rows = loop.rows(_ints(np.concatenate([pending[:, None], drafts], 1)), _ints([N + 1] * 3), None)
        raw = rows.clone()
        # the pending token was emitted by the round before and is in the history; drafts count along their chain
        lib.bs_history_update(loop.hist, out_tokens=_ints(pending[:, None]), out_len=_ints([1] * 3))
        for b in range(3):
            emitted[b].append(int(pending[b]))
        lib.bs_logits_adjust(rows, rows, gamma, 1, draft_tokens=_ints(drafts), history=loop.hist, repetition=rep, presence=pres, frequency=freq, status=loop.status)
        acc, ol_, ot = _ints([0] * 3), _ints([0] * 3), _ints(np.zeros((3, N + 1)))
        lib.bs_softmax_verify(rows, None, _ints(drafts), gamma, None, 0.0, acc, None, None, vws)
        lib.bs_residual_sample(rows, None, _ints(drafts), gamma, acc, None, 0.0, ot, ol_, vws)
        tau, toks = acc.tolist(), ot.tolist()
        for b in range(3):
            seq = texts[b] + [int(pending[b])] + drafts[b].tolist()
            want = m.exact(seq, range(len(seq)), np.tril(np.ones((len(seq), len(seq)), bool)))[len(texts[b]):]
            _near(raw[b].double().cpu().numpy(), want, 0.1)
            h = ol.enter(np.zeros((1, V)), prompts=[prompts[b]], emitted=[emitted[b]])[0]
            best = []
            for r in range(N + 1):
                w = ol.adjust_row(raw[b, r].cpu().numpy(), h, drafts[b, :r].tolist(), float(rep[b]), float(pres[b]), float(freq[b]))
                assert np.abs(rows[b, r].double().cpu().numpy() - w).max() < 1e-4
                best.append(int(np.argmax(rows[b, r].cpu().numpy())))
            t = 0
            while t < N and drafts[b, t] == best[t]:
                t += 1
            assert tau[b] == t and toks[b][:t + 1] == drafts[b, :t].tolist() + [best[t]]
            texts[b] += [int(pending[b])] + drafts[b, :t].tolist()
            emitted[b] += drafts[b, :t].tolist()
            pending[b] = best[t]
        if max(tau):
            lib.bs_history_update(loop.hist, out_tokens=_ints(drafts), out_len=acc)
        loop.kept = ol_.clone()
    assert not loop.status.any()


def test_a_round_of_trees_keeps_keys_at_their_angles(lib):
    """Keys of a tree are rotated by depth, so the accepted path can move to the front as it is: the next round sees the text."""
    rng = np.random.default_rng(8)
    m, prompts, N = Model(lib, 1), _prompts(rng), 6
    loop = Loop(lib, m, prompts, N)
    loop.prompts(prompts)
    parent = [0, 0, 1, 1, 2, 4]                               # of nodes 1 to 6
    par = _ints([parent] * 3)
    tree = rng.integers(0, V, (3, N + 1))
    rows = loop.rows(_ints(tree), _ints([N + 1] * 3), par)
    see = np.zeros((N + 1, N + 1), bool)
    for n in range(N + 1):
        see[n, [0] + ol.path(parent, n)] = True
    for b, p in enumerate(prompts):
        L = len(p)
        mask = np.zeros((L + N + 1,) * 2, bool)
        mask[:L, :L] = np.tril(np.ones((L, L), bool))
        mask[L:, :L], mask[L:, L:] = True, see
        want = m.exact(p + tree[b].tolist(), list(range(L)) + [L + op.depth(parent, n) for n in range(N + 1)], mask)[L:]
        _near(rows[b].double().cpu().numpy(), want, 0.1)
    # the path 1, 4, 6 of sequence 0, 2, 5 of sequence 1, nothing of sequence 2
    nodes, tau = _ints([[1, 4, 6, -1, -1, -1], [2, 5, -1, -1, -1, -1], [-1] * 6]), _ints([3, 2, 0])
    lib.bs_cache_keep_path(nodes, tau, loop.seq, loop.table, loop.kc, loop.ks, loop.vc, loop.vs, loop.status)
    loop.kept = _ints([4, 3, 1])
    texts = [prompts[0] + tree[0, [0, 1, 4, 6]].tolist(), prompts[1] + tree[1, [0, 2, 5]].tolist(), prompts[2] + tree[2, [0]].tolist()]
    nxt = rng.integers(0, V, (3, N + 1))
    rows = loop.rows(_ints(nxt), _ints([N + 1] * 3), None)
    for b, p in enumerate(texts):
        seq = p + nxt[b].tolist()
        want = m.exact(seq, range(len(seq)), np.tril(np.ones((len(seq),) * 2, bool)))[len(p):]
        _near(rows[b].double().cpu().numpy(), want, 0.1)
    # rows of a tree: the penalties follow the path
    raw, f = rows.clone(), torch.full((3,), 0.5, device=DEV)
    lib.bs_logits_adjust(rows, rows, _ints([N, 2, 0]), 1, draft_tokens=_ints(tree[:, 1:]), node_parent=par, history=loop.hist, frequency=f, status=loop.status)
    for b in range(3):
        h = ol.enter(np.zeros((1, V)), prompts=[prompts[b]])[0]
        for n in range(N + 1):
            w = raw[b, n].double().cpu().numpy()
            if n <= [N, 2, 0][b]:
                w = ol.adjust_row(w, h, tree[b, ol.path(parent, n)].tolist(), f=0.5)
            assert np.abs(rows[b, n].double().cpu().numpy() - w).max() < 1e-4
    assert not loop.status.any()


def test_a_captured_prompt_is_replayed(lib):
    rng = np.random.default_rng(2)
    m, prompts = Model(lib, 2), _prompts(rng)
    loop = Loop(lib, m, prompts, 1)
    want = loop.prompts(prompts)
    lens, flat = _ints([len(p) for p in prompts]), _ints(sum(prompts, []))
    q0, k0, v0 = m.project(flat)
    pos, cu = torch.cat([torch.arange(len(p), device=DEV) for p in prompts]).to(torch.int32), loop.cu.clone()
    q, k, att = torch.empty_like(q0), torch.empty_like(k0), torch.zeros(len(flat), Hq, d, dtype=torch.bfloat16, device=DEV)
    hist, fresh = lib.new_history(3, V, DEV), torch.ones(3, dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.bs_rotary(q0, k0, pos, m.table, False, q, k)
        lib.bs_prompt_attention(q, k, v0, cu, d ** -0.5, att)
        lib.bs_history_update(hist, fresh, cu, flat)
    for _ in range(2):
        att.zero_()
        hist.fill_(9)
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(m.logits(att), want) and torch.equal(hist, loop.hist) and int(lens.sum()) == len(flat)
