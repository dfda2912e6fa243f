"""Performance cases of sampling the responses of packed groups: a paged cache of keys and values whose prompt pages a group's
K responses share, attention of new tokens (one a sequence, or a tree of drafted ones) over it, and the verification of
drafted tokens that says which of them stay.

A rollout writes its prompts into pages, forks each prompt into K sequences, and then, step by step, makes room for the next
tokens, per layer writes their keys and values and attends, once per step verifies the drafts and keeps the accepted ones; at
the end it frees the sequences and moves what is left to the front of the pool.  The sizes are those of workload.py's batches
or generic.

listed() gives the cases, draw(rng) more of the same ranges; prepare makes a case's inputs, run does one pass (in elementary
torch operations, or with the library where `own` is set), exact the same in 64 bits from the definitions.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"


# ---------------------------------------------------------------- cases


def _tree(name, dtype, heads, d, groups, k, prompt, resp, nodes, page, width=1, ragged=False, len_seed=1):
    """Attention of `nodes` tokens of each of groups * k sequences; a group's sequences share the whole pages of a prompt."""
    c = {"kind": "tree", "dtype": dtype, "hq": heads[0], "hkv": heads[1], "d": d, "groups": groups, "k": k, "p_lo": prompt[0],
         "p_hi": prompt[1], "r_lo": resp[0], "r_hi": resp[1], "nodes": nodes, "page": page, "width": width, "ragged": ragged,
         "len_seed": len_seed}
    if name:
        c["name"] = name
    return c


def _append(name, kind, dtype, heads, d, seqs, held, new, page, layers=1, width=1, base=500000.0, len_seed=1):
    """kind "prompts": `new` tokens of each sequence are written behind `held` others; "step": a tree of `new` drafted tokens
    is written in every layer, and the accepted ones are kept."""
    c = {"kind": kind, "dtype": dtype, "hq": heads[0], "hkv": heads[1], "d": d, "seqs": seqs, "p_lo": held[0], "p_hi": held[1],
         "n_lo": new[0], "n_hi": new[1], "page": page, "layers": layers, "width": width, "base": base, "len_seed": len_seed}
    if name:
        c["name"] = name
    return c


def _pages(name, kind, dtype, hkv, d, groups, k, prompt, page, layers, add=0, len_seed=1):
    """kind "fork": prompts are forked into k sequences each, with room for `add` tokens; "compact": forks, frees and moves."""
    c = {"kind": kind, "dtype": dtype, "hkv": hkv, "d": d, "groups": groups, "k": k, "p_lo": prompt[0], "p_hi": prompt[1],
         "page": page, "layers": layers, "add": add, "len_seed": len_seed}
    if name:
        c["name"] = name
    return c


def _verify(name, dtype, vocab, seqs, nodes, width=1, draft=True, greedy=0, ragged=False, hidden_vocab=0, len_seed=1):
    c = {"kind": "verify", "dtype": dtype, "vocab": vocab, "seqs": seqs, "nodes": nodes, "width": width, "draft": draft,
         "greedy": greedy, "ragged": ragged, "hidden_vocab": hidden_vocab, "len_seed": len_seed}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # plain sampling of eight sequences, one new token each (latency counts)
        _tree("tree_one_token", "bf16", (32, 8), 128, 8, 1, (300, 1601), (0, 0), 1, 16),
        # a rollout's decode step: 16 prompts of the 8B-shaped model with eight responses each, one new token each
        _tree("tree_group_decode", "bf16", (32, 8), 128, 16, 8, (1024, 6144), (1, 512), 1, 64),
        # few sequences with long caches, trees of 16 drafted tokens, 72B-shaped heads
        _tree("tree_drafts_long", "bf16", (64, 8), 128, 4, 1, (16000, 48000), (0, 0), 16, 32, width=3),
        # the largest: trees of eight drafted tokens for eight responses of each of 16 long prompts, some sequences finished
        _tree("tree_drafts_group", "bf16", (32, 8), 128, 16, 8, (2048, 6144), (64, 512), 8, 64, width=2, ragged=True),
        # the toy model in fp32, ragged trees
        _tree("tree_tiny_fp32", "fp32", (4, 4), 64, 4, 2, (64, 128), (1, 64), 5, 16, width=2, ragged=True),
        # a step of drafted trees in four layers of a small model: rotate and write every node, then keep the accepted ones
        _append("step_drafts_d64", "step", "bf16", (14, 2), 64, 24, (17, 900), (2, 8), 16, layers=4, width=2, base=1e6),
        # the prompts of an 8B-shaped batch go into their pages, rotated with their queries
        _append("append_prompts_8b", "prompts", "bf16", (32, 8), 128, 8, (0, 0), (256, 1536), 64),
        # one prompt becomes a group: copies of its last page in every layer, and room for the first tokens
        _pages("fork_one_group", "fork", "bf16", 8, 128, 1, 8, (256, 1536), 16, 8, add=8),
        # a rollout's start: 32 prompts become 256 sequences
        _pages("fork_rollout", "fork", "bf16", 8, 128, 32, 8, (256, 1536), 64, 4, add=64),
        # sequences leave and others come, and twice the pool's live pages move to its front
        _pages("compact_rollout", "compact", "bf16", 8, 128, 16, 8, (256, 1536), 64, 4),
        # chains of four drafted tokens against a large vocabulary, a quarter of the sequences greedy
        _verify("verify_chain_128k", "bf16", 128256, 32, 5, greedy=4),
        # trees with siblings against the 72B-shaped vocabulary, ragged
        _verify("verify_tree_152k", "bf16", 152064, 8, 24, width=3, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    a, b = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
    return min(a, b), max(a, b)


_HEADS = [((32, 8), 128), ((64, 8), 128), ((28, 4), 128), ((16, 4), 64), ((14, 2), 64), ((8, 8), 64), ((12, 12), 128), ((8, 1), 64)]


def _cost(case):
    w = work(case)
    return w["flops"] / 1e12 + w["bytes"] / 5e9  # about ms


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree_long", "step", "prompts", "fork", "compact", "verify", "verify"])
    seed, page = rng.randint(2, 1 << 30), rng.choice([16, 32, 64, 128, 256])
    heads, d = rng.choice(_HEADS)
    dtype = rng.choice(["bf16"] * 4 + ["fp32"])
    if kind.startswith("tree"):
        nodes = rng.choice([1, 1, 2, rng.randint(1, 64), rng.randint(1, 16)])
        if kind == "tree":
            groups, k, prompt = _log_int(rng, 1, 24), rng.choice([1, 2, 4, 8, rng.randint(1, 16)]), _span(rng, 1, 6144)
        else:
            groups, k, prompt = _log_int(rng, 1, 6), 1, _span(rng, 2000, 48000)
        case = _tree("", dtype, heads, d, groups, k, prompt, (0, 0) if rng.random() < 0.3 else _span(rng, 1, 512), nodes, page,
                     rng.randint(1, 4), rng.random() < 0.5, seed)
        many, most = "groups", "tree_drafts_group"
    elif kind in ("step", "prompts"):
        step = kind == "step"
        case = _append("", kind, dtype, heads, d, _log_int(rng, 1, 64), (0, 0) if rng.random() < 0.3 else _span(rng, 1, 4000),
                       _span(rng, 1, 32) if step else _span(rng, 1, 1536), page, rng.randint(1, 4) if step else 1,
                       rng.randint(1, 3) if step else 1, rng.choice([0.0, 10000.0, 500000.0, 1e6]), seed)
        many, most = "seqs", "append_prompts_8b"
    elif kind in ("fork", "compact"):
        case = _pages("", kind, dtype, heads[1], d, _log_int(rng, 1, 32), rng.randint(1, 12), _span(rng, 1, 2000), page,
                      rng.randint(1, 8), rng.choice([0, 1, 64, 200]) if kind == "fork" else 0, seed)
        many, most = "groups", "fork_rollout" if kind == "fork" else "compact_rollout"
    else:
        vocab = rng.choice([128256, 152064, 32000, rng.randint(200, 152064)])
        nodes = rng.choice([1, rng.randint(2, 8), rng.randint(2, 32)])
        case = _verify("", dtype, vocab, _log_int(rng, 1, 64), nodes, rng.randint(1, 3), rng.random() < 0.7,
                       rng.choice([0, 0, 1, 3]), rng.random() < 0.5, rng.choice([0, 0, 80]), seed)
        many, most = "seqs", "verify_tree_152k"
    most = _cost(next(c for c in listed() if c["name"] == most))
    while case[many] > 1 and _cost(case) > most:
        case[many] = max(1, case[many] // 2)
    for lo, hi in (("p_lo", "p_hi"), ("n_lo", "n_hi")):
        while hi in case and case[hi] > 1 and _cost(case) > most:
            case[lo], case[hi] = max(1, case[lo] // 2), max(1, case[hi] // 2)
    return case


# ---------------------------------------------------------------- layouts


def _rng(case):
    return np.random.default_rng([2602, 24082, 8, case["len_seed"]])


def _parents(rng, n, width):
    """A tree of n nodes: node 0 is its root, a node has at most `width` children."""
    par, kids = [-1], [0]
    for i in range(1, n):
        free = [j for j in range(i) if kids[j] < width]
        j = free[-1] if width == 1 or rng.random() < 0.5 else int(rng.choice(free))
        par.append(j)
        kids[j] += 1
        kids.append(0)
    return par


def _ceil(a, b):
    return -(-a // b)


class _TreeLayout:
    def __init__(self, case):
        rng, G, K, N, ps = _rng(case), case["groups"], case["k"], case["nodes"], case["page"]
        self.n, self.N = G * K, N
        P = rng.integers(case["p_lo"], case["p_hi"], size=G, endpoint=True).tolist()
        R = rng.integers(case["r_lo"], case["r_hi"], size=self.n, endpoint=True).tolist()
        self.len = [P[i // K] + R[i] for i in range(self.n)]
        self.count = rng.integers(0, N, size=self.n, endpoint=True).tolist() if case["ragged"] else [N] * self.n
        self.count[0] = max(1, self.count[0])
        self.par = [_parents(rng, N, case["width"]) for _ in range(self.n)]
        self.shared = [p // ps if K > 1 else 0 for p in P]  # whole pages of the prompt
        self.held = [_ceil(self.len[i] + self.count[i], ps) for i in range(self.n)]
        self.columns = max(1, max(self.held))
        own_pages = [self.held[i] - self.shared[i // K] for i in range(self.n)]
        self.pages = max(1, sum(own_pages) + sum(self.shared)) + 3
        order = rng.permutation(self.pages).tolist()
        self.slot = rng.permutation(self.n + 2)[:self.n].tolist()
        self.table = np.full((self.n + 2, self.columns), -1, np.int32)
        take = lambda m: [order.pop() for _ in range(m)]
        for g in range(G):
            first = take(self.shared[g])
            for i in range(g * K, (g + 1) * K):
                self.table[self.slot[i], :self.held[i]] = first + take(own_pages[i])


class _AppendLayout:
    def __init__(self, case):
        rng, n, ps = _rng(case), case["seqs"], case["page"]
        self.n = n
        self.len = rng.integers(case["p_lo"], case["p_hi"], size=n, endpoint=True).tolist()
        self.count = rng.integers(case["n_lo"], case["n_hi"], size=n, endpoint=True).tolist()
        self.N = max(self.count)
        step = case["kind"] == "step"
        self.start = [i * self.N for i in range(n)] if step else np.concatenate([[0], np.cumsum(self.count)])[:-1].tolist()
        self.rows = n * self.N if step else sum(self.count)
        self.par = [_parents(rng, self.N, case["width"]) for _ in range(n)]
        self.path, self.keep = np.full((n, self.N), -1, np.int32), []
        for i in range(n):  # the accepted nodes: a walk from the root
            at, walk = 0, [0]
            while True:
                kids = [j for j in range(at + 1, self.count[i]) if self.par[i][j] == at]
                if not kids or rng.random() < 0.25:
                    break
                at = int(rng.choice(kids))
                walk.append(at)
            self.path[i, :len(walk)] = walk
            self.keep.append(len(walk))
        self.held = [_ceil(a + b, ps) for a, b in zip(self.len, self.count)]
        self.columns, self.pages = max(self.held), sum(self.held) + 3
        order = rng.permutation(self.pages).tolist()
        self.slot = rng.permutation(n + 2)[:n].tolist()
        self.table = np.full((n + 2, self.columns), -1, np.int32)
        for i in range(n):
            self.table[self.slot[i], :self.held[i]] = [order.pop() for _ in range(self.held[i])]


class _PagesLayout:
    """Slots: prompts first, then K children of each, and for "compact" K more."""

    def __init__(self, case):
        rng, G, K, ps = _rng(case), case["groups"], case["k"], case["page"]
        self.P = rng.integers(case["p_lo"], case["p_hi"], size=G, endpoint=True).tolist()
        self.src = [g for g in range(G) for _ in range(K)]
        sets = 2 if case["kind"] == "compact" else 1
        self.dst = [[G + s * G * K + i for i in range(G * K)] for s in range(sets)]
        self.slots = G + sets * G * K
        self.held = [_ceil(p, ps) for p in self.P]
        self.columns = max(_ceil(p + case["add"], ps) for p in self.P)
        per = max(1, 1 + _ceil(case["add"], ps))
        self.pages = sum(self.held) + sets * G * K * per + 5
        order = rng.permutation(self.pages).tolist()
        self.table = np.full((self.slots, self.columns), -1, np.int32)
        for g in range(G):
            self.table[g, :self.held[g]] = [order.pop() for _ in range(self.held[g])]


class _VerifyLayout:
    def __init__(self, case):
        rng, n, N = _rng(case), case["seqs"], case["nodes"]
        self.n, self.N = n, N
        self.count = rng.integers(0, N, size=n, endpoint=True).tolist() if case["ragged"] else [N] * n
        self.count[0] = max(1, self.count[0])
        self.par = [_parents(rng, N, case["width"]) for _ in range(n)]
        self.temp = [0.0 if case["greedy"] and i % case["greedy"] == 0 else t
                     for i, t in enumerate(rng.choice([1.0, 0.7, 1.25], size=n).tolist())]

    def children(self, i):
        kids = [[] for _ in range(self.N)]
        for j in range(1, self.count[i]):
            kids[self.par[i][j]].append(j)
        return kids


def _layout(case):
    kind = case["kind"]
    return {"tree": _TreeLayout, "step": _AppendLayout, "prompts": _AppendLayout, "fork": _PagesLayout, "compact": _PagesLayout,
            "verify": _VerifyLayout}[kind](case)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(shape, seed, dtype, sigma=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    out = torch.empty(shape, dtype=dtype, device=DEV)
    step = max(1, (1 << 28) // max(1, int(np.prod(shape[1:]))))
    for r in range(0, shape[0], step):
        out[r:r + step] = torch.randn((min(step, shape[0] - r), *shape[1:]), generator=g, device=DEV).mul_(sigma)
    return out


def _ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _put_cache(st, table, length, held, pages, page, slots):
    """The cache's bookkeeping: table, lengths, pages held and how often each page is listed."""
    full = np.zeros((2, table.shape[0]), np.int32)
    full[0, slots], full[1, slots] = length, held
    refs = np.bincount(np.concatenate([table[s, :h] for s, h in zip(slots, held)] + [np.zeros(0, np.int64)]).astype(np.int64),
                       minlength=pages)
    st.update(table=_ints(table), len=_ints(full[0]), held=_ints(full[1]), refs=_ints(refs))
    if own:
        from paper_2602_24082_amd import binding as pp
        st["cache"] = pp.Cache(st["table"], st["len"], st["held"], st["refs"], page)


def prepare(case, seed):
    L, dt, s = _layout(case), _dtype(case), seed * 1000 + 31
    kind = case["kind"]
    st = {"case": case, "layout": L}
    if kind == "verify":
        return _prepare_verify(st, case, L, dt, s)
    hkv, d, ps = case["hkv"], case["d"], case["page"]
    if kind in ("fork", "compact"):
        _put_cache(st, L.table, L.P, L.held, L.pages, ps, list(range(len(L.P))))
        st["k"] = _randn((case["layers"], L.pages, hkv, ps, d), s, dt)
        st["v"] = _randn((case["layers"], L.pages, hkv, ps, d), s + 1, dt)
        st["src"], st["dst"] = _ints(L.src), [_ints(x) for x in L.dst]
        st["add"] = torch.full((len(L.src),), case["add"], dtype=torch.int32, device=DEV)
        if kind == "compact":
            _plain_fork(st, st["src"], st["dst"][0])
        return st
    _put_cache(st, L.table, L.len, L.held, L.pages, ps, L.slot)
    hq = case["hq"]
    st["slots"], st["count"], st["parents"] = _ints(L.slot), _ints(L.count), _ints(L.par)
    if kind == "tree":
        st["k"], st["v"] = _randn((L.pages, hkv, ps, d), s, dt), _randn((L.pages, hkv, ps, d), s + 1, dt)
        st["q"] = _randn((L.n, L.N, hq, d), s + 2, dt)
        st["shared"] = _ints(L.shared)
        return st
    st["k"] = _randn((case["layers"], L.pages, hkv, ps, d), s, dt)
    st["v"] = _randn((case["layers"], L.pages, hkv, ps, d), s + 1, dt)
    st["new"] = [tuple(_randn((L.rows, h, d), s + 10 * (i + 1) + j, dt) for j, h in enumerate((hkv, hkv, hq)))
                 for i in range(case["layers"])]
    st["start"] = _ints(L.start)
    st["path"], st["keep"], st["len0"] = _ints(L.path), _ints(L.keep), st["len"].clone()
    return st


def _prepare_verify(st, case, L, dt, s):
    """Logits of a model and of a drafter that is close to it; the drafts are sampled from the drafter's distributions (from the
    model's where there is no drafter)."""
    n, N, V = L.n, L.N, case["vocab"]
    g = torch.Generator(device=DEV)
    g.manual_seed(s)
    st["count"], st["parents"] = _ints(L.count), _ints(L.par)
    st["temp"] = torch.tensor(L.temp, dtype=torch.float32, device=DEV)
    st["u"] = torch.rand((n, N), generator=g, device=DEV)
    st["target"] = _randn((n, N, V), s + 1, dt, 3.0)
    seen = V - case["hidden_vocab"]
    st["target"][:, :, seen:] = -math.inf
    st["draft"] = None
    if case["draft"]:
        st["draft"] = (st["target"].float() + _randn((n, N, V), s + 2, dt, 0.8).float()).to(dt)
    tokens = torch.zeros((n, N), dtype=torch.int64, device=DEV)
    for i in range(n if N > 1 else 0):
        rows = (st["target"] if st["draft"] is None else st["draft"])[i].float() / (L.temp[i] or 1.0)
        p = torch.softmax(rows, dim=1)[torch.tensor(L.par[i][1:], device=DEV)]
        tokens[i, 1:] = torch.multinomial(p, 1, generator=g)[:, 0]
    st["tokens"] = tokens.to(torch.int32)
    return st


# ---------------------------------------------------------------- one pass


def run(st):
    kind = st["case"]["kind"]
    if own:
        return _run_own(st, kind)
    return {"tree": _plain_tree, "step": _plain_step, "prompts": _plain_prompts, "fork": _plain_fork_pass,
            "compact": _plain_compact_pass, "verify": _plain_verify}[kind](st)


def _pages_out(st):
    return {"table": st["table"], "len": st["len"], "held": st["held"], "refs": st["refs"], "k": st["k"], "v": st["v"]}


def _run_own(st, kind):
    from paper_2602_24082_amd import binding as pp
    case = st["case"]
    if kind == "tree":
        o, lse = pp.pp_tree_attn_fwd(st["cache"], st["slots"], st["q"], st["k"], st["v"], parents=st["parents"], count=st["count"],
                                     group=case["k"], shared=st["shared"])
        return {"o": o, "lse": lse}
    if kind == "verify":
        count, tokens, path, logp = pp.pp_verify_draft(st["target"], st["tokens"], st["u"], draft=st["draft"],
                                                       parents=st["parents"], count=st["count"], temperature=st["temp"],
                                                       max_children=case["width"])
        return {"count": count, "tokens": tokens, "path": path, "logp": logp}
    c, out = st["cache"], {}
    if kind == "prompts":
        k, v, q = st["new"][0]
        out["q"] = pp.pp_cache_append(c, st["slots"], k, v, st["k"][0], st["v"][0], count=st["count"], start=st["start"],
                                      max_new=st["layout"].N, q=q, rope_base=case["base"])
        out.update(k=st["k"], v=st["v"])
        return out
    if kind == "step":
        st["len"].copy_(st["len0"])
        for i, (k, v, q) in enumerate(st["new"]):
            out["q%d" % i] = pp.pp_cache_append(c, st["slots"], k, v, st["k"][i], st["v"][i], count=st["count"],
                                                max_new=st["layout"].N, parents=st["parents"], q=q, rope_base=case["base"])
        out["status"] = pp.pp_cache_accept(c, st["slots"], st["keep"], st["path"], st["k"], st["v"])
        out.update(k=st["k"], v=st["v"], len=st["len"])
        return out
    dst = st["dst"]
    if kind == "fork":
        pp.pp_cache_free(c, dst[0])
        status = [pp.pp_cache_fork(c, st["src"], dst[0], st["k"], st["v"]), pp.pp_cache_reserve(c, dst[0], st["add"])]
    else:
        status = [pp.pp_cache_fork(c, st["src"], dst[1], st["k"], st["v"])]
        pp.pp_cache_free(c, dst[0])
        status.append(pp.pp_cache_compact(c, st["k"], st["v"]))
        status.append(pp.pp_cache_fork(c, st["src"], dst[0], st["k"], st["v"]))
        pp.pp_cache_free(c, dst[1])
        status.append(pp.pp_cache_compact(c, st["k"], st["v"]))
    return {**_pages_out(st), "status": status}


# ---------------------------------------------------------------- the plain forms


def _keys_of(pool, pages, n):
    """[heads, n, d] in 32 bits: the first n tokens of the pages."""
    x = pool[pages].float().transpose(0, 1)
    return x.reshape(x.shape[0], -1, x.shape[3])[:, :n].contiguous()


def _ancestors(par, n):
    see = np.zeros((n, n), bool)
    for i in range(n):
        j = i
        while j >= 0:
            see[i, j] = True
            j = par[j]
    return see


def _plain_tree(st):
    """Every sequence by itself: softmax of the scores over its cached tokens and each node's path to the root."""
    case, L = st["case"], st["layout"]
    hq, hkv, d, ps = case["hq"], case["hkv"], case["d"], case["page"]
    G, tau = hq // hkv, 1.0 / math.sqrt(d)
    o = torch.zeros(L.n, L.N, hq, d, device=DEV)
    lse = torch.zeros(hq, L.n, L.N, device=DEV)
    for i in range(L.n):
        c, n = L.count[i], L.len[i]
        if c == 0:
            continue
        pages = st["table"][L.slot[i], :_ceil(n + c, ps)].long()
        k, v = _keys_of(st["k"], pages, n + c), _keys_of(st["v"], pages, n + c)
        q = st["q"][i, :c].float().view(c, hkv, G, d).transpose(0, 1).reshape(hkv, c * G, d)
        s = torch.matmul(q, k.transpose(1, 2)) * tau
        if c > 1:
            hidden = torch.tensor(~_ancestors(L.par[i], c), device=DEV)
            hidden = hidden[:, None, :].expand(c, G, c).reshape(c * G, c)
            s[:, :, n:].masked_fill_(hidden, -math.inf)
        m = s.max(dim=2, keepdim=True).values
        p = torch.exp(s - m)
        z = p.sum(dim=2, keepdim=True)
        og = torch.matmul(p / z, v)
        o[i, :c] = og.view(hkv, c, G, d).transpose(0, 1).reshape(c, hq, d)
        lse[:, i, :c] = (m + torch.log(z)).view(hkv, c, G).transpose(1, 2).reshape(hq, c)
    return {"o": o.to(_dtype(case)), "lse": lse.view(hq, L.n * L.N)}


def _rotate(x, pos, base):
    """Pairs (x_j, x_{j+d/2}) of rows at positions pos, turned by pos * base^(-2j/d); angles in 64 bits."""
    d = x.shape[-1]
    freq = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=DEV) / d)
    a = pos.double()[:, None] * freq
    c, s = torch.cos(a).float()[:, None, :], torch.sin(a).float()[:, None, :]
    lo, hi = x[..., :d // 2].float(), x[..., d // 2:].float()
    return torch.cat([lo * c - hi * s, hi * c + lo * s], dim=-1).to(x.dtype)


def _new_tokens(L, tree):
    """Of every new token: its row in the inputs, its sequence, its place behind the cached tokens and its rotary position."""
    row, seq, place, depth = [], [], [], []
    for i in range(L.n):
        for j in range(L.count[i]):
            row.append(L.start[i] + j)
            seq.append(i)
            place.append(j)
            depth.append(depth[-j + L.par[i][j]] + 1 if tree and j else j)
    return [torch.tensor(x, device=DEV) for x in (row, seq, place, depth)]


def _plain_append(st, layer, length):
    case, L, ps = st["case"], st["layout"], st["case"]["page"]
    if "at" not in st:
        st["at"] = _new_tokens(L, case["kind"] == "step")
    row, seq, place, depth = st["at"]
    k, v, q = st["new"][layer]
    slot = st["slots"].long()[seq]
    at, pos = length.long()[slot] + place, length.long()[slot] + depth
    page = st["table"][slot, at // ps].long()
    kr, vr = k[row], v[row]
    qr = q.clone()
    if case["base"]:
        kr = _rotate(kr, pos, case["base"])
        qr[row] = _rotate(q[row], pos, case["base"])
    st["k"][layer, page, :, at % ps] = kr
    st["v"][layer, page, :, at % ps] = vr
    dead = torch.ones(q.shape[0], dtype=torch.bool, device=DEV)
    dead[row] = False
    qr[dead] = 0
    return qr


def _plain_prompts(st):
    return {"q": _plain_append(st, 0, st["len"]), "k": st["k"], "v": st["v"]}


def _plain_step(st):
    case, L, ps = st["case"], st["layout"], st["case"]["page"]
    st["len"].copy_(st["len0"])
    out = {"q%d" % i: _plain_append(st, i, st["len"]) for i in range(case["layers"])}
    slots, keep, N = st["slots"].long(), st["keep"].long(), L.N
    j = torch.arange(N, device=DEV)
    move = (j < keep[:, None]) & (st["path"] != j)
    seq, to = move.nonzero(as_tuple=True)
    base = st["len"].long()[slots[seq]]
    src, dst = base + st["path"].long()[seq, to], base + to
    tab = st["table"].long()
    ps_, pd = tab[slots[seq], src // ps], tab[slots[seq], dst // ps]
    for pool in (st["k"], st["v"]):
        pool[:, pd, :, dst % ps] = pool[:, ps_, :, src % ps].clone()
    st["len"].index_add_(0, slots, st["keep"])
    out.update(k=st["k"], v=st["v"], len=st["len"], status=torch.zeros(2, dtype=torch.int32, device=DEV))
    return out


def _listed(st, slots):
    """The pages that the slots hold: their table rows, and which columns count."""
    rows = st["table"][slots.long()].long()
    return rows, torch.arange(rows.shape[1], device=DEV) < st["held"][slots.long()][:, None]


def _plain_free(st, slots):
    rows, used = _listed(st, slots)
    st["refs"].index_add_(0, rows[used], torch.full((int(used.sum()),), -1, dtype=torch.int32, device=DEV))
    st["held"][slots.long()] = 0
    st["len"][slots.long()] = 0


def _plain_fork(st, src, dst):
    ps, src, dst = st["case"]["page"], src.long(), dst.long()
    n = st["len"][src].long()
    full, rest = n // ps, n % ps
    col = torch.arange(st["table"].shape[1], device=DEV)
    whole = col < full[:, None]
    st["table"][dst] = torch.where(whole, st["table"][src], st["table"][dst])
    shared = st["table"][src].long()[whole]
    st["refs"].index_add_(0, shared, torch.ones(shared.numel(), dtype=torch.int32, device=DEV))
    part = (rest > 0).nonzero()[:, 0]
    new = (st["refs"] == 0).nonzero()[:part.numel(), 0]
    old = st["table"][src[part], full[part]].long()
    rows = (torch.arange(ps, device=DEV) < rest[part][:, None])[None, :, None, :, None]
    for pool in (st["k"], st["v"]):
        pool[:, new] = torch.where(rows, pool[:, old], pool[:, new])
    st["table"][dst[part], full[part]] = new.to(torch.int32)
    st["refs"][new] = 1
    st["held"][dst], st["len"][dst] = (full + (rest > 0)).to(torch.int32), n.to(torch.int32)
    return torch.zeros(2, dtype=torch.int32, device=DEV)


def _plain_reserve(st, slots, add):
    ps, slots = st["case"]["page"], slots.long()
    have = st["held"][slots].long()
    want = torch.maximum(have, (st["len"][slots] + add + ps - 1) // ps)
    col = torch.arange(st["table"].shape[1], device=DEV)
    seq, at = ((col >= have[:, None]) & (col < want[:, None])).nonzero(as_tuple=True)
    new = (st["refs"] == 0).nonzero()[:seq.numel(), 0]
    st["table"][slots[seq], at] = new.to(torch.int32)
    st["refs"][new] = 1
    st["held"][slots] = want.to(torch.int32)
    return torch.zeros(2, dtype=torch.int32, device=DEV)


def _plain_compact(st):
    refs = st["refs"]
    live = (refs > 0).sum()
    at = torch.arange(refs.numel(), device=DEV)
    hole, mover = ((refs == 0) & (at < live)).nonzero()[:, 0], ((refs > 0) & (at >= live)).nonzero()[:, 0]
    new = at.clone()
    new[mover] = hole
    for pool in (st["k"], st["v"]):
        pool[:, hole] = pool[:, mover]
    refs[hole] = refs[mover]
    refs[mover] = 0
    used = torch.arange(st["table"].shape[1], device=DEV) < st["held"][:, None]
    st["table"][used] = new[st["table"].long()[used]].to(torch.int32)
    return live.to(torch.int32).reshape(1)


def _plain_fork_pass(st):
    _plain_free(st, st["dst"][0])
    status = [_plain_fork(st, st["src"], st["dst"][0]), _plain_reserve(st, st["dst"][0], st["add"])]
    return {**_pages_out(st), "status": status}


def _plain_compact_pass(st):
    a, b = st["dst"]
    status = [_plain_fork(st, st["src"], b)]
    _plain_free(st, a)
    status.append(_plain_compact(st))
    status.append(_plain_fork(st, st["src"], a))
    _plain_free(st, b)
    status.append(_plain_compact(st))
    return {**_pages_out(st), "status": status}


def _plain_verify(st):
    """Sequence by sequence; 64 bits, as probabilities are compared with given numbers."""
    case, L = st["case"], st["layout"]
    n, N = L.n, L.N
    count = torch.zeros(n, dtype=torch.int32, device=DEV)
    tokens, path = (torch.full((n, N), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    logp = torch.zeros(n, N, device=DEV)
    u_all, drafted = st["u"].double().cpu(), st["tokens"].cpu()
    for i in range(n):
        if L.count[i] == 0:
            continue
        T, kids, u, y = L.temp[i], L.children(i), u_all[i], drafted[i].tolist()
        x = st["target"][i, :L.count[i]].double() / (T or 1.0)
        x = x - x.max(dim=1, keepdim=True).values
        p = torch.exp(x)
        p /= p.sum(dim=1, keepdim=True)
        q = None
        if st["draft"] is not None and T:
            q = torch.exp(st["draft"][i, :L.count[i]].double() / T)
            q /= q.sum(dim=1, keepdim=True)
        at, out, nodes = 0, [], [0]
        while True:
            w, Z, a, found = p[at], 1.0, 0.0, None
            best = int((st["target"][i, at] == st["target"][i, at].max()).nonzero()[0])
            for c in kids[at]:
                if not T:
                    ok = y[c] == best
                elif q is not None:
                    ok = float(u[c]) * float(q[at, y[c]]) * Z < float(w[y[c]])
                else:
                    ok = float(u[c]) * Z < float(w[y[c]])
                if ok:
                    found = c
                    break
                if not T:
                    continue
                if q is not None:
                    a += Z
                    w = torch.clamp(p[at] - a * q[at], min=0)
                    Z = float(w.sum())
                else:
                    w = w.clone()
                    Z -= float(w[y[c]])
                    w[y[c]] = 0
            if found is None:
                break
            out.append((y[found], at))
            nodes.append(found)
            at = found
        if T:
            sums = torch.cumsum(w, dim=0)
            best = int((sums <= float(u[0]) * float(sums[-1])).sum())
            if best == w.numel():
                best = int((w > 0).nonzero()[-1])
        out.append((best, at))
        m = len(out)
        count[i] = m
        tok = torch.tensor([t for t, _ in out], device=DEV)
        tokens[i, :m], path[i, :m] = tok.to(torch.int32), torch.tensor(nodes, dtype=torch.int32, device=DEV)
        logp[i, :m] = torch.log(p[torch.tensor([r for _, r in out], device=DEV), tok]).float()
    return {"count": count, "tokens": tokens, "path": path, "logp": logp}


# ---------------------------------------------------------------- work


def work(case):
    L, esz, kind = _layout(case), 2 if case["dtype"] == "bf16" else 4, case["kind"]
    if kind == "verify":
        V, rows, drafts = case["vocab"], sum(L.count), 0
        if case["draft"]:
            drafts = sum(sum(1 for k in L.children(i) if k) for i in range(L.n) if L.temp[i])
        return {"bytes": int((rows + drafts) * V * esz + 24 * L.n * L.N), "flops": int(4 * (rows + drafts) * V)}
    hkv, d, ps = case["hkv"], case["d"], case["page"]
    row = 2 * hkv * d * esz  # a token's keys and values
    if kind == "tree":
        hq, K = case["hq"], case["k"]
        new = sum(L.count)
        tokens = sum(L.len[i] + L.count[i] - L.shared[i // K] * ps for i in range(L.n) if L.count[i])
        tokens += sum(s * ps for g, s in enumerate(L.shared) if any(L.count[g * K:(g + 1) * K]))
        pairs = sum(c * n + int(_ancestors(p, c).sum()) for c, n, p in zip(L.count, L.len, L.par))
        return {"bytes": int(tokens * row + new * hq * (2 * d * esz + 4)), "flops": int(4 * d * hq * pairs)}
    if kind in ("step", "prompts"):
        new, move = sum(L.count), 0
        if kind == "step":
            move = sum(int((L.path[i, :m] != np.arange(m)).sum()) for i, m in enumerate(L.keep))
        return {"bytes": int(2 * case["layers"] * (new * (row + case["hq"] * d * esz) + move * row)),
                "flops": int(6 * case["layers"] * new * (hkv + case["hq"]) * d // 2)}
    part = sum(L.P[g] % ps for g in L.src)
    full = sum(L.P[g] // ps for g in L.src)
    if kind == "fork":
        return {"bytes": int(2 * part * row * case["layers"] + 4 * (4 * full + 2 * L.pages)), "flops": 0}
    moved = sum(1 for g in L.src if L.P[g] % ps) * ps  # each of the two sets' pages, once
    return {"bytes": int(4 * (part + moved) * row * case["layers"] + 8 * (4 * full + 2 * L.pages)), "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits


def _exact_tree(st):
    """Node by node: the tokens that it sees, listed, and torch's softmax over them."""
    case, L = st["case"], st["layout"]
    hq, hkv, d, ps = case["hq"], case["hkv"], case["d"], case["page"]
    G = hq // hkv
    o = torch.zeros(L.n, L.N, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(hq, L.n, L.N, dtype=torch.float64, device=DEV)
    table = st["table"].cpu().numpy()
    for i in range(L.n):
        n, c = L.len[i], L.count[i]
        if c == 0:
            continue
        flat = np.concatenate([np.int64(pg) * ps + np.arange(ps) for pg in table[L.slot[i], :_ceil(n + c, ps)]])[:n + c]
        page, off = torch.tensor(flat // ps, device=DEV), torch.tensor(flat % ps, device=DEV)
        hidden = np.ones((c, n + c), bool)
        hidden[:, :n] = False
        for a in range(c):
            b = a
            while b != -1:
                hidden[a, n + b] = False
                b = L.par[i][b]
        hidden = torch.tensor(hidden, device=DEV)[:, None, :].expand(c, G, n + c).reshape(c * G, n + c)
        for g in range(hkv):
            k, v = st["k"][page, g, off].double(), st["v"][page, g, off].double()
            s = torch.mm(st["q"][i, :c, g * G:(g + 1) * G].double().reshape(c * G, d), k.T.contiguous()) / math.sqrt(d)
            s = s.masked_fill(hidden, -math.inf)
            o[i, :c, g * G:(g + 1) * G] = torch.mm(torch.softmax(s, dim=1), v).view(c, G, d)
            lse[g * G:(g + 1) * G, i, :c] = torch.logsumexp(s, dim=1).view(c, G).T
    return {"o": o, "lse": lse.view(hq, -1)}


def _exact_append(st):
    """Token by token: which page and row it goes to, and each pair as a complex number times e^(i angle)."""
    case, L = st["case"], st["layout"]
    ps, d, tree = case["page"], case["d"], case["kind"] == "step"
    table, out = st["table"].cpu().numpy(), {}
    pools = [st["k"].double(), st["v"].double()]
    freq = np.array([case["base"] ** (-2.0 * j / d) if case["base"] else 0.0 for j in range(d // 2)])
    row, page, off, pos = [], [], [], []
    for i in range(L.n):
        for j in range(L.count[i]):
            steps, b = j, j
            if tree:
                steps = 0
                while L.par[i][b] >= 0:
                    steps, b = steps + 1, L.par[i][b]
            t = L.len[i] + j
            row.append(L.start[i] + j)
            page.append(int(table[L.slot[i], t // ps]))
            off.append(t % ps)
            pos.append(L.len[i] + steps)
    angle = torch.tensor(np.outer(pos, freq), device=DEV)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    row, page, off = (torch.tensor(x, device=DEV) for x in (row, page, off))

    def turned(x):
        z = torch.complex(x[row, :, :d // 2].double(), x[row, :, d // 2:].double()) * turn
        return torch.cat([z.real, z.imag], dim=2)

    for layer in range(case["layers"]):
        k, v, q = st["new"][layer]
        heads = torch.arange(k.shape[1], device=DEV)
        pools[0][layer][page[:, None], heads, off[:, None]] = turned(k)
        pools[1][layer][page[:, None], heads, off[:, None]] = v[row].double()
        qr = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
        qr[row] = turned(q)
        out["q%d" % layer if tree else "q"] = qr
    if tree:
        length = st["len"].cpu().numpy().copy()
        for i in range(L.n):
            s = L.slot[i]
            place = lambda t: (int(table[s, t // ps]), t % ps)
            for j in range(L.keep[i]):  # in order: a node never moves backwards in the list
                (a, x), (b, y) = place(length[s] + int(L.path[i, j])), place(length[s] + j)
                for pool in pools:
                    pool[:, b, :, y] = pool[:, a, :, x].clone()
            length[s] += L.keep[i]
        out["len"] = torch.tensor(length, device=DEV)
        out["status"] = torch.zeros(2, dtype=torch.int32, device=DEV)
    out.update(k=pools[0], v=pools[1])
    return out


class _Book:
    """The cache's bookkeeping on the host, page by page."""

    def __init__(self, st):
        self.table = [list(map(int, r)) for r in st["table"].cpu().numpy()]
        self.len, self.held, self.refs = (st[x].cpu().numpy().tolist() for x in ("len", "held", "refs"))
        self.pools, self.ps = [st["k"].clone(), st["v"].clone()], st["case"]["page"]

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def free(self, slots):
        for s in slots:
            for c in range(self.held[s]):
                self.refs[self.table[s][c]] -= 1
            self.held[s] = self.len[s] = 0

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            whole, rest = divmod(self.len[a], self.ps)
            for c in range(whole):
                self.table[b][c] = self.table[a][c]
                self.refs[self.table[a][c]] += 1
            self.len[b], self.held[b] = self.len[a], whole + (rest > 0)
            if rest:
                self.table[b][whole] = p = self.take()
                for pool in self.pools:
                    pool[:, p, :, :rest] = pool[:, self.table[a][whole], :, :rest]
        return [0, 0]

    def reserve(self, slots, add):
        for s in slots:
            while self.held[s] * self.ps < self.len[s] + add:
                self.table[s][self.held[s]] = self.take()
                self.held[s] += 1
        return [0, 0]

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        for p in range(live, len(self.refs)):
            if self.refs[p]:
                hole = self.refs.index(0)
                for pool in self.pools:
                    pool[:, hole] = pool[:, p]
                self.refs[hole], self.refs[p] = self.refs[p], 0
                for s, row in enumerate(self.table):
                    for c in range(self.held[s]):
                        if row[c] == p:
                            row[c] = hole
        return [live]


def _exact_pages(st):
    b, L = _Book(st), st["layout"]
    if st["case"]["kind"] == "fork":
        b.free(L.dst[0])
        status = [b.fork(L.src, L.dst[0]), b.reserve(L.dst[0], st["case"]["add"])]
    else:
        status = [b.fork(L.src, L.dst[1])]
        b.free(L.dst[0])
        status.append(b.compact())
        status.append(b.fork(L.src, L.dst[0]))
        b.free(L.dst[1])
        status.append(b.compact())
    return {"table": _ints(b.table), "len": _ints(b.len), "held": _ints(b.held), "refs": _ints(b.refs),
            "k": b.pools[0], "v": b.pools[1], "status": [_ints(s) for s in status]}


def _exact_verify(st):
    """The residual as a distribution of its own: after a rejected draft it is max(r - q, 0) (or r without the draft), and its
    sum is made 1 again."""
    L = st["layout"]
    out = {"count": np.zeros(L.n, np.int32), "tokens": np.full((L.n, L.N), -1, np.int32), "path": np.full((L.n, L.N), -1, np.int32),
           "logp": np.zeros((L.n, L.N))}
    for i in range(L.n):
        if not L.count[i]:
            continue
        T, at, m = L.temp[i], 0, 0
        out["path"][i, 0] = 0
        while True:
            logp = torch.log_softmax(st["target"][i, at].double() / (T if T > 0 else 1.0), dim=0)
            r, q = logp.exp(), None
            if T == 0:
                r = torch.zeros_like(r)
                r[int((st["target"][i, at] == st["target"][i, at].max()).nonzero()[0])] = 1.0
            elif st["draft"] is not None:
                q = torch.softmax(st["draft"][i, at].double() / T, dim=0)
            step = None
            for c in range(1, L.count[i]):
                if L.par[i][c] != at:
                    continue
                y = int(st["tokens"][i, c])
                chance = float(r[y] / q[y]) if q is not None else float(r[y])
                if float(st["u"][i, c]) < chance:
                    step = (c, y)
                    break
                if q is not None:
                    r = torch.clamp(r - q, min=0)
                else:
                    r[y] = 0
                r = r / r.sum()
            if step is None:
                break
            out["tokens"][i, m], out["logp"][i, m] = step[1], float(logp[step[1]])
            at, m = step[0], m + 1
            out["path"][i, m] = at
        above = torch.cumsum(r, dim=0) > float(st["u"][i, 0]) * float(r.sum())
        y = int(above.nonzero()[0]) if bool(above.any()) else int((r > 0).nonzero()[-1])
        out["tokens"][i, m], out["logp"][i, m], out["count"][i] = y, float(logp[y]), m + 1
    return {k: torch.tensor(v, device=DEV) for k, v in out.items()}


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "tree":
        return _exact_tree(st)
    if kind in ("step", "prompts"):
        return _exact_append(st)
    return _exact_verify(st) if kind == "verify" else _exact_pages(st)
