"""GPU tests of the sampling operators together, as a rollout uses them: prompts cached once a group and forked for its
responses, drafted steps until the responses end (reserve, append, attention of several layers on one plan, verification,
accept), slots freed and pages moved on the way, all without a copy to the host.  What the steps computed is compared with the
packed attention over the finished rows: the library's for bf16, the 64-bit oracle's for fp32, whose inputs pp_attn_fwd rounds
to bf16.

Operators are deterministic, so eager runs, runs on another stream, captured and replayed ones and two at a time agree bit
for bit.  Against the packed attention both sides are within the bounds of test_gpu_tree.py of the exact value, whose larger
terms are u P|v| + u |o| + 2 r P|v| with u the half step of the type and r the error of a score, (d + 4) e tau |q||k| + 2^-21
and, where keys and queries are rotated on both sides in 32 bits, twice 4 e tau |q||k| more."""
import threading

import numpy as np
import pytest
import torch

from oracle import pp_oracle as ora
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
LAYERS, HQ, HKV, D, V, PS = 3, 4, 2, 64, 257, 16
PROMPTS, K = [37, 16, 90], 4
PARENTS = [-1, 0, 0, 1, 1, 3]
NODES, STEPS, TEMP = len(PARENTS), 7, 0.8


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Rollout:
    """Layers that read tables at a token: what a step computes follows from its tokens and places alone, so it can be
    computed again for the finished rows.  The logits come from the layers' attention."""

    def __init__(self, dtype, base, seed=5):
        r = lambda shape, i, sigma=1.0, dt=dtype: wl.randn(shape, seed + i, dt, DEV, sigma=sigma)
        self.dtype, self.base = dtype, base
        self.wq = r((LAYERS, V, HQ, D), 1)
        self.wk, self.wv = r((LAYERS, V, HKV, D), 2, 0.5), r((LAYERS, V, HKV, D), 3)
        self.head = r((LAYERS, HQ * D, V), 4, 0.3, torch.float32)
        self.table = r((V, V), 6, 1.5, torch.float32)  # the drafter's logits after a token
        self.groups, self.n = len(PROMPTS), len(PROMPTS) * K
        rng = np.random.default_rng(seed)
        self.prompts = [rng.integers(0, V, size=p) for p in PROMPTS]
        self.u = torch.tensor(rng.random((STEPS, self.n, NODES)), dtype=torch.float32, device=DEV)
        self.noise = -torch.log(-torch.log(torch.tensor(rng.random((STEPS, self.n, NODES, V)), device=DEV))).float()
        self.cache = pp.make_cache(self.n + self.groups + 2, 12, 110, PS, DEV)
        z = lambda: torch.full((LAYERS, 110, HKV, PS, D), float("nan"), dtype=dtype, device=DEV)
        self.k, self.v = z(), z()
        self.src = ints([self.n + self.groups + 1 - g for g in range(self.groups)])
        self.slots = ints([(5 * i + 3) % self.n for i in range(self.n)])
        self.parents = ints([PARENTS] * self.n)
        self.limit = ints([PROMPTS[i // K] + 3 + 4 * (i % K) for i in range(self.n)])  # responses end at different steps
        self.last = ints([self.prompts[i // K][-1] for i in range(self.n)])
        self.temp = torch.full((self.n,), TEMP, device=DEV)
        self.step_u, self.step_noise = self.u[0].clone(), self.noise[0].clone()
        self.nodes = torch.full((self.n,), NODES, dtype=torch.int32, device=DEV)
        ws = max(pp.pp_tree_workspace_size(self.cache, self.n, K, NODES, HQ, HKV, D, pp._dtype_code(self.wq)), 1)
        self.tree_ws = torch.full((ws,), 0xff, dtype=torch.uint8, device=DEV)

    def start(self):
        """All prompt tokens but the last are cached, the last one is node 0 of the first step."""
        lens = [p - 1 for p in PROMPTS]
        tokens = torch.tensor(np.concatenate([p[:-1] for p in self.prompts]), device=DEV)
        begin, count = ints(np.cumsum([0] + lens[:-1])), ints(lens)
        assert pp.pp_cache_reserve(self.cache, self.src, count).tolist() == [0, 0]
        for i in range(LAYERS):
            pp.pp_cache_append(self.cache, self.src, self.wk[i][tokens], self.wv[i][tokens], self.k[i], self.v[i], count=count,
                               start=begin, max_new=max(lens), rope_base=self.base)
        assert pp.pp_cache_accept(self.cache, self.src, count).tolist() == [0, 0]
        assert pp.pp_cache_fork(self.cache, self.src.repeat_interleave(K), self.slots, self.k, self.v).tolist() == [0, 0]

    def step(self):
        c = self.cache
        count = torch.where(c.seq_len[self.slots.long()] < self.limit, self.nodes, 0)
        tokens = [self.last]
        for j in range(1, NODES):
            tokens.append((self.table[tokens[PARENTS[j]].long()] / TEMP + self.step_noise[:, j]).argmax(1).int())
        tokens = torch.stack(tokens, 1)
        at = tokens.long()
        status = [pp.pp_cache_reserve(c, self.slots, count)]
        shared = pp.pp_cache_shared(c, self.slots, K)
        logits, outs = 0, []
        for i in range(LAYERS):
            q = pp.pp_cache_append(c, self.slots, self.wk[i][at], self.wv[i][at], self.k[i], self.v[i], count=count,
                                   parents=self.parents, q=self.wq[i][at], rope_base=self.base)
            o, lse = pp.pp_tree_attn_fwd(c, self.slots, q, self.k[i], self.v[i], parents=self.parents, count=count, group=K,
                                         shared=shared, planned=i > 0, ws=self.tree_ws)
            outs += [o, lse]
            logits = logits + o.reshape(-1, HQ * D).float() @ self.head[i]
        target = logits.view(self.n, NODES, V)
        kept, new, path, logp = pp.pp_verify_draft(target, tokens, self.step_u, draft=self.table[at], parents=self.parents,
                                                   count=count, temperature=self.temp, max_children=2)
        status.append(pp.pp_cache_accept(c, self.slots, kept, path, self.k, self.v))
        follows = new.gather(1, (kept - 1).clamp(min=0).long()[:, None])[:, 0]
        self.last.copy_(torch.where(kept > 0, follows, self.last))
        return {"kept": kept, "new": new, "path": path, "logp": logp, "target": target, "outs": torch.stack(outs[::2]),
                "lse": torch.stack(outs[1::2]), "tokens": tokens, "status": torch.stack(status), "shared": shared}

    def run(self, graph=False, move=False, between=None):
        """The steps' outputs; `move`: the prompts' slots are freed and pages moved after the second step."""
        self.start()
        got, g = [], None
        for s in range(STEPS):
            self.step_u.copy_(self.u[s])
            self.step_noise.copy_(self.noise[s])
            if move and s == 2:
                pp.pp_cache_free(self.cache, self.src)
                pp.pp_cache_compact(self.cache, self.k, self.v)
            if not graph or s == 0:
                out = self.step()
            else:
                if g is None:
                    torch.cuda.synchronize()
                    g = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(g):
                        out = self.step()
                g.replay()
            got.append({k: x.clone() for k, x in out.items()})
            if between:
                between()
        torch.cuda.synchronize()
        return got


def same(a, b):
    for x, y in zip(a, b):
        for key in x:
            i, j = (t.view(torch.int32 if t.element_size() == 4 else torch.int16) for t in (x[key], y[key]))
            assert torch.equal(i, j), key


def packed(pack, dtype, base, q, k, v):
    """o, lse and P|v| of the packed rows, on the CPU in 64 bits."""
    if dtype == torch.bfloat16:
        assert not base
        o, lse = pp.pp_attn_fwd(pack, q, k, v)
        return o.double().cpu(), lse.double().cpu(), pp.pp_attn_fwd(pack, q, k, v.abs())[0].double().cpu()
    n = lambda x: x.double().cpu().numpy()
    fwd = lambda x: (ora.attn_fwd_rope(*pack.oracle_args(), n(q), n(k), n(x), base) if base
                     else ora.attn_fwd(*pack.oracle_args(), n(q), n(k), n(x)))
    o, lse = (torch.tensor(x) for x in fwd(v)[:2])
    return o, lse, torch.tensor(fwd(v.abs())[0])


CASES = [(torch.float32, 10000.0), (torch.float32, 0.0), (torch.bfloat16, 0.0)]


@pytest.mark.parametrize("dtype,base", CASES)
def test_steps_agree_with_the_packed_rows(dtype, base):
    r = Rollout(dtype, base)
    got = r.run()
    assert all(x["status"].abs().sum().item() == 0 for x in got)
    assert any((x["kept"] > 1).any() for x in got) and any((x["kept"] == 0).any() for x in got)
    assert all((x["shared"].cpu() == torch.tensor([(p - 1) // PS for p in PROMPTS])).all() for x in got)
    # every response's tokens (node 0 of its first step is the prompt's last), and where each was computed
    seqs, places = [[] for _ in range(r.n)], [[] for _ in range(r.n)]
    for s, x in enumerate(got):
        kept, path, tok = x["kept"].tolist(), x["path"].tolist(), x["tokens"].tolist()
        for i in range(r.n):
            seqs[i] += [tok[i][j] for j in path[i][:kept[i]]]
            places[i] += [(s, j) for j in path[i][:kept[i]]]
            assert kept[i] == 0 or x["new"][i, :kept[i] - 1].tolist() == [tok[i][j] for j in path[i][1:kept[i]]]
    lens = r.cache.seq_len.tolist()
    assert [lens[s] for s in r.slots.tolist()] == [PROMPTS[i // K] - 1 + len(q) for i, q in enumerate(seqs)]
    # rows: the prompt without its last token, then K responses that begin with it
    pack = wl.make_pack([p - 1 for p in PROMPTS], [[len(seqs[g * K + i]) for i in range(K)] for g in range(r.groups)])
    flat, where = np.zeros(pack.total_tokens, int), {}
    for g in range(r.groups):
        b = int(pack.row_start[g])
        flat[b:b + PROMPTS[g] - 1] = r.prompts[g][:-1]
        for i in range(K):
            at = b + int(pack.resp_off[g][i])
            flat[at:at + len(seqs[g * K + i])] = seqs[g * K + i]
            for j, place in enumerate(places[g * K + i]):
                where[at + j] = (g * K + i, place)
    rows, tau, u = torch.tensor(flat, device=DEV), D ** -0.5, U[dtype]
    total = 0
    for i in range(LAYERS):
        q, k, v = r.wq[i][rows], r.wk[i][rows], r.wv[i][rows]
        o, lse, pv = packed(pack, dtype, base, q, k, v)
        qk = q.float().norm(dim=2).max().item() * k.float().norm(dim=2).max().item() * tau
        err = (D + 4) * E * qk + 8 * E * qk + 2.0 ** -21 + (8 * E * qk if base else 0)
        for t, (seq, (s, j)) in where.items():
            a, b, w = got[s]["outs"][i][seq, j].double().cpu(), o[t], pv[t]
            bound = 2 * ((u + 2 * err + 2.0 ** -20 + 200 * E) * w * (1 + 4 * u) + u * b.abs())
            assert ((a - b).abs() <= bound).all(), (i, seq, s, j)
            la, lb = got[s]["lse"][i][:, seq * NODES + j].double().cpu(), lse[:, t]
            assert ((la - lb).abs() <= 2 * (err + 2.0 ** -20 + 200 * E + 4 * E * lb.abs())).all()
        total = total + o.reshape(-1, HQ * D) @ r.head[i].double().cpu()
    # the log-probs are those of the packed rows' logits: a logit's difference is at most the outputs' through the head
    slack = LAYERS * HQ * D * r.head.abs().max().item() * 2 * (2 * u + 1e-4) * 4 / TEMP
    temp = float(np.float32(TEMP))  # as the kernel has it
    ref = torch.log_softmax(total / temp, 1)
    for t, (seq, (s, j)) in where.items():
        x = got[s]
        at = x["path"][seq].tolist().index(j)
        y = int(x["new"][seq, at])
        own = torch.log_softmax(x["target"][seq, j].double() / temp, 0)[y].item()
        assert abs(x["logp"][seq, at].item() - own) <= 2.0 ** -24 * abs(own) + 1e-12
        assert abs(own - ref[t, y].item()) <= 2 * slack
    # and all pages come back
    pp.pp_cache_free(r.cache, torch.cat([r.slots, r.src]))
    assert r.cache.refs.abs().sum().item() == 0 and r.cache.held.abs().sum().item() == 0


@pytest.mark.parametrize("dtype,base", CASES[1:])
def test_captured_moved_and_on_another_stream(dtype, base):
    want = Rollout(dtype, base).run()
    junk = []

    def between():  # the program's own work between replays
        junk.append(torch.randn(1 << 18, device=DEV).sum().item())
        torch.cuda.synchronize()

    same(want, Rollout(dtype, base).run(graph=True, between=between))
    same(want, Rollout(dtype, base).run(move=True))
    same(want, Rollout(dtype, base).run(graph=True, move=True))
    r, side = Rollout(dtype, base), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = r.run()
    same(want, got)


def test_two_rollouts_at_once():
    """Two host threads, a stream and a cache each."""
    cases = [(torch.float32, 10000.0), (torch.bfloat16, 0.0)]
    want = [Rollout(*c).run() for c in cases]
    made, got, errors = [Rollout(*c) for c in cases], [None, None], []
    torch.cuda.synchronize()

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                got[i] = made[i].run()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for a, b in zip(want, got):
        same(a, b)


def test_two_graphs_share_a_workspace():
    """Two captured steps with one workspace, replayed in turn: each plans anew."""
    a, b = Rollout(torch.bfloat16, 0.0, seed=5), Rollout(torch.bfloat16, 0.0, seed=6)
    want = [Rollout(torch.bfloat16, 0.0, seed=s).run() for s in (5, 6)]
    b.tree_ws = a.tree_ws
    graphs, outs, got = [], [], [[], []]
    for r in (a, b):
        r.start()
    torch.cuda.synchronize()
    for s in range(STEPS):
        for i, r in enumerate((a, b)):
            r.step_u.copy_(r.u[s])
            r.step_noise.copy_(r.noise[s])
            if s == 0:
                out = r.step()
            elif s == 1:
                torch.cuda.synchronize()
                graphs.append(torch.cuda.CUDAGraph())
                with torch.cuda.graph(graphs[i]):
                    outs.append(r.step())
            if s > 0:
                graphs[i].replay()
                out = outs[i]
            got[i].append({k: x.clone() for k, x in out.items()})
    torch.cuda.synchronize()
    same(want[0], got[0])
    same(want[1], got[1])
