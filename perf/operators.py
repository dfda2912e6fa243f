"""Performance cases of policy optimisation on packed groups: a prompt, its K sampled responses and, for image-conditioned
models, the encoder states of the prompt's images.

A step of such training runs, beside the packed self-attention, per layer cross attention of the packed row to its encoder
states (forward, and backward in training), and once per batch the log-probs and entropies of the response tokens, the clipped
policy loss with its KL and entropy terms and its gradient, and the gradient of the logits.  Sampling the responses runs the
cross attention for a token or a few at a time.  The sizes are those of workload.py's batches or generic.

listed() gives the cases, draw(rng) more of the same ranges; prepare makes a case's inputs, run does one pass (in elementary
torch operations, or with the library where `own` is set), exact the same in 64 bits from the definitions.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"


# ---------------------------------------------------------------- cases


def _base(name, kind, dtype, rows, prompt, k, resp, pad=0, len_seed=1):
    c = {"kind": kind, "dtype": dtype, "rows": rows, "p_lo": prompt[0], "p_hi": prompt[1], "k_lo": k[0], "k_hi": k[1],
         "r_lo": resp[0], "r_hi": resp[1], "pad_hi": pad, "len_seed": len_seed}
    if name:
        c["name"] = name
    return c


def _cross(name, train, dtype, heads, d, rows, prompt, k, resp, enc, enc_pad=0, images=0, pad=0, len_seed=1):
    c = _base(name, "cross_train" if train else "cross_fwd", dtype, rows, prompt, k, resp, pad, len_seed)
    c.update({"hq": heads[0], "hkv": heads[1], "d": d, "e_lo": enc[0], "e_hi": enc[1], "enc_pad": enc_pad, "images": images})
    return c


def _tok(name, kind, dtype, vocab, rows, prompt, k, resp, entropy, hidden_vocab=0, pad=0, len_seed=1):
    c = _base(name, kind, dtype, rows, prompt, k, resp, pad, len_seed)
    c.update({"vocab": vocab, "entropy": entropy, "hidden_vocab": hidden_vocab})
    return c


def _policy(name, rows, prompt, k, resp, reduction, kl="", entropy=False, masked=False, adv_tok=False, old=True, dual=0.0,
            pad=0, len_seed=1):
    c = _base(name, "policy", "fp32", rows, prompt, k, resp, pad, len_seed)
    c.update({"reduction": reduction, "kl": kl, "entropy": entropy, "masked": masked, "adv_tok": adv_tok, "old": old,
              "dual": dual})
    return c


def listed():
    return [
        # sampling: one new token of each of eight rows looks at its image's states (latency counts)
        _cross("cross_one_token", False, "bf16", (32, 8), 128, 8, (1, 1), (0, 0), (0, 0), (300, 1601)),
        # sampling over video-length states, two to four tokens a row: bound by reading keys and values once
        _cross("cross_few_tokens_long", False, "bf16", (64, 8), 128, 4, (2, 4), (0, 0), (0, 0), (16000, 48000)),
        # a reference model scores an 8B-shaped batch, one to four image tiles a row
        _cross("cross_fwd_8b", False, "bf16", (32, 8), 128, 8, (256, 1536), (2, 2), (64, 512), (1601, 6404)),
        # one layer of 8B-shaped training with one packed row per GPU, one image
        _cross("cross_train_8b_one_row", True, "bf16", (32, 8), 128, 1, (1024, 1536), (2, 2), (128, 512), (1601, 1601)),
        # a small model of head size 64: ragged rows and states, several images in the text, tokens ahead of the first
        # image see nothing, padding in both axes
        _cross("cross_train_d64_images", True, "bf16", (14, 2), 64, 24, (17, 900), (1, 6), (1, 300), (0, 1500), enc_pad=40,
               images=4, pad=63),
        # the toy model in fp32
        _cross("cross_train_tiny_fp32", True, "fp32", (4, 4), 64, 4, (64, 128), (2, 2), (16, 64), (50, 200)),
        # the largest: a 72B-shaped layer on long rows, several image tiles
        _cross("cross_train_72b", True, "bf16", (64, 8), 128, 8, (2048, 6144), (2, 2), (64, 256), (1601, 6404)),
        # log-probs and entropies of groups of eight responses over a large bf16 vocabulary
        _tok("tok_logprob_128k", "tok", "bf16", 128256, 4, (256, 1024), (8, 8), (64, 512), True),
        # gradient of log-probs and entropies on the predicting rows, 72B-shaped vocabulary
        _tok("tok_bwd_rows_152k", "tok_bwd_rows", "bf16", 152064, 4, (300, 1200), (4, 4), (50, 500), True),
        # dense gradient of the log-probs alone; fp32 logits whose rows start on no 16-byte boundary, the last entries of the
        # vocabulary hidden with -inf
        _tok("tok_bwd_dense_odd_fp32", "tok_bwd", "fp32", 50257, 4, (64, 700), (2, 4), (20, 400), False, hidden_vocab=80),
        # the loss of a micro-batch of groups: mean over the responses, KL to the reference
        _policy("policy_micro_batch", 4, (256, 1024), (8, 8), (64, 512), "seq", kl="k3"),
        # the loss of a whole rollout batch: mean over the tokens that the mask counts, entropy bonus, advantages per token
        _policy("policy_rollout_batch", 256, (100, 1000), (8, 8), (50, 1024), "token", kl="k3", entropy=True, masked=True,
                adv_tok=True, dual=3.0, pad=63),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    a, b = _log_int(rng, lo, hi), _log_int(rng, lo, hi)
    return min(a, b), max(a, b)


def _cost(case):
    w = work(case)
    return w["flops"] / 1e12 + w["bytes"] / 5e9  # about ms


def draw(rng):
    kind = rng.choice(["cross_fwd", "cross_few", "cross_train", "cross_train", "tok", "tok_bwd", "tok_bwd_rows", "policy",
                       "policy"])
    seed, pad = rng.randint(2, 1 << 30), rng.choice([0, 0, 63])
    rows, prompt = _log_int(rng, 1, 24), _span(rng, 8, 6144)
    k_lo = rng.randint(1, 6)
    k, resp = (k_lo, k_lo + rng.randint(0, 2)), _span(rng, 1, 512)
    if kind.startswith("cross"):
        heads, d = rng.choice([((32, 8), 128), ((64, 8), 128), ((28, 4), 128), ((16, 4), 64), ((14, 2), 64), ((8, 8), 64),
                               ((12, 12), 128), ((8, 1), 64)])
        dtype = rng.choice(["bf16"] * 5 + ["fp32"])
        enc, enc_pad, images = _span(rng, 1, 8000), rng.choice([0, 0, 40]), rng.choice([0, 0, 1, 4])
        if kind == "cross_few":
            rows, prompt, k, resp = _log_int(rng, 1, 64), _span(rng, 1, 8), (0, 0), (0, 0)
            enc, images = _span(rng, 1, 48000), 0
        if dtype == "fp32":
            prompt, enc = (min(prompt[0], 700), min(prompt[1], 700)), (min(enc[0], 2000), min(enc[1], 2000))
        if rng.random() < 0.2:
            enc = (0, enc[1])  # rows of text alone among the others
        case = _cross("", kind == "cross_train", dtype, heads, d, rows, prompt, k, resp, enc, enc_pad, images, pad, seed)
        most = "cross_train_72b"
    elif kind.startswith("tok"):
        vocab = rng.choice([128256, 152064, 32000, rng.randint(200, 152064)])
        case = _tok("", kind, rng.choice(["bf16", "bf16", "fp32"]), vocab, rows, prompt, k, resp, rng.random() < 0.6,
                    rng.choice([0, 0, 80]), pad, seed)
        most = {"tok": "tok_logprob_128k", "tok_bwd": "tok_bwd_rows_152k", "tok_bwd_rows": "tok_bwd_rows_152k"}[kind]
    else:
        k_lo = rng.randint(1, 16)
        case = _policy("", _log_int(rng, 1, 256), _span(rng, 8, 1000), (k_lo, k_lo + rng.randint(0, 2)), _span(rng, 1, 1024),
                       rng.choice(["token", "seq", "sum"]), rng.choice(["", "k1", "k2", "k3", "k3"]), rng.random() < 0.4,
                       rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.8, rng.choice([0.0, 0.0, 3.0]), pad, seed)
        most = "policy_rollout_batch"
    most = _cost(next(c for c in listed() if c["name"] == most))
    while case["rows"] > 1 and _cost(case) > most:
        case["rows"] //= 2
    while _cost(case) > most:
        case["p_hi"] = max(case["p_lo"], case["p_hi"] // 2)
        case["p_lo"] = max(8, case["p_lo"] // 2)
        case["k_hi"] = max(case["k_lo"], case["k_hi"] - 1)
        case["r_hi"] = max(case["r_lo"], case["r_hi"] // 2)
        case["r_lo"] = max(1, case["r_lo"] // 2)
    return case


# ---------------------------------------------------------------- the packed layout


class _Layout:
    """Rows of a prompt, K responses back to back and padding on one token axis; encoder states of each row, and padding,
    on another."""

    def __init__(self, case):
        rng = np.random.default_rng([2602, 24082, 7, case["len_seed"]])
        B = case["rows"]
        self.P = rng.integers(case["p_lo"], case["p_hi"], size=B, endpoint=True).tolist()
        K = rng.integers(case["k_lo"], case["k_hi"], size=B, endpoint=True).tolist()
        self.R = [rng.integers(case["r_lo"], case["r_hi"], size=n, endpoint=True).tolist() for n in K]
        self.pad = rng.integers(0, case["pad_hi"], size=B, endpoint=True).tolist()
        self.n = [p + sum(r) for p, r in zip(self.P, self.R)]
        self.t0 = np.concatenate([[0], np.cumsum([n + x for n, x in zip(self.n, self.pad)])]).tolist()
        self.T, self.B, self.Kmax = self.t0[-1], B, max([len(r) for r in self.R] + [1])
        if "e_lo" in case:
            self.E = rng.integers(case["e_lo"], case["e_hi"], size=B, endpoint=True).tolist()
            self.enc_pad = rng.integers(0, case["enc_pad"], size=B, endpoint=True).tolist()
            self.e0 = np.concatenate([[0], np.cumsum([n + x for n, x in zip(self.E, self.enc_pad)])]).tolist()
            self.begin = self.end = None
            if case["images"]:
                self._images(case["images"], rng)

    def _images(self, most, rng):
        """Each token looks at the last image ahead of it in the row: the keys [begin, end) of the row's states."""
        self.begin, self.end = np.zeros(self.T, np.int32), np.zeros(self.T, np.int32)
        for b in range(self.B):
            n, E = self.n[b], self.E[b]
            m = int(rng.integers(1, most, endpoint=True))
            edge = np.linspace(0, E, m + 1).astype(np.int64)
            at = np.sort(rng.integers(0, max(1, self.P[b]), size=m))  # where each image stands in the prompt
            img = np.searchsorted(at, np.arange(n), side="right") - 1
            lo = np.where(img >= 0, edge[np.maximum(img, 0)], 0)
            hi = np.where(img >= 0, edge[np.maximum(img, 0) + 1], 0)
            self.begin[self.t0[b]:self.t0[b] + n], self.end[self.t0[b]:self.t0[b] + n] = lo, hi

    def responses(self):
        """[(row b, response k, flat start, length)]"""
        out = []
        for b in range(self.B):
            o = self.t0[b] + self.P[b]
            for k, n in enumerate(self.R[b]):
                out.append((b, k, o, n))
                o += n
        return out

    def token_slots(self):
        """Flat positions of the response tokens, and the slot b * Kmax + k of each."""
        rs = self.responses()
        pos = np.concatenate([np.arange(o, o + n) for _, _, o, n in rs] + [np.zeros(0, np.int64)])
        slot = np.concatenate([np.full(n, b * self.Kmax + k) for b, k, _, n in rs] + [np.zeros(0, np.int64)])
        return pos.astype(np.int64), slot.astype(np.int64)

    def predicting(self):
        """Flat row of the logits that predicts each response token (the last prompt token predicts every response's
        first), and the token's flat position."""
        rs = self.responses()
        row = [np.concatenate([[self.t0[b] + self.P[b] - 1], np.arange(o, o + n - 1)]) for b, _, o, n in rs if n]
        at = [np.arange(o, o + n) for _, _, o, n in rs if n]
        cat = lambda x: np.concatenate(x + [np.zeros(0, np.int64)]).astype(np.int64)
        return cat(row), cat(at)


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


def prepare(case, seed):
    L, dt, s = _Layout(case), _dtype(case), seed * 1000 + 29
    st = {"case": case, "layout": L}
    if case["kind"].startswith("cross"):
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        st["q"] = _randn((L.T, hq, d), s, dt)
        st["k"], st["v"] = _randn((L.e0[-1], hkv, d), s + 1, dt), _randn((L.e0[-1], hkv, d), s + 2, dt)
        st["begin"] = st["end"] = None
        if L.begin is not None:
            st["begin"], st["end"] = torch.tensor(L.begin, device=DEV), torch.tensor(L.end, device=DEV)
        if case["kind"] == "cross_train":
            st["do"] = _randn((L.T, hq, d), s + 3, dt)
    elif case["kind"].startswith("tok"):
        g = torch.Generator(device=DEV)
        g.manual_seed(s)
        V = case["vocab"]
        seen = V - case["hidden_vocab"]
        st["tokens"] = torch.randint(0, seen, (L.T,), generator=g, device=DEV, dtype=torch.int32)
        st["logits"] = _randn((L.T, V), s + 1, dt, 3.0)
        st["logits"][:, seen:] = -math.inf
        if case["kind"] != "tok":
            st["dtok"] = _randn((L.T,), s + 2, torch.float32, 1e-3)
            st["dent"] = _randn((L.T,), s + 3, torch.float32, 1e-3) if case["entropy"] else None
        row, at = L.predicting()
        st["row"], st["at"] = torch.tensor(row, device=DEV), torch.tensor(at, device=DEV)
    else:
        pos, slot = L.token_slots()
        st["pos"], st["slot"] = torch.tensor(pos, device=DEV), torch.tensor(slot, device=DEV)
        lp = -_randn((L.T,), s, torch.float32).abs()
        st["logp"] = lp
        st["old"] = lp + _randn((L.T,), s + 1, torch.float32, 0.15) if case["old"] else None
        st["ref"] = lp + _randn((L.T,), s + 2, torch.float32, 0.3) if case["kl"] else None
        st["entropy"] = _randn((L.T,), s + 3, torch.float32).abs() if case["entropy"] else None
        st["adv"] = _randn((L.T,) if case["adv_tok"] else (L.B, L.Kmax), s + 4, torch.float32)
        st["mask"] = (_randn((L.T,), s + 5, torch.float32) > -1.0).to(torch.uint8) if case["masked"] else None
        st["kl_coef"], st["ent_coef"] = 0.04 if case["kl"] else 0.0, 0.01 if case["entropy"] else 0.0
        st["norm"] = 1024.0 * L.B
    if own:
        from paper_2602_24082_amd import workload as wl
        st["pack"] = wl.make_pack(L.P, L.R, pad=L.pad, max_resp=L.Kmax)
        if "e_lo" in case:
            st["enc"] = wl.make_enc(L.E, pad=L.enc_pad)
    return st


CLIP_LOW, CLIP_HIGH = 0.2, 0.28


def run(st):
    kind = st["case"]["kind"]
    if own:
        return _run_own(st, kind)
    if kind.startswith("cross"):
        return _plain_cross(st)
    if kind == "tok":
        return _plain_tok(st)
    if kind.startswith("tok"):
        return _plain_tok_bwd(st)
    return _plain_policy(st)


def _run_own(st, kind):
    from paper_2602_24082_amd import binding as pp
    case, pack = st["case"], st["pack"]
    if kind.startswith("cross"):
        q, k, v, enc, keys = st["q"], st["k"], st["v"], st["enc"], {"key_begin": st["begin"], "key_end": st["end"]}
        o, lse = pp.pp_cross_attn_fwd(pack, enc, q, k, v, **keys)
        out = {"o": o, "lse": lse}
        if kind == "cross_train":
            out["dq"], out["dk"], out["dv"] = pp.pp_cross_attn_bwd(pack, enc, q, k, v, o, lse, st["do"], **keys)
        return out
    if kind == "tok":
        tok, ent = pp.pp_tok_logprob(pack, st["logits"], st["tokens"], want_entropy=case["entropy"])
        return {"tok": tok, "entropy": ent} if case["entropy"] else {"tok": tok}
    if kind == "tok_bwd_rows":
        dl, idx = pp.pp_tok_logprob_bwd_rows(pack, st["logits"], st["tokens"], st["dtok"], st["dent"])
        return {"dlogits": dl, "row_index": idx}
    if kind == "tok_bwd":
        return {"dlogits": pp.pp_tok_logprob_bwd(pack, st["logits"], st["tokens"], st["dtok"], st["dent"])}
    loss, stats, counts, dlogp, dent = pp.pp_policy_loss(
        pack, st["logp"], st["adv"], logp_old=st["old"], logp_ref=st["ref"], entropy=st["entropy"], mask=st["mask"],
        clip_low=CLIP_LOW, clip_high=CLIP_HIGH, dual_clip=case["dual"], kl_coef=st["kl_coef"], kl=case["kl"] or "k3",
        ent_coef=st["ent_coef"], reduction=case["reduction"], norm=st["norm"])
    out = {"loss": loss, "stats": stats, "counts": counts, "dlogp": dlogp}
    if dent is not None:
        out["dentropy"] = dent
    return out


# ---------------------------------------------------------------- the plain forms


def _plain_cross(st):
    """Every row and kv-head by itself: softmax of the scores over the row's states (those of the token's range), and the
    softmax's backward pass, in 32 bits."""
    case, L = st["case"], st["layout"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G, tau, dt = hq // hkv, 1.0 / math.sqrt(d), _dtype(case)
    train = "do" in st
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    o, lse = torch.zeros_like(q), torch.zeros(hq, L.T, device=DEV)
    if train:
        do, dq, dk, dv = st["do"].float(), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for b in range(L.B):
        n, E = L.n[b], L.E[b]
        if n == 0 or E == 0:
            continue
        r, e = slice(L.t0[b], L.t0[b] + n), slice(L.e0[b], L.e0[b] + E)
        hidden = None
        if st["begin"] is not None:
            j = torch.arange(E, device=DEV)
            hidden = (j < st["begin"][r, None]) | (j >= st["end"][r, None])  # [n, E]
            hidden = hidden[:, None, :].expand(n, G, E).reshape(n * G, E)
        for g in range(hkv):
            h = slice(g * G, (g + 1) * G)
            qg, kg, vg = q[r, h].reshape(n * G, d), k[e, g].contiguous(), v[e, g].contiguous()
            s = torch.mm(qg, kg.T) * tau
            if hidden is not None:
                s.masked_fill_(hidden, -math.inf)
            m = s.max(dim=1, keepdim=True).values
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            p = torch.exp(s - m)
            z = p.sum(dim=1, keepdim=True)
            some = z > 0
            p = p / torch.where(some, z, torch.ones_like(z))
            og = torch.mm(p, vg)
            o[r, h] = og.view(n, G, d)
            lse[h, r] = torch.where(some, m + torch.log(z), torch.zeros_like(z)).view(n, G).T
            if train:
                dog = do[r, h].reshape(n * G, d)
                dv[e, g] = torch.mm(p.T, dog)
                ds = p * (torch.mm(dog, vg.T) - (dog * og).sum(dim=1, keepdim=True))
                dq[r, h] = (torch.mm(ds, kg) * tau).view(n, G, d)
                dk[e, g] = torch.mm(ds.T, qg) * tau
    out = {"o": o.to(dt), "lse": lse}
    if train:
        out["dq"], out["dk"], out["dv"] = dq.to(dt), dk.to(dt), dv.to(dt)
    return out


_ROWS = 1024  # logit rows at a time


def _plain_tok(st):
    case, L = st["case"], st["layout"]
    tok, ent = torch.zeros(L.T, device=DEV), torch.zeros(L.T, device=DEV)
    for c in range(0, st["row"].numel(), _ROWS):
        row, at = st["row"][c:c + _ROWS], st["at"][c:c + _ROWS]
        x = st["logits"][row].float()
        y = x - x.max(dim=1, keepdim=True).values
        e = torch.exp(y)
        z = e.sum(dim=1)
        tok[at] = y.gather(1, st["tokens"][at].long()[:, None])[:, 0] - torch.log(z)
        if case["entropy"]:
            ent[at] = torch.log(z) - torch.where(e > 0, e * y, torch.zeros_like(y)).sum(dim=1) / z
    return {"tok": tok, "entropy": ent} if case["entropy"] else {"tok": tok}


def _plain_tok_bwd(st):
    case, L = st["case"], st["layout"]
    rows, inv = torch.unique(st["row"], return_inverse=True)
    dense = case["kind"] == "tok_bwd"
    dl = torch.zeros((L.T, case["vocab"]) if dense else (rows.numel(), case["vocab"]), dtype=_dtype(case), device=DEV)
    label = st["tokens"][st["at"]].long()
    g = st["dtok"][st["at"]]
    sum_g = torch.zeros(rows.numel(), device=DEV).index_add_(0, inv, g)
    sum_h = torch.zeros(rows.numel(), device=DEV)
    if st["dent"] is not None:
        sum_h.index_add_(0, inv, st["dent"][st["at"]])
    order = torch.argsort(inv, stable=True)
    first = torch.searchsorted(inv[order], torch.arange(0, rows.numel() + _ROWS, _ROWS, device=DEV)).tolist()
    for i, c in enumerate(range(0, rows.numel(), _ROWS)):
        row = rows[c:c + _ROWS]
        x = st["logits"][row].float()
        y = x - x.max(dim=1, keepdim=True).values
        e = torch.exp(y)
        z = e.sum(dim=1, keepdim=True)
        p = e / z
        out = -sum_g[c:c + _ROWS, None] * p
        if st["dent"] is not None:
            y = torch.where(e > 0, y - torch.log(z), torch.zeros_like(y))  # log p
            H = -(p * y).sum(dim=1, keepdim=True)
            out -= sum_h[c:c + _ROWS, None] * p * (y + H)
        at = order[first[i]:first[i + 1]]
        out.index_put_((inv[at] - c, label[at]), g[at], accumulate=True)
        if dense:
            dl[row] = out.to(dl.dtype)
        else:
            dl[c:c + _ROWS] = out.to(dl.dtype)
    return {"dlogits": dl} if dense else {"dlogits": dl, "row_index": rows.to(torch.int32)}


def _plain_policy(st):
    case, L = st["case"], st["layout"]
    pos, slot = st["pos"], st["slot"]
    if st["mask"] is not None:
        keep = st["mask"][pos] != 0
        pos, slot = pos[keep], slot[keep]
    # 64 bits: ratios are compared with the clip range's ends, and the KL term is a small difference
    lp = st["logp"][pos].double()
    delta = lp - st["old"][pos].double() if st["old"] is not None else torch.zeros_like(lp)
    adv = (st["adv"][pos] if case["adv_tok"] else st["adv"].reshape(-1)[slot]).double()
    ratio = torch.exp(delta)
    off = ((adv > 0) & (ratio > 1 + CLIP_HIGH)) | ((adv < 0) & (ratio < 1 - CLIP_LOW))
    used = torch.where(off, torch.where(adv > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW).double(), ratio)
    if case["dual"]:
        far = (adv < 0) & (ratio > case["dual"])
        off, used = off | far, torch.where(far, torch.full_like(used, case["dual"]), used)
    surr = used * adv
    dl = torch.where(off, torch.zeros_like(adv), -adv * ratio)
    kl = torch.zeros_like(lp)
    if case["kl"]:
        x = st["ref"][pos].double() - lp
        if case["kl"] == "k1":
            kl, dkl = -x, torch.ones_like(x)
        elif case["kl"] == "k2":
            kl, dkl = 0.5 * x * x, -x
        else:
            kl, dkl = torch.expm1(x) - x, -torch.expm1(x)
        dl = dl + st["kl_coef"] * dkl
    n = torch.zeros(L.B * L.Kmax, dtype=torch.float64, device=DEV).index_add_(0, slot, torch.ones_like(lp))
    if case["reduction"] == "seq":
        w = 1.0 / (n[slot] * (n > 0).sum())
    elif case["reduction"] == "token":
        w = torch.full_like(lp, 1.0) / max(1, lp.numel())
    else:
        w = torch.full_like(lp, 1.0 / st["norm"])
    ent = st["entropy"][pos].double() if st["entropy"] is not None else torch.zeros_like(lp)
    parts = [(-surr * w).sum(), (kl * w).sum(), (ent * w).sum(), (ratio * w).sum()]
    loss = parts[0] + st["kl_coef"] * parts[1] - st["ent_coef"] * parts[2]
    dlogp = torch.zeros(L.T, device=DEV)
    dlogp[pos] = (dl * w).float()
    out = {"loss": loss.float().reshape(1), "stats": torch.stack(parts).float(),
           "counts": torch.stack([torch.ones_like(off).sum(), off.sum()]).to(torch.int32), "dlogp": dlogp}
    if st["entropy"] is not None:
        dent = torch.zeros(L.T, device=DEV)
        dent[pos] = (-st["ent_coef"] * w).float()
        out["dentropy"] = dent
    return out


# ---------------------------------------------------------------- work


def work(case):
    L, esz = _Layout(case), 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind.startswith("cross"):
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        pairs = sum(n * E for n, E in zip(L.n, L.E)) if L.begin is None else int((L.end - L.begin).sum())
        q, kv, lse = L.T * hq * d * esz, sum(L.E) * hkv * d * esz, L.T * hq * 4
        nbytes = 2 * q + 2 * kv + lse + (8 * L.T if L.begin is not None else 0)
        flops = 4 * d * hq * pairs
        if kind == "cross_train":  # the backward pass reads q, k, v, o, lse and dO, and writes dq, dk and dv
            nbytes += 4 * q + 4 * kv + lse
            flops += 10 * d * hq * pairs
        return {"bytes": int(nbytes), "flops": int(flops)}
    if kind.startswith("tok"):
        row, at = L.predicting()
        n, V = len(np.unique(row)), case["vocab"]
        nbytes = n * V * esz + 4 * len(at)
        if kind == "tok":
            nbytes += 4 * L.T * (2 if case["entropy"] else 1)
        else:
            nbytes += (n if kind == "tok_bwd_rows" else L.T) * V * esz + 4 * len(at) * (2 if case["entropy"] else 1)
        return {"bytes": int(nbytes), "flops": int(n * V * ((5 if case["entropy"] else 3) + (0 if kind == "tok" else 4)))}
    n = sum(sum(r) for r in L.R)
    reads = 1 + case["old"] + bool(case["kl"]) + case["entropy"] + case["adv_tok"]
    nbytes = 4 * n * reads + (n if case["masked"] else 0) + 4 * L.T * (2 if case["entropy"] else 1)
    return {"bytes": int(nbytes), "flops": int(40 * n)}


# ---------------------------------------------------------------- the same in 64 bits


def _exact_cross(st):
    """Head by head with torch's softmax, gradients by autograd."""
    case, L = st["case"], st["layout"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    names = ("q", "k", "v") + (("do",) if "do" in st else ())
    x = {n: st[n].double() for n in names}
    out = {"o": torch.zeros_like(x["q"]), "lse": torch.zeros(hq, L.T, dtype=torch.float64, device=DEV)}
    if "do" in x:
        out.update(dq=torch.zeros_like(x["q"]), dk=torch.zeros_like(x["k"]), dv=torch.zeros_like(x["v"]))
    for b in range(L.B):
        n, E = L.n[b], L.E[b]
        t, e = L.t0[b], L.e0[b]
        lo, hi = np.zeros(n, np.int64), np.full(n, E, np.int64)
        if L.begin is not None:
            lo, hi = L.begin[t:t + n].astype(np.int64), L.end[t:t + n].astype(np.int64)
        idx = np.nonzero(hi > lo)[0]  # the other tokens see nothing: zeros
        if len(idx) == 0:
            continue
        tok = torch.tensor(t + idx, device=DEV)
        j = np.arange(E)
        seen = None
        if (lo[idx] > 0).any() or (hi[idx] < E).any():
            seen = torch.tensor((j[None] >= lo[idx, None]) & (j[None] < hi[idx, None]), device=DEV)
        for h in range(hq):
            g = h // (hq // hkv)
            qh = x["q"][tok, h].requires_grad_("do" in x)
            kh = x["k"][e:e + E, g].clone().requires_grad_("do" in x)
            vh = x["v"][e:e + E, g].clone().requires_grad_("do" in x)
            s = torch.mm(qh, kh.T.contiguous()) / math.sqrt(d)
            if seen is not None:
                s = s.masked_fill(~seen, -math.inf)
            oh = torch.mm(torch.softmax(s, dim=1), vh)
            out["o"][tok, h] = oh.detach()
            out["lse"][h, tok] = torch.logsumexp(s.detach(), dim=1)
            if "do" in x:
                gq, gk, gv = torch.autograd.grad(oh, (qh, kh, vh), x["do"][tok, h])
                out["dq"][tok, h] = gq
                out["dk"][e:e + E, g] += gk
                out["dv"][e:e + E, g] += gv
            del s, oh
    return out


def _exact_tok(st):
    case, L = st["case"], st["layout"]
    dense = case["kind"] == "tok_bwd"
    row_of = {}
    for r, t in zip(st["row"].tolist(), st["at"].tolist()):
        row_of.setdefault(r, []).append(t)
    rows = sorted(row_of)
    tok = torch.zeros(L.T, dtype=torch.float64, device=DEV)
    ent = torch.zeros_like(tok)
    dl = None
    if case["kind"] != "tok":
        dl = torch.zeros((L.T if dense else len(rows), case["vocab"]), dtype=torch.float64, device=DEV)
    for c in range(0, len(rows), 512):
        some = rows[c:c + 512]
        logp = torch.log_softmax(st["logits"][torch.tensor(some, device=DEV)].double(), dim=1)
        p = logp.exp()
        H = torch.special.entr(p).sum(dim=1)
        i = torch.tensor([i for i, r in enumerate(some) for _ in row_of[r]], device=DEV)
        t = torch.tensor([t for r in some for t in row_of[r]], device=DEV)
        y = st["tokens"][t].long()
        tok[t], ent[t] = logp[i, y], H[i]
        if dl is not None:
            a = torch.zeros(len(some), dtype=torch.float64, device=DEV)
            grad = torch.zeros_like(p)
            grad.index_put_((i, y), st["dtok"][t].double(), accumulate=True)
            grad -= p * a.index_add(0, i, st["dtok"][t].double())[:, None]
            if st["dent"] is not None:
                dH = torch.special.entr(p) - p * H[:, None]
                grad += dH * a.index_add(0, i, st["dent"][t].double())[:, None]
            dl[torch.tensor(some, device=DEV) if dense else slice(c, c + len(some))] = grad
    if dl is None:
        return {"tok": tok, "entropy": ent} if case["entropy"] else {"tok": tok}
    if dense:
        return {"dlogits": dl}
    return {"dlogits": dl, "row_index": torch.tensor(rows, dtype=torch.int32, device=DEV)}


def _exact_policy(st):
    """The definition term by term, its gradient by autograd."""
    case, L = st["case"], st["layout"]
    lp = st["logp"].double().requires_grad_(True)
    H = st["entropy"].double().requires_grad_(True) if st["entropy"] is not None else None
    counted = torch.zeros(L.T, dtype=torch.bool, device=DEV)
    counted[st["pos"]] = True if st["mask"] is None else st["mask"][st["pos"]].bool()
    slot = torch.full((L.T,), -1, dtype=torch.int64, device=DEV)
    slot[st["pos"]] = st["slot"]
    t = counted.nonzero()[:, 0]
    A = st["adv"].double()[t] if case["adv_tok"] else st["adv"].double().view(-1)[slot[t]]
    r = torch.exp(lp[t] - (st["old"].double()[t] if st["old"] is not None else lp[t].detach()))
    clipped = torch.clamp(r, 1 - CLIP_LOW, 1 + CLIP_HIGH)
    surr = torch.minimum(r * A, clipped * A)
    was = clipped * A < r * A
    if case["dual"]:
        floor = case["dual"] * A
        was = was | ((A < 0) & (surr < floor))
        surr = torch.where(A < 0, torch.maximum(surr, floor), surr)
    x = (st["ref"].double()[t] - lp[t]) if case["kl"] else None
    kl = {"": lambda: torch.zeros_like(r), "k1": lambda: -x, "k2": lambda: x ** 2 / 2,
          "k3": lambda: torch.expm1(x) - x}[case["kl"]]()
    if case["reduction"] == "token":
        w = torch.full_like(r, 1.0 / max(1, t.numel())).detach()
    elif case["reduction"] == "sum":
        w = torch.full_like(r, 1.0 / st["norm"]).detach()
    else:
        per = torch.bincount(slot[t], minlength=L.B * L.Kmax).double()
        w = (1.0 / per)[slot[t]] / (per > 0).sum()
    ent = H[t] if H is not None else torch.zeros_like(r)
    parts = [-(w * surr).sum(), (w * kl).sum(), (w * ent).sum(), (w * r).sum()]
    loss = parts[0] + st["kl_coef"] * parts[1] - st["ent_coef"] * parts[2]
    loss.backward()
    out = {"loss": loss.detach().reshape(1), "stats": torch.stack(parts).detach(),
           "counts": torch.stack([torch.tensor(t.numel(), device=DEV), was.sum()]).to(torch.int32), "dlogp": lp.grad}
    if H is not None:
        out["dentropy"] = H.grad
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("cross"):
        return _exact_cross(st)
    if case["kind"].startswith("tok"):
        return _exact_tok(st)
    return _exact_policy(st)
