"""GPU tests of the policy-optimisation operators together, as a training step calls them:
cross attention to encoder states, an output head, token log-probs and entropies, the
clipped loss, the logits' gradient and back through the cross attention; the same step on
another stream and captured into a graph.

The chain is checked against autograd in 64 bits.  Its fp32 operators are exact to a few
1e-6 of a result's size (test_gpu_cross.py, test_gpu_policy.py hold each to its own bound);
what they pass on is O(1), so the chain's results are held to 1e-4 of their greatest."""
import numpy as np
import pytest
import torch

from oracle import pp_oracle as orc
from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HQ, HKV, D, V = 4, 2, 64, 300
KW = dict(clip_low=0.2, clip_high=0.28, kl_coef=0.05, ent_coef=0.01, reduction="seq")


def _inputs(seed, dtype=torch.float32):
    pack = wl.make_pack([20, 7, 3], [[9, 30, 1], [0, 12], [5, 5, 5]], pad=[2, 0, 1])
    enc = wl.make_enc([70, 0, 33], pad=[0, 3, 5])
    T = pack.total_tokens
    r = lambda shape, i, sigma=1.0, t=dtype: wl.randn(shape, seed + i, t, DEV, sigma=sigma)
    x = {"q": r((T, HQ, D), 0), "k": r((enc.total_states, HKV, D), 1), "v": r((enc.total_states, HKV, D), 2),
         "w": r((HQ * D, V), 3, 0.3), "tokens": wl.randint((T,), V, seed + 4, DEV), "adv": r((3, 3), 5, t=torch.float32),
         "drift": r((T,), 6, 0.2, torch.float32), "ref": r((T,), 7, 0.2, torch.float32),
         "mask": (r((T,), 8, t=torch.float32) > -1).to(torch.uint8)}
    begin = torch.zeros(T, dtype=torch.int32, device=DEV)
    end = torch.full((T,), 50, dtype=torch.int32, device=DEV)
    end[3], begin[9] = 0, 60  # see nothing
    return pack, enc, x, begin, end


def _step(pack, enc, x, begin, end, old=None, ref=None):
    o, lse = pp.pp_cross_attn_fwd(pack, enc, x["q"], x["k"], x["v"], key_begin=begin, key_end=end)
    h = o.view(len(o), -1)
    logits = h @ x["w"]
    tok, ent = pp.pp_tok_logprob(pack, logits, x["tokens"], want_entropy=True)
    # a rollout's own log-probs and a reference's, a little off this policy's
    old = tok + x["drift"] if old is None else old
    ref = tok + x["ref"] if ref is None else ref
    loss, stats, counts, dtok, dent = pp.pp_policy_loss(pack, tok, x["adv"], logp_old=old, logp_ref=ref, entropy=ent,
                                                        mask=x["mask"], **KW)
    rows, idx = pp.pp_tok_logprob_bwd_rows(pack, logits, x["tokens"], dtok, dent)
    dlogits = pp.pp_tok_logprob_bwd(pack, logits, x["tokens"], dtok, dent)
    do = (dlogits @ x["w"].T).view(o.shape)
    dw = h.T @ dlogits
    dq, dk, dv = pp.pp_cross_attn_bwd(pack, enc, x["q"], x["k"], x["v"], o, lse, do, key_begin=begin, key_end=end)
    return {"loss": loss, "stats": stats, "counts": counts, "rows": rows, "idx": idx, "dlogits": dlogits, "dw": dw, "dq": dq,
            "dk": dk, "dv": dv, "tok": tok, "ent": ent}, old, ref


def test_step_against_autograd():
    pack, enc, x, begin, end = _inputs(700)
    got, old, ref = _step(pack, enc, x, begin, end)
    c = {n: t.double().cpu() for n, t in x.items()}
    leaf = {n: c[n].requires_grad_(True) for n in ("q", "k", "v", "w")}
    T = pack.total_tokens
    outs = []
    vis = orc.cross_visible(*pack.oracle_args(), enc.enc_len, begin.cpu().numpy(), end.cpu().numpy())
    for b, see in enumerate(vis):
        t = slice(int(pack.row_start[b]), int(pack.row_start[b + 1]))
        e = slice(int(enc.enc_start[b]), int(enc.enc_start[b] + enc.enc_len[b]))
        k, v = (leaf[n][e].repeat_interleave(HQ // HKV, 1) for n in ("k", "v"))
        see = torch.tensor(see)
        s = torch.einsum("thd,ehd->hte", leaf["q"][t], k) / np.sqrt(D)
        some = see.any(1)
        p = torch.zeros_like(s)
        if see.shape[1]:
            p = torch.where(some[:, None], torch.softmax(s.masked_fill(~see & some[:, None], -np.inf), 2), 0.0)
        outs.append(torch.einsum("hte,ehd->thd", p, v))
    logits = torch.cat(outs).reshape(T, -1) @ leaf["w"]
    logits.retain_grad()
    toks = orc.response_tokens(*pack.oracle_args())
    row, at = (torch.tensor([y[i] for y in toks]) for i in (0, 1))
    lp = torch.log_softmax(logits[row], 1)
    tok = lp.gather(1, c["tokens"][at].long()[:, None])[:, 0]
    ent = -(lp.exp() * lp).sum(1)
    keep = c["mask"][at] != 0
    A = torch.stack([c["adv"][y[2], y[3]] for y in toks])
    ratio = torch.exp(tok - old.double().cpu()[at])
    xr = ref.double().cpu()[at] - tok
    term = (-torch.minimum(ratio * A, ratio.clamp(0.8, 1.28) * A) + 0.05 * (torch.exp(xr) - 1 - xr) - 0.01 * ent)
    per = {}
    for y, on in zip(toks, keep.tolist()):
        if on:
            per[y[2:]] = per.get(y[2:], 0) + 1
    w = torch.tensor([1.0 / (len(per) * per[y[2:]]) if on else 0.0 for y, on in zip(toks, keep.tolist())])
    loss = (w * term).sum()
    loss.backward()
    close = lambda g, r: float((g.double().cpu() - r).abs().max()) <= 1e-4 * float(r.abs().max())
    assert abs(float(got["loss"]) - float(loss.detach())) <= 1e-5 and got["counts"].tolist()[0] == int(keep.sum())
    assert close(got["tok"][at.to(DEV)], tok.detach()) and close(got["ent"][at.to(DEV)], ent.detach())
    assert close(got["dlogits"], logits.grad) and torch.equal(got["rows"], got["dlogits"][got["idx"].long()])
    for n in ("q", "k", "v", "w"):
        assert close(got["d" + n], leaf[n].grad), n


def test_step_on_another_stream():
    pack, enc, x, begin, end = _inputs(720, torch.bfloat16)
    want, old, ref = _step(pack, enc, x, begin, end)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got, _, _ = _step(pack, enc, x, begin, end, old, ref)
    s.synchronize()
    for n in want:
        assert torch.equal(want[n], got[n]), n


@pytest.mark.parametrize("rows", [1, 40])
def test_captured_calls_replay(rows):
    """Every operator captured with its own workspace and replayed on new inputs between eager calls, which
    refill the staging buffers: with records that ride in launch arguments, and with many of them."""
    pack = wl.make_pack([20, 7] * rows, [[9, 30, 1], [0, 12]] * rows, pad=[2, 0] * rows)
    enc = wl.make_enc([70, 33] * rows, pad=[0, 3] * rows)
    T, vocab = pack.total_tokens, 200
    other = wl.make_pack([11] * 2 * rows, [[5, 6, 7]] * 2 * rows), wl.make_enc([15] * 2 * rows)
    x = {"q": (T, HQ, D), "k": (enc.total_states, HKV, D), "v": (enc.total_states, HKV, D), "do": (T, HQ, D), "lp": (T,),
         "old": (T,), "adv": (2 * rows, 3), "logits": (T, vocab), "dtok": (T,), "dent": (T,)}
    x = {n: torch.randn(shape, device=DEV) for n, shape in x.items()}
    tokens = wl.randint((T,), vocab, 5, DEV)
    mask = (torch.rand(T, device=DEV) > 0.2).to(torch.uint8)

    def workspaces(pack, enc):
        f, b = pp.pp_cross_workspace_size(pack, enc, HQ, HKV, D, pp.PP_FP32)
        n = [f, b, pp.pp_policy_workspace_size(pack)] + [pp.pp_workspace_size(pack, vocab=vocab, fwd=False, bwd=False,
                                                                             logprob=True, loss=False)[2]] * 3
        return [torch.empty(max(i, 1), dtype=torch.uint8, device=DEV) for i in n]

    def calls(pack, enc, x, tokens, mask, ws):
        o, lse = pp.pp_cross_attn_fwd(pack, enc, x["q"], x["k"], x["v"], ws=ws[0])
        grads = pp.pp_cross_attn_bwd(pack, enc, x["q"], x["k"], x["v"], o, lse, x["do"], ws=ws[1])
        loss, stats, counts, dlp, _ = pp.pp_policy_loss(pack, x["lp"], x["adv"], logp_old=x["old"], mask=mask, reduction="seq",
                                                        ws=ws[2])
        tok, ent = pp.pp_tok_logprob(pack, x["logits"], tokens, want_entropy=True, ws=ws[3])
        dl = pp.pp_tok_logprob_bwd(pack, x["logits"], tokens, x["dtok"], x["dent"], ws=ws[4])
        dr, idx = pp.pp_tok_logprob_bwd_rows(pack, x["logits"], tokens, x["dtok"], x["dent"], ws=ws[5])
        return (o, lse, *grads, loss, stats, counts, dlp, tok, ent, dl, dr, idx)

    ws, ws2 = workspaces(pack, enc), workspaces(*other)
    n2 = other[0].total_tokens
    y = {n: torch.randn((n2, *t.shape[1:]) if len(t) == T else (2 * rows, 3) if n == "adv" else
                        (other[1].total_states, HKV, D), device=DEV) for n, t in x.items()}
    calls(pack, enc, x, tokens, mask, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(pack, enc, x, tokens, mask, ws)
    for i in range(3):
        for _ in range(20):
            calls(*other, y, tokens[:n2] if n2 <= T else torch.zeros(n2, dtype=torch.int32, device=DEV),
                  torch.ones(n2, dtype=torch.uint8, device=DEV), ws2)
        for n, t in x.items():
            t.copy_(torch.randn(t.shape, generator=torch.Generator(DEV).manual_seed(i), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip(out, calls(pack, enc, x, tokens, mask, [None] * 6)):
            assert torch.equal(a, c), i
