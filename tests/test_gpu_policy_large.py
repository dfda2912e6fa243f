"""GPU tests of cross attention and the token log-probs where offsets pass 2^31 elements, and of calls
from several host threads: results are those of the same rows alone, bit for bit."""
import threading

import pytest
import torch

from paper_2602_24082_amd import binding as pp
from paper_2602_24082_amd import workload as wl

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF = torch.bfloat16


@pytest.mark.parametrize("T", [3, 60])
def test_states_behind_two_billion_elements(T):
    """A row whose states lie past 2^31 elements, behind a row that nothing looks at; and the last keys of a
    row that is itself that long."""
    hq, hkv, d, far = 16, 8, 128, 2_200_000
    own = 150
    pack, alone = wl.make_pack([0, T], [[], []]), wl.make_pack([T], [[]])
    enc, enc1 = wl.make_enc([far, own]), wl.make_enc([own])
    q, do = wl.randn((T, hq, d), 1, BF, DEV), wl.randn((T, hq, d), 2, BF, DEV)
    k1, v1 = wl.randn((own, hkv, d), 3, BF, DEV), wl.randn((own, hkv, d), 4, BF, DEV)
    want = pp.pp_cross_attn_fwd(alone, enc1, q, k1, v1)
    grads = pp.pp_cross_attn_bwd(alone, enc1, q, k1, v1, *want, do)
    k, v = (torch.zeros(far + own, hkv, d, dtype=BF, device=DEV) for _ in range(2))
    assert far * hkv * d > 2 ** 31
    k[far:], v[far:] = k1, v1
    got = pp.pp_cross_attn_fwd(pack, enc, q, k, v)
    dq, dk, dv = pp.pp_cross_attn_bwd(pack, enc, q, k, v, *got, do)
    # The batches may split their walks differently: either result is off by half a step of 2^-8 in its terms
    # and in itself, 2 x 2^-8 (c + 1) of the greatest with c the terms' sum of magnitudes, less than 7 times
    # the greatest sum.  A wrong address gives other numbers altogether.
    near = lambda a, b: float((a.float() - b.float()).abs().max()) <= 2.0 ** -4 * float(b.float().abs().max())
    assert near(got[0], want[0]) and near(got[1], want[1]) and near(dq, grads[0])
    assert near(dk[far:], grads[1]) and near(dv[far:], grads[2])
    assert not dk[:far].any() and not dv[:far].any()
    # one row of all the states, every token at its last 150
    whole = wl.make_enc([far + own])
    begin = torch.full((T,), far, dtype=torch.int32, device=DEV)
    end = torch.full((T,), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    got = pp.pp_cross_attn_fwd(alone, whole, q, k, v, key_begin=begin, key_end=end)
    assert near(got[0], want[0]) and near(got[1], want[1])
    dq, dk, dv = pp.pp_cross_attn_bwd(alone, whole, q, k, v, *got, do, key_begin=begin, key_end=end)
    assert near(dq, grads[0]) and near(dk[far:], grads[1]) and near(dv[far:], grads[2])
    assert not dk[:far].any() and not dv[:far].any()


def test_logits_behind_two_billion_elements():
    V, P = 128256, 16800
    pack, alone = wl.make_pack([P, 3], [[], [5, 4]]), wl.make_pack([3], [[5, 4]])
    x = torch.empty(pack.total_tokens, V, dtype=BF, device=DEV)
    assert P * V > 2 ** 31
    x1 = wl.randn((12, V), 5, BF, DEV, 3.0)
    x[P:] = x1
    y1 = wl.randint((12,), V, 6, DEV)
    y = torch.cat([torch.zeros(P, dtype=torch.int32, device=DEV), y1])
    w1 = wl.randn((2, 12), 7, torch.float32, DEV)
    w = torch.cat([torch.zeros(2, P, device=DEV), w1], 1).contiguous()
    want = pp.pp_tok_logprob(alone, x1, y1, want_entropy=True)
    for a, b in zip(pp.pp_tok_logprob(pack, x, y, want_entropy=True), want):
        assert torch.equal(a[P:], b) and not a[:P].any()
    rows, idx = pp.pp_tok_logprob_bwd_rows(pack, x, y, w[0], w[1])
    rows1, idx1 = pp.pp_tok_logprob_bwd_rows(alone, x1, y1, w1[0], w1[1])
    assert torch.equal(rows, rows1) and torch.equal(idx, idx1 + P)
    dense = pp.pp_tok_logprob_bwd(pack, x, y, w[0], w[1])
    assert torch.equal(dense[P:], pp.pp_tok_logprob_bwd(alone, x1, y1, w1[0], w1[1])) and not dense[:P].any()


def test_two_host_threads():
    """Calls of two threads at once, each on a stream of its own, with records of both sizes."""
    def case(seed, rows):
        pack = wl.make_pack([40, 9, 70] * rows, [[30, 8], [1], [64, 3]] * rows)
        enc = wl.make_enc([120, 0, 500] * rows)
        T = pack.total_tokens
        return dict(pack=pack, enc=enc, q=wl.randn((T, 8, 64), seed, BF, DEV), k=wl.randn((enc.total_states, 2, 64), seed + 1, BF, DEV),
                    v=wl.randn((enc.total_states, 2, 64), seed + 2, BF, DEV), do=wl.randn((T, 8, 64), seed + 3, BF, DEV),
                    logits=wl.randn((T, 400), seed + 4, BF, DEV), tokens=wl.randint((T,), 400, seed + 5, DEV),
                    adv=wl.randn((3 * rows, 2), seed + 6, torch.float32, DEV))

    def run(c):
        o, lse = pp.pp_cross_attn_fwd(c["pack"], c["enc"], c["q"], c["k"], c["v"])
        g = pp.pp_cross_attn_bwd(c["pack"], c["enc"], c["q"], c["k"], c["v"], o, lse, c["do"])
        tok, ent = pp.pp_tok_logprob(c["pack"], c["logits"], c["tokens"], want_entropy=True)
        loss, stats, counts, dlp, dent = pp.pp_policy_loss(c["pack"], tok, c["adv"], entropy=ent, ent_coef=0.1, reduction="seq")
        rows, idx = pp.pp_tok_logprob_bwd_rows(c["pack"], c["logits"], c["tokens"], dlp, dent)
        return o, lse, *g, tok, ent, loss, stats, counts, rows, idx

    cases = [case(10, 1), case(20, 60)]
    want = [run(c) for c in cases]
    torch.cuda.synchronize()
    bad = []

    def work(c, w):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            for _ in range(20):
                got = run(c)
                s.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, w)):
                    bad.append(len(c["adv"]))

    threads = [threading.Thread(target=work, args=a) for a in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
