"""Element-by-element bounds on the error of cross attention's results.

Let u be the half step of the type that the probabilities, dS and the results are rounded
to (bf16: 2^-8 relative to the value; fp32 inputs round nothing but sums: u = 2^-24) and
e = 2^-24 an fp32 rounding.  From the operator's formulas, with A.B for sums of |a| |b|:

  score     s = tau q.k, d products summed in fp32, then scaled: |err| <= (d + 4) e tau |q|.|k|
  P         exp2 of an fp32 argument of size |s - m|: relative err of P
                r = err(s) + 4 e (|s| + |m|) + 2^-21   (the hardware's exp2 and log2: a few ulps)
            and as much again through lse, m the row's greatest score
  O         P rounded, N products summed:  (u + 2 r' + N e) P.|v| + u |O|, r' the row's greatest r
  lse       r' + N e + 4 e |lse|
  delta     dO . O with O as stored:  dO.err(O) + d e dO.|O|
  dS        P (dP - delta), rounded:  |dS| (u + 2 r' + 4 e) + P (d e |dO|.|v| + err(delta))
  dQ        tau (err(dS) + N e |dS|).|k| + u |dQ|
  dK, dV    the same sums over the M rows of the kv-head's group

The backward pass is given the forward's o and lse of the library, so their errors enter
as above.  Everything is formed in 64 bits from the reference's own values.
"""
import numpy as np

E = 2.0 ** -24


def bounds(args, enc_start, enc_len, q, k, v, dout, vis, u, scale=None):
    """Allowed |error| of (o, lse, dq, dk, dv), arrays of the results' shapes."""
    row_start = args[0]
    T, hq, d = q.shape
    G = hq // k.shape[1]
    tau = 1.0 / np.sqrt(d) if scale is None else scale
    bo, bl = np.zeros((T, hq, d)), np.zeros((hq, T))
    bq, bk, bv = np.zeros((T, hq, d)), np.zeros(k.shape), np.zeros(v.shape)
    for b, see in enumerate(vis):
        t0, e0, n = int(row_start[b]), int(enc_start[b]), int(enc_len[b])
        some = see.any(axis=1)
        rows, see = t0 + np.nonzero(some)[0], see[some]
        if len(rows) == 0:
            continue
        M = len(rows) * G + 64
        for h in range(hq):
            g = h // G
            kh, vh, qh, gh = k[e0:e0 + n, g], v[e0:e0 + n, g], q[rows, h], dout[rows, h]
            ak, av, aq, ag = np.abs(kh), np.abs(vh), np.abs(qh), np.abs(gh)
            s = np.where(see, tau * (qh @ kh.T), -np.inf)
            m = s.max(axis=1, keepdims=True)
            P = np.exp(s - m)
            P /= P.sum(axis=1, keepdims=True)
            fin = np.where(see, s, 0.0)
            r = np.where(see, (d + 4) * E * tau * (aq @ ak.T) + 4 * E * (np.abs(fin) + np.abs(m)) + 2.0 ** -21, 0.0)
            r = r.max(axis=1, keepdims=True)
            O = P @ vh
            Pv = P @ av
            eO = (u + 2 * r + (n + 64) * E) * Pv + u * np.abs(O)
            bo[rows, h] = eO
            lse = m[:, 0] + 0.0
            bl[h, rows] = r[:, 0] + (n + 64) * E + 4 * E * (np.abs(lse) + np.log(n + 1))
            dP = gh @ vh.T
            delta = (P * dP).sum(axis=1, keepdims=True)
            dS = P * (dP - delta)
            ed = (ag * eO).sum(axis=1, keepdims=True) + d * E * (ag * np.abs(O)).sum(axis=1, keepdims=True)
            # terms of dS and delta cancel: their own roundings are relative to the parts
            eS = np.abs(dS) * (u + 2 * r + 4 * E) + P * (d * E * (ag @ av.T) + ed + 2 * E * (np.abs(dP) + np.abs(delta)))
            bq[rows, h] = tau * ((eS + (n + 64) * E * np.abs(dS)) @ ak) + u * np.abs(tau * dS @ kh)
            bk[e0:e0 + n, g] += tau * ((eS + M * E * np.abs(dS)).T @ aq)
            eP = P * (u + 2 * r)
            bv[e0:e0 + n, g] += (eP + M * E * P).T @ ag
    return bo, bl, bq, bk, bv


def allow(bound, ref, u, room=1e-30):
    """The bound of a sum over heads, with its own rounding to the result's type."""
    return bound * (1 + 1e-6) + u * np.abs(ref) + room
