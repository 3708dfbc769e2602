"""Plain fp64 CPU oracle of eviction by accumulated attention weight.  TEST INFRASTRUCTURE ONLY, as ``lazy_oracle``."""
from __future__ import annotations

import math

import numpy as np

from . import lazy_oracle as O


def key_weights(q, q_start, q_pos0, pool_k, chunks, chunk_start, hq, hkv, d, base, causal, lse, pairing="half",
                key_positions="nope", inv_freq=None, softmax_scale=0.0, q_prerotated=False):
    """Per request: [keys] sums over query rows and heads of exp(s - lse), and bounds of the error of an evaluation that
    keeps rotated queries and keys as sums of two bf16 numbers each and multiplies them without the two second parts'
    product.  With u = 2^-8 per rounding, every product q'k' is off by at most u^2 for each operand's rest and u^2 for
    what is left out, 3 2^-16; sums of at most 384 products in fp32 add 384 2^-24 = 1.5 2^-16 and angles good to 2e-7
    under 0.1 2^-16: together 4.6 2^-16 = 1.15 2^-14 of scale sum |q'||k'|.  The exponent's other part, lse (below 64
    here), is rounded to fp32 twice: 2^-17.  Sums of probabilities: 2^-16 covers 256 additions of 2^-24 each."""
    G = hq // hkv
    scale = softmax_scale or 1.0 / math.sqrt(d)
    alibi = pairing == "alibi"
    theta = None if alibi else O.rope_frequencies(d, base, inv_freq)
    slopes = (np.asarray(inv_freq, np.float64) if inv_freq is not None else 2.0 ** (-8.0 * (np.arange(hq) + 1) / hq)) \
        if alibi else None
    q, lse = np.asarray(q, np.float64), np.asarray(lse, np.float64)
    got = []
    for r in range(len(q_start) - 1):
        a, b = int(q_start[r]), int(q_start[r + 1])
        K, _, kpos, offs = O.request_kv(pool_k, pool_k, chunks, int(chunk_start[r]), int(chunk_start[r + 1]), hkv, d,
                                        with_offsets=True)
        qpos = int(q_pos0[r]) + np.arange(b - a)
        if not alibi:
            K = O.rotate(K, kpos if key_positions == "nope" else offs, theta, pairing)
        Q = q[a:b].transpose(1, 0, 2)
        if not alibi and not q_prerotated:
            Q = O.rotate(Q, qpos, theta, pairing)
        w, bound = np.zeros(kpos.size), np.zeros(kpos.size)
        for h in range(hq):
            s = scale * Q[h] @ K[h // G].T
            if alibi:
                s = s + slopes[h] * (kpos[None, :] - qpos[:, None])
            L = lse[a:b, h][:, None]
            hidden = np.isneginf(L) | ((kpos[None, :] > qpos[:, None]) if causal else False)
            with np.errstate(invalid="ignore", over="ignore"):
                P = np.where(hidden, 0.0, np.exp(s - L))
            E = 1.25 * 2.0 ** -14 * scale * np.abs(Q[h]) @ np.abs(K[h // G]).T + 2.0 ** -17
            w += P.sum(0)
            bound += (P * (E + 2.0 ** -16)).sum(0)
        got.append((w, bound + 1e-30))
    return got


def select(weights, budget, sink, recent):
    """Ascending indices of the kept keys of one request (python loop over a full sort)."""
    n = len(weights)
    if budget >= n:
        return list(range(n))

    def rank(j):
        w = float(weights[j])
        guarded = j < sink or j >= n - recent
        return (not guarded, 0.0 if guarded else (math.inf if math.isnan(w) else -w), not guarded and math.isnan(w), j)

    return sorted(sorted(range(n), key=rank)[:budget])
