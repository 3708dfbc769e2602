"""Plain fp64 CPU oracle of the attention's backward pass.  TEST INFRASTRUCTURE ONLY, as ``lazy_oracle``.

The forward pass is that of ``lazy_oracle.lazy_attention``: rotated queries and keys, s = scale q'.k' (+ ALiBi bias), a
key visible iff pos_k <= pos_q (causal), P = exp(s - lse).  For a loss L with dout = dL/dout, dlse = dL/dlse:

    delta_i = dout_i . out_i - dlse_i,   dS_ij = P_ij (dout_i . v_j - delta_i),   dv_j = sum_i P_ij dout_i,
    dq_i = scale R(-p_i) sum_j dS_ij k'_j,   dk_j = scale sum_i R(-p_j) dS_ij q'_i,

each stored key summing over every use.  With the gradients come first-order bounds of the error that an evaluation
makes which rounds rotated queries, rotated keys, P and dS to bf16 (relative error at most u = 2^-8 each), sums in
fp32 and rounds the result once:  a score is off by at most E_ij = 2 u scale sum_d |q'_id k'_jd|, so P by the factor
1 + E_ij, and every term of a sum by its own relative errors.

``operand`` asks for the bounds of an evaluation that keeps those operands more exactly, to a relative error of
``operand``: each as the sum of two bf16 numbers has 2^-17 (half a step of a half step), and products of two second parts
are left out, 2^-18; 2^-15 leaves as much again for fp32 sums over some hundred steps of 16 (2^-24 each).  Scores, biases
and their differences from the log-sum-exps are then bounded in fp32 too: 2^-22 (four roundings) of their magnitudes.
"""
from __future__ import annotations

import math

import numpy as np

from . import lazy_oracle as O

U = 2.0 ** -8  # largest relative error of a rounding to bf16


def _turn_back(x, pos, theta, pairing):
    return O.rotate(x, -np.asarray(pos), theta, pairing)


def _pair_sum(b, pairing):
    """Bound of a rotated vector's elements given bounds of the original's: both elements of a pair contribute."""
    if pairing == "half":
        h = b.shape[-1] // 2
        s = b[..., :h] + b[..., h:]
        return np.concatenate([s, s], -1)
    s = b[..., 0::2] + b[..., 1::2]
    return np.repeat(s, 2, -1)


def lazy_backward(q, q_start, q_pos0, pool_k, pool_v, chunks, chunk_start, hq, hkv, d, base, causal, out, lse, dout,
                  dlse=None, pairing="half", key_positions="nope", inv_freq=None, softmax_scale=0.0,
                  q_prerotated=False, operand=None):
    """Returns (dq, dk_pool, dv_pool) and their error bounds (same shapes); pools are flat fp64 arrays."""
    G = hq // hkv
    scale = softmax_scale or 1.0 / math.sqrt(d)
    alibi = pairing == "alibi"
    u = U if operand is None else operand
    theta = None if alibi else O.rope_frequencies(d, base, inv_freq)
    slopes = None
    if alibi:
        slopes = np.asarray(inv_freq, np.float64) if inv_freq is not None else \
            2.0 ** (-8.0 * (np.arange(hq) + 1) / hq)
    q, out, dout, lse = (np.asarray(x, np.float64) for x in (q, out, dout, lse))
    dq, bq = np.zeros(q.shape), np.zeros(q.shape)
    dk, bk = np.zeros(pool_k.size), np.zeros(pool_k.size)
    dv, bv = np.zeros(pool_v.size), np.zeros(pool_v.size)
    for r in range(len(q_start) - 1):
        a, b = int(q_start[r]), int(q_start[r + 1])
        lo, hi = int(chunk_start[r]), int(chunk_start[r + 1])
        K, V, kpos, offs = O.request_kv(pool_k, pool_v, chunks, lo, hi, hkv, d, with_offsets=True)
        qpos = int(q_pos0[r]) + np.arange(b - a)
        kr = kpos if key_positions == "nope" else offs
        if not alibi:
            K = O.rotate(K, kr, theta, pairing)
        Q = q[a:b].transpose(1, 0, 2)
        if not alibi and not q_prerotated:
            Q = O.rotate(Q, qpos, theta, pairing)
        hidden = (kpos[None, :] > qpos[:, None]) if causal else np.zeros((b - a, kpos.size), bool)
        GK, GV = np.zeros(K.shape), np.zeros(V.shape)
        BK, BV = np.zeros(K.shape), np.zeros(V.shape)
        for h in range(hq):
            g = h // G
            s = scale * Q[h] @ K[g].T
            if alibi:
                s = s + slopes[h] * (kpos[None, :] - qpos[:, None])
            L = lse[a:b, h]
            with np.errstate(invalid="ignore", over="ignore"):
                P = np.where(hidden | np.isneginf(L)[:, None], 0.0, np.exp(s - L[:, None]))
            E = 2 * u * scale * np.abs(Q[h]) @ np.abs(K[g]).T
            if operand is not None:
                bias = slopes[h] * np.abs(kpos[None, :] - qpos[:, None]) if alibi else 0.0
                E = E + 2.0 ** -22 * (np.abs(s) + np.where(np.isneginf(L), 0.0, np.abs(L))[:, None] + bias)
            delta = (dout[a:b, h] * out[a:b, h]).sum(-1)
            if dlse is not None:
                delta = delta - np.asarray(dlse, np.float64)[a:b, h]
            dP = dout[a:b, h] @ V[g].T
            dS = P * (dP - delta[:, None])
            # The inner sums are formed in fp32: 2^-24 a term, well below one part in 2^16 of their absolute sums.
            fine = 2.0 ** -16 * P * (np.abs(dout[a:b, h]) @ np.abs(V[g]).T +
                                     (np.abs(dout[a:b, h] * out[a:b, h])).sum(-1)[:, None])
            GV[g] += P.T @ dout[a:b, h]
            BV[g] += (P * (E + u)).T @ np.abs(dout[a:b, h])
            GK[g] += scale * dS.T @ Q[h]
            BK[g] += scale * (np.abs(dS) * (E + 2 * u) + fine).T @ np.abs(Q[h])
            gq = scale * dS @ K[g]
            gb = scale * (np.abs(dS) * (E + 2 * u) + fine) @ np.abs(K[g])
            if not alibi and not q_prerotated:
                gq, gb = _turn_back(gq, qpos, theta, pairing), _pair_sum(gb, pairing)
            dq[a:b, h] = gq
            bq[a:b, h] = gb
        if not alibi:
            GK, BK = _turn_back(GK, kr, theta, pairing), _pair_sum(BK, pairing)
        j = 0
        for i in range(lo, hi):
            c = chunks[i]
            n = int(c["len"])
            for dst, off, st, src in ((dk, "k_offset", "k_stride", GK), (bk, "k_offset", "k_stride", BK),
                                      (dv, "v_offset", "v_stride", GV), (bv, "v_offset", "v_stride", BV)):
                for g in range(hkv):
                    at = int(c[off]) + g * int(c[st]) * d
                    dst[at:at + n * d] += src[g, j:j + n].reshape(-1)
            j += n
    # Once rounded: half a step more.  1.25: second-order terms (products of two relative errors below 1/4).
    return (dq, dk, dv), tuple(1.25 * b + U * np.abs(x) + 1e-30 for b, x in ((bq, dq), (bk, dk), (bv, dv)))
