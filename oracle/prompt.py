"""Oracle for prompt attention over packed sequences.  TEST INFRASTRUCTURE ONLY.

The plain definition in float64: for row i of a sequence with L_q query and L_k key rows,
query head h and key/value head g = h // (H_q / H_kv), over the keys j that the row sees
(j <= i + L_k - L_q if causal, else all):

    s_j = scale * <q[i, h], k[j, g]>;  w = softmax(s);  O = sum_j w_j v[j, g];  lse = log sum_j exp(s_j)

A row that sees no key has O = 0 and lse = -inf.  Keys that a row does not see are not
touched at all.  Beside them two sums that bound the rounding errors of a 32-bit
computation: A = sum_j w_j |v[j]| per output element and N = scale * max_j sum_d |q_d k_jd|
per row.
"""
from __future__ import annotations

import numpy as np


def prompt_attention(q, k, v, cu_q, cu_k, scale: float, causal: bool = True):
    """q [T_q, H_q, D], k and v [T_k, H_kv, D] float64 (infinities and NaN allowed).
    Returns (O, lse, A, N); rows outside every sequence are NaN."""
    Tq, Hq, D = q.shape
    G = Hq // k.shape[1]
    O, A = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, N = np.full((Tq, Hq), np.nan), np.zeros((Tq, Hq))
    with np.errstate(invalid="ignore", over="ignore"):
        for b in range(len(cu_q) - 1):
            Lq, Lk = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
            for i in range(Lq):
                n = max(0, min(Lk, i + Lk - Lq + 1)) if causal else Lk
                for h in range(Hq):
                    row = (cu_q[b] + i, h)
                    if n == 0:
                        O[row], A[row], lse[row] = 0.0, 0.0, -np.inf
                        continue
                    kk, vv = k[cu_k[b]:cu_k[b] + n, h // G], v[cu_k[b]:cu_k[b] + n, h // G]
                    s = scale * (kk @ q[row])
                    N[row] = abs(scale) * float(np.max(np.abs(kk) @ np.abs(q[row])))
                    m = s.max()
                    e = np.exp(s - m)
                    w = e / e.sum()
                    O[row], A[row] = w @ vv, w @ np.abs(vv)
                    lse[row] = m + np.log(e.sum())
    return O, lse, A, N
