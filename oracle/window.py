"""fp64 window attention, its gradients, and how far 16-bit arithmetic may be off.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Every query is
evaluated over the list of keys that it sees, so nothing behind a mask enters
any sum.
"""
from __future__ import annotations

import numpy as np


def visible(i, q_len, kv_len, left, right, sinks):
    """Ascending key indices that query i of a sequence sees."""
    p = i + kv_len - q_len
    lo = 0 if left < 0 else max(p - left, 0)
    hi = kv_len - 1 if right < 0 else min(p + right, kv_len - 1)
    return np.array([j for j in range(max(hi + 1, 0)) if j >= lo or j < sinks], dtype=np.int64)


def mask_of(n_q, n_kv, q_len, kv_len, left, right, sinks):
    """bool [n_q, n_kv]: what each query sees."""
    m = np.zeros((n_q, n_kv), dtype=bool)
    for i in range(q_len):
        m[i, visible(i, q_len, kv_len, left, right, sinks)] = True
    return m


def window_attention(q, k, v, left, right, sinks, scale=None, q_len=None, kv_len=None, do=None):
    """O, LSE and, given do, gradients of [B, N, H, d] float64 arrays.

    Rows behind q_len or kv_len are NaN.  Returns a dict of o, lse, dq, dk, dv
    and for each of o, dq, dk, dv (as err_u, err_s) the sums that a rounding of
    the probabilities or score gradients, relative (u) or by a fixed step (s),
    is carried by; err_f likewise for the 32-bit arithmetic."""
    B, Nq, H, d = q.shape
    Nkv, Hkv = k.shape[1], k.shape[2]
    scale = d ** -0.5 if scale is None else scale
    full = lambda *s: np.full(s, np.nan)
    r = dict(o=full(B, Nq, H, d), lse=full(B, H, Nq))
    err = {x: full(B, Nq, H, d) for x in ("o_u", "o_s")}
    if do is not None:
        r.update(dq=full(B, Nq, H, d), dk=full(B, Nkv, Hkv, d), dv=full(B, Nkv, Hkv, d))
        err.update({x: full(B, Nq, H, d) for x in ("dq_u", "dq_s", "dq_f")})
        err.update({x: full(B, Nkv, Hkv, d) for x in ("dk_u", "dk_s", "dk_f", "dv_u", "dv_s")})
    for b in range(B):
        nq = Nq if q_len is None else int(q_len[b])
        nk = Nkv if kv_len is None else int(kv_len[b])
        m = mask_of(nq, nk, nq, nk, left, right, sinks)
        if do is not None:
            for x in ("dk", "dv"):
                r[x][b, :nk] = 0.0
            for x in ("dk_u", "dk_s", "dk_f", "dv_u", "dv_s"):
                err[x][b, :nk] = 0.0
        for h in range(H):
            kv = h // (H // Hkv)
            Q, K, V = q[b, :nq, h], k[b, :nk, kv].copy(), v[b, :nk, kv].copy()
            K[~m.any(0)] = 0.0  # keys that nobody sees
            V[~m.any(0)] = 0.0
            s = np.where(m, Q @ K.T * scale, -np.inf)
            top = s.max(1, initial=-np.inf, keepdims=True)
            e = np.where(m, np.exp(s - np.where(np.isinf(top), 0.0, top)), 0.0)
            z = e.sum(1, keepdims=True)
            p = e / np.where(z > 0, z, 1.0)
            with np.errstate(divide="ignore"):
                r["lse"][b, h, :nq] = (top + np.log(z))[:, 0]
            o = p @ V
            r["o"][b, :nq, h] = o
            carry_o = p @ np.abs(V)
            err["o_u"][b, :nq, h] = carry_o
            err["o_s"][b, :nq, h] = m.astype(float) @ np.abs(V)
            if do is None:
                continue
            g = do[b, :nq, h]
            dp = g @ V.T
            delta = (g * o).sum(1, keepdims=True)
            ds = p * (dp - delta)
            r["dq"][b, :nq, h] = scale * ds @ K
            r["dk"][b, :nk, kv] += scale * ds.T @ Q
            r["dv"][b, :nk, kv] += p.T @ g
            # delta is formed from an O that carries the forward pass's roundings
            e_delta = p * (np.abs(g) * (carry_o + np.abs(o))).sum(1, keepdims=True)
            f = p * (np.abs(g) @ np.abs(V).T) + e_delta
            M = m.astype(float)
            err["dq_u"][b, :nq, h] = scale * (np.abs(ds) + e_delta) @ np.abs(K)
            err["dq_s"][b, :nq, h] = scale * M @ np.abs(K)
            err["dq_f"][b, :nq, h] = scale * f @ np.abs(K)
            err["dk_u"][b, :nk, kv] += scale * (np.abs(ds) + e_delta).T @ np.abs(Q)
            err["dk_s"][b, :nk, kv] += scale * M.T @ np.abs(Q)
            err["dk_f"][b, :nk, kv] += scale * f.T @ np.abs(Q)
            err["dv_u"][b, :nk, kv] += p.T @ np.abs(g)
            err["dv_s"][b, :nk, kv] += M.T @ np.abs(g)
    r["err"] = err
    return r
