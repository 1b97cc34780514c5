"""float64 oracle of attention between sequences of two lengths with a bias by buckets
of relative position: forward, first backward and backward-over-backward, one batch
entry and query head at a time on its valid rows and keys alone, from the definitions

  S_ij = tau q_i . k_j + T[bucket(clamp(j - (s + i), -R, R)), h],  P = softmax over valid j
  dS = P (dP - D), dT[c] = sum of dS over bucket c
  F = tau (U_Q K^T + Q U_K^T) + U_T[bucket],  St = P (Pt - E), Tt[c] = sum of St over c

(the other closed forms are those of bob_oracle.py, which this file shares no code with).
An entry of -2^24 or less masks its bucket.  A row without a valid key has O = 0, L = -inf
and no part in anything else.
"""
import numpy as np

MASKED = -2.0 ** 24


def _safe(x):
    return np.asarray(x, dtype=np.float64)


def run(Q, K, V, tau, causal=False, table=None, buckets=None, q_lens=None, kv_lens=None, q_starts=None, dO=None,
        UQ=None, UK=None, UV=None, UT=None):
    """Dict of O, L; with dO also D, dQ, dK, dV, dT; with UQ, UK, UV also alpha, E, Qt, Kt, Vt, dOt, Tt."""
    Q, K, V = _safe(Q), _safe(K), _safe(V)
    B, H, Nq, d = Q.shape
    Hkv, Nk = K.shape[1:3]
    G = H // Hkv
    out = {"O": np.zeros_like(Q), "L": np.full((B, H, Nq), -np.inf)}
    if dO is not None:
        dO = _safe(dO)
        out.update(D=np.zeros((B, H, Nq)), dQ=np.zeros_like(Q), dK=np.zeros_like(K), dV=np.zeros_like(V))
    if UQ is not None:
        UQ, UK, UV = _safe(UQ), _safe(UK), _safe(UV)
        out.update(alpha=np.zeros((B, H, Nq)), E=np.zeros((B, H, Nq)), Qt=np.zeros_like(Q), dOt=np.zeros_like(Q),
                   Kt=np.zeros_like(K), Vt=np.zeros_like(V))
    if table is not None:
        table, buckets = _safe(table), np.asarray(buckets, dtype=np.int64)
        R = (len(buckets) - 1) // 2
        UT = np.zeros_like(table) if UT is None else _safe(UT)
        if dO is not None:
            out["dT"] = np.zeros_like(table)
        if UQ is not None:
            out["Tt"] = np.zeros_like(table)
    for b in range(B):
        n = Nq if q_lens is None else int(np.clip(q_lens[b], 0, Nq))
        m = Nk if kv_lens is None else int(np.clip(kv_lens[b], 0, Nk))
        s = 0 if q_starts is None else int(q_starts[b])
        step = np.arange(m)[None, :] - (s + np.arange(n))[:, None]
        valid = step <= 0 if causal else np.ones((n, m), bool)
        for h in range(H):
            kh = h // G
            q, k, v = Q[b, h, :n], K[b, kh, :m], V[b, kh, :m]
            S = tau * (q @ k.T)
            ok = valid
            if table is not None:
                c = np.clip(buckets[np.clip(step, -R, R) + R], 0, table.shape[0] - 1)
                bias = table[c, h]
                ok = valid & ~(bias <= MASKED)
                S = S + np.where(ok, bias, 0.0)
            some = ok.any(1)
            top = np.where(ok, S, -np.inf).max(1, initial=-np.inf)
            top = np.where(some, top, 0.0)
            W = np.where(ok, np.exp(np.where(ok, S, 0.0) - top[:, None]), 0.0)
            total = W.sum(1)
            P = W / np.where(some, total, 1.0)[:, None]
            out["O"][b, h, :n] = P @ v
            out["L"][b, h, :n] = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
            if dO is None:
                continue
            do = dO[b, h, :n]
            dP = do @ v.T
            D = (P * dP).sum(1)
            dS = P * (dP - D[:, None])
            out["D"][b, h, :n] = D
            out["dQ"][b, h, :n] = tau * (dS @ k)
            out["dK"][b, kh, :m] += tau * (dS.T @ q)
            out["dV"][b, kh, :m] += P.T @ do
            if table is not None:
                np.add.at(out["dT"][:, h], c, dS)
            if UQ is None:
                continue
            uq, uk, uv = UQ[b, h, :n], UK[b, kh, :m], UV[b, kh, :m]
            F = tau * (uq @ k.T + q @ uk.T)
            if table is not None:
                F = F + UT[c, h]
            alpha = (P * F).sum(1)
            Pt = do @ uv.T + F * (dP - D[:, None]) - alpha[:, None] * dP
            E = (P * Pt).sum(1)
            St = P * (Pt - E[:, None])
            Ph = P * (F - alpha[:, None])
            out["alpha"][b, h, :n], out["E"][b, h, :n] = alpha, E
            out["Qt"][b, h, :n] = tau * (St @ k + dS @ uk)
            out["Kt"][b, kh, :m] += tau * (St.T @ q + dS.T @ uq)
            out["Vt"][b, kh, :m] += Ph.T @ do
            out["dOt"][b, h, :n] = P @ uv + Ph @ v
            if table is not None:
                np.add.at(out["Tt"][:, h], c, St)
    return out
