"""float64 oracle of attention over capped scores, with a bias that falls with distance, under masks by
document, prefix and causality: forward, first backward and backward-over-backward, one batch entry and query
head at a time on its valid rows and keys alone, from the definitions

  s = tau q.k,  z = c tanh(s / c) - m_h |j - (p + i)|,  P = softmax of z over valid j
  u = 1 - tanh^2(s / c),  u' = -(2 / c) tanh(s / c) u           (1 and 0 without a cap)
  dZ = P (dP - D),  dS = u dZ
  F = u Fs,  Fs = tau (U_Q K^T + Q U_K^T),  St = u P (Pt - E) + u' dZ Fs

(alpha, Pt and E are those of bob_oracle.py, which this file shares no code with).  The mask is formed from the
documents and prefixes themselves, position by position.
"""
import numpy as np


def _f(x):
    return np.asarray(x, dtype=np.float64)


def valid_pairs(b, n, m, start, causal=False, documents=None, prefix_lens=None):
    """Which of n query rows from position `start` on see which of m keys, in entry b."""
    ok = np.zeros((n, m), bool)
    ids = None if documents is None else np.asarray(documents)[b]
    prefix = None if prefix_lens is None else int(np.asarray(prefix_lens)[b])
    spans = ids is not None or prefix is not None
    total = m if ids is None else len(ids)
    for i in range(n):
        p = start + i
        first, last = 0, m
        if ids is not None:
            if not 0 <= p < total or ids[p] < 0:
                continue
            first = p
            while first > 0 and ids[first - 1] == ids[p]:
                first -= 1
            last = p + 1
            while last < total and ids[last] == ids[p]:
                last += 1
        hi = last
        if causal or spans:
            hi = p + 1 if prefix is None else max(p + 1, min(first + max(prefix, 0), last))
        ok[i, max(first, 0):max(min(hi, m), 0)] = True
    return ok


def run(Q, K, V, tau, causal=False, cap=None, slopes=None, documents=None, prefix_lens=None, q_lens=None, kv_lens=None,
        q_starts=None, dO=None, UQ=None, UK=None, UV=None):
    """Dict of O, L; with dO also D, dQ, dK, dV; with UQ, UK, UV also alpha, E, Qt, Kt, Vt, dOt."""
    Q, K, V = _f(Q), _f(K), _f(V)
    B, H, Nq, d = Q.shape
    Hkv, Nk = K.shape[1:3]
    G = H // Hkv
    out = {"O": np.zeros_like(Q), "L": np.full((B, H, Nq), -np.inf)}
    if dO is not None:
        dO = _f(dO)
        out.update(D=np.zeros((B, H, Nq)), dQ=np.zeros_like(Q), dK=np.zeros_like(K), dV=np.zeros_like(V))
    if UQ is not None:
        UQ, UK, UV = _f(UQ), _f(UK), _f(UV)
        out.update(alpha=np.zeros((B, H, Nq)), E=np.zeros((B, H, Nq)), Qt=np.zeros_like(Q), dOt=np.zeros_like(Q),
                   Kt=np.zeros_like(K), Vt=np.zeros_like(V))
    for b in range(B):
        n = Nq if q_lens is None else int(np.clip(q_lens[b], 0, Nq))
        m = Nk if kv_lens is None else int(np.clip(kv_lens[b], 0, Nk))
        start = 0 if q_starts is None else int(q_starts[b])
        ok = valid_pairs(b, n, m, start, causal, documents, prefix_lens)
        if documents is not None or prefix_lens is not None:
            ok[(start + np.arange(n) < 0) | (start + np.arange(n) >= Nk)] = False  # positions without a span
        gap = np.abs(np.arange(m)[None, :] - (start + np.arange(n))[:, None]).astype(np.float64)
        some = ok.any(1)
        for h in range(H):
            kh = h // G
            q, k, v = Q[b, h, :n], K[b, kh, :m], V[b, kh, :m]
            s = tau * (q @ k.T)
            t = np.tanh(s / cap) if cap else np.zeros_like(s)
            u = 1 - t * t
            z = cap * t if cap else s
            if slopes is not None:
                z = z - float(slopes[h]) * gap
            top = np.where(some, np.where(ok, z, -np.inf).max(1, initial=-np.inf), 0.0)
            W = np.where(ok, np.exp(np.where(ok, z, 0.0) - top[:, None]), 0.0)
            total = np.where(some, W.sum(1), 1.0)
            P = W / total[:, None]
            out["O"][b, h, :n] = P @ v
            out["L"][b, h, :n] = np.where(some, top + np.log(total), -np.inf)
            if dO is None:
                continue
            do = dO[b, h, :n]
            dP = do @ v.T
            D = (P * dP).sum(1)
            dZ = P * (dP - D[:, None])
            dS = u * dZ
            out["D"][b, h, :n] = D
            out["dQ"][b, h, :n] = tau * (dS @ k)
            out["dK"][b, kh, :m] += tau * (dS.T @ q)
            out["dV"][b, kh, :m] += P.T @ do
            if UQ is None:
                continue
            uq, uk, uv = UQ[b, h, :n], UK[b, kh, :m], UV[b, kh, :m]
            Fs = tau * (uq @ k.T + q @ uk.T)
            F = u * Fs
            alpha = (P * F).sum(1)
            Pt = do @ uv.T + F * (dP - D[:, None]) - alpha[:, None] * dP
            E = (P * Pt).sum(1)
            St = u * P * (Pt - E[:, None])
            if cap:
                St = St - (2 / cap) * t * u * dZ * Fs
            Ph = P * (F - alpha[:, None])
            out["alpha"][b, h, :n], out["E"][b, h, :n] = alpha, E
            out["Qt"][b, h, :n] = tau * (St @ k + dS @ uk)
            out["Kt"][b, kh, :m] += tau * (St.T @ q + dS.T @ uq)
            out["Vt"][b, kh, :m] += Ph.T @ do
            out["dOt"][b, h, :n] = P @ uv + Ph @ v
    return out
