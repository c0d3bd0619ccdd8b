"""The gated delta rule in fp64, one token after another: the definition of the operator, and its gradients by the chain rule
through the recurrence.  Arrays: Q, K (B, Hk, N, dk), V (B, H, N, dv), g, beta (B, H, N), states (B, H, dk, dv)."""
import numpy as np


def _heads(X, H):
    return np.repeat(X, H // X.shape[1], axis=1)


def _token(S, k, v, g, beta):
    """(decayed state, error row, new state)"""
    Sd = np.exp(g)[..., None, None] * S
    e = v - np.einsum("bhk,bhkv->bhv", k, Sd)
    return Sd, e, Sd + k[..., :, None] * (beta[..., None] * e)[..., None, :]


def forward(Q, K, V, g, beta, scale, state=None):
    """Outputs (B, H, N, dv) and the state behind the last token."""
    H, N = V.shape[1], V.shape[2]
    Q, K, V, g, beta = (np.asarray(x, dtype=np.float64) for x in (_heads(Q, H), _heads(K, H), V, g, beta))
    S = np.zeros(V.shape[:2] + (K.shape[-1], V.shape[-1])) if state is None else np.asarray(state, dtype=np.float64)
    O = np.empty_like(V)
    for t in range(N):
        S = _token(S, K[:, :, t], V[:, :, t], g[:, :, t], beta[:, :, t])[2]
        O[:, :, t] = scale * np.einsum("bhk,bhkv->bhv", Q[:, :, t], S)
    return O, S


def backward(Q, K, V, g, beta, scale, dO, state=None, dstate=None):
    """dQ, dK, dV, dg, dbeta and the cotangent of the first state."""
    H, Hk, N = V.shape[1], Q.shape[1], V.shape[2]
    Q, K, V, g, beta, dO = (np.asarray(x, dtype=np.float64) for x in (_heads(Q, H), _heads(K, H), V, g, beta, dO))
    S = np.zeros(V.shape[:2] + (K.shape[-1], V.shape[-1])) if state is None else np.asarray(state, dtype=np.float64)
    block, marks = 32, []
    for t in range(N):
        if t % block == 0:
            marks.append(S)
        S = _token(S, K[:, :, t], V[:, :, t], g[:, :, t], beta[:, :, t])[2]
    dS = np.zeros_like(S) if dstate is None else np.asarray(dstate, dtype=np.float64)
    dQ, dK, dV, dg, db = (np.empty_like(x) for x in (Q, K, V, g, beta))
    for c in range(len(marks) - 1, -1, -1):
        S, kept = marks[c], []
        for t in range(c * block, min(N, (c + 1) * block)):
            kept.append(_token(S, K[:, :, t], V[:, :, t], g[:, :, t], beta[:, :, t]))
            S = kept[-1][2]
        for t in range(min(N, (c + 1) * block) - 1, c * block - 1, -1):
            Sd, e, S = kept[t - c * block]
            q, k, do, b = Q[:, :, t], K[:, :, t], dO[:, :, t], beta[:, :, t]
            dQ[:, :, t] = scale * np.einsum("bhkv,bhv->bhk", S, do)
            dS = dS + scale * q[..., None] * do[..., None, :]
            du = np.einsum("bhk,bhkv->bhv", k, dS)
            de = b[..., None] * du
            dV[:, :, t] = de
            db[:, :, t] = (e * du).sum(-1)
            dK[:, :, t] = np.einsum("bhkv,bhv->bhk", dS, b[..., None] * e) - np.einsum("bhkv,bhv->bhk", Sd, de)
            dS = dS - k[..., None] * de[..., None, :]
            dg[:, :, t] = (Sd * dS).sum((-1, -2))
            dS = np.exp(g[:, :, t])[..., None, None] * dS
    dQ, dK = (x.reshape(x.shape[0], Hk, H // Hk, N, x.shape[-1]).sum(2) for x in (dQ, dK))
    return dQ, dK, dV, dg, db, dS
