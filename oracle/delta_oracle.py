"""fp64 oracle of the gated delta rule and of the norms between two blocks, from their definitions, in numpy.

Delta rule, token by token, per batch b and value head h (key head h // (H / Hk)), S [d,e]:
    S_t = exp(g_t) (S_{t-1} - beta_t k_t (k_t^T S_{t-1})) + beta_t k_t v_t^T,    o_t = scale S_t^T q_t
and its adjoint step by step (no chunks, no inverses).  Arrays are heads first: q, k [B,Hk,N,d], v [B,H,N,e], g, beta [B,H,N].
"""
import numpy as np


def _f64(x):
    return np.asarray(x.detach().cpu().double().numpy() if hasattr(x, "detach") else x, dtype=np.float64)


def _shared(x, H):
    return np.repeat(x, H // x.shape[1], axis=1)


def _step(S, k, v, a, beta):
    """The decayed state, what the state holds less than v for k, the state after the token."""
    S = a[..., None, None] * S
    r = v - np.einsum("bhi,bhij->bhj", k, S)
    return S, r, S + np.einsum("bhi,bhj->bhij", k, beta[..., None] * r)


def delta_fwd(q, k, v, g, beta, scale=1.0, kv_in=None):
    """o [B,H,N,e] and the state after the last token."""
    q, k, v, g, beta = (_f64(x) for x in (q, k, v, g, beta))
    B, H, N, e = v.shape
    q, k = _shared(q, H), _shared(k, H)
    S = np.zeros((B, H, k.shape[3], e)) if kv_in is None else _f64(kv_in).copy()
    o, a = np.empty((B, H, N, e)), np.exp(g)
    for t in range(N):
        S = _step(S, k[:, :, t], v[:, :, t], a[:, :, t], beta[:, :, t])[2]
        o[:, :, t] = scale * np.einsum("bhij,bhi->bhj", S, q[:, :, t])
    return o, S


def delta_bwd(q, k, v, g, beta, do, scale=1.0, kv_in=None, grad_kv_out=None):
    """dq, dk (summed over the heads that share them), dv, dg, dbeta, and the gradient of kv_in."""
    q, k, v, g, beta, do = (_f64(x) for x in (q, k, v, g, beta, do))
    B, H, N, e = v.shape
    Hk, d = k.shape[1], k.shape[3]
    q, k = _shared(q, H), _shared(k, H)
    a = np.exp(g)
    S = np.zeros((B, H, d, e)) if kv_in is None else _f64(kv_in).copy()
    entering = []
    for t in range(N):
        entering.append(S)
        S = _step(S, k[:, :, t], v[:, :, t], a[:, :, t], beta[:, :, t])[2]
    E = np.zeros_like(S) if grad_kv_out is None else _f64(grad_kv_out).copy()
    dq, dk, dv, dg, dbeta = (np.empty_like(x) for x in (q, k, v, g, beta))
    for t in range(N - 1, -1, -1):
        kt, qt, bt = k[:, :, t], q[:, :, t], beta[:, :, t, None]
        before, r, S = _step(entering[t], kt, v[:, :, t], a[:, :, t], beta[:, :, t])
        dq[:, :, t] = scale * np.einsum("bhij,bhj->bhi", S, do[:, :, t])
        E = E + scale * np.einsum("bhi,bhj->bhij", qt, do[:, :, t])
        dn = np.einsum("bhi,bhij->bhj", kt, E)          # of beta r
        dv[:, :, t] = bt * dn
        dbeta[:, :, t] = np.sum(dn * r, -1)
        dk[:, :, t] = np.einsum("bhij,bhj->bhi", E, bt * r) - np.einsum("bhij,bhj->bhi", before, dv[:, :, t])
        E = E - np.einsum("bhi,bhj->bhij", kt, dv[:, :, t])  # of the decayed state
        dg[:, :, t] = np.sum(before * E, (-2, -1))
        E = a[:, :, t, None, None] * E
    dq, dk = (x.reshape(B, Hk, H // Hk, N, d).sum(2) for x in (dq, dk))
    return dq, dk, dv, dg, dbeta, E


ACT = {0: (lambda u: u, lambda u: np.ones_like(u)),
       1: (lambda u: 1 / (1 + np.exp(-u)), lambda u: 1 / (1 + np.exp(-u)) / (1 + np.exp(u))),
       2: (lambda u: u / (1 + np.exp(-u)), lambda u: (1 + u / (1 + np.exp(u))) / (1 + np.exp(-u)))}


def _norm(a, eps):
    m = np.mean(a * a, -1, keepdims=True) + eps
    r = np.where(m == 0, 0.0, 1 / np.sqrt(np.where(m == 0, 1.0, m)))
    return a * r, r


def block_norm_fwd(x, y, u=None, w_post=None, s=None, w_pre=None, eps=0.0, gate=0, post_norm=True):
    """h and n."""
    x, y = _f64(x), _f64(y)
    z = _norm(y, eps)[0] if post_norm else y
    z = z * (1.0 if w_post is None else _f64(w_post)) * (1.0 if u is None else ACT[gate][0](_f64(u)))
    h = x + z * (1.0 if s is None else _f64(s))
    return h, _norm(h, eps)[0] * (1.0 if w_pre is None else _f64(w_pre))


def block_norm_bwd(x, y, u, w_post, s, w_pre, dh, dn, eps=0.0, gate=0, post_norm=True):
    """dx, dy, du (None without u), dw_post, ds, dw_pre of <h, dh> + <n, dn>."""
    x, y = _f64(x), _f64(y)
    w_post, s, w_pre = (np.ones(x.shape[-1]) if w is None else _f64(w) for w in (w_post, s, w_pre))
    uu = None if u is None else _f64(u)
    act, slope = (1.0, 0.0) if u is None else (ACT[gate][0](uu), ACT[gate][1](uu))
    yn, ry = _norm(y, eps) if post_norm else (y, np.ones((*y.shape[:-1], 1)))
    hn, rh = _norm(x + s * yn * w_post * act, eps)
    dx = np.zeros_like(x) if dh is None else _f64(dh).copy()
    dw_pre = np.zeros(x.shape[-1])
    if dn is not None:
        p = _f64(dn) * w_pre
        dx = dx + rh * (p - hn * np.mean(p * hn, -1, keepdims=True))
        dw_pre = np.sum(_f64(dn) * hn, 0)
    p = dx * s * act * w_post
    dy = ry * (p - yn * np.mean(p * yn, -1, keepdims=True)) if post_norm else p
    du = None if u is None else dx * s * yn * w_post * slope
    return dx, dy, du, np.sum(dx * s * act * yn, 0), np.sum(dx * yn * w_post * act, 0), dw_pre
