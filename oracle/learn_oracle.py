"""Float64 oracle of the learner's operators (test infrastructure only, plain numpy; shares no code with the library): the gated linear
recurrence, the clipped policy loss and AdamW, each with what its gradient or its stored state is."""
from __future__ import annotations

import numpy as np


def _sigmoid(z):
    with np.errstate(over="ignore"):
        return np.where(z >= 0, 1.0 / (1.0 + np.exp(-z)), np.exp(z) / (1.0 + np.exp(z)))


# ------------------------------------------------------------------ gated linear recurrence
def gated_fwd(gate, u, is_first=None, h0=None, linear=False):
    """h [Bt,L,D]."""
    gate, u = np.asarray(gate, np.float64), np.asarray(u, np.float64)
    Bt, L, D = gate.shape
    f, v = (gate, u) if linear else (_sigmoid(gate), _sigmoid(-gate) * u)
    state = np.zeros((Bt, D)) if h0 is None else np.asarray(h0, np.float64)
    h = np.empty((Bt, L, D))
    for t in range(L):
        kept = f[:, t] * state
        if is_first is not None:
            kept = np.where(np.asarray(is_first)[:, t, None] != 0, 0.0, kept)
        state = kept + v[:, t]
        h[:, t] = state
    return h


def gated_bwd(gate, u, is_first, h0, dh, dh_last=None, linear=False):
    """dict(dgate, du, dh0) for the loss sum(dh h) + sum(dh_last h[:, -1])."""
    gate, u, dh = (np.asarray(x, np.float64) for x in (gate, u, dh))
    Bt, L, D = gate.shape
    h = gated_fwd(gate, u, is_first, h0, linear)
    f, i = (gate, np.ones_like(gate)) if linear else (_sigmoid(gate), _sigmoid(-gate))
    start = np.zeros((Bt, D)) if h0 is None else np.asarray(h0, np.float64)
    back = np.zeros((Bt, D)) if dh_last is None else np.asarray(dh_last, np.float64)
    dgate, du = np.empty_like(gate), np.empty_like(u)
    for t in range(L - 1, -1, -1):
        chi = dh[:, t] + back
        prev = h[:, t - 1] if t else start
        back = f[:, t] * chi
        if is_first is not None:
            cut = np.asarray(is_first)[:, t, None] != 0
            prev, back = np.where(cut, 0.0, prev), np.where(cut, 0.0, back)
        du[:, t] = i[:, t] * chi
        dgate[:, t] = prev * chi if linear else f[:, t] * i[:, t] * (prev - u[:, t]) * chi
    return {"dgate": dgate, "du": du, "dh0": back}


# ------------------------------------------------------------------ clipped policy loss
def policy_loss(x, action, logp_old, advantage, weight=None, logp_ref=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0, entropy_coef=0.0,
                dloss=1.0):
    """dict(loss, logp, entropy, lse, dlogits), row by row."""
    x = np.asarray(x, np.float64)
    N, K = x.shape
    weight = np.full(N, 1.0 / N) if weight is None else np.asarray(weight, np.float64)
    out = {"loss": 0.0, "logp": np.zeros(N), "entropy": np.zeros(N), "lse": np.full(N, -np.inf), "dlogits": np.zeros((N, K))}
    for n in range(N):
        a, w, A = int(action[n]), weight[n], float(advantage[n])
        if w == 0 or a < 0 or np.all(x[n] == -np.inf):
            continue
        if a >= K or np.any(np.isnan(x[n])) or np.any(x[n] == np.inf):
            out["loss"] = out["logp"][n] = out["dlogits"][n, :] = np.nan
            continue
        m = x[n].max()
        d = x[n] - m                                     # (differences first: log s is lost beside a large m)
        ls = np.log(np.exp(d).sum())
        p = np.exp(d - ls)
        lp = np.where(p > 0, d - ls, 0.0)
        H = -(p * lp).sum()
        logp, lse = d[a] - ls, m + ls
        with np.errstate(over="ignore"):
            rho = np.exp(logp - float(logp_old[n]))
        clipped = min(max(rho, 1.0 - clip_low), 1.0 + clip_high) * A
        raw = rho * A if A != 0 else 0.0
        loss, g = -min(raw, clipped) - entropy_coef * H, (-raw if raw <= clipped else 0.0)
        if logp_ref is not None and kl_coef != 0:
            d = float(logp_ref[n]) - logp
            loss, g = loss + kl_coef * (np.expm1(d) - d), g - kl_coef * np.expm1(d)
        out["loss"] += w * loss
        out["logp"][n], out["entropy"][n], out["lse"][n] = logp, H, lse
        out["dlogits"][n] = w * dloss * p * (entropy_coef * (lp + H) - g)
        out["dlogits"][n, a] += w * dloss * g
    return out


# ------------------------------------------------------------------ AdamW
M_BITS, R_BITS = (3, 7, 448.0), (4, 15, 1.9375)      # mantissa bits, bias, largest value of the codes of m and of sqrt(v)
BLOCK = 256


def code_values(bits):
    """What the codes stand for, in ascending order (m: the codes without the sign)."""
    mantissa, bias, _ = bits
    code = np.arange(1 << (4 + mantissa))
    e, q = code >> mantissa, code & ((1 << mantissa) - 1)
    return np.where(e == 0, q * 2.0 ** (1 - bias - mantissa), (q + (1 << mantissa)) * 2.0 ** (e - bias - mantissa))


def stored_m(code, scale):
    code = np.asarray(code).astype(np.int64)
    v = code_values(M_BITS)[code & 127] * np.repeat(np.asarray(scale, np.float64), BLOCK)[:code.size]
    return np.where(code >= 128, -v, v)


def stored_v(code, scale):
    return (code_values(R_BITS)[np.asarray(code).astype(np.int64)] * np.repeat(np.asarray(scale, np.float64), BLOCK)[:np.asarray(code).size]) ** 2


def adamw(p, g, m, v, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """(p, m, v) after one step."""
    p, g, m, v = (np.asarray(x, np.float64) for x in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    update = (m / (1.0 - beta1 ** step)) / (np.sqrt(v / (1.0 - beta2 ** step)) + eps)
    return p - lr * weight_decay * p - lr * update, m, v
