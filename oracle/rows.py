"""fp64 statement of the operators around a draft head, in numpy: target-only verification, the TV loss with its gradient,
distillation from a teacher's top logits.  TEST INFRASTRUCTURE ONLY, like the C oracle; shares no code with the kernels.

Rows are float32 arrays (bf16 inputs widened exactly by the caller).  Beside the values come the margins that say where a
rounding may decide: a verification is `flagged` where its accept test or its draw is a near-tie.
"""
import math

import numpy as np

ST_NONFINITE, ST_EMPTY_ROW, ST_BAD_TOKEN, ST_ZERO_RESID, ST_BAD_TEMP = 1, 2, 4, 8, 16
FLAG_MARGIN = 1e-5


def _tau(temperature, temperature_all, i):
    return float(np.float32(temperature_all if temperature is None else temperature[i]))      # (an fp32 argument of the entry points)


def _tau_ok(tau):
    return tau > 0.0 and math.isfinite(tau)


def log_softmax(z, tau):
    """(log softmax(z / tau) in fp64, status).  The largest logit is taken off first: it may be as large as a float is."""
    z = np.asarray(z, dtype=np.float64)
    if np.isnan(z).any() or (z == np.inf).any():
        return None, ST_NONFINITE
    m = z.max()
    if m == -np.inf:
        return None, ST_EMPTY_ROW
    x = (z - m) / tau
    return x - math.log(math.fsum(np.exp(x))), 0


def target_only_verify(target, draft_tokens, u_accept, u_final, draft_len=None, temperature=None, temperature_all=1.0):
    """Accept x_k while u_k < p_k(x_k); at a reject draw from p without the draft, else from the row behind the last draft."""
    B, K1, V = target.shape
    K = K1 - 1
    o = dict(accept_len=np.zeros(B, np.int32), out_tokens=np.full((B, K1), -1, np.int32), p_draft=np.zeros((B, K)), row_status=np.zeros(B, np.int32),
             margin_acc=np.full(B, np.inf), margin_cdf=np.full(B, np.inf))
    for b in range(B):
        tau = _tau(temperature, temperature_all, b)
        L = K if draft_len is None else max(0, min(int(draft_len[b]), K))
        x = draft_tokens[b, :L]
        if not _tau_ok(tau):
            o["row_status"][b] = ST_BAD_TEMP
            continue
        if ((x < 0) | (x >= V)).any():
            o["row_status"][b] = ST_BAD_TOKEN
            continue
        n = 0
        while True:
            lp, st = log_softmax(target[b, n], tau)
            if st:
                break
            r = np.exp(lp)
            if n == L:
                break
            p, u = r[x[n]], float(u_accept[b, n])
            o["p_draft"][b, n] = p
            o["margin_acc"][b] = min(o["margin_acc"][b], abs(u - p) / max(u, p))
            if not u < p:
                r[x[n]] = 0.0
                break
            n += 1
        if st:
            o["row_status"][b] = st
            o["p_draft"][b] = 0.0
            continue
        o["accept_len"][b] = n
        o["out_tokens"][b, :n] = x[:n]
        Z = math.fsum(r)
        if not Z > 0.0:
            o["row_status"][b] = ST_ZERO_RESID
            o["out_tokens"][b, n] = x[n]
            continue
        C = np.cumsum(r.astype(np.longdouble))
        t = np.longdouble(u_final[b]) * C[-1]
        y = int(np.searchsorted(C, t))
        o["out_tokens"][b, n] = y
        o["margin_cdf"][b] = float(min(t - (C[y - 1] if y else 0), C[y] - t) / r[y])
    o["flagged"] = (o["margin_acc"] < FLAG_MARGIN) | (o["margin_cdf"] < FLAG_MARGIN)
    return o


def tv_grad(target, draft, grad_tv=None, temperature=None, temperature_all=1.0):
    """tv = sum max(0, p - q), S = sum q 1[q <= p], grad = -(g / tau) q (1[q <= p] - S); and log_q (for tolerances), near: the smallest
    distance of log q and log p in a row where q counts."""
    N, V = draft.shape
    o = dict(tv=np.zeros(N), s_aux=np.zeros(N), grad_draft=np.zeros((N, V)), row_status=np.zeros(N, np.int32), log_q=np.full((N, V), -np.inf), near=np.full(N, np.inf))
    for i in range(N):
        tau = _tau(temperature, temperature_all, i)
        if not _tau_ok(tau):
            o["row_status"][i] = ST_BAD_TEMP
            continue
        (lp, sp), (lq, sq) = log_softmax(target[i], tau), log_softmax(draft[i], tau)
        if sp | sq:
            o["row_status"][i] = sp | sq
            continue
        p, q = np.exp(lp), np.exp(lq)
        # q <= p by the difference of the logits: the softmax's own rounding stays out of it
        zp, zq = target[i].astype(np.float64), draft[i].astype(np.float64)
        with np.errstate(invalid="ignore"):
            theta = tau * (lq.max() - lp.max())
            d = (zp - zp.max()) - (zq - zq.max())
        below = np.where(q > 0, d >= theta, True)
        o["near"][i] = np.abs(np.where(q > 0, d - theta, np.inf)).min()
        o["tv"][i] = min(1.0, max(0.0, 0.5 * math.fsum(np.abs(p - q))))
        o["s_aux"][i] = math.fsum(q[below])
        o["log_q"][i] = lq
        o["grad_draft"][i] = -((1.0 if grad_tv is None else float(grad_tv[i])) / tau) * q * (below - o["s_aux"][i])
    return o


def distill(draft, ids, top, lse=None, grad_loss=None, temperature=None, temperature_all=1.0):
    """KL of the entries' distribution (id -1: none) and the draft's, the rest of both as one more token where lse is given.
    Beside loss and grad_draft: `size`, what the gradient's terms add up to in magnitude, and log_q (for tolerances)."""
    N, V = draft.shape
    o = dict(loss=np.zeros(N), grad_draft=np.zeros((N, V)), row_status=np.zeros(N, np.int32), size=np.zeros((N, V)), log_q=np.full((N, V), -np.inf))
    for i in range(N):
        tau = _tau(temperature, temperature_all, i)
        have = ids[i] != -1
        at, t = ids[i][have].astype(np.int64), np.asarray(top[i], dtype=np.float64)[have]
        if not _tau_ok(tau):
            o["row_status"][i] = ST_BAD_TEMP
            continue
        if not have.any():
            continue
        if ((at < 0) | (at >= V)).any() or len(set(at.tolist())) < len(at):
            o["row_status"][i] = ST_BAD_TOKEN
            continue
        lq, st = log_softmax(draft[i], tau)
        if np.isnan(t).any() or (t == np.inf).any() or (lse is not None and not np.isfinite(lse[i])) or st == ST_NONFINITE:
            o["row_status"][i] = ST_NONFINITE
            continue
        if st or (lse is None and t.max() == -np.inf):
            o["row_status"][i] = ST_EMPTY_ROW
            continue
        lp = log_softmax(t, tau)[0] if lse is None else t / tau - float(lse[i])
        p, q = np.exp(lp), np.exp(lq)
        P = math.fsum(p)
        r = 0.0 if lse is None else max(0.0, 1.0 - P)
        rest = np.ones(V, bool)
        rest[at] = False
        loss = math.fsum(p[j] * (lp[j] - lq[at[j]]) if p[j] > 0 else 0.0 for j in range(len(at))) if not (np.isneginf(lq[at]) & (p > 0)).any() else math.inf
        s = math.fsum(q[rest])
        if r > 0:
            loss += r * (math.log(r) - math.log(s)) if s > 0 else math.inf
        g = (1.0 if grad_loss is None else float(grad_loss[i])) / tau
        d, size = q * (P + r), q * (P + r)
        if r > 0 and s > 0:
            d[rest] -= q[rest] * (r / s)
            size[rest] += q[rest] * (r / s)
        d[at] -= p
        size[at] += p
        o["loss"][i], o["grad_draft"][i], o["size"][i], o["log_q"][i] = loss, g * d, abs(g) * size, lq
    return o
