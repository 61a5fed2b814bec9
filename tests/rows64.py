"""Helpers of the tests of the operators around a draft head: inputs, calls, and what the kernels' fp32 arithmetic may be off by.

An exponential 2^t, t = (x - m) c, carries half a step of x - m, of the product and of c (or of the added low part), each 2^-24 |t| in t, so 3 ln 2 2^-24 |t|
relative, and ex2.approx's 2^-22; a sum of such terms carries their weighted mean, at most the same with the row's mean |t|, and a vector's or a
chunk's tokens added in fp32 (16 additions in a row at most: 2^-20).  `rel` is that for q = e / sum; scales and products add four more roundings."""
import numpy as np
import torch

import paper_2606_12370_b200 as P

DEV = "cuda"
LN2 = 0.6931471805599453
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}        # a rounding of the output, relative
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def padded(rows, V, dtype, fill=None, extra=0):
    """[..., V] rows on 16-byte boundaries, `extra` vectors apart; and their storage."""
    vec = 16 // torch.empty((), dtype=TYPES[dtype]).element_size()
    store = torch.empty((*rows, V + (-V) % vec + extra * vec), dtype=TYPES[dtype], device=DEV)
    store.fill_(1e4 if fill is None else fill)
    return store[..., :V], store


def rows(shape, V, dtype, seed, std=3.0, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z, _ = padded(shape, V, dtype, extra=extra)
    z.copy_(std * torch.randn((*shape, V), generator=g, device=DEV))
    return z


def uniform(shape, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (2 * torch.randint(0, 1 << 23, shape, generator=g, device=DEV) + 1).float() * 2.0 ** -24


def np32(t):
    return None if t is None else t.detach().float().cpu().numpy()


def rel(log_q):
    """[N, V] relative error allowed to q, from its logarithm; rows without one (-inf everywhere) get 0."""
    t = np.where(np.isfinite(log_q), (log_q.max(-1, keepdims=True) - log_q) / LN2, 0.0)
    with np.errstate(invalid="ignore"):
        mean = np.where(np.isfinite(log_q), np.exp(log_q) * t, 0.0).sum(-1, keepdims=True)
    return 3 * LN2 * 2.0 ** -24 * (t + mean) + 2 * 2.0 ** -22 + 2.0 ** -20 + 4 * 2.0 ** -24


def check_tv_grad(got, ref, dtype, scale):
    """scale [N]: |g| / tau."""
    assert (got["row_status"].cpu().numpy() == ref["row_status"]).all(), (got["row_status"].tolist(), ref["row_status"].tolist())
    r = rel(ref["log_q"])
    top = r.max(-1)
    mean = (np.exp(ref["log_q"]) * r).sum(-1) + 2.0 ** -20
    assert (np.abs(np32(got["tv"]) - ref["tv"]) <= 4 * mean + 2.0 ** -24).all(), np.abs(np32(got["tv"]) - ref["tv"]).max()      # (p and q, and the products with their ratio)
    assert (np.abs(np32(got["s_aux"]) - ref["s_aux"]) <= 2 * mean + 2.0 ** -24).all()
    q = np.exp(ref["log_q"]) * np.asarray(scale)[:, None]
    tol = q * (r + 2 * mean[:, None]) + STEP[dtype] * (np.abs(ref["grad_draft"]) + q * r) + 2.0 ** -120 * np.asarray(scale)[:, None]
    bad = np.abs(np32(got["grad_draft"]) - ref["grad_draft"]) > tol
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), np32(got["grad_draft"])[bad][:4], ref["grad_draft"][bad][:4], top.max())


def check_distill(got, ref, dtype, scale):
    assert (got["row_status"].cpu().numpy() == ref["row_status"]).all(), (got["row_status"].tolist(), ref["row_status"].tolist())
    r = rel(ref["log_q"])
    mean = (np.exp(ref["log_q"]) * r).sum(-1) + 2.0 ** -20
    loss = np32(got["loss"])
    fine = np.isfinite(ref["loss"])
    assert (loss[~fine] == ref["loss"][~fine]).all()
    off = np.abs(loss - ref["loss"])[fine]
    # log of the sum and of the tail's share: their relative errors; the result's own rounding
    assert (off <= (2 * mean + 2.0 ** -24 * (1 + np.abs(ref["loss"])))[fine]).all(), off.max()
    if got["grad_draft"] is None:
        return
    tol = ref["size"] * (r + 2 * mean[:, None]) + STEP[dtype] * (np.abs(ref["grad_draft"]) + ref["size"] * r) + 2.0 ** -120 * np.asarray(scale)[:, None]
    bad = np.abs(np32(got["grad_draft"]) - ref["grad_draft"]) > tol
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), np32(got["grad_draft"])[bad][:4], ref["grad_draft"][bad][:4])


def check_target_only(got, ref):
    ok = ~ref["flagged"]
    assert ok.any() or len(ok) < 3
    for k in ("accept_len", "row_status"):
        assert (got[k].cpu().numpy()[ok] == ref[k][ok]).all(), (k, got[k].tolist(), ref[k].tolist())
    bad = (got["out_tokens"].cpu().numpy() != ref["out_tokens"]).any(1) & ok
    assert not bad.any(), (np.nonzero(bad)[0][:4], got["out_tokens"].cpu().numpy()[bad][:4], ref["out_tokens"][bad][:4], ref["margin_cdf"][bad][:4])
    if got["p_draft"] is not None:
        assert (np.abs(np32(got["p_draft"]) - ref["p_draft"])[ok] <= 1e-5 * ref["p_draft"][ok]).all()


def paths(request):
    """Both ways a row is taken: in the shared memory of a cluster, and from memory by every pass."""
    P.bebop_debug_force_general_path(request.param)
    return request.param
