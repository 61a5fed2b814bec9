"""The operators around a draft head, beside the verify step itself: the total-variation loss with its gradient
("tv_grad"), distillation from the teacher's top logits ("distill"), and the verification of drafts that come without a
distribution ("target_only").

A case names the operator, its sizes (N rows, or B sequences of K drafts; V logits per row; T teacher entries per row), the
type of the logits and what varies by row.  Rows whose length is not a whole number of 16-byte vectors are padded, as the
entry points ask for.  `run` computes the plain form with elementary torch operations, or, with `own`, calls the framework.
"""
import math

import torch

own = False

MAX_BYTES = 0.75e9         # work of a drawn case, at most: less than the largest listed ones


def _tv(name, N, V, dtype="bf16", temperature="one", weights="mean"):
    """weights: what the loss gives every row pair: "mean" (1 / N), or "masked" (every eighth row is padding: weight 0)."""
    return dict(name=name, op="tv_grad", N=N, V=V, dtype=dtype, temperature=temperature, weights=weights)


def _distill(name, N, V, T, dtype="bf16", temperature="one", tail=True, ragged=False, grad=True):
    """tail: the teacher's logsumexp came with its top logits, so that what they leave out counts; ragged: rows with fewer entries
    than T, some with none (ignored positions); grad: the gradient is wanted."""
    return dict(name=name, op="distill", N=N, V=V, T=T, dtype=dtype, temperature=temperature, tail=tail, ragged=ragged, grad=grad)


def _verify(name, B, K, V, dtype="bf16", temperature="one", ragged=False):
    """ragged: draft counts uniform in 1..K."""
    return dict(name=name, op="target_only", B=B, K=K, V=V, dtype=dtype, temperature=temperature, ragged=ragged)


def listed():
    return [
        # the smallest call: four sequences' three draft positions over a toy vocabulary, latency only
        _tv("tv_grad_tiny", 12, 1024, dtype="f32"),
        # a small evaluation batch, fp32 logits, an odd vocabulary, a temperature per row
        _tv("tv_grad_f32_odd", 100, 32003, dtype="f32", temperature="rows"),
        # the draft positions of a training batch over a production vocabulary, padded positions among them
        _tv("tv_grad_train", 768, 151936, weights="masked"),
        # the largest vocabulary
        _tv("tv_grad_large_vocab", 512, 262144, temperature="half"),
        # the smallest call
        _distill("distill_tiny", 12, 1024, 8, dtype="f32", tail=False),
        # fp32, odd vocabulary, a nucleus of varying size per position, ignored positions
        _distill("distill_f32_odd", 100, 49999, 100, dtype="f32", temperature="rows", ragged=True),
        # validation loss over a middle-sized vocabulary: no gradient
        _distill("distill_loss_only", 1024, 32000, 256, tail=False, grad=False),
        # the training batch
        _distill("distill_train", 768, 151936, 64),
        # the smallest call
        _verify("target_only_tiny", 4, 3, 1024, dtype="f32"),
        # one stream of interactive decoding with look-up drafts
        _verify("target_only_one_stream", 1, 3, 151936),
        # a rollout batch
        _verify("target_only_rollout", 256, 3, 151936),
        # the full rollout batch: ragged drafts, a temperature per row
        _verify("target_only_full_batch", 1024, 4, 151936, temperature="rows", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tv_grad", "distill", "target_only"])
    n, V = _log_int(rng, 1, 1024), _log_int(rng, 1024, 262144)
    how = dict(dtype=rng.choice(["bf16", "bf16", "f32"]), temperature=rng.choice(["one", "half", "rows"]))
    if op == "tv_grad":
        c = _tv("", n, V, weights=rng.choice(["mean", "masked"]), **how)
    elif op == "distill":
        c = _distill("", n, V, _log_int(rng, 1, 512), tail=rng.random() < 0.5, ragged=rng.random() < 0.5, grad=rng.random() < 0.75, **how)
    else:
        c = _verify("", n, rng.randint(1, 8), V, ragged=rng.random() < 0.5, **how)
    del c["name"]
    key = "B" if op == "target_only" else "N"
    while work(c)["bytes"] > MAX_BYTES or c[key] * (c.get("K", 0) + 1) * c["V"] > 8e8:      # (a verify call holds rows that it does not read)
        c[key] = c[key] * 3 // 4
    return c


def _size(c):
    return 4 if c["dtype"] == "f32" else 2


# Drafts of a trained head: the target gives them between 0.4 and 1, 0.7 in the mean.
ACCEPT = (0.4, 1.0)


def _rows_needed(c):
    """Target rows that verification reads in the mean: every draft lets it go on with probability 0.7."""
    a = sum(ACCEPT) / 2
    upto = [sum(a ** k for k in range(L + 1)) for L in range(c["K"] + 1)]
    return c["B"] * (sum(upto[1:]) / c["K"] if c["ragged"] else upto[c["K"]])


def work(case):
    c = case
    if c["op"] == "tv_grad":
        n = c["N"] * c["V"]
        # both rows in, the gradient out; per pair two exponentials and sums, the comparison, the residual, the product
        return {"bytes": float(3 * n * _size(c) + 16 * c["N"]), "flops": float(14 * n)}
    if c["op"] == "distill":
        n = c["N"] * c["V"]
        return {"bytes": float((2 if c["grad"] else 1) * n * _size(c) + c["N"] * (c["T"] * (4 + _size(c)) + 16)), "flops": float((6 if c["grad"] else 4) * n)}
    n = _rows_needed(c) * c["V"]
    return {"bytes": float(n * _size(c) + 4 * c["B"] * (4 * c["K"] + 5)), "flops": float(4 * n)}


# ------------------------------------------------------------------ inputs
def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _padded(c, rows):
    """Rows of V logits, each on a 16-byte boundary."""
    V = c["V"]
    return torch.zeros((*rows, V + (-V) % (16 // _size(c))), dtype=_dtype(c), device="cuda")[..., :V]


def _temperature(c, n, g):
    if c["temperature"] == "one":
        return None
    if c["temperature"] == "half":
        t = torch.ones(n, device="cuda")
        t[: n // 2] = 0.7
        return t
    return 0.6 + 0.6 * torch.rand(n, generator=g, device="cuda")


def _model_rows(n, V, g):
    """Logits of a trained model: N(0, 3^2) and eight Zipf-ranked peaks a row."""
    t = torch.randn((n, V), generator=g, device="cuda") * 3.0
    heights = 8.0 * torch.arange(1, 9, device="cuda", dtype=torch.float32) ** (-2.0 / 3.0)
    return t.scatter_add_(1, torch.randint(0, V, (n, 8), generator=g, device="cuda"), heights.expand(n, 8))


def _uniform(shape, g):
    """(2 r + 1) 2^-24: inside (0, 1), exact in fp32."""
    return (2 * torch.randint(0, 1 << 23, shape, generator=g, device="cuda") + 1).to(torch.float32) * 2.0 ** -24


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"op": c["op"]}
    V = c["V"]
    if c["op"] == "target_only":
        B, K = c["B"], c["K"]
        s["temperature"] = tau = _temperature(c, B, g)
        z = _padded(c, (B, K + 1))
        s["draft_tokens"] = tok = torch.randint(0, V, (B, K), generator=g, device="cuda", dtype=torch.int32)
        odds = torch.logit(ACCEPT[0] + (ACCEPT[1] - ACCEPT[0]) * torch.rand((B, K), generator=g, device="cuda").clamp(1e-3, 0.999))
        for b in range(0, B, 32):
            n = min(32, B - b)
            x = _model_rows(n * (K + 1), V, g).view(n, K + 1, V)
            at = tok[b:b + n].long().unsqueeze(-1)
            ts = torch.ones((n, 1), device="cuda") if tau is None else tau[b:b + n, None]
            d = x[:, :K].scatter(2, at, -math.inf)               # the draft's logit: what gives it its probability
            x[:, :K] = d.scatter_(2, at, (ts * (torch.logsumexp(d / ts.unsqueeze(-1), -1) + odds[b:b + n])).unsqueeze(-1))
            z[b:b + n] = x
        s["target"] = z
        s["u_accept"], s["u_final"] = _uniform((B, K), g), _uniform((B,), g)
        s["draft_len"] = torch.randint(1, K + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if c["ragged"] else None
        # the outputs' buffers are what a program that calls the step in a loop keeps
        s["out"] = dict(accept_len=torch.empty(B, dtype=torch.int32, device="cuda"), out_tokens=torch.empty((B, K + 1), dtype=torch.int32, device="cuda"),
                        p_draft=torch.empty((B, K), device="cuda"), row_status=torch.empty(B, dtype=torch.int32, device="cuda"))
        return s
    N = c["N"]
    s["temperature"] = tau = _temperature(c, N, g)
    s["draft"] = draft = _padded(c, (N,))
    keep = torch.ones(N, device="cuda")
    if c["op"] == "tv_grad":
        s["target"] = target = _padded(c, (N,))
        if c["weights"] == "masked":
            keep[::8] = 0.0 if N > 8 else 1.0
        s["weight"] = keep / keep.sum()
    else:
        T = min(c["T"], V)
        s["ids"] = torch.empty((N, T), dtype=torch.int32, device="cuda")
        s["top"] = torch.empty((N, T), dtype=_dtype(c), device="cuda")
        s["lse"] = torch.empty(N, device="cuda") if c["tail"] else None
    for a in range(0, N, 64):
        n = min(64, N - a)
        t = _model_rows(n, V, g).to(_dtype(c))
        draft[a:a + n] = t + torch.randn((n, V), generator=g, device="cuda")
        if c["op"] == "tv_grad":
            target[a:a + n] = t
        else:
            top = t.float().topk(T, dim=-1)
            s["ids"][a:a + n], s["top"][a:a + n] = top.indices, top.values
            if c["tail"]:
                s["lse"][a:a + n] = torch.logsumexp(t.double() / (1.0 if tau is None else tau[a:a + n, None].double()), -1)
    if c["op"] == "distill":
        if c["ragged"]:
            have = torch.randint(1, T + 1, (N,), generator=g, device="cuda")
            have[3::16] = 0
            s["ids"].masked_fill_(torch.arange(T, device="cuda") >= have[:, None], -1)
        s["weight"] = torch.full((N,), 1.0 / N, device="cuda") if c["grad"] else None
        s["out"] = dict(loss=torch.empty(N, device="cuda"), row_status=torch.empty(N, dtype=torch.int32, device="cuda"))
    else:
        s["out"] = dict(tv=torch.empty(N, device="cuda"), s_aux=torch.empty(N, device="cuda"), row_status=torch.empty(N, dtype=torch.int32, device="cuda"))
    if c.get("grad", True):
        s["out"]["grad_draft"] = _padded(c, (N,))
    return s


# ------------------------------------------------------------------ one pass
def run(state):
    s = state
    if own:
        import paper_2606_12370_b200 as P
        if s["op"] == "tv_grad":
            return P.bebop_tv_grad(s["target"], s["draft"], temperature=s["temperature"], grad_tv=s["weight"], out=s["out"])
        if s["op"] == "distill":
            return P.bebop_distill(s["draft"], s["ids"], s["top"], target_lse=s["lse"], temperature=s["temperature"], grad_loss=s["weight"],
                                   out=s["out"], want_grad=s["weight"] is not None)
        return P.bebop_target_only_verify(s["target"], s["draft_tokens"], s["u_accept"], s["u_final"], draft_len=s["draft_len"],
                                          temperature=s["temperature"], out=s["out"])
    return {"tv_grad": _plain_tv_grad, "distill": _plain_distill, "target_only": _plain_target_only}[s["op"]](s)


def _log_softmax(z, tau):
    """log softmax(z / tau), in 64 bits."""
    x = z.double()
    if tau is not None:
        x = x / tau.double().view(-1, *[1] * (x.dim() - 1))
    x = x - x.amax(-1, keepdim=True)
    return x - x.exp().sum(-1, keepdim=True).log()


def _plain_tv_grad(s):
    # in 64 bits: which side of q = p a token is on, where the gradient jumps
    lp, lq = _log_softmax(s["target"], s["temperature"]), _log_softmax(s["draft"], s["temperature"])
    below = lq <= lp
    p, q = lp.float().exp(), lq.float().exp()
    tv = (p - q).clamp_min(0).sum(-1, dtype=torch.float64).clamp(0, 1)
    S = torch.where(below, q, 0).sum(-1, dtype=torch.float64)
    scale = s["weight"] if s["temperature"] is None else s["weight"] / s["temperature"]
    grad = q * (S.float()[:, None] - below.float()) * scale[:, None]
    return dict(grad_draft=grad.to(s["draft"].dtype), tv=tv.float(), s_aux=S.float(), row_status=torch.zeros_like(tv, dtype=torch.int32))


def _plain_distill(s):
    z, ids, N = s["draft"].float(), s["ids"].long(), s["ids"].shape[0]
    tau = torch.ones((N, 1), device=z.device) if s["temperature"] is None else s["temperature"][:, None]
    m = z.amax(-1, keepdim=True)
    e = ((z - m) / tau).exp()
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    has = ids >= 0
    t = torch.where(has, s["top"].double() / tau.double(), -math.inf)
    if s["lse"] is None:
        top = t.amax(-1, keepdim=True).nan_to_num(neginf=0.0)
        lp = t - top
        lp = lp - lp.exp().sum(-1, keepdim=True).log()
    else:
        lp = t - s["lse"].double()[:, None]
    lp = torch.where(has, lp, 0.0)
    p = torch.where(has, lp.exp(), 0.0)
    at = ids.clamp_min(0)
    zt = z.gather(1, at)
    lq = ((zt - m) / tau).double() - total.log()
    loss = (p * (lp - lq)).sum(-1)
    P = p.sum(-1, keepdim=True)
    seen = has.any(-1, keepdim=True)
    out = dict(loss=loss, row_status=torch.zeros(N, dtype=torch.int32, device=z.device))
    rest = e.scatter(1, at, torch.where(has, 0.0, e.gather(1, at)))      # (an unused entry points at token 0: put back below)
    zero = torch.zeros_like(z[:, :1])
    first = torch.where((has & (ids == 0)).any(-1, keepdim=True), zero, e[:, :1])
    rest[:, :1] = first
    r = (1.0 - P).clamp_min(0.0) if s["lse"] is not None else torch.zeros_like(P)
    share = rest.sum(-1, keepdim=True, dtype=torch.float64) / total
    if s["lse"] is not None:
        out["loss"] = loss + torch.where(r > 0, r * (r / share).log(), 0.0).squeeze(-1)
    out["loss"] = torch.where(seen.squeeze(-1), out["loss"], 0.0).float()
    if s["weight"] is not None:
        q = e / total.float()
        grad = q * (P + r).float() - (rest / total.float()) * torch.where(r > 0, r / share, 0.0).float()
        grad.scatter_add_(1, at, -p.float())
        grad = torch.where(seen, grad, 0.0) * (s["weight"][:, None] / tau)
        out["grad_draft"] = grad.to(s["draft"].dtype)
    return out


def _plain_target_only(s):
    # in 64 bits: accept tests and the running sums that a token is drawn from
    prob = _log_softmax(s["target"], s["temperature"]).exp_()
    B, K = s["draft_tokens"].shape
    tok = s["draft_tokens"].long()
    L = torch.full((B,), K, device=tok.device) if s["draft_len"] is None else s["draft_len"].long()
    k = torch.arange(K, device=tok.device)
    px = prob[:, :K].gather(2, tok.unsqueeze(-1)).squeeze(-1)
    go = (s["u_accept"].double() < px) & (k < L[:, None])
    n = go.long().cumprod(-1).sum(-1)
    r = prob[torch.arange(B, device=tok.device), n]
    rejected = n < L
    x = tok.gather(1, n.clamp_max(K - 1)[:, None])
    r.scatter_(1, x, torch.where(rejected[:, None], 0.0, r.gather(1, x)))
    C = r.cumsum(-1)
    y = (C < s["u_final"].double()[:, None] * C[:, -1:]).sum(-1)
    col = torch.arange(K + 1, device=tok.device)
    drafts = torch.cat([tok, tok[:, :1]], 1)
    out = torch.where(col < n[:, None], drafts, torch.where(col == n[:, None], y[:, None], -1))
    read = (k <= n[:, None]) & (k < L[:, None])
    return dict(accept_len=n.int(), out_tokens=out.int(), p_draft=torch.where(read, px, 0.0).float(), row_status=torch.zeros(B, dtype=torch.int32, device=tok.device))


# ------------------------------------------------------------------ the definition, row by row
def exact(case, seed):
    c, s = case, prepare(case, seed)
    tau_of = (lambda i: 1.0) if s["temperature"] is None else [float(v) for v in s["temperature"].tolist()].__getitem__
    if c["op"] == "target_only":
        return _exact_target_only(c, s, tau_of)
    N, V = s["draft"].shape
    names = ["tv", "s_aux"] if c["op"] == "tv_grad" else ["loss"]
    res = {k: torch.zeros(N, dtype=torch.float64, device="cuda") for k in names}
    grad = torch.zeros((N, V), dtype=torch.float64, device="cuda") if s["weight"] is not None else None
    for i in range(N):
        tau = tau_of(i)
        zq = s["draft"][i].double() / tau
        log_q = zq - torch.logsumexp(zq, 0)
        if c["op"] == "tv_grad":
            zp = s["target"][i].double() / tau
            log_p = zp - torch.logsumexp(zp, 0)
            p, q = torch.exp(log_p), torch.exp(log_q)
            under = torch.le(log_q, log_p).double()
            res["tv"][i] = 0.5 * (p - q).abs().sum()
            res["s_aux"][i] = torch.dot(q, under)
            grad[i] = -(s["weight"][i].double() / tau) * q * (under - res["s_aux"][i])
            continue
        here = (s["ids"][i] >= 0).nonzero().squeeze(-1)
        if here.numel() == 0:
            continue
        ids, t = s["ids"][i][here].long(), s["top"][i][here].double() / tau
        teacher = torch.zeros(V, dtype=torch.float64, device="cuda")
        logs = t - (torch.logsumexp(t, 0) if s["lse"] is None else s["lse"][i].double())
        teacher[ids] = torch.exp(logs)
        loss = torch.dot(torch.exp(logs), logs - log_q[ids])
        other = torch.ones(V, dtype=torch.bool, device="cuda")
        other[ids] = False
        q = torch.exp(log_q)
        r = max(0.0, 1.0 - float(torch.exp(logs).sum())) if s["lse"] is not None else 0.0
        d = q * (torch.exp(logs).sum() + r) - teacher
        if r > 0.0:
            left = torch.exp(torch.logsumexp(log_q[other], 0))
            loss = loss + r * (math.log(r) - torch.log(left))
            d[other] -= q[other] * (r / left)
        res["loss"][i] = loss
        if grad is not None:
            grad[i] = d * (s["weight"][i].double() / tau)
    res["row_status"] = None
    if grad is not None:
        res["grad_draft"] = grad
    return res


def _exact_target_only(c, s, tau_of):
    B, K = c["B"], c["K"]
    tok, ua, uf = s["draft_tokens"].tolist(), s["u_accept"].tolist(), s["u_final"].tolist()
    L = [K] * B if s["draft_len"] is None else s["draft_len"].tolist()
    p_draft = torch.zeros((B, K), dtype=torch.float64)
    accept, out = [], []
    for b in range(B):
        n, drawn = 0, None
        while True:
            p = torch.softmax(s["target"][b, n].double() / tau_of(b), 0)
            if n == L[b]:
                break
            px = float(p[tok[b][n]])
            p_draft[b, n] = px
            if ua[b][n] >= px:
                p[tok[b][n]] = 0.0
                break
            n += 1
        run_sum = torch.cumsum(p, 0)
        drawn = int(torch.searchsorted(run_sum, torch.tensor([uf[b]], dtype=torch.float64, device="cuda") * run_sum[-1]))
        accept.append(n)
        out.append(tok[b][:n] + [drawn] + [-1] * (K - n))
    return dict(accept_len=torch.tensor(accept, dtype=torch.int32), out_tokens=torch.tensor(out, dtype=torch.int32), p_draft=p_draft, row_status=None)
