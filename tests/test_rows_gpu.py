"""The operators around a draft head (target-only verification, the TV loss with its gradient, distillation from the target's top logits) against the fp64
oracle, at the sizes, masks and strides where they can go wrong.  Every case runs both ways a row can be taken."""
import numpy as np
import pytest
import torch

import oracle.rows as O
import paper_2606_12370_b200 as P
from rows64 import DEV, TYPES, check_distill, check_target_only, check_tv_grad, np32, padded, rows, uniform

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(params=[0, 1], ids=["resident", "from_memory"], autouse=True)
def path(request):
    P.bebop_debug_force_general_path(request.param)
    yield request.param
    P.bebop_debug_force_general_path(0)


SIZES = [("f32", 1, 5), ("bf16", 1, 3), ("bf16", 2, 9), ("f32", 7, 4), ("bf16", 8, 4), ("bf16", 1000, 3), ("f32", 1025, 5), ("bf16", 4099, 7), ("f32", 12290, 2), ("bf16", 32003, 3), ("f32", 151936, 2),
         ("bf16", 262144, 2), ("bf16", 300, 700)]


# ------------------------------------------------------------------ the TV loss and its gradient
def run_tv_grad(t, d, **kw):
    got = P.bebop_tv_grad(t, d, **kw)
    torch.cuda.synchronize()
    return got


def against_tv(t, d, dtype, g=None, tau=None, tau_all=1.0, got=None):
    got = got or run_tv_grad(t, d, temperature=tau, temperature_all=tau_all, grad_tv=g)
    ref = O.tv_grad(np32(t), np32(d), np32(g), np32(tau), tau_all)
    scale = (np.ones(len(t)) if g is None else np.abs(np32(g))) / (tau_all if tau is None else np.where(np32(tau) > 0, np32(tau), 1.0))
    check_tv_grad(got, ref, dtype, scale)
    return got, ref


@pytest.mark.parametrize("dtype,V,N", SIZES)
def test_tv_grad_sizes(dtype, V, N):
    t = rows((N,), V, dtype, 1)
    d = rows((N,), V, dtype, 2, extra=1)
    d.copy_(t + 0.3 * d)
    tau = 0.6 + 0.6 * uniform((N,), 3)
    against_tv(t, d, dtype, g=uniform((N,), 4) - 0.5, tau=tau)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tv_grad_masks(dtype):
    """Masked tokens in one row or both, masks of a large finite value and of the type's lowest, rows that are nothing but such a mask."""
    V, N = 1500, 12
    t, d = rows((N,), V, dtype, 5), rows((N,), V, dtype, 6)
    low = torch.finfo(TYPES[dtype]).min
    t[0, :700] = -INF
    d[1, 300:] = -INF
    t[2, ::2] = -INF; d[2, ::2] = -INF
    t[3, :] = -INF; t[3, 1499] = 2.0                  # all of p on one token
    t[4, 5:] = -1e9
    d[5, :1499] = low
    t[6, :] = -1e9; d[6, :] = -1e9                    # p = q = 1 / V
    t[7, :] = low; d[7, :] = -low                     # (the same; the rows' difference is beyond a float)
    t[8, :] = low                                     # uniform against the draft
    t[9, :700] = -INF; d[9, 700:] = -INF              # disjoint
    t[10, 100] = -low                                 # one token above all
    t[11] = d[11]                                     # equal rows: TV 0, S 1, no gradient
    got, ref = against_tv(t, d, dtype)
    # (disjoint rows: the same terms added up in pass 1 and, in another order, in pass 2, a vector's eight or a lane's 32 in fp32: 2^-23 and 2^-23)
    assert float(got["tv"][9]) >= 1.0 - 2.0 ** -22 and float(got["tv"][11]) == 0.0 and float(got["s_aux"][11]) == 1.0
    assert not got["grad_draft"][11].any() and not got["grad_draft"][9, 700:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tv_grad_status_and_fatal_rows(dtype):
    t, d = rows((9,), 777, dtype, 7), rows((9,), 777, dtype, 8)
    tau = torch.ones(9, device=DEV)
    t[0, 776] = float("nan"); d[1, 0] = float("nan"); t[2, 3] = INF; d[3, 776] = INF
    t[4, :] = -INF; d[5, :] = -INF
    tau[6] = 0.0; tau[7] = float("nan")
    got, _ = against_tv(t, d, dtype, tau=tau)
    assert got["row_status"].tolist() == [1, 1, 1, 1, 2, 2, 16, 16, 0]
    assert not got["grad_draft"][:8].any() and got["grad_draft"][8].any()


@pytest.mark.parametrize("tau", [1e-30, 1e-3, 40.0, 1e30])
def test_tv_grad_temperatures(tau):
    t = rows((3,), 501, "f32", 9)
    d = t + 0.1 * rows((3,), 501, "f32", 10)
    got = run_tv_grad(t, padded((3,), 501, "f32")[0].copy_(d), temperature_all=tau)
    ref = O.tv_grad(np32(t), np32(d), None, None, tau)
    check_tv_grad(got, ref, "f32", np.full(3, 1.0 / tau))


def test_tv_grad_comparisons_at_the_border():
    """Thousands of tokens whose q and p differ by less than the fp32 sums' error: the comparisons, and with them the gradients, are those of fp64."""
    V, N = 60000, 3
    t = rows((N,), V, "f32", 11)
    d = padded((N,), V, "f32")[0].copy_(t + 0.5 * torch.randn((N, V), generator=torch.Generator(device=DEV).manual_seed(12), device=DEV))
    low = torch.arange(V, device=DEV) % 7 == 0
    t[:, low] = -6 - 2 * uniform((N, int(low.sum())), 13)
    for _ in range(3):
        theta = torch.logsumexp(t.double(), 1) - torch.logsumexp(d.double(), 1)
        d[:, low] = (t[:, low].double() - theta[:, None]).float()
    got, ref = against_tv(t, d, "f32")
    assert (ref["near"] < 2e-7).all()                    # (the case is what it says)
    dist = np.abs((np32(t).astype(np.float64) - np32(d)) - theta.cpu().numpy()[:, None])
    assert (dist < 1e-7).sum() > 1000
    sure = dist > 1e-12                                  # (fp64's own sums are off by less)
    sign = np.sign(np32(got["grad_draft"]))
    assert (sign == np.sign(ref["grad_draft"]))[sure].all()


def test_tv_grad_agrees_with_differences():
    """The directional derivative of the fp64 TV, by central differences, along random directions: h = 2^-10 and 2^-11 extrapolated."""
    V, N, tau = 60, 4, 0.8
    t, d = rows((N,), V, "f32", 14, std=2.0), rows((N,), V, "f32", 15, std=2.0)
    g = np32(run_tv_grad(t, d, temperature_all=tau)["grad_draft"]).astype(np.float64)
    T, D = np32(t).astype(np.float64), np32(d).astype(np.float64)
    rng = np.random.default_rng(1)
    def tv(z):
        p, q = np.exp(T / tau), np.exp(z / tau)
        return 0.5 * np.abs(p / p.sum(1, keepdims=True) - q / q.sum(1, keepdims=True)).sum(1)
    for _ in range(20):
        v = rng.standard_normal((N, V)); v /= np.linalg.norm(v, axis=1, keepdims=True)
        d1, d2 = ((tv(D + h * v) - tv(D - h * v)) / (2 * h) for h in (2.0 ** -15, 2.0 ** -16))
        # smooth where no token crosses p = q within h: the difference's error is h^2 times a third derivative below 8 / tau^3, and 2^-52 / h of rounding
        smooth = np.abs(d1 - d2) < 1e-8
        assert smooth.any()
        assert (np.abs((g * v).sum(1) - (4 * d2 - d1) / 3)[smooth] < 1e-6).all()


def test_tv_grad_writes_its_rows_and_nothing_else():
    V, N = 1001, 6
    for dtype in ("f32", "bf16"):
        t, d = rows((N,), V, dtype, 16, extra=2), rows((N,), V, dtype, 17, extra=1)
        g, store = padded((N + 2,), V, dtype, fill=77.0, extra=3)
        r = run_tv_grad(t, d, out={"grad_draft": g[1:N + 1]}, want_tv=False, want_s_aux=False, want_status=False)
        assert r["tv"] is None and r["s_aux"] is None and r["row_status"] is None and r["grad_draft"].data_ptr() == g[1:N + 1].data_ptr()
        assert (store[:, V:] == 77).all() and (store[0] == 77).all() and (store[N + 1] == 77).all()
        assert torch.equal(r["grad_draft"], run_tv_grad(t, d)["grad_draft"])
        assert torch.equal(t[:, :3], rows((N,), V, dtype, 16, extra=2)[:, :3])


# ------------------------------------------------------------------ distillation
def teacher(N, V, T, dtype, seed, tau=None, tau_all=1.0):
    """A target's rows, their T largest logits in a random order, the rows' logsumexp."""
    z = rows((N,), V, dtype, seed)
    top = z.float().topk(T, dim=1)
    order = torch.rand((N, T), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).argsort(1)
    ids, val = top.indices.gather(1, order).int().contiguous(), top.values.gather(1, order)
    ts = torch.full((N, 1), tau_all, device=DEV, dtype=torch.float64) if tau is None else tau.double()[:, None]
    return z, ids, val.to(TYPES[dtype]), torch.logsumexp(z.double() / ts, 1).float()


def run_distill(*a, **kw):
    got = P.bebop_distill(*a, **kw)
    torch.cuda.synchronize()
    return got


def against_distill(d, ids, top, dtype, lse=None, g=None, tau=None, tau_all=1.0, **kw):
    got = run_distill(d, ids, top, target_lse=lse, temperature=tau, temperature_all=tau_all, grad_loss=g, **kw)
    ref = O.distill(np32(d), ids.cpu().numpy(), np32(top), np32(lse), np32(g), np32(tau), tau_all)
    scale = (np.ones(len(d)) if g is None else np.abs(np32(g))) / (tau_all if tau is None else np.where(np32(tau) > 0, np32(tau), 1.0))
    check_distill(got, ref, dtype, scale)
    return got, ref


@pytest.mark.parametrize("tail", [False, True], ids=["entries", "tail"])
@pytest.mark.parametrize("dtype,V,N", SIZES)
def test_distill_sizes(dtype, V, N, tail):
    T = max(1, min(V // 3, 37))
    tau = 0.6 + 0.6 * uniform((N,), 20)
    z, ids, top, lse = teacher(N, V, T, dtype, 21, tau)
    d = padded((N,), V, dtype, extra=1)[0].copy_(z + rows((N,), V, dtype, 22, std=1.0))
    against_distill(d, ids, top, dtype, lse=lse if tail else None, g=uniform((N,), 23) - 0.5, tau=tau)


@pytest.mark.parametrize("T", [1, 31, 33, 1000, 1024])
@pytest.mark.parametrize("tail", [False, True], ids=["entries", "tail"])
def test_distill_entry_counts(T, tail):
    """Lists of any length, of another type than the logits', down to every token of the vocabulary (no mass outside the entries)."""
    V = 1024
    z, ids, top, lse = teacher(4, V, T, "f32", 24)
    d = padded((4,), V, "bf16")[0].copy_(z + rows((4,), V, "f32", 25, std=1.0))
    if T == V:
        lse = lse + 1e-3                                  # (some mass the target's entries leave out, none outside them)
    got, ref = against_distill(d, ids, top, "bf16", lse=lse if tail else None)
    assert not (T == V and tail) or torch.isinf(got["loss"]).all()


@pytest.mark.parametrize("tail", [False, True], ids=["entries", "tail"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_ragged_and_ignored_rows(dtype, tail):
    V, N, T = 2500, 33, 40
    z, ids, top, lse = teacher(N, V, T, dtype, 26)
    d = padded((N,), V, dtype)[0].copy_(z + rows((N,), V, dtype, 27, std=1.0))
    have = torch.randint(0, T + 1, (N,), generator=torch.Generator(device=DEV).manual_seed(28), device=DEV)
    have[0], have[1], have[2] = 0, 1, T
    drop = torch.rand((N, T), generator=torch.Generator(device=DEV).manual_seed(29), device=DEV).argsort(1) >= have[:, None]      # (anywhere in the list)
    ids[drop] = -1
    top[drop] = float("nan")                              # what an unused entry holds does not matter
    d[0, :] = float("nan")                                # nor what an ignored row holds
    got, _ = against_distill(d, ids, top, dtype, lse=lse if tail else None)
    assert float(got["loss"][0]) == 0 and int(got["row_status"][0]) == 0 and not got["grad_draft"][0].any()


@pytest.mark.parametrize("tail", [False, True], ids=["entries", "tail"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distill_masks(dtype, tail):
    V, N, T = 900, 10, 16
    low = torch.finfo(TYPES[dtype]).min
    z, ids, top, lse = teacher(N, V, T, dtype, 30)
    d = padded((N,), V, dtype)[0].copy_(z + rows((N,), V, dtype, 31, std=1.0))
    d[0, int(ids[0, 0])] = -INF                           # the target gives mass to what the draft masks: an infinite loss
    top[1, 3] = -INF; d[1, int(ids[1, 3])] = -INF         # neither does
    outside = torch.ones(V, dtype=torch.bool, device=DEV); outside[ids[2].long()] = False
    d[2, outside] = -INF                                  # all the draft's mass on the entries
    d[3, outside] = -1e9
    d[4, :] = low                                         # q = 1 / V
    d[5, int(ids[5, 0])] = -low                           # one token above all
    d[6, ids[6].long()] = -INF                            # no entry has mass
    top[7, 1:] = -INF                                     # all the entries' mass on one
    top[8, :] = low
    d[9, :] = -1e9; d[9, 450] = 0
    if tail:
        lse[8] = float(low)
    against_distill(d, ids, top, dtype, lse=lse if tail else None)


@pytest.mark.parametrize("tail", [False, True], ids=["entries", "tail"])
def test_distill_status_and_fatal_rows(tail):
    V, N, T = 640, 14, 9
    z, ids, top, lse = teacher(N, V, T, "f32", 32)
    d = padded((N,), V, "f32")[0].copy_(z + 0.5)
    tau = torch.ones(N, device=DEV)
    d[0, int(ids[0, 2])] = float("nan"); d[1, 639] = INF; d[2, :] = -INF
    top[3, 4] = float("nan"); top[4, 0] = INF
    ids[5, 1] = V; ids[6, 8] = -2; ids[7, 3] = ids[7, 6]
    tau[8] = -1.0; ids[8, 0] = V
    top[9, :] = -INF
    ids[10, 0] = ids[10, 1]; d[10, 0] = float("nan")      # (a bad token alone decides)
    ids[11, :] = -1; d[11, :] = -INF                      # ignored
    lse[12] = float("nan")
    got, ref = against_distill(d, ids, top, "f32", lse=lse if tail else None, tau=tau)
    assert got["row_status"].tolist() == [1, 1, 2, 1, 1, 4, 4, 4, 16, 0 if tail else 2, 4, 0, 1 if tail else 0, 0]
    fatal = got["row_status"] != 0
    assert not got["grad_draft"][fatal].any() and not got["loss"][fatal].any()


def test_distill_agrees_with_differences():
    """The directional derivative of the fp64 loss by central differences: the loss is smooth (third derivative below 8 / tau^3), h = 2^-12:
    h^2 8 / (6 tau^3) + 2^-50 / h is below 3e-7; the kernel's fp32 error adds 1e-6 of the gradient's size."""
    V, N, T, tau = 50, 3, 7, 0.8
    z, ids, top, lse = teacher(N, V, T, "f32", 33, tau_all=tau)
    d = padded((N,), V, "f32")[0].copy_(z + rows((N,), V, "f32", 34, std=1.0))
    rng = np.random.default_rng(2)
    for tail in (None, lse):
        g = np32(run_distill(d, ids, top, target_lse=tail, temperature_all=tau)["grad_draft"]).astype(np.float64)
        f = lambda z: O.distill(z, ids.cpu().numpy(), np32(top), np32(tail), None, None, tau)["loss"]
        for _ in range(5):
            v, h = rng.standard_normal((N, V)), 2.0 ** -12
            v /= np.linalg.norm(v, axis=1, keepdims=True)
            D = np32(d).astype(np.float64)
            assert (np.abs((g * v).sum(1) - (f(D + h * v) - f(D - h * v)) / (2 * h)) < 3e-6).all()


def test_distill_without_gradient_and_into_buffers():
    V, N, T = 1001, 5, 12
    z, ids, top, lse = teacher(N, V, T, "bf16", 35)
    d = padded((N,), V, "bf16")[0].copy_(z + 0.25 * z.flip(1))
    full = run_distill(d, ids, top, target_lse=lse)
    r = run_distill(d, ids, top, target_lse=lse, want_grad=False, want_status=False)
    assert r["grad_draft"] is None and r["row_status"] is None and torch.equal(r["loss"], full["loss"])
    g, store = padded((N,), V, "bf16", fill=77.0, extra=2)
    out = {"grad_draft": g, "loss": torch.empty(N, device=DEV)}
    r = run_distill(d, ids, top, target_lse=lse, out=out, want_grad=False)
    assert r["loss"] is out["loss"] and r["grad_draft"] is g and torch.equal(g, full["grad_draft"]) and (store[:, V:] == 77).all()


# ------------------------------------------------------------------ target-only verification
def drafts(B, K, V, dtype, seed, tau=None, std=3.0, accept=(0.3, 1.0), extra=0):
    """Target rows whose drafts have probabilities uniform in `accept`, the drafts, the uniforms."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = rows((B, K + 1), V, dtype, seed, std=std, extra=extra)
    tok = torch.randint(0, V, (B, K), generator=g, device=DEV, dtype=torch.int32)
    ts = torch.ones(B, device=DEV) if tau is None else tau
    if V > 1:
        p = accept[0] + (accept[1] - accept[0]) * torch.rand((B, K), generator=g, device=DEV)
        others = z[:, :K].float().scatter(2, tok.long().unsqueeze(-1), -INF) / ts[:, None, None]
        zx = ts[:, None] * (torch.logsumexp(others, 2) + torch.logit(p.clamp(1e-3, 0.9995)))
        z[:, :K] = z[:, :K].scatter(2, tok.long().unsqueeze(-1), zx.unsqueeze(-1).to(z.dtype))
    return z, tok, uniform((B, K), seed + 1), uniform((B,), seed + 2)


def run_target_only(*a, **kw):
    got = P.bebop_target_only_verify(*a, **kw)
    torch.cuda.synchronize()
    return got


def against_target_only(z, tok, ua, uf, L=None, tau=None, tau_all=1.0):
    got = run_target_only(z, tok, ua, uf, draft_len=L, temperature=tau, temperature_all=tau_all)
    ref = O.target_only_verify(np32(z), tok.cpu().numpy(), ua.cpu().numpy(), uf.cpu().numpy(), None if L is None else L.cpu().numpy(), np32(tau), tau_all)
    check_target_only(got, ref)
    return got, ref


@pytest.mark.parametrize("dtype,V,B", SIZES)
@pytest.mark.parametrize("K", [1, 4])
def test_target_only_sizes(dtype, V, B, K):
    tau = 0.6 + 0.6 * uniform((B,), 40)
    against_target_only(*drafts(B, K, V, dtype, 41, tau, extra=1), tau=tau)


def test_target_only_thirty_two_drafts_and_all_lengths():
    B, K, V = 40, 32, 600
    x = drafts(B, K, V, "bf16", 42, accept=(0.9, 1.0))
    L = torch.arange(B, device=DEV, dtype=torch.int32) % 35 - 1          # (out of range lengths are taken as 0 and K)
    got, ref = against_target_only(*x, L=L)
    assert ref["accept_len"].max() > 20 and (ref["accept_len"] == 0).any()
    got, ref = against_target_only(x[0], x[1], torch.full_like(x[2], 2.0 ** -20), x[3])
    assert (got["accept_len"] == K).all()


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("dtype,std", [("bf16", 1.0), ("f32", 3.0)])
def test_target_only_draws_over_many_sequences(dtype, std, seed):
    """Flat and peaked rows, drawn from at a reject or behind the drafts: tokens as fp64 has them."""
    tau = 0.6 + 0.6 * uniform((256,), 50 + seed)
    against_target_only(*drafts(256, 2, 20000, dtype, 60 + 10 * seed, tau, std=std), tau=tau)


def test_target_only_draw_is_the_targets_distribution():
    """10^6 sequences of eight tokens: the first emitted token is distributed as p, whatever the draft (chi-squared, 7 degrees of freedom: 24.3 at 10^-3)."""
    B, V = 1 << 20, 8
    z = torch.randn((1, 2, V), generator=torch.Generator(device=DEV).manual_seed(70), device=DEV).expand(B, 2, V).contiguous()
    for draft in (int(z[0, 0].argmax()), int(z[0, 0].argmin())):
        r = run_target_only(z, torch.full((B, 1), draft, dtype=torch.int32, device=DEV), uniform((B, 1), 71), uniform((B,), 72))
        want = torch.softmax(z[0, 0].double(), 0) * B
        seen = torch.bincount(r["out_tokens"][:, 0].long(), minlength=V).double()
        assert float(((seen - want) ** 2 / want).sum()) < 24.3
        assert (r["row_status"] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_target_only_masks_and_rows_behind_the_stop(dtype):
    B, K, V = 9, 3, 1100
    low = torch.finfo(TYPES[dtype]).min
    z, tok, ua, uf = drafts(B, K, V, dtype, 80)
    never, always = 1.0 - 2.0 ** -24, 2.0 ** -24
    ua[0, 0] = never; z[0, 1:] = float("nan")             # rows behind the reject are not read
    z[1, 0, :] = -INF; z[1, 0, 7] = 1.0; tok[1, 0] = 3    # the draft has no probability: rejected, and 7 is drawn
    z[2, 0, :] = low; tok[2, 0] = 1099; ua[2, 0] = 0.5    # uniform row
    z[3, :] = -1e9                                        # uniform rows
    z[4, 0, :] = -INF; z[4, 0, int(tok[4, 0])] = 5.0      # the draft has all probability: accepted by any u < 1
    ua[4, 0] = never
    z[5, 0, :] = -INF; z[5, 0, int(tok[5, 0])] = -3.0; ua[5, 0] = 1.0       # ... and by u = 1 not: nothing is left to draw from
    ua[6] = always; z[6, K, :] = -INF; z[6, K, 1099] = 0.0                  # the bonus row has one token
    z[7, 0, :5] = -INF; uf[7] = always; ua[7, 0] = never                    # the first token with mass
    uf[8] = never; ua[8, 0] = never; z[8, 0, 900:] = -INF                   # the last
    got, ref = against_target_only(z, tok, ua, uf)
    assert int(got["row_status"][5]) == 8 and int(got["out_tokens"][5, 0]) == int(tok[5, 0])
    assert int(got["out_tokens"][1, 0]) == 7 and int(got["out_tokens"][6, K]) == 1099 and int(got["accept_len"][4]) >= 1
    assert int(got["out_tokens"][7, 0]) >= 5 and int(got["out_tokens"][8, 0]) < 900
    assert got["row_status"].tolist()[:5] == [0] * 5


def test_target_only_status_and_fatal_rows():
    B, K, V = 10, 3, 512
    z, tok, ua, uf = drafts(B, K, V, "f32", 81)
    tau = torch.ones(B, device=DEV)
    ua[:] = 2.0 ** -20
    z[0, 0, 511] = float("nan"); z[1, 2, 0] = INF; z[2, 1, :] = -INF; z[3, K, :] = -INF
    tok[4, 2] = V; tok[5, 0] = -1; tok[6, 1] = V
    tau[6] = 0.0; tau[7] = INF
    L = torch.full((B,), K, device=DEV, dtype=torch.int32)
    L[8] = 1; tok[8, 2] = -5; z[8, 2] = float("nan")      # beyond the drafts: neither tokens nor rows count
    got, ref = against_target_only(z, tok, ua, uf, L=L, tau=tau)
    assert got["row_status"].tolist() == [1, 1, 2, 2, 4, 4, 16, 16, 0, 0]
    fatal = got["row_status"] != 0
    assert not got["accept_len"][fatal].any() and (got["out_tokens"][fatal] == -1).all() and not got["p_draft"][fatal].any()


def test_target_only_nearly_certain_drafts():
    """Drafts of probability 1 - 2^-10 to 1 - 2^-22 that are rejected: the draw is from the little that is left."""
    B, V = 64, 5000
    z = rows((B, 2), V, "f32", 82)
    tok = torch.randint(0, V, (B, 1), generator=torch.Generator(device=DEV).manual_seed(83), device=DEV, dtype=torch.int32)
    others = torch.logsumexp(z[:, 0].scatter(1, tok.long(), -INF).double(), 1)
    z[:, 0] = z[:, 0].scatter(1, tok.long(), (others + torch.linspace(7, 15, B, device=DEV, dtype=torch.float64)).float()[:, None])
    got, ref = against_target_only(z, tok, torch.full((B, 1), 1.0 - 2.0 ** -24, device=DEV), uniform((B,), 84))
    assert (ref["accept_len"] == 0).all()


# ------------------------------------------------------------------ what all of them promise
def three(V=3000, dtype="bf16", seed=90):
    z, ids, top, lse = teacher(6, V, 20, dtype, seed)
    d = padded((6,), V, dtype)[0].copy_(z + rows((6,), V, dtype, seed + 1, std=1.0))
    x = drafts(6, 2, V, dtype, seed + 2)
    return [lambda **k: P.bebop_tv_grad(z, d, **k), lambda **k: P.bebop_distill(d, ids, top, target_lse=lse, **k), lambda **k: P.bebop_target_only_verify(*x, **k)]


def same(a, b):
    return all((a[k] is None and b[k] is None) or torch.equal(a[k], b[k]) for k in a)


def test_the_same_bits_every_time_on_any_stream_and_from_a_graph():
    for f in three():
        want = f()
        torch.cuda.synchronize()
        assert all(same(want, f()) for _ in range(3))
        streams = [torch.cuda.Stream() for _ in range(3)]
        got = []
        for i in range(12):                               # calls that overlap: no workspace is shared
            with torch.cuda.stream(streams[i % 3]):
                got.append(f())
        torch.cuda.synchronize()
        assert all(same(want, g) for g in got)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = f()
        for v in kept.values():
            v.zero_()
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert same(want, kept)


def test_a_call_starts_behind_the_work_before_it():
    """The launch overlaps the end of the kernel before it in the stream, but reads only what that has left."""
    V = 40000
    a, b = rows((64,), V, "bf16", 91), rows((64,), V, "bf16", 92)
    want = [run_tv_grad(a, b), run_tv_grad(b, a)]
    x, y = a.clone(), b.clone()
    for i in range(8):
        x.copy_(b if i % 2 else a); y.copy_(a if i % 2 else b)
        r = P.bebop_tv_grad(x, y)
        x.fill_(0)
        assert same(r, want[i % 2])


def test_a_wait_that_runs_out_returns_with_the_status_bit():
    for f in three():
        want = f()
        P.bebop_debug_expire_wait(1)
        r = f()
        torch.cuda.synchronize()
        assert (r["row_status"] == 32).all()
        for k in ("grad_draft", "loss", "tv", "accept_len"):
            assert k not in r or not r[k].any()
        assert same(f(), want)


def test_what_the_calls_refuse():
    t, d = rows((4,), 256, "f32", 93), rows((4,), 256, "f32", 94)
    ids, top = torch.arange(20, device=DEV, dtype=torch.int32).view(4, 5), torch.randn((4, 5), device=DEV)
    z, tok, ua, uf = drafts(4, 2, 256, "f32", 95)
    one = torch.ones(4, device=DEV)
    for f in (lambda: P.bebop_tv_grad(t, d[:3]), lambda: P.bebop_tv_grad(t, d.bfloat16()), lambda: P.bebop_tv_grad(t, d, grad_tv=one[:3]),
              lambda: P.bebop_tv_grad(t, d, grad_tv=one.double()), lambda: P.bebop_tv_grad(t, d, grad_tv=one[:1].expand(4)), lambda: P.bebop_tv_grad(t, d, temperature=one.cpu()),
              lambda: P.bebop_tv_grad(t, d, out={"tv": one[:2]}), lambda: P.bebop_tv_grad(t, d, out={"grad_draft": d.bfloat16()}),
              lambda: P.bebop_tv_grad(t, d, out={"grad_draft": torch.empty((256, 4), device=DEV).t()}),
              lambda: P.bebop_distill(d, ids.long(), top), lambda: P.bebop_distill(d, ids, top[:, :4]), lambda: P.bebop_distill(d, ids, top.t().contiguous().t()),
              lambda: P.bebop_distill(d, ids, top, target_lse=one[:2]), lambda: P.bebop_distill(d, ids, top, grad_loss=one.bfloat16()),
              lambda: P.bebop_target_only_verify(z, tok[:, :1], ua, uf), lambda: P.bebop_target_only_verify(z, tok, ua, uf[:1]),
              lambda: P.bebop_target_only_verify(z, tok.long(), ua, uf), lambda: P.bebop_target_only_verify(z, tok, ua, uf, draft_len=one),
              lambda: P.bebop_target_only_verify(z.transpose(0, 1), tok, ua, uf), lambda: P.bebop_target_only_verify(z[:, :1], tok[:, :0], ua[:, :0], uf)):
        with pytest.raises(AssertionError):
            f()
    for f in (lambda: P.bebop_tv_grad(t[0], d[0]), lambda: P.bebop_distill(z, ids, top), lambda: P.bebop_target_only_verify(t, tok, ua, uf)):
        with pytest.raises(ValueError):
            f()
    odd = torch.empty(4 * 255 + 8, device=DEV)
    for code, f in ((8, lambda: P.bebop_tv_grad(t.cpu(), d.cpu())), (3, lambda: P.bebop_tv_grad(t.half(), d.half())), (3, lambda: P.bebop_distill(d, ids, top.half())),
                    (6, lambda: P.bebop_tv_grad(t, d, temperature_all=0.0)), (6, lambda: P.bebop_distill(d, ids, top, temperature_all=float("nan"))),
                    (6, lambda: P.bebop_target_only_verify(z, tok, ua, uf, temperature_all=-1.0)),
                    (10, lambda: P.bebop_tv_grad(t, d, out={"grad_draft": d})), (10, lambda: P.bebop_tv_grad(t, d, out={"grad_draft": t})),
                    (10, lambda: P.bebop_distill(d, ids, top, out={"grad_draft": d})),
                    (4, lambda: P.bebop_tv_grad(t[:, :255], odd[1:1021].view(4, 255))), (4, lambda: P.bebop_tv_grad(t, d, out={"grad_draft": torch.empty((4, 258), device=DEV)[:, 1:257]})),
                    (2, lambda: P.bebop_tv_grad(t[:0], d[:0])), (2, lambda: P.bebop_distill(d, ids[:, :0], top[:, :0])), (2, lambda: P.bebop_target_only_verify(z[:, :1].contiguous(), tok[:, :0], ua[:, :0], uf)),
                    (2, lambda: P.bebop_distill(d, torch.zeros((4, 1025), dtype=torch.int32, device=DEV), torch.zeros((4, 1025), device=DEV))),
                    (2, lambda: P.bebop_target_only_verify(torch.zeros((4, 34, 8), device=DEV), torch.zeros((4, 33), dtype=torch.int32, device=DEV), torch.zeros((4, 33), device=DEV), uf))):
        with pytest.raises(P.BebopError) as e:
            f()
        assert e.value.code == code, code


def test_new_outputs_are_plain_tensors_of_their_own():
    for f in three(V=1001):
        r = f()
        assert len({v.untyped_storage().data_ptr() for v in r.values()}) == len(r)
        for v in r.values():
            assert not v.requires_grad and v.storage_offset() == 0 and v.is_cuda


# ------------------------------------------------------------------ together
def test_train_a_draft_head_and_verify_what_it_drafts():
    """A draft head (one matrix) takes a step on the TV loss and one on the target's top logits, with the gradients that autograd gives for the plain losses; its
    argmax drafts are then verified against the target."""
    g = torch.Generator(device=DEV).manual_seed(96)
    N, H, V, K, T = 24, 32, 1200, 3, 16
    hidden = torch.randn((N, H), generator=g, device=DEV)
    target = rows((N,), V, "f32", 97, std=2.0)
    W = (0.2 * torch.randn((H, V), generator=g, device=DEV)).requires_grad_()
    weight = torch.full((N,), 1.0 / N, device=DEV)
    top = target.topk(T, dim=1)
    lse = torch.logsumexp(target.double(), 1).float()
    p = torch.softmax(target.double(), 1)
    pt = top.values.double() - lse.double()[:, None]

    def plain_tv(z):
        return (weight.double() * 0.5 * (p - torch.softmax(z, 1)).abs().sum(1)).sum()

    def plain_top(z):
        lq = torch.log_softmax(z, 1).gather(1, top.indices)
        r, s = 1 - pt.exp().sum(1), 1 - lq.exp().sum(1)
        return (weight.double() * ((pt.exp() * (pt - lq)).sum(1) + r * (r / s).log())).sum()

    for step, plain in ((lambda z: P.bebop_tv_grad(target, z, grad_tv=weight), plain_tv),
                        (lambda z: P.bebop_distill(z, top.indices.int(), top.values, target_lse=lse, grad_loss=weight), plain_top)):
        W.grad = None
        z = hidden @ W
        r = step(z)
        z.backward(r["grad_draft"])
        got = W.grad.clone()
        W64 = W.detach().double().requires_grad_()
        plain(hidden.double() @ W64).backward()
        # the product's own fp32 (and TF32-free) sums of 24 rows and 32 inputs: 2^-24 sqrt-free bound 56 2^-24, the gradient rows 2^-19 of their size
        assert (got - W64.grad).abs().max() < 1e-5 * W64.grad.abs().max() + 1e-7
        with torch.no_grad():
            W -= 0.5 * got
    B = N // K
    drafted = (hidden @ W.detach()).argmax(1).int().view(B, K)
    z = torch.cat([target.view(B, K, V), rows((B, 1), V, "f32", 98)], 1).contiguous()
    against_target_only(z, drafted, uniform((B, K), 99), uniform((B,), 100))
