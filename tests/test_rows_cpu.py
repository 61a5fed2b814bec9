"""The operators around a draft head without a GPU: what the C ABI refuses before it touches a device, and the pins of their fp64 oracle."""
import math

import numpy as np
import pytest

import oracle
import oracle.rows as O
import paper_2606_12370_b200 as P
from paper_2606_12370_b200 import build as B

FAKE = 0x100000       # never dereferenced: every call below fails a host check first


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.load_library()


def call(lib, op, **kw):
    a = dict(target=FAKE, ldt=1024, draft=FAKE + (1 << 20), ldd=1024, tok=FAKE, dl=None, temp=None, tall=1.0, ua=FAKE, uf=FAKE, B=4, K=3, N=4, V=1024, dt=0, acc=FAKE, out=FAKE, pd=None, st=None,
             g=None, grad=FAKE + (1 << 24), ldg=1024, tv=None, sx=None, ids=FAKE, top=FAKE, tdt=0, T=8, lse=None, loss=FAKE)
    a.update(kw)
    v = a.__getitem__
    names = {"target_only": "target ldt tok dl temp tall ua uf B K V dt acc out pd st", "tv_grad": "target ldt draft ldd temp tall g N V dt grad ldg tv sx st",
             "distill": "draft ldd ids top tdt T lse temp tall g N V dt loss grad ldg st"}[op].split()
    return getattr(lib, {"target_only": "bebop_target_only_verify", "tv_grad": "bebop_tv_grad", "distill": "bebop_distill"}[op])(*map(v, names), None)


def test_target_only_refusals(lib):
    f = lambda **k: call(lib, "target_only", **k)
    assert f(B=0) == 2 and f(K=0) == 2 and f(K=33) == 2 and f(V=0) == 2 and f(B=1 << 27) == 2 and f(ldt=1000) == 2
    assert f(dt=2) == 3
    for k in ("target", "tok", "ua", "uf", "acc", "out"):
        assert f(**{k: None}) == 1, k
    assert f(target=FAKE + 4) == 4 and f(V=1021, ldt=1021) == 4
    assert f(tall=0.0) == 6 and f(tall=math.inf) == 6 and f(tall=math.nan) == 6


def test_tv_grad_refusals(lib):
    f = lambda **k: call(lib, "tv_grad", **k)
    assert f(N=0) == 2 and f(N=1 << 27) == 2 and f(V=-1) == 2 and f(ldt=1000) == 2 and f(ldd=1000) == 2 and f(ldg=1000) == 2
    assert f(dt=-1) == 3
    for k in ("target", "draft", "grad"):
        assert f(**{k: None}) == 1, k
    assert f(grad=FAKE + (1 << 24) + 8) == 4 and f(ldg=1025) == 4 and f(draft=FAKE + (1 << 20) + 4) == 4
    assert f(tall=-1.0) == 6
    end = FAKE + 4 * (3 * 1024 + 1024)                    # behind the target's last row
    assert f(grad=FAKE) == 10 and f(grad=FAKE + (1 << 20)) == 10 and f(grad=end - 16) == 10 and f(grad=FAKE + (1 << 20) - 16) == 10
    assert f(grad=FAKE + (1 << 20) + 2048, ldg=2048, V=512, ldd=1024) == 10          # (interleaved rows count as shared: the ranges meet)


def test_distill_refusals(lib):
    f = lambda **k: call(lib, "distill", **k)
    assert f(N=0) == 2 and f(T=0) == 2 and f(T=1025) == 2 and f(V=(1 << 24) + 8, ldd=(1 << 24) + 8) == 2 and f(ldg=1000) == 2
    assert f(dt=3) == 3 and f(tdt=3) == 3
    for k in ("draft", "ids", "top", "loss"):
        assert f(**{k: None}) == 1, k
    assert f(draft=FAKE + (1 << 20) + 4) == 4 and f(grad=FAKE + (1 << 24) + 4) == 4
    assert f(tall=0.0) == 6 and f(grad=FAKE + (1 << 20)) == 10
    assert P.bebop_status_string(10) not in {P.bebop_status_string(i) for i in range(10)}


# ------------------------------------------------------------------ the oracle
def model(N, V, seed, std=2.0):
    return (np.random.default_rng(seed).standard_normal((N, V)) * std).astype(np.float32)


def test_tv_grad_oracle_is_the_c_oracle_and_the_derivative_of_its_value():
    t, d = model(5, 40, 1), model(5, 40, 2)
    tau = np.array([0.7, 1.0, 1.3, 0.9, 2.0], np.float32)
    o, c = O.tv_grad(t, d, None, tau), oracle.tv(t, d, temperature=tau)
    assert np.abs(o["tv"] - c["tv"]).max() < 1e-13 and np.abs(o["s_aux"] - c["s_aux"]).max() < 1e-13
    h = 2.0 ** -14
    for j in range(40):
        for s in (1,):
            up, dn = d.astype(np.float64), d.astype(np.float64)
            up[:, j] += h; dn[:, j] -= h
            tv = lambda z: O.tv_grad(t, z, None, tau)["tv"]
            diff = (tv(up) - tv(dn)) / (2 * h)
            smooth = o["near"] > 4 * h                    # no token crosses p = q
            assert (np.abs(diff - o["grad_draft"][:, j])[smooth] < 1e-8).all()
    assert (o["near"] > 4 * h).any()
    assert np.abs(o["grad_draft"].sum(1)).max() < 1e-15   # (a shift of a row changes nothing)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_oracle_is_the_derivative_of_its_value(tail):
    N, V, T, tau = 3, 30, 6, float(np.float32(0.8))
    t, d = model(N, V, 3), model(N, V, 4)
    ids = np.argsort(-t, axis=1)[:, :T].astype(np.int32)
    top = np.take_along_axis(t, ids, 1)
    lse = np.array([math.log(math.fsum(np.exp(r.astype(np.float64) / tau))) for r in t], np.float32) if tail else None
    o = O.distill(d, ids, top, lse, None, None, tau)
    assert np.abs(o["grad_draft"].sum(1)).max() < 1e-14
    h = 2.0 ** -14
    for j in range(V):
        up, dn = d.astype(np.float64), d.astype(np.float64)
        up[:, j] += h; dn[:, j] -= h
        f = lambda z: O.distill(z, ids, top, lse, None, None, tau)["loss"]
        assert np.abs((f(up) - f(dn)) / (2 * h) - o["grad_draft"][:, j]).max() < 1e-7
    # entries of the whole vocabulary: the forward KL; the target itself: nothing to learn
    every = np.tile(np.arange(V, dtype=np.int32), (N, 1))
    kl = O.distill(d, every, t, None, None, None, tau)["loss"]
    for i in range(N):
        lp, lq = O.log_softmax(t[i], tau)[0], O.log_softmax(d[i], tau)[0]
        assert abs(kl[i] - float((np.exp(lp) * (lp - lq)).sum())) < 1e-12
    z = O.distill(t, ids, top, lse, None, None, tau)
    if tail:
        assert np.abs(z["loss"]).max() < 1e-6 and np.abs(z["grad_draft"]).max() < 1e-6       # (lse is rounded to fp32)


def test_target_only_oracle_agrees_with_a_certain_draft_distribution():
    """Target-only sampling is rejection sampling from a draft distribution with all its mass on the draft."""
    Bn, K, V = 200, 3, 12
    rng = np.random.default_rng(5)
    t = (rng.standard_normal((Bn, K + 1, V)) * 2).astype(np.float32)
    tok = rng.integers(0, V, (Bn, K)).astype(np.int32)
    ua, uf = rng.random((Bn, K)).astype(np.float32), rng.random(Bn).astype(np.float32)
    d = np.full((Bn, K, V), -np.inf, np.float32)
    np.put_along_axis(d, tok[:, :, None].astype(np.int64), 0.0, 2)
    L = rng.integers(0, K + 1, Bn).astype(np.int32)
    a, b = O.target_only_verify(t, tok, ua, uf, L, None, 0.9), oracle.verify(t, d, tok, ua, uf, draft_len=L, temperature_all=0.9)
    ok = ~a["flagged"] & ~b["flagged"]
    assert ok.mean() > 0.99
    assert (a["accept_len"] == b["accept_len"])[ok].all() and (a["out_tokens"] == b["out_tokens"])[ok].all()
    read = a["p_draft"] > 0
    assert np.abs(a["p_draft"] - b["p_draft"])[read].max() < 1e-14
