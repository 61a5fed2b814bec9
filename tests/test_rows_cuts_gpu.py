"""The operators around a draft head where rows are cut: runs of warps and chunks that end anywhere, many rows to a CTA with all kinds of rows among them, the largest vocabularies, and draws whose
target lies next to the border of a token."""
import numpy as np
import pytest
import torch

import oracle.rows as O
import paper_2606_12370_b200 as P
from rows64 import DEV, TYPES, check_distill, check_target_only, check_tv_grad, np32, padded, rows, uniform

pytestmark = pytest.mark.gpu
INF = float("inf")


def teacher(N, V, T, dtype, seed):
    z = rows((N,), V, dtype, seed)
    top = z.float().topk(T, dim=1)
    return z, top.indices.int().contiguous(), top.values.contiguous(), torch.logsumexp(z.double(), 1).float()


def all_three(V, N, dtype, seed):
    """Each operator on N rows of V tokens, against the oracle."""
    t = rows((N,), V, dtype, seed)
    d = rows((N,), V, dtype, seed + 1, extra=1)
    d.copy_(t + 0.3 * d)
    got = P.bebop_tv_grad(t, d)
    check_tv_grad(got, O.tv_grad(np32(t), np32(d)), dtype, np.ones(N))
    z, ids, top, lse = teacher(N, V, min(V, 50), dtype, seed + 2)
    got = P.bebop_distill(d, ids, top, target_lse=lse)
    check_distill(got, O.distill(np32(d), ids.cpu().numpy(), np32(top), np32(lse)), dtype, np.ones(N))
    x = rows((N, 3), V, dtype, seed + 3)
    tok = x[:, :2].float().argmax(2).int()
    ua, uf = uniform((N, 2), seed + 4), uniform((N,), seed + 5)
    got = P.bebop_target_only_verify(x, tok, ua, uf)
    check_target_only(got, O.target_only_verify(np32(x), tok.cpu().numpy(), ua.cpu().numpy(), uf.cpu().numpy()))


# a vector is 4 or 8 tokens, a row of a warp 32 vectors, a chunk 6 of them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [127, 128, 129, 255, 257, 767, 769, 1535, 1536, 1537, 1800, 6145, 12287, 12289, 24577, 49151, 98305])
def test_runs_and_chunks_that_end_anywhere(dtype, V):
    all_three(V, 3, dtype, V)


@pytest.mark.parametrize("V,N", [(4100, 400), (70001, 160)])
def test_more_rows_than_the_device_holds_at_a_time(V, N):
    """Rows of other lengths of run than the ring has slots, taken one after the other by the same CTA."""
    all_three(V, N, "bf16", 7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_all_kinds_of_rows_one_after_the_other(dtype):
    """What a row leaves behind -- marks, sums, open comparisons -- reaches no other row of its CTA."""
    N, V, T = 2000, 530, 20
    t = rows((N,), V, dtype, 300)
    d = rows((N,), V, dtype, 301)
    d.copy_(t + 0.3 * d)
    low = torch.finfo(TYPES[dtype]).min
    for z, at in ((t, 3), (d, 5)):
        z[at::29, 7] = float("nan"); z[at + 1::31, V - 1] = INF; z[at + 2::37, :] = -INF; z[at + 3::41, :] = -1e9; z[at + 4::43, : V - 3] = low
    d[10::17] = t[10::17]                                    # no token is above another
    tau = 0.6 + 0.6 * uniform((N,), 302)
    tau[11::53] = -1.0
    got = P.bebop_tv_grad(t, d, temperature=tau)
    scale = 1 / np.where(np32(tau) > 0, np32(tau), 1.0)
    check_tv_grad(got, O.tv_grad(np32(t), np32(d), temperature=np32(tau)), dtype, scale)
    _, ids, top, lse = teacher(N, V, T, "f32", 303)
    ids[2::23, 4] = -1; ids[4::47] = -1; ids[6::59, 0] = V; ids[8::61, 1] = ids[8::61, 2]
    got = P.bebop_distill(d, ids, top, target_lse=lse, temperature=tau)
    ref = O.distill(np32(d), ids.cpu().numpy(), np32(top), np32(lse), temperature=np32(tau))
    # (an entry at -3.4e38 and tau below 1: a loss of p 3.4e38 / tau lies above the largest float, and rounds to inf)
    assert (np.abs(ref["loss"]) > 3.4028235677973366e38).any() or dtype == "bf16"
    ref["loss"] = np.where(np.abs(ref["loss"]) > 3.4028235677973366e38, np.inf, ref["loss"])
    check_distill(got, ref, dtype, scale)
    x = torch.stack([d, t], 1)
    x = padded((N, 2), V, dtype)[0].copy_(x)
    tok = torch.randint(-1, V, (N, 1), generator=torch.Generator(device=DEV).manual_seed(304), device=DEV, dtype=torch.int32)
    ua, uf = uniform((N, 1), 305), uniform((N,), 306)
    got = P.bebop_target_only_verify(x, tok, ua, uf, temperature=tau)
    check_target_only(got, O.target_only_verify(np32(x), tok.cpu().numpy(), ua.cpu().numpy(), uf.cpu().numpy(), temperature=np32(tau)))


@pytest.mark.parametrize("dtype,V", [("f32", 1 << 24), ("bf16", 13000001), ("bf16", 3000003)])
def test_the_largest_vocabularies(dtype, V):
    """Sixteen CTAs a row; of distillation the marks of one row alone fill their shared memory.  Checked on the device: sums in double."""
    t = rows((2,), V, dtype, 310, std=2.0)
    d = rows((2,), V, dtype, 311, std=0.5)
    d.copy_(t + d)
    log = lambda z: torch.log_softmax(z.double(), 1)
    lp, lq = log(t), log(d)
    got = P.bebop_tv_grad(t, d)
    # (sums of terms that are off by 2^-20 at most, all of their weighted mean)
    tv = 0.5 * (lp.exp() - lq.exp()).abs().sum(1)
    assert (got["row_status"] == 0).all() and ((got["tv"].double() - tv).abs() <= 2.0 ** -18).all()
    below = lq <= lp
    s = (lq.exp() * below).sum(1, keepdim=True)
    assert ((got["s_aux"].double() - s[:, 0]).abs() <= 2.0 ** -18).all()
    ref = -lq.exp() * (below.double() - s)
    near = (lq - lp).abs() < 1e-9
    step = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    assert ((got["grad_draft"].double() - ref).abs() <= lq.exp() * 2.0 ** -17 + step * ref.abs())[~near].all()
    ids = torch.randperm(V, generator=torch.Generator(device=DEV).manual_seed(312), device=DEV)[:2048].view(2, 1024).int()
    ids[:, 0], ids[:, 1] = 0, V - 1
    top = t.float().gather(1, ids.long()) + 12
    got = P.bebop_distill(d, ids, top)
    p = torch.softmax(top.double(), 1)
    loss = (p * (p.log() - lq.gather(1, ids.long()))).sum(1)
    assert (got["row_status"] == 0).all() and ((got["loss"].double() - loss).abs() <= 2.0 ** -18 * (1 + loss)).all()
    ref = lq.exp().scatter_add(1, ids.long(), -p)
    size = lq.exp().scatter_add(1, ids.long(), p)
    assert ((got["grad_draft"].double() - ref).abs() <= size * 2.0 ** -17 + step * ref.abs()).all()
    x = padded((1, 2), V, dtype)[0]
    x[0].copy_(t)
    tok = torch.tensor([[V - 1]], device=DEV, dtype=torch.int32)
    for u in (0.001, 0.5, 0.99):
        got = P.bebop_target_only_verify(x, tok, torch.full((1, 1), 1.0, device=DEV), torch.full((1,), u, device=DEV))
        e = lp[0].exp()
        e[V - 1] = 0
        c = e.cumsum(0)
        target = float(torch.tensor(u, dtype=torch.float32)) * c[-1]
        y = int(got["out_tokens"][0, 0])
        assert int(got["accept_len"][0]) == 0 and float(c[y] - e[y] - target) <= 1e-12 and float(target - c[y]) <= 1e-12


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,std", [(300, 3.0), (5000, 1.0), (40000, 2.0)])
def test_draws_next_to_the_border_of_a_token(dtype, V, std):
    """u_final as near to a border of the distribution as floats allow, on either side: closer than fp32 sums tell."""
    B = 256
    x = rows((B, 2), V, dtype, 320 + V, std=std)
    tok = torch.zeros((B, 1), dtype=torch.int32, device=DEV)
    c = torch.softmax(x[:, 1].double(), 1).cumsum(1)
    at = torch.randint(0, V - 1, (B,), generator=torch.Generator(device=DEV).manual_seed(321), device=DEV)
    uf = (c.gather(1, at[:, None])[:, 0] / c[:, -1]).float()
    uf[1::4] = torch.nextafter(uf[1::4], torch.zeros_like(uf[1::4])); uf[2::4] = torch.nextafter(uf[2::4], torch.ones_like(uf[2::4]))
    uf = uf.clamp(2.0 ** -24, 1 - 2.0 ** -24)
    L = torch.zeros(B, dtype=torch.int32, device=DEV)
    for row in (0, 1):                                       # behind the drafts, and at a rejected draft
        z = padded((B, 2), V, dtype)[0]
        z[:, 0], z[:, 1] = x[:, 1], x[:, 1]
        lens = L if row == 0 else L + 1
        ua = torch.full((B, 1), 1.0, device=DEV)
        got = P.bebop_target_only_verify(z, tok, ua, uf, draft_len=lens)
        ref = O.target_only_verify(np32(z), tok.cpu().numpy(), ua.cpu().numpy(), uf.cpu().numpy(), lens.cpu().numpy())
        # (what 64 bits cannot tell either: 1e-12 of the row)
        p = torch.softmax(x[:, 1].double(), 1)
        m = p.gather(1, torch.as_tensor(ref["out_tokens"][:, 0], device=DEV).long()[:, None])[:, 0].cpu().numpy()
        sure = ref["margin_cdf"] * m > 1e-12
        assert sure.mean() > 0.95 and (got["accept_len"].cpu().numpy() == 0).all()
        wrong = (got["out_tokens"].cpu().numpy() != ref["out_tokens"]).any(1) & sure
        assert not wrong.any(), np.nonzero(wrong)[0][:5]


def test_a_shape_met_first_in_a_capture_and_calls_from_several_threads():
    """What the host works out for a shape (cuts, how many clusters fit) needs no call before the capture, and no lock."""
    import threading
    def calls(V, seed):
        t, d = rows((37,), V, "bf16", seed), rows((37,), V, "bf16", seed + 1)
        _, ids, top, lse = teacher(37, V, 11, "bf16", seed + 2)
        x = rows((5, 3), V, "bf16", seed + 3)
        tok = x[:, :2].float().argmax(2).int()
        ua, uf = uniform((5, 2), seed + 4), uniform((5,), seed + 5)
        return [lambda: P.bebop_tv_grad(t, d), lambda: P.bebop_distill(d, ids, top, target_lse=lse), lambda: P.bebop_target_only_verify(x, tok, ua, uf)]
    for f in calls(23456, 330):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kept = f()
        graph.replay()
        torch.cuda.synchronize()
        want = f()
        assert all((kept[k] is None and want[k] is None) or torch.equal(kept[k], want[k]) for k in want)
    jobs = [(calls(V, V), [None] * 3) for V in (1111, 5555, 23457, 44444)]
    torch.cuda.synchronize()

    def work(fs, out):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                for i, f in enumerate(fs):
                    out[i] = f()
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    for fs, out in jobs:
        for f, got in zip(fs, out):
            want = f()
            assert all((got[k] is None and want[k] is None) or torch.equal(got[k], want[k]) for k in want)
