"""GPU parity of the router's balance loss, the gradient of its logits and the
dense router backward, against the fp64 oracle.

u = 2^-24.  A probability: exp is good to 2 ulp, its argument z - max is rounded
once (|z - max| u absolute), the sum over the experts takes at most 4 + 6 steps, the
quotient 2: p is off by (20 + max|z - max|) 2 u of itself.  counts are exact.  dprob is formed in
fp64 and rounded once.  The products are fp32 sums: the number of terms bounds the
roundings; a bf16 dX adds half a step (2^-8) and may keep 16 bits of dlogits (2^-16)."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

from gpu_harness import log

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def draw(T, E, k, B, pad, seed=0):
    g = torch.Generator().manual_seed(1000 * T + 10 * E + seed)
    z = 3 * torch.randn(T, E, generator=g)
    idx = torch.topk(z, k, dim=1)[1].int()
    seg = torch.cat((torch.zeros(1), torch.sort(torch.randint(0, T + 1, (B - 1,), generator=g))[0], torch.tensor([T]))).int()
    keep = (torch.rand(T, generator=g) >= pad).to(torch.uint8)
    gate = torch.softmax(torch.gather(z, 1, idx.long()), 1)
    return [t.to(DEV) for t in (z, idx, seg, keep, gate, torch.randn(T, k, generator=g))]


def loss_of(z, idx, coef, seg=None, keep=None):
    T, E = z.shape
    B = 1 if seg is None else len(seg) - 1
    counts = torch.full((B, E), -7, dtype=torch.int32, device=DEV)
    dprob, loss = torch.full((B, E), float("nan"), device=DEV), torch.full((1,), float("nan"), device=DEV)
    ws = torch.full((api.moe_balance_loss_workspace_size(T, E, B),), 0xFF, dtype=torch.uint8, device=DEV)
    api.moe_balance_loss(z, idx, coef, counts, dprob, loss, ws, seg=seg, keep=keep)
    return counts, dprob, loss


def check(z, idx, seg, keep, gate, dg, coef=0.02, up=1.5):
    T, E = z.shape
    k = idx.shape[1]
    hs, hk = (None if seg is None else seg.cpu().numpy()), (None if keep is None else keep.cpu().numpy())
    counts, dprob, loss = loss_of(z, idx, coef, seg, keep)
    z64 = f64(z)
    c, dp, l = O.balance_loss(z64, idx.cpu().numpy(), k, coef, hs, hk)
    np.testing.assert_array_equal(counts.cpu().numpy(), c)
    np.testing.assert_allclose(f64(dprob), dp, rtol=2 * U, atol=0)
    with np.errstate(invalid="ignore"):
        top = z64.max(1, keepdims=True)
        reach = np.where(np.isfinite(z64), np.abs(z64 - np.where(np.isfinite(top), top, 0)), 0)
    rel = 2 * U * (20 + reach.max(1, initial=0))[:, None]
    assert abs(float(loss) - l) <= (float(rel.max(initial=0)) + 66 * U) * abs(l)
    dl = torch.full_like(z, float("nan"))
    dloss = torch.tensor([up], device=DEV)
    api.moe_balance_loss_bwd(z, dprob, dloss, dl, seg=seg, keep=keep, gate=gate, idx=idx if gate is not None else None,
                             dgate=dg)
    want = O.balance_loss_backward(z64, dp, up, hs, hk, f64(gate), idx.cpu().numpy(), f64(dg))
    p = O.full_softmax(z64)
    w = np.zeros((T, E))
    for b in range(len(dp)):
        w[slice(None) if hs is None else slice(hs[b], hs[b + 1])] = dp[b]
    tol = abs(up) * p * (2 * rel + 16 * U) * (np.abs(w) + (p * np.abs(w)).sum(1, keepdims=True))
    if gate is not None:
        ga, da = np.abs(f64(gate)), np.abs(f64(dg))
        share = (k + 6) * U * ga * (da + (ga * da).sum(1, keepdims=True))
        for j in range(k):
            e = idx.cpu().numpy()[:, j]
            ok = (e >= 0) & (e < E)
            np.add.at(tol, (np.nonzero(ok)[0], e[ok]), share[ok, j])
        tol = tol + k * U * np.abs(want)
    err = np.abs(f64(dl) - want)
    assert np.all(err <= tol), (float((err - tol).max()), np.argwhere(err > tol)[:3])
    return counts, dprob, loss, dl


CASES = [(1, 1, 1, 1, 0.0), (1, 8, 2, 3, 0.0), (5, 3, 3, 1, 0.0), (64, 8, 2, 1, 0.0), (65, 16, 4, 4, 0.2), (200, 9, 2, 7, 0.3),
         (333, 17, 5, 64, 0.1), (1000, 64, 6, 5, 0.0), (777, 65, 8, 3, 0.5), (129, 100, 16, 1, 0.1), (500, 129, 3, 2, 0.0),
         (300, 256, 16, 300, 0.2), (4096, 64, 8, 1, 0.0), (130, 33, 1, 4000, 0.0)]


@pytest.mark.parametrize("T,E,k,B,pad", CASES)
def test_loss_and_logits_gradient(T, E, k, B, pad):
    z, idx, seg, keep, gate, dg = draw(T, E, k, B, pad)
    check(z, idx, seg, keep if pad else None, gate, dg)
    check(z, idx, None, keep, None, None)
    check(z, idx, None, None, gate, dg, coef=-0.5, up=-2.0)


def test_sequences_that_leave_tokens_out():
    """Tokens before the first and behind the last sequence, empty sequences, all of a
    sequence masked, everything masked, one token kept."""
    z, idx, _, keep, gate, dg = draw(150, 12, 3, 1, 0.0)
    seg = torch.tensor([10, 10, 70, 70, 71, 140], dtype=torch.int32, device=DEV)
    counts, dprob, loss, dl = check(z, idx, seg, None, None, None)
    assert not counts[0].any() and int(counts.sum()) == 3 * 130 and not dl[:10].any() and not dl[140:].any()
    keep[10:70] = 0
    counts, dprob, loss, dl = check(z, idx, seg, keep, None, None)
    assert not counts[1].any() and not dprob[1].any() and not dl[10:70].any()
    keep[:] = 0
    counts, dprob, loss, dl = check(z, idx, seg, keep, gate, dg)
    assert float(loss) == 0 and not counts.any() and not dprob.any() and bool(dl.any())
    keep[100] = 9
    counts, _, _, dl = check(z, idx, None, keep, None, None)
    assert int(counts.sum()) == 3 and not dl[99].any()
    # no tokens at all
    e = torch.empty(0, 12, device=DEV)
    counts, dprob, loss = loss_of(e, torch.empty(0, 3, dtype=torch.int32, device=DEV), 0.1, torch.zeros(5, dtype=torch.int32, device=DEV))
    assert float(loss) == 0 and not counts.any() and not dprob.any()


def test_infinities_nan_and_bad_entries():
    z, idx, seg, keep, gate, dg = draw(96, 70, 2, 3, 0.0)
    z[:, 5] = float("-inf")                            # an expert that nobody may take
    z[7] = float("-inf")                               # a row that a mask leaves empty
    z[8, :69] = float("-inf")                          # one expert left
    z[9] = torch.finfo(torch.float32).min              # a mask of the type's lowest value: even
    idx[20, 0], idx[21, 1], idx[22] = -1, 70, 3        # no expert, no expert, the same one twice
    counts, _, _, dl = check(z, idx, seg, None, gate, dg)
    _, _, _, dl = check(z, idx, seg, None, None, None)
    assert int(counts.sum()) == 2 * 96 - 2 and not dl[7].any() and not dl[8].any()
    assert not dl[:9, 5].any() and not dl[10:, 5].any()    # row 9 holds the lowest value there, not -inf
    # NaN in masked rows stays out; in a live row it reaches that row's gradient and the loss
    keep[30:34] = 0
    clean = check(z, idx, seg, keep, None, None)
    y = z.clone()
    y[30], y[31, 2], y[33] = float("nan"), float("inf"), float("-inf")
    for a, b in zip(loss_of(y, idx, 0.02, seg, keep), clean):
        assert torch.equal(a, b)
    out = torch.empty_like(z)
    api.moe_balance_loss_bwd(y, clean[1], torch.tensor([1.5], device=DEV), out, seg=seg, keep=keep)
    assert torch.equal(out, clean[3])
    y = z.clone()
    y[40, 3] = float("nan")
    c, dp, l = loss_of(y, idx, 0.02, seg, keep)
    assert torch.isnan(l).all() and torch.equal(c, clean[0]) and torch.equal(dp, clean[1])
    api.moe_balance_loss_bwd(y, dp, None, out, seg=seg, keep=keep)
    assert torch.isnan(out[40]).all() and torch.isfinite(out[:40]).all() and torch.isfinite(out[41:]).all()
    # the gradient in the logits' place
    want = torch.empty_like(z)
    api.moe_balance_loss_bwd(z, dp, None, want, seg=seg, keep=keep)
    same = z.clone()
    api.moe_balance_loss_bwd(same, dp, None, same, seg=seg, keep=keep)
    assert torch.equal(same, want)


def router(dl, X, Wr, dx=True, dw=True, db=True, old=None):
    T, E = dl.shape
    d = X.shape[1]
    new = lambda *s, t=torch.float32: torch.full(s, float("nan"), dtype=t, device=DEV)  # noqa: E731
    out = dict(dX=new(T, d, t=X.dtype) if dx else None, dWr=new(E, d) if dw else None, dbias=new(E) if db else None)
    if old is not None:
        out = {n: old[n].clone() for n in out}
    ws = torch.full((max(1, api.moe_router_bwd_workspace_size(T, d, E)),), 0xFF, dtype=torch.uint8, device=DEV)
    api.moe_router_bwd(dl, X if dw else None, Wr if dx else None, ws, accumulate_dx=old is not None,
                       accumulate_dw=old is not None, **out)
    return out


def check_router(out, dl, X, Wr, old=None):
    a, x, w = f64(dl), f64(X), f64(Wr)
    T, E = a.shape
    base = {n: 0.0 if old is None else f64(old[n]) for n in out}
    bf = X.dtype == torch.bfloat16
    for n, want, tol in (("dX", a @ w, (2.0 ** -16 if bf else 0) + (E + 4) * U, ), ("dWr", a.T @ x, (T + 40) * U),
                         ("dbias", a.sum(0), (T + 40) * U)):
        if out[n] is None:
            continue
        mag = {"dX": np.abs(a) @ np.abs(w), "dWr": np.abs(a).T @ np.abs(x), "dbias": np.abs(a).sum(0)}[n]
        want = want + base[n]
        tol = tol * mag + 2 * U * np.abs(base[n]) + ((2.0 ** -8 if bf and n == "dX" else U) * np.abs(want))
        err = np.abs(f64(out[n]) - want)
        assert np.all(err <= tol), (n, float((err / np.maximum(tol, 1e-300)).max()), np.argwhere(err > tol)[:3])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,E", [(1, 8, 1), (3, 24, 5), (31, 136, 8), (32, 128, 16), (65, 264, 33), (64, 512, 64),
                                   (200, 1000, 65), (130, 72, 129), (257, 144, 256), (1500, 2048, 64), (3000, 40, 9)])
def test_router_backward(T, d, E, dt):
    g = torch.Generator().manual_seed(T + d + E)
    dl = (torch.randn(T, E, generator=g) * torch.exp(2 * torch.randn(T, 1, generator=g))).to(DEV)
    X, Wr = torch.randn(T, d, generator=g).to(dt).to(DEV), torch.randn(E, d, generator=g).to(dt).to(DEV)
    out = router(dl, X, Wr)
    check_router(out, dl, X, Wr)
    old = dict(dX=torch.randn(T, d, generator=g).to(dt).to(DEV), dWr=torch.randn(E, d, generator=g).to(DEV),
               dbias=torch.randn(E, generator=g).to(DEV))
    check_router(router(dl, X, Wr, old=old), dl, X, Wr, old)
    for how in (dict(dx=False), dict(dw=False), dict(db=False), dict(dw=False, db=False), dict(dx=False, dw=False)):
        part = router(dl, X, Wr, **how)
        check_router(part, dl, X, Wr)
        if not (part["dX"] is None and part["dWr"] is None):   # dbias alone has no type: the fp32 kernel sums it
            assert all(v is None or torch.equal(v, out[n]) for n, v in part.items()), how


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,E", [(33 * 64, 264, 20), (33 * 64, 2048, 64), (35 * 64 + 1, 136, 130), (65 * 64, 512, 33)])
def test_router_backward_slabs_that_do_not_divide(T, d, E, dt):
    """More slabs of 64 tokens than parts of the token range, and no multiple of them:
    whole slabs in each part leave fewer parts."""
    test_router_backward(T, d, E, dt)


def test_router_backward_without_tokens_and_sparse():
    e = torch.empty(0, 8, device=DEV)
    X = torch.empty(0, 16, device=DEV)
    out = router(e, X, torch.randn(8, 16, device=DEV))
    assert not out["dWr"].any() and not out["dbias"].any()
    # against the sparse backward: gradients on the selected experts alone
    T, d, E, k = 100, 264, 24, 4
    z, idx, _, _, gate, dg = draw(T, E, k, 1, 0.0)
    Wr = torch.randn(E, d, device=DEV)
    dl = torch.empty_like(z)
    api.moe_balance_loss_bwd(z, torch.zeros(1, E, device=DEV), None, dl, gate=gate, idx=idx, dgate=dg)
    want = torch.empty(T, d, device=DEV)
    api.moe_route_bwd(gate, idx, dg, Wr, want)
    got = router(dl, torch.randn(T, d, device=DEV), Wr)["dX"]
    assert float((got - want).norm()) <= 1e-6 * float(want.norm())


def test_router_products_past_32_bits():
    """X and dX of 2^31 + 2^18 elements, a bf16 d of 2048."""
    d, E = 2048, 4
    T = (1 << 20) + 128
    dl = torch.zeros(T, E, device=DEV)
    dl[-1, 1], dl[5, 3], dl[1 << 20, 2] = 2.0, 1.0, -1.0
    X = torch.ones(T, d, dtype=torch.bfloat16, device=DEV)
    X[-1] = 3.0
    Wr = torch.randn(E, d, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16).to(DEV)
    out = router(dl, X, Wr)
    assert torch.equal(out["dWr"].cpu(), torch.tensor([0., 6., -1., 1.])[:, None].expand(E, d))
    assert out["dbias"].tolist() == [0, 2, -1, 1]
    assert torch.equal(out["dX"][-1], 2 * Wr[1]) and torch.equal(out["dX"][1 << 20], -Wr[2]) and not out["dX"][6].any()
    assert int((out["dX"] != 0).any(1).sum()) == 3


def test_gradient_by_differences():
    """The GPU's own loss, nudged along a random direction: its third derivative is of
    the loss's size, so a step of 1e-2 is off by 1e-4, and 2^-24 of the loss over the step by 1e-5."""
    z, idx, seg, keep, _, _ = draw(60, 20, 3, 4, 0.2)
    _, dprob, _ = loss_of(z, idx, 1.0, seg, keep)
    dl = torch.empty_like(z)
    api.moe_balance_loss_bwd(z, dprob, None, dl, seg=seg, keep=keep)
    h, dirn = 1e-2, torch.randn(z.shape, generator=torch.Generator().manual_seed(1)).to(DEV)
    up, dn = (float(loss_of(z + s * h * dirn, idx, 1.0, seg, keep)[2]) for s in (1, -1))
    assert abs((up - dn) / (2 * h) - float((dl * dirn).sum())) <= 1e-3 * float((dl * dirn).abs().sum())


def test_captured_and_replayed():
    T, E, k, d = 400, 64, 6, 264
    z, idx, seg, keep, gate, dg = draw(T, E, k, 5, 0.1)
    X, Wr = (torch.randn(n, d, device=DEV).to(torch.bfloat16) for n in (T, E))
    out = dict(counts=torch.empty(5, E, dtype=torch.int32, device=DEV), dprob=torch.empty(5, E, device=DEV),
               loss=torch.empty(1, device=DEV), dl=torch.empty(T, E, device=DEV),
               dX=torch.empty_like(X), dWr=torch.empty(E, d, device=DEV), dbias=torch.empty(E, device=DEV))
    ws = torch.empty(max(api.moe_balance_loss_workspace_size(T, E, 5), api.moe_router_bwd_workspace_size(T, d, E)),
                     dtype=torch.uint8, device=DEV)

    def go():
        api.moe_balance_loss(z, idx, 0.1, out["counts"], out["dprob"], out["loss"], ws, seg=seg, keep=keep)
        api.moe_balance_loss_bwd(z, out["dprob"], out["loss"], out["dl"], seg=seg, keep=keep, gate=gate, idx=idx, dgate=dg)
        api.moe_router_bwd(out["dl"], X, Wr, ws, dX=out["dX"], dWr=out["dWr"], dbias=out["dbias"])
    go()
    torch.cuda.synchronize()
    want = {n: t.clone() for n, t in out.items()}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    side = torch.cuda.Stream()
    for _ in range(3):
        for t in out.values():
            t.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in out)
        ws.fill_(0xFF)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            go()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], want[n]) for n in out)
