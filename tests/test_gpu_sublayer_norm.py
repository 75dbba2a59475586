"""GPU parity of the sublayer norms, forward and backward, against the fp64 oracle.

Tolerances, element by element.  u = 2^-24 is an fp32 rounding.  A thread sums at
most 16 elements of a row in a chain, then come at most 6 steps within its wave and
16 waves: a row sum is off by at most 40 u of the sum of its terms' magnitudes, a
row's scale by 24 u.  A bf16 output adds half a step, 2^-8 of its value.  A gain's
gradient sums over the rows in chains: the rows of a block, the blocks of a group,
the groups; their number bounds the roundings.  The backward gets the same S and
scales on both sides, the forward's N is compared with the oracle on the GPU's own S."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

from gpu_harness import log

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}

SHAPES = [(1, 8), (3, 24), (8, 4096), (5, 128), (70, 136), (65, 512), (33, 520), (1, 1000), (1000, 1000), (129, 2048),
          (7, 2056), (4, 8192), (2500, 64), (600, 4104)]


def f64(t):
    return None if t is None else t.double().cpu().numpy()


def draw(T, d, dt, seed=0):
    g = torch.Generator().manual_seed(seed + 7 * T + d)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    big = dict(X=n(T, d), Y=0.3 * n(T, d), dS=n(T, d), dN=n(T, d), S=1.5 * n(T, d))
    return {**{m: v.to(dt).to(DEV) for m, v in big.items()}, "gate": n(T).to(DEV),
            "w_post": (1 + 0.2 * n(d)).to(DEV), "w_pre": (1 + 0.2 * n(d)).to(DEV)}


def off(got, want, tol, what):
    err = np.abs(f64(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), (what, np.argwhere(bad)[:3], float((err / np.maximum(tol, 1e-300)).max()))


def forward(v, dt, alpha, post, eps, gate=None, w_post=None, w_pre=None, Y=True, S=True, N=True):
    T, d = v["X"].shape
    new = lambda *s, t=torch.float32: torch.full(s, float("nan"), dtype=t, device=DEV)  # noqa: E731
    out = dict(S=new(T, d, t=dt) if S else None, N=new(T, d, t=dt) if N else None,
               rstd_y=new(T) if post and Y else None, rstd_s=new(T) if N else None)
    api.moe_sublayer_norm(v["X"], v["Y"] if Y else None, out["S"], out["N"], alpha=alpha, gate=gate, w_post=w_post,
                          w_pre=w_pre, post_norm=post, eps=eps, rstd_y=out["rstd_y"], rstd_s=out["rstd_s"])
    return out


def check_forward(out, v, dt, alpha, post, eps, gate, w_post, w_pre, Y=True):
    X, y = f64(v["X"]), f64(v["Y"]) if Y else None
    g, a, b = f64(gate), f64(w_post), f64(w_pre)
    S, _ = O.sublayer_norm(X, y, g, a, b, alpha, post, eps)
    terms = np.abs(alpha * X) + (0 if y is None else np.abs(S - alpha * X))
    off(out["S"], S, HALF[dt] * np.abs(S) + 40 * U * terms, "S")
    kept = f64(out["S"])
    den = np.sqrt((kept ** 2).mean(1, keepdims=True) + eps)
    N = kept / np.where(den > 0, den, 1) * (1 if b is None else b)
    off(out["N"], N, (HALF[dt] + 32 * U) * np.abs(N), "N")
    off(out["rstd_s"], np.where(den > 0, 1 / np.where(den > 0, den, 1), 0)[:, 0], 32 * U / np.maximum(den[:, 0], 1e-30), "rstd_s")
    if post and Y:
        ry = 1 / np.sqrt((y ** 2).mean(1) + eps)
        off(out["rstd_y"], ry, 32 * U * ry, "rstd_y")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward(T, d, dt):
    v = draw(T, d, dt)
    for post, full in ((True, True), (True, False), (False, True), (False, False)):
        w = (v["gate"], v["w_post"], v["w_pre"]) if full else (None, None, None)
        out = forward(v, dt, 1.25, post, 1e-6, *w)
        check_forward(out, v, dt, 1.25, post, 1e-6, *w)
    # the pre-norm alone
    out = forward(v, dt, 1.0, False, 1e-5, w_pre=v["w_pre"], Y=False)
    assert torch.equal(out["S"], v["X"])
    check_forward(out, v, dt, 1.0, False, 1e-5, None, None, v["w_pre"], Y=False)


def backward(v, dt, alpha, post, rs, ry, gate=None, w_post=None, w_pre=None, dS=True, dN=True, Y=True, acc=None):
    T, d = v["S"].shape
    new = lambda *s, t=torch.float32: torch.full(s, float("nan"), dtype=t, device=DEV)  # noqa: E731
    out = dict(dX=new(T, d, t=dt), dY=new(T, d, t=dt) if Y else None, dgate=new(T) if Y else None,
               dw_post=new(d) if Y else None, dw_pre=new(d))
    if acc is not None:
        out["dw_post"], out["dw_pre"] = acc[0].clone(), acc[1].clone()
    ws = torch.full((max(1, api.moe_sublayer_norm_bwd_workspace_size(T, d)),), 0xFF, dtype=torch.uint8, device=DEV)
    api.moe_sublayer_norm_bwd(v["dS"] if dS else None, v["dN"] if dN else None, v["S"], v["Y"] if Y else None, rs,
                              out["dX"], out["dY"], ws, alpha=alpha, rstd_y=ry, gate=gate, w_post=w_post, w_pre=w_pre,
                              post_norm=post, dgate=out["dgate"], dw_post=out["dw_post"], dw_pre=out["dw_pre"],
                              accumulate_dw=acc is not None)
    return out


def scales(v, eps=1e-6):
    r = lambda t: (t.double().square().mean(1) + eps).rsqrt().float()  # noqa: E731
    return r(v["S"]), r(v["Y"])


def check_backward(out, v, dt, alpha, post, rs, ry, gate, w_post, w_pre, dS=True, dN=True, Y=True, acc=None):
    T, d = v["S"].shape
    ds, dn = f64(v["dS"]) if dS else None, f64(v["dN"]) if dN else None
    S, y = f64(v["S"]), f64(v["Y"]) if Y else None
    g, a, b = f64(gate), f64(w_post), f64(w_pre)
    want = O.sublayer_norm_backward(ds, dn, S, y, f64(rs), f64(ry) if post else None, g, a, b, alpha)
    # magnitudes of what an element is summed from
    q = np.abs(dn * (1 if b is None else b)) if dN else np.zeros((T, d))
    x = np.abs(S) * f64(rs)[:, None]
    D = (np.abs(ds) if dS else 0) + f64(rs)[:, None] * (q + x * (x * q).mean(1, keepdims=True))
    off(out["dX"], want["dX"], HALF[dt] * np.abs(want["dX"]) + 60 * U * abs(alpha) * D, "dX")
    rows = T + 16          # roundings of a sum over the rows, at most
    base = (0, 0) if acc is None else (f64(acc[0]), f64(acc[1]))
    off(out["dw_pre"], want["dw_pre"] + base[1], (rows + 8) * U * ((np.abs(dn) if dN else 0 * x) * x).sum(0) + U * np.abs(base[1]), "dw_pre")
    if not Y:
        return
    u = np.abs(y) * (f64(ry)[:, None] if post else 1)
    ga, wa = 1 if g is None else np.abs(g)[:, None], 1 if a is None else np.abs(a)
    dv = ga * D * wa
    mag = (f64(ry)[:, None] * (dv + u * (u * dv).mean(1, keepdims=True))) if post else dv
    off(out["dY"], want["dY"], HALF[dt] * np.abs(want["dY"]) + 120 * U * mag, "dY")
    off(out["dgate"], want["dgate"], 120 * U * (D * u * wa).sum(1), "dgate")
    off(out["dw_post"], want["dw_post"] + base[0], (rows + 80) * U * (ga * D * u).sum(0) + U * np.abs(base[0]), "dw_post")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", SHAPES)
def test_backward(T, d, dt):
    v = draw(T, d, dt, 1)
    rs, ry = scales(v)
    every = (v["gate"], v["w_post"], v["w_pre"])
    for post, w, how in ((True, every, {}), (False, every, {}), (True, (None,) * 3, {}), (False, (None,) * 3, {}),
                         (True, every, dict(dS=False)), (True, every, dict(dN=False)), (False, (None, None, v["w_pre"]), dict(Y=False))):
        out = backward(v, dt, 1.25, post, rs, ry if post else None, *w, **how)
        check_backward(out, v, dt, 1.25, post, rs, ry, *w, **how)
    assert T < 2 or d < 64 or float(f64(out["dw_pre"]).std()) > 0
    acc = (torch.randn(d, device=DEV), torch.randn(d, device=DEV))
    out = backward(v, dt, 1.0, True, rs, ry, *every, acc=acc)
    check_backward(out, v, dt, 1.0, True, rs, ry, *every, acc=acc)


def test_gradients_by_differences():
    """The GPU's own forward, nudged along random directions, in fp32: central
    differences of a linear functional of S and N against the backward.  With step h
    the difference is off by its third derivative (h^2, scale 1: below 1e-4 of the norm here)
    and by 2^-24 of the functional's terms over h."""
    T, d, h = 6, 72, 2e-3
    v = draw(T, d, torch.float32, 2)
    names = ("X", "Y", "gate", "w_post", "w_pre")

    def value(w):
        out = forward(w, torch.float32, 0.8, True, 1e-6, w["gate"], w["w_post"], w["w_pre"])
        return out, float((out["S"].double() * v["dS"].double()).sum() + (out["N"].double() * v["dN"].double()).sum())
    out, _ = value(v)
    v["S"] = out["S"]
    grads = backward(v, torch.float32, 0.8, True, out["rstd_s"], out["rstd_y"], v["gate"], v["w_post"], v["w_pre"])
    of = dict(X="dX", Y="dY", gate="dgate", w_post="dw_post", w_pre="dw_pre")
    for n in names:
        dirn = torch.randn(v[n].shape, generator=torch.Generator().manual_seed(len(n))).to(DEV)
        up, dn = ({**v, n: v[n] + s * h * dirn} for s in (1, -1))
        diff = (value(up)[1] - value(dn)[1]) / (2 * h)
        want = float((grads[of[n]].double() * dirn.double()).sum())
        scale = float((grads[of[n]].double().abs() * dirn.double().abs()).sum())
        assert abs(diff - want) <= 2e-3 * scale, (n, diff, want, scale)


def test_rows_of_zeros_nan_and_infinity():
    T, d = 9, 136
    v = draw(T, d, torch.bfloat16, 3)
    v["X"][2] = 0
    v["Y"][2] = 0
    v["Y"][4] = 0                                      # only the block's output is 0
    v["X"][6, 3] = float("nan")
    v["Y"][7, 100] = float("inf")
    w = (v["gate"], v["w_post"], v["w_pre"])
    out = forward(v, torch.bfloat16, 1.0, True, 0.0, *w)
    assert not out["S"][2].any() and not out["N"][2].any() and out["rstd_s"][2] == 0 and out["rstd_y"][2] == 0
    assert torch.equal(out["S"][4], v["X"][4]) and out["rstd_y"][4] == 0
    assert torch.isnan(out["N"][6]).all() and torch.isnan(out["N"][7]).any()
    fine = [0, 1, 3, 5, 8]
    ref = forward({**v, "X": v["X"][fine], "Y": v["Y"][fine]}, torch.bfloat16, 1.0, True, 0.0, w[0][fine].clone(), *w[1:])
    for n in ("S", "N"):
        assert torch.equal(out[n][fine], ref[n])
    # a zero row with eps 0 has no gradient through its norm
    v["S"][2] = 0
    rs, ry = scales(v, 0.0)
    rs[2] = ry[2] = 0
    b = backward({**v, "Y": torch.zeros_like(v["Y"])}, torch.bfloat16, 1.0, True, rs, torch.zeros_like(ry), *w)
    assert torch.equal(b["dX"][2], v["dS"][2]) and not b["dY"].any()


def test_outputs_over_their_inputs():
    """S over X, N over Y; dX over dS, dY over dN: the same bits as apart."""
    for T, d in ((37, 264), (9, 4096)):
        v = draw(T, d, torch.bfloat16, 4)
        w = (v["gate"], v["w_post"], v["w_pre"])
        want = forward(v, torch.bfloat16, 1.5, True, 1e-6, *w)
        X, Y = v["X"].clone(), v["Y"].clone()
        api.moe_sublayer_norm(X, Y, X, Y, alpha=1.5, gate=w[0], w_post=w[1], w_pre=w[2])
        assert torch.equal(X, want["S"]) and torch.equal(Y, want["N"])
        rs, ry = scales(v)
        want = backward(v, torch.bfloat16, 1.5, True, rs, ry, *w)
        dS, dN = v["dS"].clone(), v["dN"].clone()
        ws = torch.empty(api.moe_sublayer_norm_bwd_workspace_size(T, d), dtype=torch.uint8, device=DEV)
        api.moe_sublayer_norm_bwd(dS, dN, v["S"], v["Y"], rs, dS, dN, ws, alpha=1.5, rstd_y=ry, gate=w[0], w_post=w[1],
                                  w_pre=w[2])
        assert torch.equal(dS, want["dX"]) and torch.equal(dN, want["dY"])


def test_partial_outputs_and_no_rows():
    T, d = 20, 256
    v = draw(T, d, torch.bfloat16, 5)
    w = (v["gate"], v["w_post"], v["w_pre"])
    both = forward(v, torch.bfloat16, 1.0, True, 1e-6, *w)
    assert torch.equal(forward(v, torch.bfloat16, 1.0, True, 1e-6, *w, S=False)["N"], both["N"])
    assert torch.equal(forward(v, torch.bfloat16, 1.0, True, 1e-6, *w, N=False)["S"], both["S"])
    rs, ry = scales(v)
    every = backward(v, torch.bfloat16, 1.0, True, rs, ry, *w)
    ws = torch.empty(api.moe_sublayer_norm_bwd_workspace_size(T, d), dtype=torch.uint8, device=DEV)
    for only in ("dX", "dY", "dgate", "dw_post", "dw_pre"):
        out = torch.full_like(every[only], float("nan"))
        kw = {n: (out if n == only else None) for n in ("dgate", "dw_post", "dw_pre")}
        api.moe_sublayer_norm_bwd(v["dS"], v["dN"], v["S"], v["Y"], rs, out if only == "dX" else None,
                                  out if only == "dY" else None, ws, rstd_y=ry, gate=w[0], w_post=w[1], w_pre=w[2], **kw)
        assert torch.equal(out, every[only]), only
    e = torch.empty(0, d, dtype=torch.bfloat16, device=DEV)
    dw = torch.full((d,), 3.0, device=DEV)
    api.moe_sublayer_norm(e, e, e, None)
    api.moe_sublayer_norm_bwd(e, None, None, e, None, e, None, ws, rstd_y=torch.empty(0, device=DEV), dw_post=dw,
                              accumulate_dw=True)
    assert bool((dw == 3).all())
    api.moe_sublayer_norm_bwd(e, None, None, e, None, e, None, ws, rstd_y=torch.empty(0, device=DEV), dw_post=dw)
    assert not dw.any()


def test_rows_past_32_bits_and_long_sums():
    """T d = 2^31 + 2^20 elements; gains' gradients over all rows of a constant."""
    d, T = 8192, (1 << 18) + 128
    X = torch.ones(T, d, dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(4, d, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).to(DEV)
    X[-4:] = tail
    N = torch.empty_like(X)
    api.moe_sublayer_norm(X, None, None, N)
    den = (tail.double().square().mean(1, keepdim=True) + 1e-6).sqrt()
    want = (tail.double() / den).cpu().numpy()
    off(N[-4:], want, (2.0 ** -8 + 32 * U) * np.abs(want), "N")
    assert bool((N[:-4] == 1).all())
    dw = torch.empty(d, device=DEV)
    ws = torch.empty(api.moe_sublayer_norm_bwd_workspace_size(T, d), dtype=torch.uint8, device=DEV)
    one = torch.ones(T, device=DEV)
    api.moe_sublayer_norm_bwd(None, X, X, None, one, None, None, ws, dw_pre=dw)
    want = (T - 4) + tail.double().square().sum(0).cpu().numpy()
    off(dw, want, 1024 * U * want, "dw_pre")            # ones add exactly below 2^24


def test_two_graphs_one_workspace():
    """Two captured backwards that share a workspace, replayed in turn on one stream."""
    cases = []
    for T, d in ((50, 264), (700, 512)):
        v = draw(T, d, torch.bfloat16, T)
        rs, ry = scales(v)
        cases.append((v, rs, ry))
    ws = torch.empty(max(api.moe_sublayer_norm_bwd_workspace_size(*c[0]["S"].shape) for c in cases), dtype=torch.uint8, device=DEV)
    graphs = []
    for v, rs, ry in cases:
        T, d = v["S"].shape
        out = dict(dX=torch.empty_like(v["S"]), dY=torch.empty_like(v["S"]), dgate=torch.empty(T, device=DEV),
                   dw_post=torch.empty(d, device=DEV), dw_pre=torch.empty(d, device=DEV))

        def go(v=v, rs=rs, ry=ry, out=out):
            api.moe_sublayer_norm_bwd(v["dS"], v["dN"], v["S"], v["Y"], rs, out["dX"], out["dY"], ws, rstd_y=ry,
                                      gate=v["gate"], w_post=v["w_post"], w_pre=v["w_pre"], dgate=out["dgate"],
                                      dw_post=out["dw_post"], dw_pre=out["dw_pre"])
        go()
        torch.cuda.synchronize()
        want = {n: t.clone() for n, t in out.items()}
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            go()
        graphs.append((g, go, out, want))
    for _ in range(3):
        for g, go, out, want in graphs:
            for replay in (g.replay, go):
                for t in out.values():
                    t.fill_(float("nan"))
                replay()
                torch.cuda.synchronize()
                assert all(torch.equal(out[n], want[n]) for n in out)
