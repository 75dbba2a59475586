"""GPU parity of the microscaled 4-bit rows and of the grouped SwiGLU forward on
them, against the fp64 oracle.

Codes, scale bytes and dequantised values are exact: every step of the
definition is (a power of two, a rounding to 8 magnitudes).  The forward's H is
rounded to 4 bits between the products, so a row whose fp32 H lies next to a
border of that rounding may take the other code; rows with such an element
(nearer than 2e-5 of the block's scale, where fp32 sums differ from exact ones by
some 1e-6 of H) are left out, counted and bounded.  The others must agree with the
exact result of the same codes within the rounding to bf16 (half an ulp, 2^-8) and
the fp32 sums: (I / 64 + 16) 2^-23 sum |h w|."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api
from paper_2508_19078_amd.profiling import QuantizedStack

from gpu_harness import host, log

pytestmark = pytest.mark.gpu
DEV = "cuda"


def quantize(W):
    cs, ss = api.mxfp4_shapes(*W.shape)
    codes = torch.full(cs, 0xAA, dtype=torch.uint8, device=DEV)
    scale = torch.full(ss, 0xAA, dtype=torch.uint8, device=DEV)
    api.moe_quantize_mxfp4(W, codes, scale)
    return codes, scale


def unpacked(codes, cols):
    c = codes.cpu().numpy()
    return np.stack((c & 15, c >> 4), -1).reshape(len(c), -1)[:, :cols]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 24), (5, 32), (17, 40), (8, 128), (33, 136), (7, 688), (1000, 264),
                                       (2, 4096)])
def test_rows_are_exact(rows, cols, dt):
    rng = np.random.default_rng([rows, cols])
    W = torch.from_numpy((rng.standard_normal((rows, cols)) * np.exp(4 * rng.standard_normal((rows, 1))))
                         .astype(np.float32)).to(dt)
    W[rows // 2] = 0
    W.view(-1)[:8] = torch.tensor([0.25, -0.25, 0.75, 5, -7, 6, 3.5, -0.0])     # ties, the cut, -0
    codes, scale = quantize(W.to(DEV))
    want, byte = O.mxfp4_rows(W.double().numpy())
    np.testing.assert_array_equal(unpacked(codes, cols), want)
    np.testing.assert_array_equal(scale.cpu().numpy()[:, :byte.shape[1]], byte)
    assert not unpacked(codes, 10 ** 6)[:, cols:].any() and not scale.cpu().numpy()[:, byte.shape[1]:].any()
    for out_dt in (torch.bfloat16, torch.float32):
        out = torch.full((rows, cols), float("nan"), dtype=out_dt, device=DEV)
        api.moe_dequant_mxfp4(codes, scale, out)
        np.testing.assert_array_equal(out.double().cpu().numpy(), O.mxfp4_values(want, byte))


def test_rows_of_extremes():
    big, tiny = torch.finfo(torch.float32).max, 2.0 ** -149
    W = torch.zeros(8, 64)
    W[0, 0], W[0, 1] = big, -big / 2
    W[1, 5] = tiny                                     # a block of subnormals: byte 0
    W[2, :3] = torch.tensor([2.0 ** -126, 2.0 ** -127, 3 * 2.0 ** -128])
    W[3, 3] = float("inf")
    W[4, 4] = float("nan")
    W[5, 40] = -float("inf")                           # the other block stays a number
    W[5, 0] = 1.0
    W[6] = -0.0
    codes, scale = quantize(W.to(DEV))
    out = torch.empty(8, 64, device=DEV)
    api.moe_dequant_mxfp4(codes, scale, out)
    out, s = out.cpu(), scale.cpu()
    for r in (0, 1, 2, 6, 7):
        c, b = O.mxfp4_rows(W[r:r + 1].double().numpy())
        np.testing.assert_array_equal(unpacked(codes[r:r + 1], 64), c)
        np.testing.assert_array_equal(s[r, :2].numpy(), b[0])
        np.testing.assert_array_equal(out[r:r + 1].double().numpy(), O.mxfp4_values(c, b))
    for r, blk in ((3, 0), (4, 0), (5, 1)):
        assert s[r, blk] == 255 and not unpacked(codes[r:r + 1], 64)[0, 32 * blk:32 * blk + 32].any()
        assert torch.isnan(out[r, 32 * blk:32 * blk + 32]).all()
        assert torch.isfinite(out[r, 32 * (1 - blk):32 * (1 - blk) + 32]).all()
    assert out[5, 0] == 1.0


def test_rows_past_32_bits():
    rows, cols = 1_050_000, 2048                       # 2.15e9 elements
    W = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(64, cols, generator=torch.Generator().manual_seed(0)).to(torch.bfloat16)
    W[-64:] = tail.to(DEV)
    W[1_048_570:1_048_580] = tail[:10].to(DEV)         # across element 2^31
    codes, scale = quantize(W)
    want, byte = O.mxfp4_rows(tail.double().numpy())
    np.testing.assert_array_equal(unpacked(codes[-64:], cols), want)
    np.testing.assert_array_equal(scale[-64:].cpu().numpy(), byte)
    np.testing.assert_array_equal(unpacked(codes[1_048_570:1_048_580], cols), want[:10])
    W.fill_(float("nan"))
    api.moe_dequant_mxfp4(codes, scale, W)
    np.testing.assert_array_equal(W[-64:].double().cpu().numpy(), O.mxfp4_values(want, byte))
    assert not W[:1_048_570].any()


# ---------------------------------------------------------------- forward ----

CASES = {
    # name: (T, d, E, k, I, shared, experts drawn from)
    "one_token": (1, 136, 6, 2, 88, 0, 6),
    "below_every_tile": (3, 8, 4, 2, 8, 1, 4),
    "ragged_tails_empty_slots": (300, 272, 8, 2, 208, 1, 6),
    "row_ends_inside_a_block": (77, 168, 5, 3, 688, 0, 5),
    "shared_only": (77, 128, 0, 1, 96, 2, 0),
    "one_expert": (130, 256, 1, 1, 128, 0, 1),
    "all_on_two_of_many": (257, 264, 100, 2, 136, 0, 2),
    "most_choices": (40, 392, 32, 16, 72, 0, 32),
    "wide_tiles": (900, 512, 4, 2, 384, 0, 4),
}


def draw(T, d, E, k, I, sh, E_drawn, seed=0):
    rng = np.random.default_rng([T, d, E, I, seed])
    S = E + sh
    X = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(torch.bfloat16)
    idx = (np.argsort(rng.random((T, E_drawn)), axis=1)[:, :k] if E else np.zeros((T, k))).astype(np.int32)
    gate = np.full((T, k), 1.0 / k, dtype=np.float32)
    w = {}
    for m, (r, c) in dict(g=(I, d), u=(I, d), d=(d, I)).items():
        w[m] = torch.from_numpy((rng.standard_normal((S * r, c)) / np.sqrt(c)).astype(np.float32)).to(torch.bfloat16)
    if E:
        offsets, tok, _, _ = O.permute_maps(idx, gate, np.arange(E), E)
    else:
        offsets, tok = np.zeros(1, dtype=np.int64), np.zeros(0, dtype=np.int64)
    return X, w, offsets, np.concatenate((tok, np.zeros(T * k - len(tok), dtype=np.int64)))


def tables(w, d, E, k, I, sh):
    q = {m: quantize(w[m].to(DEV)) for m in "gud"}
    rows = dict(g=I, u=I, d=d)
    cut = lambda t, r: [t[i * r:(i + 1) * r] for i in range(E + sh)]  # noqa: E731
    return api.LayerTablesMX4(d, I, E, sh, *(cut(q[m][0], rows[m]) for m in "gud"),
                              *(cut(q[m][1], rows[m]) for m in "gud"))


def run(tab, X, offsets, tok, T, k, sh, d, ws=None):
    out = torch.full((T * (k + sh), d), 7.0, dtype=torch.bfloat16, device=DEV)
    if ws is None:
        ws = torch.full((api.moe_grouped_swiglu_fwd_mx4_workspace_size(tab, T, k),), 0xFF, dtype=torch.uint8, device=DEV)
    api.moe_grouped_swiglu_fwd_mx4(tab, X.to(DEV), torch.from_numpy(tok.astype(np.int32)).to(DEV),
                                   torch.from_numpy(offsets.astype(np.int32)).to(DEV), T, k, out, ws)
    return out


def exact_rows(x, wg, wu, wd):
    """(O, its tolerance, rows whose H has an element next to a border)."""
    H, Y = O.swiglu_mx4_fwd(x, wg, wu, wd)
    q = O.mxfp4_round(H)
    _, byte = O.mxfp4_rows(H)
    s = np.repeat(np.exp2(byte.astype(float) - 127), 32, axis=1)[:, :H.shape[1]]
    a = np.abs(H) / s
    near = np.abs(a[..., None] - np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])).min(-1) < 2e-5
    top = np.maximum.reduceat(a, np.arange(0, H.shape[1], 32), axis=1)
    near_top = (np.abs(top - 4) < 2e-5) | (np.abs(top - 8) < 2e-5)
    tol = 2.0 ** -8 * np.abs(Y) + (H.shape[1] / 64 + 16) * 2.0 ** -23 * (np.abs(q) @ np.abs(wd).T)
    return Y, tol, near.any(1) | near_top.any(1)


def check(got, X, w, offsets, tok, T, d, E, k, I, sh, slots=None):
    x = X.double().numpy()
    left = total = 0
    for s in range(E + sh) if slots is None else slots:
        r0, n = (int(offsets[s]), int(offsets[s + 1] - offsets[s])) if s < E else (T * k + (s - E) * T, T)
        if n == 0:
            continue
        xs = x[tok[r0:r0 + n]] if s < E else x
        wg, wu, wd = (O.mxfp4_round(w[m][s * r:(s + 1) * r].double().numpy()) for m, r in (("g", I), ("u", I), ("d", d)))
        want, tol, near = exact_rows(xs, wg, wu, wd)
        g = got[r0:r0 + n].double().cpu().numpy()
        err = np.abs(g - want) / tol
        assert np.all(err[~near] <= 1), (s, float(err[~near].max()), np.argwhere(err > 1)[:5])
        assert np.linalg.norm(g - want) <= 0.05 * np.linalg.norm(want)       # a moved code moves its row, not far
        left += int(near.sum())
        total += n
    log(f"  {total} rows, {left} next to a border")
    assert left <= max(1, 0.2 * total)
    return total


@pytest.mark.parametrize("name", list(CASES))
def test_forward(name):
    T, d, E, k, I, sh, E_drawn = CASES[name]
    log(f"mx4 forward {name}")
    X, w, offsets, tok = draw(*CASES[name])
    got = run(tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    check(got, X, w, offsets, tok, T, d, E, k, I, sh)
    N = int(offsets[-1])
    assert bool((got[N:T * k] == 7.0).all())           # rows behind the last slot's


@pytest.mark.parametrize("T", [1, 2, 7, 31, 32, 33, 64, 65, 127, 129, 255, 500, 1100])
def test_forward_lengths(T):
    """Both sides of every tile's number of rows, a shared slot of exactly T rows."""
    d, E, k, I, sh = 200, 3, 2, 136, 1
    X, w, offsets, tok = draw(T, d, E, k, I, sh, E)
    got = run(tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    assert check(got, X, w, offsets, tok, T, d, E, k, I, sh) == T * (k + sh)


def test_forward_with_numbers_that_are_none():
    """A NaN or an infinity in a token's activations reaches that token's rows and
    no others; one in a weight block its column's users."""
    T, d, E, k, I, sh = 140, 160, 2, 1, 96, 1
    X, w, offsets, tok = draw(T, d, E, k, I, sh, E)
    tab = tables(w, d, E, k, I, sh)
    want = run(tab, X, offsets, tok, T, k, sh, d)
    bad = X.clone()
    bad[17, 150], bad[99, 3] = float("nan"), float("-inf")
    got = run(tab, bad, offsets, tok, T, k, sh, d)
    hit = torch.zeros(T * (k + sh), dtype=torch.bool)
    hit[:T * k] = torch.from_numpy(np.isin(tok, (17, 99)))
    hit[T * k + 17] = hit[T * k + 99] = True
    assert torch.isnan(got[hit.to(DEV)]).all()
    assert torch.equal(got[~hit.to(DEV)], want[~hit.to(DEV)])
    w["d"][5, 40] = float("nan")                       # W_down of slot 0: one output column
    got = run(tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    n0 = int(offsets[1])
    assert torch.isnan(got[:n0, 5]).all()
    want[:n0, 5] = got[:n0, 5] = 0
    assert torch.equal(got, want)


def test_forward_past_32_bits():
    """O of 2.6e9 elements; the rows at both ends and across element 2^31."""
    T, d, E, k, I = 40_000, 4096, 16, 16, 16
    X, w, offsets, tok = draw(8, d, E, k, I, 0, E)
    X = X.repeat(T // 8, 1)
    tab = tables(w, d, E, k, I, 0)
    offsets = np.arange(E + 1) * T                     # every token on every expert
    tok = np.tile(np.arange(T), E)
    got = run(tab, X, offsets, tok, T, k, 0, d)
    for s in (0, 13, 15):
        wg, wu, wd = (O.mxfp4_round(w[m][s * r:(s + 1) * r].double().numpy()) for m, r in (("g", I), ("u", I), ("d", d)))
        want, tol, near = exact_rows(X[:8].double().numpy(), wg, wu, wd)
        g = got[s * T:(s + 1) * T].view(-1, 8, d)
        assert bool((g == g[0]).all())
        assert np.all((np.abs(g[0].double().cpu().numpy() - want) / tol)[~near] <= 1)


def test_forward_on_another_stream_and_in_two_graphs():
    """Two graphs, captured on a side stream, each with its own layer and workspace,
    replayed several times with eager work between; and one workspace that two eager
    calls share in a row."""
    args = []
    for seed, (T, d, E, k, I, sh) in enumerate([(70, 136, 4, 2, 104, 1), (9, 256, 3, 1, 72, 0)]):
        X, w, offsets, tok = draw(T, d, E, k, I, sh, E, seed)
        tab = tables(w, d, E, k, I, sh)
        args.append([tab, X.to(DEV), torch.from_numpy(tok.astype(np.int32)).to(DEV),
                     torch.from_numpy(offsets.astype(np.int32)).to(DEV), T, k,
                     torch.empty((T * (k + sh), d), dtype=torch.bfloat16, device=DEV),
                     torch.empty(api.moe_grouped_swiglu_fwd_mx4_workspace_size(tab, T, k), dtype=torch.uint8, device=DEV)])
    want = []
    shared = torch.empty(max(a[-1].numel() for a in args), dtype=torch.uint8, device=DEV)
    for a in args:
        api.moe_grouped_swiglu_fwd_mx4(*a[:-1], shared)
        want.append(a[6].clone())
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), []
    for a in args:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            api.moe_grouped_swiglu_fwd_mx4(*a)
        graphs.append(g)
    for _ in range(3):
        for a, g, v in zip(args, graphs, want):
            a[6].fill_(3.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(a[6], v)
            a[6].fill_(5.0)
            with torch.cuda.stream(side):
                side.wait_stream(torch.cuda.default_stream())
                api.moe_grouped_swiglu_fwd_mx4(*a)
            torch.cuda.synchronize()
            assert torch.equal(a[6], v)


# ------------------------------------------------------------ profiling pass --

@pytest.mark.parametrize("dt,d,I,sh", [("bf16", 128, 64, 1), ("bf16", 136, 88, 0), ("f32", 128, 72, 1)])
def test_profiling_pass_with_4_bit_experts(dt, d, I, sh):
    """Teacher-forced: each layer's routing and update against the oracle's on the
    GPU's own normalised input of that layer, so both sides quantise the same values.
    The update differs by roundings of the expert outputs and their sum to bf16 (2^-8
    each, norms) and by the few H codes next to a border: 1e-2; the fp32 stack runs on
    the quantised matrices' values in fp32: 1e-5."""
    T, E, k, n = 61, 8, 2, 2        # (the stack's histograms need E to be a multiple of 4)
    rng = np.random.default_rng([d, I])
    tdt = torch.bfloat16 if dt == "bf16" else torch.float32
    layers = []
    for _ in range(n):
        lay = dict(Wr=rng.standard_normal((E, d)) / np.sqrt(d), wg=rng.standard_normal((E, I, d)) / np.sqrt(d),
                   wu=rng.standard_normal((E, I, d)) / np.sqrt(d), wd=rng.standard_normal((E, d, I)) / np.sqrt(I))
        if sh:
            lay.update(sg=lay["wg"][:sh] * 0.5, su=lay["wu"][1:1 + sh], sd=lay["wd"][2:2 + sh])
        layers.append({m: torch.from_numpy(v.astype(np.float32)).to(tdt).to(DEV) for m, v in lay.items()})
    X0 = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(tdt).to(DEV)
    st = QuantizedStack(layers, T, k, record=True, experts="mxfp4")
    assert st.fused == (dt == "bf16") and not hasattr(st, "Dg") == st.fused
    st.run(X0)
    torch.cuda.synchronize()
    for l, lay in enumerate(layers):
        tr = st.trace[l]
        lay64 = {m: v.double().cpu().numpy() for m, v in lay.items()}
        Xn = tr["Xn"].double().cpu().numpy()
        q, s = O.quantize_int8_rows(lay64["Wr"].astype(np.float32))
        lg = O.profile_logits(Xn, q, s)
        sure = O.topk_gap(lg, k) > 1e-5
        idx = host(tr["idx"])
        assert np.array_equal(np.sort(idx[sure], 1), np.sort(O.topk_select(lg, k)[sure], 1))
        Y = np.zeros((T, d))
        fwd = O.swiglu_mx4_fwd if dt == "bf16" else lambda x, a, b, c: (None, O.swiglu_fwd(x, a, b, c)[3])
        deq = lambda W: O.mxfp4_round(W.reshape(-1, W.shape[-1])).reshape(W.shape)  # noqa: E731
        wg, wu, wd = (deq(lay64[m]) for m in ("wg", "wu", "wd"))
        for e in range(E):
            t, j = np.nonzero(idx == e)
            if len(t):
                Y[t] += host(tr["gate"])[t, j][:, None] * fwd(Xn[t], wg[e], wu[e], wd[e])[1]
        for i in range(sh):
            Y += fwd(Xn, *(deq(lay64[m][i]) for m in ("sg", "su", "sd")))[1]
        err = np.linalg.norm(host(tr["Y"]) - Y) / np.linalg.norm(Y)
        log(f"  4-bit stack {dt} d={d} layer {l}: rel err {err:.2e}")
        assert err < (1e-2 if dt == "bf16" else 1e-5)
    with pytest.raises(ValueError):
        QuantizedStack(layers, T, k, experts="fp4")
