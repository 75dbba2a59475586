"""GPU parity of the 8-bit float rows and of the grouped SwiGLU forward on them, against
the fp64 oracle.

Codes of bf16 matrices are exact (their quotients lie on a tie exactly or at least 2^-14
from one); of fp32 ones a quotient within 2^-22 of a tie may take the other code.  Scales
and dequantised values are exact.

The forward's products run on the matrix unit, which aligns the products of 8
consecutive k to the largest sum of their operands' exponents, e, and drops what of each
lies below 2^(e - 13), towards zero.  The oracle's products are formed the same way here
(`unit_product`), so that what is left are fp32 sums.  H is rounded to 8 bits between the
products, so an element next to a border of that rounding may take the other code, a step
away.  The tolerance of an output is
  2^-8 |O|                      its rounding to bf16 (half a step)
  + (n + 16) 2^-23 sum |h w|    fp32 sums over n blocks, the scales' product, H's scale
  + sum over elements next to a border of step * scale * |w|
with H's own error bounded the same way: the sums of its two products, and (|a| + 8) 2^-23
for the logistic function and the products behind it.

Against the formula itself, without the dropped bits: they move an H by r = 2^-13 of it or
less (norms), a code by a step (at most 2^-3 of it) where that crosses a border, in a part of at
most 2 * 16 r of the elements, and so O by 2^-3 sqrt(2^-8) = 2^-7 at most; with the rounding to
bf16 1e-2 of its norm."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api
from paper_2508_19078_amd.profiling import QuantizedStack

from gpu_harness import host, log

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def quantize(W, block_rows=128):
    codes = torch.full(W.shape, 0xAA, dtype=torch.uint8, device=DEV)
    scale = torch.full(api.fp8_scale_shape(*W.shape, block_rows), -7.0, device=DEV)
    api.moe_quantize_fp8(W, codes, scale, block_rows)
    return codes, scale


def values(codes):
    return codes.cpu().view(torch.float8_e4m3fn).double().numpy()


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows,cols", [(1, 8), (3, 24), (17, 40), (8, 128), (33, 136), (7, 688), (127, 264), (129, 120), (300, 1032),
                                       (2, 4096)])
def test_rows(rows, cols, block_rows, dt):
    rng = np.random.default_rng([rows, cols])
    W = torch.from_numpy((rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1)))).astype(np.float32)).to(dt)
    W[rows // 2] = 0
    W.view(-1)[:8] = torch.tensor([0.25, -0.25, 0.75, 5, -7, 6, 3.5, -0.0])
    codes, scale = quantize(W.to(DEV), block_rows)
    W64 = W.double().numpy()
    want, ws = O.fp8_rows(W64, block_rows)
    np.testing.assert_array_equal(host(scale), ws.astype(np.float32))
    got = values(codes)
    if dt is F32:
        s = O.fp8_spread(ws, rows, cols, block_rows)
        q = np.abs(np.divide(W64, s, out=np.zeros_like(W64), where=s > 0))
        step = np.exp2(np.maximum(np.frexp(q)[1] - 1, -6) - 3)
        tie = np.abs(q / step - np.floor(q / step) - 0.5) <= q / step * 2.0 ** -22
        assert tie.mean() < 1e-3 and np.all(np.abs(got - want)[tie] <= step[tie])
        got[tie] = want[tie]
    np.testing.assert_array_equal(got, want)
    val = values(codes) * O.fp8_spread(host(scale).astype(np.float64), rows, cols, block_rows)
    for out_dt in (BF, F32):
        out = torch.full((rows, cols), float("nan"), dtype=out_dt, device=DEV)
        api.moe_dequant_fp8(codes, scale, out, block_rows)
        assert torch.equal(out.cpu(), torch.from_numpy(val.astype(np.float32)).to(out_dt))
    # torch's own type of these bits
    c2 = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=DEV)
    api.moe_quantize_fp8(W.to(DEV), c2, torch.empty_like(scale), block_rows)
    assert torch.equal(c2.view(torch.uint8), codes)


@pytest.mark.parametrize("scale", [1.0, 7.0 / 448, 2.0 ** -40, 2.0 ** 100, 2.0 ** -110])
def test_ties_of_bf16(scale):
    """Every bf16 mantissa pair that can tie: rows whose largest value has each mantissa,
    holding the values of all mantissas."""
    top = torch.arange(128, 256).float() * scale
    rows = torch.empty(128, 128)
    rows[:, 0] = top
    rows[:, 1:] = top[:, None] * 0 + torch.arange(129, 256).float()[None, :] * scale * 2.0 ** -(torch.arange(127) % 9 + 1).float()
    W = rows.to(BF)
    assert torch.equal(W.float(), rows)
    codes, s = quantize(W.to(DEV), 1)
    want, ws = O.fp8_rows(W.double().numpy(), 1)
    np.testing.assert_array_equal(values(codes), want)
    np.testing.assert_array_equal(host(s), ws.astype(np.float32))


@pytest.mark.parametrize("block_rows", [1, 128])
def test_rows_of_extremes(block_rows):
    big, tiny = torch.finfo(F32).max, 2.0 ** -149
    rows = [{0: big, 1: -big / 2, 2: 1.0}, {5: tiny}, {0: 2.0 ** -118, 1: 2.0 ** -120, 2: -3 * 2.0 ** -126}, {3: float("inf"), 4: 1.0},
            {4: float("nan")}, {140: float("-inf"), 0: 1.0}, {}, {0: 448 * 2.0 ** -126, 1: 2.0 ** -126, 130: 2.0 ** -140}]
    for r, cells in enumerate(rows):                       # each in a block of its own
        W = torch.zeros(3, 256)
        for c, v in cells.items():
            W[1, c] = v
        W[0, 0] = -0.0
        codes, scale = quantize(W.to(DEV), block_rows)
        want, ws = O.fp8_rows(W.double().numpy(), block_rows)
        np.testing.assert_array_equal(host(scale), ws.astype(np.float32), err_msg=str(r))
        np.testing.assert_array_equal(values(codes), want)
        out = torch.empty(3, 256, device=DEV)
        api.moe_dequant_fp8(codes, scale, out, block_rows)
        # a smallest subnormal of the product may round either way only where the oracle's does
        val = want * O.fp8_spread(ws, 3, 256, block_rows)
        np.testing.assert_array_equal(host(out), val.astype(np.float32))


def test_every_code_of_dequantisation():
    codes = torch.arange(256, dtype=torch.uint8, device=DEV).view(2, 128)
    want = codes.cpu().view(torch.float8_e4m3fn).double()
    for s in (1.0, 0.3, 2.0 ** 110, 2.0 ** -126, 0.0, float("nan")):
        for dt in (F32, BF):
            out = torch.empty(2, 128, dtype=dt, device=DEV)
            api.moe_dequant_fp8(codes, torch.full((1, 1), s, device=DEV), out)
            np.testing.assert_array_equal(out.float().cpu().numpy(), (want * float(np.float32(s))).float().to(dt).float().numpy())


def test_rows_past_32_bits():
    rows, cols = 1_050_112, 2048                           # 2.15e9 elements
    W = torch.zeros(rows, cols, dtype=BF, device=DEV)
    tail = torch.randn(128, cols, generator=torch.Generator().manual_seed(0)).to(BF)
    W[-128:] = tail.to(DEV)
    W[1_048_570:1_048_580] = tail[:10].to(DEV)             # across element 2^31
    for block_rows in (1, 128):
        codes, scale = quantize(W, block_rows)
        want, ws = O.fp8_rows(tail.double().numpy(), block_rows)
        np.testing.assert_array_equal(values(codes[-128:]), want)
        np.testing.assert_array_equal(host(scale[-len(ws):]), ws.astype(np.float32))
        out = torch.empty(rows, cols, dtype=BF, device=DEV)
        api.moe_dequant_fp8(codes, scale, out, block_rows)
        ref = torch.from_numpy((want * O.fp8_spread(ws, 128, cols, block_rows)).astype(np.float32)).to(BF)
        assert torch.equal(out[-128:].cpu(), ref)
        assert not out[:1_048_448].any()
        if block_rows == 1:
            assert torch.equal(out[1_048_570:1_048_580].cpu(), ref[:10])


# ---------------------------------------------------------------- forward ----

CASES = {
    # name: (T, d, E, k, I, shared, experts drawn from)
    "one_token": (1, 144, 6, 2, 80, 0, 6),
    "below_every_tile": (3, 16, 4, 2, 16, 1, 4),
    "ragged_tails_empty_slots": (300, 272, 8, 2, 208, 1, 6),
    "row_ends_inside_a_block": (77, 176, 5, 3, 688, 0, 5),
    "shared_only": (77, 128, 0, 1, 96, 2, 0),
    "one_expert": (130, 256, 1, 1, 128, 0, 1),
    "all_on_two_of_many": (257, 272, 100, 2, 144, 0, 2),
    "most_choices": (40, 400, 32, 16, 80, 0, 32),
    "large_tiles": (900, 640, 4, 2, 400, 0, 4),
    "large_tiles_ragged": (777, 1168, 3, 2, 1168, 1, 3),
    "many_slabs": (200, 2064, 2, 1, 1040, 0, 2),
}


def draw(T, d, E, k, I, sh, E_drawn, seed=0):
    rng = np.random.default_rng([T, d, E, I, seed])
    S = E + sh
    X = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(BF)
    idx = (np.argsort(rng.random((T, E_drawn)), axis=1)[:, :k] if E else np.zeros((T, k))).astype(np.int32)
    gate = np.full((T, k), 1.0 / k, dtype=np.float32)
    w = {}
    for m, (r, c) in dict(g=(I, d), u=(I, d), d=(d, I)).items():
        # scale blocks of different magnitudes, so that a wrong block shows
        v = rng.standard_normal((S, r, c)) / np.sqrt(c)
        v *= np.exp(0.5 * rng.standard_normal((S, -(-r // 128), -(-c // 128)))).repeat(128, 1).repeat(128, 2)[:, :r, :c]
        w[m] = torch.from_numpy(v.astype(np.float32)).to(BF)
    if E:
        offsets, tok, _, _ = O.permute_maps(idx, gate, np.arange(E), E)
    else:
        offsets, tok = np.zeros(1, dtype=np.int64), np.zeros(0, dtype=np.int64)
    return X, w, offsets, np.concatenate((tok, np.zeros(T * k - len(tok), dtype=np.int64)))


def tables(w, d, E, k, I, sh):
    q = {m: [quantize(x.contiguous().to(DEV)) for x in w[m]] for m in "gud"}
    return api.LayerTablesFP8(d, I, E, sh, *([c for c, _ in q[m]] for m in "gud"), *([s for _, s in q[m]] for m in "gud"))


def run(tab, X, offsets, tok, T, k, sh, d, ws=None):
    out = torch.full((T * (k + sh), d), 7.0, dtype=BF, device=DEV)
    if ws is None:
        ws = torch.full((api.moe_grouped_swiglu_fwd_fp8_workspace_size(tab, T, k),), 0xFF, dtype=torch.uint8, device=DEV)
    api.moe_grouped_swiglu_fwd_fp8(tab, X.to(DEV), torch.from_numpy(tok.astype(np.int32)).to(DEV),
                                   torch.from_numpy(offsets.astype(np.int32)).to(DEV), T, k, out, ws)
    return out


def unit_product(x, wc, ws):
    """(x W^T in fp64 as the matrix unit forms it, sum |x w|) of x quantised by rows and of
    W's codes and scales."""
    xc, xs = O.fp8_rows(x)
    n, d = x.shape
    pad = -d % 128
    xc, w = np.pad(xc, ((0, 0), (0, pad))), np.pad(wc, ((0, 0), (0, pad)))
    ex, ew = (np.maximum(np.frexp(v)[1] - 1, -6) for v in (xc, w))
    ws = np.repeat(ws, 128, axis=0)[:len(wc)]
    out, mag = np.zeros((n, len(wc))), np.zeros((n, len(wc)))
    for b in range(xc.shape[1] // 128):
        c = slice(128 * b, 128 * b + 128)
        f = xs[:, b][:, None] * ws[:, b][None, :]
        for r in range(0, n, 16):
            q = slice(r, min(n, r + 16))
            p = xc[q, None, c] * w[None, :, c]
            e = np.where(p != 0, ex[q, None, c] + ew[None, :, c], -99).reshape(*p.shape[:2], 16, 8)
            unit = np.exp2(e.max(-1, keepdims=True) - 13.0)
            out[q] += f[q] * (np.trunc(p.reshape(e.shape) / unit) * unit).sum((-1, -2))
            mag[q] += f[q] * np.abs(p).sum(-1)
    return out, mag


def exact_rows(x, wg, wu, wd):
    """(O, its tolerance, part of H next to a border) for (codes, scales) of the weights."""
    u = 2.0 ** -23
    (a, ma), (b, mb) = unit_product(x, *wg), unit_product(x, *wu)
    n = -(-x.shape[1] // 128) + 16
    silu = a * O.sigmoid(a)
    H = silu * b
    dH = 1.1 * np.abs(b) * n * u * ma + np.abs(silu) * n * u * mb + (np.abs(a) + 8) * u * np.abs(H)
    val, scale = O.fp8_rows(H)
    Y, _ = unit_product(H, *wd)
    s = O.fp8_spread(scale, *H.shape, 1)
    safe = np.where(s > 0, s, 1.0)
    q = np.abs(H) / safe
    # H's block scale is off by its largest element's relative error
    cols = np.arange(0, H.shape[1], 128)
    off = np.maximum.reduceat(dH, cols, axis=1) / np.maximum(np.maximum.reduceat(np.abs(H), cols, axis=1), 1e-300)
    off = np.repeat(off, 128, axis=1)[:, :H.shape[1]] + 4 * u
    step = np.exp2(np.maximum(np.frexp(q)[1] - 1, -6) - 3)
    t = q / step
    reach = (dH / safe + q * off) / step
    near = np.abs(t - np.floor(t) - 0.5) <= reach
    h = np.abs(val) * s
    aw = np.abs(wd[0] * O.fp8_spread(wd[1], *wd[0].shape, 128)).T
    # a code that moves also moves what is dropped of its group of 8: within the step's own room
    tol = 2.0 ** -8 * np.abs(Y) + (H.shape[1] / 128 + 16) * u * (h @ aw) + (h * off) @ aw + 2 * (near * (1 + reach) * step * s) @ aw
    return Y, tol + 2.0 ** -133, float(near.mean())


def check(got, X, w, offsets, tok, T, d, E, k, I, sh, slots=None):
    x = X.double().numpy()
    total, border = 0, 0.0
    for s in range(E + sh) if slots is None else slots:
        r0, n = (int(offsets[s]), int(offsets[s + 1] - offsets[s])) if s < E else (T * k + (s - E) * T, T)
        if n == 0:
            continue
        xs = x[tok[r0:r0 + n]] if s < E else x
        g = got[r0:r0 + n].double().cpu().numpy()
        wq = [O.fp8_rows(w[m][s].double().numpy(), 128) for m in "gud"]
        # all rows against the formula, by norms; some, both ends among them, one by one
        _, Y = O.swiglu_fp8_fwd(xs, *(c * O.fp8_spread(sc, *c.shape, 128) for c, sc in wq))
        assert np.linalg.norm(g - Y) <= 1e-2 * np.linalg.norm(Y), np.linalg.norm(g - Y) / np.linalg.norm(Y)
        some = np.unique(np.linspace(0, n - 1, min(n, max(8, int(4e7 / (d * I))))).astype(int))
        want, tol, near = exact_rows(xs[some], *wq)
        err = np.abs(g[some] - want) / tol
        assert np.all(err <= 1), (s, float(err.max()), np.argwhere(err > 1)[:5])
        total += n
        border += near * n
    log(f"  {total} rows, {border / max(total, 1):.1e} of H next to a border")
    return total


@pytest.mark.parametrize("name", list(CASES))
def test_forward(name):
    T, d, E, k, I, sh, E_drawn = CASES[name]
    log(f"fp8 forward {name}")
    X, w, offsets, tok = draw(*CASES[name])
    got = run(tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    check(got, X, w, offsets, tok, T, d, E, k, I, sh)
    N = int(offsets[-1])
    assert bool((got[N:T * k] == 7.0).all())           # rows behind the last slot's


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 31, 32, 33, 64, 65, 127, 129, 255, 257, 500, 1100])
def test_forward_lengths(T):
    """Both sides of every tile's number of rows, a shared slot of exactly T rows."""
    d, E, k, I, sh = 208, 3, 2, 144, 1
    X, w, offsets, tok = draw(T, d, E, k, I, sh, E)
    got = run(tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    assert check(got, X, w, offsets, tok, T, d, E, k, I, sh) == T * (k + sh)


@pytest.mark.parametrize("T", [3, 140, 900])
def test_forward_with_numbers_that_are_none(T):
    """A NaN or an infinity in a token's activations reaches that token's rows and
    no others; one in a weight block its columns' users."""
    d, E, k, I, sh = 160, 2, 1, 144, 1
    X, w, offsets, tok = draw(T, d, E, k, I, sh, E)
    tab = tables(w, d, E, k, I, sh)
    want = run(tab, X, offsets, tok, T, k, sh, d)
    bad = X.clone()
    b0, b1 = 1, T - 1
    bad[b0, 150], bad[b1, 3] = float("nan"), float("-inf")
    got = run(tab, bad, offsets, tok, T, k, sh, d)
    hit = torch.zeros(T * (k + sh), dtype=torch.bool)
    hit[:T * k] = torch.from_numpy(np.isin(tok, (b0, b1)))
    hit[T * k + b0] = hit[T * k + b1] = True
    assert torch.isnan(got[hit.to(DEV)]).all()
    assert torch.equal(got[~hit.to(DEV)], want[~hit.to(DEV)])
    w["d"][0, 130, 140] = float("nan")                 # W_down of slot 0: the second block of columns
    got = run(tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    n0 = int(offsets[1])
    assert torch.isnan(got[:n0, 128:]).all()
    want[:n0, 128:] = got[:n0, 128:] = 0
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
        want, tol, _ = exact_rows(X[:8].double().numpy(), *(O.fp8_rows(w[m][s].double().numpy(), 128) for m in "gud"))
        g = got[s * T:(s + 1) * T].view(-1, 8, d)
        assert bool((g == g[0]).all())
        assert np.all(np.abs(g[0].double().cpu().numpy() - want) <= tol)


def test_forward_on_another_stream_and_in_two_graphs():
    """Two graphs, captured on a side stream, each with its own layer and workspace,
    replayed several times with eager work between; and one workspace that two eager
    calls share in a row."""
    args = []
    for seed, (T, d, E, k, I, sh) in enumerate([(70, 144, 4, 2, 112, 1), (9, 256, 3, 1, 80, 0), (2, 256, 3, 1, 80, 1)]):
        X, w, offsets, tok = draw(T, d, E, k, I, sh, E, seed)
        tab = tables(w, d, E, k, I, sh)
        args.append([tab, X.to(DEV), torch.from_numpy(tok.astype(np.int32)).to(DEV),
                     torch.from_numpy(offsets.astype(np.int32)).to(DEV), T, k,
                     torch.empty((T * (k + sh), d), dtype=BF, device=DEV),
                     torch.empty(api.moe_grouped_swiglu_fwd_fp8_workspace_size(tab, T, k), dtype=torch.uint8, device=DEV)])
    want = []
    shared = torch.empty(max(a[-1].numel() for a in args), dtype=torch.uint8, device=DEV)
    for a in args:
        api.moe_grouped_swiglu_fwd_fp8(*a[:-1], shared)
        want.append(a[6].clone())
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), []
    for a in args:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            api.moe_grouped_swiglu_fwd_fp8(*a)
        graphs.append(g)
    for _ in range(3):
        for a, g, v in zip(args, graphs, want):
            a[6].fill_(3.0)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(a[6], v)
            a[6].fill_(5.0)
            side.wait_stream(torch.cuda.default_stream())
            with torch.cuda.stream(side):
                api.moe_grouped_swiglu_fwd_fp8(*a)
            torch.cuda.synchronize()
            assert torch.equal(a[6], v)


# ------------------------------------------------------------ profiling pass --

@pytest.mark.parametrize("dt,d,I,sh", [("bf16", 128, 64, 1), ("bf16", 136, 88, 0), ("f32", 128, 72, 1)])
def test_profiling_pass_with_8_bit_float_experts(dt, d, I, sh):
    """Teacher-forced: each layer's routing and update against the oracle's on the
    GPU's own normalised input of that layer, so both sides quantise the same values.
    The update differs by roundings of the expert outputs and their sum to bf16 (2^-8
    each, norms) and the few H codes next to a border: 1e-2 (d or I off 16: the
    dequantised matrices in the bf16 forward); fp32 on the quantised values: 1e-5."""
    T, E, k, n = 61, 8, 2, 2
    rng = np.random.default_rng([d, I])
    tdt = BF if dt == "bf16" else F32
    layers = []
    for _ in range(n):
        lay = dict(Wr=rng.standard_normal((E, d)) / np.sqrt(d), wg=rng.standard_normal((E, I, d)) / np.sqrt(d),
                   wu=rng.standard_normal((E, I, d)) / np.sqrt(d), wd=rng.standard_normal((E, d, I)) / np.sqrt(I))
        if sh:
            lay.update(sg=lay["wg"][:sh] * 0.5, su=lay["wu"][1:1 + sh], sd=lay["wd"][2:2 + sh])
        layers.append({m: torch.from_numpy(v.astype(np.float32)).to(tdt).to(DEV) for m, v in lay.items()})
    X0 = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(tdt).to(DEV)
    st = QuantizedStack(layers, T, k, record=True, experts="fp8")
    fused = dt == "bf16" and d % 16 == 0 and I % 16 == 0
    assert st.fused == fused and hasattr(st, "Dg") != fused
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
        fwd = O.swiglu_fp8_fwd if fused else lambda x, a, b, c: (None, O.swiglu_fwd(x, a, b, c)[3])
        store = (lambda v: torch.from_numpy(v).to(BF).double().numpy()) if dt == "bf16" and not fused else (lambda v: v)
        deq = lambda W: store(np.stack([O.fp8_round(x, 128) for x in W]))  # noqa: E731
        wg, wu, wd = (deq(lay64[m]) for m in ("wg", "wu", "wd"))
        for e in range(E):
            t, j = np.nonzero(idx == e)
            if len(t):
                Y[t] += host(tr["gate"])[t, j][:, None] * fwd(Xn[t], wg[e], wu[e], wd[e])[1]
        if sh:
            sg, su, sd = (deq(lay64[m]) for m in ("sg", "su", "sd"))
            for i in range(sh):
                Y += fwd(Xn, sg[i], su[i], sd[i])[1]
        err = np.linalg.norm(host(tr["Y"]) - Y) / np.linalg.norm(Y)
        log(f"  8-bit stack {dt} d={d} layer {l}: rel err {err:.2e}")
        assert err < (1e-2 if dt == "bf16" else 1e-5)
