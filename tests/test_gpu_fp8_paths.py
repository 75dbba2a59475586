"""The kernels behind moe_grouped_swiglu_fwd_fp8, each at the sizes where it can go wrong: the
ones for a few tokens, the 128- and 256-row tiles (with their half-height forms) and both
sides of the rules between them.  A case names the path it is there for and asks the
library's own rule (fm::fp8_tile), so that a retuned rule does not leave it on another.

Formulas and tolerances as in test_gpu_fp8."""
import ctypes

import numpy as np
import oracle as O
import pytest
import torch

from paper_2508_19078_amd import api

import test_gpu_fp8 as M

FEW, SMALL, LARGE = 0, 128, 256


def path(T, d, E, k, I, sh):
    f = getattr(api.lib(), "_ZN2fm8fp8_tileEPK13moe_layer_fp8ii")   # fm::fp8_tile(const moe_layer_fp8*, int, int)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    L = api.moe_layer_fp8(d, I, E, sh, *[None] * 6)
    return f(ctypes.addressof(L), T, k)


FEW_CASES = {
    # name: (T, d, E, k, I, shared, experts drawn from)
    "one_token": (1, 4096, 6, 2, 688, 0, 6),                  # I ends inside a block, k split over idle waves too
    "two_tokens_on_one_expert": (2, 4096, 2, 1, 272, 0, 1),
    "ragged_ends_and_empty_slots": (3, 1040, 5, 2, 1040, 1, 3),
    "many_empty_slots": (3, 1040, 70, 2, 1024, 0, 70),        # the slots' ballot goes round twice
    "seven_tokens_shared_alone": (7, 2064, 0, 1, 528, 2, 0),
    "eight_tokens_on_all": (8, 4096, 8, 8, 272, 0, 8),
    "many_slabs_per_wave": (2, 6160, 2, 2, 2320, 0, 2),       # a second round of requests in both
    "one_expert": (8, 1040, 1, 1, 1024, 0, 1),
    "sixteen_tokens": (16, 528, 4, 2, 272, 0, 4),             # more than eight rows in a slot
    "narrowest": (16, 16, 3, 1, 16, 1, 2),
}
# both sides of a limit of the rule
LIMITS = [
    ((8, 1040, 3, 1, 2048, 0, 3), FEW), ((9, 1040, 3, 1, 2048, 0, 3), SMALL),          # tokens
    ((16, 528, 2, 1, 2048, 0, 2), FEW), ((17, 528, 2, 1, 2048, 0, 2), SMALL),
    ((4, 272, 5, 4, 4096, 0, 5), FEW), ((4, 272, 6, 4, 4096, 0, 6), SMALL),            # slots times I / 8
    ((16, 272, 8, 2, 512, 0, 8), FEW), ((16, 272, 8, 2, 528, 0, 8), SMALL),
    ((8, 6912, 2, 1, 128, 1, 2), FEW), ((8, 7168, 2, 1, 128, 1, 2), SMALL),            # rows in LDS
    ((271, 144, 2, 1, 144, 1, 2), SMALL), ((272, 144, 1, 1, 144, 0, 1), LARGE),        # rows per slot
]
SMALL_CASES = {
    "empty_slots_between": (150, 528, 40, 2, 272, 0, 9),
    "three_slabs": (200, 384, 3, 2, 384, 1, 3),               # the ring is as long as the product
    "one_slab": (100, 128, 3, 2, 128, 0, 3),
    "two_slabs": (100, 144, 3, 2, 160, 0, 3),
    "four_slabs_and_a_part": (100, 528, 3, 1, 560, 0, 3),     # a second group of scales
    "columns_end_inside_tiles": (70, 656, 2, 1, 400, 2, 2),
    "tiles_of_two_rows": (260, 272, 2, 1, 272, 0, 2),
    "gate_and_up_of_66_slabs": (20, 8336, 2, 1, 144, 0, 2),   # a second group of weight scales
    "down_of_66_slabs": (20, 144, 2, 1, 8336, 0, 2),
}
LARGE_CASES = {
    "one_slab": (300, 128, 1, 1, 128, 0, 1),
    "two_slabs": (600, 144, 2, 2, 160, 0, 2),
    "five_slabs": (600, 640, 2, 1, 640, 0, 1),
    "nine_slabs_ragged": (530, 1040, 2, 1, 1072, 1, 2),
    "a_row_more_than_the_half_tile": (385, 272, 1, 1, 272, 0, 1),
    "the_half_tile": (384, 272, 1, 1, 272, 0, 1),
    "gate_and_up_of_66_slabs": (290, 8336, 1, 1, 144, 0, 1),
    "more_tiles_than_blocks": (4000, 144, 4, 2, 1168, 0, 4),
}


def test_paths():
    for cases, want in ((FEW_CASES, FEW), (SMALL_CASES, SMALL), (LARGE_CASES, LARGE)):
        for name, case in cases.items():
            assert path(*case[:6]) == want, name
    for case, want in LIMITS:
        assert path(*case[:6]) == want, case


def forward(case):
    T, d, E, k, I, sh, _ = case
    X, w, offsets, tok = M.draw(*case)
    got = M.run(M.tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    M.check(got, X, w, offsets, tok, T, d, E, k, I, sh)
    assert bool((got[int(offsets[-1]):T * k] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(FEW_CASES))
def test_few_tokens(name):
    forward(FEW_CASES[name])


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 8])
def test_few_tokens_drop_nothing_of_gate_and_up(T):
    """Large products that cancel, from different groups of 8, and small ones that 8-bit
    products would drop beside them: what is left decides H.  All codes are exact; the
    output is off by its rounding to bf16 and by what tells H's codes in fp32 from those
    in 64 bits, a step at most."""
    d, I = 128, 16
    assert path(T, d, 2, 1, I, 0) == FEW
    X = torch.zeros(T, d)
    X[:, :16] = 2.0 ** -6
    X[:, 0] = X[:, 8] = 448
    W = torch.ones(2, I, d)
    W[:, :, 8] = -1
    w = dict(g=W.to(M.BF), u=W.to(M.BF), d=torch.ones(2, d, I, dtype=M.BF))
    offsets, tok = np.array([0, 0, T]), np.arange(T)
    got = M.run(M.tables(w, d, 2, 1, I, 0), X.to(M.BF), offsets, tok, T, 1, 0, d).double().cpu().numpy()
    H, want = O.swiglu_fp8_fwd(X.double().numpy(), *(w[m][1].double().numpy() for m in "gud"))
    assert abs(H[0, 0] - 0.21875 ** 2 / (1 + np.exp(-0.21875))) < 1e-12
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * want)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c, _ in LIMITS], ids=["-".join(map(str, c)) for c, _ in LIMITS])
def test_both_sides_of_the_rule(case):
    forward(case)


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(SMALL_CASES))
def test_small_tiles(name):
    forward(SMALL_CASES[name])


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(LARGE_CASES))
def test_large_tiles(name):
    forward(LARGE_CASES[name])


@pytest.mark.gpu
@pytest.mark.parametrize("T,want", [(3, FEW), (100, SMALL), (600, LARGE)])
def test_h_at_the_top_of_fp32(T, want):
    """Finite blocks of H whose largest value lies between 2^126 and the top of fp32: 448 over
    it is a normal number, its plain reciprocal is not."""
    d, E, I = 256, 2, 272
    assert path(T, d, E, 1, I, 0) == want
    X, w, offsets, tok = M.draw(T, d, E, 1, I, 0, E)
    X = X.abs()
    w["g"] = w["g"].abs() * 0.75                              # the gate's sums are some 3 to 20
    a, u = (np.concatenate([X.double().numpy() @ x.double().numpy().T for x in w[m]]) for m in "gu")
    H = np.abs(a * O.sigmoid(a) * u)
    e = np.floor(127.9 - np.log2(H.max()))                    # 7 % are left for what quantisation adds
    tops = np.maximum.reduceat(H * 2.0 ** e, np.arange(0, I, 128), axis=1)
    assert (tops > 2.0 ** 126).mean() > 0.05 and a.min() > 2
    w["u"], w["d"] = w["u"] * 2.0 ** e, w["d"] * 2.0 ** -100
    got = M.run(M.tables(w, d, E, 1, I, 0), X, offsets, tok, T, 1, 0, d)
    M.check(got, X, w, offsets, tok, T, d, E, 1, I, 0)


def dropped(xc, xs, wc, ws):
    """Variance of what the matrix unit drops of each sum of x W^T: of the products of 8
    consecutive k, each the part below 2^(e - 13), of its product's sign, with e the largest
    sum of exponents among them (whole scale blocks only).  A product has 6 bits behind its
    leading one, so that those within 7 binades of the largest lose nothing."""
    ex, ew = (np.maximum(np.frexp(v)[1] - 1, -6) for v in (xc, wc))
    out = np.zeros((len(xc), len(wc)))
    for b in range(xc.shape[1] // 128):
        f = xs[:, b][:, None] * np.repeat(ws[:, b], 128)[None, :len(wc)]
        for g in range(128 * b, 128 * b + 128, 8):
            c = slice(g, g + 8)
            p = np.abs(xc[:, None, c] * wc[None, :, c])
            unit = np.exp2(np.where(p != 0, ex[:, None, c] + ew[None, :, c], -99).max(-1, keepdims=True) - 13.0)
            out += f ** 2 * (np.mod(p, unit) ** 2).sum(-1)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("T,want", [(3, FEW), (100, SMALL), (600, LARGE)])
def test_how_many_codes_of_h_the_matrix_unit_moves(T, want):
    """W_down as the unit matrix, so that O holds what H's codes stand for, counted against the
    formula's.  A code moves where the error of its H over the block's scale crosses a border:
    with probability E|error| / step, at most the standard deviation in steps.  That is
    the sums' (`dropped`; a few tokens drop nothing of them), carried through the formula, and
    that of the block's largest H, which is its scale's.  A quarter and four standard deviations of the
    count on top; with one bit less in the unit more than twice as many move."""
    d, I = 256, 128
    assert path(T, d, 1, 1, I, 0) == want
    X, w, offsets, tok = M.draw(T, d, 1, 1, I, 0, 1)
    w["d"] = torch.eye(d, I).to(M.BF)[None]
    got = M.run(M.tables(w, d, 1, 1, I, 0), X, offsets, tok, T, 1, 0, d).double().cpu().numpy()
    x = X.double().numpy()[tok]
    (xc, xs), wg, wu = O.fp8_rows(x), *(O.fp8_rows(w[m][0].double().numpy(), 128) for m in "gu")
    a, u = ((xc * O.fp8_spread(xs, T, d, 1)) @ (c * O.fp8_spread(s, I, d, 128)).T for c, s in (wg, wu))
    sig = O.sigmoid(a)
    H = a * sig * u
    var = 0.0 if want == FEW else (u * sig * (1 + a * (1 - sig))) ** 2 * dropped(xc, xs, *wg) + (a * sig) ** 2 * dropped(xc, xs, *wu)
    var = var + (H * 16 * 2.0 ** -23) ** 2                     # fp32 sums and the logistic function, amply
    val, s = O.fp8_rows(H)
    q, top = np.abs(H) / s, np.abs(H).argmax(1)[:, None]
    off = np.take_along_axis(var, top, 1) / np.take_along_axis(H, top, 1) ** 2
    step = np.exp2(np.maximum(np.frexp(q)[1] - 1, -6) - 3)
    p = np.minimum(np.sqrt(var / s ** 2 + q ** 2 * off) / step, 1).sum()
    moved = int((np.abs(got[:, :I] - val * s) > 0.25 * step * s).sum())
    M.log(f"  {moved} of {H.size} codes moved, {p:.1f} expected at most")
    assert not got[:, I:].any()
    assert moved <= 1.25 * p + 4 * np.sqrt(p) + 1
