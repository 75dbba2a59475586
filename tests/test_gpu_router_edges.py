"""The router's dense backward where it can go wrong.  u = 2^-24; the products' tolerances are test_gpu_balance's."""
import numpy as np
import pytest
import torch

from paper_2508_19078_amd import api

import test_gpu_balance as B

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("T,d,E", [(70, 40, 4), (64, 2048, 64), (200, 136, 130)])
def test_dx_takes_all_bits_of_dlogits(T, d, E):
    """Two experts with one row of Wr and gradients that nearly cancel: what is left
    stands in the low bits.  At most 6 products of parts are not 0, each exact: 6 sums."""
    g = torch.Generator().manual_seed(T)
    dl = torch.zeros(T, E)
    dl[:, 0] = torch.randn(T, generator=g)
    dl[:, E - 1] = -dl[:, 0] * (1 + 2.0 ** -15 * torch.rand(T, generator=g))
    Wr = torch.randn(E, d, generator=g).bfloat16()
    Wr[E - 1] = Wr[0]
    out = B.router(dl.to(DEV), torch.zeros(T, d, dtype=torch.bfloat16, device=DEV), Wr.to(DEV), dw=False, db=False)["dX"]
    a, w = B.f64(dl), B.f64(Wr)
    want = a @ w
    tol = 12 * U * (np.abs(a) @ np.abs(w)) + 2.0 ** -8 * np.abs(want)
    assert np.all(np.abs(B.f64(out) - want) <= tol)


def products(a, x):
    """(sum_t a[t,i] x[t,j], the same of magnitudes), term by term in fp64."""
    with np.errstate(invalid="ignore", over="ignore"):
        p = a[:, :, None] * x[:, None, :]
        return p.sum(0), np.abs(p).sum(0)


def same(got, want, tol, what):
    g = B.f64(got)
    np.testing.assert_array_equal(np.isnan(g), np.isnan(want), err_msg=what)
    inf = np.isinf(want)
    np.testing.assert_array_equal(np.isinf(g), inf, err_msg=what)
    np.testing.assert_array_equal(g[inf], want[inf], err_msg=what)
    ok = np.isfinite(want)
    assert np.all(np.abs(g[ok] - want[ok]) <= tol[ok]), what


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,E", [(65, 24, 5), (130, 136, 33), (150, 72, 130), (129, 264, 64)])
def test_infinities_and_nan(T, d, E, dt):
    """They reach what the formula says and nothing else: an infinity stays one (the fp32
    dlogits are taken apart for bf16 products, and a part may be 0), and rows behind the
    last token are no terms of the sum."""
    g = torch.Generator().manual_seed(T + d)
    dl, X, Wr = (torch.randn(s, generator=g) for s in ((T, E), (T, d), (E, d)))
    dl[::3] = dl[::3].bfloat16().float()               # one part holds them
    dl[dl == 0] = 0.5
    X[10, 3], X[T - 1, 5], X[4, 9] = INF, -INF, NAN
    X[20, 7], X[21, 7] = INF, -INF
    Wr[0] *= 2.0 ** -10
    Wr[2, 7], Wr[0, 8], Wr[3, 11] = INF, -INF, NAN
    dl[6, 1], dl[7, 2], dl[8, 3] = INF, -INF, NAN
    dl[9, 0], X[9] = torch.finfo(torch.float32).max, X[9] * 2.0 ** -20   # rounds to an infinity in 8 bits
    X, Wr = X.to(dt), Wr.to(dt)
    out = B.router(dl.to(DEV), X.to(DEV), Wr.to(DEV))
    a, x, w = B.f64(dl), B.f64(X), B.f64(Wr)
    want, mag = products(a, x)
    with np.errstate(invalid="ignore"):
        same(out["dWr"], want, (T + 40) * U * mag + U * np.abs(want), "dWr")
        want, mag = products(a.T, w)
        half = 2.0 ** -8 if dt == torch.bfloat16 else U
        same(out["dX"], want, (E + 4) * U * mag + half * np.abs(want), "dX")
        same(out["dbias"], a.sum(0), (T + 40) * U * np.abs(a).sum(0), "dbias")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_parts_of_the_tokens_add_up_in_64_bits(dt):
    """One gradient in each slab of 64 tokens: 2^25, thirty times 1, -2^25.  The slabs lie
    in different parts of the token range, whose sums meet in 64 bits: 30, exactly."""
    T, d, E = 2048, 2048, 4
    dl = torch.zeros(T, E, device=DEV)
    dl[64:1984:64, 1] = 1.0
    dl[0, 1], dl[T - 1, 1] = 2.0 ** 25, -2.0 ** 25
    X = torch.ones(T, d, dtype=dt, device=DEV)
    out = B.router(dl, X, torch.zeros(E, d, dtype=dt, device=DEV), dx=False)
    assert bool((out["dWr"][1] == 30).all()) and out["dbias"].tolist() == [0, 30, 0, 0]
    assert not out["dWr"][[0, 2, 3]].any()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,E", [(5000, 40, 4), (3001, 2048, 64), (2000, 136, 200)])
def test_bias_gradient_is_a_sum_in_64_bits(T, d, E, dt):
    """2^25, ones and -2^25 in each of two columns: the ones' number, exactly."""
    dl = torch.ones(T, E, device=DEV)
    dl[0, 1], dl[T - 1, 1] = 2.0 ** 25, -2.0 ** 25
    dl[5, E - 1], dl[64, E - 1] = -2.0 ** 25, 2.0 ** 25
    want = torch.full((E,), float(T), device=DEV)
    want[1] = want[E - 1] = T - 2
    X, Wr = torch.zeros(T, d, dtype=dt, device=DEV), torch.zeros(E, d, dtype=dt, device=DEV)
    assert torch.equal(B.router(dl, X, Wr)["dbias"], want)
    assert torch.equal(B.router(dl, X, Wr, dx=False, dw=False)["dbias"], want)      # the fp32 kernel, of bias alone


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("e", [-60, -100, -118, -126])
def test_tiny_gradients_keep_their_bits(e, dt):
    """dlogits down to fp32's smallest normal numbers, whose lower parts are subnormal: off
    by the products' roundings, or by fp32's smallest step in each of the sum's terms.  In
    bf16, dlogits are taken apart into bf16 values: the upper halves of what is left, cut at
    the 16th bit, which for a subnormal stands for 2^-133.  What three cuts leave is below
    2^-133, whatever the value: a term is off by that times the other factor."""
    T, d, E = 130, 72, 20
    g = torch.Generator().manual_seed(-e)
    dl = (1 + torch.rand(T, E, generator=g)) * 2.0 ** e * (1 - 2 * torch.randint(0, 2, (T, E), generator=g))
    X, Wr = (torch.randn(n, d, generator=g).to(dt) for n in (T, E))
    out = B.router(dl.to(DEV), X.to(DEV), Wr.to(DEV))
    a, x, w = B.f64(dl), B.f64(X), B.f64(Wr)
    step = 2.0 ** -149
    for n, (want, mag), terms in (("dWr", products(a, x), T), ("dX", products(a.T, w), E)):
        half = 2.0 ** -8 if n == "dX" and dt == torch.bfloat16 else U
        tol = (terms + 40) * U * mag + half * np.abs(want) + (3 * terms + (2.0 ** 15 if half > U else 0)) * step
        if dt == torch.bfloat16:
            tol = tol + 2.0 ** -133 * (np.abs(x).sum(0) if n == "dWr" else np.abs(w).sum(0))
        err = np.abs(B.f64(out[n]) - want)
        assert np.all(err <= tol), (n, float((err / tol).max()))
