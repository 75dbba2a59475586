"""The router's dense backward where it can go wrong.  u = 2^-24; the products' tolerances are test_gpu_balance's."""
import numpy as np
import pytest
import torch

from paper_2508_19078_amd import api

import test_gpu_balance as B

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24


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
