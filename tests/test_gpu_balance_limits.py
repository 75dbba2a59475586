"""The balance loss and the gradient of its logits over more tokens than one launch can
take.  u = 2^-24."""
import numpy as np
import pytest
import torch

from paper_2508_19078_amd import api

import test_gpu_balance as B

pytestmark = pytest.mark.gpu
DEV, U, INF = "cuda", 2.0 ** -24, float("inf")


def test_tokens_past_one_launch_of_the_loss():
    """2^29 + 40 tokens: a thread for each eighth of one passes the 2^32 of a launch."""
    T = (1 << 29) + 40
    z = torch.zeros(T, 1, device=DEV)
    idx = torch.zeros(T, 1, dtype=torch.int32, device=DEV)
    idx[-3:], idx[5] = -1, -1
    seg = torch.tensor([0, T - 8, T], dtype=torch.int32, device=DEV)
    counts, dprob, loss = B.loss_of(z, idx, 0.25, seg)
    assert counts.tolist() == [[T - 9], [5]]
    want = np.array([0.25 * (T - 9) / (T * (T - 8.0)), 0.25 * 5 / (T * 8.0)])
    np.testing.assert_allclose(B.f64(dprob)[:, 0], want, rtol=2 * U)
    assert abs(float(loss) - (want * [T - 8, 8]).sum()) <= 60 * U * 0.25
    gate = torch.ones(T, 1, device=DEV)
    out = z                                            # in the logits' place
    api.moe_balance_loss_bwd(z, dprob, None, out, seg=seg, gate=gate, idx=idx, dgate=gate)
    assert not out.any()                               # one expert: nothing to move to
    gate[-20:], gate[100] = 0.5, 0.25                  # (gates that are no softmax: the formula's)
    ones = torch.ones_like(gate)
    idx[-3:], idx[5] = 0, 0
    api.moe_balance_loss_bwd(z, dprob, None, out, seg=seg, gate=gate, idx=idx, dgate=ones)
    assert bool((out[-20:] == 0.25).all()) and float(out[100]) == 0.25 * 0.75 and int((out != 0).sum()) == 21


def test_tokens_past_one_launch_of_the_logits_gradient():
    """2^27 + 24 tokens of 17 experts: 32 lanes a token."""
    T, E = (1 << 27) + 24, 17
    z = torch.zeros(T, E, device=DEV)
    z[-5, 3] = -INF
    keep = torch.ones(T, dtype=torch.uint8, device=DEV)
    keep[-2:], keep[7] = 0, 0
    dprob = torch.arange(E, dtype=torch.float32, device=DEV)[None].contiguous()
    api.moe_balance_loss_bwd(z, dprob, None, z, keep=keep)
    w = np.arange(E)
    even = (w - w.mean()) / E
    # p is rounded once or not at all, the sum of p w some 7 times, then two more
    tol = 40 * U * (w + w.mean()) / E
    assert bool((z[8:T - 5] == z[0]).all()) and not z[-2:].any() and not z[7].any()
    assert np.all(np.abs(B.f64(z[0]) - even) <= tol)
    p = np.where(w == 3, 0, 1 / 16)
    assert np.all(np.abs(B.f64(z[-5]) - p * (w - (p * w).sum())) <= 2 * tol)
