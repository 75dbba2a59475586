"""MXFP4 rows at the ends of both types' ranges, in and out, against the fp64 oracle:
the quantisation and the dequantisation of bf16 are code of their own for these.

Codes and scale bytes are exact.  Values are exact down to 2^-126; a smaller one may
come out as 0."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

import test_gpu_mxfp4 as M

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN, INF = float("nan"), float("inf")


def rows(dt):
    """(W [n, 64], the blocks (row, block) that hold no number)."""
    big = torch.finfo(dt).max
    tiny = 2.0 ** -149 if dt == torch.float32 else 2.0 ** -133
    W = torch.zeros(18, 64)
    W[0, :4] = torch.tensor([big, -big / 2, big / 8, 3 * 2.0 ** 125])   # cut at 6
    W[1, 5] = tiny                                            # below byte 0's smallest code
    W[2, :3] = torch.tensor([2.0 ** -126, -2.0 ** -127, 3 * 2.0 ** -128])
    # the largest of a block on either side of 2^-124: bytes 0 and 1
    W[3, :5] = torch.tensor([1.9375 * 2.0 ** -125, -1.5 * 2.0 ** -125, 2.0 ** -126, 2.0 ** -128, -1.25 * 2.0 ** -127])
    W[4, :5] = torch.tensor([2.0 ** -124, -1.5 * 2.0 ** -125, 1.25 * 2.0 ** -126, 2.0 ** -127, -0.75 * 2.0 ** -127])
    W[5, 31], W[5, 32] = -2.0 ** -124, 1.75 * 2.0 ** -125     # one block each side
    W[6] = -0.0
    W[7, 8:16] = torch.tensor([0.25, -0.25, 0.75, 5, -7, 6, 3.5, -2.5])
    W[8] = torch.linspace(-8, 8, 64)
    none = []
    for r, (at, v) in enumerate([((3,), INF), ((4,), NAN), ((40,), -INF), ((63,), NAN), ((0, 32), NAN), ((31,), -INF)], 9):
        W[r] = torch.linspace(-3, 5, 64)
        W[r, list(at)] = v
        none += [(r, a // 32) for a in at]
    W[15, 7], W[15, 39] = INF, big                            # beside the largest finite block
    none.append((15, 0))
    W[16, 0], W[16, 1] = NAN, INF
    none.append((16, 0))
    return W.to(dt), none


@pytest.mark.parametrize("out_dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_rows(dt, out_dt):
    W, none = rows(dt)
    n = len(W)
    codes, scale = M.quantize(W.to(DEV))
    out = torch.full((n, 64), 7.0, dtype=out_dt, device=DEV)
    api.moe_dequant_mxfp4(codes, scale, out)
    out, s, c = out.double().cpu().numpy(), scale.cpu().numpy()[:, :2], M.unpacked(codes, 64)
    clean = W.double().numpy().reshape(n, 2, 32)
    for r, b in none:
        clean[r, b] = 0
    want, byte = O.mxfp4_rows(clean.reshape(n, 64))
    value = O.mxfp4_values(want, byte)
    assert byte[3, 0] == 0 and byte[4, 0] == 1 and want[3, :5].any() and want[4, :5].any()   # what the rows are there for
    for r in range(n):
        for b in range(2):
            at = slice(32 * b, 32 * b + 32)
            if (r, b) in none:
                assert s[r, b] == 255 and not c[r, at].any() and np.isnan(out[r, at]).all(), (r, b)
                continue
            assert s[r, b] == byte[r, b], (r, b)
            np.testing.assert_array_equal(c[r, at], want[r, at])
            v, g = value[r, at], out[r, at]
            assert np.all((g == v) | ((g == 0) & (np.abs(v) < 2.0 ** -126))), (r, b)


@pytest.mark.parametrize("out_dt", [torch.bfloat16, torch.float32])
def test_every_code_at_every_scale(out_dt):
    """Dequantisation alone: 16 codes under each scale byte that a quantisation leaves
    (the largest finite block's is 252)."""
    codes = torch.arange(16, dtype=torch.uint8)
    codes = (codes[0::2] | codes[1::2] << 4).repeat(254, 2).contiguous()
    byte = torch.cat((torch.arange(253), torch.tensor([255]))).to(torch.uint8)
    scale = torch.zeros(254, 4, dtype=torch.uint8)
    scale[:, 0] = byte
    out = torch.full((254, 32), 7.0, dtype=out_dt, device=DEV)
    api.moe_dequant_mxfp4(codes.to(DEV), scale.to(DEV), out)
    out = out.double().cpu().numpy()
    want = O.mxfp4_values(M.unpacked(codes, 32)[:253], np.arange(253)[:, None])
    tiny = np.abs(want) < 2.0 ** -126
    assert np.all((out[:253] == want) | (tiny & (out[:253] == 0)))
    assert np.isnan(out[253]).all()
