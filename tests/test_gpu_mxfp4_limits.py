"""More rows than one launch of the quantisation can take."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_rows_past_one_launch():
    """2^28 + 3 rows of 8 columns: 16 threads a row pass the 2^32 of a launch."""
    rows, cols = (1 << 28) + 3, 8
    W = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    tail = torch.randn(40, cols, generator=torch.Generator().manual_seed(0)).bfloat16()
    at = [slice(0, 10), slice((1 << 27) - 5, (1 << 27) + 5), slice((1 << 28) - 5, (1 << 28) + 3)]   # the launches' ends
    for i, s in enumerate(at):
        W[s] = tail[10 * i:10 * i + s.stop - s.start].to(DEV)
    cs, ss = api.mxfp4_shapes(rows, cols)
    codes = torch.full(cs, 0xAA, dtype=torch.uint8, device=DEV)
    scale = torch.full(ss, 0xAA, dtype=torch.uint8, device=DEV)
    api.moe_quantize_mxfp4(W, codes, scale)
    want, byte = O.mxfp4_rows(tail.double().numpy())
    n = 0
    for i, s in enumerate(at):
        w = want[10 * i:10 * i + s.stop - s.start]
        c = codes[s].cpu().numpy()
        np.testing.assert_array_equal(np.stack((c & 15, c >> 4), -1).reshape(len(c), -1)[:, :cols], w)
        assert not c[:, cols // 2:].any()
        np.testing.assert_array_equal(scale[s].cpu().numpy()[:, 0], byte[10 * i:10 * i + s.stop - s.start, 0])
        n += int((scale[s] != 0).sum())
    assert int((scale != 0).sum()) == n                # all other rows are zero blocks
    W.fill_(float("nan"))
    api.moe_dequant_mxfp4(codes, scale, W)
    for i, s in enumerate(at):
        np.testing.assert_array_equal(W[s].double().cpu().numpy(),
                                      O.mxfp4_values(want, byte)[10 * i:10 * i + s.stop - s.start])
    assert bool((W[10:(1 << 27) - 5] == 0).all())
