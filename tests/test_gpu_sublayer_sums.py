"""The gains' gradients are sums over the rows in 64 bits, within a block and over them."""
import pytest
import torch

from paper_2508_19078_amd import api

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_blocks_add_up_in_64_bits(dt):
    """512 rows in as many blocks: 2^25, 510 times 1, -2^25."""
    T, d = 512, 2048
    a, b = torch.ones(T, d, dtype=dt, device=DEV), torch.ones(T, d, dtype=dt, device=DEV)
    a[0], b[0] = 2.0 ** 12, 2.0 ** 13
    a[-1], b[-1] = -2.0 ** 12, 2.0 ** 13
    ws = torch.empty(api.moe_sublayer_norm_bwd_workspace_size(T, d), dtype=torch.uint8, device=DEV)
    dw = torch.full((2, d), float("nan"), device=DEV)
    # dw_post = sum dS Y
    api.moe_sublayer_norm_bwd(a, None, None, b, None, None, None, ws, post_norm=False, dw_post=dw[0])
    assert bool((dw[0] == 510).all())
    # dw_pre = sum dN S rstd
    api.moe_sublayer_norm_bwd(None, a, b, None, torch.ones(T, device=DEV), None, None, ws, post_norm=False, dw_pre=dw[1])
    assert bool((dw[1] == 510).all())
    # and on top of what was there, rounded once
    dw[1] = 2.0 ** -20
    api.moe_sublayer_norm_bwd(None, a, b, None, torch.ones(T, device=DEV), None, None, ws, post_norm=False, dw_pre=dw[1],
                              accumulate_dw=True)
    assert bool((dw[1] == torch.tensor(510 + 2.0 ** -20, device=DEV)).all())


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 256, 2048])
def test_rows_of_a_block_add_up_in_64_bits(d, dt):
    """Rows 2048 apart, which one block walks: 2^25, 31 times 1, -2^25; none of the others."""
    T = 32 * 2048 + 1
    a, b = torch.zeros(T, d, dtype=dt, device=DEV), torch.ones(T, d, dtype=dt, device=DEV)
    a[2048:T - 1:2048] = 1
    a[0], b[0] = 2.0 ** 12, 2.0 ** 13
    a[-1], b[-1] = -2.0 ** 12, 2.0 ** 13
    ws = torch.empty(api.moe_sublayer_norm_bwd_workspace_size(T, d), dtype=torch.uint8, device=DEV)
    dw = torch.full((2, d), float("nan"), device=DEV)
    api.moe_sublayer_norm_bwd(a, None, None, b, None, None, None, ws, post_norm=False, dw_post=dw[0])
    api.moe_sublayer_norm_bwd(None, a, b, None, torch.ones(T, device=DEV), None, None, ws, post_norm=False, dw_pre=dw[1])
    assert bool((dw == 31).all()), dw.unique().tolist()
