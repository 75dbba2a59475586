"""Sizes that are refused because a launch could not hold them (no GPU)."""
import test_abi_operators as A
from test_abi_operators import L  # noqa: F401  (the built library)

from paper_2508_19078_amd import api


def test_router_backward_of_more_than_2_30_weights(L):  # noqa: F811
    for E, d in ((256, 1 << 24), (256, (1 << 22) + 8), (1, 2147483640), (200, 1 << 23)):
        rc, msg = A.call(L, "moe_router_bwd", A.ROUTER, E=E, d=d, bytes=1 << 62)
        assert rc == api.MOE_ERR_UNSUPPORTED and "2^30" in msg and f"d={d}" in msg, (rc, msg)
