"""Refusals of the 4-bit, balance-loss, router-backward and sublayer-norm entry
points, through the C ABI and the binding.  Arguments are validated before any
HIP call, so these run without a GPU."""
import ctypes
import os

import pytest
import torch

from paper_2508_19078_amd import api

FAKE = 0x100000          # aligned, never dereferenced: validation fails first
MIS = FAKE + 4
F, I32, U8 = torch.float32, torch.int32, torch.uint8


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(api.LIB_PATH):
        from paper_2508_19078_amd import build
        build.build(verbose=False)
    return api.lib()


def call(L, name, defaults, **over):
    args = [over.get(n, v) for n, v in defaults]
    assert set(over) <= {n for n, _ in defaults}, over
    return getattr(L, name)(*args), L.moe_last_error().decode()


BALANCE = (("logits", FAKE), ("idx", FAKE), ("seg", None), ("keep", None), ("T", 16), ("E", 8), ("k", 2), ("B", 1),
           ("coef", 0.01), ("counts", FAKE), ("dprob", FAKE), ("loss", FAKE), ("ws", FAKE), ("bytes", 1 << 20), ("st", None))
DLOGITS = (("logits", FAKE), ("dprob", FAKE), ("dloss", None), ("seg", None), ("keep", None), ("gate", None),
           ("idx", None), ("dgate", None), ("T", 16), ("E", 8), ("k", 2), ("B", 1), ("out", FAKE), ("st", None))
ROUTER = (("dl", FAKE), ("X", FAKE), ("Wr", FAKE), ("dtype", api.MOE_BF16), ("T", 16), ("d", 64), ("E", 8),
          ("dX", FAKE + 64), ("acc_dx", 0), ("dWr", FAKE), ("dbias", FAKE), ("acc_dw", 0), ("ws", FAKE),
          ("bytes", 1 << 20), ("st", None))
NORM = (("X", FAKE), ("Y", FAKE), ("gate", None), ("w_post", None), ("w_pre", None), ("T", 4), ("d", 64),
        ("dtype", api.MOE_BF16), ("alpha", 1.0), ("post", 1), ("eps", 1e-6), ("S", FAKE), ("N", FAKE + 64),
        ("rstd_y", None), ("rstd_s", None), ("st", None))
NORM_BWD = (("dS", FAKE), ("dN", FAKE), ("S", FAKE), ("Y", FAKE), ("gate", None), ("w_post", None), ("w_pre", None),
            ("rstd_y", FAKE), ("rstd_s", FAKE), ("T", 4), ("d", 64), ("dtype", api.MOE_BF16), ("alpha", 1.0),
            ("post", 1), ("dX", FAKE), ("dY", FAKE + 64), ("dgate", None), ("dw_post", FAKE), ("dw_pre", FAKE),
            ("acc", 0), ("ws", FAKE), ("bytes", 1 << 20), ("st", None))
QUANT = (("W", FAKE), ("dtype", api.MOE_BF16), ("rows", 4), ("cols", 64), ("codes", FAKE), ("scale", FAKE), ("st", None))
DEQUANT = (("codes", FAKE), ("scale", FAKE), ("rows", 4), ("cols", 64), ("dtype", api.MOE_BF16), ("out", FAKE),
           ("st", None))

ARG, UNS, ALI, WSP = api.MOE_ERR_ARG, api.MOE_ERR_UNSUPPORTED, api.MOE_ERR_ALIGN, api.MOE_ERR_WORKSPACE
BAD = [
    ("moe_balance_loss", BALANCE, dict(k=9), UNS, "k=9"),
    ("moe_balance_loss", BALANCE, dict(E=257), UNS, "E=257"),
    ("moe_balance_loss", BALANCE, dict(E=64, k=17), UNS, "k=17"),
    ("moe_balance_loss", BALANCE, dict(T=-1), ARG, "T=-1"),
    ("moe_balance_loss", BALANCE, dict(T=(1 << 30) + 1), UNS, "2^30"),
    ("moe_balance_loss", BALANCE, dict(B=2), ARG, "without seg"),
    ("moe_balance_loss", BALANCE, dict(B=0), ARG, "B=0"),
    ("moe_balance_loss", BALANCE, dict(seg=FAKE, B=4097), UNS, "B=4097"),
    ("moe_balance_loss", BALANCE, dict(coef=float("nan")), ARG, "coef"),
    ("moe_balance_loss", BALANCE, dict(logits=None), ARG, "logits"),
    ("moe_balance_loss", BALANCE, dict(loss=None), ARG, "loss"),
    ("moe_balance_loss", BALANCE, dict(seg=MIS), ALI, "seg"),
    ("moe_balance_loss", BALANCE, dict(bytes=16), WSP, "workspace"),
    ("moe_balance_loss", BALANCE, dict(ws=None), ARG, "ws"),
    ("moe_balance_loss_bwd", DLOGITS, dict(gate=FAKE), ARG, "together"),
    ("moe_balance_loss_bwd", DLOGITS, dict(gate=FAKE, idx=FAKE, dgate=FAKE, k=9), UNS, "k=9"),
    ("moe_balance_loss_bwd", DLOGITS, dict(dprob=None), ARG, "dprob"),
    ("moe_balance_loss_bwd", DLOGITS, dict(out=MIS), ALI, "dlogits"),
    ("moe_balance_loss_bwd", DLOGITS, dict(E=300), UNS, "E=300"),
    ("moe_router_bwd", ROUTER, dict(d=60), UNS, "d=60"),
    ("moe_router_bwd", ROUTER, dict(T=2147483647, d=8), UNS, "2^30"),
    ("moe_router_bwd", ROUTER, dict(dtype=api.MOE_I8), UNS, "dtype"),
    ("moe_router_bwd", ROUTER, dict(Wr=None), ARG, "Wr"),
    ("moe_router_bwd", ROUTER, dict(X=None), ARG, "X"),
    ("moe_router_bwd", ROUTER, dict(dX=FAKE), ARG, "alias"),
    ("moe_router_bwd", ROUTER, dict(bytes=64), WSP, "workspace"),
    ("moe_router_bwd", ROUTER, dict(dbias=MIS), ALI, "dbias"),
    ("moe_sublayer_norm", NORM, dict(d=60), UNS, "d=60"),
    ("moe_sublayer_norm", NORM, dict(d=8200), UNS, "d=8200"),
    ("moe_sublayer_norm", NORM, dict(eps=-1.0), ARG, "eps"),
    ("moe_sublayer_norm", NORM, dict(alpha=float("inf")), ARG, "alpha"),
    ("moe_sublayer_norm", NORM, dict(Y=None), ARG, "without Y"),
    ("moe_sublayer_norm", NORM, dict(Y=None, post=0, gate=FAKE), ARG, "without Y"),
    ("moe_sublayer_norm", NORM, dict(S=None, N=None), ARG, "both"),
    ("moe_sublayer_norm", NORM, dict(N=None, rstd_s=FAKE), ARG, "rstd_s"),
    ("moe_sublayer_norm", NORM, dict(post=0, rstd_y=FAKE), ARG, "rstd_y"),
    ("moe_sublayer_norm", NORM, dict(N=FAKE), ARG, "alias"),
    ("moe_sublayer_norm", NORM, dict(gate=MIS), ALI, "gate"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(dS=None, dN=None), ARG, "both"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(S=None), ARG, "S must"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(rstd_s=None), ARG, "rstd_s"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(rstd_y=None), ARG, "rstd_y"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(Y=None), ARG, "without Y"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(dY=FAKE), ARG, "alias"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(bytes=8), WSP, "workspace"),
    ("moe_sublayer_norm_bwd", NORM_BWD, dict(dw_pre=MIS), ALI, "dw_pre"),
    ("moe_quantize_mxfp4", QUANT, dict(cols=12), UNS, "cols=12"),
    ("moe_quantize_mxfp4", QUANT, dict(rows=0), ARG, "rows=0"),
    ("moe_quantize_mxfp4", QUANT, dict(cols=2147483640), UNS, "2^30"),
    ("moe_quantize_mxfp4", QUANT, dict(dtype=api.MOE_I8), UNS, "dtype"),
    ("moe_quantize_mxfp4", QUANT, dict(scale=None), ARG, "scale"),
    ("moe_quantize_mxfp4", QUANT, dict(codes=MIS), ALI, "codes"),
    ("moe_dequant_mxfp4", DEQUANT, dict(cols=-8), ARG, "cols=-8"),
    ("moe_dequant_mxfp4", DEQUANT, dict(out=MIS), ALI, "out"),
]


@pytest.mark.parametrize("name,defaults,over,code,word", BAD,
                         ids=[f"{n[4:]}-{'-'.join(f'{a}={b}' for a, b in o.items())}" for n, _, o, _, _ in BAD])
def test_refusals(L, name, defaults, over, code, word):
    rc, msg = call(L, name, defaults, **over)
    assert rc == code and word in msg, (rc, msg)


def test_calls_without_tokens_enqueue_nothing(L):
    assert call(L, "moe_balance_loss_bwd", DLOGITS, T=0, logits=None, dprob=None, out=None)[0] == api.MOE_OK
    assert call(L, "moe_router_bwd", ROUTER, T=0, dl=None, X=None, Wr=None, dWr=None, dbias=None)[0] == api.MOE_OK
    assert call(L, "moe_router_bwd", ROUTER, T=0, dl=None, X=None, acc_dw=1)[0] == api.MOE_OK
    assert call(L, "moe_sublayer_norm", NORM, T=0, X=None, Y=None, S=None, N=None)[0] == api.MOE_OK
    assert call(L, "moe_sublayer_norm_bwd", NORM_BWD, T=0, acc=1)[0] == api.MOE_OK
    # ... but the shape is still validated
    assert call(L, "moe_sublayer_norm", NORM, T=0, d=12)[0] == UNS
    assert call(L, "moe_balance_loss_bwd", DLOGITS, T=0, E=0)[0] == ARG


MX4 = dict(layer=dict(d=64, I=32, S_routed=4, S_shared=1, q_gate=FAKE, q_up=FAKE, q_down=FAKE, s_gate=FAKE, s_up=FAKE,
                      s_down=FAKE))


def mx4(L, layer=(), **over):
    lay = api.moe_layer_mx4(**{**MX4["layer"], **dict(layer)})
    d = dict(X=FAKE, tok=FAKE, off=FAKE, T=16, k=2, O=FAKE, ws=FAKE, bytes=1 << 24)
    d.update(over)
    rc = L.moe_grouped_swiglu_fwd_mx4(ctypes.addressof(lay), d["X"], d["tok"], d["off"], d["T"], d["k"], d["O"], d["ws"],
                                      d["bytes"], None)
    return rc, L.moe_last_error().decode()


@pytest.mark.parametrize("layer,over,code,word", [
    (dict(d=60), {}, UNS, "d=60"),
    (dict(d=2147483640, I=8), {}, UNS, "2^30"),
    (dict(I=0), {}, ARG, "I=0"),
    (dict(d=1 << 20, I=1 << 13), {}, UNS, "2^32 weights"),
    (dict(S_routed=513), {}, ARG, "S_routed=513"),
    (dict(S_routed=0, S_shared=0), {}, ARG, "S_routed=0"),
    (dict(s_up=None), {}, ARG, "s_up"),
    ({}, dict(k=0), ARG, "k=0"),
    ({}, dict(k=17), ARG, "k=17"),
    ({}, dict(T=1 << 26), UNS, "2^32 values"),
    ({}, dict(tok=None), ARG, "perm_token"),
    ({}, dict(O=None), ARG, "O must"),
    ({}, dict(X=MIS), ALI, "X"),
    ({}, dict(bytes=100), WSP, "workspace"),
])
def test_mx4_forward_refusals(L, layer, over, code, word):
    rc, msg = mx4(L, layer, **over)
    assert rc == code and word in msg, (rc, msg)


def test_mx4_forward_without_tokens_and_workspace_sizes(L):
    assert mx4(L, T=0, X=None, O=None, ws=None, bytes=0)[0] == api.MOE_OK
    assert L.moe_grouped_swiglu_fwd_mx4(None, FAKE, FAKE, FAKE, 1, 1, FAKE, FAKE, 1, None) == ARG
    lay = api.moe_layer_mx4(**MX4["layer"])
    sizes = [L.moe_grouped_swiglu_fwd_mx4_workspace_size(ctypes.addressof(lay), T, 2) for T in (0, 1, 16, 4096)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert L.moe_balance_loss_workspace_size(-1, 8, 1) == 0
    assert L.moe_router_bwd_workspace_size(64, 64, 8) > 0
    assert L.moe_sublayer_norm_bwd_workspace_size(0, 64) == 0


def test_binding_refuses_memory_the_library_cannot_read():
    t = lambda *s, dt=F: torch.zeros(*s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError, match="device memory"):
        api.moe_quantize_mxfp4(t(4, 40), t(4, 32, dt=U8), t(4, 4, dt=U8))
    with pytest.raises(ValueError, match="device memory"):
        api.moe_sublayer_norm(t(4, 16), None, t(4, 16), None)
    with pytest.raises(ValueError, match="q_gate"):
        api.LayerTablesMX4(64, 32, 2, 0, *[[t(1, dt=U8)] * 2] * 6, device="cpu")
    with pytest.raises(ValueError, match="2 slots"):
        api.LayerTablesMX4(64, 32, 2, 0, *[[t(1, dt=U8)]] * 6, device="cpu")
    assert api.mxfp4_shapes(7, 688) == ((7, 352), (7, 24))


@pytest.mark.gpu
def test_binding_refuses_tensors_it_would_misread():
    """Wrong shapes, types and layouts, before anything is enqueued."""
    t = lambda *s, dt=F: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    with pytest.raises(ValueError, match="counts"):
        api.moe_balance_loss(t(4, 8), t(4, 2, dt=I32), 0.1, t(2, 8, dt=I32), t(1, 8), t(1), t(64))
    with pytest.raises(ValueError, match="dprob"):
        api.moe_balance_loss_bwd(t(4, 8), t(1, 8), None, t(4, 8), seg=t(3, dt=I32))
    with pytest.raises(ValueError, match="dWr"):
        api.moe_router_bwd(t(4, 8), t(4, 16), t(8, 16), t(64), dWr=t(8, 8))
    with pytest.raises(ValueError, match="gate"):
        api.moe_sublayer_norm(t(4, 16), t(4, 16), t(4, 16), t(4, 16), gate=t(4, 1))
    with pytest.raises(ValueError, match="rstd_s"):
        api.moe_sublayer_norm_bwd(t(4, 16), t(4, 16), t(4, 16), None, t(5), t(4, 16), None, t(64))
    with pytest.raises(ValueError, match="scale"):
        api.moe_quantize_mxfp4(t(4, 40), t(4, 32, dt=U8), t(4, 2, dt=U8))
    with pytest.raises(ValueError, match="codes"):
        api.moe_dequant_mxfp4(t(4, 20, dt=U8), t(4, 4, dt=U8), t(4, 40))
    with pytest.raises(TypeError, match="int64"):
        api.moe_balance_loss(t(4, 8), t(4, 2, dt=torch.int64), 0.1, t(1, 8, dt=I32), t(1, 8), t(1), t(64))
    with pytest.raises(TypeError, match="float32"):
        api.moe_sublayer_norm(t(4, 16, dt=torch.bfloat16), t(4, 16), t(4, 16, dt=torch.bfloat16), None)
    with pytest.raises(ValueError, match="contiguous"):
        api.moe_sublayer_norm(t(4, 32)[:, ::2], None, t(4, 16), None)
    with pytest.raises(api.MoeError, match="aligned"):
        api.moe_sublayer_norm(t(4, 16), t(4, 16), t(4, 16), None, gate=t(5)[1:])


def test_workspaces_for_more_tokens_serve_fewer(L):
    for d, E in ((264, 20), (2048, 64), (136, 130)):
        sizes = [L.moe_router_bwd_workspace_size(T, d, E) for T in range(0, 6400, 32)]
        assert sizes == sorted(sizes)
        sizes = [L.moe_balance_loss_workspace_size(T, E, 4) for T in range(0, 6400, 16)]
        assert sizes == sorted(sizes)
        sizes = [L.moe_sublayer_norm_bwd_workspace_size(T, d) for T in range(0, 6400, 16)]
        assert sizes == sorted(sizes)
