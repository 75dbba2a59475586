"""Refusals of the routing from scores, 8-bit float and gradient entry points, through the
C ABI and the binding.  Arguments are validated before any HIP call, so these run
without a GPU."""
import ctypes
import os

import pytest
import torch

from paper_2508_19078_amd import api

FAKE = 0x100000          # aligned, never dereferenced: validation fails first
MIS = FAKE + 4
F, I32, U8, D = torch.float32, torch.int32, torch.uint8, torch.float64
ARG, UNS, ALI, WSP = api.MOE_ERR_ARG, api.MOE_ERR_UNSUPPORTED, api.MOE_ERR_ALIGN, api.MOE_ERR_WORKSPACE


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


# ---------------------------------------------------------------- routing ----

def route(L, g=(), bwd=False, **over):
    g = dict(E=64, k=6, score="sigmoid", n_group=8, topk_group=4, group_top=2) | dict(g)
    score = g.pop("score")
    st = api.gating(**{**g, "score": "softmax"})
    st.score = api.SCORES.get(score, score)
    d = dict(logits=FAKE, bias=None, keep=None, T=16, idx=FAKE, gate=FAKE, counts=None, dgate=FAKE, out=FAKE + 4096, acc=0)
    d.update(over)
    p = ctypes.addressof(st)
    if bwd:
        rc = L.moe_route_scored_bwd(p, d["logits"], d["idx"], d["dgate"], d["T"], d["out"], d["acc"], None)
    else:
        rc = L.moe_route_scored(p, d["logits"], d["bias"], d["keep"], d["T"], d["idx"], d["gate"], d["counts"], None)
    return rc, L.moe_last_error().decode()


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("g,over,code,word", [
    (dict(E=0), {}, ARG, "E=0"),
    (dict(E=257, n_group=1, topk_group=1), {}, UNS, "E=257"),
    (dict(k=17, E=128), {}, UNS, "k=17"),
    (dict(k=0), {}, ARG, "k=0"),
    (dict(E=4, k=5, n_group=1, topk_group=1), {}, UNS, "k=5"),
    (dict(score=2), {}, UNS, "score=2"),
    (dict(n_group=7), {}, ARG, "n_group=7"),
    (dict(n_group=0), {}, ARG, "n_group=0"),
    (dict(n_group=64, group_top=1, topk_group=8), {}, UNS, "n_group=64"),
    (dict(topk_group=9), {}, ARG, "topk_group=9"),
    (dict(topk_group=0), {}, ARG, "topk_group=0"),
    (dict(n_group=32, topk_group=2), {}, ARG, "2 groups of 2"),
    (dict(group_top=3), {}, UNS, "group_top=3"),
    (dict(E=32, n_group=32, topk_group=8), {}, ARG, "group_top=2"),
    (dict(scale=float("nan")), {}, ARG, "scale"),
    (dict(scale=float("inf")), {}, ARG, "scale"),
    ({}, dict(T=-1), ARG, "T=-1"),
    ({}, dict(T=(1 << 30) + 1), UNS, "2^30"),
    ({}, dict(logits=None), ARG, "logits"),
    ({}, dict(idx=None), ARG, "idx"),
    ({}, dict(logits=MIS), ALI, "logits"),
    ({}, dict(idx=MIS), ALI, "idx"),
])
def test_routing_refusals(L, bwd, g, over, code, word):
    rc, msg = route(L, g, bwd, **over)
    assert rc == code and word in msg, (rc, msg)


def test_routing_refusals_of_one_direction(L):
    for over, code, word in ((dict(gate=None), ARG, "gate"), (dict(gate=MIS), ALI, "gate"), (dict(bias=MIS), ALI, "sel_bias"),
                             (dict(keep=MIS), ALI, "keep"), (dict(counts=MIS), ALI, "counts")):
        rc, msg = route(L, **over)
        assert rc == code and word in msg, (rc, msg)
    for over, code, word in ((dict(dgate=None), ARG, "dgate"), (dict(out=None), ARG, "dlogits"), (dict(out=MIS), ALI, "dlogits"),
                             (dict(dgate=MIS), ALI, "dgate"), (dict(out=FAKE, acc=1), ARG, "alias")):
        rc, msg = route(L, bwd=True, **over)
        assert rc == code and word in msg, (rc, msg)
    assert L.moe_route_scored(None, FAKE, None, None, 1, FAKE, FAKE, None, None) == ARG
    assert L.moe_route_scored_bwd(None, FAKE, FAKE, FAKE, 1, FAKE, 0, None) == ARG


def test_routing_without_tokens_enqueues_nothing(L):
    assert route(L, T=0, logits=None, idx=None, gate=None)[0] == api.MOE_OK
    assert route(L, bwd=True, T=0, logits=None, idx=None, dgate=None, out=None)[0] == api.MOE_OK
    assert route(L, dict(n_group=7), T=0)[0] == ARG          # the gating is still validated


LOGITS = (("X", FAKE), ("Wr", FAKE), ("dtype", api.MOE_BF16), ("bias", None), ("T", 16), ("d", 64), ("E", 8),
          ("logits", FAKE), ("st", None))
UPDATE = (("counts", FAKE), ("E", 8), ("rate", 0.001), ("bias", FAKE), ("st", None))
QUANT = (("W", FAKE), ("dtype", api.MOE_BF16), ("rows", 4), ("cols", 64), ("block", 128), ("codes", FAKE), ("scale", FAKE),
         ("st", None))
DEQUANT = (("codes", FAKE), ("scale", FAKE), ("rows", 4), ("cols", 64), ("block", 128), ("dtype", api.MOE_BF16), ("out", FAKE),
           ("st", None))


@pytest.mark.parametrize("name,defaults,over,code,word", [
    ("moe_router_logits", LOGITS, dict(E=257), UNS, "E=257"),
    ("moe_router_logits", LOGITS, dict(d=60), UNS, "d=60"),
    ("moe_router_logits", LOGITS, dict(T=-1), ARG, "T=-1"),
    ("moe_router_logits", LOGITS, dict(dtype=api.MOE_I8), UNS, "dtype"),
    ("moe_router_logits", LOGITS, dict(logits=None), ARG, "logits"),
    ("moe_router_logits", LOGITS, dict(X=MIS), ALI, "X"),
    ("moe_router_logits", LOGITS, dict(logits=MIS), ALI, "logits"),
    ("moe_route_bias_update", UPDATE, dict(E=0), ARG, "E=0"),
    ("moe_route_bias_update", UPDATE, dict(E=257), UNS, "E=257"),
    ("moe_route_bias_update", UPDATE, dict(rate=float("nan")), ARG, "rate"),
    ("moe_route_bias_update", UPDATE, dict(counts=None), ARG, "counts"),
    ("moe_route_bias_update", UPDATE, dict(bias=MIS), ALI, "sel_bias"),
    ("moe_quantize_fp8", QUANT, dict(rows=0), ARG, "rows=0"),
    ("moe_quantize_fp8", QUANT, dict(cols=60), UNS, "cols=60"),
    ("moe_quantize_fp8", QUANT, dict(block=64), UNS, "block_rows=64"),
    ("moe_quantize_fp8", QUANT, dict(block=0), UNS, "block_rows=0"),
    ("moe_quantize_fp8", QUANT, dict(dtype=api.MOE_I8), UNS, "dtype"),
    ("moe_quantize_fp8", QUANT, dict(scale=None), ARG, "scale"),
    ("moe_quantize_fp8", QUANT, dict(codes=MIS), ALI, "codes"),
    ("moe_dequant_fp8", DEQUANT, dict(cols=0), ARG, "cols=0"),
    ("moe_dequant_fp8", DEQUANT, dict(block=2), UNS, "block_rows=2"),
    ("moe_dequant_fp8", DEQUANT, dict(dtype=api.MOE_I8), UNS, "out_dtype"),
    ("moe_dequant_fp8", DEQUANT, dict(out=None), ARG, "out"),
    ("moe_dequant_fp8", DEQUANT, dict(scale=MIS), ALI, "scale"),
])
def test_refusals(L, name, defaults, over, code, word):
    rc, msg = call(L, name, defaults, **over)
    assert rc == code and word in msg, (rc, msg)


def test_logits_of_no_tokens(L):
    assert call(L, "moe_router_logits", LOGITS, T=0, X=None, Wr=None, logits=None)[0] == api.MOE_OK


# ---------------------------------------------------------- 8-bit forward ----

def fp8(L, layer=(), **over):
    lay = api.moe_layer_fp8(**{**dict(d=64, I=32, S_routed=4, S_shared=1, q_gate=FAKE, q_up=FAKE, q_down=FAKE, s_gate=FAKE,
                                      s_up=FAKE, s_down=FAKE), **dict(layer)})
    d = dict(X=FAKE, tok=FAKE, off=FAKE, T=16, k=2, O=FAKE, ws=FAKE, bytes=1 << 24)
    d.update(over)
    rc = L.moe_grouped_swiglu_fwd_fp8(ctypes.addressof(lay), d["X"], d["tok"], d["off"], d["T"], d["k"], d["O"], d["ws"],
                                      d["bytes"], None)
    return rc, L.moe_last_error().decode()


@pytest.mark.parametrize("layer,over,code,word", [
    (dict(d=72), {}, UNS, "d=72"),
    (dict(I=40), {}, UNS, "I=40"),
    (dict(d=2147483632, I=16), {}, UNS, "2^30"),
    (dict(I=0), {}, ARG, "I=0"),
    (dict(d=1 << 20, I=1 << 13), {}, UNS, "2^32 weights"),
    (dict(d=16, I=(1 << 24) + 16), {}, UNS, "2^24"),
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
def test_fp8_forward_refusals(L, layer, over, code, word):
    rc, msg = fp8(L, layer, **over)
    assert rc == code and word in msg, (rc, msg)


def test_fp8_forward_without_tokens_and_workspace_sizes(L):
    assert fp8(L, T=0, X=None, O=None, ws=None, bytes=0)[0] == api.MOE_OK
    assert L.moe_grouped_swiglu_fwd_fp8(None, FAKE, FAKE, FAKE, 1, 1, FAKE, FAKE, 1, None) == ARG
    lay = api.moe_layer_fp8(64, 32, 4, 1, *[FAKE] * 6)
    sizes = [L.moe_grouped_swiglu_fwd_fp8_workspace_size(ctypes.addressof(lay), T, 2) for T in (0, 1, 9, 16, 4096)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert L.moe_grouped_swiglu_fwd_fp8_workspace_size(None, 1, 2) == 0


# -------------------------------------------------------------- gradients ----

def tensor_set(**over):
    return api.moe_tensor_set(**{**dict(n=3, dtype=api.MOE_F32, data=FAKE, start=FAKE, total=100), **over})


@pytest.mark.parametrize("over,code,word", [
    (dict(n=0), ARG, "n=0"),
    (dict(n=(1 << 20) + 1), UNS, "2^20"),
    (dict(total=-1), ARG, "total=-1"),
    (dict(total=(1 << 48) + 1), UNS, "2^48"),
    (dict(dtype=api.MOE_I8), UNS, "dtype"),
    (dict(data=None), ARG, "data"),
    (dict(start=None), ARG, "start"),
    (dict(start=MIS), ALI, "start"),
])
def test_tensor_set_refusals(L, over, code, word):
    bad_set, good_set = tensor_set(**over), tensor_set()
    bad, good = ctypes.addressof(bad_set), ctypes.addressof(good_set)
    for f, args in ((L.moe_grad_norm, (bad, 0, FAKE, FAKE, FAKE, 1 << 20, None)),
                    (L.moe_grad_clip, (bad, FAKE, 1.0, 0.0, None, None)), (L.moe_grad_clip, (good, FAKE, 1.0, 0.0, bad, None))):
        rc = f(*args)
        assert rc == code and word in L.moe_last_error().decode(), (rc, L.moe_last_error())


def test_norm_and_clip_refusals(L):
    s = tensor_set()
    p = ctypes.addressof(s)
    ws = L.moe_grad_norm_workspace_size()
    for args, code, word in (((None, 0, FAKE, FAKE, FAKE, ws), ARG, "g must"), ((p, 0, None, FAKE, FAKE, ws), ARG, "sumsq"),
                             ((p, 0, FAKE, FAKE, None, ws), ARG, "ws"), ((p, 0, FAKE, FAKE, FAKE, ws - 1), WSP, "workspace"),
                             ((p, 0, FAKE, MIS, FAKE, ws), ALI, "norm"), ((p, 0, MIS, FAKE, FAKE, ws), ALI, "sumsq")):
        assert L.moe_grad_norm(*args, None) == code and word in L.moe_last_error().decode()
    for args, code, word in (((p, None, 1.0, 0.0, None), ARG, "sumsq"), ((p, FAKE, -1.0, 0.0, None), ARG, "max_norm"),
                             ((p, FAKE, float("inf"), 0.0, None), ARG, "max_norm"), ((p, FAKE, float("nan"), 0.0, None), ARG, "max_norm"),
                             ((p, FAKE, 1.0, -1.0, None), ARG, "eps"), ((p, FAKE, 1.0, float("nan"), None), ARG, "eps")):
        assert L.moe_grad_clip(*args, None) == code and word in L.moe_last_error().decode()
    for over in (dict(n=2), dict(total=99), dict(dtype=api.MOE_BF16)):
        other = tensor_set(**over)
        assert L.moe_grad_clip(p, FAKE, 1.0, 0.0, ctypes.addressof(other), None) == ARG
        assert "out:" in L.moe_last_error().decode()


# ---------------------------------------------------------------- binding ----

def test_binding_refuses_memory_the_library_cannot_read():
    t = lambda *s, dt=F: torch.zeros(*s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError, match="device memory"):
        api.moe_quantize_fp8(t(4, 40), t(4, 40, dt=U8), t(1, 1))
    with pytest.raises(ValueError, match="device memory"):
        api.moe_route_scored(api.gating(8, 2), t(4, 8), t(4, 2, dt=I32), t(4, 2))
    with pytest.raises(ValueError, match="device memory"):
        api.TensorSet([t(4)])
    with pytest.raises(ValueError, match="no tensors"):
        api.TensorSet([])
    with pytest.raises(ValueError, match="score"):
        api.gating(8, 2, score="tanh")
    with pytest.raises(ValueError, match="2 slots"):
        api.LayerTablesFP8(64, 32, 2, 0, *[[t(1, dt=U8)]] * 6, device="cpu")
    with pytest.raises(ValueError, match="q_gate"):
        api.LayerTablesFP8(64, 32, 2, 0, *[[t(1, dt=U8)] * 2] * 6, device="cpu")
    assert api.fp8_scale_shape(129, 688) == (2, 6) and api.fp8_scale_shape(129, 688, 1) == (129, 6)


@pytest.mark.gpu
def test_binding_refuses_tensors_it_would_misread():
    t = lambda *s, dt=F: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    g = api.gating(8, 2)
    with pytest.raises(ValueError, match="logits"):
        api.moe_route_scored(g, t(4, 9), t(4, 2, dt=I32), t(4, 2))
    with pytest.raises(ValueError, match="gate"):
        api.moe_route_scored(g, t(4, 8), t(4, 2, dt=I32), t(4, 3))
    with pytest.raises(TypeError, match="int64"):
        api.moe_route_scored(g, t(4, 8), t(4, 2, dt=torch.int64), t(4, 2))
    with pytest.raises(ValueError, match="sel_bias"):
        api.moe_route_scored(g, t(4, 8), t(4, 2, dt=I32), t(4, 2), sel_bias=t(7))
    with pytest.raises(ValueError, match="contiguous"):
        api.moe_route_scored(g, t(4, 16)[:, ::2], t(4, 2, dt=I32), t(4, 2))
    with pytest.raises(ValueError, match="dlogits"):
        api.moe_route_scored_bwd(g, t(4, 8), t(4, 2, dt=I32), t(4, 2), t(3, 8))
    with pytest.raises(ValueError, match="counts"):
        api.moe_route_bias_update(t(7, dt=I32), t(8), 0.1)
    with pytest.raises(ValueError, match="logits"):
        api.moe_router_logits(t(4, 16), t(8, 16), None, t(4, 7))
    with pytest.raises(ValueError, match="scale"):
        api.moe_quantize_fp8(t(4, 40), t(4, 40, dt=U8), t(4, 1))
    with pytest.raises(api.MoeError, match="block_rows=0"):
        api.moe_quantize_fp8(t(4, 40), t(4, 40, dt=U8), t(4, 1), block_rows=0)
    with pytest.raises(ValueError, match="codes"):
        api.moe_dequant_fp8(t(4, 20, dt=U8), t(1, 1), t(4, 40))
    with pytest.raises(ValueError, match="aligned"):
        q, s = [t(32, 64, dt=U8).view(-1)[4:][:1024].view(16, 64)], [t(1, 1)]
        api.LayerTablesFP8(64, 16, 1, 0, q, q, [t(64, 16, dt=U8)], s, s, s)
    x = t(12)
    for shared in ([x, t(4), x], [x[8:], None, x[:9]], [x, x[4:5]]):
        with pytest.raises(ValueError, match="share memory"):
            api.TensorSet(shared)
    assert api.TensorSet([x[8:], x[:0], x[:8], x[12:]]).sizes == [4, 0, 8, 0]
    a = api.TensorSet([t(4), None, t(3, 5)])
    with pytest.raises(TypeError, match="bfloat16"):
        api.TensorSet([t(4), t(4, dt=torch.bfloat16)])
    with pytest.raises(TypeError, match="float64"):
        api.moe_grad_norm(a, t(1), t(1), t(2048))
    with pytest.raises(ValueError, match="other sizes"):
        api.moe_grad_clip(a, t(1, dt=D), 1.0, out=api.TensorSet([t(4), t(3, 5)]))
    with pytest.raises(api.MoeError, match="workspace"):
        api.moe_grad_norm(a, t(1, dt=D), t(1), t(8))


def results(grads, outs):
    api._check_results(api._spans(outs), api._spans(grads))


def test_results_that_would_be_written_while_they_are_read():
    """Addresses alone decide, so host tensors stand for device ones."""
    x, y, z = torch.zeros(64), torch.zeros(32), torch.zeros(64)
    a, b = x[8:24], x[24:40]
    grads = [a, None, b, y]
    for outs in (grads, [z[:16], None, z[16:32], y], [a, None, z[:16], z[16:48]], [x[:8], None, x[40:56], z[:32]], [x[:0], None, z[:0], x[8:8]]):
        results(grads, outs)
    for outs, word in (([x[9:25], None, z[:16], y], r"out\[0\] and grads\[0\]"), ([x[7:23], None, z[:16], y], r"out\[0\] and grads\[0\]"),
                       ([z[:16], None, a, y], r"out\[2\] and grads\[0\]"), ([b, None, a, y], "share memory"),
                       ([z[:16], None, z[16:32], x[:32]], r"out\[3\] and grads\[0\]"), ([z[:16], None, z[16:32], x[39:]], r"out\[3\] and grads\[2\]"),
                       ([z[:16], y[:16], z[16:32], z[32:]], r"out\[1\] and grads\[3\]"), ([x, None, z[:16], y], r"out\[0\] and grads"),
                       ([a[:15], None, z[:16], y], r"out\[0\] and grads\[0\]")):
        with pytest.raises(ValueError, match=word):
            results(grads, outs)
    many = [t[1:] for t in torch.zeros(4096).split(4)]
    results(many, many)
    results(many, [torch.zeros(3) for _ in many])
    with pytest.raises(ValueError, match=r"out\[700\] and grads\[701\]"):
        results(many, many[:700] + [many[701]])


@pytest.mark.gpu
def test_binding_refuses_results_that_share_memory():
    t = lambda *s, dt=F: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    x, sumsq = t(300), t(1, dt=D)
    grads = api.TensorSet([x[:100], None, x[100:200]])
    for outs in ([x[1:101], None, x[150:250]], [x[100:200], None, x[:100]], [x[:100], None, x[101:201]]):
        with pytest.raises(ValueError, match="share memory"):
            api.moe_grad_clip(grads, sumsq, 1.0, out=api.TensorSet(outs))
    apart, mixed = api.TensorSet([t(100), None, x[200:]]), api.TensorSet([x[:100], None, x[200:]])
    for _ in range(2):                                     # compared once, and again with another set between
        for out in (apart, mixed, grads):
            api.moe_grad_clip(grads, sumsq, 1.0, out=out)
    assert not x.any()
