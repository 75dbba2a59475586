"""GPU parity of the global gradient norm and of clipping, against fp64.

sumsq: squares and sums in fp64, n roundings of 2^-53 at most, relative (all terms are
positive): n 2^-52.  norm: one rounding to fp32.  Clipped values: the coefficient's
rounding and the product's in fp32, 2^-23 relative and a smallest subnormal, and for bf16
the rounding of the result, 2^-8."""
import math

import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

from gpu_harness import log

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def tensors(sizes, dt, seed=0, offset=0):
    """Tensors of these sizes (None: frozen), each `offset` elements off its allocation's
    alignment."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        if n is None:
            out.append(None)
            continue
        base = torch.full((n + offset + 9,), 7.0, dtype=dt, device=DEV)
        v = base[offset:offset + n]
        v.copy_((torch.randn(n, generator=g) * math.exp(i % 5 - 2)).to(dt))
        out.append(v)
    return out


def norm_of(sets, ws=None, norm=True):
    sumsq = torch.full((1,), float("nan"), dtype=torch.float64, device=DEV)
    nrm = torch.full((1,), float("nan"), device=DEV) if norm else None
    ws = torch.full((api.moe_grad_norm_workspace_size(),), 0xFF, dtype=torch.uint8, device=DEV) if ws is None else ws
    for i, s in enumerate(sets):
        api.moe_grad_norm(s, sumsq, nrm, ws, accumulate=i > 0)
    return sumsq, nrm


def check(ts, dt, over=3.0, out_offset=None, eps=1e-6):
    s = api.TensorSet(ts, dt)
    live = [t for t in ts if t is not None]
    host = [t.double().cpu().numpy() for t in live]
    want = O.grad_sumsq(host)
    sumsq, nrm = norm_of([s])
    n = sum(t.numel() for t in live)
    assert abs(sumsq.item() - want) <= max(n, 1) * 2.0 ** -52 * want
    assert abs(nrm.item() - math.sqrt(want)) <= (2.0 ** -24 + 1e-12) * math.sqrt(want)
    max_norm = np.float32(math.sqrt(want) / over)
    coef = O.clip_coefficient(want, float(max_norm), eps=float(np.float32(eps)))
    outs = ts
    if out_offset is not None:
        outs = tensors([None if t is None else t.numel() for t in ts], dt, 99, out_offset)
    before = [t.clone() for t in live]
    api.moe_grad_clip(s, sumsq, max_norm, out=None if out_offset is None else api.TensorSet(outs, dt), eps=eps)
    for t, o, b, h in zip(live, [o for o in outs if o is not None], before, host):
        if out_offset is not None:
            assert torch.equal(t, b)                       # the gradients are left as they were
        got = o.double().cpu().numpy()
        tol = (2.0 ** -23 + (2.0 ** -8 if dt is BF else 0)) * np.abs(h * coef) + (2.0 ** -133 if dt is BF else 2.0 ** -149)
        assert np.all(np.abs(got - h * coef) <= tol)
        # what lies around a result is left as it was
        base = o._base if o._base is not None else o
        off = o.storage_offset()
        assert bool((base[:off] == 7).all()) and bool((base[off + o.numel():] == 7).all())


SIZES = {
    "one_element": [1],
    "empty_tensors": [0, 5, 0, 0, 3, 0],
    "odd": [1, 2, 3, 7, 63, 64, 65, 1000, 4097],
    "frozen": [None, 100, None, None, 2049, None],
    "many_small": [i % 37 for i in range(700)],
    "many_of_one": [1] * 5000,
    "one_large": [3_000_001],
    "large_and_small": [5, 2_000_003, 17, 1_000_000, 1],
}


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("name", list(SIZES))
def test_norm_and_clip(name, dt):
    log(f"grads {name} {dt}")
    check(tensors(SIZES[name], dt), dt)
    check(tensors(SIZES[name], dt, 1), dt, out_offset=0)


@pytest.mark.parametrize("dt", [F32, BF])
@pytest.mark.parametrize("offset,out_offset", [(1, 0), (0, 1), (3, 3), (1, 2), (7, 5)])
def test_alignments(dt, offset, out_offset):
    """Tensors and results off their 16-byte boundaries, each by its own distance."""
    for sizes in ([1, 5, 70, 1030], [300_001, 9]):
        check(tensors(sizes, dt, 2, offset), dt, out_offset=out_offset)
        check(tensors(sizes, dt, 3, offset), dt)


@pytest.mark.parametrize("dt", [F32, BF])
def test_below_the_limit_nothing_changes(dt):
    ts = tensors([100, 3000], dt)
    before = [t.clone() for t in ts]
    s = api.TensorSet(ts)
    sumsq, nrm = norm_of([s])
    api.moe_grad_clip(s, sumsq, nrm.item() * 1.01)
    assert all(torch.equal(a, b) for a, b in zip(ts, before))
    out = [torch.empty_like(t) for t in ts]
    api.moe_grad_clip(s, sumsq, nrm.item() * 1.01, out=api.TensorSet(out))
    assert all(torch.equal(a, b) for a, b in zip(out, before))


def test_everything_frozen_or_empty():
    for ts in ([None, None], [torch.empty(0, device=DEV)]):
        s = api.TensorSet(ts, F32, device=DEV)
        sumsq, nrm = norm_of([s])
        assert sumsq.item() == 0 and nrm.item() == 0
        api.moe_grad_clip(s, sumsq, 1.0)
        api.moe_grad_clip(s, sumsq, 0.0, out=s, eps=0.0)
    ts = tensors([50], F32)                                # no norm is allowed: everything becomes 0
    s = api.TensorSet(ts)
    api.moe_grad_clip(s, norm_of([s])[0], 0.0)
    assert not ts[0].any()
    api.moe_grad_clip(s, norm_of([s])[0], 0.0, eps=0.0)    # 0 / 0: left alone
    assert not ts[0].any()


@pytest.mark.parametrize("value", [1e-30, 2.0 ** -149, 1e30, 3e38])
def test_squares_that_fp32_cannot_hold(value):
    t = torch.full((70_000,), value, device=DEV)
    sumsq, nrm = norm_of([api.TensorSet([t])])
    v = float(t[0])
    assert abs(sumsq.item() / (70_000 * v * v) - 1) < 1e-11
    want = min(math.sqrt(70_000) * v, float("inf"))
    assert nrm.item() == np.float32(want) or abs(nrm.item() / want - 1) < 2.0 ** -23


def test_infinities_and_nan():
    for bad, kept in ((float("inf"), 0.0), (float("nan"), float("nan"))):
        t = torch.ones(3000, device=DEV)
        t[1234] = bad
        s = api.TensorSet([t])
        sumsq, nrm = norm_of([s])
        assert nrm.isinf().item() if bad == float("inf") else nrm.isnan().item()
        api.moe_grad_clip(s, sumsq, 1.0)
        assert t[1234].isnan().item()
        rest = torch.cat((t[:1234], t[1235:]))
        assert bool((rest == 0).all()) if kept == 0.0 else bool(rest.isnan().all())
    t = torch.ones(3000, dtype=BF, device=DEV)
    t[5] = float("nan")
    s = api.TensorSet([t])
    api.moe_grad_clip(s, norm_of([s])[0], 1.0)
    assert bool(t.isnan().all())


def test_sets_add_up_and_norm_may_be_left_out():
    a, b = tensors([1000, 77], F32), tensors([5000], BF, 4)
    sumsq, nrm = norm_of([api.TensorSet(a), api.TensorSet(b)])
    want = O.grad_sumsq([t.double().cpu().numpy() for t in a + b])
    assert abs(sumsq.item() / want - 1) < 1e-12 and abs(nrm.item() / math.sqrt(want) - 1) < 2.0 ** -23
    assert torch.equal(norm_of([api.TensorSet(a), api.TensorSet(b)], norm=False)[0], sumsq)


def test_results_repeat_and_a_workspace_serves_calls_in_a_row():
    ts = tensors([1_000_003, 5], F32)
    s, small = api.TensorSet(ts), api.TensorSet(tensors([3], F32, 5))
    ws = torch.empty(api.moe_grad_norm_workspace_size(), dtype=torch.uint8, device=DEV)
    first = norm_of([s], ws)[0].clone()
    for _ in range(3):
        norm_of([small], ws)
        assert torch.equal(norm_of([s], ws)[0], first)


def test_past_32_bits():
    n = 2 ** 32 + 100_003                                  # bf16, 8.6 GB
    t = torch.zeros(n, dtype=BF, device=DEV)
    for at in (0, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, n - 1):
        t[at] = 2.0
    s = api.TensorSet([None, t, None])
    sumsq, nrm = norm_of([s])
    assert sumsq.item() == 24.0
    api.moe_grad_clip(s, sumsq, math.sqrt(24.0) / 2, eps=0.0)
    for at in (0, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, n - 1):
        assert t[at].item() == 1.0
    assert norm_of([s])[0].item() == 6.0


def test_two_graphs_and_another_stream():
    """Norm and clip captured twice, replayed with eager work between, each with its own
    workspace."""
    steps = []
    for seed, sizes in enumerate(([3000, None, 70_001], [5] * 300)):
        ts = tensors([n for n in sizes], F32, seed)
        out = [None if t is None else torch.empty_like(t) for t in ts]
        steps.append(dict(s=api.TensorSet(ts), to=api.TensorSet(out), out=[o for o in out if o is not None],
                          sumsq=torch.empty(1, dtype=torch.float64, device=DEV), norm=torch.empty(1, device=DEV),
                          ws=torch.empty(api.moe_grad_norm_workspace_size(), dtype=torch.uint8, device=DEV)))

    def run(s):
        api.moe_grad_norm(s["s"], s["sumsq"], s["norm"], s["ws"])
        api.moe_grad_clip(s["s"], s["sumsq"], 1.0, out=s["to"])
    want = []
    for s in steps:
        run(s)
        want.append([s["norm"].clone()] + [o.clone() for o in s["out"]])
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), []
    for s in steps:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            run(s)
        graphs.append(g)
    for _ in range(3):
        for s, g, w in zip(steps, graphs, want):
            for replay in (True, False):
                for o in s["out"]:
                    o.fill_(9.0)
                s["ws"].fill_(0xFF)
                torch.cuda.synchronize()
                if replay:
                    g.replay()
                else:
                    with torch.cuda.stream(side):
                        run(s)
                torch.cuda.synchronize()
                for a, b in zip([s["norm"]] + s["out"], w):
                    assert torch.equal(a, b)
