"""A fine-tuning step of a layer whose router scores by sigmoids or by a softmax over all
experts, as MoELayerRunner runs it: logits, routing, experts, combine, and back to the
experts', the router's and the input's gradients, their global norm and clipping, the
selection bias.  Against torch autograd in fp64 on the same selection.  fp32 throughout:
every product holds some 1e-6, the gradients' norms are held to 2e-5."""
import dataclasses

import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api
from paper_2508_19078_amd.layer import MoELayerRunner
from paper_2508_19078_amd.workloads import WORKLOADS

from gpu_harness import log

pytestmark = pytest.mark.gpu
GATINGS = {"sigmoid": dict(score="sigmoid", n_group=4, topk_group=2, group_top=2, scale=2.5), "softmax": dict(renorm=False)}


def runner(name, **over):
    w = dataclasses.replace(WORKLOADS["tiny"], dtype="f32", merge=None, n_shared=1, n_tune=None, **over)
    r = MoELayerRunner(w, gating=api.gating(w.E, w.k, **GATINGS[name]))
    r.merge(torch.ones(w.E, dtype=torch.int32, device="cuda"))
    return r


def rel(a, b):
    return float(((a.double() - b).norm() / b.norm()).detach())


@pytest.mark.parametrize("name", list(GATINGS))
def test_step_against_autograd(name):
    r = runner(name)
    w, how = r.w, GATINGS[name]
    r.sel_bias.copy_(0.2 * torch.randn(w.E, generator=torch.Generator().manual_seed(1)))
    bias0 = r.sel_bias.double().cpu().numpy()
    r.route()
    r.forward()
    r.backward(dgate=True)
    r.router_backward()
    torch.cuda.synchronize()
    grads = [r.dWg, r.dWu, r.dWd, r.dWr, r.dbias]
    d64 = lambda t: t.double().detach().clone().requires_grad_(True)  # noqa: E731
    X, Wr, bias = d64(r.X), d64(r.Wr), d64(r.bias)
    mats = [[d64(t) for t in stack] + [d64(t) for t in sh] for stack, sh in ((r.Wg, r.Sg), (r.Wu, r.Su), (r.Wd, r.Sd))]
    z = X @ Wr.T + bias
    want, wgate, key = O.route_scored(r.logits.cpu().numpy(), w.k, sel_bias=bias0, **how)
    assert np.array_equal(r.idx.cpu().numpy(), want)
    idx = r.idx.long()
    s = torch.sigmoid(z) if how.get("score") == "sigmoid" else torch.softmax(z, 1)
    sel = s.gather(1, idx)
    gate = how.get("scale", 1.0) * (sel / sel.sum(1, keepdim=True) if how.get("renorm", True) else sel)
    assert rel(r.gate, gate) < 1e-5

    def expert(x, e):
        a = x @ mats[0][e].T
        return (a * torch.sigmoid(a) * (x @ mats[1][e].T)) @ mats[2][e].T
    Y = expert(X, w.E)
    for e in range(w.E):
        t, j = (idx == e).nonzero(as_tuple=True)
        Y = Y.index_add(0, t, gate[t, j][:, None] * expert(X[t], e))
    assert rel(r.Y, Y.detach()) < 1e-5
    (Y * r.dY.double()).sum().backward()
    for got, ref in ((r.dX, X.grad), (r.dWr, Wr.grad), (r.dbias, bias.grad),
                     *((g, torch.stack([m.grad if m.grad is not None else torch.zeros_like(m) for m in ms]))
                       for g, ms in zip(grads, mats))):
        assert rel(got, ref) < 2e-5, rel(got, ref)
    # the norm of all of them, and what clipping leaves
    before = [g.clone() for g in grads]
    sumsq = O.grad_sumsq([g.double().cpu().numpy() for g in grads])
    norm = r.clip(float(np.sqrt(sumsq)) / 4)
    assert abs(norm.item() / np.sqrt(sumsq) - 1) < 1e-6
    for g, b in zip(grads, before):
        assert bool((g.double() - b.double() / 4).abs().max() <= 2.0 ** -22 * b.abs().max())
    n = r.load.cpu().numpy()
    assert np.array_equal(n, np.bincount(want.ravel(), minlength=w.E))
    r.balance(0.001)
    np.testing.assert_allclose(r.sel_bias.cpu().numpy(), O.bias_update(n, bias0, np.float32(0.001)), rtol=1e-6, atol=1e-9)
    assert not r.load.any()
    log(f"  scored step {name}: norm {norm.item():.4g}, load {n.min()} to {n.max()}")


def test_step_captured_and_replayed():
    r = runner("sigmoid")

    def step():
        r.load.zero_()
        r.route()
        r.forward()
        r.backward(dgate=True)
        r.router_backward()
        r.clip(0.5)
    step()
    torch.cuda.synchronize()
    outs = (r.idx, r.gate, r.Y, r.dX, r.dWg, r.dWd, r.dWr, r.dbias, r.norm, r.load)
    want = [t.clone() for t in outs]
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for _ in range(3):
        for t in outs:
            t.fill_(1)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for t, v in zip(outs, want):
            assert torch.equal(t, v)
        step()
        torch.cuda.synchronize()
        for t, v in zip(outs, want):
            assert torch.equal(t, v)


def test_gating_of_another_layer_is_refused():
    w = WORKLOADS["tiny"]
    with pytest.raises(ValueError, match="gating"):
        MoELayerRunner(w, gating=api.gating(w.E + 1, w.k))
