"""The operators around the MoE layer run together, as a fine-tuning step of one
residual block uses them, against torch autograd in fp64.

    N1 = norm(X) w1                                   moe_sublayer_norm
    idx, g = topk(N1 Wr^T + b)                        moe_route_topk
    aux = balance loss of the logits                  moe_balance_loss
    Y = combine of the experts on N1                  moe_permute .. moe_unpermute
    S = alpha X + r (norm(Y) w2), N2 = norm(S) w3     moe_sublayer_norm
    L = <N2, C> + <S, D> + aux

and back to every gradient: the block's input, the three gains, the residual gate, the
router's weight and bias, the tuned experts' matrices.  fp32 throughout.  Every
operator holds some 1e-6 of its own sums; over the chain (two norms, three products,
softmax) the gradients' norms are held to 2e-5.  The selection is taken from
the GPU in both; no token's k-th gap is below 1e-4 in these draws.

The same block once more with its experts in 4 bits (a frozen participant's
forward), eager and captured."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

from gpu_harness import log

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Block:
    def __init__(self, T, d, E, k, I, sh, dt, seg, seed=0):
        g = torch.Generator().manual_seed(seed)
        n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        S = E + sh
        self.T, self.d, self.E, self.k, self.I, self.sh, self.dt = T, d, E, k, I, sh, dt
        put = lambda t, ty=torch.float32: t.to(ty).to(DEV)  # noqa: E731
        self.X, self.C, self.D = (put(n(T, d), dt) for _ in range(3))
        self.Wr, self.bias = put(n(E, d) / d ** 0.5, dt), put(0.1 * n(E))
        self.w1, self.w2, self.w3 = (put(1 + 0.1 * n(d)) for _ in range(3))
        self.res = put(torch.rand(T, generator=g) + 0.5)
        self.wg, self.wu, self.wd = put(n(S, I, d) / d ** 0.5, dt), put(n(S, I, d) / d ** 0.5, dt), put(n(S, d, I) / I ** 0.5, dt)
        self.seg, self.alpha, self.coef = put(torch.tensor(seg), torch.int32), 0.9, 0.05
        self.keep = put((torch.rand(T, generator=g) > 0.2), torch.uint8)
        e = lambda *s, t=dt: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
        f, i32, B, R = torch.float32, torch.int32, len(seg) - 1, T * (k + sh)
        self.N1, self.S, self.N2, self.Y, self.dX, self.dN1, self.dY = (e(T, d) for _ in range(7))
        self.r1, self.r2, self.ry, self.dres = (e(T, t=f) for _ in range(4))
        self.idx, self.gate, self.logits = e(T, k, t=i32), e(T, k, t=f), e(T, E, t=f)
        self.counts, self.dprob, self.loss, self.dl = e(B, E, t=i32), e(B, E, t=f), e(1, t=f), e(T, E, t=f)
        self.offsets, self.tok, self.pg, self.inv = e(E + 1, t=i32), torch.zeros(T * k, dtype=i32, device=DEV), e(T * k, t=f), e(T, k, t=i32)
        self.Xp, self.O, self.dO, self.dXp = e(T * k, d), e(R, d), e(R, d), e(R, d)
        self.Ag, self.Au, self.H = e(R, I), e(R, I), e(R, I)
        self.dWg, self.dWu, self.dWd = (torch.zeros_like(w, dtype=f) for w in (self.wg, self.wu, self.wd))
        self.tuned = [s for s in range(S) if s % 3 != 1]                    # some experts are frozen
        dw = lambda t: [t[s] if s in self.tuned else None for s in range(S)]  # noqa: E731
        self.tab = api.LayerTables(d, I, dt, E, sh, list(self.wg), list(self.wu), list(self.wd), dw(self.dWg), dw(self.dWu), dw(self.dWd))
        q = {}
        for name, w in (("g", self.wg), ("u", self.wu), ("d", self.wd)):
            cs, ss = api.mxfp4_shapes(w.shape[1], w.shape[2])
            codes, scale = e(S, *cs, t=torch.uint8), e(S, *ss, t=torch.uint8)
            api.moe_quantize_mxfp4(w.view(-1, w.shape[2]), codes.view(-1, cs[1]), scale.view(-1, ss[1]))
            q[name] = codes, scale
        self.tab4 = api.LayerTablesMX4(d, I, E, sh, *(list(q[m][0]) for m in "gud"), *(list(q[m][1]) for m in "gud"))
        self.q = q
        size = max(api.moe_permute_workspace_size(T, k, E), api.moe_grouped_swiglu_fwd_workspace_size(self.tab, T, k),
                   api.moe_balance_loss_workspace_size(T, E, B), api.moe_router_bwd_workspace_size(T, d, E),
                   api.moe_sublayer_norm_bwd_workspace_size(T, d), api.moe_grouped_swiglu_fwd_mx4_workspace_size(self.tab4, T, k))
        self.ws = e(size, t=torch.uint8)                                    # one for every call but the products' backward
        self.ws_bwd = e(api.moe_grouped_swiglu_bwd_workspace_size(self.tab, T, k), t=torch.uint8)
        self.dWr, self.dbias, self.dw1, self.dw2, self.dw3 = e(E, d, t=f), e(E, t=f), e(d, t=f), e(d, t=f), e(d, t=f)

    def forward(self, four_bit=False):
        T, k, E = self.T, self.k, self.E
        api.moe_sublayer_norm(self.X, None, None, self.N1, w_pre=self.w1, rstd_s=self.r1)
        api.moe_route_topk(self.N1, self.Wr, self.bias, k, self.idx, self.gate, self.logits)
        api.moe_balance_loss(self.logits, self.idx, self.coef, self.counts, self.dprob, self.loss, self.ws, seg=self.seg, keep=self.keep)
        api.moe_permute(self.N1, self.idx, self.gate, None, E, self.offsets, self.tok, self.pg, self.inv, self.Xp, self.ws)
        if four_bit:
            api.moe_grouped_swiglu_fwd_mx4(self.tab4, self.N1, self.tok, self.offsets, T, k, self.O, self.ws)
        else:
            api.moe_grouped_swiglu_fwd(self.tab, self.N1, self.Xp, self.offsets, T, k, self.Ag, self.Au, self.H, self.O, self.ws)
        api.moe_unpermute(self.tab, self.O, self.inv, self.pg, T, k, self.Y)
        api.moe_sublayer_norm(self.X, self.Y, self.S, self.N2, alpha=self.alpha, gate=self.res, w_post=self.w2, w_pre=self.w3,
                              rstd_y=self.ry, rstd_s=self.r2)

    def backward(self):
        T, k = self.T, self.k
        api.moe_sublayer_norm_bwd(self.D, self.C, self.S, self.Y, self.r2, self.dX, self.dY, self.ws, alpha=self.alpha,
                                  rstd_y=self.ry, gate=self.res, w_post=self.w2, w_pre=self.w3, dgate=self.dres,
                                  dw_post=self.dw2, dw_pre=self.dw3)
        dgate = torch.empty(T, k, device=DEV)
        api.moe_unpermute_bwd(self.tab, self.dY, self.O, self.inv, self.offsets, self.pg, T, k, self.dO, dgate)
        api.moe_grouped_swiglu_bwd(self.tab, self.N1, self.Xp, self.offsets, T, k, self.Ag, self.Au, self.H, self.dO, self.dXp, False, self.ws_bwd)
        api.moe_permute_bwd(self.tab, self.dXp, self.inv, T, k, self.dN1)
        api.moe_balance_loss_bwd(self.logits, self.dprob, None, self.dl, seg=self.seg, keep=self.keep, gate=self.gate, idx=self.idx, dgate=dgate)
        api.moe_router_bwd(self.dl, self.N1, self.Wr, self.ws, dX=self.dN1, dWr=self.dWr, dbias=self.dbias, accumulate_dx=True)
        # the stream's share is already in dX: the pre-norm's adds to it
        api.moe_sublayer_norm_bwd(self.dX, self.dN1, self.X, None, self.r1, self.dX, None, self.ws, w_pre=self.w1,
                                  post_norm=False, dw_pre=self.dw1)


def reference(b, idx):
    """The block in torch fp64 with leaves for every gradient, the selection given."""
    leaf = {n: getattr(b, n).double().cpu().requires_grad_() for n in ("X", "Wr", "bias", "w1", "w2", "w3", "res", "wg", "wu", "wd")}
    norm = lambda v: torch.nn.functional.rms_norm(v, (b.d,), eps=1e-6)  # noqa: E731
    X = leaf["X"]
    N1 = norm(X) * leaf["w1"]
    z = N1 @ leaf["Wr"].T + leaf["bias"]
    g = torch.softmax(torch.gather(z, 1, idx), 1)
    ffn = lambda v, s: (torch.nn.functional.silu(v @ leaf["wg"][s].T) * (v @ leaf["wu"][s].T)) @ leaf["wd"][s].T  # noqa: E731
    Y = sum(((g * (idx == e)).sum(1, keepdim=True) * ffn(N1, e) for e in range(b.E)), torch.zeros_like(X))
    Y = Y + sum(ffn(N1, b.E + i) for i in range(b.sh))
    S = b.alpha * X + leaf["res"][:, None] * norm(Y) * leaf["w2"]
    N2 = norm(S) * leaf["w3"]
    p, keep, seg, aux = torch.softmax(z, 1), b.keep.cpu().bool(), b.seg.tolist(), 0.0 * X.sum()
    n = sum(int(keep[i:j].sum()) for i, j in zip(seg, seg[1:]))
    for i, j in zip(seg, seg[1:]):
        m = keep[i:j]
        if m.any():
            f = torch.bincount(idx[i:j][m].flatten(), minlength=b.E).double() / (int(m.sum()) * b.k)
            aux = aux + b.coef * int(m.sum()) / n * b.E * (f * p[i:j][m].mean(0)).sum()
    L = (N2 * b.C.double().cpu()).sum() + (S * b.D.double().cpu()).sum() + aux
    L.backward()
    return leaf, dict(N1=N1, S=S, N2=N2, Y=Y, loss=aux.reshape(1)), z


@pytest.mark.parametrize("T,d,E,k,I,sh,seg", [(70, 64, 8, 2, 48, 1, (0, 20, 20, 66)), (1, 40, 4, 1, 24, 0, (0, 1)),
                                              (333, 136, 12, 4, 72, 2, (0, 100, 333))])
def test_training_step(T, d, E, k, I, sh, seg):
    b = Block(T, d, E, k, I, sh, torch.float32, seg)
    b.forward()
    b.backward()
    torch.cuda.synchronize()
    idx = b.idx.long().cpu()
    leaf, out, z = reference(b, idx)
    gap = O.topk_gap(z.detach().numpy(), k)
    assert np.array_equal(np.sort(O.topk_select(z.detach().numpy(), k), 1), np.sort(idx.numpy(), 1)) and gap.min() > 1e-4
    rel = lambda a, r: float((a.double().cpu() - r).norm() / (r.norm() if r.any() else 1.0))  # noqa: E731
    err = {n: rel(getattr(b, n), v.detach()) for n, v in out.items()}
    dwt = dict(wg=b.dWg, wu=b.dWu, wd=b.dWd)
    err.update({"d" + n: rel(getattr(b, "d" + n), leaf[n].grad) for n in ("X", "Wr", "bias", "w1", "w2", "w3", "res")})
    err.update({"d" + n: rel(dwt[n][b.tuned], leaf[n].grad[b.tuned]) for n in dwt})
    log("  " + ", ".join(f"{n} {e:.1e}" for n, e in err.items()))
    assert all(e < 2e-5 for e in err.values()), err
    frozen = [s for s in range(E + sh) if s not in b.tuned]
    assert not any(dwt[n][frozen].any() for n in dwt)


def test_step_captured_and_replayed():
    b = Block(200, 128, 8, 2, 64, 1, torch.bfloat16, (0, 50, 180))

    def step():
        b.forward()
        b.backward()
    names = ("N1", "S", "N2", "counts", "dprob", "loss", "dl", "dX", "dWr", "dbias", "dw1", "dw2", "dw3", "dres", "dWg", "dWd")
    step()
    torch.cuda.synchronize()
    want = {n: getattr(b, n).clone() for n in names}
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        for n in names:
            if n not in ("dWg", "dWd"):                 # frozen experts' rows are not written
                getattr(b, n).fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(b, n), want[n]) for n in names)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(getattr(b, n), want[n]) for n in names)


def test_forward_with_4_bit_experts():
    """bf16 block, experts in 4 bits: the stream against the oracle's 4-bit experts on
    the GPU's own N1 (roundings to bf16 of the rows, their sum, Y's norm and S: 1e-2 of
    the norm)."""
    b = Block(150, 128, 8, 2, 96, 1, torch.bfloat16, (0, 150))
    b.forward(four_bit=True)
    torch.cuda.synchronize()
    N1, idx, gate = b.N1.double().cpu().numpy(), b.idx.cpu().numpy(), b.gate.double().cpu().numpy()
    deq = lambda w: O.mxfp4_round(w.double().cpu().numpy())  # noqa: E731
    Y = np.zeros((b.T, b.d))
    for s in range(b.E + b.sh):
        t, j = np.nonzero(idx == s) if s < b.E else (np.arange(b.T), None)
        if len(t):
            o = O.swiglu_mx4_fwd(N1[t], deq(b.wg[s]), deq(b.wu[s]), deq(b.wd[s]))[1]
            Y[t] += o if j is None else gate[t, j][:, None] * o
    S, _ = O.sublayer_norm(b.X.double().cpu().numpy(), Y, b.res.double().cpu().numpy(), b.w2.double().cpu().numpy(), None, b.alpha)
    rel = np.linalg.norm(b.S.double().cpu().numpy() - S) / np.linalg.norm(S)
    log(f"  4-bit block: stream rel err {rel:.2e}")
    assert rel < 1e-2
    want = b.S.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.forward(four_bit=True)
    for _ in range(3):
        b.S.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.S, want)
        b.forward()
        torch.cuda.synchronize()
