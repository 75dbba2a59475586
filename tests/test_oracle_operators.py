"""CPU pins of the oracle's 4-bit rows, balance loss, dense router backward and
sublayer norms: hand-worked values, torch autograd in fp64 and central
differences."""
import numpy as np
import pytest
import torch

import oracle as O


# ------------------------------------------------------------- 4-bit rows ----

def test_mxfp4_hand_worked_block():
    # largest magnitude 7: 2^2 <= 7 < 2^3, scale 2^0; ties go to the even code
    x = np.zeros(32)
    x[:20] = [7, 6, 5, 5.0001, 4, 3.5, 3.4999, 2.5, 2.5001, 1.75, 1.25, 0.75, 0.25, 0.2501, -0.25, -0.75, -5, -7, 0.5,
              -0.0]
    codes, byte = O.mxfp4_rows(x[None])
    assert byte.tolist() == [[127]]
    want = [6, 6, 4, 6, 4, 4, 3, 2, 3, 2, 1, 1, 0, 0.5, 0, -1, -4, -6, 0.5, 0]
    np.testing.assert_array_equal(O.mxfp4_values(codes, byte)[0, :20], want)
    assert codes[0, 19] == 8 and codes[0, 20] == 0 and codes[0, 14] == 8
    # the same block times a power of two has the same codes
    for e in (-60, 3, 90):
        c2, b2 = O.mxfp4_rows(x[None] * 2.0 ** e)
        assert np.array_equal(c2, codes) and b2[0, 0] == 127 + e


def test_mxfp4_blocks_edges_and_error():
    rng = np.random.default_rng(0)
    W = rng.standard_normal((50, 72)) * np.exp(rng.standard_normal((50, 1)) * 3)
    W[3] = 0
    W[4, :32] = 2.0 ** -149                       # below the smallest scale: all codes 0
    codes, byte = O.mxfp4_rows(W)
    assert byte.shape == (50, 3) and byte[3].max() == 0 and byte[4, 0] == 0
    V = O.mxfp4_values(codes, byte)
    assert not V[3].any() and not V[4, :32].any()
    # half the widest step (2, above 4) of the block's scale, or the cut above 6
    s = np.repeat(np.exp2(byte.astype(float) - 127), 32, axis=1)[:, :72]
    assert np.all(np.abs(V - W) <= np.where(np.abs(W) > 6 * s, np.abs(W) - 6 * s, s) * (1 + 1e-12))
    top = np.abs(W[:, :32]).max(axis=1)
    ok = byte[:, 0] > 0
    assert np.all((top[ok] / s[ok, 0] >= 4) & (top[ok] / s[ok, 0] < 8))
    np.testing.assert_array_equal(O.mxfp4_round(V), V)      # values are kept


def test_swiglu_mx4_on_representable_inputs_is_the_plain_one():
    rng = np.random.default_rng(1)
    x = O.mxfp4_round(rng.standard_normal((6, 40)))
    wg, wu = (O.mxfp4_round(rng.standard_normal((32, 40))) for _ in range(2))
    wd = np.zeros((5, 32))
    wd[np.arange(5), np.arange(5)] = 1.0
    H, Y = O.swiglu_mx4_fwd(x, wg, wu, wd)
    np.testing.assert_allclose(H, torch.nn.functional.silu(torch.tensor(x @ wg.T)).numpy() * (x @ wu.T), rtol=1e-12,
                               atol=1e-12)
    np.testing.assert_array_equal(Y, O.mxfp4_round(H)[:, :5])


# ----------------------------------------------------------- balance loss ----

def torch_loss(z, idx, k, coef, seg, keep):
    """The loss by its definition in torch fp64, choices fixed."""
    p = torch.softmax(z, 1)
    E, loss = z.shape[1], 0.0
    n = sum(int(keep[seg[b]:seg[b + 1]].sum()) for b in range(len(seg) - 1))
    for b in range(len(seg) - 1):
        m = keep[seg[b]:seg[b + 1]]
        if m.any():
            f = torch.bincount(idx[seg[b]:seg[b + 1]][m].flatten(), minlength=E).double() / (int(m.sum()) * k)
            loss = loss + coef * int(m.sum()) / n * E * (f * p[seg[b]:seg[b + 1]][m].mean(0)).sum()
    return loss


@pytest.mark.parametrize("seg,pad", [((0, 12), 0.0), ((0, 0, 5, 5, 11), 0.3)])
def test_balance_loss_and_gradient_by_autograd(seg, pad):
    rng = np.random.default_rng(2)
    T, E, k = 12, 5, 2
    z = rng.standard_normal((T, E)) * 2
    idx = np.argsort(-z, axis=1)[:, :k]
    keep = rng.random(T) >= pad
    counts, dprob, loss = O.balance_loss(z, idx, k, 0.03, seg, keep)
    zt = torch.tensor(z, requires_grad=True)
    want = torch_loss(zt, torch.tensor(idx), k, 0.03, seg, torch.tensor(keep))
    assert abs(loss - want.item()) < 1e-14
    assert counts.sum() == k * keep[seg[0]:seg[-1]].sum()
    want.backward()
    got = O.balance_loss_backward(z, dprob, 1.0, seg, keep)
    np.testing.assert_allclose(got, zt.grad.numpy(), rtol=0, atol=1e-15)
    assert not got[seg[-1]:].any() and not got[~keep].any()
    # differences of the loss itself, with the gates' share beside it
    gate, dg = rng.random((T, k)), rng.standard_normal((T, k))
    both = O.balance_loss_backward(z, dprob, 2.0, seg, keep, gate, idx, dg)
    share = O.route_topk_backward(np.eye(E), idx, gate, dg)[0]
    np.testing.assert_allclose(both, 2.0 * got + share, rtol=0, atol=1e-14)
    h = 1e-6
    for t, e in ((0, 1), (4, 3), (10, 0)):
        zp, zm = z.copy(), z.copy()
        zp[t, e] += h
        zm[t, e] -= h
        diff = (O.balance_loss(zp, idx, k, 0.03, seg, keep)[2] - O.balance_loss(zm, idx, k, 0.03, seg, keep)[2]) / (2 * h)
        assert abs(diff - got[t, e]) < 1e-9


def test_balance_loss_special_rows():
    # even choices and probabilities: the loss is coef
    z = np.zeros((8, 4))
    idx = (np.arange(8)[:, None] + np.arange(2)) % 4
    assert abs(O.balance_loss(z, idx, 2, 0.5)[2] - 0.5) < 1e-15
    # a row of -inf has no probabilities, its choices count; outside choices do not
    z = np.zeros((2, 3))
    z[0] = -np.inf
    counts, dprob, loss = O.balance_loss(z, np.array([[0], [7]]), 1, 1.0)
    assert counts.tolist() == [[1, 0, 0]] and abs(loss - 3 * 0.5 * (1 / 3) / 2) < 1e-15
    assert not O.balance_loss_backward(z, dprob, 1.0)[0].any()
    # nothing kept
    counts, dprob, loss = O.balance_loss(z, np.zeros((2, 1), int), 1, 1.0, keep=np.zeros(2))
    assert loss == 0 and not dprob.any() and not counts.any()


# ------------------------------------------------------------------ norms ----

@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("plain", [True, False])
def test_sublayer_norm_and_gradients_by_autograd(post, plain):
    rng = np.random.default_rng(3)
    T, d, eps, alpha = 5, 12, 1e-3, 1.5
    X, Y = rng.standard_normal((2, T, d))
    gate, w_post, w_pre = (None,) * 3 if plain else (rng.random(T), rng.standard_normal(d), rng.standard_normal(d))
    dS, dN = rng.standard_normal((2, T, d))
    tt = {n: torch.tensor(v, requires_grad=True) for n, v in
          dict(X=X, Y=Y, gate=gate, w_post=w_post, w_pre=w_pre).items() if v is not None}
    u = torch.nn.functional.rms_norm(tt["Y"], (d,), eps=eps) if post else tt["Y"]
    v = u * tt.get("w_post", 1.0)
    St = alpha * tt["X"] + (tt["gate"][:, None] if not plain else 1.0) * v
    Nt = torch.nn.functional.rms_norm(St, (d,), eps=eps) * tt.get("w_pre", 1.0)
    S, N = O.sublayer_norm(X, Y, gate, w_post, w_pre, alpha, post, eps)
    np.testing.assert_allclose(S, St.detach().numpy(), rtol=1e-13, atol=1e-13)
    np.testing.assert_allclose(N, Nt.detach().numpy(), rtol=1e-13, atol=1e-13)
    ((St * torch.tensor(dS)).sum() + (Nt * torch.tensor(dN)).sum()).backward()
    rs = 1 / np.sqrt((S * S).mean(1) + eps)
    ry = 1 / np.sqrt((Y * Y).mean(1) + eps) if post else None
    got = O.sublayer_norm_backward(dS, dN, S, Y, rs, ry, gate, w_post, w_pre, alpha)
    for n, g in dict(X="dX", Y="dY", gate="dgate", w_post="dw_post", w_pre="dw_pre").items():
        if n in tt:
            np.testing.assert_allclose(got[g], tt[n].grad.numpy(), rtol=1e-11, atol=1e-11)


def test_sublayer_norm_without_a_block_and_zero_rows():
    X = np.random.default_rng(4).standard_normal((3, 8))
    X[1] = 0
    S, N = O.sublayer_norm(X, None, eps=0.0, alpha=2.0)
    np.testing.assert_array_equal(S, 2 * X)
    np.testing.assert_allclose(N, O.rms_norm_rows(X, 0.0), rtol=1e-13, atol=0)
    assert not N[1].any()


def test_stack_with_4_bit_experts():
    """Representable weights and one layer: the stack's update equals the 4-bit
    experts called by hand; int8 experts give another one."""
    rng = np.random.default_rng(5)
    T, d, E, k, I = 9, 32, 4, 2, 32
    lay = dict(Wr=rng.standard_normal((E, d)), bias=np.zeros(E),
               wg=O.mxfp4_round(rng.standard_normal((E * I, d))).reshape(E, I, d),
               wu=O.mxfp4_round(rng.standard_normal((E * I, d))).reshape(E, I, d),
               wd=O.mxfp4_round(rng.standard_normal((E * d, I))).reshape(E, d, I))
    X0 = rng.standard_normal((T, d))
    counts, idx, gate, Xs = O.quantized_stack_profile(X0, [lay], k, experts="mxfp4")
    Xn = O.rms_norm_rows(X0)
    want = X0.copy()
    for t in range(T):
        for j in range(k):
            e = idx[0][t, j]
            want[t] += gate[0][t, j] * O.swiglu_mx4_fwd(Xn[t:t + 1], lay["wg"][e], lay["wu"][e], lay["wd"][e])[1][0]
    np.testing.assert_allclose(Xs[1], want, rtol=1e-12, atol=1e-12)
    c8, i8, _, X8 = O.quantized_stack_profile(X0, [lay], k)
    assert np.array_equal(c8[0], counts[0]) and np.abs(X8[1] - want).max() > 1e-3
