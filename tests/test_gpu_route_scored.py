"""GPU parity of the routing from scores, its gradient, the router's logits and the bias
update, against the fp64 oracle.

Selections and counts are exact: the library selects as keys in fp64 do, and so does the
oracle; inputs that tie do so exactly.  Gates: an exponential and its argument (up to
|z| half steps of it), a quotient and two sums of at most 256 terms, half a step of fp32
each: (48 + 2 max|z|) 2^-24 relative, the gradient the same relative to the sum of the
magnitudes it is a difference of."""
import itertools

import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

from gpu_harness import host, log

pytestmark = pytest.mark.gpu
DEV = "cuda"

CASES = {
    # name: (T, E, k, gating, selection bias)
    "one_token": (1, 16, 4, dict(), False),
    "one_expert": (7, 1, 1, dict(score="sigmoid"), True),
    "odd": (37, 60, 5, dict(renorm=False), False),
    "odd_experts": (19, 37, 3, dict(score="sigmoid", renorm=False, scale=-1.5), True),
    "softmax_bias": (130, 64, 6, dict(scale=2.5), True),
    "sigmoid_groups": (300, 64, 6, dict(score="sigmoid", n_group=8, topk_group=3), True),
    "sigmoid_groups_of_two_best": (301, 256, 8, dict(score="sigmoid", n_group=8, topk_group=4, group_top=2, scale=2.5), True),
    "softmax_groups_of_two_best": (65, 160, 6, dict(n_group=8, topk_group=3, group_top=2, renorm=False), False),
    "sigmoid_two_best_without_bias": (65, 128, 6, dict(score="sigmoid", n_group=16, topk_group=3, group_top=2), False),
    "groups_that_all_stay": (33, 96, 7, dict(n_group=4, topk_group=4, group_top=2), True),
    "all_experts": (16, 16, 16, dict(score="sigmoid"), True),
    "all_of_the_kept": (50, 48, 6, dict(n_group=16, topk_group=2, renorm=False), True),
    "most_groups": (64, 96, 4, dict(score="sigmoid", n_group=32, topk_group=31, group_top=1), True),
    "groups_of_one": (17, 32, 3, dict(n_group=32, topk_group=5), False),
    "most": (515, 256, 16, dict(score="sigmoid"), True),
}


def draw(T, E, bias, seed=0, spread=1.0):
    rng = np.random.default_rng([T, E, seed])
    z = (spread * (rng.standard_normal((T, E)) + rng.standard_normal(E))).astype(np.float32)
    return z, (0.1 * rng.standard_normal(E)).astype(np.float32) if bias else None


def cuda(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def route(g, z, b=None, keep=None, counts=None):
    T = len(z)
    idx = torch.full((T, g.k), -7, dtype=torch.int32, device=DEV)
    gate = torch.full((T, g.k), float("nan"), device=DEV)
    api.moe_route_scored(g, cuda(z), idx, gate, sel_bias=cuda(b), counts=counts, keep=cuda(keep))
    return idx, gate


def backward(g, z, idx, dg, accumulate_to=None):
    out = torch.full(z.shape, float("nan"), device=DEV) if accumulate_to is None else cuda(accumulate_to)
    api.moe_route_scored_bwd(g, cuda(z), cuda(idx.astype(np.int32)), cuda(dg), out, accumulate=accumulate_to is not None)
    return host(out).astype(np.float64)


def tolerance(z):
    f = np.abs(z[np.isfinite(z)])
    return (48 + 2 * (f.max() if f.size else 0)) * 2.0 ** -24


def check(z, b, k, how, keep=None):
    T, E = z.shape
    g = api.gating(E, k, **how)
    counts = torch.full((E,), 3, dtype=torch.int32, device=DEV)
    idx, gate = route(g, z, b, keep, counts)
    want, wgate, _ = O.route_scored(z, k, sel_bias=b, **how)
    np.testing.assert_array_equal(host(idx), want)
    rel = tolerance(z)
    assert np.all(np.abs(host(gate) - wgate) <= rel * np.abs(wgate) + 2.0 ** -149), np.abs(host(gate) - wgate).max()
    kept = want if keep is None else want[keep != 0]
    np.testing.assert_array_equal(host(counts), 3 + np.bincount(kept.ravel(), minlength=E))
    return g, want


def check_backward(g, z, idx, how, seed=0):
    rng = np.random.default_rng(seed)
    dg = rng.standard_normal(idx.shape).astype(np.float32)
    score, renorm, scale = how.get("score", "softmax"), how.get("renorm", True), how.get("scale", 1.0)
    want = O.route_scored_backward(z, idx, dg, score, renorm, scale)
    # magnitudes of what the gradient is a difference of
    s = O.scores(z, score)
    ok = (idx >= 0) & (idx < z.shape[1])
    at = np.where(ok, idx, 0)
    sel = np.take_along_axis(s, at, 1) * ok
    if renorm:
        share = np.abs(O.gates_of(np.where(ok, np.take_along_axis(z, at, 1), -np.inf), np.broadcast_to(np.arange(idx.shape[1]), idx.shape),
                                  score, True, 1.0))
    else:
        share = sel
    mag = np.zeros(z.shape)
    total = (share * np.abs(dg)).sum(1, keepdims=True)
    for j in range(idx.shape[1]):
        np.add.at(mag, (np.arange(len(z)), at[:, j]), abs(scale) * (share[:, j] * (np.abs(dg[:, j]) + total[:, 0])) * ok[:, j])
    if score == "softmax" and not renorm:
        mag += abs(scale) * s * total
    for acc in (None, rng.standard_normal(z.shape).astype(np.float32)):
        got = backward(g, z, idx, dg, acc)
        base = 0.0 if acc is None else acc.astype(np.float64)
        tol = 2 * tolerance(z) * mag + (0 if acc is None else 2.0 ** -24 * np.abs(base + want)) + 2.0 ** -140
        assert np.all(np.abs(got - base - want) <= tol), (np.abs(got - base - want) / tol).max()


@pytest.mark.parametrize("name", list(CASES))
def test_routing_and_gradient(name):
    T, E, k, how, bias = CASES[name]
    log(f"route_scored {name}")
    z, b = draw(T, E, bias)
    keep = (np.arange(T) % 3 != 1).astype(np.uint8)
    g, idx = check(z, b, k, how, keep)
    check_backward(g, z, idx, how)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("how", [dict(), dict(score="sigmoid", n_group=4, topk_group=2, group_top=2)])
def test_ties_go_to_the_lower_expert(how, bias):
    """bf16 logits and a bias of few values: many keys tie exactly."""
    z, _ = draw(200, 64, False)
    z = torch.from_numpy(z).to(torch.bfloat16).float().numpy()
    z[3], z[4, ::2] = 1.0, z[4, 0]
    z[5] = np.where(np.arange(64) % 2, 0.0, -0.0)
    b = np.where(np.arange(64) % 3, 0.25, 0.0).astype(np.float32) if bias else None
    check(z, b, 6, how)


@pytest.mark.parametrize("spread", [1e-7, 1e-5, 30.0, 300.0])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True])
def test_keys_that_fp32_cannot_tell_apart(score, bias, spread):
    """Scores within an fp32 step of each other, scores that vanish, saturated ones."""
    z, b = draw(96, 64, bias, 1, spread)
    how = dict(score=score, n_group=4, topk_group=2, group_top=2)
    if bias:
        b = b * np.float32(1e-7)
    # without a bias, groups of saturated scores tie in fp64 as in the oracle
    g, idx = check(z, b, 5, how)
    check_backward(g, z, idx, how)


def test_bias_whose_steps_are_as_large_as_scores():
    """Keys in fp32 are whole eighths here, and scores make up for the differences of the
    biases: their sums lie on both sides of a tie and round apart, either way."""
    rng = np.random.default_rng(0)
    for i, j in itertools.combinations(range(8), 2):
        at = np.array([i, j]) / 8
        s = 15 / 16 - at + 2.0 ** -25 * rng.uniform(-3, 3, (8192, 2))
        check(np.log(s / (1 - s)).astype(np.float32), (15938355 / 8 + at).astype(np.float32), 1, dict(score="sigmoid"))


@pytest.mark.parametrize("how", [dict(), dict(renorm=False), dict(score="sigmoid"), dict(score="sigmoid", renorm=False),
                                 dict(n_group=4, topk_group=2, group_top=2), dict(score="sigmoid", n_group=4, topk_group=2)])
@pytest.mark.parametrize("bias", [False, True])
def test_masked_logits(how, bias):
    z, b = draw(24, 32, bias, 2)
    inf, nan, low = np.inf, np.nan, np.finfo(np.float32).min
    z[0] = -inf                              # nothing left
    z[1] = nan
    z[2, 1:] = -inf                          # fewer than k left
    z[3, 2:] = low
    z[4, 5], z[4, 6], z[4, 7] = inf, inf, nan
    z[5] = inf
    z[6, ::2] = nan
    z[7] = low
    z[8, 3] = np.finfo(np.float32).max
    if bias:
        b[3], b[9], b[10] = -inf, nan, 2.0   # switched off
    g = api.gating(32, 4, **how)
    idx, gate = route(g, z, b)
    want, wgate, _ = O.route_scored(z, 4, sel_bias=b, **how)
    np.testing.assert_array_equal(host(idx), want)
    np.testing.assert_allclose(host(gate), wgate, rtol=1e-5, atol=1e-30)
    dg = np.random.default_rng(0).standard_normal(want.shape).astype(np.float32)
    got = backward(g, z, want, dg)
    wantd = O.route_scored_backward(z, want, dg, how.get("score", "softmax"), how.get("renorm", True), 1.0)
    np.testing.assert_allclose(got, wantd, rtol=1e-5, atol=1e-6)


def test_gradient_of_indices_that_a_caller_made():
    """An expert named twice or three times, entries outside the experts, a row of them."""
    z, _ = draw(6, 12, False)
    idx = np.array([[3, 3, 1], [5, -1, 5], [-1, 12, 99], [7, 7, 7], [0, 11, 2], [-2147483648, 4, 2147483647]])
    for how in (dict(), dict(renorm=False), dict(score="sigmoid"), dict(score="sigmoid", renorm=False, scale=0.5)):
        check_backward(api.gating(12, 3, **how), z, idx, how)


def test_gradient_over_its_logits():
    z, b = draw(70, 64, True)
    for how in (dict(score="sigmoid"), dict(renorm=False)):
        g = api.gating(64, 6, **how)
        idx, _ = route(g, z, b)
        dg = torch.randn(70, 6, generator=torch.Generator().manual_seed(0)).to(DEV)
        zd, apart = cuda(z), torch.empty(70, 64, device=DEV)
        api.moe_route_scored_bwd(g, zd, idx, dg, apart)
        api.moe_route_scored_bwd(g, zd, idx, dg, zd)
        assert torch.equal(zd, apart)


@pytest.mark.parametrize("T", [1, 3, 4, 15, 16, 17, 31, 33, 64, 1000, 17000])
def test_lengths(T):
    """Both sides of a block's tokens, and blocks that take several times as many; the
    outputs behind the last token stay as they were."""
    z, b = draw(T, 64, True)
    g = api.gating(64, 6, "sigmoid", 8, 3, 2, True, 2.5)
    idx = torch.full((T + 20, 6), -7, dtype=torch.int32, device=DEV)
    gate = torch.full((T + 20, 6), -7.0, device=DEV)
    counts = torch.zeros(64, dtype=torch.int32, device=DEV)
    api.moe_route_scored(g, cuda(z), idx[:T], gate[:T], sel_bias=cuda(b), counts=counts)
    want, wgate, _ = O.route_scored(z, 6, "sigmoid", 8, 3, 2, True, 2.5, b)
    np.testing.assert_array_equal(host(idx)[:T], want)
    assert np.all(np.abs(host(gate)[:T] - wgate) <= tolerance(z) * wgate)
    assert bool((idx[T:] == -7).all()) and bool((gate[T:] == -7).all())
    np.testing.assert_array_equal(host(counts), np.bincount(want.ravel(), minlength=64))
    out = torch.full((T + 20, 64), -7.0, device=DEV)
    dg = np.random.default_rng(T).standard_normal((T, 6)).astype(np.float32)
    api.moe_route_scored_bwd(g, cuda(z), idx[:T], cuda(dg), out[:T])
    np.testing.assert_allclose(host(out)[:T], O.route_scored_backward(z, want, dg, "sigmoid", True, 2.5), rtol=1e-4, atol=1e-6)
    assert bool((out[T:] == -7).all())


def test_past_32_bits():
    """2.2e9 logits: rows across element 2^31 and the last ones, of a repeated pattern."""
    E, k, base = 256, 8, 64
    T = 8_500_032
    z, b = draw(base, E, True)
    zd = cuda(z).repeat(T // base, 1)
    g = api.gating(E, k, "sigmoid", 8, 4, 2, True, 2.5)
    idx, gate = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    api.moe_route_scored(g, zd, idx, gate, sel_bias=cuda(b))
    want, _, _ = O.route_scored(z, k, "sigmoid", 8, 4, 2, True, 2.5, b)
    assert bool((idx.view(-1, base, k) == cuda(want.astype(np.int32))).all())
    assert bool((gate.view(-1, base, k) == gate[:base]).all())
    dg = torch.ones(T, k, device=DEV)
    dg[:, 0] = 2.0
    api.moe_route_scored_bwd(g, zd, idx, dg, zd)
    assert bool((zd.view(-1, base, E) == zd[:base]).all())
    np.testing.assert_allclose(host(zd[:base]), O.route_scored_backward(z, want, host(dg[:base]), "sigmoid", True, 2.5),
                               rtol=1e-4, atol=1e-6)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d,E,bias", [(1, 128, 16, False), (37, 136, 60, True), (300, 256, 64, True), (20000, 256, 8, False),
                                        (65, 264, 256, True)])
def test_router_logits(T, d, E, bias, dt):
    """The bits of moe_route_topk's logits, and the product: d + 1 roundings of fp32."""
    rng = np.random.default_rng([T, d, E])
    X = torch.from_numpy(rng.standard_normal((T, d)).astype(np.float32)).to(dt).to(DEV)
    Wr = torch.from_numpy((rng.standard_normal((E, d)) / np.sqrt(d)).astype(np.float32)).to(dt).to(DEV)
    b = cuda(rng.standard_normal(E).astype(np.float32)) if bias else None
    got, topk = (torch.full((T, E), float("nan"), device=DEV) for _ in range(2))
    api.moe_router_logits(X, Wr, b, got)
    k = min(2, E)
    api.moe_route_topk(X, Wr, b, k, torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV), topk)
    assert torch.equal(got, topk)
    x, w = host(X.double()), host(Wr.double())
    want = x @ w.T + (host(b) if bias else 0)
    assert np.all(np.abs(host(got) - want) <= (d + 1) * 2.0 ** -24 * (np.abs(x) @ np.abs(w).T + (np.abs(host(b)) if bias else 0)))


def test_bias_update():
    rng = np.random.default_rng(0)
    for E in (1, 3, 64, 65, 256):
        n = rng.integers(0, 2 ** 31 - 1, E).astype(np.int32)
        n[0] = 7
        if E == 3:
            n[:] = (5, 4, 6)               # the mean itself: not moved
        b = rng.standard_normal(E).astype(np.float32)
        bd = cuda(b)
        api.moe_route_bias_update(cuda(n), bd, 0.001)
        want = b + np.float32(0.001) * np.sign(int(n.astype(np.int64).sum()) - n.astype(np.int64) * E).astype(np.float32)
        np.testing.assert_array_equal(host(bd), want.astype(np.float32))


def test_two_graphs_and_another_stream():
    """A training step's calls captured twice, replayed with eager work between."""
    steps = []
    for seed, (T, E, k, how) in enumerate([(70, 64, 6, dict(score="sigmoid", n_group=8, topk_group=3)), (33, 60, 5, dict(renorm=False))]):
        z, b = draw(T, E, True, seed)
        s = dict(g=api.gating(E, k, **how), z=cuda(z), b=cuda(b), idx=torch.empty(T, k, dtype=torch.int32, device=DEV),
                 gate=torch.empty(T, k, device=DEV), counts=torch.zeros(E, dtype=torch.int32, device=DEV),
                 dg=torch.randn(T, k, device=DEV), dz=torch.empty(T, E, device=DEV))
        steps.append(s)

    def run(s):
        s["counts"].zero_()
        api.moe_route_scored(s["g"], s["z"], s["idx"], s["gate"], sel_bias=s["b"], counts=s["counts"])
        api.moe_route_scored_bwd(s["g"], s["z"], s["idx"], s["dg"], s["dz"])
    names = ("idx", "gate", "counts", "dz")
    want = []
    for s in steps:
        run(s)
        want.append([s[n].clone() for n in names])
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), []
    for s in steps:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=side):
            run(s)
        graphs.append(gr)
    for _ in range(3):
        for s, gr, w in zip(steps, graphs, want):
            for how in ("replay", "stream"):
                for n in names:
                    s[n].fill_(9)
                if how == "replay":
                    gr.replay()
                else:
                    side.wait_stream(torch.cuda.default_stream())
                    with torch.cuda.stream(side):
                        run(s)
                torch.cuda.synchronize()
                for n, v in zip(names, w):
                    assert torch.equal(s[n], v), n


SHIFTS = [-1e9, -3e7, -1000, -230, -120, -100, -60, -40, -33, -20, 20, 33, 40, 60, 100, 230, 1000, 3e7]
SHIFTED = {
    # name: (T, E, k, gating)
    "64_experts": (300, 64, 6, dict()),
    "odd_experts_plain": (90, 37, 3, dict(renorm=False)),
    "groups_of_two_best": (130, 160, 6, dict(n_group=8, topk_group=3, group_top=2)),
    "sigmoid_groups": (130, 128, 6, dict(score="sigmoid", n_group=8, topk_group=3)),
    "sigmoid_256_experts": (130, 256, 8, dict(score="sigmoid")),
    "many_tokens": (3000, 64, 6, dict()),
}


@pytest.mark.parametrize("name", list(SHIFTED))
@pytest.mark.parametrize("shift", SHIFTS)
def test_logits_far_from_zero(shift, name):
    """A softmax does not see a shift of its logits, and a window below the largest of them
    ends at a number that fp32 may have to round, to either side."""
    T, E, k, how = SHIFTED[name]
    z, _ = draw(T, E, False, 3)
    z = (z + np.float32(shift)).astype(np.float32)
    g, idx = check(z, None, k, how)
    check_backward(g, z, idx, how)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_logits_around_every_power_of_two(score):
    """Rows whose largest logit lies a few steps of fp32 to either side of a power of two, of
    either sign, or 32 above it; the others lie steps, ones and more than 32 below."""
    rng = np.random.default_rng(4)
    z = []
    for e in range(-20, 127):
        for base in (2.0 ** e, -2.0 ** e, 32 + 2.0 ** e, 32 - 2.0 ** e):
            for n in (-9, -1, 0, 1, 2, 40):
                top = np.float32(base)
                top = np.float32(top + n * np.spacing(np.abs(top)))
                below = np.concatenate((np.spacing(np.abs(top)) * np.arange(6), 2.0 ** rng.uniform(-18, 0, 6), np.arange(1, 13),
                                        32 + 2.0 ** rng.uniform(-20, 3, 8)))
                z.append(top - rng.permutation(below).astype(np.float32))
    check(np.stack(z).astype(np.float32), None, 4, dict(score=score, renorm=score == "softmax"))


@pytest.mark.parametrize("shift", [-1e6, -100, -15, -7.5, -5, -3.8, -3, -2, 2, 3, 3.8, 7.5, 100, 1e6])
@pytest.mark.parametrize("T,E,k,how", [(300, 64, 6, dict(score="sigmoid")), (130, 256, 8, dict(score="sigmoid", n_group=8, topk_group=4, group_top=2)),
                                       (130, 60, 5, dict(n_group=5, topk_group=2)), (130, 128, 4, dict(renorm=False))])
def test_biases_far_from_zero(T, E, k, how, shift):
    z, b = draw(T, E, True, 5)
    check(z, (b + np.float32(shift)).astype(np.float32), k, how)


@pytest.mark.parametrize("off", [-50, -1e3, -1e4, -1e5, -1e6, -1e7, -1e9])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,ks,how", [(64, (3, 6), dict(n_group=8, topk_group=3, group_top=2)), (256, (4, 8), dict(n_group=8, topk_group=4, group_top=2)),
                                      (128, (1, 4), dict(n_group=2, topk_group=1, group_top=2)), (64, (6, 14), dict(n_group=16, topk_group=4)),
                                      (60, (2, 5), dict(n_group=5, topk_group=2, group_top=2)), (48, (4, 5), dict(n_group=16, topk_group=5, group_top=2)),
                                      (256, (1, 8), dict(n_group=2, topk_group=1, group_top=2)), (48, (5, 11), dict(n_group=16, topk_group=4))])
def test_groups_with_experts_switched_off(E, ks, how, score, off):
    """One expert per group, or every expert of three groups, carries no bias and the others a
    large negative one: ranks hold keys whose steps are far larger than the largest key's.
    The choices end among the experts that are on, and reach those that are off.
    Scores lie about as close as those steps, so that fp32 ranks of different groups tie or
    change places."""
    how, n = dict(how, score=score), how["n_group"]
    rng = np.random.default_rng([E, n])
    b = np.full((n, E // n), off, dtype=np.float32)
    if how.get("group_top") == 2:
        b[np.arange(n), rng.integers(0, E // n, n)] = 0
    else:
        b[:3] = 0
    for steps in (0.5, 4, 64):
        spread = min(1.0, steps * abs(off) * 2.0 ** -23 * (4 if score == "sigmoid" else E))
        for k in ks:
            check((0.3 + spread * rng.standard_normal((1500, E))).astype(np.float32), b.ravel(), k, how)


@pytest.mark.parametrize("how", [dict(n_group=8, topk_group=3, group_top=2), dict(n_group=8, topk_group=3), dict(n_group=16, topk_group=9, group_top=2)])
def test_groups_with_biases_of_every_size(how):
    """Biases of both signs from 1e-3 to the largest of fp32, the type's lowest value and
    -inf among them; ranks that fp32 cannot hold."""
    rng = np.random.default_rng(6)
    low = np.finfo(np.float32).min
    for E in (64, 96, 256):
        for trial in range(12):
            b = np.exp(rng.uniform(-7, 86 if trial % 2 else 30, E)) * rng.choice((-1, -1, -1, 1), E)
            b[rng.random(E) < 0.3] = (low, -np.inf, 0, -3e38)[trial % 4]
            b[rng.random(E) < 0.2] = (0, low, low, -2.9e38)[trial % 4]
            z, _ = draw(150, E, False, trial, (1.0, 1e-6)[trial % 2])
            with np.errstate(over="ignore"):
                check(z, b.astype(np.float32), 6, dict(how, score=("sigmoid", "softmax")[trial // 2 % 2]))


def test_groups_masked_by_the_lowest_value():
    """Whole groups off by the type's lowest value: one rank that fp32 cannot hold, or that
    ties with others."""
    z, _ = draw(400, 64, False, 7)
    b = np.zeros((8, 8), dtype=np.float32)
    b[[1, 2, 4, 5, 6]] = np.finfo(np.float32).min
    for kept in (2, 3, 4):
        for top in (1, 2):
            check(z, b.ravel(), 6, dict(score="sigmoid", n_group=8, topk_group=kept, group_top=top))
