"""The kernels behind moe_grouped_swiglu_fwd_mx4, each at the sizes where it can go
wrong: the ones for a few tokens, the 256-row tiles (with their 128-row form) and both
sides of the rules between them.  A case names the path it is there for and asks the
library's own rule (fm::mx4_tile), so that a retuned rule does not leave it on another.

Formulas, exclusions and tolerances as in test_gpu_mxfp4: rows of which an element of H
lies next to a border of its rounding are left out, counted and bounded.  The bound of
a fifth is met by the oracle's own count, which does not depend on the GPU."""
import ctypes

import numpy as np
import pytest
import torch

import oracle as O
from paper_2508_19078_amd import api

import test_gpu_mxfp4 as M
from gpu_harness import log

DEV = "cuda"
FEW, SMALL, LARGE = 0, 128, 256


def path(T, d, E, k, I, sh):
    f = getattr(api.lib(), "_ZN2fm8mx4_tileEPK13moe_layer_mx4ii")   # fm::mx4_tile(const moe_layer_mx4*, int, int)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_int, ctypes.c_int]
    L = api.moe_layer_mx4(d, I, E, sh, *[None] * 6)
    return f(ctypes.addressof(L), T, k)


# ------------------------------------------------------------- a few tokens ----

FEW_CASES = {
    # name: (T, d, E, k, I, shared, experts drawn from)
    "one_token": (1, 4096, 6, 2, 688, 0, 6),                  # I ends inside a 128-block, k split over idle waves too
    "two_tokens_on_one_expert": (2, 4096, 2, 1, 264, 0, 1),
    "ragged_ends_and_empty_slots": (3, 1048, 5, 2, 1032, 1, 3),   # d and I end inside a 32-block
    "many_empty_slots": (3, 1032, 70, 2, 1024, 0, 70),        # the slots' ballot goes round twice
    "seven_tokens_shared_alone": (7, 2056, 0, 1, 520, 2, 0),
    "eight_tokens_on_all": (8, 4096, 8, 8, 264, 0, 8),
    "eight_tokens": (8, 1048, 4, 2, 1032, 2, 3),
    "one_expert": (8, 1032, 1, 1, 1024, 0, 1),
}
# both sides of a limit of the rule
LIMITS = [
    ((8, 1032, 3, 1, 1024, 0, 3), FEW), ((9, 1032, 3, 1, 1024, 0, 3), SMALL),          # tokens
    ((2, 264, 8, 4, 4096, 0, 4), SMALL), ((2, 264, 2, 2, 4096, 0, 2), FEW),            # slots times I / 8
    ((8, 8, 2, 1, 8, 0, 2), FEW), ((9, 8, 2, 1, 8, 0, 2), SMALL),                      # below every block
    ((8, 9216, 2, 1, 120, 1, 2), FEW), ((8, 13824, 2, 1, 120, 1, 2), SMALL),           # rows in LDS
]


def test_paths():
    for name, case in FEW_CASES.items():
        assert path(*case[:6]) == FEW, name
    for case, want in LIMITS:
        assert path(*case[:6]) == want, case
    for name, (T, d, E, k, I, sh, _) in LARGE_CASES.items():
        assert path(T, d, E, k, I, sh) == LARGE, name


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(FEW_CASES))
def test_few_tokens(name):
    T, d, E, k, I, sh, _ = case = FEW_CASES[name]
    assert path(*case[:6]) == FEW
    X, w, offsets, tok = M.draw(*case)
    got = M.run(M.tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    M.check(got, X, w, offsets, tok, T, d, E, k, I, sh)


@pytest.mark.gpu
@pytest.mark.parametrize("case,want", LIMITS, ids=["-".join(map(str, c)) for c, _ in LIMITS])
def test_both_sides_of_the_rule(case, want):
    T, d, E, k, I, sh, _ = case
    assert path(*case[:6]) == want
    X, w, offsets, tok = M.draw(*case)
    got = M.run(M.tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    M.check(got, X, w, offsets, tok, T, d, E, k, I, sh)


@pytest.mark.gpu
def test_few_tokens_more_rows_than_tokens():
    """Merged experts: a token may choose a slot several times.  Rows that no slot holds
    are left as they were."""
    T, d, E, k, I = 8, 1032, 3, 4, 1024
    X, w, _, _ = M.draw(T, d, E, 1, I, 0, E)
    offsets = np.array([0, 0, 27, 29])
    tok = np.concatenate((np.sort(np.arange(27) % T), [1, 6], np.zeros(3, dtype=np.int64)))
    assert path(T, d, E, k, I, 0) == FEW
    got = M.run(M.tables(w, d, E, k, I, 0), X, offsets, tok, T, k, 0, d)
    M.check(got, X, w, offsets, tok, T, d, E, k, I, 0)
    assert bool((got[29:] == 7.0).all())


@pytest.mark.gpu
def test_few_tokens_with_numbers_that_are_none():
    T, d, E, k, I, sh = 6, 1048, 3, 2, 1032, 1
    assert path(T, d, E, k, I, sh) == FEW
    X, w, offsets, tok = M.draw(T, d, E, k, I, sh, E)
    tab = M.tables(w, d, E, k, I, sh)
    want = M.run(tab, X, offsets, tok, T, k, sh, d)
    bad = X.clone()
    bad[2, 1047], bad[5, 3] = float("nan"), float("-inf")
    got = M.run(tab, bad, offsets, tok, T, k, sh, d)
    hit = torch.zeros(T * (k + sh), dtype=torch.bool)
    hit[:T * k] = torch.from_numpy(np.isin(tok, (2, 5)))
    hit[T * k + 2] = hit[T * k + 5] = True
    assert torch.isnan(got[hit.to(DEV)]).all()
    assert torch.equal(got[~hit.to(DEV)], want[~hit.to(DEV)])
    w["d"][1047, 1030] = float("nan")                  # W_down of slot 0: its last output column
    got = M.run(M.tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    n0 = int(offsets[1])
    assert n0 > 0 and torch.isnan(got[:n0, 1047]).all()
    want[:n0, 1047] = got[:n0, 1047] = 0
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_few_tokens_captured_and_on_another_stream():
    case = T, d, E, k, I, sh, _ = FEW_CASES["ragged_ends_and_empty_slots"]
    X, w, offsets, tok = M.draw(*case)
    tab = M.tables(w, d, E, k, I, sh)
    X, out = X.to(DEV), torch.empty(T * (k + sh), d, dtype=torch.bfloat16, device=DEV)
    tok, offsets = (torch.from_numpy(v.astype(np.int32)).to(DEV) for v in (tok, offsets))
    ws = torch.empty(api.moe_grouped_swiglu_fwd_mx4_workspace_size(tab, T, k), dtype=torch.uint8, device=DEV)
    go = lambda: api.moe_grouped_swiglu_fwd_mx4(tab, X, tok, offsets, T, k, out, ws)  # noqa: E731
    go()
    torch.cuda.synchronize()
    want, X0 = out.clone(), X.clone()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(g, stream=side):
        go()
    for _ in range(3):
        out.fill_(3.0)
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        X.mul_(-0.5)                                   # the replay reads what is there now
        g.replay()
        torch.cuda.synchronize()
        assert not torch.equal(out, want)
        X.copy_(X0)
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.default_stream())
            out.fill_(5.0)
            go()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# ------------------------------------------------------------ 256-row tiles ----

LARGE_CASES = {
    # name: (T, d, E, k, I, shared, rows per routed slot)
    # gate-up: 9 column tiles and a half slab; down: 5 slabs, a half slab, the scales' last
    # group moved back, a column tile of 8; tiles of 1, 127, 128, 129 and 255 rows
    "uneven_slots_and_a_shared_one": (7001, 264, 6, 4, 1032, 1,
                                      (20 * 256 + 1, 18 * 256 + 127, 22 * 256 + 128, 0, 19 * 256 + 129, 25 * 256 + 255)),
    # 3 slabs in both products, each with its last scales moved back; a slot below one tile
    "three_slabs": (10900, 520, 5, 4, 648, 0, (50 * 256 + 200, 100, 45 * 256, 40 * 256 + 64, 30 * 256 + 1)),
    # one slab in both, no end off a 128-block
    "one_slab_many_slots": (9000, 256, 16, 16, 256, 1, tuple(8300 + 37 * i for i in range(16))),
}


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(LARGE_CASES))
def test_large_tiles(name):
    """Every row against the oracle: the tokens repeat 64 different ones."""
    T, d, E, k, I, sh, rows = LARGE_CASES[name]
    assert path(T, d, E, k, I, sh) == LARGE and len(rows) == E and sum(rows) <= T * k
    base, w, _, _ = M.draw(64, d, E, 1, I, sh, E)
    X = base[torch.arange(T) % 64]
    offsets = np.concatenate(([0], np.cumsum(rows)))
    N = int(offsets[-1])
    tok = np.random.default_rng(N).integers(0, T, T * k)
    got = M.run(M.tables(w, d, E, k, I, sh), X, offsets, tok, T, k, sh, d)
    assert bool((got[N:T * k] == 7.0).all())
    left = 0
    for s in range(E + sh):
        r0, n = (int(offsets[s]), rows[s]) if s < E else (T * k + (s - E) * T, T)
        wg, wu, wd = (O.mxfp4_round(w[m][s * r:(s + 1) * r].double().numpy()) for m, r in (("g", I), ("u", I), ("d", d)))
        want, tol, near = M.exact_rows(base.double().numpy(), wg, wu, wd)
        left += int(near.sum())
        which = torch.from_numpy(tok[r0:r0 + n] if s < E else np.arange(T)).to(DEV) % 64
        want, tol, sure = (torch.from_numpy(v).to(DEV)[which] for v in (want, tol, ~near))
        g = got[r0:r0 + n].double()
        bad = ~((g - want).abs() <= tol) & sure[:, None]
        assert not bad.any(), (s, bad.nonzero()[:5].tolist())
        # the same token in the same slot: the same bits, in whichever tile it lies
        first = torch.full((64,), n, dtype=torch.long, device=DEV).scatter_reduce(
            0, which, torch.arange(n, device=DEV), "amin")
        assert torch.equal(got[r0:r0 + n], got[r0:r0 + n][first[which]])
    log(f"  {name}: {left} of {64 * (E + sh)} next to a border")
    assert left <= 0.2 * 64 * (E + sh)
