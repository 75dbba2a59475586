"""What the tables of 4-bit experts refuse and keep: the kernels read the addresses in
them without a check."""
import gc
import types

import pytest
import torch

from paper_2508_19078_amd import api

import test_gpu_mxfp4 as M

pytestmark = pytest.mark.gpu
DEV, U8 = "cuda", torch.uint8


def off(shape, by):
    """A contiguous tensor of this shape that starts `by` bytes behind an aligned address."""
    n = shape[0] * shape[1]
    return torch.zeros(n + by, dtype=U8, device=DEV)[by:].view(shape)


@pytest.mark.parametrize("at,name", enumerate(["q_gate", "q_up", "q_down", "s_gate", "s_up", "s_down"]))
def test_misaligned_matrices_are_refused(at, name):
    d, I = 64, 32
    (cg, sg), (cd, sd) = api.mxfp4_shapes(I, d), api.mxfp4_shapes(d, I)
    shapes = [cg, cg, cd, sg, sg, sd]
    args = [[off(s, 0), off(s, 4 if i > 2 else 16)] for i, s in enumerate(shapes)]
    api.LayerTablesMX4(d, I, 1, 1, *args)
    for by in (1, 2) + ((8,) if at < 3 else ()):
        bad = [list(a) for a in args]
        bad[at][1] = off(shapes[at], by)
        with pytest.raises(ValueError, match=rf"{name}\[1\] is not"):
            api.LayerTablesMX4(d, I, 1, 1, *bad)


def test_tables_of_another_device_are_refused():
    X, w, offsets, tok = M.draw(4, 64, 2, 1, 32, 0, 2)
    tab = M.tables(w, 64, 2, 1, 32, 0)
    elsewhere = types.SimpleNamespace(struct=tab.struct, tabs=[torch.zeros(1)])
    with pytest.raises(ValueError, match="tables are on cpu"):
        M.run(elsewhere, X, offsets, tok, 4, 1, 0, 64, ws=torch.empty(1 << 20, dtype=U8, device=DEV))


def test_the_tables_keep_the_matrices():
    """Also when the caller's lists are emptied and the memory would serve others."""
    T, d, E, k, I = 33, 136, 3, 1, 72
    X, w, offsets, tok = M.draw(T, d, E, k, I, 0, E)
    q = {m: M.quantize(w[m].to(DEV)) for m in "gud"}
    rows = dict(g=I, u=I, d=d)
    lists = [[q[m][j][i * rows[m]:(i + 1) * rows[m]].clone() for i in range(E)] for j in (0, 1) for m in "gud"]
    tab = api.LayerTablesMX4(d, I, E, 0, *lists)
    want = M.run(M.tables(w, d, E, k, I, 0), X, offsets, tok, T, k, 0, d)
    kept = [[t.data_ptr() for t in x] for x in lists]
    for x in lists:
        x.clear()
    gc.collect()
    assert [[t.data_ptr() for t in x] for x in tab.keep] == kept
    assert torch.equal(M.run(tab, X, offsets, tok, T, k, 0, d), want)
