"""Refusals of dense layers, dropout and the label loss, and their reference's own pins.  No GPU work is
issued: every call here is refused on the host."""
import ctypes
import math
import os

import pytest
import torch

import layers_ref as ref
import paper_2110_07029_amd as asgd
from test_logits_cpu import A, BIG, MATRICES, Ws, csr, mat, refused

E, R = asgd.ASGD_EINVAL, asgd.ASGD_ERANGE
BF16 = asgd.ASGD_BF16


def at(i):
    """Addresses that are far apart."""
    return A + (i << 32)


def layer(m=4, n=6, k=8, dtype=asgd.ASGD_F32):
    return {"x": mat(m, k, dtype=dtype, data=at(1)), "w": mat(n, k, dtype=dtype, data=at(2)), "y": mat(m, n, data=at(3))}


def dense(**change):
    a = {**layer(), **change}
    asgd.asgd_dense(a.pop("x"), a.pop("w"), a.pop("y"), **{"workspace": BIG, **a})


def backward(**change):
    a = {**layer(), "dy": mat(4, 6, data=at(3)), "dx": mat(4, 8, data=at(4)), "dw": mat(6, 8, data=at(5)), "db": at(6), **change}
    a.pop("y")
    asgd.asgd_dense_backward(a.pop("dy"), a.pop("x"), a.pop("w"), **{"workspace": BIG, **a})


def loss(**change):
    a = {"h": mat(4, 8, data=at(1)), "w": mat(100, 8, data=at(2)), "y": csr(indptr=at(3), indices=at(4)), "loss_rows": at(5),
         "lse": at(6), "dh": mat(4, 8, data=at(7)), "dw": mat(100, 8, data=at(8)), "db": at(9), "bias": at(10),
         "weights": at(11), **change}
    asgd.asgd_label_loss(a.pop("h"), a.pop("w"), a.pop("y"), a.pop("loss_rows"), **{"workspace": BIG, **a})


@pytest.mark.parametrize("change,status,word", MATRICES)
def test_bad_matrices_are_refused(change, status, word):
    m = mat(**{**change, "data": change.get("data", at(9))})
    for name in ("x", "w", "y", "pre"):
        if name == "w" and status == R and "rows" in change:
            continue
        refused(status, word, dense, **{name: m})
    refused(status, word, backward, dx=m)
    refused(status, word, asgd.asgd_dropout, m, 0.1, 0, mat())
    refused(status, word, loss, h=m)
    if "rows" not in change or status != R:
        refused(status, word, loss, w=m)
    refused(status, word, asgd.asgd_dense_workspace, m, mat())
    refused(status, word, asgd.asgd_dense_backward_workspace, m, mat())
    refused(status, word, asgd.asgd_label_loss_workspace, m, mat())


def ep(**k):
    return asgd.dense_epilogue(**k)


def test_dense_layers_are_checked():
    refused(E, "columns", dense, x=mat(4, 9, data=at(1)))
    refused(E, "type", dense, x=mat(4, 8, dtype=BF16, data=at(1)))
    refused(E, "y has another shape", dense, y=mat(4, 7, data=at(3)))
    refused(E, "y has another shape", dense, y=mat(5, 6, data=at(3)))
    refused(E, "pre has another shape", dense, pre=mat(4, 7, data=at(4)))
    refused(E, "residual has another shape", dense, epilogue=ep(residual=mat(6, 4, data=at(4))))
    for act in (-1, 4):
        refused(E, "act", dense, epilogue=ep(act=act))
        refused(E, "act", backward, epilogue=ep(act=act))
    for p in (-0.1, 1.0, 2.0, math.nan, math.inf):
        refused(E, "[0, 1)", dense, epilogue=ep(drop=p))
        refused(E, "[0, 1)", backward, epilogue=ep(drop=p))
        refused(E, "[0, 1)", asgd.asgd_dropout, mat(), p, 0, mat(data=at(1)))
    e = ep()
    e.bias = A + 2
    refused(E, "bias", dense, epilogue=e)
    with pytest.raises(ValueError):
        dense(epilogue=ep(bias=torch.zeros(5)))
    for bad in (torch.zeros(6, dtype=torch.float64), torch.zeros(2, 3), torch.zeros(12)[::2]):
        with pytest.raises(ValueError):
            ep(bias=bad)
    lib, by = asgd.load(), ctypes.byref
    a = {k: by(v) for k, v in layer().items()}
    assert lib.asgd_dense(None, a["w"], None, None, a["y"], A, 1 << 40, None) == E
    assert lib.asgd_dense(a["x"], None, None, None, a["y"], A, 1 << 40, None) == E
    assert lib.asgd_dense(a["x"], a["w"], None, None, None, A, 1 << 40, None) == E
    assert lib.asgd_dense_workspace(a["x"], a["w"], None) == E
    assert lib.asgd_dense_backward_workspace(a["x"], a["w"], None) == E


def test_sums_over_more_than_two_to_the_twenty_columns_are_refused():
    k = 1 << 20
    long = dict(x=mat(4, k + 1, data=at(1)), w=mat(6, k + 1, data=at(2)))
    refused(R, "2^20 columns", dense, **long)
    refused(R, "2^20 columns", backward, **long)
    refused(R, "2^20 columns", asgd.asgd_dense_workspace, *long.values())
    refused(R, "2^20 columns", asgd.asgd_dense_backward_workspace, *long.values())
    refused(R, "2^20 columns", loss, h=long["x"], w=mat(100, k + 1, data=at(2)))
    refused(R, "2^20 columns", asgd.asgd_label_loss_workspace, *long.values(), False)
    refused(R, "workspace", dense, x=mat(4, k, data=at(1)), w=mat(6, k, data=at(2)), workspace=Ws(0))
    asgd.asgd_label_loss_workspace(mat(4, k), mat(6, k), True)
    # (a dropout of that width sums nothing)
    refused(E, "overlaps", asgd.asgd_dropout, mat(4, k + 1), 0.1, 0, mat(4, k + 1, data=A + 4))


def test_outputs_that_share_memory_are_refused():
    refused(E, "overlaps", dense, y=mat(4, 6, data=at(1) + 32))
    refused(E, "overlaps", dense, y=mat(4, 6, data=at(2)))
    refused(E, "overlaps", dense, epilogue=ep(residual=mat(4, 6, data=at(3) + 4)))
    refused(E, "overlaps", dense, epilogue=ep(residual=mat(4, 6, ld=7, data=at(3))))
    refused(E, "overlaps", dense, epilogue=ep(residual=mat(4, 6, dtype=BF16, data=at(3))))
    refused(E, "overlaps", dense, pre=mat(4, 6, data=at(3)))
    refused(E, "overlaps", dense, pre=mat(4, 6, data=at(4)), epilogue=ep(residual=mat(4, 6, data=at(4))))
    # columns of one buffer: side by side they are fine (the call goes on to the workspace), else not
    side = dict(x=mat(4, 8, 20, data=at(1)), w=mat(6, 8, ld=9, data=at(2)))
    for shift, fine in ((8, True), (14, True), (7, False), (15, False), (20 + 8, True), (-12, True), (-6, True), (-5, False), (-13, False)):
        y = mat(4, 6, 20, data=at(1) + 4 * shift)
        if fine:
            refused(R, "workspace", dense, **side, y=y, workspace=Ws(0))
        else:
            refused(E, "overlaps", dense, **side, y=y)
    for name, shape in (("dx", (4, 8)), ("dw", (6, 8))):
        for i in (1, 2, 3):
            refused(E, "overlaps an input", backward, **{name: mat(*shape, data=at(i))})
        refused(E, "gradients overlap", backward, **{name: mat(*shape, data=at(6))})
    refused(E, "gradients overlap", backward, dx=mat(4, 8, data=at(5)))
    refused(E, "overlaps an input", backward, db=at(2) + 8)
    refused(E, "overlaps an input", backward, pre=mat(4, 6, data=at(4)))
    refused(E, "overlaps", asgd.asgd_dropout, mat(), 0.1, 0, mat(data=A + 4))
    refused(E, "overlaps", asgd.asgd_dropout, mat(), 0.1, 0, mat(data=at(1)), residual=mat(data=at(1) + 400))
    refused(E, "output overlaps an input", loss, loss_rows=at(1))
    refused(E, "output overlaps an input", loss, db=at(10) + 4)
    refused(E, "output overlaps an input", loss, lse=at(3))
    refused(E, "output overlaps an input", loss, dw=mat(100, 8, data=at(2)))
    refused(E, "outputs overlap", loss, lse=at(5) + 12)
    refused(E, "outputs overlap", loss, dh=mat(4, 8, data=at(8) + 64))


def test_gradients_are_checked():
    refused(E, "needs pre", backward, epilogue=ep(act=asgd.ASGD_ACT_RELU))
    refused(E, "all NULL", backward, dx=None, dw=None, db=None)
    refused(E, "dx has another shape", backward, dx=mat(4, 6, data=at(4)))
    refused(E, "dw has another shape", backward, dw=mat(8, 6, data=at(5)))
    refused(E, "dy has another shape", backward, dy=mat(4, 8, data=at(3)))
    refused(E, "pre has another shape", backward, pre=mat(4, 8, data=at(7)))
    refused(E, "db", backward, db=at(6) + 2)
    with pytest.raises(ValueError):
        backward(db=torch.zeros(5))


def test_the_label_loss_is_checked():
    refused(E, "columns", loss, h=mat(4, 9, data=at(1)))
    refused(E, "type", loss, h=mat(4, 8, dtype=BF16, data=at(1)))
    refused(R, "2^22", loss, w=mat(1 << 22, 8, data=at(2)))
    refused(E, "y is NULL", loss, y=None)
    for change, word in ((dict(rows=5), "n_rows"), (dict(cols=99), "n_cols"), (dict(nnz=-1), "nnz"), (dict(indptr=None), "indptr"),
                         (dict(indices=None), "indices"), (dict(indptr=at(3) + 2), "aligned")):
        refused(E, word, loss, y=csr(**{"indptr": at(3), "indices": at(4), **change}))
    refused(R, "2^30", loss, y=csr(nnz=1 << 30, indptr=at(3), indices=at(4)))
    refused(E, "loss_rows", loss, loss_rows=None)
    for name in ("bias", "weights", "loss_rows", "lse", "db"):
        refused(E, "4-byte", loss, **{name: at(12) + 2})
    for name, n in (("bias", 100), ("weights", 4), ("loss_rows", 4), ("lse", 4), ("db", 100)):
        with pytest.raises(ValueError):
            loss(**{name: torch.zeros(n - 1)})
        with pytest.raises(ValueError):
            loss(**{name: torch.zeros(n, dtype=torch.float16)})
    refused(E, "dh has another shape", loss, dh=mat(4, 7, data=at(7)))
    refused(E, "dw has another shape", loss, dw=mat(99, 8, data=at(8)))
    lib = asgd.load()
    assert lib.asgd_label_loss_workspace(ctypes.byref(mat(4, 8)), ctypes.byref(mat(100, 8)), 1, None) == E


@pytest.mark.parametrize("dtype", [asgd.ASGD_F32, BF16, asgd.ASGD_F16])
def test_workspaces(dtype):
    for m, n, k in ((1, 4096, 1024), (33, 77, 515), (4000, 4000, 64)):
        x, w, y = mat(m, k, dtype=dtype, data=at(1)), mat(n, k, dtype=dtype, data=at(2)), mat(m, n, data=at(3))
        need, back = asgd.asgd_dense_workspace(x, w), asgd.asgd_dense_backward_workspace(x, w)
        if need:
            refused(R, "workspace", asgd.asgd_dense, x, w, y, workspace=Ws(need - 1))
            refused(E, "NULL", asgd.asgd_dense, x, w, y, workspace=Ws(need, None))
            refused(E, "256", asgd.asgd_dense, x, w, y, workspace=Ws(need, A + 128))
        refused(R, "workspace", asgd.asgd_dense_backward, y, x, w, db=at(4), workspace=Ws(back - 1))
    h, w = mat(40, 61, dtype=dtype, data=at(1)), mat(5000, 61, dtype=dtype, data=at(2))
    y = csr(40, 5000, indptr=at(3), indices=at(4))
    less, need = asgd.asgd_label_loss_workspace(h, w, False), asgd.asgd_label_loss_workspace(h, w, True)
    assert less < need
    refused(R, "workspace", asgd.asgd_label_loss, h, w, y, at(5), workspace=Ws(less - 1))
    refused(R, "workspace", asgd.asgd_label_loss, h, w, y, at(5), db=at(6), workspace=Ws(need - 1))
    # the largest label matrix has a workspace, too
    asgd.asgd_label_loss_workspace(mat(1 << 20, 128), mat((1 << 22) - 1, 128), True)
    # rows in place need none of their own, rows out of line a copy
    assert asgd.asgd_dense_workspace(mat(4000, 64), mat(4000, 64)) == 0
    assert asgd.asgd_dense_workspace(mat(4000, 63), mat(4000, 63)) >= 2 * 4000 * 64 * 4


def test_reference_of_the_random_bits():
    # splitmix64 as published: the first outputs of the generator that starts at 0
    with open(os.path.join(os.path.dirname(__file__), "golden", "splitmix64_seed0.txt")) as f:
        first = [int(x.split()[1], 0) for x in f if not x.startswith("#")][0]  # of state 0

    def mix(v):
        v = (v + 0x9E3779B97F4A7C15) % 2 ** 64
        v = (v ^ (v >> 30)) * 0xBF58476D1CE4E5B9 % 2 ** 64
        v = (v ^ (v >> 27)) * 0x94D049BB133111EB % 2 ** 64
        return v ^ (v >> 31)
    assert mix(0) == first
    k = ref.kept(3, 5, 0.5, 0)
    for i in range(3):
        for j in range(5):
            word = mix(mix(0) ^ (i * 2 ** 22 + j // 2))
            assert k[i, j] == ((word >> 32 * (j % 2)) % 2 ** 32 >= 2 ** 31)


def test_reference_of_layers_and_loss_against_automatic_differentiation():
    g = torch.Generator().manual_seed(1)
    x, w, b, dy = (torch.randn(*s, generator=g, dtype=torch.float64, requires_grad=True) for s in ((5, 7), (6, 7), (6,), (5, 6)))
    for name, f in (("relu", torch.relu), ("gelu", torch.nn.functional.gelu), ("silu", torch.nn.functional.silu), ("none", lambda t: t)):
        a, _, y, _ = ref.dense(x, w, b, name, 0.4, 3)
        want = f(x @ w.T + b) * ref.mask(5, 6, 0.4, 3, "cpu")
        assert torch.allclose(y, want, atol=1e-12)
        gx, gw, gb = torch.autograd.grad((want * dy).sum(), (x, w, b))
        got = ref.dense_grad(dy.detach(), x.detach(), w.detach(), a.detach(), "f32", name, 0.4, 3)
        for k, t in (("dx", gx), ("dw", gw), ("db", gb)):
            assert torch.allclose(got[k][0], t, atol=1e-12), (name, k)
    lists, weights = [[1, 3], [], [2, 2, 9], [5], [0, -1]], torch.rand(5, dtype=torch.float64, generator=g)
    out = ref.label_loss(x.detach(), w.detach(), lists, b.detach(), weights, "f32")
    logp = torch.log_softmax(x @ w.T + b, 1)
    rows = [[1, 3], [], [2, 2], [5], [0]]
    loss = torch.stack([-logp[i, r].mean() if r else logp[i, 0] * 0 for i, r in enumerate(rows)])
    assert torch.allclose(out["loss"][0], loss)
    for k, t in zip(("dh", "dw", "db"), torch.autograd.grad((loss * weights).sum(), (x, w, b))):
        assert torch.allclose(out[k][0], t, atol=1e-12), k


def test_what_shares_memory_is_found_element_by_element():
    # outputs of one row and of several against w [n x 8] in rows of 21, wherever they begin.  A matrix of one row has no
    # stride, whatever its ld says.
    for n, rows, ld in ((6, 1, 6), (6, 1, 33), (30, 1, 30), (6, 3, 21), (1, 1, 7), (1, 5, 9)):
        held = {21 * i + j for i in range(n) for j in range(8)}
        step = ld if rows > 1 else 0
        for start in range(-max(ld, n) * rows - 8, 21 * n + 8, 1 if n < 10 else 7):
            taken = {start + i * step + j for i in range(rows) for j in range(n)}
            call = dict(x=mat(rows, 8, data=at(1)), w=mat(n, 8, 21, data=at(2)), y=mat(rows, n, ld, data=at(2) + 4 * start))
            if held & taken:
                refused(E, "overlaps", dense, **call)
            else:
                refused(R, "workspace", dense, **call, workspace=Ws(0))
    # the residual itself, whatever the strides of one row say; of another type it is not itself
    x, w = mat(1, 8, data=at(1)), mat(6, 8, 9, data=at(2))
    for ld in (6, 9):
        refused(R, "workspace", dense, x=x, w=w, y=mat(1, 6, ld, data=at(3)), epilogue=ep(residual=mat(1, 6, data=at(3))), workspace=Ws(0))
    refused(E, "overlaps", dense, x=x, y=mat(1, 6, data=at(3)), epilogue=ep(residual=mat(1, 6, dtype=BF16, data=at(3))))
    # the bias's gradient in the gaps between dw's rows
    for col, fine in ((8, True), (14, True), (7, False), (15, False)):
        change = dict(dw=mat(6, 8, 20, data=at(5)), db=at(5) + 4 * (40 + col), w=w)
        if fine:
            refused(R, "workspace", backward, **change, workspace=Ws(0))
        else:
            refused(E, "overlap", backward, **change)
