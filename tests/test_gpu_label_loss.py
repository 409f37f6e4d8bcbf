"""The label loss and its gradients on the GPU, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import layers_ref as ref
import paper_2110_07029_amd as asgd
from gpu_util import flush
from test_gpu_layers import NAN, INF, normal, placed, room, scratch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _say(request):
    flush(request.node.name)
    asgd.load()


def csr(lists, labels, before=0):
    """(asgd_csr, tensors that it borrows); `before` entries of another batch lie in front."""
    flat = [2 ** 30] * before + [i for r in lists for i in r] + [2 ** 30]
    ends = before + np.concatenate([[0], np.cumsum([len(r) for r in lists])])
    keep = [torch.tensor(ends, dtype=torch.int32, device="cuda"), torch.tensor(flat, dtype=torch.int32, device="cuda")]
    return asgd.asgd_csr(len(lists), labels, int(ends[-1]) - before, keep[0].data_ptr(), keep[1].data_ptr(), None), keep


def random_lists(seed, rows, labels, mean):
    r = np.random.default_rng(seed)
    out = [r.choice(labels, min(labels, int(k)), replace=False).tolist() for k in r.integers(0, 2 * mean + 1, rows)]
    if rows == 1 and not out[0]:
        out[0] = [0]
    return out


class Call:
    """One call with outputs in rooms of their own."""

    def __init__(self, h, w, lists, bias=None, weights=None, dtype="f32", out=None, shift=0, pad=0, grads=("dh", "dw", "db"),
                 before=0):
        B, D = h.shape
        L = w.shape[0]
        self.y, self.keep = csr(lists, L, before)
        self.loss, self.lse = (torch.full((B + 1,), NAN, device="cuda") for _ in range(2))
        self.dh, self.clean_h = room(B, D, out or dtype, shift, pad)
        self.dw, self.clean_w = room(L, D, out or dtype, shift, pad)
        self.db = torch.full((L + 1,), NAN, device="cuda")
        self.h, self.w, self.bias, self.weights, self.grads = h, w, bias, weights, grads
        self.types = {"loss": "f32", "lse": "f32", "dh": out or dtype, "dw": out or dtype, "db": "f32"}
        self.ws = scratch(asgd.asgd_label_loss_workspace(asgd.matrix(h), asgd.matrix(w), bool(grads)))
        self.B, self.L = B, L

    def run(self):
        a = asgd.matrix
        asgd.asgd_label_loss(a(self.h), a(self.w), self.y, self.loss, bias=self.bias, weights=self.weights, lse=self.lse,
                             dh=a(self.dh) if "dh" in self.grads else None, dw=a(self.dw) if "dw" in self.grads else None,
                             db=self.db if "db" in self.grads else None, workspace=self.ws,
                             stream=torch.cuda.current_stream())
        return self

    def outputs(self):
        out = {"loss": self.loss[:self.B], "lse": self.lse[:self.B]}
        out.update({k: v for k, v in (("dh", self.dh), ("dw", self.dw), ("db", self.db[:self.L])) if k in self.grads})
        return out

    def check(self, lists, dtype):
        want = ref.label_loss(self.h, self.w, lists, self.bias, self.weights, dtype)
        for name, got in self.outputs().items():
            ref.near(got, *want[name], self.types[name], name)
        self.clean_h()
        self.clean_w()
        assert bool(self.loss[self.B].isnan()) and bool(self.lse[self.B].isnan()) and bool(self.db[self.L].isnan())


SIZES = [(1, 1, 1, 1), (1, 2, 8, 1), (1, 3000, 128, 3), (3, 7, 5, 2), (31, 1000, 64, 1), (33, 130, 40, 5), (128, 1000, 128, 3),
         (129, 257, 131, 5), (300, 300, 128, 75), (64, 20000, 128, 5), (700, 515, 264, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,L,D,mean", SIZES)
def test_loss_and_gradients_of_all_sizes(B, L, D, mean, dtype):
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=2 * D ** -0.5), dtype)
    lists = random_lists(3, B, L, mean)
    Call(h, w, lists, normal(4, L), dtype=dtype).run().check(lists, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,shift,pad", [(128, 0, 8), (61, 1, 5), (136, 8, 24)])
def test_strided_rows_with_weights(D, shift, pad, dtype):
    B, L = 150, 900
    h, w = placed(normal(1, B, D), dtype, shift, pad), placed(normal(2, L, D, scale=0.2), dtype, shift, pad)
    lists = random_lists(5, B, L, 4)
    weights = torch.rand(B, generator=torch.Generator().manual_seed(1)).cuda() * 3e-3
    weights[::7] = 0.0
    weights[3] *= -1.0
    Call(h, w, lists, None, weights, dtype, shift=shift, pad=pad, before=9).run().check(lists, dtype)


@pytest.mark.parametrize("dtype,B,L", [("f32", 8192, 4500), ("bf16", 16384, 4200)])
def test_several_pieces_of_labels(dtype, B, L):
    h, w = placed(normal(1, B, 16), dtype), placed(normal(2, L, 16, scale=0.5), dtype)
    lists = random_lists(6, B, L, 1)
    Call(h, w, lists, normal(3, L), dtype=dtype).run().check(lists, dtype)


def test_large_tiles():
    B, L, D = 3600, 3700, 136
    h, w = placed(normal(1, B, D), "bf16"), placed(normal(2, L, D, scale=0.2), "bf16")
    lists = random_lists(6, B, L, 2)
    Call(h, w, lists, normal(3, L), dtype="bf16").run().check(lists, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_wide_labels_on_few_rows(dtype):
    for B, L in ((1, 70001), (5, 70001), (40, 30001)):
        h, w = placed(normal(1, B, 128), dtype), placed(normal(2, L, 128, scale=0.2), dtype)
        lists = random_lists(7, B, L, 5)
        Call(h, w, lists, normal(3, L), dtype=dtype).run().check(lists, dtype)


@pytest.mark.parametrize("grads", [(), ("dh",), ("dw",), ("db",), ("dh", "db")])
def test_parts_of_the_outputs_are_the_same(grads):
    B, L, D = 100, 3000, 128
    h, w, lists = normal(1, B, D).bfloat16(), normal(2, L, D, scale=0.2).bfloat16(), random_lists(8, B, L, 3)
    whole = Call(h, w, lists, dtype="bf16").run().outputs()
    part = Call(h, w, lists, dtype="bf16", grads=grads).run().outputs()
    assert set(part) == {"loss", "lse", *grads}
    for k, v in part.items():
        assert torch.equal(v, whole[k]), k


def test_gradients_of_16_bits_into_floats():
    B, L, D = 60, 400, 128
    h, w, lists = normal(1, B, D).bfloat16(), normal(2, L, D, scale=0.2).bfloat16(), random_lists(8, B, L, 3)
    Call(h, w, lists, dtype="bf16", out="f32").run().check(lists, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_empty_rows_ids_out_of_range_and_repeats(dtype):
    B, L, D = 40, 300, 64
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.3), dtype)
    lists = random_lists(9, B, L, 3)
    lists[0] = []
    lists[1] = [-1, L, 2 ** 31 - 1, -2 ** 31]
    lists[2] = [5, -7, 5, 5, L + 3, 6]
    lists[3] = [L - 1] * 700 + [0]
    lists[39] = []
    c = Call(h, w, lists, normal(4, L), dtype=dtype).run()
    c.check(lists, dtype)
    for i in (0, 1, 39):
        assert float(c.loss[i]) == 0.0 and bool((c.dh[i] == 0).all())
    assert bool(c.lse[:B].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_rows_without_labels_hold_reaches_nothing(dtype):
    B, L, D = 50, 200, 61
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.3), dtype)
    weights = torch.full((B,), 0.01, device="cuda")
    lists = random_lists(9, B, L, 3)
    for i in (0, 7, 49):
        lists[i] = []
    quiet = Call(h, w, lists, None, weights, dtype).run().outputs()
    h[0], h[7, 3], h[49] = NAN, INF, 1e30
    weights[0], weights[7], weights[49] = NAN, INF, 1e30
    loud = Call(h, w, lists, None, weights, dtype).run().outputs()
    live = [i for i in range(B) if lists[i]]
    for k in ("loss", "dh"):
        assert torch.equal(loud[k], quiet[k]), k
    for k in ("dw", "db"):
        assert torch.equal(loud[k], quiet[k]), k
    assert torch.equal(loud["lse"][live], quiet["lse"][live])


def test_no_row_has_labels():
    for lists in ([[]] * 6, [[-1]] * 6):
        c = Call(normal(1, 6, 32), normal(2, 50, 32), lists).run()
        c.check(lists, "f32")
        assert all(bool((v == 0).all()) for k, v in c.outputs().items() if k != "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_labels_of_bias_minus_infinity(dtype):
    B, L, D = 70, 1000, 128
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.2), dtype)
    bias = normal(4, L)
    bias[100:700] = -INF  # whole tiles of them
    lists = [[0, 99, 999], [700]] * 35
    c = Call(h, w, lists, bias, dtype=dtype).run()
    c.check(lists, dtype)
    assert bool((c.dw[100:700] == 0).all()) and bool((c.db[100:700] == 0).all())


def test_logits_that_are_not_finite():
    B, L, D = 40, 500, 32
    h, w = normal(1, B, D), normal(2, L, D, scale=0.3)
    lists = [[1, 2]] * B
    h[5, 1] = NAN
    h[6, 1] = INF  # (its logits are infinities of both signs)
    c = Call(h, w, lists).run()
    rest = [i for i in range(B) if i not in (5, 6)]
    assert bool(c.loss[[5, 6]].isnan().all()) and bool(c.dh[[5, 6]].isnan().all())
    assert bool(c.dw.isnan().all()) and bool(c.db[:L].isnan().all())
    assert bool(c.loss[rest].isfinite().all()) and bool(c.dh[rest].isfinite().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_large_logits_and_certain_rows(dtype):
    # logits of hundreds, of which one decides: p is 1 and 0, what is left of the gradient is about nothing
    B, L, D = 64, 700, 64
    h, w = placed(normal(1, B, D, scale=20.0), dtype), placed(normal(2, L, D), dtype)
    best = (h.double() @ w.double().T).argmax(1).tolist()
    lists = [[j] for j in best]
    Call(h, w, lists, dtype=dtype).run().check(lists, dtype)


def test_gradients_meet_differences():
    B, L, D = 20, 90, 24
    h, w, bias = normal(1, B, D), normal(2, L, D, scale=0.4), normal(3, L)
    lists = random_lists(4, B, L, 3)
    weights = torch.rand(B, generator=torch.Generator().manual_seed(3)).cuda()
    c = Call(h, w, lists, bias, weights).run()

    def value(h, w, b):
        return float((Call(h, w, lists, b, weights, grads=()).run().loss[:B].double() * weights.double()).sum())
    for i, d in enumerate((c.dh, c.dw, c.db[:L])):
        t = (h, w, bias)[i]
        v, e = normal(30 + i, *t.shape), 2.0 ** -8
        args = [[u + s * e * v if j == i else u for j, u in enumerate((h, w, bias))] for s in (1, -1)]
        diff, slope = (value(*args[0]) - value(*args[1])) / (2 * e), float((d.double() * v.double()).sum())
        # Along v a row's logits move by e u exactly, and the third derivative of its log-sum-exp is the third central
        # moment of u under p: 2 max |u|^3 at most.  A sixth of it times e^2, weighted; and the values' own rounding, some
        # 2^-20 of a loss of about 5 a row, over e.
        u = v @ w.T if i == 0 else h @ v.T if i == 1 else v.expand(B, L)
        tol = e * e / 6 * float((weights * 2 * u.abs().amax(1) ** 3).sum()) + 2.0 ** -20 * 5 * B / e
        assert abs(diff - slope) <= tol, (i, diff, slope, tol)


def test_the_same_call_gives_the_same_bits_and_streams_agree():
    B, L, D = 500, 5000, 128
    h, w, lists = normal(1, B, D).bfloat16(), normal(2, L, D, scale=0.2).bfloat16(), random_lists(8, B, L, 5)
    first = Call(h, w, lists, dtype="bf16").run().outputs()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(Call(h, w, lists, dtype="bf16").run())
    torch.cuda.synchronize()
    for c in got:
        for k, v in c.outputs().items():
            assert torch.equal(v, first[k]), k


def test_captured_and_replayed():
    B, L, D = 100, 2000, 128
    h, w, lists = normal(1, B, D).bfloat16(), normal(2, L, D, scale=0.2).bfloat16(), random_lists(8, B, L, 3)
    c = Call(h, w, lists, normal(3, L), dtype="bf16").run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.run()
    for i in range(4):
        h.copy_(normal(20 + i, B, D))
        for t in c.outputs().values():
            t.fill_(NAN)
        c.ws.fill_(0xA5)
        g.replay()
        torch.cuda.synchronize()
        replayed = {k: v.clone() for k, v in c.outputs().items()}
        c.run()
        torch.cuda.synchronize()
        for k, v in c.outputs().items():
            assert torch.equal(v, replayed[k]), (i, k)


def test_layers_under_the_label_loss_as_they_are_used():
    """Two dense layers with dropout and a residual under the label loss, forward and back, against automatic
    differentiation of the same network in 64 bits."""
    B, D, L = 96, 128, 1500
    x = normal(1, B, D)
    w1, b1, w2, b2 = normal(2, 200, D, scale=0.1), normal(3, 200), normal(4, D, 200, scale=0.1), normal(5, D)
    wl, bl = normal(6, L, D, scale=0.2), normal(7, L)
    lists = random_lists(9, B, L, 4)
    a = asgd.matrix
    st = torch.cuda.current_stream()

    def ws(n):
        return scratch(n)
    pre1, y1, y2, h = (torch.empty(B, n, device="cuda") for n in (200, 200, D, D))
    e1 = asgd.dense_epilogue(bias=b1, act=asgd.ASGD_ACT_GELU, drop=0.2, seed=1)
    e2 = asgd.dense_epilogue(bias=b2, residual=a(x))
    asgd.asgd_dense(a(x), a(w1), a(y1), epilogue=e1, pre=a(pre1), workspace=ws(asgd.asgd_dense_workspace(a(x), a(w1))), stream=st)
    asgd.asgd_dense(a(y1), a(w2), a(y2), epilogue=e2, workspace=ws(asgd.asgd_dense_workspace(a(y1), a(w2))), stream=st)
    asgd.asgd_dropout(a(y2), 0.3, 2, a(h), stream=st)
    c = Call(h, wl, lists, bl).run()
    dy2, dy1, dx = torch.empty_like(y2), torch.empty_like(y1), torch.empty_like(x)
    g = {k: torch.empty_like(t) for k, t in (("w1", w1), ("b1", b1), ("w2", w2), ("b2", b2))}
    asgd.asgd_dropout(a(c.dh), 0.3, 2, a(dy2), stream=st)
    asgd.asgd_dense_backward(a(dy2), a(y1), a(w2), dx=a(dy1), dw=a(g["w2"]), db=g["b2"], epilogue=e2,
                             workspace=ws(asgd.asgd_dense_backward_workspace(a(y1), a(w2))), stream=st)
    asgd.asgd_dense_backward(a(dy1), a(x), a(w1), pre=a(pre1), dx=a(dx), dw=a(g["w1"]), db=g["b1"], epilogue=e1,
                             workspace=ws(asgd.asgd_dense_backward_workspace(a(x), a(w1))), stream=st)
    asgd.asgd_dropout(a(dx), 0.0, 0, a(dx), residual=a(dy2), stream=st)  # the residual's way back
    torch.cuda.synchronize()

    leaves = {k: t.detach().cpu().double().requires_grad_() for k, t in
              (("x", x), ("w1", w1), ("b1", b1), ("w2", w2), ("b2", b2), ("wl", wl), ("bl", bl))}
    v = leaves
    t1 = torch.nn.functional.gelu(v["x"] @ v["w1"].T + v["b1"]) * ref.mask(B, 200, 0.2, 1, "cpu")
    t2 = t1 @ v["w2"].T + v["b2"] + v["x"]
    logp = torch.log_softmax((t2 * ref.mask(B, D, 0.3, 2, "cpu")) @ v["wl"].T + v["bl"], 1)
    loss = torch.stack([-logp[i, r].mean() if r else logp[i, 0] * 0 for i, r in enumerate(lists)])
    loss.mean().backward()
    assert torch.allclose(c.loss[:B].cpu().double(), loss.detach(), rtol=1e-5, atol=1e-5)
    got = {"x": dx, "w1": g["w1"], "b1": g["b1"], "w2": g["w2"], "b2": g["b2"], "wl": c.dw, "bl": c.db[:L]}
    for k, t in got.items():
        want = v[k].grad
        # sums of up to 1,500 fp32 products in a chain of five: some 5 sqrt(1500) 2^-24 of the norm, 1.2e-5; twice that
        assert float((t.cpu().double() - want).norm()) <= 2.4e-5 * float(want.norm()), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_very_long_lists_and_many_targets_in_a_tile(dtype):
    # row 0 names one label 70,000 times and another 5 times behind them: the first 65,535 entries count; the other rows
    # name so many labels that every tile has more targets than it lists
    B, L, D = 200, 260, 40
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.3), dtype)
    lists = [[7] * 70000 + [9] * 5] + [list(range(i % 3, L, 2)) for i in range(1, B)]
    c = Call(h, w, lists, normal(4, L), dtype=dtype).run()
    c.check([[7] * 65535] + lists[1:], dtype)


def test_more_tiles_than_a_launch_has_threads():
    # 65,536 rows against 2^22 - 1 labels of width 136: 16.8 million tiles.  Some rows' log-sum-exp in 64 bits.
    B, L, D = 65536, (1 << 22) - 1, 136
    g = torch.Generator(device="cuda").manual_seed(1)
    h = torch.randn(B, D, generator=g, device="cuda").bfloat16()
    w = (torch.randn(L, D, generator=g, device="cuda") * 0.1).bfloat16()
    y = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    ids = torch.randint(0, L, (B,), generator=g, device="cuda").int()
    loss, lse = torch.full((B,), NAN, device="cuda"), torch.full((B,), NAN, device="cuda")
    ws = torch.empty(asgd.asgd_label_loss_workspace(asgd.matrix(h), asgd.matrix(w), False), dtype=torch.uint8, device="cuda")
    asgd.asgd_label_loss(asgd.matrix(h), asgd.matrix(w), asgd.asgd_csr(B, L, B, y.data_ptr(), ids.data_ptr(), None), loss,
                         lse=lse, workspace=ws, stream=torch.cuda.current_stream())
    assert bool(lse.isfinite().all()) and bool(loss.isfinite().all())
    for i in (0, 1, 12345, 65535):
        z = w.double() @ h[i].double()
        want = torch.logsumexp(z, 0)
        ez = (D + 2) * ref.U * float((w.double().abs() @ h[i].double().abs()).max())
        # (bounds as in the reference)
        tol = 2 * ez + (200 + 2 * L / 32768 + 4 * np.log(L)) * ref.U + 4 * ref.U * float(want)
        assert abs(float(lse[i]) - float(want)) <= tol, (i, float(lse[i]), float(want), tol)
        assert abs(float(loss[i]) - float(want - z[ids[i].long()])) <= 2 * tol, i
    del w, h, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("B,L,D,mean,dtype", [
    (3600, 3700, 1000, 2, "bf16"), (3600, 3700, 1000, 2, "f16"),  # large tiles of long rows
    (256, 300, 128, 75, "bf16"), (256, 300, 128, 75, "f16"),      # narrow rows: more targets than a workgroup lists
    (256, 20000, 120, 3, "bf16"), (255, 4097, 64, 3, "f16"),      # narrow rows: the most whose gradients take one pass, and about
    (300, 70000, 520, 3, "bf16"), (300, 70000, 520, 3, "f16"),    # medium tiles, the sum over labels split
    (5, 30000, 200, 3, "bf16"), (32, 30000, 200, 3, "f32")])      # few rows
def test_sizes_behind_each_choice_of_tiles(B, L, D, mean, dtype):
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=2 * D ** -0.5), dtype)
    lists = random_lists(3, B, L, mean)
    Call(h, w, lists, normal(4, L), dtype=dtype).run().check(lists, dtype)


@pytest.mark.parametrize("B", [33000, 70000, 131073])
def test_narrow_rows_in_many_blocks(B):
    # each choice of ranges of labels; rows of integers in few bits, whose logits are exact
    L, D = 700, 24
    g = torch.Generator().manual_seed(B)
    h, w = (torch.randint(-2, 3, s, generator=g).to(torch.bfloat16).cuda() for s in ((B, D), (L, D)))
    ids = torch.randint(0, L, (B,), generator=g)
    c = Call(h, w, [[i] for i in ids.tolist()], dtype="bf16", grads=()).run()
    z = h.double() @ w.double().T
    want = torch.logsumexp(z, 1)
    # exponentials as in the reference; the logits are exact
    tol = (200 + 2 * L / 32768 + 4 * np.log(L)) * ref.U + 4 * ref.U * want.abs()
    assert bool(((c.lse[:B].double() - want).abs() <= tol).all())
    target = z[torch.arange(B), ids.cuda()]
    assert bool(((c.loss[:B].double() - (want - target)).abs() <= tol + 12 * ref.U * (want.abs() + target.abs())).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_weights_whose_largest_has_no_labels(dtype):
    # the gradients' scale is that of rows with labels, in whatever order the weights come
    B, L, D = 600, 300, 64
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.3), dtype)
    lists = [[] if i % 3 == 1 else [-1, L] if i % 3 == 2 else [i % L] for i in range(B)]
    up = torch.arange(1, B + 1, dtype=torch.float32).cuda() * 1e-6
    for weights in (up, up.flip(0), up.flip(0) * -1.0):
        weights = weights.clone()
        weights[1], weights[599] = 1e30, INF
        c = Call(h, w, lists, normal(4, L), weights, dtype=dtype).run()
        weights[1] = weights[599] = 0.0  # (rows without labels: the reference needs finite ones)
        c.check(lists, dtype)


@pytest.mark.parametrize("B,L,D,mean,shift,pad,dtype", [
    (300, 41000, 128, 3, 0, 0, "bf16"), (257, 40000, 64, 75, 0, 8, "f16"), (1000, 40500, 120, 5, 0, 0, "f16"),
    (700, 66000, 61, 1, 1, 5, "bf16"), (2000, 40960, 8, 2, 0, 0, "bf16"), (1100, 41000, 128, 300, 0, 0, "bf16"),
    (300, 140000, 128, 3, 0, 0, "f16")])
def test_gradients_of_many_narrow_rows(B, L, D, mean, shift, pad, dtype):
    h, w = placed(normal(1, B, D), dtype, shift, pad), placed(normal(2, L, D, scale=2 * D ** -0.5), dtype, shift, pad)
    lists = random_lists(3, B, L, mean)
    lists[1], lists[2], lists[130] = [L - 1, L, -1, L - 1], [], [7] * 3
    weights = torch.rand(B, generator=torch.Generator().manual_seed(1)).cuda() * 3e-3
    weights[::7] = 0.0
    h[2] = NAN  # (a row without labels)
    c = Call(h, w, lists, normal(4, L), weights, dtype, shift=shift, pad=pad, before=9).run()
    bits = {k: v.clone() for k, v in c.outputs().items()}
    c.run()
    for k, v in c.outputs().items():
        assert torch.equal(v.nan_to_num(5.0), bits[k].nan_to_num(5.0)), k
    assert bool(c.lse[2].isnan()) and float(c.loss[2]) == 0.0
    c.lse[2] = 0.0
    h[2] = 0.0
    want = ref.label_loss(h, w, lists, c.bias, weights, dtype)
    for k, got in c.outputs().items():
        if k == "lse":
            got[2] = want["lse"][0][2]
        ref.near(got, *want[k], c.types[k], k)
    c.clean_h()
    c.clean_w()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_label_of_every_row_and_parts_of_the_outputs(dtype):
    # more targets in a workgroup's share than it lists
    B, L, D = 4200, 40000, 32
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.4), dtype)
    lists = [[5, 6 + i % 90, 5] for i in range(B)]
    c = Call(h, w, lists, normal(4, L), dtype=dtype, out="f32").run()
    c.check(lists, dtype)
    whole = {k: v.clone() for k, v in c.outputs().items()}
    for grads in (("dh",), ("dw",), ("db",)):
        part = Call(h, w, lists, normal(4, L), dtype=dtype, out="f32", grads=grads).run().outputs()
        assert set(part) == {"loss", "lse", *grads}
        for k, v in part.items():
            assert torch.equal(v, whole[k]), k


def test_many_narrow_rows_without_labels():
    # zeros, whatever the rows and the biases hold
    B, L, D = 300, 40000, 128
    h, w, bias = placed(normal(1, B, D), "bf16"), placed(normal(2, L, D), "bf16"), normal(4, L)
    h[3], bias[7], bias[8] = NAN, NAN, INF
    for weights in (None, torch.ones(B, device="cuda")):
        for lists in ([[] for _ in range(B)], [[-1, L] for _ in range(B)]):
            c = Call(h, w, lists, bias, weights, "bf16").run()
            for k, v in c.outputs().items():
                assert k == "lse" or bool((v == 0).all()), k


def test_many_narrow_rows_whose_logits_are_not_finite():
    B, L, D = 300, 40000, 64
    h, w, bias = placed(normal(1, B, D), "f16"), placed(normal(2, L, D, scale=0.3), "f16"), normal(4, L)
    lists = [[i] for i in range(B)]
    h[5] = NAN
    c = Call(h, w, lists, bias, dtype="f16").run()
    assert bool(c.loss[5].isnan()) and bool(c.dh[5].isnan().all()) and bool(c.dw.isnan().all()) and bool(c.db[:L].isnan().all())
    rest = [i for i in range(B) if i != 5]
    assert bool(c.loss[rest].isfinite().all()) and bool(c.dh[rest].isfinite().all())
    # labels of bias -inf have no probability
    h[5], bias[1000:1200] = 0.0, -INF
    c = Call(h, w, lists, bias, dtype="f16").run()
    c.check(lists, "f16")
    assert bool((c.dw[1000:1200] == 0).all()) and bool((c.db[1000:1200] == 0).all())


def test_medium_tiles_in_single_precision():
    # dz W in medium tiles with the labels split
    B, L, D = 995, 5000, 1208
    h, w = placed(normal(1, B, D), "f32"), placed(normal(2, L, D, scale=2 * D ** -0.5), "f32")
    lists = random_lists(3, B, L, 2)
    Call(h, w, lists, normal(4, L), dtype="f32").run().check(lists, "f32")
