"""The label loss over rows of 16 bits up to 128 wide, where single labels or rows decide: what single precision must still
hold, masks, infinities and lists that a few labels fill."""
import pytest
import torch

import layers_ref as ref
import paper_2110_07029_amd as asgd
from gpu_util import flush
from test_gpu_label_loss import Call, random_lists
from test_gpu_layers import INF, NAN, normal, placed

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _say(request):
    flush(request.node.name)
    asgd.load()


def bias_gradient(h, w, lists, bias):
    """db in 64 bits, a range of labels at a time."""
    B, L = h.shape[0], w.shape[0]
    hd = h.double()
    n = torch.tensor([len(r) for r in lists], device="cuda").double()
    lse = torch.full((B,), -INF, dtype=torch.float64, device="cuda")
    step = 100_000
    z_of = [(a, min(L, a + step)) for a in range(0, L, step)]

    def logits(a, b):
        return hd @ w[a:b].double().T + (bias[a:b].double() if bias is not None else 0.0)
    for a, b in z_of:
        lse = torch.logaddexp(lse, torch.logsumexp(logits(a, b), 1))
    db = torch.cat([((logits(a, b) - lse[:, None]).exp() * (n > 0)[:, None]).sum(0) for a, b in z_of])
    rows = torch.repeat_interleave(torch.arange(B, device="cuda"), n.long())
    ids = torch.tensor([i for r in lists for i in r], device="cuda")
    return db.index_add_(0, ids, -1.0 / n[rows]) / B


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [0.05, 0.18])
def test_bias_gradient_of_many_tiles_a_workgroup(scale, dtype):
    # 256 live rows and 41 tiles of labels in each workgroup.  db is formed in fp32 throughout: its norm is that of the labels
    # that stand in lists, of which each goes through 1/n and its product with the weight (2 roundings), the difference to p
    # (1), sums over 32 lanes (5) and 8 waves (up to 8) and the scale (1): 17 roundings of either sign, 2^-24 / sqrt 3 at most in
    # the mean square, 2.4 2^-24 together.  The exponentials' own error has no part in that: all labels' p are 4 % of the norm.
    B, L = 256, 670_091
    h, w = placed(normal(1, B, 128), dtype), placed(normal(2, L, 128, scale=scale), dtype)
    bias = normal(4, L, scale=0.3)
    lists = [r or [i] for i, r in enumerate(random_lists(3, B, L, 5))]
    c = Call(h, w, lists, bias, dtype=dtype).run()
    first = {k: v.clone() for k, v in c.outputs().items()}
    want = bias_gradient(h, w, lists, bias)
    for _ in range(12):
        got = c.db[:L].double()
        assert float((got - want).norm()) <= 3e-7 * float(want.norm())
        # (one label's logit formed from a piece of another's row moves its db by about a tenth of the labels' mean, 1 / L)
        assert float((got - want).abs().amax()) <= 1e-3 / L + 17 * ref.U * float(want.abs().amax())
        c.run()
        for k, v in c.outputs().items():
            assert torch.equal(v, first[k]), k


LOWEST = torch.finfo(torch.float32).min


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("low", [LOWEST, -1e30, -1e10, -1e9])
@pytest.mark.parametrize("B,L,D", [(100, 70_000, 128), (300, 70_000, 128), (300, 45_000, 61), (40, 3_000, 64)])
def test_labels_masked_by_very_low_biases(B, L, D, low, dtype):
    # whole tiles of them: the first of each range of tiles, runs, and all but one label
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=2 * D ** -0.5), dtype)
    lane = torch.arange(L, device="cuda") // 64
    for masked in (lane % 3 == 0, lane % 3 != 0, lane > 0, lane < L // 64):
        bias = torch.where(masked, low, normal(4, L))
        free = (~masked).nonzero()[:, 0].tolist()
        lists = [[free[(7 * i) % len(free)], free[(11 * i + 1) % len(free)]] for i in range(B)]
        lists[3] = []
        Call(h, w, lists, bias, dtype=dtype).run().check(lists, dtype)
        alone = Call(h, w, lists, bias, dtype=dtype, grads=()).run()
        alone.check(lists, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("low", [LOWEST, -1e10, -300.0, -INF])
@pytest.mark.parametrize("B,L", [(100, 70_000), (300, 70_000), (256, 20_001)])
def test_one_label_that_is_certain(B, L, low, dtype):
    # p is 1 and 0 exactly, so nothing is left of the gradients
    h, w = placed(normal(1, B, 128), dtype), placed(normal(2, L, 128, scale=0.1), dtype)
    for one in (0, 12_345, L - 1):
        bias = torch.full((L,), low, device="cuda")
        bias[one] = 0.5
        c = Call(h, w, [[one]] * B, bias, dtype=dtype).run()
        c.check([[one]] * B, dtype)
        for k in ("dh", "dw", "db"):
            assert bool((c.outputs()[k] == 0).all()), k


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,L", [(100, 70_000), (300, 70_000)])
def test_all_labels_masked_alike(B, L, dtype):
    # logits of the lowest value whatever h and w are: as likely as each other
    h, w = placed(normal(1, B, 128), dtype), placed(normal(2, L, 128, scale=0.1), dtype)
    lists = [[i, 2 * i + 500] for i in range(B)]
    c = Call(h, w, lists, torch.full((L,), LOWEST, device="cuda"), dtype=dtype).run()
    assert bool((c.lse[:B] == LOWEST).all())
    want = torch.full((L,), 1.0 / L, dtype=torch.float64, device="cuda")
    ids = torch.tensor(lists, device="cuda").flatten()
    want.index_add_(0, ids, torch.full_like(ids, -0.5 / B, dtype=torch.float64))
    # sums of B equal terms that are good to 8 steps
    assert bool(((c.db[:L].double() - want).abs() <= (B + 8) * ref.U * (1.0 / L + want.abs())).all())
    assert all(bool(c.outputs()[k].isfinite().all()) for k in ("dh", "dw", "db"))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,L", [(100, 70_000), (300, 45_000), (40, 3_000)])
def test_logits_far_from_zero(B, L, dtype):
    # a bias that all labels share moves the log-sum-exp and nothing else; 2^14 leaves logits of few bits exact
    g = torch.Generator().manual_seed(1)
    h, w = (torch.randint(-2, 3, s, generator=g).float() for s in ((B, 128), (L, 128)))
    h, w = placed(h.cuda(), dtype), placed((w / 8).cuda(), dtype)
    lists = random_lists(3, B, L, 3)
    near = Call(h, w, lists, torch.zeros(L, device="cuda"), dtype=dtype).run().outputs()
    for shift in (-16384.0, 16384.0, -131072.0):
        far = Call(h, w, lists, torch.full((L,), shift, device="cuda"), dtype=dtype).run().outputs()
        for k in ("dh", "dw", "db"):
            assert torch.equal(far[k], near[k]), (shift, k)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,L", [(100, 70_000), (300, 41_000), (320, 41_000), (500, 70_001)])
def test_infinities_in_a_label_reach_no_row_without_labels(B, L, dtype):
    # A -inf against a column of ones makes a label's logit -inf in every live row, as a bias of -inf does.  Rows without
    # labels (and those that fill up the last tile of 64) take part in nothing, whatever 0 times that is.
    h, w = placed(normal(1, B, 128), dtype), placed(normal(2, L, 128, scale=0.1), dtype)
    h[:, 5] = 1.0
    lists = [r or [77] for r in random_lists(3, B, L, 3)]
    lists[7], lists[B - 1] = [], [-1, L]
    bias = normal(4, L)
    for rows in (lists, [r or [3] for r in lists]):
        rows = [[i for i in r if i not in (40, 1000, L - 1)] or [2] * bool(r) for r in rows]
        masked = bias.clone()
        for j in (40, 1000, L - 1):
            masked[j] = -INF
        want = {k: v.clone() for k, v in Call(h, w, rows, masked, dtype=dtype).run().outputs().items()}
        sick = w.clone()
        sick[40, 5] = sick[1000, 5] = sick[L - 1, 5] = -INF
        got = Call(h, sick, rows, bias, dtype=dtype).run().outputs()
        for k in ("loss", "lse", "dw", "db"):
            assert torch.equal(got[k], want[k]) and bool(want[k].isfinite().all()), k
        other = [c for c in range(128) if c != 5]  # (0 times the infinity itself is NaN, in the column that has it)
        assert torch.equal(got["dh"][:, other], want["dh"][:, other])


def test_a_label_that_is_not_finite_in_live_rows():
    # NaN of a live row stays NaN: 0 weights do not hide it
    B, L = 300, 41_000
    h, w = placed(normal(1, B, 128), "bf16"), placed(normal(2, L, 128, scale=0.1), "bf16")
    lists, bias = [[i] for i in range(B)], normal(4, L)
    lists[9] = []
    weights = torch.full((B,), 1e-3, device="cuda")
    weights[8] = 0.0
    bias[500] = NAN
    c = Call(h, w, lists, bias, weights, "bf16").run()
    live = [i for i in range(B) if i != 9]
    assert bool(c.loss[live].isnan().all()) and float(c.loss[9]) == 0.0 and bool((c.dh[9] == 0).all())
    assert bool(c.dw.isnan().all()) and bool(c.db[:L].isnan().all()) and bool(c.dh[live].isnan().all())


def crowded(kind, B, L):
    """Lists of which a few labels, rows or tiles have far more than their part."""
    lists = [[(37 * i) % L] for i in range(B)]
    if kind == "labels":  # some in every row: more than a workgroup lists for all of its rows, in one block of 128 and in its neighbour
        for i, r in enumerate(lists):
            r += [130, 131 + i % 40, 200, 255] + [300] * (i % 2)
    elif kind == "tile":  # a tile of rows that names a whole block of labels, and a tile of labels that 128 rows name
        for i in range(64, 128):
            lists[i] = list(range(256, 384))
        for i in range(256, 384):
            lists[i] = list(range(6400, 6464))
    elif kind == "range":  # rows that name the first labels, each many
        for i in range(256):
            lists[i] = list(range(i % 7, 448, 13))
    else:  # repeats fill a list as well
        for i in range(0, B, 3):
            lists[i] += [500] * 20 + [L - 1] * (i % 5)
    lists[5], lists[B - 2] = [], [-1, L]
    return lists


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["labels", "tile", "range", "repeats"])
@pytest.mark.parametrize("B,L", [(1501, 70_000), (700, 140_000)])
def test_lists_that_a_few_labels_or_rows_fill(B, L, kind, dtype):
    h, w = placed(normal(1, B, 32), dtype), placed(normal(2, L, 32, scale=0.4), dtype)
    lists = crowded(kind, B, L)
    c = Call(h, w, lists, normal(4, L), dtype=dtype, out="f32", before=3).run()
    first = {k: v.clone() for k, v in c.outputs().items()}
    c.check(lists, dtype)
    c.run()
    for k, v in c.outputs().items():
        assert torch.equal(v, first[k]), k


def test_lists_of_many_tiles_in_groups():
    # more than 255 tiles of rows, so that tiles share a place in the list; every row names a label of one block
    B, L = 20_000, 41_000
    g = torch.Generator().manual_seed(1)
    h, w = (torch.randint(-2, 3, s, generator=g).float() for s in ((B, 8), (L, 8)))
    h, w = placed(h.cuda(), "bf16"), placed((w / 4).cuda(), "bf16")
    lists = [[640 + i % 100, (31 * i) % L] for i in range(B)]
    c = Call(h, w, lists, None, None, "bf16", out="f32").run()
    z = h.double() @ w.double().T
    p = z.sub_(torch.logsumexp(z, 1)[:, None]).exp_()
    rows = torch.arange(B, device="cuda").repeat_interleave(2)
    p.index_put_((rows, torch.tensor(lists, device="cuda").flatten()), torch.full_like(rows, -0.5, dtype=torch.float64), accumulate=True)
    # one rounding of dz to 8 bits, and what sums of B (or L) terms round
    size = p.abs()
    for got, want, most, n in ((c.dw, p.T @ h.double(), size.T @ h.double().abs(), B), (c.dh, p @ w.double(), size @ w.double().abs(), L)):
        tol = ((2.0 ** -8 + 2.0 ** -18) * most + (n + 66) * ref.U * most) / B
        assert bool(((got.double() - want / B).abs() <= tol).all())
    db, most = p.sum(0) / B, size.sum(0) / B
    assert bool(((c.db[:L].double() - db).abs() <= 2.0 ** -18 * most).all())


def test_crowded_labels_cost_little_more_than_even_ones():
    # 2,048 rows of 75 labels out of 205,443: evenly drawn a workgroup's share has 380, here some have 2,200 to 6,300.  Looking
    # through the rows' lists at every tile of such a share took 1.9 times the even lists' time; in windows it is 1.1.
    B, L, K = 2048, 205_443, 75
    h, w = placed(normal(1, B, 128), "bf16"), placed(normal(2, L, 128, scale=0.18), "bf16")
    g = torch.Generator().manual_seed(1)
    even = torch.randint(0, L, (B, K), generator=g)
    crowded_ids = even.clone()
    crowded_ids[:, :3] = torch.tensor([512 * 7 + 1, 512 * 7 + 130, 512 * 7 + 131])
    crowded_ids[:, 3] = 512 * 40 + 5
    crowded_ids[::12, 4] = 512 * 40 + 6
    best = []
    for ids in (even, crowded_ids):
        c = Call(h, w, ids.tolist(), dtype="bf16")
        took = []
        for _ in range(9):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            c.run()
            b.record()
            torch.cuda.synchronize()
            took.append(a.elapsed_time(b))
        best.append(min(took))
    assert best[1] <= 1.6 * best[0], best


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_the_largest_weight_of_many_rows(dtype):
    # more rows than are looked at in one go; lists that begin with ids that do not count, and the largest weights on rows
    # without any that does
    B, L, D = 5001, 300, 40
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=0.3), dtype)
    lists = [[-1] * (i % 9) + [L] * (i % 3) + [i % L] * (i % 4 != 1) for i in range(B)]
    up = torch.arange(1, B + 1, dtype=torch.float32).cuda() * 1e-7
    for weights, largest in ((up, B - 2), (up.flip(0), 0), (-up, 4096 + 7)):
        weights = weights.clone()
        weights[4097] = 1e30  # (4097 % 4 == 1: no labels)
        weights[5] = INF
        weights[largest] = -3e-3
        c = Call(h, w, lists, normal(4, L), weights, dtype).run()
        weights[4097] = weights[5] = 0.0  # (the reference needs finite ones)
        c.check(lists, dtype)


# rows of integers of a few bits: their logits are multiples of 1/16 below 2^6, exact in every order of summation
PATHS = [(200, 70_000, 128, "bf16"), (256, 30_001, 64, "f16"), (4000, 41_000, 64, "bf16"), (1000, 45_000, 128, "f16"),
         (300, 3_000, 264, "bf16"), (700, 9_001, 136, "f16"), (300, 3_000, 128, "f32"), (1100, 5_000, 40, "f32"), (20, 20_000, 200, "f32")]


def few_bits(B, L, D, dtype):
    g = torch.Generator().manual_seed(1)
    h, w = (torch.randint(-2, 3, s, generator=g).float() for s in ((B, D), (L, D)))
    return placed(h.cuda(), dtype), placed((w / 16).cuda(), dtype)


@pytest.mark.parametrize("B,L,D,dtype", PATHS)
def test_probabilities_of_exact_logits(B, L, D, dtype):
    # Every row's label is 0, so db of the others is the mean of their probabilities.  One is good to |z - top| + 4 half steps
    # (the argument's product, the exponential, 1 / sum and two products), 12 or so: of either sign from row to row, so
    # 12 / sqrt 20 of them are left of 20 rows or more; sums over rows round some 20 times, of either sign.  Together
    # 7 half steps of 2^-24, 4.2e-7, in the norm.
    h, w = few_bits(B, L, D, dtype)
    c = Call(h, w, [[0]] * B, None, dtype=dtype).run()
    z = h.double() @ w.double().T
    z_top, lse = z.amax(1), torch.logsumexp(z, 1)
    want = z.sub_(lse[:, None]).exp_().sum(0) / B
    off = (c.db[1:L].double() - want[1:]).norm() / want[1:].norm()
    assert float(off) <= 7 * ref.U, float(off)
    # (sums of tens of thousands of exponentials, in parts: 20 half steps of 1 at most)
    assert bool(((c.lse[:B].double() - lse).abs() <= ref.U * (lse.abs() + 20)).all())
    # In the mean square: lse lies between 8 and 16, where half a step is 8 2^-24, as much over sqrt 3 (4.62) for any part of it;
    # the logarithm of the sum, below 8, is off by a step of its own at most (8, where it is above 4); the sum by 12 half
    # steps, of either sign, of each of the exponentials that make it up, 1 together: sqrt(4.62^2 + 8^2 + 1) = 9.3
    assert bool((lse > 8).all()) and bool((lse < 16).all()) and bool((lse - z_top < 8).all())
    assert float((c.lse[:B].double() - lse).norm()) <= 9.3 * ref.U * B ** 0.5


@pytest.mark.parametrize("B,L,D,dtype", PATHS)
def test_probabilities_do_not_go_through_the_rounded_log_sum_exp(B, L, D, dtype):
    # 2^14 in every bias leaves logits exact and takes 10 bits of the log-sum-exp's fraction
    h, w = few_bits(B, L, D, dtype)
    lists = random_lists(3, B, L, 3)
    near = Call(h, w, lists, torch.zeros(L, device="cuda"), dtype=dtype).run().outputs()
    far = Call(h, w, lists, torch.full((L,), 16384.0, device="cuda"), dtype=dtype).run().outputs()
    for k in ("dh", "dw", "db"):
        assert torch.equal(far[k], near[k]), k


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 264), ("f32", 64)])
def test_several_masked_labels_in_a_list(dtype, D):
    # the mean of their logits is finite though the sum is not
    B, L = 30, 500
    h, w = placed(normal(1, B, D, scale=0.1), dtype), placed(normal(2, L, D, scale=0.1), dtype)
    bias = normal(4, L)
    bias[:300] = LOWEST
    lists = [list(range(1 + 9 * i)) for i in range(B)]
    lists[7] = [3] * 65_535
    c = Call(h, w, lists, bias, dtype=dtype, grads=()).run()
    assert bool(c.loss[:B].isfinite().all()) and bool(c.lse[:B].isfinite().all())
    want = torch.tensor([-float(bias[r].double().mean()) for r in lists], dtype=torch.float64, device="cuda")
    # (n sums and a product with 1/n: n + 2 half steps)
    n = torch.tensor([len(r) for r in lists], device="cuda")
    assert bool(((c.loss[:B].double() - want).abs() <= (n + 2) * ref.U * want.abs()).all())
    # and where all labels are masked, lse and the mean are both the lowest value
    c = Call(h, w, [r or [1] for r in lists], torch.full((L,), LOWEST, device="cuda"), dtype=dtype, grads=()).run()
    assert bool((c.lse[:B] == LOWEST).all()) and bool((c.loss[:B].abs() <= 65_537 * ref.U * -LOWEST).all())


@pytest.mark.parametrize("low", [LOWEST, -1e10])
@pytest.mark.parametrize("B,L,D,dtype", [(300, 9_000, 136, "bf16"), (64, 5_000, 264, "f16"), (200, 5_000, 64, "f32"), (3, 30_000, 200, "f32")])
def test_wider_rows_under_the_same_masks(B, L, D, dtype, low):
    h, w = placed(normal(1, B, D), dtype), placed(normal(2, L, D, scale=2 * D ** -0.5), dtype)
    block = torch.arange(L, device="cuda") // 64
    for masked in (block % 3 == 0, block > 0, block < L // 64):
        bias = torch.where(masked, low, normal(4, L))
        free = (~masked).nonzero()[:, 0].tolist()
        lists = [[free[(7 * i) % len(free)], free[(11 * i + 1) % len(free)]] for i in range(B)]
        lists[1] = []
        Call(h, w, lists, bias, dtype=dtype).run().check(lists, dtype)
    lists = [[i, 2 * i + 500] for i in range(B)]
    c = Call(h, w, lists, torch.full((L,), LOWEST, device="cuda"), dtype=dtype).run()
    want = torch.full((L,), 1.0 / L, dtype=torch.float64, device="cuda")
    ids = torch.tensor(lists, device="cuda").flatten()
    want.index_add_(0, ids, torch.full_like(ids, -0.5 / B, dtype=torch.float64))
    assert bool(((c.db[:L].double() - want).abs() <= (B + 8) * ref.U * (1.0 / L + want.abs())).all())
