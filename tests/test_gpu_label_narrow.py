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
