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
