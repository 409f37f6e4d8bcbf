"""Dense layers, dropout and the label loss in 64 bits, with bounds on what fp32 sums and one rounding per
output may be off.  Everything runs on the device of its inputs."""
import math

import numpy as np
import torch

import paper_2110_07029_amd as asgd

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# Half a step relative to a value; and what is lost near zero: fp16 has steps of 2^-24 there, the other two have
# normal values down to 2^-126, below which matrix cores and the base-2 exponential may return zero.
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
U = 2.0 ** -24
ACTS = {"none": asgd.ASGD_ACT_NONE, "relu": asgd.ASGD_ACT_RELU, "gelu": asgd.ASGD_ACT_GELU, "silu": asgd.ASGD_ACT_SILU}


def kept(rows, cols, p, seed):
    """bool [rows, cols] (numpy): which elements stay, from the documented bits; rows: their number or some of them."""
    u = np.uint64

    def mix(v):
        v = v + u(0x9E3779B97F4A7C15)
        v = (v ^ (v >> u(30))) * u(0xBF58476D1CE4E5B9)
        v = (v ^ (v >> u(27))) * u(0x94D049BB133111EB)
        return v ^ (v >> u(31))

    with np.errstate(over="ignore"):
        i, j = np.array(range(rows) if isinstance(rows, int) else rows, dtype=u)[:, None], np.arange(cols, dtype=u)
        word = mix(mix(np.array([seed], u)) ^ (i * u(2 ** 22) + j // u(2)))
    return ((word >> (u(32) * (j % u(2)))) & u(2 ** 32 - 1)) >= u(math.floor(p * 2.0 ** 32))


def scale_of(p):
    return float(np.float32(1.0 / (1.0 - p)))


def mask(rows, cols, p, seed, device):
    return torch.from_numpy(kept(rows, cols, p, seed)).to(device).double() * scale_of(p)


def act(name, a):
    if name == "relu":
        return torch.relu(a)
    if name == "gelu":
        return a * 0.5 * torch.erfc(-a / math.sqrt(2))
    return a * torch.sigmoid(a) if name == "silu" else a


def slope(name, a):
    if name == "relu":
        return (a > 0).double()
    if name == "gelu":
        return 0.5 * torch.erfc(-a / math.sqrt(2)) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = torch.sigmoid(a)
        return s + a * s * (1 - s)
    return torch.ones_like(a)


def rounded(t, dtype):
    return HALF[dtype] * t.abs() + TINY[dtype]


def dense(x, w, bias=None, name="none", p=0.0, seed=0, res=None):
    """(a, |error of a| bound, y, |error of y| bound) before outputs are rounded.  Sums of k products in any order are
    within (k + 2) 2^-24 of the sum of absolute values; act changes by at most 1.13 times what a does, and its own
    evaluation is good to some 8 steps of max(|a|, |y|)."""
    x, w = x.double(), w.double()
    k = x.shape[1]
    b = torch.zeros(w.shape[0], dtype=torch.float64, device=x.device) if bias is None else bias.double()
    a = x @ w.T + b
    ea = (k + 2) * U * (x.abs() @ w.abs().T + b.abs())
    y, ey = act(name, a), 1.13 * ea
    if name != "none":
        ey = ey + 8 * U * a.abs()
    if p:
        m = mask(*a.shape, p, seed, x.device)
        y, ey = y * m, ey * m + U * (y * m).abs()
    if res is not None:
        y = y + res.double()
        ey = ey + U * y.abs()
    return a, ea, y, ey


def dense_grad(dy, x, w, pre, dtype, name="none", p=0.0, seed=0):
    """{dx, dw, db} and bounds: dA is good to some 16 steps and rounded once to the operands' type."""
    x, w, dy = x.double(), w.double(), dy.double()
    da = dy if name == "none" else dy * slope(name, pre.double())
    e = 16 * U * dy.abs()
    if p:
        m = mask(*dy.shape, p, seed, dy.device)
        da, e = da * m, e * m + U * (da * m).abs()
    M, N = dy.shape
    er = e + rounded(da, dtype)
    return {"dx": (da @ w, er @ w.abs() + (N + 2) * U * (da.abs() @ w.abs())),
            "dw": (da.T @ x, er.T @ x.abs() + (M + 2) * U * (da.abs().T @ x.abs())),
            "db": (da.sum(0), e.sum(0) + (M + 2) * U * da.abs().sum(0))}


def label_loss(h, w, lists, bias, weights, dtype):
    """{loss, lse, dh, dw, db} and bounds.  lists: ids per row, any."""
    h, w = h.double(), w.double()
    B, D = h.shape
    L = w.shape[0]
    dev = h.device
    live = [[i for i in r if 0 <= i < L] for r in lists]
    n = torch.tensor([len(r) for r in live], dtype=torch.float64, device=dev)
    on = n > 0
    hz = torch.where(on[:, None], h, 0.0)  # (what rows without labels hold reaches no gradient)
    b = torch.zeros(L, dtype=torch.float64, device=dev) if bias is None else bias.double()
    z = h @ w.T + b
    ez = (D + 2) * U * (h.abs() @ w.abs().T + torch.where(b.isfinite(), b.abs(), 0.0))
    lse = torch.logsumexp(z, 1)
    # exponentials of x are good to (|x| + 2) 2^-23, of which e^x |x| sums to ln L at most
    elog = (200 + 2 * L / 32768 + 4 * math.log(max(2, L))) * U
    elog = elog + 2 * U * torch.where(lse.isfinite(), lse.abs(), 0.0)
    p = (z - lse[:, None]).exp()
    err_lse = torch.where(p > 0, ez, 0.0).amax(1) + elog
    t = torch.zeros(B, L, dtype=torch.float64, device=dev)
    flat = [(i, j) for i, r in enumerate(live) for j in r]
    loss, eloss = torch.zeros_like(lse), torch.zeros_like(lse)
    if flat:
        rows, ids = (torch.tensor(v, device=dev) for v in zip(*flat))
        t.index_put_((rows, ids), (1.0 / n)[rows], accumulate=True)
        mean = torch.zeros_like(lse).index_add_(0, rows, z[rows, ids] / n[rows])
        size = torch.zeros_like(lse).index_add_(0, rows, z[rows, ids].abs() / n[rows])
        off = torch.zeros_like(lse).index_add_(0, rows, ez[rows, ids] / n[rows])
        loss = torch.where(on, lse - mean, 0.0)
        eloss = torch.where(on, elog + err_lse + off + (n + 8) * U * (size + lse.abs()), 0.0)
    weight = torch.full_like(lse, 1.0 / B) if weights is None else weights.double()
    wt = torch.where(on, weight, 0.0)[:, None]
    dz = torch.where(on[:, None], wt * (p - t), 0.0)
    far = torch.where(p > 0, (z - lse[:, None]).abs(), 0.0)
    e = wt.abs() * (p * (torch.where(p > 0, ez, 0.0) + err_lse[:, None] + (2 * far + 8) * U) + 8 * U * (p + t))
    top = wt.abs().amax()
    # (exponentials below 2^-126 are zero, and so are factors of a product below it: 2^-126 each, and so once more)
    e = torch.where(on[:, None], e + 2.0 ** -126 * (wt.abs() + top), 0.0)
    er = e + HALF[dtype] * dz.abs() + (TINY[dtype] * 2.0 ** -15 * top if dtype == "f16" else 0.0)
    out = {"loss": (loss, eloss), "lse": (lse, err_lse + elog)}
    wa, ha = w.abs(), hz.abs()
    out["dh"] = (dz @ w, er @ wa + (L + 66) * U * (dz.abs() @ wa))
    out["dw"] = (dz.T @ hz, er.T @ ha + (B + 2) * U * (dz.abs().T @ ha))
    out["db"] = (dz.sum(0), e.sum(0) + (B + 4) * U * dz.abs().sum(0))
    return out


def near(got, want, bound, dtype, what):
    """got is want to within the bound and one rounding to its type."""
    got = got.double()
    tol = bound + rounded(want.abs() + bound, dtype)
    bad = ~((got - want).abs() <= tol) & ~((got == want) | (got.isnan() & want.isnan()))
    if bool(bad.any()):
        at = bad.nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: "
                             f"{got[tuple(at)].item()!r} for {want[tuple(at)].item()!r} +- {tol[tuple(at)].item()!r}")
