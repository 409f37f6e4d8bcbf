"""What the operators for a network of the caller's own under the label layer are timed on:
dense layers, dropout and the label loss, with their gradients.

A case is a dict of plain values.  ``kind`` names the operator:

* ``loss``: softmax cross-entropy of hidden rows against a label matrix that the caller
  owns, with the gradients of rows, label matrix and biases, without logits in memory:
  ``asgd_label_loss``.
* ``dense``: a product with bias, activation, dropout and residual: ``asgd_dense``.
* ``dense_grad``: its gradients for input, weight and bias: ``asgd_dense_backward``.
* ``dropout``: dropout from a counter-based generator, plus a residual: ``asgd_dropout``.

Label counts, batches and the width 128 are those of the package's workloads; wider rows
stand for a dense network under the label layer.  ``own`` selects the library's calls; the
other branch of each operator is its plain form in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
ACTS = ("none", "relu", "gelu", "silu")


# ---------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------
def _loss(name, rows, labels, width, dtype, per_row, grads, bias, weights):
    # per_row: labels of a row on average (1: exactly one, and some rows without any)
    return {"name": name, "kind": "loss", "rows": rows, "labels": labels, "width": width, "dtype": dtype,
            "per_row": per_row, "grads": grads, "bias": bias, "weights": weights}


def _dense(name, kind, rows, outs, ins, dtype, act, drop, residual, keep, pad):
    # keep: the pre-activation is stored for a backward pass; pad: elements between rows
    return {"name": name, "kind": kind, "rows": rows, "outs": outs, "ins": ins, "dtype": dtype, "act": act,
            "drop": drop, "residual": residual, "keep": keep, "pad": pad}


def _dropout(name, rows, cols, dtype, drop, residual, pad):
    return {"name": name, "kind": "dropout", "rows": rows, "cols": cols, "dtype": dtype, "drop": drop,
            "residual": residual, "pad": pad}


def listed():
    return [
        # A step's loss over the smallest label set, fp32: launches and latency.
        _loss("loss tiny", 128, 1_000, 128, "f32", 3, True, True, False),
        # A step over the wide label set at the label layer's own width: bound by the label matrix.
        _loss("loss wide", 256, 670_091, 128, "bf16", 5, True, True, False),
        # One label a row under wide hidden rows, every row with a weight of its own: bound by the products.
        _loss("loss tokens", 4_096, 32_001, 2_048, "bf16", 1, True, False, True),
        # Held-out rows: the loss alone.
        _loss("loss evaluation", 1_024, 205_443, 128, "f16", 75, False, True, False),
        # A single request through a hidden layer: bound by the weight.
        _dense("dense one row", "dense", 1, 4_096, 1_024, "bf16", "gelu", 0.0, False, False, 0),
        # A training batch through a hidden layer, everything in the epilogue.
        _dense("dense batch", "dense", 8_192, 4_096, 1_024, "bf16", "gelu", 0.1, True, True, 0),
        # Ragged sizes in rows that are out of line.
        _dense("dense odd", "dense", 777, 1_001, 515, "f16", "silu", 0.2, True, True, 3),
        # The second hidden layer of the smallest model, fp32: latency.
        _dense("dense hidden grad", "dense_grad", 128, 128, 128, "f32", "relu", 0.0, False, True, 0),
        # The training batch's way back.
        _dense("dense batch grad", "dense_grad", 8_192, 4_096, 1_024, "bf16", "gelu", 0.1, False, True, 0),
        # A long fp32 batch with few units: the weight's gradient sums over many rows.
        _dense("dense long grad", "dense_grad", 16_384, 256, 200, "f32", "silu", 0.0, False, True, 0),
        # A batch of hidden rows: latency.
        _dropout("dropout hidden rows", 256, 128, "f32", 0.5, False, 0),
        # A block's output added to its residual: bound by memory.
        _dropout("dropout residual", 16_384, 4_096, "bf16", 0.1, True, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("loss", "loss", "loss", "dense", "dense", "dense_grad", "dense_grad", "dropout"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    drop = rng.choice((0.0, 0.1, 0.3))
    if kind == "loss":
        width = rng.choice((128, _log(rng, 32, 2_048), 8 * _log(rng, 8, 256)))
        labels = _log(rng, 1_000, min(670_091, 100_000_000 // width))
        most = min(4_096, 200_000_000 // labels, int((3e10 if dtype == "f32" else 2.6e11) // (labels * width)))
        case = _loss("", _log(rng, 1, max(1, most)), labels, width, dtype, rng.choice((1, 1, 5, 75)),
                     rng.random() < 0.75, rng.random() < 0.5, rng.random() < 0.5)
    elif kind == "dropout":
        rows = _log(rng, 1, 16_384)
        case = _dropout("", rows, _log(rng, 64, min(8_192, 64_000_000 // rows)), dtype, rng.choice((0.1, 0.3, 0.5)),
                        rng.random() < 0.5, rng.choice((0, 0, 1, 8)))
    else:
        outs, ins = (rng.choice((_log(rng, 64, 4_096), 8 * _log(rng, 16, 512))) for _ in range(2))
        most = min(16_384, int((3e9 if dtype == "f32" else 3e10) // (outs * ins)))
        case = _dense("", kind, _log(rng, 1, max(1, most)), outs, ins, dtype, rng.choice(ACTS), drop,
                      kind == "dense" and rng.random() < 0.5, kind == "dense_grad" or rng.random() < 0.5,
                      rng.choice((0, 0, 1, 8)))
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
class _Random:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, scale, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda") * scale

    def ints(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda")


def _padded(t, dtype, pad):
    """t as a matrix of the type whose rows lie `pad` elements apart."""
    if not pad:
        return t.to(dtype)
    big = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=dtype, device="cuda")
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def _room(rows, cols, dtype, pad):
    return torch.empty(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _prepare_loss(case, r):
    B, L, D = case["rows"], case["labels"], case["width"]
    dtype = DTYPES[case["dtype"]]
    w = r.normal(2.0 / math.sqrt(D), L, D)
    if case["per_row"] == 1:
        count = (r.ints(0, 16, B) > 0).long()
        if B == 1:
            count[:] = 1
    else:
        count = r.ints(0, 2 * case["per_row"] + 1, B)
    most = max(1, 2 * case["per_row"])
    indptr = torch.zeros(B + 1, dtype=torch.int64, device="cuda")
    indptr[1:] = count.cumsum(0)
    n = int(indptr[-1])
    row = torch.repeat_interleave(torch.arange(B, device="cuda"), count, output_size=n)
    place = torch.arange(n, device="cuda") - indptr[row]
    ids = place * (L // most) + r.ints(0, L // most, n)  # distinct in a row, in order
    # hidden rows that lean to their labels, as after some training
    h = r.normal(1.0, B, D)
    lean = torch.zeros(B, D, device="cuda")
    lean.index_add_(0, row, w[ids])
    h += 3.0 * lean / (lean.norm(dim=1, keepdim=True) + 1e-6)
    s = {"h": h.to(dtype), "w": w.to(dtype), "labels": L, "indptr": indptr.int(), "ids": ids.int(), "nnz": n}
    s["bias"] = r.normal(0.3, L) if case["bias"] else None
    s["weights"] = torch.rand(B, generator=r.g, device="cuda") / B if case["weights"] else None
    s["loss"], s["lse"] = (torch.empty(B, device="cuda") for _ in range(2))
    s["grads"] = case["grads"]
    if case["grads"]:
        s["dh"], s["dw"], s["db"] = torch.empty_like(s["h"]), torch.empty_like(s["w"]), torch.empty(L, device="cuda")
    return s


def _prepare_dense(case, r):
    M, N, K, pad = case["rows"], case["outs"], case["ins"], case["pad"]
    dtype = DTYPES[case["dtype"]]
    x, w, bias = r.normal(1.0, M, K), r.normal(1.0 / math.sqrt(K), N, K), r.normal(0.3, N)
    s = {"x": _padded(x, dtype, pad), "w": _padded(w, dtype, pad), "bias": bias, "act": case["act"],
         "drop": case["drop"], "seed": int(r.ints(0, 2 ** 62, 1)), "res": None}
    if case["kind"] == "dense":
        if case["residual"]:
            s["res"] = _padded(r.normal(1.0, M, N), dtype, pad)
        s["pre"] = _room(M, N, dtype, pad) if case["keep"] else None
        s["y"] = _room(M, N, dtype, pad)
    else:
        s["dy"] = _padded(r.normal(1.0, M, N), dtype, pad)
        # what the forward pass left
        s["pre"] = _padded(s["x"].float() @ s["w"].float().T + bias, dtype, pad)
        s["dx"], s["dw"], s["db"] = _room(M, K, dtype, pad), _room(N, K, dtype, pad), torch.empty(N, device="cuda")
    return s


def _prepare_dropout(case, r):
    M, N, pad = case["rows"], case["cols"], case["pad"]
    dtype = DTYPES[case["dtype"]]
    return {"x": _padded(r.normal(1.0, M, N), dtype, pad), "drop": case["drop"], "seed": int(r.ints(0, 2 ** 62, 1)),
            "res": _padded(r.normal(1.0, M, N), dtype, pad) if case["residual"] else None, "y": _room(M, N, dtype, pad)}


def prepare(case, seed):
    make = {"loss": _prepare_loss, "dense": _prepare_dense, "dense_grad": _prepare_dense, "dropout": _prepare_dropout}
    return dict(make[case["kind"]](case, _Random(seed)), kind=case["kind"])


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------
def _signed(v):
    return v - 2 ** 64 if v >= 2 ** 63 else v


def _shifted(v, n):
    return (v >> n) & ((1 << (64 - n)) - 1)


def _splitmix(v):
    """splitmix64 of 64-bit words held in int64 (products wrap)."""
    v = v + _signed(0x9E3779B97F4A7C15)
    v = (v ^ _shifted(v, 30)) * _signed(0xBF58476D1CE4E5B9)
    v = (v ^ _shifted(v, 27)) * _signed(0x94D049BB133111EB)
    return v ^ _shifted(v, 31)


def _kept(rows, cols, drop, seed, device):
    """1 / (1 - drop) where an element stays, 0 where it is dropped.  Neighbours in a row
    share the 64 bits of their counter, the even column has the low half."""
    key = _splitmix(torch.tensor([seed], dtype=torch.int64, device=device))
    pairs = (cols + 1) // 2
    at = (torch.arange(rows, device=device)[:, None] << 22) | torch.arange(pairs, device=device)
    bits = _splitmix(key ^ at)
    both = torch.stack((bits & 0xFFFFFFFF, _shifted(bits, 32)), -1).view(rows, 2 * pairs)[:, :cols]
    return (both >= math.floor(drop * 2 ** 32)).float() * (1.0 / (1.0 - drop))


def _act(name, a):
    if name == "relu":
        return a.clamp(min=0)
    if name == "gelu":
        return 0.5 * a * (1 + torch.erf(a * math.sqrt(0.5)))
    if name == "silu":
        return a / (1 + (-a).exp())
    return a


def _slope(name, a):
    if name == "relu":
        return (a > 0).float()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(a * math.sqrt(0.5))) + a * (-0.5 * a * a).exp() * (1 / math.sqrt(2 * math.pi))
    if name == "silu":
        g = 1 / (1 + (-a).exp())
        return g * (1 + a * (1 - g))
    return torch.ones_like(a)


def _plain_loss(s):
    h, w = s["h"].float(), s["w"].float()
    z = h @ w.T
    if s["bias"] is not None:
        z += s["bias"]
    B = h.shape[0]
    count = s["indptr"].diff().long()
    row = torch.repeat_interleave(torch.arange(B, device=h.device), count, output_size=s["nnz"])
    ids = s["ids"].long()
    share = 1.0 / count.clamp(min=1)
    live = (count > 0).float()
    top = z.amax(1)
    e = (z - top[:, None]).exp()
    total = e.sum(1)
    lse = top + total.log()
    target = torch.zeros(B, device=h.device).index_put_((row,), z[row, ids], accumulate=True)
    loss = (lse - target * share) * live
    out = {"loss": loss, "lse": lse}
    if s["grads"]:
        weight = torch.full_like(live, 1.0 / B) if s["weights"] is None else s["weights"]
        dz = e.mul_((live / total)[:, None])
        dz.index_put_((row, ids), -share[row], accumulate=True)
        dz *= weight[:, None]
        out["dh"] = (dz @ w).to(s["h"].dtype)
        out["dw"] = (dz.T @ h).to(s["w"].dtype)
        out["db"] = dz.sum(0)
    return out


def _plain_dense(s):
    a = s["x"].float() @ s["w"].float().T + s["bias"]
    y = _act(s["act"], a)
    if s["drop"]:
        y = y * _kept(*y.shape, s["drop"], s["seed"], y.device)
    if s["res"] is not None:
        y = y + s["res"].float()
    out = {"y": y.to(s["y"].dtype)}
    if s["pre"] is not None:
        out["pre"] = a.to(s["pre"].dtype)
    return out


def _plain_dense_grad(s):
    d = s["dy"].float() * _slope(s["act"], s["pre"].float())
    if s["drop"]:
        d = d * _kept(*d.shape, s["drop"], s["seed"], d.device)
    return {"dx": (d @ s["w"].float()).to(s["dx"].dtype), "dw": (d.T @ s["x"].float()).to(s["dw"].dtype), "db": d.sum(0)}


def _plain_dropout(s):
    y = s["x"].float() * _kept(*s["x"].shape, s["drop"], s["seed"], s["x"].device)
    if s["res"] is not None:
        y = y + s["res"].float()
    return {"y": y.to(s["y"].dtype)}


# ---------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------
def _workspace(s, need):
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(1, need()), dtype=torch.uint8, device="cuda")
    return s["workspace"]


def _own_loss(s, asgd, stream):
    h, w = asgd.matrix(s["h"]), asgd.matrix(s["w"])
    y = asgd.asgd_csr(s["h"].shape[0], s["labels"], s["nnz"], s["indptr"].data_ptr(), s["ids"].data_ptr(), None)
    ws = _workspace(s, lambda: asgd.asgd_label_loss_workspace(h, w, s["grads"]))
    out = {"loss": s["loss"], "lse": s["lse"]}
    if not s["grads"]:
        asgd.asgd_label_loss(h, w, y, s["loss"], bias=s["bias"], lse=s["lse"], workspace=ws, stream=stream)
        return out
    asgd.asgd_label_loss(h, w, y, s["loss"], bias=s["bias"], weights=s["weights"], lse=s["lse"],
                         dh=asgd.matrix(s["dh"]), dw=asgd.matrix(s["dw"]), db=s["db"], workspace=ws, stream=stream)
    return dict(out, dh=s["dh"], dw=s["dw"], db=s["db"])


def _own_epilogue(s, asgd, bias):
    acts = {"none": asgd.ASGD_ACT_NONE, "relu": asgd.ASGD_ACT_RELU, "gelu": asgd.ASGD_ACT_GELU, "silu": asgd.ASGD_ACT_SILU}
    return asgd.dense_epilogue(bias=bias, act=acts[s["act"]], drop=s["drop"], seed=s["seed"],
                               residual=None if s["res"] is None else asgd.matrix(s["res"]))


def _own_dense(s, asgd, stream):
    x, w = asgd.matrix(s["x"]), asgd.matrix(s["w"])
    asgd.asgd_dense(x, w, asgd.matrix(s["y"]), epilogue=_own_epilogue(s, asgd, s["bias"]),
                    pre=None if s["pre"] is None else asgd.matrix(s["pre"]),
                    workspace=_workspace(s, lambda: asgd.asgd_dense_workspace(x, w)), stream=stream)
    return {"y": s["y"]} if s["pre"] is None else {"y": s["y"], "pre": s["pre"]}


def _own_dense_grad(s, asgd, stream):
    x, w = asgd.matrix(s["x"]), asgd.matrix(s["w"])
    asgd.asgd_dense_backward(asgd.matrix(s["dy"]), x, w, pre=asgd.matrix(s["pre"]), epilogue=_own_epilogue(s, asgd, None),
                             dx=asgd.matrix(s["dx"]), dw=asgd.matrix(s["dw"]), db=s["db"],
                             workspace=_workspace(s, lambda: asgd.asgd_dense_backward_workspace(x, w)), stream=stream)
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_dropout(s, asgd, stream):
    asgd.asgd_dropout(asgd.matrix(s["x"]), s["drop"], s["seed"], asgd.matrix(s["y"]),
                      residual=None if s["res"] is None else asgd.matrix(s["res"]), stream=stream)
    return {"y": s["y"]}


def run(state):
    if own:
        import paper_2110_07029_amd as asgd
        call = {"loss": _own_loss, "dense": _own_dense, "dense_grad": _own_dense_grad, "dropout": _own_dropout}
        return call[state["kind"]](state, asgd, torch.cuda.current_stream())
    return {"loss": _plain_loss, "dense": _plain_dense, "dense_grad": _plain_dense_grad,
            "dropout": _plain_dropout}[state["kind"]](state)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    size = SIZE[case["dtype"]]
    if case["kind"] == "loss":
        B, L, D = case["rows"], case["labels"], case["width"]
        once = size * (B + L) * D + 4 * B * (case["per_row"] + 1) + 8 * B + (4 * L if case["bias"] else 0)
        if not case["grads"]:
            return {"bytes": once, "flops": 2.0 * B * L * D}
        # rows, label matrix and biases read, their gradients written; the product and its two gradients
        return {"bytes": once + size * (B + L) * D + 4 * L, "flops": 6.0 * B * L * D}
    if case["kind"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": size * n * (3 if case["residual"] else 2), "flops": 12.0 * n}
    M, N, K = case["rows"], case["outs"], case["ins"]
    if case["kind"] == "dense":
        return {"bytes": size * ((M + N) * K + M * N * (1 + case["residual"] + case["keep"])) + 4 * N,
                "flops": 2.0 * M * N * K}
    return {"bytes": size * (2 * (M + N) * K + 2 * M * N) + 4 * N, "flops": 4.0 * M * N * K}


# ---------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------
def _stays(rows, cols, drop, seed):
    """Which elements stay: each element's own 32 bits, from unsigned 64-bit words on the host."""
    u = np.uint64

    def mix(v):
        v = v + u(0x9E3779B97F4A7C15)
        v = (v ^ (v >> u(30))) * u(0xBF58476D1CE4E5B9)
        v = (v ^ (v >> u(27))) * u(0x94D049BB133111EB)
        return v ^ (v >> u(31))

    with np.errstate(over="ignore"):
        key = mix(np.array([seed], u))
        j = np.arange(cols, dtype=u)
        out = np.empty((rows, cols), bool)
        for i in range(0, rows, 512):
            r = np.arange(i, min(rows, i + 512), dtype=u)[:, None]
            word = mix(key ^ (r * u(1 << 22) + j // u(2)))
            out[i:i + 512] = ((word >> (u(32) * (j % u(2)))) & u(0xFFFFFFFF)) >= u(int(drop * 2.0 ** 32))
    return torch.from_numpy(out).cuda()


def _exact_loss(s):
    h, w = s["h"].double(), s["w"].double()
    B = h.shape[0]
    z = torch.mm(h, w.T)
    if s["bias"] is not None:
        z.add_(s["bias"].double())
    lse = torch.logsumexp(z, 1)
    ends, ids = s["indptr"].tolist(), s["ids"].long()
    loss = torch.zeros(B, dtype=torch.float64, device=h.device)
    z_at = [z[i, ids[a:b]] for i, (a, b) in enumerate(zip(ends, ends[1:]))]
    for i, v in enumerate(z_at):
        if v.numel():
            loss[i] = lse[i] - v.mean()
    out = {"loss": loss, "lse": lse}
    if s["grads"]:
        z.sub_(lse[:, None]).exp_()
        for i, v in enumerate(z_at):
            if v.numel():
                z[i].index_add_(0, ids[ends[i]:ends[i + 1]], torch.full_like(v, -1.0 / v.numel()))
            else:
                z[i] = 0.0
        z.mul_(1.0 / B if s["weights"] is None else s["weights"].double()[:, None])
        out.update(dh=torch.mm(z, w), dw=torch.mm(z.T.contiguous(), h), db=z.sum(0))
    return out


def _exact_dense(s):
    a = torch.mm(s["x"].double(), s["w"].double().T) + s["bias"].double()
    y = {"none": lambda v: v, "relu": torch.relu, "gelu": lambda v: v * 0.5 * torch.erfc(-v / math.sqrt(2)),
         "silu": lambda v: v * torch.sigmoid(v)}[s["act"]](a)
    if s["drop"]:
        y = torch.where(_stays(*y.shape, s["drop"], s["seed"]), y / (1 - s["drop"]), 0.0)
    if s["res"] is not None:
        y = y + s["res"].double()
    return {"y": y} if s["pre"] is None else {"y": y, "pre": a}


def _exact_dense_grad(s):
    a = s["pre"].double()
    if s["act"] == "relu":
        f = torch.where(a > 0, 1.0, 0.0).double()
    elif s["act"] == "gelu":
        f = 0.5 * torch.erfc(-a / math.sqrt(2)) + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    elif s["act"] == "silu":
        f = torch.sigmoid(a) + a * torch.sigmoid(a) * torch.sigmoid(-a)
    else:
        f = torch.ones_like(a)
    d = s["dy"].double() * f
    if s["drop"]:
        d = torch.where(_stays(*d.shape, s["drop"], s["seed"]), d / (1 - s["drop"]), 0.0)
    return {"dx": torch.mm(d, s["w"].double()), "dw": torch.mm(d.T.contiguous(), s["x"].double()), "db": d.sum(0)}


def _exact_dropout(s):
    y = torch.where(_stays(*s["x"].shape, s["drop"], s["seed"]), s["x"].double() / (1 - s["drop"]), 0.0)
    return {"y": y if s["res"] is None else y + s["res"].double()}


def exact(case, seed):
    make = {"loss": _exact_loss, "dense": _exact_dense, "dense_grad": _exact_dense_grad, "dropout": _exact_dropout}
    return make[case["kind"]](prepare(case, seed))
