"""What the operators on label logits are timed on: the 4-bit label matrix and its
product, the k best labels under rules, and distillation from a teacher's top logits.

A case is a dict of plain values.  ``kind`` names the operator:

* ``quantize``: a matrix to MXFP4 (32 elements share a power-of-two scale, elements are
  e2m1) and back to the fp32 values that the codes stand for: ``asgd_fp4_quantize`` and
  ``asgd_fp4_dequantize``.
* ``logits``: hidden rows (bf16, or MXFP4) times a label matrix in MXFP4, plus the
  labels' bias: ``asgd_fp4_logits``.
* ``topk``: the k best labels of logit rows after penalties for labels already answered,
  biases and a mask of allowed labels, and the log-sum-exp of what was ranked:
  ``asgd_logits_topk``.
* ``distill``: the loss against a teacher's top logits and its gradient for every logit:
  ``asgd_distill``.

Sizes span the package's workloads: 1,000 to 670,091 labels, single rows to batches of
1,024, hidden width 128.  ``own`` selects the library's calls; the other branch of each
operator is its plain form in elementary torch operations.
"""
import math

import torch

own = False

H = 128
BLOCK = 32  # elements that share a scale
EMPTY = 2 ** 31 - 1  # the id of a place that no label fills
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------
def _quantize(name, rows, cols, dtype):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype}


def _logits(name, rows, labels, acts, out, bias):
    return {"name": name, "kind": "logits", "rows": rows, "labels": labels, "acts": acts, "out": out, "bias": bias}


def _topk(name, rows, labels, dtype, k, seen, bias, row_bias, mask):
    # seen, row_bias: entries per row on average; mask: share of labels allowed (0: no mask)
    return {"name": name, "kind": "topk", "rows": rows, "labels": labels, "dtype": dtype, "k": k, "seen": seen,
            "bias": bias, "row_bias": row_bias, "mask": mask}


def _distill(name, rows, labels, dtype, k, temperature):
    return {"name": name, "kind": "distill", "rows": rows, "labels": labels, "dtype": dtype, "k": k,
            "temperature": temperature}


def listed():
    return [
        # One batch of hidden rows before a product with a 4-bit label matrix: latency counts.
        _quantize("quantize hidden rows", 256, H, "bf16"),
        # The output layer of the wide-label model, laid out once for serving.
        _quantize("quantize label matrix", 670_091, H, "f32"),
        # A single request: every label's logit for one row, bound by reading the label matrix.
        _logits("logits one row", 1, 670_091, "bf16", "f32", True),
        # A served batch of the wide-feature model, both operands in 4 bits, 16-bit logits.
        _logits("logits batch", 256, 205_443, "fp4", "bf16", True),
        # An evaluation block of the wide-label model: bound by writing the logits.
        _logits("logits evaluation", 1_024, 670_091, "bf16", "f32", True),
        # A few rows of the smallest model, no rules but a prior: latency counts.
        _topk("topk few labels", 16, 1_000, "f32", 1, 0, True, 0, 0.0),
        # A single request over the wide label space, after 40 answers.
        _topk("topk one row", 1, 670_091, "f32", 5, 40, True, 8, 0.0),
        # A teacher's top logits for a batch: 16-bit logits, every rule.
        _topk("topk served batch", 256, 205_443, "bf16", 32, 75, True, 5, 0.9),
        # An evaluation block with the labels of each row's catalogue allowed.
        _topk("topk evaluation", 1_024, 670_091, "f32", 5, 5, True, 0, 0.5),
        # A step of the smallest model.
        _distill("distill tiny", 128, 1_000, "f32", 5, 2.0),
        # A step of the mid model, with as many teacher labels as a prediction gives.
        _distill("distill mid", 256, 30_000, "f32", 32, 1.0),
        # A step of the wide-label model, 16-bit logits and gradients.
        _distill("distill wide", 256, 670_091, "bf16", 32, 2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantize", "logits", "topk", "topk", "distill", "distill"))
    rows, labels = _log(rng, 1, 1_024), _log(rng, 1_000, 670_091)
    if kind == "quantize":
        case = _quantize("", _log(rng, 256, 670_091), BLOCK * rng.randint(1, 4), rng.choice(("f32", "bf16", "f16")))
    elif kind == "logits":
        case = _logits("", rows, labels, rng.choice(("bf16", "fp4")), rng.choice(("f32", "bf16", "f16")),
                       rng.random() < 0.7)
    elif kind == "topk":
        case = _topk("", rows, labels, rng.choice(("f32", "bf16", "f16")), rng.randint(1, 64), rng.choice((0, 5, 75)),
                     rng.random() < 0.5, rng.choice((0, 5)), rng.choice((0.0, 0.02, 0.5, 0.9)))
    else:
        case = _distill("", min(rows, 512), labels, rng.choice(("f32", "bf16", "f16")), rng.randint(1, 64),
                        rng.choice((1.0, 1.5, 4.0)))
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

    def lists(self, mean, rows, cols):
        """Ragged lists of ids, 0 to 2 * mean a row: (indptr, indices) as int32."""
        count = self.ints(0, 2 * mean + 1, rows)
        indptr = torch.zeros(rows + 1, dtype=torch.int64, device="cuda")
        indptr[1:] = count.cumsum(0)
        total = int(indptr[-1])
        return indptr.int(), self.ints(0, cols, total).int(), total


def _pow2(e):
    """2^e in fp32 for whole e in [-127, 127], from its bits (a library's pow may round)."""
    e = e.int()
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _encode(x):
    """MXFP4 codes and scales of fp32 rows: (uint8 [rows, cols / 2], uint8 [rows, cols / 32])."""
    rows, cols = x.shape
    b = x.reshape(rows, cols // BLOCK, BLOCK)
    e = torch.frexp(b.abs().amax(-1))[1].clamp(-124, 130) - 3
    y = b * _pow2(-e[..., None])
    grid = torch.tensor(E2M1, device=x.device)
    # nearest grid value (these inputs only have to be valid codes)
    code = torch.bucketize(y.abs().clamp(max=6.0), (grid[1:] + grid[:-1]) / 2)
    code = (code + 8 * (y < 0)).reshape(rows, cols // 2, 2).to(torch.uint8)
    return code[..., 0] | (code[..., 1] << 4), (e + 127).to(torch.uint8)


def _prepare_quantize(case, r):
    # values whose scale differs from block to block, as a trained layer's rows do
    x = r.normal(1.0, case["rows"], case["cols"]) * torch.exp(r.normal(1.0, case["rows"], 1))
    x = x.to(DTYPES[case["dtype"]])
    return {"x": x, "codes": torch.empty(case["rows"], case["cols"] // 2, dtype=torch.uint8, device="cuda"),
            "scales": torch.empty(case["rows"], case["cols"] // BLOCK, dtype=torch.uint8, device="cuda"),
            "values": torch.empty(case["rows"], case["cols"], device="cuda")}


def _prepare_logits(case, r):
    B, L = case["rows"], case["labels"]
    h = r.normal(0.5, B, H).clamp(min=0)  # hidden units after ReLU
    s = {"acts": case["acts"], "h": h.bfloat16()}
    if case["acts"] == "fp4":
        s["h_codes"], s["h_scales"] = _encode(h)
    s["codes"], s["scales"] = _encode(r.normal(0.15, L, H))
    s["bias"] = r.normal(0.3, L) if case["bias"] else None
    s["z"] = torch.empty(B, L, dtype=DTYPES[case["out"]], device="cuda")
    return s


def _prepare_topk(case, r):
    B, L, k = case["rows"], case["labels"], case["k"]
    s = {"k": k, "z": r.normal(2.0, B, L).to(DTYPES[case["dtype"]]), "repetition": 1.3, "frequency": 0.2,
         "presence": 0.4, "seen": None, "row_bias": None, "mask": None}
    s["bias"] = r.normal(0.3, L) if case["bias"] else None
    if case["seen"]:
        indptr, ids, n = r.lists(case["seen"], B, L)
        # a third of them are the labels that stand at the start of the vocabulary, so some repeat
        ids = torch.where(r.ints(0, 3, n) == 0, ids % 20, ids)
        s["seen"] = (indptr, ids, n)
    if case["row_bias"]:
        indptr, ids, n = r.lists(case["row_bias"], B, max(1, L // 64))
        # distinct ids in a row: each place of a list has a range of its own
        place = torch.arange(n, device="cuda") - indptr[:-1].long().repeat_interleave(indptr.diff().long())
        s["row_bias"] = (indptr, (ids * 64 % L // 16 * 16 + place % 16).clamp(max=L - 1).int(), r.normal(3.0, n), n)
    if case["mask"]:
        words = -(-L // 32)
        m = torch.zeros(B, words, dtype=torch.int32, device="cuda")
        for bit in range(32):
            on = torch.rand(B, words, generator=r.g, device="cuda") < case["mask"]
            m |= on.int() << bit
        m[49::50] = 0  # rows that allow nothing
        s["mask"] = m
    s["ids"] = torch.empty(B, k, dtype=torch.int32, device="cuda")
    s["scores"] = torch.empty(B, k, device="cuda")
    s["lse"] = torch.empty(B, device="cuda")
    return s


def _prepare_distill(case, r):
    B, L, k = case["rows"], case["labels"], case["k"]
    z = r.normal(2.0, B, L)
    # the teacher's labels: distinct in a row, and already likely under the student
    step = max(1, L // k)
    ids = torch.arange(k, device="cuda") * step + r.ints(0, step, B, k)
    t = (r.normal(1.5, B, k) + 9.0).sort(1, descending=True).values
    z.scatter_add_(1, ids, 0.5 * t + r.normal(1.0, B, k))
    ids = ids.int()
    # some rows of the teacher hold fewer labels, or none
    short = (torch.arange(k, device="cuda") >= k - r.ints(0, k + 1, B, 1)) & (r.ints(0, 8, B, 1) == 0)
    ids[short], t[short] = EMPTY, -math.inf
    return {"z": z.to(DTYPES[case["dtype"]]), "t_ids": ids, "t_logits": t, "T": case["temperature"],
            "loss": torch.empty(B, device="cuda"), "grad": torch.empty(B, L, dtype=DTYPES[case["dtype"]], device="cuda")}


def prepare(case, seed):
    make = {"quantize": _prepare_quantize, "logits": _prepare_logits, "topk": _prepare_topk,
            "distill": _prepare_distill}[case["kind"]]
    return dict(make(case, _Random(seed)), kind=case["kind"])


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------
def _plain_quantize(s):
    x = s["x"].float()
    b = x.view(x.shape[0], -1, BLOCK)
    e = (torch.frexp(b.abs().amax(-1, keepdim=True))[1] - 3).clamp(-127, 127)
    y = b * _pow2(-e)
    m = y.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    m = (torch.round(m / step) * step).clamp(max=6.0)
    return {"values": (torch.copysign(m, y) * _pow2(e)).view(x.shape)}


def _decode(codes, scales):
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    both = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1, BLOCK)
    return (table[both.int()] * _pow2(scales.int()[..., None] - 127)).view(codes.shape[0], -1)


def _plain_logits(s):
    h = _decode(s["h_codes"], s["h_scales"]) if s["acts"] == "fp4" else s["h"].float()
    z = h @ _decode(s["codes"], s["scales"]).T
    if s["bias"] is not None:
        z = z + s["bias"]
    return {"z": z.to(s["z"].dtype)}


def _rows_of(indptr, total):
    return torch.repeat_interleave(torch.arange(indptr.numel() - 1, device=indptr.device), indptr.diff().long(),
                                   output_size=total)


def _plain_topk(s):
    z, k = s["z"], s["k"]
    B, L = z.shape
    x = z.double()
    if s["seen"] is not None:
        indptr, ids, n = s["seen"]
        c = torch.zeros(B, L, dtype=torch.float64, device=z.device)
        c.index_put_((_rows_of(indptr, n), ids.long()), torch.ones(n, dtype=c.dtype, device=z.device), accumulate=True)
        pen = torch.where(x > 0, x / s["repetition"], x * s["repetition"]) - s["frequency"] * c - s["presence"]
        x = torch.where(c > 0, pen, x)
    if s["bias"] is not None:
        x = x + s["bias"].double()
    if s["row_bias"] is not None:
        indptr, ids, v, n = s["row_bias"]
        x[_rows_of(indptr, n), ids.long()] += v.double()
    score = x.float() + 0.0  # (a negative zero ties with zero)
    ok = ~score.isnan()
    if s["mask"] is not None:
        bits = (s["mask"][:, :, None] >> torch.arange(32, device=z.device, dtype=torch.int32)) & 1
        ok &= bits.view(B, -1)[:, :L].bool()
    # one key per label: by score, then by id
    bits = score.view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (order << 32) | (L - 1 - torch.arange(L, device=z.device))
    key = torch.where(ok, key, -(2 ** 63))
    best = key.topk(k, 1).values
    full = best != -(2 ** 63)
    at = (L - 1 - (best & 0xFFFFFFFF)).clamp(0, L - 1)
    ids = torch.where(full, at, EMPTY).int()
    scores = torch.where(full, score.gather(1, at), -math.inf)
    kept = torch.where(ok, score, -math.inf)
    top = kept.amax(1, keepdim=True)
    top = torch.where(top.isfinite(), top, 0.0)
    lse = top[:, 0] + (kept - top).exp().sum(1).log()
    return {"ids": ids, "scores": scores, "lse": lse}


def _plain_distill(s):
    T, dtype = s["T"], s["z"].dtype
    z = s["z"].float() / T
    B, L = z.shape
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    valid = (s["t_ids"] >= 0) & (s["t_ids"] < L) & s["t_logits"].isfinite()
    at = torch.where(valid, s["t_ids"], 0).long()
    t = torch.where(valid, s["t_logits"] / T, -math.inf)
    q = (t - t.amax(1, keepdim=True)).exp()
    q = torch.where(valid, q / q.sum(1, keepdim=True), 0.0)
    log_p = z.gather(1, at) - top - total.log()
    loss = T * T * torch.where(q > 0, q * (q.log() - log_p), 0.0).sum(1)
    some = valid.any(1, keepdim=True)
    g = torch.where(some, e / total * (T / B), 0.0)
    g.scatter_add_(1, at, q * (-T / B))
    return {"loss": loss, "grad": g.to(dtype)}


# ---------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------
def _own_quantize(s, asgd, stream):
    q = asgd.fp4_matrix(s["codes"], s["scales"])
    asgd.asgd_fp4_quantize(asgd.matrix(s["x"]), q, stream)
    asgd.asgd_fp4_dequantize(q, asgd.matrix(s["values"]), stream)
    return {"values": s["values"]}


def _own_logits(s, asgd, stream):
    h = asgd.fp4_matrix(s["h_codes"], s["h_scales"]) if s["acts"] == "fp4" else asgd.matrix(s["h"])
    asgd.asgd_fp4_logits(h, asgd.fp4_matrix(s["codes"], s["scales"]), asgd.matrix(s["z"]), bias=s["bias"],
                         stream=stream)
    return {"z": s["z"]}


def _own_csr(asgd, rows, cols, entries):
    if entries is None:
        return None
    values = entries[2] if len(entries) == 4 else None
    return asgd.asgd_csr(rows, cols, entries[-1], entries[0].data_ptr(), entries[1].data_ptr(),
                         None if values is None else values.data_ptr())


def _own_topk(s, asgd, stream):
    B, L = s["z"].shape
    if "workspace" not in s:
        s["workspace"] = torch.empty(asgd.asgd_logits_topk_workspace(B, L, s["k"]), dtype=torch.uint8, device="cuda")
    rules = asgd.logit_rules(bias=s["bias"], allowed=s["mask"], seen=_own_csr(asgd, B, L, s["seen"]),
                             repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                             row_bias=_own_csr(asgd, B, L, s["row_bias"]))
    asgd.asgd_logits_topk(asgd.matrix(s["z"]), s["k"], s["ids"], s["scores"], rules=rules, lse=s["lse"],
                          workspace=s["workspace"], stream=stream)
    return {"ids": s["ids"], "scores": s["scores"], "lse": s["lse"]}


def _own_distill(s, asgd, stream):
    B, L = s["z"].shape
    if "workspace" not in s:
        s["workspace"] = torch.empty(asgd.asgd_distill_workspace(B, L, s["t_ids"].shape[1]), dtype=torch.uint8,
                                     device="cuda")
    asgd.asgd_distill(asgd.matrix(s["z"]), s["t_ids"], s["t_logits"], s["T"], s["loss"], grad=asgd.matrix(s["grad"]),
                      workspace=s["workspace"], stream=stream)
    return {"loss": s["loss"], "grad": s["grad"]}


def run(state):
    if own:
        import paper_2110_07029_amd as asgd
        call = {"quantize": _own_quantize, "logits": _own_logits, "topk": _own_topk, "distill": _own_distill}
        return call[state["kind"]](state, asgd, torch.cuda.current_stream())
    return {"quantize": _plain_quantize, "logits": _plain_logits, "topk": _plain_topk,
            "distill": _plain_distill}[state["kind"]](state)


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    B = case["rows"]
    if case["kind"] == "quantize":
        n = B * case["cols"]
        # the matrix read, codes and scales written and read back, the values written
        return {"bytes": n * (SIZE[case["dtype"]] + 2 * 17 / 32 + 4), "flops": 4.0 * n}
    L = case["labels"]
    n = B * L
    if case["kind"] == "logits":
        acts = B * H * (17 / 32 if case["acts"] == "fp4" else 2)
        return {"bytes": L * H * 17 / 32 + (4 * L if case["bias"] else 0) + acts + n * SIZE[case["out"]],
                "flops": 2.0 * n * H}
    if case["kind"] == "topk":
        lists = B * (4 * case["seen"] + 8 * case["row_bias"])
        # a logit that is not allowed need not be read, but shares its memory line with others
        return {"bytes": n * SIZE[case["dtype"]] + (n / 8 if case["mask"] else 0) + (4 * L if case["bias"] else 0) +
                lists + 8 * B * case["k"] + 4 * B, "flops": 5.0 * n}
    return {"bytes": 2 * n * SIZE[case["dtype"]] + 8 * B * case["k"] + 4 * B, "flops": 8.0 * n}


# ---------------------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------------------
def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _values(codes, scales):
    codes = codes.long()
    low, high = codes % 16, codes // 16
    one = lambda c: torch.where(c % 8 < 2, (c % 2) * 0.5,  # noqa: E731
                                (1 + (c % 2) * 0.5) * _two_to((c % 8) // 2 - 1)) * (1 - 2.0 * (c // 8))
    v = torch.empty(codes.shape[0], codes.shape[1] * 2, dtype=torch.float64, device=codes.device)
    v[:, 0::2], v[:, 1::2] = one(low), one(high)
    return v * _two_to(scales.long() - 127).repeat_interleave(BLOCK, 1)


def _exact_quantize(s):
    x = s["x"].double()
    size = x.abs().view(x.shape[0], -1, BLOCK).amax(-1)
    # the scale puts the block's largest value into [4, 8)
    scale = _two_to(torch.floor(torch.log2(size)) - 2)
    scale = torch.where(size / scale < 4, scale / 2, torch.where(size / scale >= 8, scale * 2, scale))
    y = x / scale.repeat_interleave(BLOCK, 1)
    table = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    mid = (table[1:] + table[:-1]) / 2
    # a value on a midpoint goes to the even code
    code = torch.bucketize(y.abs(), mid)
    on = (code < 7) & (y.abs() == mid[code.clamp(max=6)])
    code = torch.where(on & (code % 2 == 1), code + 1, code)
    return {"values": table[code] * y.sign() * scale.repeat_interleave(BLOCK, 1)}


def _exact_logits(s):
    h = _values(s["h_codes"], s["h_scales"]) if s["acts"] == "fp4" else s["h"].double()
    z = torch.mm(h, _values(s["codes"], s["scales"]).T)
    return {"z": z if s["bias"] is None else z.add_(s["bias"].double())}


def _exact_topk(s):
    z, k = s["z"], s["k"]
    B, L = z.shape
    out = {"ids": torch.full((B, k), EMPTY, dtype=torch.int32, device=z.device),
           "scores": torch.full((B, k), -math.inf, dtype=torch.float64, device=z.device),
           "lse": torch.full((B,), -math.inf, dtype=torch.float64, device=z.device)}
    for r in range(B):
        x = z[r].double()
        if s["seen"] is not None:
            a, b = s["seen"][0][r:r + 2].tolist()
            ids, times = s["seen"][1][a:b].long().unique(return_counts=True)
            v = x[ids]
            v[v > 0] /= s["repetition"]
            v[x[ids] <= 0] *= s["repetition"]
            x[ids] = v - s["frequency"] * times - s["presence"]
        if s["bias"] is not None:
            x += s["bias"]
        if s["row_bias"] is not None:
            a, b = s["row_bias"][0][r:r + 2].tolist()
            x[s["row_bias"][1][a:b].long()] += s["row_bias"][2][a:b].double()
        x = x.float()  # the score is the rounded value: labels that round to the same one tie
        ids = torch.arange(L, device=z.device)
        if s["mask"] is not None:
            ids = ids[(s["mask"][r][ids // 32] >> (ids % 32).int()) % 2 != 0]
        got, at = x[ids].sort(descending=True, stable=True)
        n = min(k, ids.numel())
        out["ids"][r, :n], out["scores"][r, :n] = ids[at[:n]].int(), got[:n].double()
        if n:
            out["lse"][r] = torch.logsumexp(got.double(), 0)
    return out


def _exact_distill(s):
    T, z = s["T"], s["z"]
    B, L = z.shape
    loss = torch.zeros(B, dtype=torch.float64, device=z.device)
    grad = torch.zeros(B, L, dtype=torch.float64, device=z.device)
    for r in range(B):
        on = (s["t_ids"][r] < L) & (s["t_ids"][r] >= 0)
        if not bool(on.any()):
            continue
        ids = s["t_ids"][r][on].long()
        log_q = torch.log_softmax(s["t_logits"][r][on].double() / T, 0)
        log_p = torch.log_softmax(z[r].double() / T, 0)
        loss[r] = T * T * (log_q.exp() * (log_q - log_p[ids])).sum()
        target = torch.zeros(L, dtype=torch.float64, device=z.device).index_add_(0, ids, log_q.exp())
        grad[r] = (log_p.exp() - target) * T / B
    return {"loss": loss, "grad": grad}


def exact(case, seed):
    make = {"quantize": _exact_quantize, "logits": _exact_logits, "topk": _exact_topk, "distill": _exact_distill}
    return make[case["kind"]](prepare(case, seed))
