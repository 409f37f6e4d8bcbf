"""The operators over label logits on the GPU, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import logits_ref as ref
import paper_2110_07029_amd as asgd
from gpu_util import flush

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
U = 2.0 ** -24  # half a step of fp32


@pytest.fixture(autouse=True)
def _say(request):
    flush(request.node.name)
    asgd.load()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(ref.DTYPES[dtype])).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


def strided(a, dtype, shift, pad):
    """a on the GPU as a view that starts `shift` elements into rows of its width + pad."""
    rows, cols = a.shape
    big = torch.full((rows, cols + pad), NAN, dtype=ref.DTYPES[dtype], device="cuda")
    v = big[:, shift:shift + cols]
    v.copy_(torch.from_numpy(a))
    return v


def scratch(n):
    # (an odd value in every byte: nothing may rely on what is there)
    return torch.full((max(n, 1),), 0xA5, dtype=torch.uint8, device="cuda")


def lists(rows, cols=None, values=False):
    """Lists per row as (asgd_csr, tensors that it borrows)."""
    ids = [r[0] if values else r for r in rows]
    indptr = np.concatenate([[0], np.cumsum([len(r) for r in ids])]).astype(np.int32)
    flat = np.concatenate([np.asarray(r, np.int32) for r in ids] + [np.zeros(0, np.int32)]).astype(np.int32)
    keep = [dev(indptr), dev(np.append(flat, 0).astype(np.int32))]
    if values:
        keep.append(dev(np.append(np.concatenate([np.asarray(r[1], np.float32) for r in rows]), 0).astype(np.float32)))
    return asgd.asgd_csr(len(rows), cols, len(flat), *[t.data_ptr() for t in keep]), keep


# ---------------------------------------------------------------- MXFP4
def awkward(rows, cols, seed):
    """Values over the whole range of scales, with midpoints, zeros and single extremes."""
    r = np.random.default_rng(seed)
    x = r.normal(0, 1, (rows, cols)) * np.exp2(r.integers(-20, 20, (rows, 1)))
    half = r.random((rows, cols)) < 0.3
    grid = np.arange(0, 33) / 4.0
    x = np.where(half, r.choice(grid, (rows, cols)) * np.exp2(r.integers(-4, 4, (rows, 1))) * r.choice([-1, 1], (rows, cols)), x)
    x[r.random((rows, cols)) < 0.1] = 0.0
    x[rows // 2, :32] = 0.0
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,shift,pad", [(1, 32, 0, 0), (3, 64, 1, 5), (257, 128, 0, 0), (130, 128, 3, 7),
                                                 (64, 4096, 8, 8), (33, 160, 0, 1)])
def test_quantize_and_back_are_exact(dtype, rows, cols, shift, pad):
    t = strided(awkward(rows, cols, rows + cols), dtype, shift, pad)
    codes = torch.full((rows, cols // 2), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, cols // 32), 0xEE, dtype=torch.uint8, device="cuda")
    q = asgd.fp4_matrix(codes, scales)
    asgd.asgd_fp4_quantize(asgd.matrix(t), q, torch.cuda.current_stream())
    v, c, s = ref.quantize(host(t))
    assert np.array_equal(scales.cpu().numpy(), s)
    got = ref.unpack(codes.cpu().numpy())
    # (the code of a zero may carry either sign)
    assert np.array_equal(np.where(got == 8, 0, got), np.where(c == 8, 0, c))
    for out in ("f32", "bf16", "f16"):
        big = torch.full((rows, cols + pad), 7.0, dtype=ref.DTYPES[out], device="cuda")
        view = big[:, shift:shift + cols]
        asgd.asgd_fp4_dequantize(q, asgd.matrix(view), torch.cuda.current_stream())
        want = torch.from_numpy(v).to(ref.DTYPES[out])  # one rounding
        # (an element beyond fp16 is infinite, and its block NaN)
        assert torch.allclose(view.cpu(), want, rtol=0, atol=0, equal_nan=True)
        rest = torch.cat((big[:, :shift], big[:, shift + cols:]), 1)
        assert bool((rest == 7.0).all())


def test_quantize_extremes():
    x = np.zeros((12, 32), np.float32)
    big = float(np.finfo(np.float32).max)
    x[0, 5] = INF
    x[1, 31] = NAN
    x[2, 0], x[2, 1] = -INF, NAN
    x[3, :3] = big, -big, 1.0
    x[4, :3] = 1e-45, -3e-45, 0.0                     # subnormal fp32
    x[5, :3] = 2.0 ** -126, 2.0 ** -127, 2.0 ** -128
    x[6, 7] = -5.0
    x[7, :4] = 2.0 ** 127, 2.0 ** 125 * 1.25, 2.0 ** 100, -(2.0 ** 126)
    x[8, :] = -0.0
    x[9, :3] = 3.9999998, 4.0, 2.0
    x[10, :2] = 7.9999995, 0.25
    x[11, :2] = 2.0 ** -125, 2.0 ** -129
    v, c, s = ref.quantize(x.astype(np.float64))
    codes = torch.empty((12, 16), dtype=torch.uint8, device="cuda")
    scales = torch.empty((12, 1), dtype=torch.uint8, device="cuda")
    q = asgd.fp4_matrix(codes, scales)
    asgd.asgd_fp4_quantize(asgd.matrix(dev(x)), q)
    out = torch.empty((12, 32), device="cuda")
    asgd.asgd_fp4_dequantize(q, asgd.matrix(out))
    assert np.array_equal(scales.cpu().numpy(), s)
    got = host(out)
    assert np.array_equal(np.isnan(got), np.isnan(v))
    ok = ~np.isnan(v)
    assert np.array_equal(got[ok], v.astype(np.float32)[ok])


def test_dequantize_every_code_and_scale():
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1)).reshape(256, 256)
    scales = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 16))
    q = asgd.fp4_matrix(dev(codes), s := dev(scales))
    c = dev(codes)
    q = asgd.fp4_matrix(c, s)
    out = torch.empty((256, 512), device="cuda")
    asgd.asgd_fp4_dequantize(q, asgd.matrix(out))
    want = ref.values_of(codes, scales).astype(np.float32)
    got = out.cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[:255], want[:255])


def label_matrix(L, seed, spread=3):
    r = np.random.default_rng(seed)
    codes = r.integers(0, 256, (L, 64)).astype(np.uint8)
    scales = (127 - 3 + r.integers(-spread, spread + 1, (L, 4))).astype(np.uint8)
    return codes, scales


def product_bound(a, w, bias):
    """128 exact products added in fp32 in any order and, at worst, cut off instead of rounded
    (one step an addition), then the bias and the final rounding (half a step each)."""
    mag = np.abs(a) @ np.abs(w).T
    z = a @ w.T
    return 128 * 2 * U * mag + 2 * U * (np.abs(z) + np.abs(bias))


@pytest.mark.parametrize("acts", ["bf16", "fp4"])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,L,shift,pad,with_bias", [(1, 1, 0, 0, True), (1, 33, 0, 0, False), (2, 31, 1, 3, True),
                                                     (31, 1000, 0, 0, True), (33, 1001, 2, 9, True),
                                                     (64, 257, 0, 0, False), (129, 4099, 1, 1, True),
                                                     (5, 30_000, 0, 0, True), (300, 515, 0, 5, True),
                                                     (16, 700, 3, 4, True), (17, 700, 1, 1, True)])
def test_fp4_logits(acts, out, B, L, shift, pad, with_bias):
    r = np.random.default_rng(B * 7 + L)
    codes, scales = label_matrix(L, L)
    bias = r.normal(0, 1, L).astype(np.float32) if with_bias else np.zeros(L, np.float32)
    w = ref.values_of(codes, scales)
    keep = [dev(codes), dev(scales), dev(bias)]
    if acts == "fp4":
        hc, hs = label_matrix(B, B + 1)
        h = ref.values_of(hc, hs)
        keep += [dev(hc), dev(hs)]
        arg = asgd.fp4_matrix(*keep[3:])
    else:
        t = strided(np.maximum(r.normal(0, 1, (B, 128)), 0), "bf16", 8, 16)
        h = host(t)
        keep.append(t)
        arg = asgd.matrix(t)
    big = torch.full((B, L + pad), 7.0, dtype=ref.DTYPES[out], device="cuda")
    z = big[:, shift:shift + L]
    asgd.asgd_fp4_logits(arg, asgd.fp4_matrix(*keep[:2]), asgd.matrix(z), bias=keep[2] if with_bias else None,
                         stream=torch.cuda.current_stream())
    want = h @ w.T + bias
    bound = product_bound(h, w, bias)
    bound = bound + (ref.half_step(np.abs(want) + bound, out) if out != "f32" else 0)
    err = np.abs(host(z) - want)
    assert (err <= bound).all(), (err - bound).max()
    assert bool((torch.cat((big[:, :shift], big[:, shift + L:]), 1) == 7.0).all())


def test_fp4_logits_of_nan_blocks_stay_in_their_rows_and_labels():
    codes, scales = label_matrix(70, 1)
    scales[5, 2] = 255
    hc, hs = label_matrix(40, 2)
    hs[33, 0] = 255
    keep = [dev(v) for v in (codes, scales, hc, hs)]
    z = torch.empty((40, 70), device="cuda")
    asgd.asgd_fp4_logits(asgd.fp4_matrix(*keep[2:]), asgd.fp4_matrix(*keep[:2]), asgd.matrix(z))
    nan = np.isnan(host(z))
    want = np.zeros((40, 70), bool)
    want[33], want[:, 5] = True, True
    assert np.array_equal(nan, want)
    # bf16 rows, many and few: NaN and infinities of a row stay in it
    h = torch.ones((40, 128), dtype=torch.bfloat16, device="cuda")
    h[3, 7], h[4, 100] = NAN, INF
    for n in (40, 20):
        z = torch.empty((n, 70), device="cuda")
        asgd.asgd_fp4_logits(asgd.matrix(h[:n]), asgd.fp4_matrix(*keep[:2]), asgd.matrix(z))
        got = host(z)
        want = np.zeros((n, 70), bool)
        want[3], want[:, 5] = True, True
        weights = ref.values_of(codes, scales)[:, 100]
        want[4] |= weights == 0  # 0 * inf
        assert np.array_equal(np.isnan(got), want)
        ok = ~want[4]
        assert np.array_equal(got[4][ok], np.sign(weights[ok]) * INF)


# ---------------------------------------------------------------- ranking under rules
def rank(z, k, rules=None, stream=None, with_scores=True, with_lse=True):
    B, L = z.shape
    ids = torch.full((B, k), -7, dtype=torch.int32, device="cuda")
    sc = torch.full((B, k), 7.0, device="cuda") if with_scores else None
    lse = torch.full((B,), 7.0, device="cuda") if with_lse else None
    ws = scratch(asgd.asgd_logits_topk_workspace(B, L, k))
    asgd.asgd_logits_topk(asgd.matrix(z), k, ids, sc, rules=rules, lse=lse, workspace=ws,
                          stream=torch.cuda.current_stream() if stream is None else stream)
    return ids, sc, lse


def check_rank(got, s, k, allowed=None, L=None):
    ids, top, lse = ref.topk(s, k, allowed)
    assert np.array_equal(got[0].cpu().numpy(), ids)
    assert np.array_equal(got[1].cpu().numpy(), top)
    g = host(got[2])
    assert np.array_equal(np.isinf(g), np.isinf(lse)) and not np.isnan(g).any()
    inf = np.isinf(lse)
    assert np.array_equal(g[inf], lse[inf])
    bound = ref.lse_bound(lse, s.shape[1])
    err = np.abs(g[~inf] - lse[~inf])
    assert (err <= bound[~inf]).all(), err.max()


def words(allowed):
    B, L = allowed.shape
    bits = np.zeros((B, (L + 31) // 32 * 32), np.uint64)
    bits[:, :L] = allowed
    w = (bits.reshape(B, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return w.astype(np.uint32).view(np.int32)


RANKS = [(1, 1, 1), (1, 5, 8), (3, 63, 4), (2, 64, 64), (5, 1000, 1), (16, 1000, 33), (7, 4097, 5), (1, 30_000, 32),
         (2, 30_001, 64), (1, 205_443, 5), (40, 8191, 7), (2100, 130, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,L,k", RANKS)
def test_topk_without_rules(dtype, B, L, k):
    r = np.random.default_rng(B + L + k)
    z = strided(r.normal(0, 2, (B, L)), dtype, (B + k) % 9, 9)
    got = rank(z, k)
    check_rank(got, ref.scores(host(z)), k)
    only = rank(z, k, with_scores=False, with_lse=False)
    assert torch.equal(only[0], got[0])


def random_rules(r, B, L, seen_mean, bias, row_bias, mask, shared=False):
    o, keep, kw = {}, [], {}
    if bias:
        o["bias"] = r.normal(0, 1, L).astype(np.float32)
        keep.append(dev(o["bias"]))
        kw["bias"] = keep[-1]
    if seen_mean:
        # a few ids many times, ids out of range, empty lists
        o["seen"] = [np.where(r.random(n) < 0.3, r.integers(0, min(L, 5), n), r.integers(-3, L + 3, n))
                     for n in r.integers(0, 2 * seen_mean + 1, B)]
        c, t = lists(o["seen"], L)
        keep.append(t)
        kw.update(seen=c, repetition=1.3, frequency=0.2, presence=0.4)
        o.update(repetition=1.3, frequency=0.2, presence=0.4)
    if row_bias:
        o["row_bias"] = [(r.integers(-2, L + 2, n), r.normal(0, 4, n).astype(np.float32))
                         for n in r.integers(0, 2 * row_bias + 1, B)]
        c, t = lists(o["row_bias"], L, values=True)
        keep.append(t)
        kw["row_bias"] = c
    allowed = None
    if mask:
        allowed = r.random((1 if shared else B, L)) < mask
        if not shared:
            allowed[B // 2] = False
        w = dev(words(allowed))
        keep.append(w)
        kw["allowed"] = w[0] if shared else w
        allowed = np.broadcast_to(allowed, (B, L))
    return o, asgd.logit_rules(**kw), allowed, keep


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,L,k,seen,bias,row_bias,mask,shared", [
    (1, 1, 1, 2, True, 1, 0.5, False), (3, 40, 64, 10, True, 5, 0.6, False), (4, 1000, 5, 20, False, 0, 0.0, False),
    (4, 1000, 5, 0, True, 0, 0.02, False), (9, 4096, 16, 0, False, 4, 0.5, True), (1, 30_000, 5, 300, True, 8, 0.9, True),
    (3, 30_011, 32, 2000, True, 60, 0.01, False), (2, 205_443, 64, 75, True, 5, 0.9, False),
    (50, 8193, 3, 75, False, 5, 0.0, False), (2100, 67, 2, 3, True, 2, 0.5, False)])
def test_topk_with_rules(dtype, B, L, k, seen, bias, row_bias, mask, shared):
    r = np.random.default_rng(B * L + k)
    z = strided(r.normal(0, 2, (B, L)), dtype, (L + k) % 7, 7)
    o, rules, allowed, keep = random_rules(r, B, L, seen, bias, row_bias, mask, shared)
    check_rank(rank(z, k, rules), ref.scores(host(z), **o), k, allowed)


ORDERS = ["ascending", "descending", "equal", "minus infinity", "lowest", "two values", "zeros of both signs", "nan",
          "infinite", "mostly nan"]


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("L,k", [(50, 64), (9000, 5), (40_000, 64)])
def test_topk_of_awkward_rows(order, L, k):
    r = np.random.default_rng(L)
    x = np.sort(r.normal(0, 1, (2, L)).astype(np.float32), 1)
    x = {"ascending": x, "descending": x[:, ::-1], "equal": np.full_like(x, 0.25), "minus infinity": np.full_like(x, -INF),
         "lowest": np.full_like(x, np.finfo(np.float32).min), "two values": np.where(r.random(x.shape) < 0.5, 1.0, -1.0),
         "zeros of both signs": np.where(r.random(x.shape) < 0.5, 0.0, -0.0),
         "nan": np.where(r.random(x.shape) < 0.1, NAN, x), "infinite": np.where(r.random(x.shape) < 0.02, INF, x),
         "mostly nan": np.full_like(x, NAN)}[order].astype(np.float32).copy()
    if order == "infinite":
        x[:, 3] = -INF
    if order == "mostly nan":
        x[0, L // 2] = -1.0
    check_rank(rank(dev(x), k), ref.scores(x) + np.float32(0), k)
    # the same where a mask leaves some of them, with NaN and infinities behind it
    allowed = r.random(x.shape) < 0.3
    y = x.copy()
    y[~allowed] = r.choice([NAN, INF, -INF, 3e38], int((~allowed).sum()))
    w = dev(words(allowed))
    check_rank(rank(dev(y), k, asgd.logit_rules(allowed=w)), ref.scores(x) + np.float32(0), k, allowed)


def test_topk_seen_ids_that_repeat_and_cancel():
    # one label seen 70,000 times, biases of infinities, penalties that turn the order around
    L = 5000
    x = np.linspace(-3, 3, L, dtype=np.float32)[None].copy()
    seen = [np.concatenate([np.full(70_000, L - 1), np.arange(L - 40, L - 1), [L - 2]])]
    row_bias = [(np.array([7, 8, 7, 9, 9]), np.array([50, INF, 2, -INF, 4], np.float32))]
    c, keep = lists(seen, L)
    c2, keep2 = lists(row_bias, L, values=True)
    kw = dict(repetition=1.7, frequency=0.001, presence=-0.5)
    got = rank(dev(x), 64, asgd.logit_rules(seen=c, row_bias=c2, **kw))
    check_rank(got, ref.scores(x, seen=seen, row_bias=row_bias, **kw), 64)


def test_topk_negative_zeros_tie_with_zeros():
    L = 3000
    r = np.random.default_rng(1)
    z = np.where(r.random((2, L)) < 0.5, -0.0, 0.0).astype(np.float32)
    bias = np.where(r.random(L) < 0.7, -0.0, 0.0).astype(np.float32)
    b = dev(bias)
    got = rank(dev(z), 64, asgd.logit_rules(bias=b))
    assert np.array_equal(got[0].cpu().numpy(), np.tile(np.arange(64), (2, 1)))
    assert bool((got[1] == 0).all())


def test_topk_lists_with_malformed_indptr_are_read_inside_their_entries():
    L = 300
    x = np.random.default_rng(0).normal(0, 1, (4, L)).astype(np.float32)
    ids = dev(np.array([5, 6, 7, 8], np.int32))
    # entries [0, 4): rows reach before, past and across them
    ip = dev(np.array([0, 900, -50, 2, 4], np.int32))
    c = asgd.asgd_csr(4, L, 4, ip.data_ptr(), ids.data_ptr(), None)
    seen = [[5, 6, 7, 8], [], [5, 6], [7, 8]]
    got = rank(dev(x), 5, asgd.logit_rules(seen=c, presence=3.0))
    check_rank(got, ref.scores(x, seen=seen, presence=3.0), 5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,low,count,k", [(200_000, 0, 3000, 64), (200_000, 150_000, 9000, 5), (3000, 0, 2900, 64),
                                           (4100, 4000, 100, 64)])
def test_topk_lists_that_crowd_a_range(dtype, L, low, count, k):
    # more distinct ids side by side than a table holds, in both lists, each of them up to three times
    r = np.random.default_rng(L + count)
    ids = low + r.permutation(count)[:count]
    seen = [np.concatenate([ids, ids[::2], ids[::7]]), [], ids[:3]]
    row_bias = [(ids[::3], r.normal(0, 3, len(ids[::3])).astype(np.float32)), ([low], np.array([9.0], np.float32)), ([], [])]
    z = strided(r.normal(0, 2, (3, L)), dtype, 1, 3)
    c, keep = lists(seen, L)
    c2, keep2 = lists(row_bias, L, values=True)
    kw = dict(repetition=1.1, frequency=0.3, presence=0.1)
    check_rank(rank(z, k, asgd.logit_rules(seen=c, row_bias=c2, **kw)),
               ref.scores(host(z), seen=seen, row_bias=row_bias, **kw), k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("listed", [50, 63])
def test_topk_short_rows_with_listed_labels_and_unaligned_ends(dtype, listed):
    # rows of one piece: listed labels wait, then the labels before and after the whole vectors, then a round that
    # passes one label of every lane
    r = np.random.default_rng(listed)
    L = 3998
    z = strided(r.normal(0, 2, (40, L)), dtype, 1, 9)
    seen = [r.permutation(np.arange(20, L - 20))[:listed] for _ in range(40)]
    c, keep = lists(seen, L)
    check_rank(rank(z, 64, asgd.logit_rules(seen=c, presence=-1.0)), ref.scores(host(z), seen=seen, presence=-1.0), 64)


def test_topk_twice_is_bitwise_the_same_and_stays_in_its_rows():
    B, L, k = 30, 50_000, 20
    r = np.random.default_rng(77)
    z = dev(r.normal(0, 2, (B, L)).astype(np.float32))
    o, rules, allowed, keep = random_rules(r, B, L, 400, True, 30, 0.8)
    big = [torch.full((B + 2, k), -7, dtype=torch.int32, device="cuda"), torch.full((B + 2, k), 7.0, device="cuda"),
           torch.full((B + 2,), 7.0, device="cuda")]
    ids, sc, lse = (t[1:B + 1] for t in big)
    first = None
    for _ in range(4):
        ws = scratch(asgd.asgd_logits_topk_workspace(B, L, k))
        asgd.asgd_logits_topk(asgd.matrix(z), k, ids, sc, rules=rules, lse=lse, workspace=ws)
        now = [t.clone() for t in (ids, sc, lse)]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = first or now
    for t, v in zip(big, (-7, 7.0, 7.0)):
        assert bool((t[0] == v).all() and (t[-1] == v).all())
    check_rank(first, ref.scores(host(z), **o), k, allowed)


# Where ceil(v log2 e), formed from the rounded product, lay far above the exact one.
FAR = [3000000512.0, -3000000768.0, 3182850800.0, 3.0366761e9, -3.0031217e9, 1.6e9, -1.9e9, 4.2e9, 2.0 ** 28, -(2.0 ** 28),
       2.0 ** 32, -(2.0 ** 32)]


def far_scores(r, B):
    """Best scores of either sign from 2^23 to 2^34."""
    v = np.exp2(r.uniform(23, 34, B)) * r.choice([-1, 1], B)
    v[:len(FAR)] = FAR[:B]
    return v


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L", [(300, 1), (300, 130), (64, 9001), (40, 140_000)])
def test_topk_lse_of_very_large_scores(dtype, B, L):
    r = np.random.default_rng(L)
    top = far_scores(r, B)
    # labels at the best score, next to it, and far below
    x = top[:, None] - np.abs(top[:, None]) * r.choice([0.0, 2.0 ** -22, 2.0 ** -7, 0.1, 1.0], (B, L), p=[.1, .2, .2, .2, .3])
    x[:, L // 2] = top
    z = strided(x, dtype, 1, 3)
    check_rank(rank(z, 5), ref.scores(host(z)), 5)


@pytest.mark.parametrize("B,L", [(100, 300), (20, 60_000)])
def test_topk_lse_of_very_large_listed_scores(B, L):
    # the best label is one that the lists name: its score goes through their own sum
    r = np.random.default_rng(B)
    top = far_scores(r, B)
    x = r.normal(0, 2, (B, L)).astype(np.float32)
    x[top < 0] += 2 * top[top < 0, None].astype(np.float32)
    at = r.integers(0, L, B)
    row_bias = [(np.array([j]), np.array([t], np.float32)) for j, t in zip(at, top)]
    x[np.arange(B), at] = 0.5
    c, keep = lists(row_bias, L, values=True)
    seen = [np.array([j, j]) for j in at]
    c2, keep2 = lists(seen, L)
    check_rank(rank(dev(x), 3, asgd.logit_rules(seen=c2, row_bias=c, frequency=0.25)),
               ref.scores(x, seen=seen, row_bias=row_bias, frequency=0.25), 3)


# ---------------------------------------------------------------- distillation
def teacher(r, B, L, k, empty=0.2):
    ids = np.stack([r.permutation(max(L, k))[:k] for _ in range(B)]).astype(np.int32)
    ids = np.where(ids >= L, ref.EMPTY, ids).astype(np.int32)
    t = r.normal(4, 1.5, (B, k)).astype(np.float32)
    short = r.random((B, k)) < empty * (r.random((B, 1)) < 0.5)
    ids[short], t[short] = ref.EMPTY, -INF
    if B > 2:
        ids[1], t[1] = ref.EMPTY, -INF  # a row without a teacher
    return ids, t


def distill(z, ids, t, T, grad=None, weights=None, stream=None):
    B, L = z.shape
    loss = torch.full((B,), 7.0, device="cuda")
    ws = scratch(asgd.asgd_distill_workspace(B, L, ids.shape[1]))
    asgd.asgd_distill(asgd.matrix(z), ids, t, T, loss, grad=None if grad is None else asgd.matrix(grad),
                      weights=weights, workspace=ws, stream=torch.cuda.current_stream() if stream is None else stream)
    return loss


def distill_bounds(z, ids, t, T, w, p, q, dtype):
    """Per entry of the gradient: p's and q's relative errors, then the output's rounding.  p: one step
    for every addition of its sum (columns / 256 on a lane and 96 merges), and for its exponent
    x = (z - m) log2(e) / T, fp32 as written (|x| / 2 + 4 half steps in the worst case, 16-bit
    outputs) or carried in two parts (8).  q: half a step per rounding of its argument and 600 additions at most."""
    B, L = z.shape
    x = (np.nanmax(np.where(np.isinf(z), np.nan, z), 1, initial=0, keepdims=True) - np.where(np.isinf(z), 0, z)) / T * 1.45
    adds = (L / 256 + 96) * 2 * U
    rel_p = adds + (np.abs(x) + 16) * 2 * U
    on = np.isfinite(t)
    span = np.where(on, t, -1e30).max(1) - np.where(on, t, 1e30).min(1)
    rel_q = ((np.maximum(span, 0) / T + 8 + ids.shape[1]) * 2 * U)[:, None]
    scale = (np.asarray(w) * T)[:, None]
    err = np.abs(scale) * (rel_p * p + rel_q * q + 2 * U * np.abs(p - q) + 1e-38)
    return err + (ref.half_step(np.abs(scale * (p - q)) + err, dtype) if dtype != "f32" else 0)


DISTILL = [(1, 1, 1, 1.0), (1, 7, 3, 2.0), (3, 64, 5, 0.5), (4, 1000, 32, 1.0), (128, 1000, 5, 2.0), (5, 8193, 512, 4.0),
           (2, 30_000, 32, 1.0), (3, 65_537, 64, 1.5), (1, 205_443, 100, 2.0), (2100, 65, 4, 1.0),
           (520, 33_001, 6, 1.0), (40, 8200, 9, 3.0), (30, 2049, 3, 1.0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,L,k,T", DISTILL)
def test_distill_loss_and_gradient(dtype, B, L, k, T):
    r = np.random.default_rng(B + L + k)
    z = strided(r.normal(0, 2, (B, L)), dtype, (B + L) % 5, 9)
    ids, t = teacher(r, B, L, k)
    w = r.uniform(0.1, 2.0, B).astype(np.float32)
    big = torch.full((B, L + 9), 7.0, dtype=z.dtype, device="cuda")
    grad = big[:, 4:4 + L]  # another phase than z's
    loss = distill(z, dev(ids), dev(t), T, grad, dev(w))
    x = host(z)
    want, g, p, q = ref.distill(x, ids, t, T, w)
    err = np.abs(host(grad) - g)
    bound = distill_bounds(x, ids, t, T, w, p, q, dtype)
    assert (err <= bound).all(), ((err / bound).max(), err.max())
    assert bool((big[:, :4] == 7.0).all() and (big[:, 4 + L:] == 7.0).all())
    # loss: the logarithms and their arguments, T^2 times
    size = T * T * (np.abs(x).max(1) / T * 2 + np.log(L) + 16)
    lerr = np.abs(host(loss) - want)
    lbound = size * (16 + k / 8 + L / 512) * 2 * U
    assert (lerr <= lbound).all(), (lerr / lbound).max()
    empty = ~((ids >= 0) & (ids < L) & np.isfinite(t)).any(1)
    assert (host(loss)[empty] == 0).all() and (host(grad)[empty] == 0).all()
    # the loss alone, and the gradient in the logits' place, with the mean over the rows
    assert torch.equal(distill(z, dev(ids), dev(t), T), loss)
    apart = torch.empty_like(z)
    assert torch.equal(distill(z, dev(ids), dev(t), T, apart), loss)
    # (a copy at z's alignment, which decides the order of the sums)
    inplace = strided(x, dtype, (B + L) % 5, 9)
    wide = torch.empty(z.shape, dtype=z.dtype, device="cuda")
    distill(z, dev(ids), dev(t), T, wide)
    assert torch.equal(distill(inplace, dev(ids), dev(t), T, inplace), loss) and torch.equal(inplace, wide)
    assert torch.equal(apart, wide)


def test_distill_repeated_and_invalid_entries():
    B, L = 6, 500
    r = np.random.default_rng(9)
    x = r.normal(0, 2, (B, L)).astype(np.float32)
    ids = r.integers(0, L, (B, 8)).astype(np.int32)
    t = r.normal(0, 1, (B, 8)).astype(np.float32)
    ids[0, :] = 17                        # one label eight times
    ids[1, 2], ids[1, 3] = -1, L          # outside
    t[2, 1], t[2, 2], t[2, 3] = NAN, INF, -INF
    t[3, :] = [80, -80, 0, 3, 88, -3, 2, 1]  # far apart
    t[4, :] = NAN
    grad = torch.empty((B, L), device="cuda")
    loss = distill(dev(x), dev(ids), dev(t), 1.0, grad)
    want, g, p, q = ref.distill(x, ids, t, 1.0)
    tt = np.where(np.isfinite(t), t, np.nan)
    err = np.abs(host(grad) - g)
    bound = distill_bounds(x, ids, np.where(np.isnan(tt), -INF, t).astype(np.float32), 1.0, np.full(B, 1 / B), p, q, "f32")
    assert (err <= bound).all(), (err / bound).max()
    assert (np.abs(host(loss) - want) <= 200 * 32 * 2 * U).all()
    assert host(loss)[4] == 0 and (host(grad)[4] == 0).all()


def test_distill_infinite_logits():
    x = np.random.default_rng(1).normal(0, 1, (6, 300)).astype(np.float32)
    x[0, 10] = NAN
    x[1, 20] = INF
    x[2, 30:200] = -INF                   # masked labels, one of them the teacher's
    x[3, :] = -INF
    x[4, :] = np.finfo(np.float32).min    # equal, at the type's lowest value
    x[5, 1:] = -INF
    ids = np.tile(np.array([5, 40, 0], np.int32), (6, 1))
    t = np.tile(np.array([1.0, 0.5, 2.0], np.float32), (6, 1))
    ids[5, :2] = 0
    grad = torch.empty((6, 300), device="cuda")
    loss = host(distill(dev(x), dev(ids), dev(t), 2.0, grad))
    g = host(grad)
    want, wg, p, q = ref.distill(x, ids, t, 2.0)
    assert np.isnan(loss[:2]).all() and np.isnan(g[:2]).all()
    assert loss[2] == INF and loss[3] == INF
    for i in (2, 3, 4, 5):
        assert np.abs(g[i] - wg[i]).max() <= 64 * 2 * U, i
    assert (g[2, 30:40] == 0).all()
    assert abs(loss[4] - want[4]) <= 64 * 2 * U * 16 and abs(loss[5] - want[5]) <= 64 * 2 * U * 4


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("L", [40_003, 300_002])
def test_distill_infinities_repeats_and_empty_teachers_of_long_rows(L, shift):
    B, T = 8, 2.0
    x = np.random.default_rng(L).normal(0, 1, (B, L)).astype(np.float32)
    x[0, L // 2] = NAN
    x[1, L - 1] = INF
    x[2, 30:L // 2] = -INF                # masked labels, one of them the teacher's
    x[3, :] = -INF
    x[4, :] = np.finfo(np.float32).min
    x[5, 1:] = -INF
    x[6, 5] = NAN                         # and no teacher
    ids = np.tile(np.array([5, 40, 0, L - 1, L - 2, 17], np.int32), (B, 1))
    t = np.random.default_rng(1).normal(0, 1, (B, 6)).astype(np.float32)
    ids[2] = [40, 3, 3, L, -1, L - 1]
    ids[5] = 0
    ids[6] = ref.EMPTY
    ids[7] = [L - 1, 0, L - 1, 0, 20_000, 20_000]
    big = torch.full((B, L + 9), 7.0, device="cuda")
    grad = big[:, 4:4 + L]
    loss = distill(strided(x, "f32", shift, 3), dev(ids), dev(t), T, grad)
    assert bool((big[:, :4] == 7.0).all() and (big[:, 4 + L:] == 7.0).all())
    assert torch.equal(distill(strided(x, "f32", shift, 3), dev(ids), dev(t), T)[2:], loss[2:])
    loss, g = host(loss), host(grad)
    want, wg, p, q = ref.distill(x, ids, t, T)
    assert np.isnan(loss[:2]).all() and np.isnan(g[:2]).all()
    assert loss[2] == INF and loss[3] == INF and loss[6] == 0 and (g[6] == 0).all()
    assert (g[2, 30:40] == 0).all() and (g[3, 100:1000] == 0).all()
    some = [2, 3, 7]
    on = (ids >= 0) & (ids < L)
    bound = distill_bounds(x[some], ids[some], np.where(on, t, -INF)[some], T, np.full(3, 1 / B), p[some], q[some], "f32")
    err = np.abs(g[some] - wg[some])
    assert (err <= bound).all(), (err / bound).max()
    # equal logits, and a single one: exponentials of 0, the sum's additions, a division, q's roundings, a difference
    bound = T / B * (L / 256 + 96 + 16 + 24) * 2 * U * (p[4:6] + q[4:6])
    err = np.abs(g[4:6] - wg[4:6])
    assert (err <= bound).all(), (err / bound).max()
    size = T * T * (8 / T * 2 + np.log(L) + 16)
    assert (np.abs(loss[[4, 5, 7]] - want[[4, 5, 7]]) <= size * (16 + 1 + L / 512) * 2 * U).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [300, 40_000, 200_000])
@pytest.mark.parametrize("T", [1e-6, 1e-3, 1e3, 1e6])
def test_distill_at_the_ends_of_the_temperatures(dtype, L, T):
    r = np.random.default_rng(L)
    x = np.round(r.normal(0, 2, (2, L)), 1)  # (gaps of 0.1 at the least between different logits)
    x[0, 7] = -INF
    z = strided(x, dtype, 1, 3)
    ids = r.integers(0, L, (2, 3)).astype(np.int32)
    t = np.array([[1.0, 2.0, 3.0], [0.0, 0.0, 1.0]], np.float32)
    grad = torch.empty((2, L), dtype=z.dtype, device="cuda")
    distill(z, dev(ids), dev(t), T, grad)
    xx = host(z)
    _, g, p, q = ref.distill(xx, ids, t, float(np.float32(T)))
    # (an exponent of thousands has an error of its own; there p is below 1e-30 on both sides)
    bound = distill_bounds(np.where(p > 1e-30, xx, -INF), ids, t, T, np.full(2, 0.5), p, q, dtype) + T * 1e-30
    err = np.abs(host(grad) - g)
    assert np.isfinite(host(grad)).all() and (err <= bound).all(), (err / bound).max()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [9, 300, 40_003, 200_000])
@pytest.mark.parametrize("T", [1e-6, 0.25, 0.5, 1.0, 3.0])
def test_distill_loss_of_teachers_labels_masked_by_the_lowest_value(dtype, L, T):
    # T^2 times (gap / T) is finite where gap / T is not
    r = np.random.default_rng(L)
    low = float(torch.finfo(ref.DTYPES[dtype]).min)
    x = r.normal(0, 2, (5, L))
    x[0, 3] = x[1, L // 2:] = low
    x[2, L - 1] = 0.75 * low
    x[3, 1:] = low
    x[3, 0], x[4, 0], x[4, 2] = 0.9 * -low, 0.5 * -low, 0.5 * low  # (and gaps beyond the type)
    z = strided(x, dtype, 1, 3)
    ids = np.array([[3, 0], [L - 1, 1], [L - 1, L - 1], [2, 0], [2, 0]], np.int32)
    t = (np.array([[0.0, 0.5], [1.0, 0.0], [-1.0, 0.0], [0.0, 2.0], [0.0, 0.0]]) * min(T, 1.0)).astype(np.float32)
    grad = torch.empty((5, L), dtype=z.dtype, device="cuda")
    loss = distill(z, dev(ids), dev(t), T, grad)
    assert torch.equal(distill(z, dev(ids), dev(t), T), loss)
    xx = host(z)
    want, g, p, q = ref.distill(xx, ids, t, float(np.float32(T)))
    with np.errstate(over="ignore"):
        infinite = np.isinf(want.astype(np.float32))
    got = host(loss)
    assert np.array_equal(np.isinf(got), infinite) and (got[infinite] == INF).all()
    # in half steps: q has its argument's (at most 2) two, its exponential's two, the sum's as many again, weighted, and
    # one, and a division's and a product's: 15; the gap's rounding, three products and two additions are six more
    ok = ~infinite
    assert (np.abs(got - want)[ok] <= 24 * U * want[ok]).all(), (got, want)
    assert (np.abs(host(grad) - g) <= distill_bounds(np.where(p > 1e-30, xx, -INF), ids, t, T, np.full(5, 0.2), p, q, dtype)
            + T * 1e-30).all()


def test_distill_gradient_against_differences():
    # the loss in fp32 moves by its gradient times the step, up to the loss's own rounding
    B, L, T = 3, 50, 1.3
    r = np.random.default_rng(2)
    x = r.normal(0, 1, (B, L)).astype(np.float32)
    ids, t = teacher(r, B, L, 6)
    w = np.ones(B, np.float32)
    grad = torch.empty((B, L), device="cuda")
    loss = host(distill(dev(x), dev(ids), dev(t), T, grad, dev(w)))
    step = 2.0 ** -6
    for j in range(L):
        up, down = x.copy(), x.copy()
        up[:, j] += np.float32(step)
        down[:, j] -= np.float32(step)
        width = (up[:, j].astype(np.float64) - down[:, j])
        d = (host(distill(dev(up), dev(ids), dev(t), T)) - host(distill(dev(down), dev(ids), dev(t), T))) / width
        # central differences: third derivative at most 1 / T in size, so step^2 / 6; rounding
        # 32 half steps of the loss over the width
        bound = step * step / 6 + 32 * U * (np.abs(loss) + 8 * T * T) / step
        assert (np.abs(d - host(grad)[:, j]) <= bound).all()


# ---------------------------------------------------------------- streams, graphs, far offsets
def test_rows_past_two_to_the_31_elements():
    B, L, ld = 520, 1000, (1 << 22) + 8
    flush("  allocating 4.4 GB")
    big = torch.zeros((B, ld), dtype=torch.bfloat16, device="cuda")
    assert (B - 1) * ld > 2 ** 31
    r = np.random.default_rng(4)
    x = r.normal(0, 2, (B, L))
    z = big[:, 3:3 + L]
    z.copy_(torch.from_numpy(x))
    check_rank(rank(z, 5), ref.scores(host(z)), 5)
    ids, t = teacher(r, B, L, 5)
    near = strided(x, "bf16", 3, 8)  # the same rows, close together and at the same alignment
    alone = torch.empty((B, L), dtype=torch.bfloat16, device="cuda")
    loss = distill(near, dev(ids), dev(t), 1.0, alone)
    assert torch.equal(distill(z, dev(ids), dev(t), 1.0, z), loss)
    assert torch.equal(z, alone)


def test_distill_past_a_million_workgroups():
    B, L, T = 1600, (1 << 22) - 3, 1.0
    flush("  allocating 13.4 GB")
    r = np.random.default_rng(7)
    row = r.normal(0, 2, L)
    z = torch.empty((B, L), dtype=torch.bfloat16, device="cuda")
    z.copy_(dev(row))
    ids, t = teacher(r, B, 1000, 5)
    at = [0, 2, 799, B - 1]
    x = host(z[:1]).repeat(len(at), 0)
    w = r.uniform(0.5, 2.0, B).astype(np.float32)
    loss = host(distill(z, dev(ids), dev(t), T, z, dev(w)))[at]
    want, g, p, q = ref.distill(x, ids[at], t[at], T, w[at])
    err = np.abs(host(z[at]) - g)
    assert (err <= distill_bounds(x, ids[at], t[at], T, w[at], p, q, "bf16")).all()
    size = T * T * (np.abs(x).max(1) / T * 2 + np.log(L) + 16)
    assert (np.abs(loss - want) <= size * (16 + 1 + L / 512) * 2 * U).all()


def test_fp4_rows_past_two_to_the_31_elements():
    B, L, ld = 520, 1000, (1 << 22) + 8
    flush("  allocating 8.8 GB")
    big = torch.zeros((B, ld), dtype=torch.bfloat16, device="cuda")
    r = np.random.default_rng(5)
    x = big[:, 5:133]
    x.copy_(torch.from_numpy(r.normal(0, 1, (B, 128))))
    codes = torch.empty((B, 64), dtype=torch.uint8, device="cuda")
    scales = torch.empty((B, 4), dtype=torch.uint8, device="cuda")
    h = asgd.fp4_matrix(codes, scales)
    asgd.asgd_fp4_quantize(asgd.matrix(x), h)
    v, c, s = ref.quantize(host(x))
    assert np.array_equal(ref.values_of(codes.cpu().numpy(), scales.cpu().numpy()), v)
    wc, wsc = (dev(t) for t in label_matrix(L, 9))
    w = asgd.fp4_matrix(wc, wsc)
    for n in (B, 20, 10):  # many rows and few
        z = big[:n, 200:200 + L] if n > 32 else big[-n:, 200:200 + L]
        a = asgd.fp4_matrix(codes[:n] if n > 32 else codes[-n:], scales[:n] if n > 32 else scales[-n:])
        asgd.asgd_fp4_logits(a, w, asgd.matrix(z))
        near = torch.empty((n, L), dtype=torch.bfloat16, device="cuda")
        asgd.asgd_fp4_logits(a, w, asgd.matrix(near))
        assert torch.equal(z, near)
        assert bool((big[:, 200 + L:200 + L + 64] == 0).all() and (big[:, 133:200] == 0).all())
    big[:, 5:133].zero_()
    asgd.asgd_fp4_dequantize(h, asgd.matrix(x))
    assert torch.equal(x.cpu(), torch.from_numpy(v).bfloat16())


def test_two_streams_at_once():
    r = np.random.default_rng(8)
    x = [dev(r.normal(0, 2, (3, 50_000)).astype(np.float32)) for _ in range(2)]
    alone = [rank(v, 16) for v in x]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream() for _ in range(2)]
    for s in st:
        s.wait_stream(torch.cuda.current_stream())
    both = []
    for _ in range(4):
        for v, s in zip(x, st):
            with torch.cuda.stream(s):
                both.append(rank(v, 16, stream=s))
    torch.cuda.synchronize()
    for i, got in enumerate(both):
        assert all(torch.equal(a, b) for a, b in zip(got, alone[i % 2]))


def test_captured_and_replayed():
    r = np.random.default_rng(11)
    B, L, k = 4, 20_000, 8
    z = dev(r.normal(0, 2, (B, L)).astype(np.float32))
    h = dev(np.maximum(r.normal(0, 1, (B, 128)), 0), "bf16")
    w2 = dev(r.normal(0, 0.2, (L, 128)).astype(np.float32))
    codes = torch.empty((L, 64), dtype=torch.uint8, device="cuda")
    scales = torch.empty((L, 4), dtype=torch.uint8, device="cuda")
    o, rules, allowed, keep = random_rules(r, B, L, 20, True, 4, 0.9)
    grad, loss = torch.empty_like(z), torch.empty(B, device="cuda")
    ids = torch.empty((B, k), dtype=torch.int32, device="cuda")
    sc, lse = torch.empty((B, k), device="cuda"), torch.empty(B, device="cuda")
    ws1 = scratch(asgd.asgd_logits_topk_workspace(B, L, k))
    ws2 = scratch(asgd.asgd_distill_workspace(B, L, k))

    def run():
        st = torch.cuda.current_stream()
        q = asgd.fp4_matrix(codes, scales)
        asgd.asgd_fp4_quantize(asgd.matrix(w2), q, st)
        asgd.asgd_fp4_logits(asgd.matrix(h), q, asgd.matrix(z), stream=st)
        asgd.asgd_logits_topk(asgd.matrix(z), k, ids, sc, rules=rules, lse=lse, workspace=ws1, stream=st)
        asgd.asgd_distill(asgd.matrix(z), ids, sc, 2.0, loss, grad=asgd.matrix(grad), workspace=ws2, stream=st)

    outs = (z, ids, sc, lse, loss, grad)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for n in range(3):
        h.copy_(dev(np.maximum(r.normal(0, 1, (B, 128)), 0), "bf16"))
        run()
        want = [v.clone() for v in outs]
        for v in outs:
            v.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), n


def test_memory_that_is_not_the_devices_is_refused():
    z = dev(np.zeros((2, 100), np.float32))
    ids = torch.empty((2, 1), dtype=torch.int32, device="cuda")
    on_host = torch.zeros((2, 100))
    ws = scratch(asgd.asgd_logits_topk_workspace(2, 100, 1))
    cases = [lambda: asgd.asgd_logits_topk(asgd.matrix(on_host), 1, ids, workspace=ws),
             lambda: asgd.asgd_logits_topk(asgd.matrix(z), 1, ids.cpu(), workspace=ws),
             lambda: asgd.asgd_logits_topk(asgd.matrix(z), 1, ids, rules=asgd.logit_rules(bias=torch.zeros(100)),
                                           workspace=ws),
             lambda: asgd.asgd_distill(asgd.matrix(z), ids.cpu(), z, 1.0, z, k=1,
                                       workspace=scratch(asgd.asgd_distill_workspace(2, 100, 1))),
             lambda: asgd.asgd_distill(asgd.matrix(z), ids, z, 1.0, z, k=1, workspace=torch.zeros(1 << 16, dtype=torch.uint8)
                                       [-on_host.data_ptr() % 256:])]
    for c in cases:
        with pytest.raises(asgd.AsgdError) as e:
            c()
        assert e.value.status == asgd.ASGD_EINVAL
    # and the refusals leave nothing behind
    check_rank(rank(z, 1), ref.scores(host(z)), 1)
