"""Refusals of the entry points over label logits, and their references' own pins.  No GPU work
is issued: every call here is refused on the host."""
import ctypes

import numpy as np
import pytest
import torch

import logits_ref as ref
import paper_2110_07029_amd as asgd

A = 1 << 20  # an address that is aligned for everything and never used


def mat(rows=4, cols=100, ld=None, dtype=asgd.ASGD_F32, data=A):
    return asgd.asgd_matrix(rows, cols, cols if ld is None else ld, dtype, data)


def fp4(rows=4, cols=128, codes=A, scales=A):
    return asgd.asgd_fp4(rows, cols, codes, scales)


class Ws:
    """Scratch memory that only claims a size."""

    def __init__(self, n, at=A):
        self.n, self.at = n, at

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def element_size(self):
        return 1


BIG = Ws(1 << 40)


def refused(status, word, call, *a, **k):
    with pytest.raises(asgd.AsgdError) as e:
        call(*a, **k)
    assert e.value.status == status, e.value
    assert word in str(e.value), e.value


MATRICES = [
    (dict(rows=0), asgd.ASGD_EINVAL, ">= 1"), (dict(cols=0, ld=1), asgd.ASGD_EINVAL, ">= 1"),
    (dict(rows=-3), asgd.ASGD_EINVAL, ">= 1"), (dict(rows=(1 << 20) + 1), asgd.ASGD_ERANGE, "2^20"),
    (dict(cols=1 << 22), asgd.ASGD_ERANGE, "2^22"), (dict(ld=99), asgd.ASGD_EINVAL, "ld"),
    (dict(ld=(1 << 40) + 1), asgd.ASGD_ERANGE, "ld"), (dict(dtype=3), asgd.ASGD_EINVAL, "type"),
    (dict(dtype=-1), asgd.ASGD_EINVAL, "type"), (dict(data=None), asgd.ASGD_EINVAL, "NULL"),
    (dict(data=A + 2), asgd.ASGD_EINVAL, "aligned"), (dict(dtype=asgd.ASGD_BF16, data=A + 1), asgd.ASGD_EINVAL, "aligned"),
]


@pytest.mark.parametrize("change,status,word", MATRICES)
def test_bad_matrices_are_refused(change, status, word):
    refused(status, word, asgd.asgd_logits_topk, mat(**change), 1, A, workspace=BIG)
    refused(status, word, asgd.asgd_distill, mat(**change), A, A, 1.0, A, k=1, workspace=BIG)
    refused(status, word, asgd.asgd_fp4_quantize, mat(**change), fp4())
    refused(status, word, asgd.asgd_fp4_dequantize, fp4(), mat(**change))


FP4S = [(dict(rows=0), asgd.ASGD_EINVAL, ">= 1"), (dict(cols=48), asgd.ASGD_EINVAL, "32"),
        (dict(rows=1 << 22), asgd.ASGD_ERANGE, "2^22"), (dict(rows=1 << 21, cols=1024), asgd.ASGD_ERANGE, "2^31"),
        (dict(codes=None), asgd.ASGD_EINVAL, "non-NULL"), (dict(scales=None), asgd.ASGD_EINVAL, "non-NULL"),
        (dict(codes=A + 8), asgd.ASGD_EINVAL, "aligned"), (dict(scales=A + 2), asgd.ASGD_EINVAL, "aligned")]


@pytest.mark.parametrize("change,status,word", FP4S)
def test_bad_fp4_matrices_are_refused(change, status, word):
    q = fp4(**change)
    refused(status, word, asgd.asgd_fp4_quantize, mat(4, 128), q)
    refused(status, word, asgd.asgd_fp4_dequantize, q, mat(4, 128))
    refused(status, word, asgd.asgd_fp4_logits, q, fp4(100), mat())
    refused(status, word, asgd.asgd_fp4_logits, mat(4, 128, dtype=asgd.ASGD_BF16), q, mat())


def test_fp4_shapes_are_checked():
    E = asgd.ASGD_EINVAL
    h = mat(4, 128, dtype=asgd.ASGD_BF16)
    refused(E, "shape", asgd.asgd_fp4_quantize, mat(5, 128), fp4())
    refused(E, "shape", asgd.asgd_fp4_quantize, mat(4, 96), fp4())
    refused(E, "shape", asgd.asgd_fp4_dequantize, fp4(), mat(4, 160))
    refused(E, "bf16", asgd.asgd_fp4_logits, mat(4, 128), fp4(100), mat())
    refused(E, "128", asgd.asgd_fp4_logits, mat(4, 64, dtype=asgd.ASGD_BF16), fp4(100), mat())
    refused(E, "128", asgd.asgd_fp4_logits, h, fp4(100, 256), mat())
    refused(E, "rows x labels", asgd.asgd_fp4_logits, h, fp4(101), mat())
    refused(E, "rows x labels", asgd.asgd_fp4_logits, h, fp4(100), mat(3))
    refused(E, "16-byte", asgd.asgd_fp4_logits, mat(4, 128, 130, asgd.ASGD_BF16), fp4(100), mat())
    refused(E, "16-byte", asgd.asgd_fp4_logits, mat(4, 128, 128, asgd.ASGD_BF16, A + 8), fp4(100), mat())
    refused(E, "bias", asgd.asgd_fp4_logits, h, fp4(100), mat(), bias=A + 1)
    lib = asgd.load()
    by = ctypes.byref
    assert lib.asgd_fp4_logits(None, None, by(fp4(100)), None, by(mat()), None) == E
    assert lib.asgd_fp4_logits(by(h), by(fp4()), by(fp4(100)), None, by(mat()), None) == E
    assert lib.asgd_fp4_quantize(None, by(fp4()), None) == E
    assert lib.asgd_logits_topk(None, None, 1, A, None, None, A, 1 << 40, None) == E
    assert lib.asgd_distill(None, A, A, 1, 1.0, None, A, None, A, 1 << 40, None) == E


def csr(rows=4, cols=100, nnz=5, indptr=A, indices=A, values=A):
    return asgd.asgd_csr(rows, cols, nnz, indptr, indices, values)


RULES = [(dict(seen=csr(rows=3)), "n_rows"), (dict(seen=csr(cols=99)), "n_cols"), (dict(seen=csr(nnz=-1)), "nnz"),
         (dict(seen=csr(indptr=None)), "indptr"), (dict(seen=csr(indices=None)), "indices"),
         (dict(row_bias=csr(rows=5)), "n_rows"), (dict(row_bias=csr(values=None)), "values"),
         (dict(repetition=-1.0), "repetition"), (dict(repetition=float("nan")), "repetition"),
         (dict(repetition=float("inf")), "repetition"), (dict(frequency=float("nan")), "frequency"),
         (dict(presence=float("inf")), "presence")]


@pytest.mark.parametrize("change,word", RULES)
def test_bad_rules_are_refused(change, word):
    refused(asgd.ASGD_EINVAL, word, asgd.asgd_logits_topk, mat(), 1, A, rules=asgd.logit_rules(**change), workspace=BIG)


@pytest.mark.parametrize("change", [dict(seen=csr(indptr=A + 2)), dict(seen=csr(indices=A + 1)), dict(row_bias=csr(values=A + 2)),
                                    dict(row_bias=csr(indices=A + 3))])
def test_misaligned_lists_are_refused(change):
    refused(asgd.ASGD_EINVAL, "4-byte aligned", asgd.asgd_logits_topk, mat(), 1, A, rules=asgd.logit_rules(**change),
            workspace=BIG)


def test_rule_masks_and_outputs_are_checked():
    E, R = asgd.ASGD_EINVAL, asgd.ASGD_ERANGE
    r = asgd.asgd_logit_rules(allowed=A, allowed_ld=3)
    refused(E, "allowed_ld", asgd.asgd_logits_topk, mat(), 1, A, rules=r, workspace=BIG)
    refused(R, "2^30", asgd.asgd_logits_topk, mat(), 1, A, rules=asgd.logit_rules(seen=csr(nnz=1 << 30)), workspace=BIG)
    r = asgd.asgd_logit_rules(allowed=A, allowed_ld=-1)
    refused(E, "allowed_ld", asgd.asgd_logits_topk, mat(), 1, A, rules=r, workspace=BIG)
    refused(E, "aligned", asgd.asgd_logits_topk, mat(), 1, A, rules=asgd.asgd_logit_rules(bias=A + 2), workspace=BIG)
    for k in (0, -1, 65):
        refused(E, "k must", asgd.asgd_logits_topk, mat(), k, A, workspace=BIG)
        refused(E, "k must", asgd.asgd_logits_topk_workspace, 4, 100, k)
    refused(E, "ids", asgd.asgd_logits_topk, mat(), 1, None, workspace=BIG)
    refused(E, "aligned", asgd.asgd_logits_topk, mat(), 1, A + 1, workspace=BIG)
    refused(E, "aligned", asgd.asgd_logits_topk, mat(), 1, A, scores=A + 2, workspace=BIG)
    need = asgd.asgd_logits_topk_workspace(1, 670_091, 5)
    assert need > 0
    big = mat(1, 670_091)
    refused(R, "workspace", asgd.asgd_logits_topk, big, 5, A, workspace=Ws(need - 1))
    refused(R, "workspace", asgd.asgd_logits_topk, big, 5, A)
    refused(E, "256-byte", asgd.asgd_logits_topk, big, 5, A, workspace=Ws(need, A + 128))
    refused(R, "2^22", asgd.asgd_logits_topk_workspace, 1, 1 << 22, 1)
    refused(E, ">= 1", asgd.asgd_logits_topk_workspace, 0, 10, 1)


def test_distill_arguments_are_checked():
    E, R = asgd.ASGD_EINVAL, asgd.ASGD_ERANGE
    call = lambda z=None, k=3, T=1.0, ids=A, t=A, loss=A, **o: asgd.asgd_distill(  # noqa: E731
        mat() if z is None else z, ids, t, T, loss, k=k, **{"workspace": BIG, **o})
    for k in (0, 513):
        refused(E, "k must", call, k=k)
        refused(E, "k must", asgd.asgd_distill_workspace, 4, 100, k)
    for T in (0.0, -1.0, float("nan"), float("inf")):
        refused(E, "temperature", call, T=T)
    for T in (1e-7, 2e6):
        refused(R, "temperature", call, T=T)
    for o in (dict(ids=None), dict(t=None), dict(loss=None)):
        refused(E, "non-NULL", call, **o)
    refused(E, "aligned", call, loss=A + 2)
    refused(E, "aligned", call, weights=A + 2)
    far = A + (1 << 16)
    refused(E, "shape or type", call, grad=mat(5, data=far))
    refused(E, "shape or type", call, grad=mat(4, 99, data=far))
    refused(E, "shape or type", call, grad=mat(dtype=asgd.ASGD_BF16, data=far))
    refused(E, "overlaps", call, grad=mat(data=A + 400))
    refused(E, "overlaps", call, grad=mat(ld=101))
    need = asgd.asgd_distill_workspace(4, 100, 3)
    refused(R, "workspace", call, workspace=Ws(need - 1))
    refused(R, "2^20", asgd.asgd_distill_workspace, (1 << 20) + 1, 10, 1)


def test_model_entry_points_refuse_null_models():
    E = asgd.ASGD_EINVAL
    refused(E, "NULL", asgd.asgd_model_fp4_labels, None, fp4())
    refused(E, "NULL", asgd.asgd_predict_rules_workspace, None, 1, 1)
    x = csr()
    refused(E, "NULL", asgd.asgd_predict_topk_rules, None, x, 1, A, workspace=BIG)
    refused(E, "NULL", asgd.asgd_distill_step, None, x, A, A, 1.0, 0.1, k=1)


def test_tensor_helpers_check_layout():
    t = torch.zeros(4, 64)
    m = asgd.matrix(t[:, 3:50])
    assert (m.n_rows, m.n_cols, m.ld, m.dtype, m.data) == (4, 47, 64, asgd.ASGD_F32, t.data_ptr() + 12)
    assert asgd.matrix(t[:1]).ld == 64 and asgd.matrix(t.bfloat16()).dtype == asgd.ASGD_BF16
    for bad in (t.T, t[0], t.double(), t[:, ::2]):
        with pytest.raises(ValueError):
            asgd.matrix(bad)
    c, s = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    assert asgd.fp4_matrix(c, s).n_cols == 128
    for a, b in ((c, s[:3]), (c.float(), s), (c[:, :8], s), (torch.zeros(4, 128, dtype=torch.uint8)[:, ::2], s)):
        with pytest.raises(ValueError):
            asgd.fp4_matrix(a, b)
    w = torch.zeros(4, 7, dtype=torch.int32)
    assert asgd.logit_rules(allowed=w).allowed_ld == 7 and asgd.logit_rules(allowed=w[0]).allowed_ld == 0
    assert asgd.logit_rules(allowed=w[:1]).allowed_ld == 7


def test_rule_tensors_of_other_types_and_strides_are_refused():
    b, w = torch.zeros(100), torch.zeros(4, 7, dtype=torch.int32)
    for bad in (b.bfloat16(), b.half(), b.double(), b.int(), b[::2], b[None], b[0]):
        with pytest.raises(ValueError, match="bias"):
            asgd.logit_rules(bias=bad)
    for bad in (w.long(), w.short(), w.bool(), w.float(), w[:, ::2], w[0, ::2], w.T, w[None], w[0, 0]):
        with pytest.raises(ValueError, match="allowed"):
            asgd.logit_rules(allowed=bad)
    r = asgd.logit_rules(bias=b[3:], allowed=w[1:, 2:5])
    assert (r.bias, r.allowed, r.allowed_ld) == (b.data_ptr() + 12, w.data_ptr() + 4 * 9, 7)
    assert asgd.logit_rules(allowed=w.view(torch.uint32)).allowed_ld == 7
    assert asgd.logit_rules(allowed=w[:1].expand(4, 7)).allowed_ld == 0  # one mask for all rows
    assert asgd.logit_rules(bias=b[::50][:1]).bias == b.data_ptr()       # one entry has no stride
    assert asgd.logit_rules(allowed=w[:, ::7]).allowed_ld == 7


def test_rule_tensors_too_short_for_the_logits_are_refused(monkeypatch):
    w = torch.zeros(4, 4, dtype=torch.int32)
    bad = [(dict(bias=torch.zeros(99)), "of 99 labels"), (dict(allowed=w[:3]), "for 3 rows"),
           (dict(allowed=w[:1]), "for 1 rows"), (dict(allowed=w[:, :3]), "of 96 labels"),
           (dict(allowed=w[0, :3]), "of 96 labels")]
    monkeypatch.setitem(asgd._binding._n_labels, None, 100)
    for kw, word in bad:
        rules = asgd.logit_rules(**kw)
        with pytest.raises(ValueError, match=word):
            asgd.asgd_logits_topk(mat(), 1, A, rules=rules, workspace=BIG)
        with pytest.raises(ValueError, match=word):
            asgd.asgd_predict_topk_rules(None, csr(), 1, A, rules=rules, workspace=BIG)
    # what covers the logits goes on to the library, which refuses something else
    for kw in (dict(bias=torch.zeros(100), allowed=w), dict(allowed=w[0]), dict(allowed=w[:1].expand(4, 4))):
        refused(asgd.ASGD_EINVAL, "k must", asgd.asgd_logits_topk, mat(), 0, A, rules=asgd.logit_rules(**kw), workspace=BIG)


def test_reference_pins():
    # hand-computed: the largest magnitude 7.1 gives scale 2^0, 5 and 0.25 are midpoints
    x = np.zeros((1, 32))
    x[0, :6] = [7.1, 5.0, 0.25, -0.75, 2.6, 1e-3]
    v, c, s = ref.quantize(x)
    assert s[0, 0] == 127 and list(v[0, :6]) == [6.0, 4.0, 0.0, -1.0, 3.0, 0.0] and list(c[0, :4]) == [7, 6, 0, 10]
    # a teacher with one label: the loss is T^2 times its cross-entropy
    z = np.array([[1.0, 2.0, 0.5]])
    loss, g, p, _ = ref.distill(z, np.array([[1]]), np.array([[3.0]]), 2.0)
    e = np.exp(z[0] / 2)
    assert np.isclose(loss[0], -4 * np.log(e[1] / e.sum())) and np.allclose(g[0], 2 * (e / e.sum() - [0, 1, 0]))
    s = ref.scores(np.array([[2.0, -2.0, 1.0]]), seen=[[0, 1, 0]], repetition=2.0, frequency=0.5, presence=0.25)
    assert list(s[0]) == [1.0 - 1.25, -4.0 - 0.75, 1.0]


def test_distill_gradient_agrees_with_differences():
    r = np.random.default_rng(3)
    z, T = r.normal(0, 2, (2, 9)), 1.7
    ids, t = np.array([[1, 4, 4], [7, 99, 0]]), r.normal(0, 1, (2, 3))
    w = np.array([0.3, 1.1])
    _, g, _, _ = ref.distill(z, ids, t, T, w)
    for i in range(2):
        for j in range(9):
            d = np.zeros_like(z)
            d[i, j] = 1e-5
            up, down = (ref.distill(z + s * d, ids, t, T, w)[0] for s in (1, -1))
            assert abs(w @ (up - down) / 2e-5 - g[i, j]) < 1e-8
