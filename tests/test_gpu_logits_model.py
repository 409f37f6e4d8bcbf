"""The operators over label logits on a model: a teacher served from a 4-bit label matrix under
rules, and its top logits into a student's distillation steps."""
import numpy as np
import pytest
import torch

import logits_ref as ref
import paper_2110_07029_amd as asgd
from gpu_util import H, RTOL_BF16, RTOL_FP32, Setup, assert_update_close, flush
from paper_2110_07029_amd import synth
from test_gpu_logits import check_rank, dev, host, random_rules, scratch

pytestmark = pytest.mark.gpu

TINY = synth.TINY


def workload(L):
    import dataclasses
    return dataclasses.replace(TINY, n_labels=L)


def first_layer(p, x):
    a = np.tile(p["b1"].astype(np.float64), (x.n_rows, 1))
    for i in range(x.n_rows):
        q = slice(x.indptr[i], x.indptr[i + 1])
        a[i] += x.values[q].astype(np.float64) @ p["W1"][x.indices[q]].astype(np.float64)
    return a


def predict(s, B, k, rules=None, w=None, rows=None, r0=0):
    ids = torch.full((B, k), -7, dtype=torch.int32, device="cuda")
    sc, lse = torch.full((B, k), 7.0, device="cuda"), torch.full((B,), 7.0, device="cuda")
    ws = scratch(asgd.asgd_predict_rules_workspace(s.m, B if rows is None else rows, k))
    asgd.asgd_predict_topk_rules(s.m, s.xb(r0, r0 + B), k, ids, sc, lse, rules=rules, w=w, workspace=ws)
    return ids, sc, lse


def trained_scale(s, seed):
    """Weights that spread the logits."""
    r = np.random.default_rng(seed)
    asgd.asgd_model_set_params(s.m, asgd.ASGD_PARAM_W1, r.normal(0, 0.5, (s.F, H)).astype(np.float32))
    asgd.asgd_model_set_params(s.m, asgd.ASGD_PARAM_W2, r.normal(0, 0.15, (s.L, H)).astype(np.float32))
    asgd.asgd_model_set_params(s.m, asgd.ASGD_PARAM_B2, r.normal(0, 0.3, s.L).astype(np.float32))


@pytest.mark.parametrize("bf16,flags,extra", [(True, 0, 0), (False, 0, 0), (True, asgd.ASGD_UNFUSED_OUTPUT, 0), (False, 0, 1)])
@pytest.mark.parametrize("B,L,rows", [(1, 1000, None), (70, 1003, None), (70, 1003, 32), (300, 517, 299), (300, 517, 1)])
def test_predict_under_rules_ranks_the_models_logits(bf16, flags, extra, B, L, rows):
    s = Setup(workload(L), 300, 300, bf16=bf16, flags=flags, extra=extra)
    try:
        trained_scale(s, B)
        z = torch.empty((B, L), device="cuda")
        asgd.asgd_debug_forward(s.m, s.xb(0, B), None, z_dev=z)
        r = np.random.default_rng(B + L)
        for args in ((0, False, 0, 0.0), (10, True, 3, 0.7)):
            o, rules, allowed, keep = random_rules(r, B, L, *args)
            check_rank(predict(s, B, 6, rules, rows=rows), ref.scores(host(z), **o), 6, allowed)
        # without rules: the plain prediction
        ids, sc = torch.empty((B, 6), dtype=torch.int32, device="cuda"), torch.empty((B, 6), device="cuda")
        asgd.asgd_predict_topk(s.m, s.xb(0, B), 6, ids, sc)
        got = predict(s, B, 6, rows=rows)
        if not bf16 or flags == 0:
            assert (got[0] == ids).float().mean() > 0.99
    finally:
        s.free()


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("B,L,rows", [(5, 1000, None), (130, 2049, 33)])
def test_predict_through_a_4_bit_label_matrix(bf16, B, L, rows):
    s = Setup(workload(L), 200, 200, bf16=bf16)
    try:
        trained_scale(s, 5)
        codes = torch.empty((L, 64), dtype=torch.uint8, device="cuda")
        scales = torch.empty((L, 4), dtype=torch.uint8, device="cuda")
        w = asgd.fp4_matrix(codes, scales)
        asgd.asgd_model_fp4_labels(s.m, w)
        p = s.params()
        v, c, sb = ref.quantize(p["W2"].astype(np.float64))
        assert np.array_equal(scales.cpu().numpy(), sb)
        assert np.array_equal(ref.values_of(codes.cpu().numpy(), sb), v)
        # the same through the product and the ranking by themselves
        a1 = torch.empty((B, H), device="cuda")
        asgd.asgd_debug_forward(s.m, s.xb(0, B), None, a1_dev=a1)
        h = a1.clamp(min=0).bfloat16()
        z = torch.empty((B, L), device="cuda")
        asgd.asgd_fp4_logits(asgd.matrix(h), w, asgd.matrix(z), bias=dev(p["b2"]))
        o, rules, allowed, keep = random_rules(np.random.default_rng(1), B, L, 5, True, 2, 0.8)
        check_rank(predict(s, B, 5, rules, w, rows), ref.scores(host(z), **o), 5, allowed)
        # and the logits are those of the 4-bit matrix
        want = np.maximum(first_layer(p, s.ds.x.rows(0, B)), 0) @ v.T + p["b2"]
        assert np.abs(host(z) - want).max() <= 2.0 ** -8 * (np.abs(want).max() + 10)
    finally:
        s.free()


def distill_oracle(p, x, ids, t, T, lr, extra):
    """Parameters after one step, the loss, and per parameter the sums over absolute values."""
    p = {k: v.astype(np.float64) for k, v in p.items()}
    a1 = first_layer(p, x)
    h = h1 = np.maximum(a1, 0)
    if extra:
        a2 = h1 @ p["Wh"].T + p["bh"]
        h = np.maximum(a2, 0)
    z = h @ p["W2"].T + p["b2"]
    loss, dz, pr, q = ref.distill(z, ids, t, T)
    size = T / x.n_rows * (pr + q)
    g = {"W2": dz.T @ h, "b2": dz.sum(0)}
    mag = {"W2": size.T @ np.abs(h), "b2": size.sum(0)}
    d, md = dz @ p["W2"], size @ np.abs(p["W2"])
    if extra:
        d, md = d * (a2 > 0), md * (a2 > 0)
        g.update(Wh=d.T @ h1, bh=d.sum(0))
        mag.update(Wh=md.T @ h1, bh=md.sum(0))
        d, md = d @ p["Wh"], md @ np.abs(p["Wh"])
    d, md = d * (a1 > 0), md * (a1 > 0)
    g["b1"], mag["b1"] = d.sum(0), md.sum(0)
    g["W1"], mag["W1"] = np.zeros_like(p["W1"]), np.zeros_like(p["W1"])
    for i in range(x.n_rows):
        f = slice(x.indptr[i], x.indptr[i + 1])
        np.add.at(g["W1"], x.indices[f], x.values[f].astype(np.float64)[:, None] * d[i])
        np.add.at(mag["W1"], x.indices[f], np.abs(x.values[f].astype(np.float64))[:, None] * md[i])
    after = {k: p[k] - lr * g[k] for k in g}
    near = np.abs(a1) < 1e-3  # units whose sign the operands' rounding may decide
    return after, loss.mean(), {k: lr * v for k, v in mag.items()}, near


@pytest.mark.parametrize("bf16,extra", [(False, 0), (True, 0), (False, 1), (True, 1)])
@pytest.mark.parametrize("B,L,k,T", [(1, 33, 1, 1.0), (17, 1000, 5, 2.0), (130, 1001, 32, 1.0), (300, 70, 64, 4.0)])
def test_distill_step_updates(bf16, extra, B, L, k, T):
    s = Setup(workload(L), 300, 300, bf16=bf16, flags=asgd.ASGD_UNFUSED_OUTPUT, extra=extra)
    try:
        trained_scale(s, 3)
        before = s.params()
        r = np.random.default_rng(B * L)
        ids = np.stack([np.resize(r.permutation(L), k) for _ in range(B)]).astype(np.int32)
        t = r.normal(3, 1, (B, k)).astype(np.float32)
        if B > 3:
            ids[2], t[2] = ref.EMPTY, -np.inf
            ids[3, 0] = L  # a padding column's index is no label
        x, _ = s.host_batch(0, B)
        lr = 0.25
        loss = asgd.asgd_distill_step(s.m, s.xb(0, B), dev(ids), dev(t), T, lr, want_loss=True)
        after = s.params()
        want, want_loss, mag, _ = distill_oracle(before, x, ids, t, T, lr, extra)
        rtol = RTOL_BF16 if bf16 else RTOL_FP32
        assert abs(loss - want_loss) <= rtol * abs(want_loss), (loss, want_loss)
        assert asgd.asgd_model_last_loss(s.m) == loss
        for n in want:
            assert_update_close(n, before[n], after[n], want[n], rtol, mag[n])
        # the same step twice from the same weights
        for n, v in before.items():
            from gpu_util import SELECT
            asgd.asgd_model_set_params(s.m, SELECT[n], v)
        asgd.asgd_distill_step(s.m, s.xb(0, B), dev(ids), dev(t), T, lr)
        again = s.params()
        assert all(np.array_equal(again[n], after[n]) for n in after)
    finally:
        s.free()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L", [(40, 40_003), (3, 150_001)])
def test_distill_step_of_long_rows(bf16, B, L):
    # rows beyond a workgroup's registers, gradient in place on the model's padded rows, label tiles over all XCDs
    k, T, lr = 20, 2.0, 0.25
    s = Setup(workload(L), 64, 64, bf16=bf16, flags=asgd.ASGD_UNFUSED_OUTPUT)
    try:
        trained_scale(s, 4)
        before = s.params()
        r = np.random.default_rng(L)
        ids = r.integers(0, L, (B, k)).astype(np.int32)
        t = r.normal(3, 1, (B, k)).astype(np.float32)
        ids[0, 0], ids[0, 1], ids[0, 2] = L, L - 1, 0  # a padding column, the last label and the first
        ids[1], t[1] = ref.EMPTY, -np.inf              # no teacher
        ids[2, 4:] = ids[2, 0]                         # one label seventeen times
        x, _ = s.host_batch(0, B)
        loss = asgd.asgd_distill_step(s.m, s.xb(0, B), dev(ids), dev(t), T, lr, want_loss=True)
        after = s.params()
        want, want_loss, mag, _ = distill_oracle(before, x, ids, t, T, lr, 0)
        rtol = RTOL_BF16 if bf16 else RTOL_FP32
        assert abs(loss - want_loss) <= rtol * abs(want_loss), (loss, want_loss)
        for n in want:
            assert_update_close(n, before[n], after[n], want[n], rtol, mag[n])
        from gpu_util import SELECT
        for n, v in before.items():
            asgd.asgd_model_set_params(s.m, SELECT[n], v)
        asgd.asgd_distill_step(s.m, s.xb(0, B), dev(ids), dev(t), T, lr)
        again = s.params()
        assert all(np.array_equal(again[n], after[n]) for n in after)
    finally:
        s.free()


def test_rules_too_short_for_the_models_labels_are_refused():
    s = Setup(workload(100), 20, 20)
    try:
        for kw in (dict(bias=torch.zeros(99, device="cuda")), dict(allowed=torch.zeros(3, dtype=torch.int32, device="cuda")),
                   dict(allowed=torch.zeros((1, 4), dtype=torch.int32, device="cuda"))):
            with pytest.raises(ValueError):
                predict(s, 4, 2, asgd.logit_rules(**kw))
        b = torch.zeros(100, device="cuda")
        predict(s, 4, 2, asgd.logit_rules(bias=b))
    finally:
        s.free()


def test_distill_step_needs_stored_logits_and_checks_its_arguments():
    s = Setup(workload(100), 20, 20)
    u = Setup(workload(100), 20, 20, flags=asgd.ASGD_UNFUSED_OUTPUT)
    ids, t = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    try:
        with pytest.raises(asgd.AsgdError) as e:
            asgd.asgd_distill_step(s.m, s.xb(0, 4), ids, t, 1.0, 0.1)
        assert e.value.status == asgd.ASGD_ESTATE
        for kw, word in ((dict(k=513), "k must"), (dict(k=0), "k must"), (dict(T=0.0), "temperature"),
                         (dict(lr=float("nan")), "lr"), (dict(ids=ids.cpu()), "device memory")):
            with pytest.raises(asgd.AsgdError) as e:
                asgd.asgd_distill_step(u.m, u.xb(0, 4), kw.get("ids", ids), t, kw.get("T", 1.0), kw.get("lr", 0.1),
                                       k=kw.get("k", 2))
            assert e.value.status == asgd.ASGD_EINVAL and word in str(e.value)
        codes, scales = torch.zeros((99, 64), dtype=torch.uint8, device="cuda"), torch.zeros((99, 4), dtype=torch.uint8, device="cuda")
        for call in (lambda: asgd.asgd_model_fp4_labels(s.m, asgd.fp4_matrix(codes, scales)),
                     lambda: predict(s, 4, 2, w=asgd.fp4_matrix(codes, scales)), lambda: predict(s, 4, 65)):
            with pytest.raises(asgd.AsgdError) as e:
                call()
            assert e.value.status == asgd.ASGD_EINVAL
        with pytest.raises(asgd.AsgdError) as e:
            asgd.asgd_predict_topk_rules(s.m, s.xb(0, 4), 2, ids, workspace=scratch(256))
        assert e.value.status == asgd.ASGD_ERANGE
    finally:
        s.free()
        u.free()


@pytest.mark.parametrize("bf16", [True, False])
def test_teacher_from_4_bits_under_rules_into_a_students_steps(bf16):
    """The set as it is used: quantize the teacher, take its top logits under rules, and step the
    student; then a training step and a prediction on the same student, as ever."""
    L, B, k, T = 1500, 64, 16, 2.0
    te = Setup(workload(L), 128, 128, bf16=True, seed=5)
    st = Setup(workload(L), 128, 128, bf16=bf16, flags=asgd.ASGD_UNFUSED_OUTPUT, ds=te.ds)
    try:
        trained_scale(te, 8)
        codes = torch.empty((L, 64), dtype=torch.uint8, device="cuda")
        scales = torch.empty((L, 4), dtype=torch.uint8, device="cuda")
        w = asgd.fp4_matrix(codes, scales)
        asgd.asgd_model_fp4_labels(te.m, w)
        o, rules, allowed, keep = random_rules(np.random.default_rng(3), B, L, 5, True, 2, 0.5)
        for step in range(3):
            r0 = 32 * step
            ids, sc, lse = predict(te, B, k, rules, w, rows=40, r0=r0)
            before = st.params()
            loss = asgd.asgd_distill_step(st.m, st.xb(r0, r0 + B), ids, sc, T, 0.5, want_loss=True)
            flush(f"  step {step}: loss {loss:.5f}")
            want, want_loss, mag, _ = distill_oracle(before, st.host_batch(r0, r0 + B)[0], ids.cpu().numpy(),
                                                     sc.cpu().numpy(), T, 0.5, 0)
            rtol = RTOL_BF16 if bf16 else RTOL_FP32
            assert abs(loss - want_loss) <= rtol * want_loss
            after = st.params()
            for n in want:
                assert_update_close(n, before[n], after[n], want[n], rtol, mag[n])
            assert (ids.cpu().numpy()[B // 2] == ref.EMPTY).all()  # the row that the mask empties
        asgd.asgd_train_step(st.m, st.xb(0, B), st.yb(0, B), 0.1, want_loss=True)
        check = predict(st, 8, 3)
        z = torch.empty((8, L), device="cuda")
        asgd.asgd_debug_forward(st.m, st.xb(0, 8), None, z_dev=z)
        check_rank(check, ref.scores(host(z)), 3)
    finally:
        te.free()
        st.free()
