"""The example's students: norm, head, a teacher's alternatives, distillation loss, weight gradient from the kept bytes, the norm's gradient, group update,
one behind the other as they are used.  The gradient row of one of them against the same formulas in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import student_oracle as so

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "language_model_workers.py")
    spec = importlib.util.spec_from_file_location("language_model_workers", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_students_run(example):
    teacher = torch.randn(example.VOCAB, example.WIDTH, device="cuda").bfloat16()
    losses = example.distil(teacher, rounds=3)
    assert len(losses) == 3 and all(np.isfinite(losses)) and all(v >= 0 for v in losses)


def test_gradient_row(example):
    """Every step's result from the step before it, as the call got it: what the row holds is the chain of them."""
    V, K, T = example.VOCAB, example.WIDTH, example.TOKENS
    teacher = torch.randn(V, K, device="cuda").bfloat16() * 0.3
    student, params = example.Student(0, "cuda"), example.Student.parameters("cuda").bfloat16()
    residual = torch.randn(T, K, device="cuda").bfloat16()
    stats = student.gradient(params, teacher, residual)
    gain, h = params[V * K:].double().cpu().numpy(), student.total.double().cpu().numpy()
    rstd = 1.0 / np.sqrt((h * h).mean(axis=1) + 1e-6)
    y = h * rstd[:, None] * gain
    assert (np.abs(student.y.double().cpu().numpy() - y) <= np.abs(y) * (4 * so.U + 2.0 ** -8) + 1e-38).all()
    logits, ids, logp = student.logits.double().cpu().numpy(), student.ids.cpu().numpy(), student.logp.cpu().numpy()
    rows = [so.Distilled(logits[t], 1.0, None, ids[t], logp[t], 0.0, False) for t in range(T)]
    want = sum(r.kl for r in rows) / T
    assert abs(float(stats[0]) - want) <= sum(r.kl_error for r in rows) / T + 8 * so.U * abs(want)
    d = np.stack([r.d for r in rows]) / T
    bound = np.stack([r.d_error + 4 * so.U * np.abs(r.d) for r in rows]) / T
    got = student.dlogits.double().cpu().numpy()
    assert (np.abs(got - d) <= bound + 2.0 ** -8 * (np.abs(d) + bound) + 1e-38).all()
    # the head's gradient is that of the kept values, sums of T products in fp32
    kept = torch.zeros(T, K, device="cuda")
    star.star_act_unpack(student.packed, kept)
    kept = kept.double().cpu().numpy()
    row = student.row.double().cpu().numpy()
    head, size = got.T @ kept, np.abs(got).T @ np.abs(kept)
    assert (np.abs(row[:V * K].reshape(V, K) - head) <= so.U * (T + 8) * size + 1e-38).all()
    # the gain's, from dy as the norm's gradient got it
    dy = student.dy.double().cpu().numpy()
    dx, dgain, dx_bound, dgain_size = so.norm_grad(dy, h, gain, rstd, None)
    assert (np.abs(row[V * K:] - dgain) <= so.U * dgain_size * (T + 6) + so.U * np.abs(dgain) + 1e-38).all()
    dx_bound = dx_bound + 4 * so.U * np.abs(dx)
    assert (np.abs(student.dx.double().cpu().numpy() - dx) <= dx_bound + 2.0 ** -8 * (np.abs(dx) + dx_bound) + 1e-38).all()


def test_whole_step_against_differences(example):
    """The loss along a direction of all parameters, in fp32 with inputs that 8 bits hold exactly: gradient row against differences."""
    T, K, V, k = 32, 16, 50, 8
    g = torch.Generator().manual_seed(3)
    h = torch.randint(-7, 8, (T, K), generator=g).float().cuda()
    h[0] = 7.0
    ids = torch.stack([torch.randperm(V, generator=g)[:k] for _ in range(T)]).cuda()
    logp = torch.log_softmax(torch.randn(T, V, generator=g), dim=1).cuda().gather(1, ids).contiguous()
    head, gain = torch.randn(V, K, generator=g).cuda() * 0.3, 1.0 + 0.2 * torch.randn(K, generator=g).cuda()

    def run(w, gn, row=None):
        y, rstd = torch.empty_like(h), torch.empty(T, device="cuda")
        star.star_rms_norm(h, gn, y, rstd_out=rstd)
        logits, stats = y @ w.t(), torch.empty(4, device="cuda")
        d = None if row is None else torch.empty_like(logits)
        star.star_distill_loss(logits, ids, logp, stats, dlogits=d, scale=1.0)
        if row is not None:
            dx = torch.empty_like(h)
            star.star_rms_norm_grad(d @ w, h, gn, rstd, dx, dgain=row[V * K:])
            row[:V * K] = (d.t() @ y).reshape(-1)
        return float(stats[0])

    row = torch.zeros(V * K + K, device="cuda")
    run(head, gain, row)
    step = 1e-2
    for seed in range(3):
        g = torch.Generator().manual_seed(10 + seed)
        dw, dg = torch.randn(V, K, generator=g).cuda() * 0.3, torch.randn(K, generator=g).cuda() * 0.3
        slope = (run(head + step * dw, gain + step * dg) - run(head - step * dw, gain - step * dg)) / (2 * step)
        want = float((row[:V * K].double() * dw.reshape(-1).double()).sum() + (row[V * K:].double() * dg.double()).sum())
        # a loss of size 30 in fp32: 2e-6 * 30 / 1e-2; third derivatives of order 30: times 1e-4 / 6 and the direction's size cubed
        assert slope == pytest.approx(want, abs=2e-2, rel=2e-3)
