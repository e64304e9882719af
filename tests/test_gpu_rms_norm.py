"""The root-mean-square norm with the residual's addition and its gradient against the plain form in 64 bits, within bounds that count roundings
(student_oracle); its output in 8 bits against star_act_pack of it, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import student_oracle as so
from test_gpu_worker_losses import TYPES, f32

pytestmark = pytest.mark.gpu

EPS = 1e-6
# (a wave a row, four of them a workgroup; 256 and 1024 threads a row; a row's end at every place of a chunk)
WIDTHS = [1, 2, 7, 8, 64, 250, 255, 256, 511, 512, 1000, 1024, 2048, 2049, 4096, 5003, 8192, 8200, 16384, 16391, 32761, 32768]


def rows(T, K, dtype, rng, pad=0, shift=0, scale=1.0):
    """A tensor in rows K + pad apart that begins at element `shift` of its buffer, NaN around it, and its values in 64 bits."""
    host = torch.from_numpy((rng.standard_normal((T, K)) * scale).astype(np.float32)).to(TYPES[dtype])
    whole = torch.full((shift + T * (K + pad) + 8,), float("nan"), dtype=TYPES[dtype], device="cuda")
    view = whole[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]
    view.copy_(host.cuda())
    return view, host.double().numpy()


def room(T, K, dtype, pad=0, shift=0):
    whole = torch.full((shift + T * (K + pad) + 64,), 7.0, dtype=TYPES[dtype], device="cuda")
    view = whole[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]

    def check():
        mask = torch.ones_like(whole, dtype=torch.bool)
        mask[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K] = False
        assert bool((whole[mask] == 7.0).all()), "written outside the rows"
    return view, check


def round_to(dtype):
    return lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TYPES[dtype]).double().numpy()


def within(got, want, bound, what):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0], np.broadcast_to(bound, got.shape)[bad][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gain_dtype", ["f32", "bf16", None])
@pytest.mark.parametrize("K", WIDTHS)
def test_norm_and_gradient(K, gain_dtype, dtype):
    T = 5 if K > 1024 else 37
    with_residual = K % 3 != 1
    rng = np.random.default_rng([K, T])
    pads = [(0, 0), (3, 1), (8, 0), (5, 3)] if K % 2 else [(0, 0)] * 4
    x, x64 = rows(T, K, dtype, rng, *pads[0])
    res, res64 = rows(T, K, dtype, rng, *pads[1], scale=3.0) if with_residual else (None, None)
    gain = None if gain_dtype is None else torch.from_numpy((1 + 0.3 * rng.standard_normal(K)).astype(np.float32)).to(TYPES[gain_dtype]).cuda()
    g64 = np.ones(K) if gain is None else gain.double().cpu().numpy()
    total, check_total = room(T, K, dtype, *pads[2]) if with_residual else (None, lambda: None)
    y, check_y = room(T, K, dtype, *pads[3])
    rstd = torch.full((T,), 9.0, device="cuda")
    packed = torch.full((star.star_act_bytes(T, K),), 99, dtype=torch.uint8, device="cuda")
    star.star_rms_norm(x, gain, y, residual=res, sum_out=total, rstd_out=rstd, packed=packed, eps=EPS)
    check_total(), check_y()
    h, want, r = so.norm(x64, res64, g64, EPS, round_to(dtype))
    if with_residual:
        assert np.array_equal(total.double().cpu().numpy(), h)
    within(rstd, r, 2 * so.U * r, "rstd")
    within(y, want, np.abs(want) * (4 * so.U + so.HALF_STEP[dtype]) + 1e-38, "y")
    kept = torch.zeros_like(packed)
    star.star_act_pack(y, kept)
    assert torch.equal(kept, packed)

    dy, dy64 = rows(T, K, dtype, rng, *pads[1], scale=0.01)
    dres, dres64 = rows(T, K, dtype, rng, *pads[2], scale=0.01) if with_residual else (None, None)
    dx, check_dx = room(T, K, dtype, *pads[3])
    taken = x if total is None else total
    for dg_dtype, accumulate in (("f32", False), ("bf16", False), ("f32", True)):
        row = torch.full((K + 9,), 0.5, dtype=TYPES[dg_dtype], device="cuda")
        dgain = row[5:5 + K]
        star.star_rms_norm_grad(dy, taken, gain, rstd, dx, dresidual=dres, dgain=dgain, accumulate=accumulate)
        check_dx()
        wdx, wdg, bound, size = so.norm_grad(dy64, h, g64, r, dres64)
        bound = bound + 4 * so.U * np.abs(wdx)                    # (rstd as it was handed over carries one rounding)
        within(dx, wdx, bound + so.HALF_STEP[dtype] * (np.abs(wdx) + bound) + 1e-38, "dx")
        # a workgroup's chain of at most T terms of 3 roundings each
        wdg = wdg + (0.5 if accumulate else 0.0)
        error = so.U * size * (T + 6)
        within(dgain, wdg, error + so.HALF_STEP[dg_dtype] * (np.abs(wdg) + error) + 1e-38, "dgain")
        assert bool((row[:5] == 0.5).all()) and bool((row[5 + K:] == 0.5).all())
    alone, check_alone = room(T, K, dtype)
    star.star_rms_norm_grad(dy, taken, gain, rstd, alone, dresidual=dres)
    assert torch.equal(alone, dx)
    check_alone()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,K", [(1, 4096), (31, 512), (32, 100), (33, 100), (600, 2056), (2100, 64), (2100, 1030), (4099, 1)])
def test_many_rows(T, K, dtype):
    """More rows than workgroups of the gradient; the last block of the packed form not full."""
    rng = np.random.default_rng([K, T])
    x, x64 = rows(T, K, dtype, rng)
    gain = torch.from_numpy((1 + 0.3 * rng.standard_normal(K)).astype(np.float32)).cuda()
    g64 = gain.double().cpu().numpy()
    y, rstd, packed = torch.zeros_like(x), torch.zeros(T, device="cuda"), torch.zeros(star.star_act_bytes(T, K), dtype=torch.uint8, device="cuda")
    star.star_rms_norm(x, gain, y, rstd_out=rstd, packed=packed)
    h, want, r = so.norm(x64, None, g64, EPS, None)
    within(y, want, np.abs(want) * (4 * so.U + so.HALF_STEP[dtype]) + 1e-38, "y")
    kept = torch.zeros_like(packed)
    star.star_act_pack(y, kept)
    assert torch.equal(kept, packed)
    dy, dy64 = rows(T, K, dtype, rng, scale=0.01)
    dx, dgain = torch.zeros_like(x), torch.zeros(K, device="cuda")
    star.star_rms_norm_grad(dy, x, gain, rstd, dx, dgain=dgain)
    wdx, wdg, bound, size = so.norm_grad(dy64, h, g64, r, None)
    bound = bound + 4 * so.U * np.abs(wdx)
    within(dx, wdx, bound + so.HALF_STEP[dtype] * (np.abs(wdx) + bound) + 1e-38, "dx")
    within(dgain, wdg, so.U * size * (T / 100 + 40) + so.U * np.abs(wdg) + 1e-38, "dgain")     # (chains of T / 256 rows and fewer, 4 waves)
    again = torch.zeros(K, device="cuda")
    star.star_rms_norm_grad(dy, x, gain, rstd, dx, dgain=again)
    assert torch.equal(again, dgain)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [40, 1031, 4096, 12000])
def test_in_the_inputs_place(K, dtype):
    T, rng = 9, np.random.default_rng(K)
    x, _ = rows(T, K, dtype, rng, 3, 1)
    res, _ = rows(T, K, dtype, rng, 3, 1)
    gain = torch.ones(K, device="cuda") * 1.5
    total, y, rstd = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(T, device="cuda")
    packed = torch.zeros(star.star_act_bytes(T, K), dtype=torch.uint8, device="cuda")
    star.star_rms_norm(x, gain, y, residual=res, sum_out=total, rstd_out=rstd, packed=packed)
    for sum_at, y_at in (("x", "r"), ("r", "x"), ("r", None), ("x", None), (None, "x"), (None, "r")):
        a, _ = rows(T, K, dtype, np.random.default_rng(0), 3, 1)
        b, _ = rows(T, K, dtype, np.random.default_rng(0), 3, 1)
        a.copy_(x), b.copy_(res)
        place = {"x": a, "r": b}
        s2, y2, p2 = place.get(sum_at, torch.zeros_like(x)), place.get(y_at, torch.zeros_like(x)), torch.zeros_like(packed)
        star.star_rms_norm(a, gain, y2, residual=b, sum_out=s2, packed=p2)
        assert torch.equal(s2, total) and torch.equal(y2, y) and torch.equal(p2, packed), (sum_at, y_at)
    plain, p1 = torch.zeros_like(x), torch.zeros_like(packed)
    star.star_rms_norm(x, gain, plain, packed=p1)
    a, p2 = x.clone(), torch.zeros_like(packed)
    star.star_rms_norm(a, gain, a, packed=p2)                     # y over x
    assert torch.equal(a, plain) and torch.equal(p1, p2)
    dy, _ = rows(T, K, dtype, rng, 3, 1)
    dx, dg = torch.zeros_like(x), torch.zeros(K, device="cuda")
    star.star_rms_norm_grad(dy, total, gain, rstd, dx, dresidual=res, dgain=dg)
    for which in range(3):
        v = [dy.clone(), total.clone(), res.clone()]
        dg2 = torch.zeros(K, device="cuda")
        star.star_rms_norm_grad(v[0], v[1], gain, rstd, v[which], dresidual=v[2], dgain=dg2)
        assert torch.equal(v[which], dx) and torch.equal(dg2, dg), which


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [100, 4096, 9001])
def test_sizes_of_values(K, dtype):
    """Rows of zeros, of values whose squares fp32 does not hold, large and small, and of inf and NaN, which stay in their rows."""
    x = torch.randn(7, K, generator=torch.Generator().manual_seed(K))
    x[0] = 0.0
    x[1] *= 1e25
    x[2] *= 1e-25
    x[3] *= 1e-3
    x[4, K // 2] = float("inf")
    x[5, K - 1] = float("nan")
    x = x.to(TYPES[dtype])
    y, rstd = torch.zeros_like(x).cuda(), torch.zeros(7, device="cuda")
    star.star_rms_norm(x.cuda(), None, y, rstd_out=rstd, eps=1e-12)
    h = x.double().numpy()
    for t in (0, 1, 2, 3, 6):
        want = h[t] / np.sqrt((h[t] ** 2).mean() + np.float64(np.float32(1e-12)))
        # (a rstd of 1e-25 is still a normal number; h rstd and y are rounded once each)
        within(y[t], want, np.abs(want) * (4 * so.U + so.HALF_STEP[dtype]) + 1e-38, t)
    assert bool(torch.isnan(y[4, K // 2])) and bool(torch.isnan(y[5]).all())
    assert bool((y[4, :K // 2] == 0).all())                       # rstd 0, and inf times 0


def test_nothing_at_all():
    x = torch.zeros(0, 8, device="cuda")
    star.star_rms_norm(x, None, torch.zeros_like(x), rstd_out=torch.zeros(0, device="cuda"), packed=torch.zeros(0, dtype=torch.uint8, device="cuda"))
    dgain = torch.full((8,), 3.0, device="cuda")
    star.star_rms_norm_grad(x, x, None, torch.zeros(0, device="cuda"), torch.zeros_like(x), dgain=dgain, accumulate=True)
    assert dgain.tolist() == [3.0] * 8
    star.star_rms_norm_grad(x, x, None, torch.zeros(0, device="cuda"), torch.zeros_like(x), dgain=dgain)
    assert dgain.tolist() == [0.0] * 8


def test_gradient_against_differences():
    T, K, h = 4, 60, 1e-2
    rng = np.random.default_rng(3)
    x, _ = rows(T, K, "f32", rng)
    gain, up = f32(1 + 0.3 * rng.standard_normal(K)), f32(rng.standard_normal((T, K)))

    def value(a, g):
        y = torch.zeros_like(a)
        star.star_rms_norm(a, g, y)
        return float((y.double() * up.double()).sum())

    rstd, y, dx, dgain = torch.zeros(T, device="cuda"), torch.zeros_like(x), torch.zeros_like(x), torch.zeros(K, device="cuda")
    star.star_rms_norm(x, gain, y, rstd_out=rstd)
    star.star_rms_norm_grad(up, x, gain, rstd, dx, dgain=dgain)
    for _ in range(4):
        v, w = f32(rng.standard_normal((T, K))), f32(rng.standard_normal(K))
        # a value of size 20 in fp32: 1e-5 / h; third derivatives of order 10: h^2
        slope = (value(x + h * v, gain) - value(x - h * v, gain)) / (2 * h)
        assert slope == pytest.approx(float((dx.double() * v.double()).sum()), abs=1e-2, rel=2e-3)
        slope = (value(x, gain + h * w) - value(x, gain - h * w)) / (2 * h)
        assert slope == pytest.approx(float((dgain.double() * w.double()).sum()), abs=1e-2, rel=2e-3)


def test_on_other_streams_and_in_a_graph():
    """Two graphs that share a workspace, replayed in turn between eager calls."""
    T, K = 700, 1536
    rng = np.random.default_rng(4)
    x, _ = rows(T, K, "bf16", rng)
    res, dy = torch.zeros_like(x), torch.zeros_like(x)
    gain = torch.ones(K, device="cuda")
    space = torch.zeros(1 << 23, dtype=torch.uint8, device="cuda")

    def room():
        return [torch.zeros_like(x), torch.zeros_like(x), torch.zeros(T, device="cuda"), torch.zeros(star.star_act_bytes(T, K), dtype=torch.uint8, device="cuda"),
                torch.zeros_like(x), torch.zeros(K, device="cuda")]

    def step(o, **more):
        stream = {k: v for k, v in more.items() if k == "stream"}
        star.star_rms_norm(x, gain, o[1], residual=res, sum_out=o[0], rstd_out=o[2], packed=o[3], **stream)
        star.star_rms_norm_grad(dy, o[0], gain, o[2], o[4], dresidual=res, dgain=o[5], **more)

    want, held, graphs = room(), [room(), room()], []
    step(want)
    torch.cuda.synchronize()
    for o in held:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(o, workspace=space)
    for n in range(4):
        for v in (x, res, dy):
            v.copy_(torch.randn(T, K, device="cuda").to(x.dtype))
        step(want)
        for o in held:
            for v in o:
                v.fill_(5)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o in held:
            assert all(torch.equal(a, b) for a, b in zip(want, o)), n
    side, got = torch.cuda.Stream(), room()
    side.wait_stream(torch.cuda.current_stream())
    step(got, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_rows_far_into_a_long_buffer():
    T, K, ld = 3, 1000, 2 ** 31 + 16
    buffer = torch.zeros((T - 1) * ld + K, dtype=torch.bfloat16, device="cuda")
    x = buffer.as_strided((T, K), (ld, 1))
    host = torch.randn(T, K).bfloat16()
    x.copy_(host.cuda())
    gain, rstd = torch.ones(K, device="cuda"), torch.zeros(T, device="cuda")
    y = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")
    star.star_rms_norm(x, gain, y, rstd_out=rstd)
    h, want, r = so.norm(host.double().numpy(), None, np.ones(K), EPS, None)
    within(y, want, np.abs(want) * (4 * so.U + so.HALF_STEP["bf16"]), "y")
    dgain = torch.zeros(K, device="cuda")
    star.star_rms_norm_grad(y, x, gain, rstd, x, dgain=dgain)
    wdx, wdg, bound, size = so.norm_grad(y.double().cpu().numpy(), h, np.ones(K), r, None)
    bound = bound + 4 * so.U * np.abs(wdx)
    within(x, wdx, bound + so.HALF_STEP["bf16"] * (np.abs(wdx) + bound) + 1e-38, "dx")
