"""Losses on logits and their gradients against the plain forms in 64 bits, within bounds that count roundings
(worker_oracle).  Sizes go where the kernels turn: one token, rows shorter than a wave, vocabularies that put rows off
16 bytes, rows longer than a workgroup holds, padded rows, targets at either end of a row, tokens that do not count."""
import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import worker_oracle as wo

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(T, V, dtype, *, seed=0, pad=0, masked=0.0, shift=0):
    """Logits in rows V + pad apart that begin at element `shift` of their buffer, as (device tensor, float64 values), and
    targets: both ends of a row among them, some not to count."""
    rng = np.random.default_rng([seed, T, V, pad])
    x = rng.standard_normal((T, V + pad)).astype(np.float32) * 2.0
    y = rng.integers(0, V, T)
    y[0] = V - 1
    if T > 1:
        y[1] = 0
    x[np.arange(T), y] += np.where(rng.random(T) < 0.5, 7.0, 0.0)
    off = rng.random(T) < masked
    y[off] = rng.choice([-100, -1, V, V + 3, 2 ** 40], int(off.sum()))
    host = torch.from_numpy(x).to(TYPES[dtype])
    buffer = torch.full((shift + T * (V + pad),), float("nan"), dtype=TYPES[dtype], device="cuda")
    buffer[shift:] = host.cuda().reshape(-1)
    dev = buffer[shift:].view(T, V + pad)[:, :V]
    return dev, host[:, :V].double().numpy(), y.astype(np.int64), rng


def guarded(logits, pad=0, shift=0):
    """Room for a gradient whose surroundings are known: (view, check that nothing outside it was written)."""
    T, V = logits.shape
    whole = torch.full((shift + T * (V + pad) + 64,), 7.0, dtype=logits.dtype, device="cuda")
    view = whole[shift:shift + T * (V + pad)].view(T, V + pad)[:, :V]

    def check():
        mask = torch.ones_like(whole, dtype=torch.bool)
        mask[shift:shift + T * (V + pad)].view(T, V + pad)[:, :V] = False
        assert bool((whole[mask] == 7.0).all()), "written outside the gradient"
    return view, check


def f32(a):
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


def i64(a):
    return torch.from_numpy(np.asarray(a, np.int64)).cuda()


def close(got, want, bound, what):
    got = got.double().cpu().numpy() if isinstance(got, torch.Tensor) else got
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size}, first at {np.argwhere(bad)[0]}: {got[bad][0]} against {want[bad][0]}, bound {np.broadcast_to(bound, got.shape)[bad][0]}"


SIZES = [(1, 1, 0), (1, 7, 0), (3, 8, 0), (2, 63, 1), (5, 64, 0), (4, 1000, 5), (7, 1003, 0), (1, 32000, 0), (3, 32003, 0),
         (2, 50021, 11), (2, 65536, 0), (1, 131072, 0), (2, 131075, 3), (1, 262147, 0), (300, 515, 0), (600, 1024, 8), (1, 600000, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V,pad", SIZES)
def test_logprobs_and_gradient(T, V, pad, dtype):
    temperature = 0.7 if T % 2 else 1.0
    x, x64, y, rng = make(T, V, dtype, pad=pad, masked=0.2 if T > 2 else 0.0, shift=pad % 4)
    logp, lse = torch.full((T,), 9.0, device="cuda"), torch.full((T,), 9.0, device="cuda")
    star.star_token_logprobs(x, i64(y), logp, lse_out=lse, temperature=temperature)
    wlogp, wlse, p, live, bound = wo.rows(x64, y, temperature)
    close(logp, wlogp, bound, "logp")
    close(lse, wlse, bound, "lse")
    only = torch.full((T,), 9.0, device="cuda")
    star.star_token_logprobs(x, i64(y), only, temperature=temperature)
    assert torch.equal(only, logp)
    dlogp = rng.standard_normal(T).astype(np.float32)
    if T > 3:
        dlogp[3] = 0.0
    d, check = guarded(x, pad=(pad + 3) % 8, shift=1)
    star.star_token_logprobs_grad(x, i64(y), lse, f32(dlogp), d, temperature=temperature)
    c = dlogp.astype(np.float64) * live / temperature
    want = wo.dlogits_of(p, y, live, c)
    # (the normaliser that the gradient was given carries its own error, and scaling it one more of its size)
    lse_bound = bound + 4 * wo.U * np.abs(wlse)
    close(d, want, wo.gradient_bound(want, p, y, live, c, 4 * wo.U * c, lse_bound, dtype), "dlogits")
    check()


def policy_inputs(T, V, dtype, **more):
    x, x64, y, rng = make(T, V, dtype, **more)
    return x, x64, y, rng


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kl,high", [(0.0, 0.2), (0.05, 0.28)])
@pytest.mark.parametrize("T,V,pad", SIZES)
def test_policy_loss(T, V, pad, kl, high, dtype):
    temperature, low, scale = (1.0 if T % 2 else 0.7), 0.2, 0.5
    x, x64, y, rng = make(T, V, dtype, seed=1, pad=pad, masked=0.3 if T > 2 else 0.0, shift=pad % 3)
    w = rng.random(T).astype(np.float32)
    if T > 4:
        w[2] = 0.0
    logp64, _, p, live, bound = wo.rows(x64, y, temperature, w)
    # log ratios in steps of 0.01: no border (log 0.8, 1.2, 1.28) within 0.002 of one
    old = (logp64 + np.round(rng.standard_normal(T) * 20) * 0.01).astype(np.float32)
    ref = (logp64 + 0.3 * rng.standard_normal(T)).astype(np.float32)
    adv = rng.standard_normal(T).astype(np.float32)
    if T > 5:
        adv[5] = 0.0
    stats, logp = torch.zeros(4, device="cuda"), torch.zeros(T, device="cuda")
    d, check = guarded(x, pad=pad, shift=pad % 3)
    star.star_policy_loss(x, i64(y), f32(old), f32(adv), stats, dlogits=d, ref_logp=f32(ref) if kl else None, weights=f32(w), scale=scale,
                          clip_low=low, clip_high=high, kl_coef=kl, temperature=temperature, logp_out=logp)
    close(logp, logp64, bound, "logp")
    L, K, clipped, slope, size = wo.policy_terms(logp64, old.astype(np.float64), ref.astype(np.float64), adv.astype(np.float64), low, high, kl)
    sw = scale * w.astype(np.float64) * live
    err = size * (bound + 12 * wo.U) + wo.U * np.abs(L) * 8 + 2 * wo.U * np.abs(adv)
    close(stats[0:1], np.array([(sw * L).sum()]), (sw * err).sum() + 4 * wo.U * np.abs(sw * L).sum() + 1e-30, "loss")
    kerr = np.abs(np.expm1(ref - logp64)) * (bound + 2 * wo.U * np.abs(ref)) + 4 * wo.U * (K + np.abs(ref - logp64))
    close(stats[1:2], np.array([(sw * K).sum()]), (sw * kerr).sum() + 4 * wo.U * (sw * K).sum() + 1e-30, "kl")
    close(stats[2:4], np.array([(sw * clipped).sum(), sw.sum()]), 4 * wo.U * sw.sum() + 1e-30, "shares")
    c = sw * slope / temperature
    want = wo.dlogits_of(p, y, live, c)
    c_err = sw / temperature * (size * (bound + 12 * wo.U + 2 * wo.U * np.abs(old)) + 8 * wo.U * np.abs(slope))
    close(d, want, wo.gradient_bound(want, p, y, live, c, c_err, bound, dtype), "dlogits")
    check()
    # the loss alone, and the gradient in place of the logits
    alone = torch.zeros(4, device="cuda")
    kw = dict(ref_logp=f32(ref) if kl else None, weights=f32(w), scale=scale, clip_low=low, clip_high=high, kl_coef=kl, temperature=temperature)
    star.star_policy_loss(x, i64(y), f32(old), f32(adv), alone, **kw)
    assert torch.allclose(alone, stats, rtol=1e-5, atol=1e-6)
    again = torch.zeros(4, device="cuda")
    star.star_policy_loss(x, i64(y), f32(old), f32(adv), again, dlogits=x, **kw)
    assert torch.equal(again, stats) and torch.equal(x, d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,V,weighted", [
    ([1, 1], 40, False), ([3, 0], 1000, False), ([0, 0, 2, 5], 1003, True), ([7, 9, 1, 30], 32003, False), ([260, 300], 517, True),
    ([2, 3] * 130, 129, True), ([1, 0] * 300, 16, False), ([90, 80, 70, 60, 50, 40], 4096, False)])
@pytest.mark.parametrize("smooth", [0.0, 0.1])
def test_preference_loss(lengths, V, weighted, smooth, dtype):
    T, beta, temperature = sum(lengths), 0.3, 0.9
    x, x64, y, rng = make(T, V, dtype, seed=2, pad=3, masked=0.2 if T > 4 else 0.0)
    w = rng.random(T).astype(np.float32) if weighted else None
    if weighted:
        w[T // 2] = 0.0
    offsets = np.concatenate([[0], np.cumsum(lengths)])
    logp64, _, p, live, bound = wo.rows(x64, y, temperature, w)
    ref = (logp64 + 0.4 * rng.standard_normal(T)).astype(np.float32)
    pairs, scale = len(lengths) // 2, 0.7
    loss, margins, logp = torch.zeros(1, device="cuda"), torch.full((pairs,), 9.0, device="cuda"), torch.zeros(T, device="cuda")
    d, check = guarded(x, pad=1)
    star.star_preference_loss(x, i64(y), f32(ref), offsets, loss, dlogits=d, weights=None if w is None else f32(w), scale=scale, beta=beta,
                              label_smoothing=smooth, temperature=temperature, logp_out=logp, margins_out=margins)
    close(logp, logp64, bound, "logp")
    wl, wm, c = wo.preference(logp64, ref.astype(np.float64), live, w, offsets, beta, smooth, scale)
    token = bound * (1 if w is None else np.abs(w))
    pair_err = np.array([beta * token[offsets[2 * b]:offsets[2 * b + 2]].sum() for b in range(pairs)])
    close(margins, wm, pair_err + 2 * wo.U * np.abs(wm) + 1e-30, "margins")
    close(loss, np.array([wl]), scale * pair_err.sum() + 4 * wo.U * abs(wl), "loss")
    c = c / temperature
    # slope: derivative of the sigmoid at most 1/4; beta, smoothing and scale as fp32 numbers 3 u
    per_token = np.zeros(T)
    for b in range(pairs):
        per_token[offsets[2 * b]:offsets[2 * b + 2]] = scale * beta * pair_err[b] / 4 / temperature
    c_err = (per_token + scale * beta * smooth * wo.U) * (1 if w is None else np.abs(w)) + 10 * wo.U * np.abs(c)
    want = wo.dlogits_of(p, y, live, c)
    close(d, want, wo.gradient_bound(want, p, y, live, c, c_err, bound + 4 * wo.U * 20, dtype), "dlogits")
    check()
    alone = torch.zeros(1, device="cuda")
    star.star_preference_loss(x, i64(y), f32(ref), offsets, alone, weights=None if w is None else f32(w), scale=scale, beta=beta,
                              label_smoothing=smooth, temperature=temperature)
    assert torch.equal(alone, loss)


def test_nothing_at_all():
    x, y, e = torch.zeros(0, 5, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, device="cuda")
    stats, loss = torch.full((4,), 3.0, device="cuda"), torch.full((1,), 3.0, device="cuda")
    star.star_policy_loss(x, y, e, e, stats, dlogits=torch.zeros_like(x))
    star.star_preference_loss(x, y, e, [0], loss, dlogits=torch.zeros_like(x))
    assert stats.tolist() == [0.0] * 4 and loss.tolist() == [0.0]
    star.star_preference_loss(x, y, e, [0, 0, 0], loss)          # one pair of two empty answers: margin 0
    assert abs(float(loss[0]) - np.log(2)) < 1e-6


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 5000, 140001])
def test_no_token_counts(V, dtype):
    T = 3
    x = torch.full((T, V), float("nan"), dtype=TYPES[dtype], device="cuda")          # a row that does not count is not read
    y = i64([-100, V, -1])
    logp, lse, stats, d = (torch.full((n,), 9.0, device="cuda") for n in (T, T, 4, 1))
    d = torch.full((T, V), 9.0, dtype=TYPES[dtype], device="cuda")
    star.star_token_logprobs(x, y, logp, lse_out=lse)
    assert logp.tolist() == [0.0] * T and lse.tolist() == [0.0] * T
    z = torch.zeros(T, device="cuda")
    star.star_policy_loss(x, y, z, z, stats, dlogits=d, kl_coef=0.1, ref_logp=z)
    assert stats.tolist() == [0.0] * 4 and bool((d == 0).all())
    d.fill_(9.0)
    star.star_token_logprobs_grad(x, y, lse, z + 1, d)
    assert bool((d == 0).all())
    d.fill_(9.0)
    loss = torch.zeros(1, device="cuda")
    star.star_preference_loss(x, y, z, [0, 1, 3], loss, dlogits=d)
    assert bool((d == 0).all()) and abs(float(loss[0]) - np.log(2)) < 1e-6
    # weights of 0 say the same of targets that are tokens
    d.fill_(9.0)
    star.star_policy_loss(x, i64([0, 1, 2]), z, z, stats, dlogits=d, weights=z)
    assert stats.tolist() == [0.0] * 4 and bool((d == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [96, 2051, 70003])
def test_infinite_and_lowest_logits(V, dtype):
    """Banned tokens (-inf, or the type's lowest value), rows of nothing but them, NaN and +inf."""
    low = torch.finfo(TYPES[dtype]).min
    x = torch.randn(6, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
    x[0, V // 3:] = float("-inf")
    x[1, V // 3:] = low
    x[2] = low
    x[3] = float("-inf")
    x[4, V // 2] = float("nan")
    x[5, V // 2] = float("inf")
    y = np.array([5, 6, 7, 8, 9, 10])
    ref = torch.log_softmax(x.double(), dim=1).numpy()
    dev, n = x.cuda(), torch.zeros(6, device="cuda")
    lse = torch.zeros(6, device="cuda")
    star.star_token_logprobs(dev, i64(y), n, lse_out=lse)
    got = n.cpu().numpy()
    want = ref[np.arange(6), y]
    tol = wo.U * (V / 64 + 300)
    assert np.all(np.abs(got[:3] - want[:3]) <= tol) and np.all(np.isnan(got[3:]))
    d = torch.full_like(dev, 9.0)
    stats = torch.zeros(4, device="cuda")
    w = f32([1, 1, 1, 0, 0, 0])
    star.star_policy_loss(dev, i64(y), n.nan_to_num(), f32(np.ones(6)), stats, dlogits=d, weights=w, scale=1.0)
    p = np.exp(ref[:3])
    want = p.copy()
    want[np.arange(3), y[:3]] -= 1.0                                  # slope -A r = -1 at r = 1
    close(d[:3], want, 1e-4 * np.abs(want) + wo.HALF_STEP[dtype] * np.abs(want) + 1e-38, "dlogits")
    assert bool((d[:2, V // 3:] == 0).all()) and bool((d[3:] == 0).all())
    assert abs(float(stats[0]) + 3.0) < 1e-4


def test_ratios_that_run_over():
    """exp(logp - old) beyond fp32: held by the clip for a positive advantage, infinite for a negative one, and free
    for one of 0."""
    V = 64
    x = torch.zeros(3, V, device="cuda")
    y, old, adv = i64([1, 2, 3]), f32([-200, -200, -200]), f32([1.0, 0.0, -1.0])
    for n, loss, grad_zero in ((1, -1.2, True), (2, -1.2, True), (3, float("inf"), False)):
        stats, d = torch.zeros(4, device="cuda"), torch.full((n, V), 9.0, device="cuda")
        star.star_policy_loss(x[:n], y[:n], old[:n], adv[:n], stats, dlogits=d, scale=1.0)
        assert float(stats[0]) == pytest.approx(loss)
        assert bool((d[:2] == 0).all())
        if not grad_zero:
            assert not bool(torch.isfinite(d[2]).any())


def test_ties_take_the_unclipped_side():
    """ratio exactly 1 with a clip range of 0: both sides are equal, the derivative is the unclipped one."""
    V = 8
    x, y = torch.zeros(1, V, device="cuda"), i64([3])
    logp = torch.zeros(1, device="cuda")
    star.star_token_logprobs(x, y, logp)
    stats, d = torch.zeros(4, device="cuda"), torch.zeros(1, V, device="cuda")
    star.star_policy_loss(x, y, logp, f32([2.0]), stats, dlogits=d, clip_low=0.0, clip_high=0.0, scale=1.0)
    want = np.full((1, V), 2.0 / V)
    want[0, 3] -= 2.0
    close(d, want, 1e-5, "dlogits")
    assert float(stats[2]) == 0.0


@pytest.mark.parametrize("which", ["policy", "preference"])
def test_gradient_against_differences(which):
    """The loss that the library returns, at logits + h v and - h v, against its own gradient along v."""
    T, V, h = 6, 300, 2e-2
    x, x64, y, rng = make(T, V, "f32", seed=5)
    y = i64(y)
    logp = torch.zeros(T, device="cuda")
    star.star_token_logprobs(x, y, logp, temperature=0.8)
    old, ref = logp - f32([0.05, -0.1, 0.0, 0.5, -0.5, 0.1]), logp + f32(rng.standard_normal(T) * 0.3)
    adv = f32([1, -1, 2, 1, -1, -2])

    def loss(z, d=None):
        if which == "policy":
            s = torch.zeros(4, device="cuda")
            star.star_policy_loss(z, y, old, adv, s, dlogits=d, ref_logp=ref, kl_coef=0.1, temperature=0.8, scale=1.0)
        else:
            s = torch.zeros(1, device="cuda")
            star.star_preference_loss(z, y, ref, [0, 2, 3, 5, 6], s, dlogits=d, beta=0.5, label_smoothing=0.1, temperature=0.8, scale=1.0)
        return float(s[0])

    d = torch.zeros_like(x)
    loss(x, d)
    for k in range(4):
        v = f32(rng.standard_normal((T, V)) * 0.2)
        v[torch.arange(T), y] += 1.0 if k % 2 else -1.0
        slope = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
        # losses of size 10 in fp32: 1e-6 / h; third derivatives of order 10: h^2
        assert slope == pytest.approx(float((d.double() * v.double()).sum()), abs=6e-3, rel=2e-3)


def test_on_a_stream_of_its_own():
    T, V = 64, 20000
    x, _, y, rng = make(T, V, "bf16", seed=7, masked=0.2)
    y, z, adv = i64(y), torch.zeros(T, device="cuda"), f32(rng.standard_normal(T))
    want, wd = torch.zeros(4, device="cuda"), torch.zeros_like(x)
    star.star_policy_loss(x, y, z - 10, adv, want, dlogits=wd)
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.zeros_like(x)
    late, stats, d = torch.zeros_like(x), torch.zeros(4, device="cuda"), torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            other.copy_(x)                     # the logits arrive late, on this stream
        late.copy_(other)
        star.star_policy_loss(late, y, z - 10, adv, stats, dlogits=d)
    stats2, d2 = torch.zeros(4, device="cuda"), torch.zeros_like(x)
    side2 = torch.cuda.Stream()
    side2.wait_stream(side)
    star.star_policy_loss(late, y, z - 10, adv, stats2, dlogits=d2, stream=side2)
    side.synchronize(), side2.synchronize()
    assert torch.equal(stats, want) and torch.equal(d, wd) and torch.equal(stats2, want) and torch.equal(d2, wd)


@pytest.mark.parametrize("T", [5, 700])
def test_in_a_graph(T):
    V = 3001
    x, _, y, rng = make(T, V, "bf16", seed=8, masked=0.1)
    y, z, adv = i64(y), torch.full((T,), -8.0, device="cuda"), f32(rng.standard_normal(T))
    offsets = [0, T // 3, T]
    stats, d, loss, d2 = torch.zeros(4, device="cuda"), torch.zeros_like(x), torch.zeros(1, device="cuda"), torch.zeros_like(x)

    def step():
        star.star_policy_loss(x, y, z, adv, stats, dlogits=d, ref_logp=z, kl_coef=0.01)
        star.star_preference_loss(x, y, z, offsets, loss, dlogits=d2)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(torch.randn(T, V, device="cuda").to(x.dtype) * 2)
        step()
        want = [t.clone() for t in (stats, d, loss, d2)]
        for t in (stats, d, loss, d2):
            t.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (stats, d, loss, d2)):
            assert torch.equal(a, b), i


def test_rows_far_into_a_long_buffer():
    """Row offsets beyond 2^32 bytes and elements: the last rows of a buffer of 9 GB."""
    T, V, ld = 3, 1000, 2 ** 31 + 16
    buffer = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    x = buffer.as_strided((T, V), (ld, 1))
    host = torch.randn(T, V).bfloat16()
    x.copy_(host.cuda())
    y = np.array([1, 500, 999])
    logp = torch.zeros(T, device="cuda")
    star.star_token_logprobs(x, i64(y), logp)
    want, _, p, live, bound = wo.rows(host.double().numpy(), y, 1.0)
    close(logp, want, bound, "logp")
    stats = torch.zeros(4, device="cuda")
    star.star_policy_loss(x, i64(y), logp, f32([1, 1, 1]), stats, dlogits=x, scale=1.0)
    wd = wo.dlogits_of(p, y, live, -np.ones(T))
    close(x, wd, wo.gradient_bound(wd, p, y, live, np.ones(T), 64 * wo.U * np.ones(T), bound, "bf16"), "dlogits")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(300, 1000), (5000, 77), (6, 20000), (200, 9000)])
def test_gradient_and_sums_agree_on_the_clip(T, V, dtype):
    """A clip range of 0 and old log-probabilities that are the present ones: the ratios lie on the border up to what rounding the
    log-probabilities left.  A token is counted as clipped exactly where its gradient row is zero."""
    x, _, y, rng = make(T, V, dtype, seed=11)
    y, logp, stats, d = i64(y), torch.zeros(T, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros_like(x)
    star.star_token_logprobs(x, y, logp)
    star.star_policy_loss(x, y, logp, f32(rng.choice([-1, 1], T)), stats, dlogits=d, clip_low=0.0, clip_high=0.0, scale=1.0)
    assert float(stats[2]) == float((d == 0).all(dim=1).sum())


# more rows than are cut into sections, at every size where a row's place changes: 9 001 to 17 501 chunks of 16 bytes
@pytest.mark.parametrize("V,dtype", [(36001, "f32"), (50021, "f32"), (65536, "f32"), (70001, "f32"), (72003, "bf16"), (100003, "bf16"), (131072, "bf16"),
                                     (150001, "bf16")])
def test_policy_loss_of_long_rows(V, dtype):
    test_policy_loss(129, V, 1, 0.05, 0.28, dtype)


def test_infinite_logits_in_long_rows():
    """Rows of nothing but the lowest value, banned tokens, NaN: where a row is kept in several places all of them see it."""
    T = 130
    for V, dtype in ((40001, "f32"), (90001, "bf16"), (131071, "bf16"), (65535, "f32")):
        low = torch.finfo(TYPES[dtype]).min
        x = torch.randn(T, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
        x[0], x[1], x[2, : V - 20], x[3, 20:] = low, float("-inf"), float("-inf"), low
        x[4, V - 1], x[5, V // 2] = float("nan"), float("inf")
        y = np.full(T, V - 10)
        y[3] = 10
        y[6:] = -100
        ref = torch.log_softmax(x[:6].double(), dim=1).numpy()
        dev, stats, logp, d = x.cuda(), torch.zeros(4, device="cuda"), torch.zeros(T, device="cuda"), torch.full((T, V), 9.0, dtype=TYPES[dtype], device="cuda")
        star.star_policy_loss(dev, i64(y), f32(np.zeros(T)), f32(np.ones(T)), stats, dlogits=d, logp_out=logp, scale=1.0, clip_high=float("inf"))
        got = logp.cpu().double().numpy()
        live = [0, 2, 3]
        assert np.all(np.abs(got[live] - ref[live, y[live]]) <= wo.U * (V / 64 + 300)) and np.all(np.isnan(got[[1, 4, 5]])) and np.all(got[6:] == 0)
        r = np.exp(ref[live, y[live]])
        want = np.exp(ref[live]) * r[:, None]
        want[np.arange(3), y[live]] -= r
        close(d[live], want, (1e-4 + wo.HALF_STEP[dtype]) * np.abs(want) + 1e-38, "dlogits")
        assert bool((d[6:] == 0).all()) and bool(torch.isnan(d[1]).all()) and bool(torch.isnan(d[4]).all())


@pytest.mark.parametrize("smooth,banned,want", [(0.0, "other", 0.0), (1.0, "preferred", 0.0), (0.0, "preferred", float("inf")), (0.1, "other", float("inf"))])
def test_margins_without_bounds(smooth, banned, want):
    """An answer whose policy excludes one of its tokens: the margin is infinite, and costs nothing on the side whose share is 0."""
    V = 40
    x = torch.zeros(4, V, device="cuda")
    x[2 if banned == "other" else 0, 5] = float("-inf")
    y, ref = i64([5, 5, 5, 5]), f32([-3.7, -3.7, -3.7, -3.7])
    loss, margins, d = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), torch.full((4, V), 9.0, device="cuda")
    star.star_preference_loss(x, y, ref, [0, 2, 4], loss, dlogits=d, scale=1.0, label_smoothing=smooth, margins_out=margins)
    assert float(margins[0]) == (float("inf") if banned == "other" else float("-inf"))
    assert float(loss[0]) == want
    assert bool(torch.isfinite(d).all()) and (want != 0.0 or bool((d == 0).all()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,V", [(3, 100), (3, 70003), (130, 40001)])
def test_an_advantage_of_zero_hides_no_nan(T, V, dtype):
    """A row without a log-probability has no loss either, and no gradient, whatever its advantage."""
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
    x[1, V // 2] = float("nan")
    y = np.full(T, 5)
    y[3:] = -100
    dev, old = x.cuda(), f32(np.full(T, -10.0))
    stats, d = torch.zeros(4, device="cuda"), torch.full_like(dev, 9.0)
    star.star_policy_loss(dev, i64(y), old, f32(np.zeros(T)), stats, dlogits=d)
    assert bool(torch.isnan(stats[0])) and bool(torch.isnan(d[1]).all())
    assert bool((d[0] == 0).all()) and bool((d[2:] == 0).all())
    star.star_policy_loss(dev, i64(y), old, f32(np.zeros(T)), stats)
    assert bool(torch.isnan(stats[0]))
    # and nothing of it where the token does not count
    star.star_policy_loss(dev, i64(y), old, f32(np.zeros(T)), stats, dlogits=d, weights=f32(np.arange(T) != 1))
    assert float(stats[0]) == 0.0 and bool((d == 0).all())


def test_kl_of_policies_close_to_each_other():
    """e^d - d - 1 where almost everything cancels: one word in the vocabulary, so that logp is 0 and d is ref_logp.  Beyond 1/4 the difference of
    expm1 (2 steps off at most, 4 u of a number up to 8.3 times the result) and d; below, a series in Horner's form, 8 roundings."""
    x, y, z = torch.zeros(1, 1, device="cuda"), i64([0]), f32([0.0])
    size = [1e-15, 1e-10, 1e-7, 3e-6, 1e-5, 1e-4, 1e-3, 0.01, 0.1, 0.2, 0.2499, 0.2501, 0.4, 1.0, 3.0, 10.0]
    for d in [0.0] + size + [-v for v in size]:
        ref = np.float32(d)
        v = float(ref)
        want = sum(v ** n / np.prod(np.arange(1.0, n + 1)) for n in range(30, 1, -1)) if abs(v) < 1 else np.expm1(v) - v
        stats = torch.zeros(4, device="cuda")
        star.star_policy_loss(x, y, z, z, stats, ref_logp=f32([ref]), kl_coef=1.0, scale=1.0)
        kl = float(stats[1])
        assert kl >= 0.0 and abs(kl - want) <= 40 * wo.U * want, (d, kl, want)
        assert float(stats[0]) == kl


# up to 128 long rows, in sections of 256 times 2, 4 and 8 chunks
@pytest.mark.parametrize("T,V,dtype", [(20, 70003, "f32"), (40, 70003, "f32"), (128, 66001, "f32"), (20, 140003, "bf16"), (33, 140003, "bf16"), (127, 131075, "bf16"),
                                       (128, 16389, "bf16")])
def test_losses_of_rows_in_sections(T, V, dtype):
    test_policy_loss(T, V, 1, 0.05, 0.28, dtype)
    test_logprobs_and_gradient(T, V, 3, dtype)


@pytest.mark.parametrize("T", [1023, 1535, 1536])
def test_policy_loss_on_both_sides_of_a_turn(T):
    """fp32 rows of more than 10240 chunks lie with two to a unit or alone, by their number."""
    V = 41001
    x = torch.randn(T, V, generator=torch.Generator(device="cuda").manual_seed(T), device="cuda")
    y = np.arange(T) * 17 % V
    y[::5] = -1
    z = torch.full((T,), -11.0, device="cuda")
    stats, d = torch.zeros(4, device="cuda"), torch.full_like(x, 9.0)
    star.star_policy_loss(x, i64(y), z, z * 0 - 1, stats, dlogits=d, clip_low=1e3, clip_high=float("inf"), scale=1.0)
    for a in range(0, T, 128):
        logp = torch.log_softmax(x[a:a + 128].double(), dim=1)
        live = torch.from_numpy(y[a:a + 128] >= 0).cuda()
        at = torch.nonzero(live)[:, 0]
        p = torch.exp(logp)
        p[at, i64(y[a:a + 128])[at]] -= 1.0
        r = torch.exp(logp[at, i64(y[a:a + 128])[at]] + 11.0)
        want = torch.zeros_like(p)
        want[at] = -p[at] * r[:, None]                         # slope -A r = r
        # r and p 2^-24 times a row's chain of V / 512 + 64 additions, and what exp makes of it
        assert bool(((d[a:a + 128] - want).abs() <= 4 * wo.U * (V / 512 + 64) * want.abs() + 1e-38).all()), a
