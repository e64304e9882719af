"""Rows whose values are large against their differences: a mask's value all over, logits shifted by a constant, temperatures at the ends of
their range.  Log-probabilities and gradients depend on differences only, and so do the bounds here: they are those of the same rows
less their maximum (worker_oracle).  Vocabularies and rows take every way through the launches."""
import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import worker_oracle as wo

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BASES = [30.0, 1000.0, -1000.0, 1e6, -1e6, 4e6, 1e10, -1e10, 1e30, -1e30, "most", "least"]
TEMPERATURES = [1e-4, 1e-3, 0.7, 1.0, 1e4]
# (vocabulary, rows): a wave a row with 1, 2, 4, 8 chunks a lane, workgroups of 256 and 1024, sections (up to 128 rows), then more
# rows than are cut into sections at every size where a row's place changes
SHAPES = {"f32": [(37, 12), (500, 12), (1003, 12), (2001, 12), (4001, 12), (8001, 12), (16001, 130), (32001, 130), (40001, 130), (50021, 130), (65001, 130),
                  (70001, 130), (16001, 12), (70001, 12)],
          "bf16": [(77, 12), (1003, 12), (2001, 12), (4003, 12), (8003, 12), (16001, 12), (32003, 130), (65001, 130), (80003, 130), (104003, 130), (131003, 130),
                   (140003, 130), (32003, 12), (140003, 12)]}


def large_rows(V, T, dtype, seed=0):
    """Row t: a third of it BASES[t], a third within 8 of the type's steps below, the rest far below or -inf; rows beyond the bases do not
    count.  (device tensor, float64 values, targets among the first two thirds)"""
    rng = np.random.default_rng([seed, V, T])
    info = torch.finfo(TYPES[dtype])
    x = torch.zeros(T, V, dtype=TYPES[dtype])
    y = np.full(T, -100, np.int64)
    for t, base in enumerate(BASES):
        top = torch.tensor(info.max if base == "most" else info.min if base == "least" else base, dtype=TYPES[dtype])
        bits = top.view(torch.int32 if dtype == "f32" else torch.int16)
        steps = torch.from_numpy(rng.integers(0, 9, V)).to(bits.dtype)
        kind = rng.random(V)
        kind[0], kind[V - 1] = 0.0, 0.5                      # (both ends of a row hold what matters)
        near = (bits + (steps if float(top) < 0 else -steps)).view(TYPES[dtype]) if base != "least" else top.expand(V)
        low = torch.from_numpy(np.where(rng.random(V) < 0.5, -np.inf, info.min)).to(TYPES[dtype])
        if base == "least":
            low = torch.full((V,), float("-inf"), dtype=TYPES[dtype])
        row = torch.where(torch.from_numpy(kind < 1 / 3), top, torch.where(torch.from_numpy(kind < 2 / 3), near, low))
        x[t] = row
        y[t] = rng.choice(np.nonzero(kind < 1 / 3)[0])
    return x.cuda(), x.double().numpy(), y


def expected(x64, y, temperature):
    """(logp, lse, p, live, bound) from the rows less their maxima; lse with them."""
    T = float(np.float32(temperature))                       # (the call takes it as such)
    m = x64.max(axis=1)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        logp, log_s, p, live, bound = wo.rows(x64 - m[:, None], y, T)
    return logp, log_s + np.where(live, m / T, 0.0), p, live, bound


def f32(a):
    return torch.from_numpy(np.asarray(a, np.float32)).cuda()


def close(got, want, bound, what):
    got = got.double().cpu().numpy()
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size}, first at {np.argwhere(bad)[0]}: {got[bad][0]} against {want[bad][0]}, bound {np.broadcast_to(bound, got.shape)[bad][0]}"


def close_lse(got, want, bound):
    """One rounding to fp32 (which may run over) more than the bound."""
    with np.errstate(over="ignore", invalid="ignore"):
        over = np.abs(want) > float(np.finfo(np.float32).max)
        got = got.double().cpu().numpy()
        assert np.array_equal(got[over], np.sign(want[over]) * np.inf)
        assert np.all(np.abs(got - want)[~over] <= (bound + 4 * wo.U * np.abs(want))[~over])


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("dtype,V,T", [(d, *s) for d in SHAPES for s in SHAPES[d]])
def test_logprobs_and_policy_loss(dtype, V, T, temperature):
    x, x64, y = large_rows(V, T, dtype)
    wlogp, wlse, p, live, bound = expected(x64, y, temperature)
    yd = torch.from_numpy(y).cuda()
    logp, lse = torch.full((T,), 9.0, device="cuda"), torch.full((T,), 9.0, device="cuda")
    star.star_token_logprobs(x, yd, logp, lse_out=lse, temperature=temperature)
    close(logp, wlogp, bound, "logp")
    close_lse(lse, wlse, bound)
    # ratio 1, up to the rounding of old_logp; a positive advantage: the slope is -ratio
    old = wlogp.astype(np.float32)
    stats, d, out = torch.zeros(4, device="cuda"), torch.full_like(x, 9.0), torch.full((T,), 9.0, device="cuda")
    star.star_policy_loss(x, yd, f32(old), f32(np.ones(T)), stats, dlogits=d, scale=1.0, temperature=temperature, logp_out=out)
    close(out, wlogp, bound, "logp of the loss")
    c = -np.exp(wlogp - old) * live / float(np.float32(temperature))
    want = wo.dlogits_of(p, y, live, c)
    close(d, want, wo.gradient_bound(want, p, y, live, c, np.abs(c) * (bound + 16 * wo.U), bound, dtype), "dlogits")
    close(stats[0:1], np.array([-np.exp(wlogp - old)[live].sum()]), float((bound + 16 * wo.U)[live].sum()) + 4 * wo.U * len(BASES), "loss")
    alone = torch.zeros(4, device="cuda")
    star.star_policy_loss(x, yd, f32(old), f32(np.ones(T)), alone, scale=1.0, temperature=temperature)
    assert torch.allclose(alone, stats, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("dtype,V,T", [(d, *s) for d in SHAPES for s in SHAPES[d]])
def test_preference_loss(dtype, V, T, temperature):
    x, x64, y = large_rows(V, T, dtype, seed=1)
    wlogp, _, p, live, bound = expected(x64, y, temperature)
    rng = np.random.default_rng(V)
    ref = (wlogp + 0.4 * rng.standard_normal(T)).astype(np.float32)
    offsets, beta, smooth, scale = np.array([0, 3, 5, 8, T]), 0.3, 0.1, 0.7
    yd, loss, margins = torch.from_numpy(y).cuda(), torch.zeros(1, device="cuda"), torch.zeros(2, device="cuda")
    logp, d = torch.full((T,), 9.0, device="cuda"), torch.full_like(x, 9.0)
    star.star_preference_loss(x, yd, f32(ref), offsets, loss, dlogits=d, scale=scale, beta=beta, label_smoothing=smooth, temperature=temperature,
                              logp_out=logp, margins_out=margins)
    close(logp, wlogp, bound, "logp")
    wl, wm, c = wo.preference(wlogp, ref.astype(np.float64), live, None, offsets, beta, smooth, scale)
    pair_err = np.array([beta * bound[offsets[2 * b]:offsets[2 * b + 2]].sum() for b in range(2)])
    close(margins, wm, pair_err + 2 * wo.U * np.abs(wm) + 1e-30, "margins")
    close(loss, np.array([wl]), scale * pair_err.sum() + 4 * wo.U * abs(wl), "loss")
    c = c / float(np.float32(temperature))
    c_err = (scale * beta * pair_err.max() / 4 + scale * beta * smooth * wo.U) / temperature + 10 * wo.U * np.abs(c)
    want = wo.dlogits_of(p, y, live, c)
    close(d, want, wo.gradient_bound(want, p, y, live, c, c_err, bound, dtype), "dlogits")
    star.star_preference_loss(x, yd, f32(ref), offsets, loss, dlogits=x, scale=scale, beta=beta, label_smoothing=smooth, temperature=temperature)
    assert torch.equal(x, d)                                   # in the logits' place


def check_gradient(x, x64, y, temperature, dtype):
    """star_token_logprobs_grad from star_token_logprobs' normaliser, into other memory and in place."""
    T = len(y)
    wlogp, wlse, p, live, bound = expected(x64, y, temperature)
    yd, logp, lse = torch.from_numpy(y).cuda(), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    star.star_token_logprobs(x, yd, logp, lse_out=lse, temperature=temperature)
    close(logp, wlogp, bound, "logp")
    close_lse(lse, wlse, bound)
    dlogp = np.random.default_rng(T).standard_normal(T).astype(np.float32)
    d = torch.full_like(x, 9.0)
    star.star_token_logprobs_grad(x, yd, lse, f32(dlogp), d, temperature=temperature)
    c = dlogp.astype(np.float64) * live / float(np.float32(temperature))
    want = wo.dlogits_of(p, y, live, c)
    # up to 64, of bf16 rows 1024, the normaliser is taken as it was rounded; beyond, the row's own sum is
    rounded = np.where(np.abs(wlse) <= (64.001 if dtype == "f32" else 1024.01), wo.U * np.abs(wlse), 0.0)
    close(d, want, wo.gradient_bound(want, p, y, live, c, 4 * wo.U * c, bound + rounded, dtype), "dlogits")
    star.star_token_logprobs_grad(x, yd, lse, f32(dlogp), x, temperature=temperature)
    assert torch.equal(x, d)


@pytest.mark.parametrize("temperature", TEMPERATURES)
@pytest.mark.parametrize("dtype,V,T", [(d, *s) for d in SHAPES for s in SHAPES[d]])
def test_gradient_of_logprobs(dtype, V, T, temperature):
    x, x64, y = large_rows(V, T, dtype, seed=2)
    check_gradient(x, x64, y, temperature, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature", [0.05, 1.0])
@pytest.mark.parametrize("T,V,pad", [(9, 77, 3), (9, 1003, 0), (9, 4001, 5), (9, 33003, 1), (9, 131075, 0), (600, 8003, 0)])
def test_gradient_of_shifted_logits(T, V, pad, temperature, dtype):
    """Ordinary rows, a constant added: in a launch that holds rows on both sides of 64."""
    rng = np.random.default_rng([T, V])
    shift = np.resize([0.0, 10.0, 30.0, 50.0, -50.0, 200.0, -1000.0, 1000.0, 3000.0], T)
    host = torch.from_numpy((rng.standard_normal((T, V + pad)) * 2 * min(1.0, 4 * temperature) + shift[:, None]).astype(np.float32)).to(TYPES[dtype])
    x = host.cuda()[:, :V]
    y = rng.integers(0, V, T)
    y[:2] = 0, V - 1
    if T > 20:
        y[rng.random(T) < 0.3] = -1
    check_gradient(x, host[:, :V].double().numpy(), y.astype(np.int64), temperature, dtype)


@pytest.mark.parametrize("dtype,V,T", [(d, *s) for d in SHAPES for s in SHAPES[d]])
def test_rows_without_a_log_probability(dtype, V, T):
    """Rows that hold NaN or +inf, or nothing but -inf, have a gradient of NaN; their neighbours, and pairs, none of it."""
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
    x[1, V // 2], x[2, V - 1], x[3], x[5, V // 2] = float("nan"), float("inf"), float("-inf"), float("nan")
    y = np.full(T, -100)
    y[:5] = [0, 1, 2, 3, V - 1]                                # (row 5 does not count)
    dev, yd = x.cuda(), torch.from_numpy(y).cuda()
    logp, lse, d = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.full_like(dev, 9.0)
    star.star_token_logprobs(dev, yd, logp, lse_out=lse)
    assert torch.isnan(logp[:5]).tolist() == [False, True, True, True, False] and bool((logp[5:] == 0).all())
    star.star_token_logprobs_grad(dev, yd, lse, torch.ones(T, device="cuda"), d)
    assert torch.isnan(d).all(dim=1)[:5].tolist() == [False, True, True, True, False]
    assert bool(torch.isfinite(d[[0, 4]]).all()) and bool((d[5:] == 0).all())
    want = -torch.softmax(x[[0, 4]].double(), dim=1)
    want[[0, 1], [0, V - 1]] += 1.0
    p = np.abs(want.numpy())
    close(d[[0, 4]], want.numpy(), 1e-4 * p + wo.HALF_STEP[dtype] * p + 1e-6 * (p > 0.5) + 1e-38, "dlogits")
    margins, loss = torch.zeros(2, device="cuda"), torch.zeros(1, device="cuda")
    star.star_preference_loss(dev, yd, torch.zeros(T, device="cuda"), [0, 2, 4, 5, T], loss, dlogits=d, margins_out=margins)
    assert torch.isnan(margins).tolist() == [True, False] and bool(torch.isnan(loss[0]))
    assert bool(torch.isnan(d[:4]).all()) and bool(torch.isfinite(d[4]).all()) and bool((d[5:] == 0).all())


def test_more_rows_than_one_launch_holds():
    """2^21 rows and more go into several launches: all entry points, against torch in 64 bits on the device."""
    T, V = 2 ** 21 + 77, 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, V, generator=g, device="cuda")
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[::7] = -1
    live, at = y >= 0, torch.arange(T, device="cuda")
    p = torch.softmax(x.double(), dim=1)
    want = torch.where(live, torch.log_softmax(x.double(), dim=1)[at, y.clamp(min=0)], 0.0)
    onehot = torch.zeros(T, V, dtype=torch.float64, device="cuda")
    onehot[at, y.clamp(min=0)] = 1.0
    slope = torch.where(live[:, None], onehot - p, 0.0)
    logp, lse, d = torch.full((T,), 9.0, device="cuda"), torch.zeros(T, device="cuda"), torch.full_like(x, 9.0)
    star.star_token_logprobs(x, y, logp, lse_out=lse)
    assert float((logp - want).abs().max()) < 64 * wo.U
    star.star_token_logprobs_grad(x, y, lse, torch.ones(T, device="cuda"), d)
    assert float((d - slope).abs().max()) < 64 * wo.U
    adv, stats, again = torch.randn(T, generator=g, device="cuda"), torch.zeros(4, device="cuda"), torch.full((T,), 9.0, device="cuda")
    star.star_policy_loss(x, y, logp, adv, stats, dlogits=d, logp_out=again, scale=1.0)
    assert torch.equal(logp, again)
    # (ratios of 1, up to the rounding of log-probabilities below 16 in size)
    assert float((d + adv[:, None].double() * slope).abs().max()) < 6 * 96 * wo.U
    assert float(stats[0]) == pytest.approx(float(-adv.double()[live].sum()), abs=64 * wo.U * float(adv.abs().sum())) and float(stats[3]) == float(live.sum())
    loss, margins, half = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"), T // 2
    star.star_preference_loss(x, y, torch.zeros(T, device="cuda"), [0, half, T], loss, dlogits=d, beta=1e-3, scale=1.0, margins_out=margins)
    m = 1e-3 * (want[:half].sum() - want[half:].sum())
    assert float(margins[0]) == pytest.approx(float(m), abs=1e-3 * 64 * wo.U * T)
    c = -1e-3 / (1 + torch.exp(margins[0].double()))
    sign = torch.where(at < half, 1.0, -1.0)[:, None]
    assert float((d - c * sign * slope).abs().max()) < 1e-3 * 64 * wo.U
