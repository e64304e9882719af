"""The distillation loss on a teacher's alternatives and its gradient against the plain form in 64 bits, within bounds that count roundings
(student_oracle)."""
import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import student_oracle as so
from test_gpu_worker_losses import TYPES, close, f32, guarded, i64, make

pytestmark = pytest.mark.gpu


def teacher(x64, k, rng, temperature, noise=0.7, ragged=True):
    """Ids and log-probabilities of a teacher near the student: its k likeliest words, fewer in some rows."""
    T, V = x64.shape
    ids, logp = np.full((T, k), -1, np.int64), np.full((T, k), -np.inf, np.float32)
    for t in range(T):
        z = x64[t] + noise * rng.standard_normal(V)
        i, p = so.top(z, k, temperature)
        if ragged and t % 3 == 1:
            i, p = i[:max(1, k - k // 3)], p[:max(1, k - k // 3)]
        ids[t, :len(i)], logp[t, :len(p)] = i, p
    return ids, logp


def check_loss(x, x64, y, ids, tlogp, w, dtype, *, ce=0.0, renormalise=False, temperature=1.0, scale=0.5, pad=0, shift=0, rows=None):
    T, V = x64.shape
    stats, kl = torch.full((4,), 9.0, device="cuda"), torch.full((T,), 9.0, device="cuda")
    d, check = guarded(x, pad=pad, shift=shift)
    args = dict(targets=None if y is None else i64(y), weights=None if w is None else f32(w), scale=scale, ce_coef=ce, renormalise=renormalise,
                temperature=temperature)
    star.star_distill_loss(x, i64(ids), f32(tlogp), stats, dlogits=d, kl_out=kl, **args)
    got, got_kl = d.double().cpu().numpy(), kl.double().cpu().numpy()
    sums, errors = np.zeros(4), np.zeros(4)
    for t in range(T):
        wt = 1.0 if w is None else float(w[t])
        if (y is not None and not 0 <= y[t] < V) or wt == 0.0:
            assert (got[t] == 0).all() and got_kl[t] == 0, t
            continue
        r = so.Distilled(x64[t], temperature, None if y is None else y[t], ids[t], tlogp[t], ce, renormalise)
        assert abs(got_kl[t] - r.kl) <= r.kl_error + so.U * abs(r.kl), (t, got_kl[t], r.kl, r.kl_error)
        c = scale * wt / temperature
        want, bound = c * r.d, c * (r.d_error + 4 * so.U * np.abs(r.d))
        bound = bound + so.HALF_STEP[dtype] * (np.abs(want) + bound) + 1e-38
        bad = ~(np.abs(got[t] - want) <= bound)
        assert not bad.any(), (t, int(bad.sum()), np.argwhere(bad)[:4].ravel(), got[t][bad][:4], want[bad][:4], bound[bad][:4])
        s = scale * wt
        sums += s * np.array([r.kl + ce * r.nll, r.kl, r.nll, 1.0])
        errors += s * np.array([r.kl_error + ce * r.nll_error, r.kl_error, r.nll_error, 0.0])
    close(stats, sums, errors + 8 * so.U * np.abs(sums) + 1e-30, "stats")
    check()
    alone = torch.zeros(4, device="cuda")
    star.star_distill_loss(x, i64(ids), f32(tlogp), alone, **args)
    assert torch.equal(alone, stats)
    star.star_distill_loss(x, i64(ids), f32(tlogp), alone, dlogits=x, **args)          # in the logits' place
    assert torch.equal(alone, stats) and torch.equal(x, d)


SIZES = [(1, 2, 0), (2, 7, 0), (3, 8, 1), (5, 64, 0), (4, 1000, 5), (7, 1003, 0), (3, 4096, 0), (2, 4111, 3), (3, 16390, 0), (1, 32000, 0), (3, 32003, 0),
         (2, 50021, 11), (2, 65543, 1), (1, 131072, 0), (2, 140003, 3), (1, 262147, 0), (150, 515, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ce,renormalise", [(0.0, False), (0.3, False), (0.0, True), (0.3, True)])
@pytest.mark.parametrize("T,V,pad", SIZES)
def test_distillation(T, V, pad, ce, renormalise, dtype):
    temperature, k = (2.0 if T % 2 else 1.0), [1, 20, 64, 128, 65][(T + V + pad) % 5]
    x, x64, y, rng = make(T, V, dtype, seed=4, pad=pad, masked=0.3 if T > 2 else 0.0, shift=pad % 3)
    w = rng.random(T).astype(np.float32)
    if T > 4:
        w[2] = 0.0
    ids, tlogp = teacher(x64, k, rng, temperature)
    check_loss(x, x64, y, ids, tlogp, w, dtype, ce=ce, renormalise=renormalise, temperature=temperature, pad=pad, shift=pad % 3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5000, 140003])
def test_without_targets_and_weights(V, dtype):
    x, x64, _, rng = make(3, V, dtype, seed=6)
    ids, tlogp = teacher(x64, 20, rng, 1.0)
    check_loss(x, x64, None, ids, tlogp, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [130, 9000, 140003])
def test_words_in_any_order(V, dtype):
    """Repeated and unknown words, the first and the last of a row, shares of 0, the taken token among the words and not."""
    T, k = 4, 100
    x, x64, y, rng = make(T, V, dtype, seed=8, pad=1, shift=1)
    ids = rng.integers(0, V, (T, k))
    tlogp = np.log(rng.random((T, k)) / k).astype(np.float32)
    ids[:, 0], ids[:, 1], ids[:, 2], ids[:, 3], ids[:, 50], ids[:, 99] = V - 1, 0, V - 1, 1, ids[:, 49], 0
    ids[:, 7], ids[:, 9] = -1, V
    ids[0, 11], ids[1, 11], ids[2, 11] = 2 ** 40, -2 ** 40, y[2]
    tlogp[:, 3], tlogp[:, 21] = -np.inf, -np.inf
    check_loss(x, x64, y, ids, tlogp, None, dtype, ce=0.4)
    x, x64, y, _ = make(T, V, dtype, seed=8, pad=1, shift=1)
    check_loss(x, x64, y, ids, tlogp, None, dtype, ce=0.4, renormalise=True)


def test_all_words_in_one_place():
    """Words that one thread owns all of: one after the other, and a whole stride apart."""
    for V, dtype, stride in ((140003, "bf16", 8 * 1024), (70003, "bf16", 8 * 1024), (70001, "f32", 4 * 1024), (3000, "f32", 4 * 256), (9000, "bf16", 1)):
        x, x64, y, rng = make(2, V, dtype, seed=9)
        n = min(100, (V - 10) // stride)
        ids = 5 + np.arange(n)[None, :] * stride + np.zeros((2, 1), np.int64)
        tlogp = np.log(rng.random((2, n)) / (n + 1)).astype(np.float32)
        check_loss(x, x64, y, ids, tlogp, None, dtype, ce=0.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [200, 70003, 140003])
def test_a_sure_student(V, dtype):
    """All but 1e-9 to 1e-30 of the student's probability on the named words: the rest's share keeps its digits."""
    T, k = 3, 4
    x, _, y, rng = make(T, V, dtype, seed=10)
    x[:, 10:14] = torch.tensor([[20.0, 21, 22, 23], [40.0, 41, 42, 43], [80.0, 81, 82, 83]], device="cuda").to(x.dtype)
    x64 = x.double().cpu().numpy()
    ids = np.tile(np.arange(10, 14), (T, 1))
    tlogp = np.log(np.array([[0.1, 0.2, 0.3, 0.3999], [0.25, 0.25, 0.25, 0.2499], [0.1, 0.2, 0.3, 0.39]])).astype(np.float32)
    check_loss(x, x64, y, ids, tlogp, None, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [60, 300, 3000, 40001, 140003])
def test_logits_of_any_size(V, dtype):
    """Values far apart, values far from 0 that lie close together, and named words far above and far below the others."""
    rng = np.random.default_rng(V)
    x = np.stack([rng.standard_normal(V) * 1e5, 3e4 + rng.standard_normal(V), -1e6 + rng.standard_normal(V), rng.standard_normal(V), rng.standard_normal(V)])
    x[3, :4] += 300.0
    x[4, :4] -= 300.0
    x = torch.from_numpy(x.astype(np.float32)).to(TYPES[dtype])
    x64 = x.double().numpy()
    ids = np.tile(np.arange(6) * 7 % V, (5, 1))
    ids[3:] = np.arange(6)
    tlogp = np.log(np.tile([0.3, 0.2, 0.1, 0.1, 0.1, 0.1], (5, 1))).astype(np.float32)
    kl, d = torch.zeros(5, device="cuda"), torch.zeros(5, V, dtype=TYPES[dtype], device="cuda")
    star.star_distill_loss(x.cuda(), i64(ids), f32(tlogp), torch.zeros(4, device="cuda"), dlogits=d, kl_out=kl, scale=1.0, temperature=0.9)
    temperature = float(np.float32(0.9))
    for t in range(5):
        r = so.Distilled(x64[t], temperature, None, ids[t], tlogp[t], 0.0, False)
        assert abs(float(kl[t]) - r.kl) <= r.kl_error + so.U * abs(r.kl), (t, float(kl[t]), r.kl, r.kl_error)
        c = 1.0 / temperature
        want, bound = c * r.d, c * (r.d_error + 4 * so.U * np.abs(r.d))
        assert (np.abs(d[t].double().cpu().numpy() - want) <= bound + so.HALF_STEP[dtype] * (np.abs(want) + bound) + 1e-38).all(), t


def test_a_student_that_agrees():
    """The teacher's numbers are the student's own: the divergence is that of their rounding to fp32 (squared, below 1e-12), never negative, and the gradient
    vanishes but for roundings."""
    T, V, k = 4, 5000, 50
    x, x64, y, rng = make(T, V, "f32", seed=11)
    ids, tlogp = teacher(x64, k, rng, 1.0, noise=0.0, ragged=False)
    stats, kl, d = torch.zeros(4, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros_like(x)
    star.star_distill_loss(x, i64(ids), f32(tlogp), stats, dlogits=d, kl_out=kl, scale=1.0)
    for t in range(T):
        r = so.Distilled(x64[t], 1.0, None, ids[t], tlogp[t], 0.0, False)
        assert abs(float(kl[t]) - r.kl) <= r.kl_error and r.kl_error < 1e-6
        assert (np.abs(d[t].double().cpu().numpy() - r.d) <= r.d_error + 1e-38).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [96, 70003, 140003])
def test_banned_words(V, dtype):
    x = torch.randn(7, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
    x[0, V // 3:] = float("-inf")                    # student bans words that the teacher does not name
    x[1, 5:] = float("-inf")                         # nothing left beside the named words
    x[2, 1] = float("-inf")                          # bans a word that the teacher names
    x[3] = float("-inf")
    x[4, V // 2] = float("nan")
    x[5, V // 2] = float("inf")
    x[6, 2] = float("nan")                           # at a named word
    ids = np.tile(np.arange(5), (7, 1))
    tlogp = np.log(np.tile([0.3, 0.2, 0.1, 0.1, 0.2], (7, 1))).astype(np.float32)
    dev, stats, kl, d = x.cuda(), torch.zeros(4, device="cuda"), torch.zeros(7, device="cuda"), torch.full((7, V), 9.0, dtype=TYPES[dtype], device="cuda")
    star.star_distill_loss(dev, i64(ids), f32(tlogp), stats, dlogits=d, kl_out=kl, scale=1.0)
    got, kl = d.double().cpu().numpy(), kl.double().cpu().numpy()
    for t in (0, 1):
        r = so.Distilled(x[t].double().numpy(), 1.0, None, ids[t], tlogp[t], 0.0, False)
        assert abs(kl[t] - r.kl) <= r.kl_error
        bound = r.d_error + 4 * so.U * np.abs(r.d)
        assert (np.abs(got[t] - r.d) <= bound + so.HALF_STEP[dtype] * (np.abs(r.d) + bound) + 1e-38).all()
    assert (got[0, V // 3:] == 0).all() and (got[1, 5:] == 0).all()
    assert kl[2] == np.inf and np.isfinite(got[2]).all() and abs(got[2, 1] + 0.2) < 1e-3
    assert np.isnan(kl[3:]).all() and np.isnan(got[3:]).all()


@pytest.mark.parametrize("shift", [-300.0, -60.0, 200.0])
def test_renormalised_numbers_of_any_scale(shift):
    """Renormalised, a teacher's numbers may be logits: a constant in them makes no difference but for their own rounding (|shift| u)."""
    T, V, k = 3, 900, 30
    x, x64, y, rng = make(T, V, "f32", seed=15)
    ids, tlogp = teacher(x64, k, rng, 1.0, ragged=False)
    moved = (tlogp.astype(np.float64) + shift).astype(np.float32)
    kl, d = torch.zeros(T, device="cuda"), torch.zeros_like(x)
    star.star_distill_loss(x, i64(ids), f32(moved), torch.zeros(4, device="cuda"), dlogits=d, kl_out=kl, renormalise=True, scale=1.0)
    for t in range(T):
        r = so.Distilled(x64[t], 1.0, None, ids[t], (moved[t].astype(np.float64) - shift).astype(np.float64), 0.0, True)
        assert abs(float(kl[t]) - r.kl) <= r.kl_error + so.U * abs(r.kl)
        bound = r.d_error + 4 * so.U * np.abs(r.d)
        assert (np.abs(d[t].double().cpu().numpy() - r.d) <= bound + so.U * np.abs(r.d) + 1e-38).all()


def test_a_teacher_that_says_nothing():
    V = 700
    x, x64, y, rng = make(3, V, "f32", seed=12)
    ids = np.array([[-1, V, 2 ** 33], [3, 4, 5], [-1, -1, -1]])
    tlogp = np.array([[-1.0, -1.0, -1.0], [-np.inf] * 3, [-np.inf] * 3], np.float32)
    for renormalise in (False, True):
        stats, kl, d = torch.zeros(4, device="cuda"), torch.full((3,), 9.0, device="cuda"), torch.full_like(x, 9.0)
        star.star_distill_loss(x, i64(ids), f32(tlogp), stats, dlogits=d, kl_out=kl, renormalise=renormalise, scale=1.0)
        kl = kl.double().cpu().numpy()
        if renormalise:
            assert (kl == 0).all() and bool((d == 0).all())
        else:
            # all of it is the rest's share of 1: nothing where no word is named, -log p of the rest where some are
            p = np.exp(so.log_softmax(x64[1], 1.0)[0])
            assert abs(kl[0]) <= 1e-6 and abs(kl[2]) <= 1e-6 and kl[1] == pytest.approx(-np.log(1 - p[3:6].sum()), abs=1e-6)
            assert float(d[0].abs().max()) <= 1e-6 and float(d[1, 3]) == pytest.approx(p[3], rel=1e-5)


def test_rows_that_do_not_count_are_not_read():
    for V in (100, 5000, 140001):
        x = torch.full((3, V), float("nan"), device="cuda")
        ids, tlogp = torch.zeros(3, 2, dtype=torch.int64, device="cuda"), torch.zeros(3, 2, device="cuda")
        for args in (dict(targets=i64([-100, V, -1])), dict(weights=torch.zeros(3, device="cuda")), dict(targets=i64([0, 1, 2]), weights=torch.zeros(3, device="cuda"))):
            stats, kl, d = torch.full((4,), 9.0, device="cuda"), torch.full((3,), 9.0, device="cuda"), torch.full_like(x, 9.0)
            star.star_distill_loss(x, ids, tlogp, stats, dlogits=d, kl_out=kl, **args)
            assert stats.tolist() == [0.0] * 4 and kl.tolist() == [0.0] * 3 and bool((d == 0).all())


def test_nothing_at_all():
    x, stats = torch.zeros(0, 5, device="cuda"), torch.full((4,), 3.0, device="cuda")
    star.star_distill_loss(x, torch.zeros(0, 2, dtype=torch.int64, device="cuda"), torch.zeros(0, 2, device="cuda"), stats, dlogits=torch.zeros_like(x))
    assert stats.tolist() == [0.0] * 4


def test_gradient_against_differences():
    T, V, h = 5, 300, 2e-2
    x, x64, y, rng = make(T, V, "f32", seed=5)
    ids, tlogp = teacher(x64, 20, rng, 0.8)
    w = f32(rng.random(T))
    for renormalise in (False, True):
        def loss(z, d=None):
            s = torch.zeros(4, device="cuda")
            star.star_distill_loss(z, i64(ids), f32(tlogp), s, targets=i64(y), dlogits=d, weights=w, ce_coef=0.2, renormalise=renormalise, temperature=0.8,
                                   scale=1.0)
            return float(s[0])

        d = torch.zeros_like(x)
        loss(x, d)
        for k in range(4):
            v = f32(rng.standard_normal((T, V)) * 0.2)
            v[torch.arange(T), i64(ids[:, 0])] += 1.0 if k % 2 else -1.0
            slope = (loss(x + h * v) - loss(x - h * v)) / (2 * h)
            # losses of size 10 in fp32: 1e-6 / h; third derivatives of order 10: h^2
            assert slope == pytest.approx(float((d.double() * v.double()).sum()), abs=6e-3, rel=2e-3)


@pytest.mark.parametrize("T", [1000, 5000])
def test_sums_over_many_tokens(T):
    """More tokens than one workgroup adds up, twice in a row on one workspace."""
    V, k = 40, 6
    x, x64, y, rng = make(T, V, "f32", seed=13, masked=0.1)
    ids, tlogp = teacher(x64, k, rng, 1.0)
    w = rng.random(T).astype(np.float32)
    stats = [torch.zeros(4, device="cuda") for _ in range(2)]
    kl = torch.zeros(T, device="cuda")
    space = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    for s in stats:
        star.star_distill_loss(x, i64(ids), f32(tlogp), s, targets=i64(y), weights=f32(w), kl_out=kl, ce_coef=0.1, scale=1.0, workspace=space)
    assert torch.equal(*stats)
    live = (y >= 0) & (y < V)
    rows = [so.Distilled(x64[t], 1.0, y[t], ids[t], tlogp[t], 0.1, False) for t in np.nonzero(live)[0]]
    ww = w[live].astype(np.float64)
    kls, nlls = np.array([r.kl for r in rows]), np.array([r.nll for r in rows])
    want = np.array([(ww * (kls + np.float64(np.float32(0.1)) * nlls)).sum(), (ww * kls).sum(), (ww * nlls).sum(), ww.sum()])
    error = np.array([(ww * np.array([r.kl_error + 0.1 * r.nll_error for r in rows])).sum(), (ww * np.array([r.kl_error for r in rows])).sum(),
                      (ww * np.array([r.nll_error for r in rows])).sum(), 0.0])
    close(stats[0], want, error + 4 * so.U * np.abs(want), "stats")


def test_on_other_streams_and_in_a_graph():
    """Two graphs that share a workspace, replayed in turn between eager calls."""
    T, V, k = 1500, 3001, 12
    x, x64, y, rng = make(T, V, "bf16", seed=7, masked=0.1)
    ids = i64(rng.integers(0, V, (T, k)))
    tlogp, y = f32(np.log(rng.random((T, k)) / k)), i64(y)
    space = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")

    def step(out, renormalise, **more):
        star.star_distill_loss(x, ids, tlogp, out[0], targets=y, dlogits=out[2], kl_out=out[1], ce_coef=0.1, renormalise=renormalise, **more)

    def room():
        return [torch.zeros(4, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros_like(x)]

    want = [room(), room()]
    held = [room(), room()]
    graphs = []
    for i in range(2):
        step(want[i], bool(i))
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            step(held[i], bool(i), workspace=space)
    for n in range(4):
        x.copy_(torch.randn(T, V, device="cuda").to(x.dtype) * 2)
        for i in range(2):
            step(want[i], bool(i))
            for v in held[i]:
                v.fill_(5)
        torch.cuda.synchronize()
        for i in range(2):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(want[i], held[i])), (n, i)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = room()
    step(got, True, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want[1], got))


def test_rows_far_into_a_long_buffer():
    T, V, ld = 3, 1000, 2 ** 31 + 16
    buffer = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    x = buffer.as_strided((T, V), (ld, 1))
    host = torch.randn(T, V).bfloat16()
    x.copy_(host.cuda())
    rng = np.random.default_rng(1)
    ids, tlogp = teacher(host.double().numpy(), 9, rng, 1.0)
    stats = torch.zeros(4, device="cuda")
    star.star_distill_loss(x, i64(ids), f32(tlogp), stats, dlogits=x, scale=1.0)
    for t in range(T):
        r = so.Distilled(host[t].double().numpy(), 1.0, None, ids[t], tlogp[t], 0.0, False)
        bound = r.d_error + 4 * so.U * np.abs(r.d)
        assert (np.abs(x[t].double().cpu().numpy() - r.d) <= bound + so.HALF_STEP["bf16"] * (np.abs(r.d) + bound) + 1e-38).all()


def test_a_teacher_and_a_student_together():
    """A teacher's pass as the student's call takes it: alternatives of one model, the loss of another on them, down to the teacher itself."""
    T, V, k = 40, 7001, 128
    x, x64, y, rng = make(T, V, "bf16", seed=14, masked=0.2)
    theirs = (x.float() + 0.5 * torch.randn(T, V, device="cuda")).to(x.dtype)
    ids, top = torch.zeros(T, k, dtype=torch.int64, device="cuda"), torch.zeros(T, k, device="cuda")
    star.star_top_logprobs(theirs, i64(y), None, top_ids=ids, top_logp=top, temperature=1.5)
    check_loss(x, x64, y, ids.cpu().numpy(), top.cpu().numpy(), None, "bf16", temperature=1.5)
    stats = torch.zeros(4, device="cuda")
    star.star_distill_loss(theirs, ids, top, stats, targets=i64(y), temperature=1.5)
    assert 0.0 <= float(stats[1]) < 1e-6 and float(stats[3]) > 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 3000, 8192, 40001, 140003])
def test_rows_that_are_nowhere_above_zero(V, dtype):
    """All of a row below 0, one thread's words alone, and the largest of them 0 or -0."""
    x, _, y, rng = make(4, V, dtype, seed=12)
    x[0] -= 100.0
    x[1, V // 2:] -= 100.0
    x[2:] = -x[2:].abs()
    x[2, V // 3], x[3, V // 3] = 0.0, -0.0
    x64 = x.double().cpu().numpy()
    ids, tlogp = teacher(x64, 20, rng, 1.0)
    check_loss(x, x64, y, ids, tlogp, None, dtype, ce=0.2)


@pytest.mark.parametrize("share,side", [("named", 0.25), ("named", -0.25), ("rest", 0.25), ("rest", -0.25)])
def test_divergence_where_its_form_turns(share, side):
    """Student and teacher a quarter apart in log p, step by step of a logit through the border, values that fp32 rounds to it among them."""
    n, log_q = 1001, {0.25: -0.9375, -0.25: -0.4375}[side] if share == "named" else {0.25: np.log(0.6), -0.25: np.log(0.4)}[side]
    log_q = np.float32(log_q)
    left = -np.expm1(np.float64(log_q))
    p0 = np.exp(np.float64(log_q) + side) if share == "named" else 1.0 - left * np.exp(side)
    middle = np.array([np.log(1.0 / p0 - 1.0)], np.float32).view(np.int32)[0]
    z = np.zeros((n, 2), np.float32)
    z[:, 1] = (middle + np.arange(n, dtype=np.int32) - n // 2).view(np.float32)
    logp = np.stack([so.log_softmax(row, 1.0)[0] for row in z.astype(np.float64)])
    d = logp[:, 0] - np.float64(log_q) if share == "named" else logp[:, 1] - np.log(left)
    assert (d < side).any() and (d > side).any()
    assert ((np.abs(d) < 0.25) & (np.abs(d.astype(np.float32)) == 0.25)).any()
    ids, tlogp = np.zeros((n, 1), np.int64), np.full((n, 1), log_q)
    check_loss(f32(z), z.astype(np.float64), None, ids, tlogp, None, "f32")
