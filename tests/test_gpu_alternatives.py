"""Log-probabilities with entropy and alternatives, and the gradient of any function of them, against the plain forms in 64 bits within bounds
that count roundings (student_oracle).  Ids have to be equal: of equal logits the lowest id first."""
import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import student_oracle as so
from test_gpu_worker_losses import TYPES, close, f32, guarded, i64, make

pytestmark = pytest.mark.gpu


def alternatives(x, y, k, temperature=1.0, **more):
    """Calls with outputs that hold something else before: (logp, entropy, lse, ids, top)."""
    T = x.shape[0]
    logp, entropy, lse = (torch.full((T,), 9.0, device="cuda") for _ in range(3))
    ids, top = torch.full((T, k), 7, dtype=torch.int64, device="cuda"), torch.full((T, k), 9.0, device="cuda")
    star.star_top_logprobs(x, y, None if y is None else logp, entropy_out=entropy, lse_out=lse, top_ids=ids if k else None, top_logp=top if k else None,
                           temperature=temperature, **more)
    return logp, entropy, lse, ids, top


def check_rows(x64, y, k, temperature, got, rows=None):
    logp, entropy, lse, ids, top = (v.double().cpu().numpy() if v.is_floating_point() else v.cpu().numpy() for v in got)
    T, V = x64.shape
    for t in range(T) if rows is None else rows:
        if y is not None and not 0 <= y[t] < V:
            assert entropy[t] == 0 and logp[t] == 0 and lse[t] == 0 and (ids[t] == -1).all() and (top[t] == 0).all()
            continue
        want, z, m = so.log_softmax(x64[t], temperature)
        error = so.logp_error(x64[t], temperature)
        H, H_error = so.entropy(x64[t], temperature)
        assert abs(entropy[t] - H) <= H_error, (t, "entropy", entropy[t], H, H_error)
        norm = float(z[0] - want[0]) if np.isfinite(z[0]) else float(z.max() - want.max())
        assert abs(lse[t] - norm) <= error.max() + 4 * so.U * abs(norm), (t, "lse")
        if y is not None:
            assert logp[t] == want[y[t]] or abs(logp[t] - want[y[t]]) <= error[y[t]], (t, "logp")       # (a banned token: -inf on both sides)
        wid, wtop = so.top(x64[t], k, temperature)
        assert (ids[t] == wid).all(), (t, ids[t], wid)
        there = wid >= 0
        assert (np.abs(top[t][there] - wtop[there]) <= error[wid[there]]).all(), (t, "top")
        assert (top[t][~there] == -np.inf).all()


SIZES = [(1, 1, 0), (2, 7, 0), (3, 8, 1), (5, 64, 0), (4, 1000, 5), (7, 1003, 0), (3, 4096, 0), (2, 4111, 3), (1, 32000, 0), (3, 32003, 0), (2, 50021, 11),
         (2, 65536, 0), (1, 131072, 0), (2, 131075, 3), (1, 262147, 0), (200, 515, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [0, 1, 5, 64, 128])
@pytest.mark.parametrize("T,V,pad", SIZES)
def test_alternatives(T, V, pad, k, dtype):
    temperature = 0.7 if T % 2 else 1.0
    x, x64, y, rng = make(T, V, dtype, pad=pad, masked=0.2 if T > 2 else 0.0, shift=pad % 4)
    got = alternatives(x, i64(y), k, temperature)
    check_rows(x64, y, k, temperature, got)
    # without targets all rows count
    every = alternatives(x, None, k, temperature)
    check_rows(x64, None, k, temperature, every, rows=range(min(T, 8)))
    live = torch.from_numpy((y >= 0) & (y < V)).cuda()
    for a, b in zip(got[1:], every[1:]):
        assert torch.equal(a[live], b[live])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [1, 20, 128])
@pytest.mark.parametrize("V", [5, 129, 3000, 40001, 140003])
def test_ties_go_to_the_lower_id(V, k, dtype):
    """Rows of one value, of two, of zeros of both signs, of a largest value that stands k / 2 times, rising and falling ones."""
    g = torch.Generator().manual_seed(V)
    x = torch.zeros(7, V)
    x[1] = torch.randint(0, 2, (V,), generator=g).float()
    x[2] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0)
    x[3] = torch.randn(V, generator=g).clamp(max=1.0)
    x[3, torch.randperm(V, generator=g)[:max(1, k // 2)]] = 3.0
    x[4] = torch.arange(V) * (20.0 / V)
    x[5] = torch.arange(V, 0, -1) * (20.0 / V)
    x[6] = -1e4
    x = x.to(TYPES[dtype])
    check_rows(x.double().numpy(), None, k, 1.0, alternatives(x.cuda(), None, k))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [96, 2051, 70003, 140003])
def test_banned_words_and_rows_without_probabilities(V, dtype):
    low, k = torch.finfo(TYPES[dtype]).min, 40
    x = torch.randn(8, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
    x[0, V // 3:] = float("-inf")
    x[1, 3:] = float("-inf")                       # fewer words than alternatives
    x[2, V // 3:] = low
    x[3] = low                                     # equal, and far from 0
    x[3, V // 2] = 0.5
    x[4] = float("-inf")
    x[4, V - 1] = 2.0                              # one word
    x[5] = float("-inf")
    x[6, V // 2] = float("nan")
    x[7, V // 2] = float("inf")
    y = np.array([5, 1, 7, V // 2, V - 1, 9, 10, 11])
    got = alternatives(x.cuda(), i64(y), k)
    # (a word that lies 3e38 below has a log-probability of -3e38, rounded)
    check_rows(x.double().numpy(), y, k, 1.0, got, rows=range(5))
    logp, entropy, lse, ids, top = (v.cpu() for v in got)
    assert bool(torch.isnan(logp[5:]).all()) and bool(torch.isnan(entropy[5:]).all())
    assert bool((ids[5:] == -1).all()) and bool(torch.isnan(top[5:]).all())
    assert float(entropy[4]) == 0.0 and float(logp[4]) == 0.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,scale", [(300, 1e5), (300, 1e30), (40001, 3e4), (140003, 1e6)])
def test_logits_of_any_size(V, scale, dtype):
    """Values far apart, and values far from 0 that lie close together."""
    g = torch.Generator().manual_seed(1)
    x = torch.stack([torch.randn(V, generator=g) * scale, scale + torch.randn(V, generator=g), -scale + torch.randn(V, generator=g)]).to(TYPES[dtype])
    y = np.array([0, 1, 2])
    check_rows(x.double().numpy(), y, 17, 0.9, alternatives(x.cuda(), i64(y), 17, 0.9))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,k", [(500, 128), (512, 33), (1024, 128), (1030, 32), (2060, 128), (4096, 127), (4100, 64), (8200, 128), (16400, 128), (32800, 100), (600001, 64),
                                 (600001, 128)])
def test_both_sides_of_a_turn(V, k, dtype):
    """Rows at either side of every size at which their threads change, and far more words than are held; a few that stand out, as models have them."""
    x, x64, y, rng = make(4, V, dtype, seed=21, pad=1, shift=1)
    x[1, rng.integers(0, V, 48)] += 12.0
    x[2, : V // 2] = float("-inf")                 # what is held first may be all banned
    x[3, 17:] = x[3, 17:].clamp(max=0.5)           # many of one value
    x64 = x.double().cpu().numpy()
    check_rows(x64, y, k, 1.0, alternatives(x, i64(y), k))


def test_entropy_of_sure_and_of_uniform_rows():
    V = 1000
    x = torch.zeros(4, V)
    x[1, 3] = 12.0
    x[2, 3] = 40.0
    x[3, :2] = 30.0                                # two words of one half each
    got = alternatives(x.cuda(), None, 2)
    check_rows(x.double().numpy(), None, 2, 1.0, got)
    assert abs(float(got[1][0]) - np.log(V)) <= 1e-6 and abs(float(got[1][3]) - np.log(2)) <= 1e-6


GRADS = [(1, 1, 0), (2, 7, 0), (3, 8, 1), (4, 1000, 5), (7, 1003, 0), (2, 4111, 3), (3, 16390, 0), (2, 32003, 0), (2, 65543, 1), (1, 131072, 0), (2, 140003, 3),
         (1, 262147, 0), (100, 515, 0)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("parts", ["all", "entropy", "top", "logp"])
@pytest.mark.parametrize("T,V,pad", GRADS)
def test_gradient(T, V, pad, parts, dtype):
    temperature, k = (0.7 if T % 2 else 1.0), (0 if parts in ("entropy", "logp") else 40)
    x, x64, y, rng = make(T, V, dtype, seed=3, pad=pad, masked=0.2 if T > 2 else 0.0, shift=pad % 3)
    dlogp = rng.standard_normal(T).astype(np.float32) if parts in ("all", "logp") else None
    dH = rng.standard_normal(T).astype(np.float32) if parts in ("all", "entropy") else None
    ids = dtop = None
    if k:
        ids = rng.integers(0, V, (T, k))
        ids[:, 0] = np.clip(y, 0, V - 1)                       # the taken token among them
        ids[:, 1], ids[:, 2] = V - 1, 0
        if k > 8:
            ids[:, 5], ids[:, 7], ids[:, 6] = ids[:, 4], ids[:, 4], ids[:, 0]      # the same word again
            ids[:, 8] = rng.choice([-1, V, -2 ** 40, 2 ** 40], T)
        dtop = rng.standard_normal((T, k)).astype(np.float32)
    d, check = guarded(x, pad=(pad + 3) % 8, shift=1)
    args = dict(dlogp=None if dlogp is None else f32(dlogp), dentropy=None if dH is None else f32(dH), top_ids=None if ids is None else i64(ids),
                dtop=None if dtop is None else f32(dtop), temperature=temperature)
    star.star_top_logprobs_grad(x, i64(y), d, **args)
    got = d.double().cpu().numpy()
    for t in range(T):
        if not 0 <= y[t] < V:
            assert (got[t] == 0).all()
            continue
        want, bound = so.top_grad(x64[t], temperature, y[t], 0.0 if dlogp is None else float(dlogp[t]), 0.0 if dH is None else float(dH[t]),
                                  [] if ids is None else ids[t], [] if dtop is None else dtop[t].astype(np.float64), dtype)
        bad = ~(np.abs(got[t] - want) <= bound)
        assert not bad.any(), (t, int(bad.sum()), np.argwhere(bad)[:4].ravel(), got[t][bad][:4], want[bad][:4], bound[bad][:4])
    check()
    again = torch.full_like(x, 5.0)
    star.star_top_logprobs_grad(x, i64(y), again, **args)
    assert torch.equal(again, d)                               # the same from run to run, also where words repeat
    star.star_top_logprobs_grad(x, i64(y), x, **args)          # in the logits' place
    assert torch.equal(x, d)


def test_all_words_in_one_place():
    """128 entries that one thread owns all of, each word twice, in rows longer than the registers hold."""
    for V, dtype in ((140003, "bf16"), (300, "f32"), (70001, "f32")):
        x, x64, y, rng = make(2, V, dtype, seed=9)
        first = V // 2
        ids = np.stack([np.arange(128) // 2 % V, first + np.arange(128) % 8 * (1 if dtype == "bf16" else 0)])
        dtop = rng.standard_normal((2, 128)).astype(np.float32)
        d = torch.full_like(x, 9.0)
        star.star_top_logprobs_grad(x, i64(y), d, top_ids=i64(ids), dtop=f32(dtop))
        for t in range(2):
            want, bound = so.top_grad(x64[t], 1.0, y[t], 0.0, 0.0, ids[t], dtop[t].astype(np.float64), dtype)
            assert (np.abs(d[t].double().cpu().numpy() - want) <= bound).all()


def test_gradient_against_differences():
    T, V, h, k = 5, 300, 2e-2, 6
    x, x64, y, rng = make(T, V, "f32", seed=5)
    y = i64(y)
    a, b, c = f32(rng.standard_normal(T)), f32(rng.standard_normal(T)), f32(rng.standard_normal((T, k)))
    ids = alternatives(x, y, k, 0.8)[3]

    def value(z):
        logp, entropy, lse, _, _ = alternatives(z, y, 0, 0.8)
        named = z.double().gather(1, ids) / 0.8 - lse.double()[:, None]
        return float((a.double() * logp.double()).sum() + (b.double() * entropy.double()).sum() + (c.double() * named).sum())

    d = torch.zeros_like(x)
    star.star_top_logprobs_grad(x, y, d, dlogp=a, dentropy=b, top_ids=ids, dtop=c, temperature=0.8)
    for _ in range(4):
        v = f32(rng.standard_normal((T, V)) * 0.2)
        slope = (value(x + h * v) - value(x - h * v)) / (2 * h)
        # a value of size 10 in fp32: 1e-6 / h; third derivatives of order 10: h^2
        assert slope == pytest.approx(float((d.double() * v.double()).sum()), abs=6e-3, rel=2e-3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [96, 70003, 140003])
def test_gradient_of_banned_words(V, dtype):
    x = torch.randn(4, V, generator=torch.Generator().manual_seed(V)).to(TYPES[dtype])
    x[0, V // 3:] = float("-inf")
    x[1] = float("-inf")
    x[2, 5] = float("nan")
    dev, y = x.cuda(), i64([1, 2, 3, -1])
    one, d = torch.ones(4, device="cuda"), torch.full_like(x.cuda(), 9.0)
    ids, dtop = i64([[0, V - 1]] * 4), f32([[1.0, 0.5]] * 4)
    star.star_top_logprobs_grad(dev, y, d, dlogp=one, dentropy=one, top_ids=ids, dtop=dtop)
    got = d.double().cpu().numpy()
    want, bound = so.top_grad(x[0].double().numpy(), 1.0, 1, 1.0, 1.0, [0, V - 1], [1.0, 0.5], dtype)
    assert (np.abs(got[0] - want) <= bound).all()
    assert (got[0, V // 3:V - 1] == 0).all() and got[0, V - 1] == 0.5         # a banned word that the function names
    assert np.isnan(got[1]).all() and np.isnan(got[2]).all() and (got[3] == 0).all()


def test_on_other_streams_and_in_a_graph():
    T, V, k = 60, 9000, 10
    x, _, y, rng = make(T, V, "bf16", seed=7, masked=0.2)
    y, dH = i64(y), f32(rng.standard_normal(T))

    def step(out, z):
        logp, entropy, ids, top, d = out
        star.star_top_logprobs(z, y, logp, entropy_out=entropy, top_ids=ids, top_logp=top)
        star.star_top_logprobs_grad(z, y, d, dlogp=logp, dentropy=dH, top_ids=ids, dtop=top)

    def room():
        return [torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(T, k, dtype=torch.int64, device="cuda"),
                torch.zeros(T, k, device="cuda"), torch.zeros_like(x)]

    want, got, held = room(), room(), room()
    step(want, x)
    torch.cuda.synchronize()
    side, other, late = torch.cuda.Stream(), torch.zeros_like(x), torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            other.copy_(x)
        late.copy_(other)
        step(got, late)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(held, x)
    for i in range(4):
        x.copy_(torch.randn(T, V, device="cuda").to(x.dtype) * 2)
        step(want, x)
        for v in held:
            v.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, held)), i


def test_rows_far_into_a_long_buffer():
    T, V, ld = 3, 1000, 2 ** 31 + 16
    buffer = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda")
    x = buffer.as_strided((T, V), (ld, 1))
    host = torch.randn(T, V).bfloat16()
    x.copy_(host.cuda())
    y = np.array([1, 500, 999])
    got = alternatives(x, i64(y), 9)
    check_rows(host.double().numpy(), y, 9, 1.0, got)
    star.star_top_logprobs_grad(x, i64(y), x, dlogp=f32(np.ones(T)), dentropy=f32(np.ones(T)))
    for t in range(T):
        want, bound = so.top_grad(host[t].double().numpy(), 1.0, y[t], 1.0, 1.0, [], [], "bf16")
        assert (np.abs(x[t].double().cpu().numpy() - want) <= bound).all()


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
    check_rows(x64, y, 20, 1.0, alternatives(x, i64(y), 20, 1.0))
    one, ids, dtop = f32(rng.standard_normal(4)), rng.integers(0, V, (4, 20)), rng.standard_normal((4, 20)).astype(np.float32)
    d = torch.zeros_like(x)
    star.star_top_logprobs_grad(x, i64(y), d, dlogp=one, dentropy=one, top_ids=i64(ids), dtop=f32(dtop))
    for t in range(4):
        want, bound = so.top_grad(x64[t], 1.0, y[t], float(one[t]), float(one[t]), ids[t], dtop[t].astype(np.float64), dtype)
        assert (np.abs(d[t].double().cpu().numpy() - want) <= bound).all(), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [900, 2000, 4000, 8000, 16000, 32000, 60000])
def test_numbers_of_a_row_are_the_same_without_alternatives(V, dtype):
    """Log-probability, entropy and normaliser do not depend on whether a list is asked for: thousands of rows on a card that is full of them, bit for
    bit.  Logits far below 0, where a sum in the place of a maximum would be above all of them."""
    T = 4096
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (torch.randn(T, V, generator=g, device="cuda") * 3 - 50).to(TYPES[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    y[::7] = -1
    listed = alternatives(x, y, 1, 0.7)
    for _ in range(3):
        alone = alternatives(x, y, 0, 0.7)
        assert all(torch.equal(a, b) for a, b in zip(listed[:3], alone[:3]))
    rows = [0, 1, 2, T // 2, T - 1]
    check_rows(x[rows].double().cpu().numpy(), y[rows].cpu().numpy(), 0, float(np.float32(0.7)), [v[rows] for v in alone])
