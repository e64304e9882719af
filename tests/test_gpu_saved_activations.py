"""Activations kept in 8 bits, and the weight gradient formed from them.  The kept values have to be equal, bit by bit; so do sums
of products of small whole numbers, which fp32 holds exactly; sums of other numbers stay within the roundings of as many
additions."""
import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
import worker_oracle as wo

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def activations(T, K, dtype, seed=0, pad=0, shift=0):
    rng = np.random.default_rng([seed, T, K])
    x = rng.standard_normal((T, K)).astype(np.float32) * np.exp(rng.standard_normal(K)).astype(np.float32)
    if K > 2:
        x[:, K // 2] *= 300.0
        x[: T // 2, K // 3] = 0.0
    x = torch.from_numpy(x).to(TYPES[dtype])
    buffer = torch.full((shift + T * (K + pad),), float("nan"), dtype=TYPES[dtype], device="cuda")
    view = buffer[shift:].view(T, K + pad)[:, :K]
    view.copy_(x.cuda())
    return view, x.float().numpy()


def pack(x):
    T, K = x.shape
    packed = torch.full((star.star_act_bytes(T, K) + 32,), 0xAB, dtype=torch.uint8, device="cuda")
    star.star_act_pack(x, packed)
    assert bool((packed[-32:] == 0xAB).all())
    return packed[:-32]


SIZES = [(1, 1), (1, 16), (2, 3), (31, 17), (32, 16), (33, 40), (64, 64), (100, 250), (257, 129), (5, 1000), (1000, 5), (96, 515)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,K", SIZES)
@pytest.mark.parametrize("pad,shift", [(0, 0), (3, 1)])
def test_kept_values_and_layout(T, K, dtype, pad, shift):
    x, x32 = activations(T, K, dtype, pad=pad, shift=shift)
    packed = pack(x)
    assert np.array_equal(packed.cpu().numpy(), wo.packed_bytes(x32))
    want, _ = wo.kept(x32)
    for out_type in ("f32", "bf16"):
        whole = torch.full((shift + T * (K + pad) + 16,), 7.0, dtype=TYPES[out_type], device="cuda")
        out = whole[shift:shift + T * (K + pad)].view(T, K + pad)[:, :K]
        star.star_act_unpack(packed, out)
        assert np.array_equal(out.double().cpu().numpy(), want)
        out.fill_(7.0)
        assert bool((whole == 7.0).all())


def test_every_border_of_the_format():
    """A block's largest value on and beside 448 * 2^e, values half way between neighbours, subnormal ones, and the ends
    of the range of fp32."""
    e4m3 = [0.0] + [m / 8 * 2.0 ** -6 for m in range(1, 8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8) if (e, m) != (8, 7)]
    half = [(a + b) / 2 for a, b in zip(e4m3, e4m3[1:])]
    values = np.array(e4m3 + half, np.float64)
    values = np.concatenate([values, -values, values * (1 + 2.0 ** -20), values * (1 - 2.0 ** -20)])
    columns = []
    for e in (0, -7, 9, -117, -130, 60, 119):
        for most in (448.0, 448.0 * (1 + 2.0 ** -23), 449.0, 447.9, 256.0, 224.0):
            with np.errstate(over="ignore"):
                for start in range(0, len(values), 31):
                    block = np.concatenate([[most], values[start:start + 31], np.zeros(31)])[:32] * 2.0 ** e
                    columns.append(np.clip(block, -3.4028234663852886e38, 3.4028234663852886e38))
    x32 = np.stack(columns, axis=1).astype(np.float32)
    x = torch.from_numpy(x32).cuda()
    packed = pack(x)
    out = torch.zeros_like(x)
    star.star_act_unpack(packed, out)
    assert np.array_equal(out.cpu().numpy().astype(np.float64), wo.kept(x32)[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_values(dtype):
    x = torch.randn(40, 20).to(TYPES[dtype])
    x[3, 4], x[35, 5], x[7, 6] = float("nan"), float("inf"), float("-inf")
    x[:, 7] = float("inf")
    if dtype == "f32":
        x[0, 8], x[1, 8] = 3.4028234663852886e38, -3.4e38
    dev = x.cuda()
    packed, out = pack(dev), torch.zeros_like(dev)
    star.star_act_unpack(packed, out)
    want, _ = wo.kept(x.float().numpy())
    assert np.array_equal(out.double().cpu().numpy(), want, equal_nan=True)
    assert int(torch.isnan(out).sum()) == 3 + 40


def exact_case(T, N, K, dy_type, seed=0):
    """Whole numbers whose sums of products fp32 holds exactly, and that the kept form holds exactly."""
    rng = np.random.default_rng([seed, T, N, K])
    top = 2 if T > 20000 else 4
    dy = rng.integers(-top, top + 1, (T, N)).astype(np.float32)
    x = rng.integers(-8, 9, (T, K)).astype(np.float32) * 2.0 ** rng.integers(-2, 3, K)
    if dy_type == "f32" and T <= 64:
        # 24 bits of which every one counts: all three parts are needed
        dy = (rng.integers(2 ** 23, 2 ** 24, (T, N)) * rng.choice([-1, 1], (T, N))).astype(np.float32)
        x = np.zeros((T, K), np.float32)
        x[rng.integers(0, T, K), np.arange(K)] = rng.choice([-1, 0.5, 2], K)
    return torch.from_numpy(dy).to(TYPES[dy_type]), torch.from_numpy(x.astype(np.float32))


GRAD_SIZES = [(1, 1, 1), (1, 64, 64), (3, 5, 7), (31, 16, 16), (32, 128, 128), (33, 130, 127), (64, 256, 256), (65, 300, 515), (250, 1024, 1000),
              (96, 17, 2049), (1000, 129, 40), (1031, 512, 64), (8192, 16, 24), (40001, 33, 65), (2048, 257, 260), (512, 2048, 1024)]


@pytest.mark.parametrize("dy_type", ["bf16", "f32"])
@pytest.mark.parametrize("dw_type", ["f32", "bf16"])
@pytest.mark.parametrize("T,N,K", GRAD_SIZES)
def test_weight_gradient_of_whole_numbers(T, N, K, dy_type, dw_type):
    dy, x = exact_case(T, N, K, dy_type)
    packed = pack(x.cuda())
    want = dy.double().t().numpy() @ x.double().numpy()
    dw = torch.full((N * K + 8,), 7.0, dtype=TYPES[dw_type], device="cuda")
    row = dw[3:3 + N * K].view(N, K)                   # a stretch of a gradient row that begins at an odd element
    star.star_act_weight_grad(dy.cuda(), packed, row)
    rounded = torch.from_numpy(want).to(torch.float32)
    assert np.array_equal(rounded.double().numpy(), want)
    assert torch.equal(row.cpu(), rounded.to(TYPES[dw_type]))
    assert bool((dw[:3] == 7.0).all()) and bool((dw[3 + N * K:] == 7.0).all())
    # added to what is there: half of it, negated, so that every element has to change
    before = (-(rounded / 2)).to(TYPES[dw_type])
    row.copy_(before.cuda())
    star.star_act_weight_grad(dy.cuda(), packed, row, accumulate=True)
    assert torch.equal(row.cpu(), (before.float() + rounded).to(TYPES[dw_type]))


@pytest.mark.parametrize("dy_type", ["bf16", "f32"])
@pytest.mark.parametrize("T,N,K,pad,shift", [(77, 100, 90, 0, 0), (77, 104, 96, 8, 0), (300, 256, 300, 3, 1), (4097, 192, 320, 0, 0), (2000, 1000, 1000, 24, 8)])
def test_weight_gradient_of_other_numbers(T, N, K, pad, shift, dy_type):
    rng = np.random.default_rng([3, T, N])
    x, x32 = activations(T, K, "bf16", seed=3)
    dy = torch.from_numpy(rng.standard_normal((T, N)).astype(np.float32) * 1e-3).to(TYPES[dy_type])
    buffer = torch.full((shift + T * (N + pad),), float("nan"), dtype=TYPES[dy_type], device="cuda")
    dev = buffer[shift:].view(T, N + pad)[:, :N]
    dev.copy_(dy.cuda())
    dw = torch.zeros(N, K, device="cuda")
    packed = pack(x)
    star.star_act_weight_grad(dev, packed, dw)
    kept, _ = wo.kept(x32)
    d64 = dy.double().numpy()
    want, size = d64.T @ kept, np.abs(d64).T @ np.abs(kept)
    # one rounding (of up to a whole step) for every addition
    bound = 2 * wo.U * (T + 64) * size + 1e-38
    assert np.all(np.abs(dw.double().cpu().numpy() - want) <= bound)
    again = torch.zeros_like(dw)
    star.star_act_weight_grad(dev, packed, again)
    assert torch.equal(again, dw)                       # the same bits from run to run


@pytest.mark.parametrize("dy_type", ["bf16", "f32"])
@pytest.mark.parametrize("T", [33, 64, 500])
def test_weight_gradient_of_infinite_values(T, dy_type):
    """inf and NaN in one column of dy or x reach that row or column of dw, and nothing else; those behind the last token
    reach nothing."""
    N, K = 70, 90
    dy, x = exact_case(T, N, K, "bf16", seed=9)
    dy = dy.to(TYPES[dy_type])
    x[:, 11] = 1.0
    dy[T - 1, 4], dy[0, 9], x[T - 1, 7] = float("inf"), float("nan"), float("nan")
    whole = torch.full((T + 32, N), float("nan"), dtype=TYPES[dy_type], device="cuda")
    whole[:T] = dy.cuda()
    dw = torch.zeros(N, K, device="cuda")
    star.star_act_weight_grad(whole[:T], pack(x.cuda()), dw)
    got = dw.cpu().double()
    clean = torch.ones(N, K, dtype=torch.bool)
    clean[4], clean[9], clean[:, 7] = False, False, False
    want = dy.double().nan_to_num(0, 0, 0).t() @ x.double().nan_to_num(0)
    assert bool((got[clean] == want[clean]).all())
    assert bool(torch.isnan(got[9]).all()) and bool(torch.isnan(got[:, 7]).all())
    assert not bool(torch.isfinite(got[4, 11])) and float(got[4, 11]) == float("inf")


def test_no_tokens():
    dw = torch.full((5, 9), 7.0, device="cuda")
    empty, packed = torch.zeros(0, 5, device="cuda"), torch.zeros(0, dtype=torch.uint8, device="cuda")
    star.star_act_weight_grad(empty, packed, dw, accumulate=True)
    assert bool((dw == 7.0).all())
    star.star_act_weight_grad(empty, packed, dw)
    assert bool((dw == 0.0).all())


def test_gradient_against_differences():
    """loss = sum of c_ij y_ij with y = kept(x) W^T: its change along a step of W is the gradient's part there."""
    T, N, K = 40, 24, 48
    x, x32 = activations(T, K, "bf16", seed=4)
    c = torch.randn(T, N, generator=torch.Generator().manual_seed(1)).bfloat16()
    packed, dw, held = pack(x), torch.zeros(N, K, device="cuda"), torch.zeros(T, K, device="cuda")
    star.star_act_weight_grad(c.cuda(), packed, dw)
    star.star_act_unpack(packed, held)
    W = torch.randn(N, K, generator=torch.Generator().manual_seed(2)).double()
    V = torch.randn(N, K, generator=torch.Generator().manual_seed(3)).double()
    loss = lambda w: float((c.double() * (held.cpu().double() @ w.t())).sum())  # noqa: E731
    h = 0.5                                             # the loss is linear in W
    assert float((dw.cpu().double() * V).sum()) == pytest.approx((loss(W + h * V) - loss(W - h * V)) / (2 * h), rel=1e-4, abs=1e-4 * float(dw.abs().max()) * 30)


def test_long_offsets():
    """Tokens whose rows of dy lie beyond 2^32 bytes, and a packed form whose last block does."""
    T, N, ld = 96, 32, 2 ** 26 + 8
    buffer = torch.zeros((T - 1) * ld + N, dtype=torch.bfloat16, device="cuda")
    dy = buffer.as_strided((T, N), (ld, 1))
    a, x = exact_case(T, N, 48, "bf16", seed=5)
    dy.copy_(a.cuda())
    dw = torch.zeros(N, 48, device="cuda")
    star.star_act_weight_grad(dy, pack(x.cuda()), dw)
    assert np.array_equal(dw.double().cpu().numpy(), a.double().t().numpy() @ x.double().numpy())


def test_in_a_graph_and_on_a_stream():
    T, N, K = 4100, 96, 200                              # long enough to be cut into parts
    x, _ = activations(T, K, "bf16", seed=6)
    dy = torch.randn(T, N, device="cuda").bfloat16()
    packed = torch.zeros(star.star_act_bytes(T, K), dtype=torch.uint8, device="cuda")
    dw, out = torch.zeros(N, K, device="cuda"), torch.zeros_like(x)

    def step():
        star.star_act_pack(x, packed)
        star.star_act_weight_grad(dy, packed, dw)
        star.star_act_unpack(packed, out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        dy.copy_(torch.randn(T, N, device="cuda"))
        x.copy_(torch.randn(T, K, device="cuda"))
        step()
        want, kept = dw.clone(), out.clone()
        dw.fill_(5.0), out.fill_(5.0), packed.fill_(1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dw, want) and torch.equal(out, kept)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    dw.fill_(5.0)
    torch.cuda.synchronize()
    star.star_act_weight_grad(dy, packed, dw, stream=side)
    side.synchronize()
    assert torch.equal(dw, want)


@pytest.mark.parametrize("N,K,dy_type", [(257, 3_000_000, "f32"), (1025, 2_450_000, "bf16")])
def test_weight_gradient_of_the_widest_layers(N, K, dy_type):
    """The last tile's rows lie so far beyond the end of dw that the distance does not fit 31 bits: what lies behind dw stays as it is."""
    T, behind = 32, 1 << 30
    g = torch.Generator(device="cuda").manual_seed(N)
    x = torch.randint(-8, 9, (T, K), generator=g, device="cuda").bfloat16()
    dy = torch.randint(-4, 5, (T, N), generator=g, device="cuda").to(TYPES[dy_type])
    packed = torch.zeros(star.star_act_bytes(T, K), dtype=torch.uint8, device="cuda")
    star.star_act_pack(x, packed)
    whole = torch.full((N * K + behind,), 7.0, device="cuda")
    dw = whole[:N * K].view(N, K)
    star.star_act_weight_grad(dy, packed, dw)
    for a in range(0, N, 64):
        assert torch.equal(dw[a:a + 64], dy[:, a:a + 64].float().t().contiguous() @ x.float()), a
    for a in range(N * K, N * K + behind, 1 << 28):
        assert bool((whole[a:a + (1 << 28)] == 7.0).all())


@pytest.mark.parametrize("T,N,ld", [(1, 1, 8), (1, 7, 8), (65, 17, 24), (64, 101, 104), (33, 127, 128), (32, 129, 136), (250, 1001, 1008), (250, 1002, 1008),
                                    (251, 1003, 1008), (64, 1005, 1008), (64, 1007, 1008), (40, 513, 520), (64, 2051, 2056)])
def test_weight_gradient_of_an_odd_number_of_columns(T, N, ld):
    """bf16 rows on 16-byte addresses that end inside of 16 bytes and inside of 4: the last token's last columns, with NaN behind them."""
    K = 80
    dy, x = exact_case(T, N, K, "bf16", seed=12)
    dy[T - 1] = 3.0
    dy[T - 1, N - 1] = -2.0
    x[T - 1] = 1.0
    buffer = torch.full((T * ld,), float("nan"), dtype=torch.bfloat16, device="cuda")
    dev = buffer.view(T, ld)[:, :N]
    dev.copy_(dy.cuda())
    dw = torch.full((N, K), 7.0, device="cuda")
    star.star_act_weight_grad(dev, pack(x.cuda()), dw)
    assert np.array_equal(dw.double().cpu().numpy(), dy.double().t().numpy() @ x.double().numpy())


def test_long_packed_form():
    """A packed form of more than 2^32 bytes, whose last block is all that reaches the gradient and what is brought back."""
    T, N, K = 2 ** 20 + 40, 24, 4096
    x = torch.empty(T, K, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    for a in range(0, T, 2 ** 17):
        x[a:a + 2 ** 17] = torch.randint(-8, 9, (min(2 ** 17, T - a), K), generator=g, device="cuda")
    packed = torch.full((star.star_act_bytes(T, K) + 32,), 0xAB, dtype=torch.uint8, device="cuda")
    assert packed.numel() > 2 ** 32
    star.star_act_pack(x, packed)
    assert bool((packed[-32:] == 0xAB).all())
    dy = torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    dy[-39:] = torch.randint(-4, 5, (39, N), generator=g, device="cuda").bfloat16()
    dw = torch.zeros(N, K, device="cuda")
    star.star_act_weight_grad(dy, packed, dw)
    assert torch.equal(dw, dy[-39:].float().t().contiguous() @ x[-39:].float())
    out = torch.zeros_like(x)
    star.star_act_unpack(packed, out)
    for a in range(0, T, 2 ** 17):
        assert torch.equal(out[a:a + 2 ** 17], x[a:a + 2 ** 17]), a


# The tiles that only large or thin outputs take: 64 for bf16 (one thin side, whole and in parts), 128 for fp32, 256 for both (whole and in parts);
# ld: rows of dy on 16-byte addresses, or not
@pytest.mark.parametrize("T,N,K,ld,dy_type", [
    (70, 40, 70001, 40, "bf16"), (70, 39, 70001, 39, "bf16"), (70, 39, 70001, 40, "bf16"), (65, 70001, 40, 70008, "bf16"), (5000, 40, 30001, 40, "bf16"),
    (5000, 33, 30001, 35, "bf16"), (70, 4090, 4001, 4096, "bf16"), (70, 4089, 4001, 4096, "bf16"), (129, 4090, 4001, 4090, "bf16"),
    (20000, 4090, 2001, 4096, "bf16"), (20001, 4090, 2001, 4091, "bf16"), (70, 2100, 4001, 2100, "f32"), (3000, 2100, 2000, 2101, "f32"),
    (60, 4090, 4001, 4090, "f32"), (70, 4090, 4001, 4091, "f32"), (20000, 4090, 2001, 4090, "f32")])
@pytest.mark.parametrize("dw_type", ["f32", "bf16"])
def test_weight_gradient_in_every_tile(T, N, K, ld, dy_type, dw_type):
    dy, x = exact_case(T, N, K, dy_type, seed=13)
    dy[T - 1] = 3.0
    buffer = torch.full((T, ld), float("nan"), dtype=TYPES[dy_type], device="cuda")
    dev, x = buffer[:, :N], x.cuda()
    dev.copy_(dy.cuda())
    packed = pack(x)
    want = dev.float().t().contiguous() @ x                            # (sums that fp32 holds exactly, in any order)
    dw = torch.full((N * K + 8,), 7.0, dtype=TYPES[dw_type], device="cuda")
    row = dw[3:3 + N * K].view(N, K)
    star.star_act_weight_grad(dev, packed, row)
    assert torch.equal(row, want.to(TYPES[dw_type]))
    before = (-(want / 2)).to(TYPES[dw_type])
    row.copy_(before)
    star.star_act_weight_grad(dev, packed, row, accumulate=True)
    assert torch.equal(row, (before.float() + want).to(TYPES[dw_type]))
    assert bool((dw[:3] == 7.0).all()) and bool((dw[3 + N * K:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_kept_values_of_a_large_matrix(dtype):
    """More blocks of columns than are packed one to a workgroup; rows apart by an odd distance."""
    T, K = 1001, 6007
    x, x32 = activations(T, K, dtype, seed=14, pad=4, shift=1)
    out = torch.zeros(T, K, device="cuda")
    star.star_act_unpack(pack(x), out)
    assert np.array_equal(out.double().cpu().numpy(), wo.kept(x32)[0])
