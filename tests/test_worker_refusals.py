"""What the worker-side entry points refuse, with the status that says why, before anything touches a device; and the
sizes of their host-only functions."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2512_09685_amd as star
from paper_2512_09685_amd import worker

NULL, SHAPE, GROUP, HPARAM, DTYPE = 1, 2, 3, 4, 5
F32, BF16 = 0, 1
P = 1 << 20          # an address that no check looks behind


@pytest.fixture(scope="module")
def lib():
    return worker._library()


def _policy(scale=1.0, low=0.2, high=0.2, kl=0.0, temperature=1.0):
    return ctypes.byref(worker._PolicyParams(scale, low, high, kl, temperature))


def _preference(scale=1.0, beta=0.1, smooth=0.0, temperature=1.0):
    return ctypes.byref(worker._PreferenceParams(scale, beta, smooth, temperature))


LOGITS = dict(x=P, dtype=BF16, tokens=3, vocab=10, ld=10, targets=P)
BAD_LOGITS = [
    (dict(x=None), NULL), (dict(targets=None), NULL), (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(tokens=-1), SHAPE), (dict(tokens=(1 << 22) + 1), SHAPE), (dict(vocab=0), SHAPE), (dict(vocab=-4), SHAPE),
    (dict(vocab=(1 << 30) + 1, ld=1 << 31), SHAPE), (dict(ld=9), SHAPE), (dict(ld=1 << 62), SHAPE), (dict(x=P + 1), SHAPE),
    (dict(dtype=F32, x=P + 2), SHAPE), (dict(targets=P + 4), SHAPE),
]
BAD_TEMPERATURE = [0.0, -1.0, float("nan"), float("inf"), 1e-45, 5e-5, 2e4]


def _head(change):
    a = {**LOGITS, **change}
    return [a["x"], a["dtype"], a["tokens"], a["vocab"], a["ld"], a["targets"]]


@pytest.mark.parametrize("change,status", BAD_LOGITS)
def test_logits_refused(lib, change, status):
    h = _head(change)
    assert lib.star_token_logprobs(*h, 1.0, P, None, P, 1 << 30, 0) == status
    assert star.last_error()
    assert lib.star_token_logprobs_grad(*h, 1.0, P, P, 2 * P, 1 << 32, 0) == status
    assert lib.star_policy_loss(*h, P, None, P, None, _policy(), 2 * P, 1 << 32, None, P, P, 1 << 30, 0) == status
    n = max(0, h[2])
    offsets = np.array([0, n, n], np.int64)
    assert lib.star_preference_loss(*h, P, None, 1, offsets.ctypes.data, _preference(), 2 * P, 1 << 32, None, None, P, P, 1 << 30,
                                    0) == status


@pytest.mark.parametrize("t", BAD_TEMPERATURE)
def test_temperature_refused(lib, t):
    h = _head({})
    assert lib.star_token_logprobs(*h, t, P, None, P, 1 << 30, 0) == HPARAM
    assert lib.star_token_logprobs_grad(*h, t, P, P, P, 10, 0) == HPARAM
    assert lib.star_policy_loss(*h, P, None, P, None, _policy(temperature=t), P, 10, None, P, P, 1 << 30, 0) == HPARAM
    o = np.array([0, 1, 3], np.int64)
    assert lib.star_preference_loss(*h, P, None, 1, o.ctypes.data, _preference(temperature=t), P, 10, None, None, P, P, 1 << 30,
                                    0) == HPARAM


def test_outputs_and_gradients_refused(lib):
    h = _head({})
    assert lib.star_token_logprobs(*h, 1.0, None, None, P, 1 << 30, 0) == NULL
    for lse, dlogp, out, ld, status in ((None, P, P, 10, NULL), (P, None, P, 10, NULL), (P, P, None, 10, NULL),
                                        (P, P, P, 9, SHAPE), (P, P, P + 1, 10, SHAPE), (P, P, P, 11, SHAPE)):   # last: in place
        assert lib.star_token_logprobs_grad(*h, 1.0, lse, dlogp, out, ld, 0) == status


@pytest.mark.parametrize("params,status", [
    (dict(scale=float("inf")), HPARAM), (dict(scale=float("nan")), HPARAM), (dict(low=-0.1), HPARAM), (dict(low=float("nan")), HPARAM),
    (dict(high=-1.0), HPARAM), (dict(kl=-0.5), HPARAM), (dict(kl=float("inf")), HPARAM), (dict(kl=float("nan")), HPARAM)])
def test_policy_params_refused(lib, params, status):
    assert lib.star_policy_loss(*_head({}), P, P, P, None, _policy(**params), P, 10, None, P, P, 1 << 30, 0) == status


def test_policy_pointers_refused(lib):
    def call(params=_policy(), old=P, ref=None, adv=P, stats=P, ws=P, size=1 << 20):
        return lib.star_policy_loss(*_head({}), old, ref, adv, None, params, 2 * P, 10, None, stats, ws, size, 0)
    assert call(params=None) == NULL
    assert call(old=None) == NULL
    assert call(adv=None) == NULL
    assert call(stats=None) == NULL
    assert call(params=_policy(kl=0.1)) == NULL            # a KL term needs the reference
    need = lib.star_policy_loss_workspace(BF16, 3, 10)
    assert need > 0
    assert call(ws=None, size=0) == NULL
    assert call(size=need - 1) == SHAPE
    assert call(ws=P + 8) == SHAPE


@pytest.mark.parametrize("offsets,tokens,status", [
    ([1, 2, 3], 3, GROUP), ([0, 2, 2], 3, GROUP), ([0, 2, 4], 3, GROUP), ([0, 3, 2, 2, 3], 3, GROUP), ([0, -1, 3], 3, GROUP)])
def test_offsets_refused(lib, offsets, tokens, status):
    o = np.array(offsets, np.int64)
    assert lib.star_preference_loss(*_head(dict(tokens=tokens)), P, None, len(offsets) // 2, o.ctypes.data, _preference(), 2 * P, 10,
                                    None, None, P, P, 1 << 30, 0) == status


def test_preference_refused(lib):
    o = np.array([0, 1, 3], np.int64)

    def call(params=_preference(), pairs=1, offsets=o.ctypes.data, ref=P, loss=P, ws=P, size=1 << 20):
        return lib.star_preference_loss(*_head({}), ref, None, pairs, offsets, params, 2 * P, 10, None, None, loss, ws, size, 0)
    assert call(params=None) == NULL
    assert call(offsets=None) == NULL
    assert call(ref=None) == NULL
    assert call(loss=None) == NULL
    assert call(pairs=-1) == SHAPE
    for bad in (dict(scale=float("nan")), dict(beta=float("inf")), dict(smooth=-0.1), dict(smooth=1.5), dict(smooth=float("nan"))):
        assert call(params=_preference(**bad)) == HPARAM
    need = lib.star_preference_loss_workspace(BF16, 3, 10, 1)
    assert call(ws=None, size=0) == NULL
    assert call(size=need - 1) == SHAPE
    assert call(ws=P + 4) == SHAPE


@pytest.mark.parametrize("args,status", [
    (dict(x=None), NULL), (dict(packed=None), NULL), (dict(dtype=7), DTYPE), (dict(tokens=-1), SHAPE), (dict(width=-1), SHAPE),
    (dict(ld=7), SHAPE), (dict(ld=1 << 62), SHAPE), (dict(tokens=1 << 41, width=1 << 20, ld=1 << 20), SHAPE), (dict(x=P + 1), SHAPE), (dict(packed=P + 8), SHAPE)])
def test_pack_and_unpack_refused(lib, args, status):
    a = {**dict(x=P, dtype=BF16, tokens=5, width=8, ld=8, packed=P), **args}
    assert lib.star_act_pack(a["x"], a["dtype"], a["tokens"], a["width"], a["ld"], a["packed"], 0) == status
    assert lib.star_act_unpack(a["packed"], a["tokens"], a["width"], a["x"], a["dtype"], a["ld"], 0) == status


@pytest.mark.parametrize("args,status", [
    (dict(dy=None), NULL), (dict(packed=None), NULL), (dict(dw=None), NULL), (dict(dy_dtype=2), DTYPE), (dict(dw_dtype=-3), DTYPE),
    (dict(tokens=-1), SHAPE), (dict(out=-1), SHAPE), (dict(width=-1), SHAPE), (dict(ld=5), SHAPE), (dict(dy=P + 1), SHAPE),
    (dict(packed=P + 4), SHAPE), (dict(dw=P + 2), SHAPE), (dict(out=1 << 20, ld=1 << 20, width=1 << 20), SHAPE),
    (dict(out=1 << 40, ld=1 << 40, width=1 << 40), SHAPE)])
def test_weight_grad_refused(lib, args, status):
    a = {**dict(dy=P, dy_dtype=BF16, tokens=5, out=6, ld=6, packed=P, width=8, dw=P, dw_dtype=F32), **args}
    assert lib.star_act_weight_grad(a["dy"], a["dy_dtype"], a["tokens"], a["out"], a["ld"], a["packed"], a["width"], a["dw"],
                                    a["dw_dtype"], 0, P, 1 << 40, 0) == status


def test_weight_grad_workspace_refused(lib):
    need = lib.star_act_weight_grad_workspace(BF16, 65536, 64, 64)     # long sums on a small matrix: cut into parts
    assert need >= 2 * 64 * 64 * 4
    args = [P, BF16, 65536, 64, 64, P, 64, P, F32, 0]
    assert lib.star_act_weight_grad(*args, None, 0, 0) == NULL
    assert lib.star_act_weight_grad(*args, P, need - 1, 0) == SHAPE
    assert lib.star_act_weight_grad(*args, P + 8, need, 0) == SHAPE


def test_empty_calls_need_nothing(lib):
    assert lib.star_token_logprobs(None, BF16, 0, 10, 10, None, 1.0, None, None, None, 0, 0) == 0
    assert lib.star_token_logprobs_grad(None, F32, 0, 10, 10, None, 1.0, None, None, None, 10, 0) == 0
    assert lib.star_act_pack(None, F32, 0, 8, 8, None, 0) == 0
    assert lib.star_act_pack(None, F32, 8, 0, 0, None, 0) == 0
    assert lib.star_act_unpack(None, 8, 0, None, F32, 0, 0) == 0
    assert lib.star_act_weight_grad(None, F32, 8, 0, 0, None, 8, None, F32, 0, None, 0, 0) == 0
    assert lib.star_act_weight_grad(None, F32, 8, 8, 8, None, 0, None, F32, 0, None, 0, 0) == 0


@pytest.mark.parametrize("tokens,width,bytes_", [(0, 8, 0), (1, 1, 16 * 33), (32, 16, 16 * 33), (33, 17, 2 * 32 * 33), (64, 4096, 2 * 4096 * 33)])
def test_act_bytes(tokens, width, bytes_):
    assert star.star_act_bytes(tokens, width) == bytes_


def test_act_bytes_of_no_size():
    assert star.star_act_bytes(-1, 8) == 0 and star.star_act_bytes(8, -1) == 0 and star.star_act_bytes(1 << 41, 1 << 41) == 0


def test_binding_refuses_tensors_of_other_kinds():
    T, V = 4, 10
    x, y = torch.zeros(T, V), torch.zeros(T, dtype=torch.int64)
    f = torch.zeros(T)
    with pytest.raises(TypeError):
        star.star_token_logprobs(x.half(), y, f, stream=0)
    with pytest.raises(ValueError):
        star.star_token_logprobs(x.t(), y, f, stream=0)                       # rows not contiguous
    with pytest.raises(ValueError):
        star.star_token_logprobs(x[:1].expand(T, V), y, f, stream=0)          # rows on top of each other
    with pytest.raises(ValueError):
        star.star_token_logprobs(x, y.int(), f, stream=0)
    with pytest.raises(ValueError):
        star.star_token_logprobs(x, y, f[:3], stream=0)
    with pytest.raises(ValueError):
        star.star_token_logprobs(x, y, f.double(), stream=0)
    with pytest.raises(TypeError):
        star.star_token_logprobs_grad(x, y, f, f, x.bfloat16(), stream=0)
    with pytest.raises(ValueError):
        star.star_token_logprobs_grad(x, y, f, f, torch.zeros(T, V + 1), stream=0)
    with pytest.raises(ValueError):
        star.star_preference_loss(x, y, f, [0, 4], f[:1], stream=0)
    with pytest.raises(TypeError):
        star.star_act_pack(x.double(), torch.zeros(9999, dtype=torch.uint8), stream=0)
    with pytest.raises(ValueError):
        star.star_act_pack(x, torch.zeros(star.star_act_bytes(T, V) - 1, dtype=torch.uint8), stream=0)
    packed = torch.zeros(star.star_act_bytes(T, V), dtype=torch.uint8)
    with pytest.raises(ValueError):
        star.star_act_unpack(packed, torch.zeros(T + 32, V), stream=0)
    with pytest.raises(ValueError):
        star.star_act_weight_grad(torch.zeros(T, 6), packed, torch.zeros(5, V), stream=0)
    with pytest.raises(ValueError):
        star.star_act_weight_grad(torch.zeros(T, 6), packed, torch.zeros(V, 6).t(), stream=0)
    with pytest.raises(star.StarError) as e:
        star.star_policy_loss(x, y, f, f, torch.zeros(4), kl_coef=0.1, stream=0)
    assert e.value.status == NULL


def test_binding_refuses_host_memory():
    """Tensors that are all well formed but lie on the host: no kernel gets their addresses."""
    T, V = 4, 10
    x, y, f = torch.zeros(T, V), torch.zeros(T, dtype=torch.int64), torch.zeros(T)
    packed = torch.zeros(star.star_act_bytes(T, V), dtype=torch.uint8)
    for call in (lambda: star.star_token_logprobs(x, y, f, stream=0),
                 lambda: star.star_token_logprobs_grad(x, y, f, f, x.clone(), stream=0),
                 lambda: star.star_policy_loss(x, y, f, f, torch.zeros(4), stream=0),
                 lambda: star.star_preference_loss(x, y, f, [0, 2, 4], f[:1], stream=0),
                 lambda: star.star_act_pack(x, packed, stream=0),
                 lambda: star.star_act_unpack(packed, x, stream=0),
                 lambda: star.star_act_weight_grad(torch.zeros(T, 6), packed, torch.zeros(6, V), stream=0)):
        with pytest.raises(ValueError, match="GPU memory"):
            call()


def test_results_stay_inside_the_weight_gradient(tmp_path):
    """The range that a block of results may write, for tiles that reach beyond the last row of the widest matrices."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "grad_range_check"
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-fsanitize=undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__=1",
                        "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2512_09685_amd", "csrc"),
                        "-I", os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include"),
                        os.path.join(root, "tests", "grad_range_check.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "blocks in range" in r.stdout, (r.stdout, r.stderr)


@pytest.mark.parametrize("off", [0, 8, -8])
def test_log_probabilities_over_an_input_refused(lib, off):
    """logp_out over what the call reads again behind it: 3 tokens, 12 bytes each."""
    far, out, o = 4 * P, P + 64, np.array([0, 1, 3], np.int64)
    for which in range(4):
        v = [far, 2 * far, 3 * far, 4 * far]                     # old_logp, ref_logp, advantages, weights
        v[which] = out + off
        assert lib.star_policy_loss(*_head({}), *v, _policy(), None, 0, out, P, None, 0, 0) == SHAPE and "overlaps" in star.last_error()
        v[which] = out + 12                                      # side by side: the next check's answer
        assert lib.star_policy_loss(*_head({}), *v, _policy(), None, 0, out, P, None, 0, 0) == NULL
    for ref, w in ((out + off, far), (far, out + off)):
        args = [ref, w, 1, o.ctypes.data, _preference(), None, 0, out, None, P, None, 0, 0]
        assert lib.star_preference_loss(*_head({}), *args) == SHAPE and "overlaps" in star.last_error()
