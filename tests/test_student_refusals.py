"""What the entry points of a worker that learns from a teacher refuse, with the status that says why, before anything touches a device."""
import ctypes

import pytest
import torch

import paper_2512_09685_amd as star
from paper_2512_09685_amd import worker
from test_worker_refusals import BAD_LOGITS, BAD_TEMPERATURE, BF16, DTYPE, F32, HPARAM, NULL, P, SHAPE, _head


@pytest.fixture(scope="module")
def lib():
    return worker._library()


def _params(scale=1.0, ce=0.0, temperature=1.0, renormalise=0):
    return ctypes.byref(worker._DistillParams(scale, ce, temperature, renormalise))


def _top(lib, head, t=1.0, k=4, logp=P, entropy=2 * P, lse=3 * P, ids=4 * P, top=5 * P):
    return lib.star_top_logprobs(*head, t, k, logp, entropy, lse, ids, top, None, 0, 0)


def _top_grad(lib, head, t=1.0, dlogp=P, dentropy=P, k=4, ids=P, dtop=P, out=2 * P, ld=1 << 32):
    return lib.star_top_logprobs_grad(*head, t, dlogp, dentropy, k, ids, dtop, out, ld, 0)


def _distill(lib, head, k=4, ids=P, teacher=P, weights=None, params=None, out=2 * P, ld=1 << 32, kl=None, stats=P, ws=P, size=1 << 30):
    return lib.star_distill_loss(*head, k, ids, teacher, weights, params or _params(), out, ld, kl, stats, ws, size, 0)


@pytest.mark.parametrize("change,status", [c for c in BAD_LOGITS if c[0] != dict(targets=None)])
def test_logits_refused(lib, change, status):
    h = _head(change)
    assert _top(lib, h) == status and star.last_error()
    assert _top_grad(lib, h) == status
    assert _distill(lib, h) == status


@pytest.mark.parametrize("t", BAD_TEMPERATURE)
def test_temperature_refused(lib, t):
    assert _top(lib, _head({}), t=t) == HPARAM
    assert _top_grad(lib, _head({}), t=t) == HPARAM
    assert _distill(lib, _head({}), params=_params(temperature=t)) == HPARAM


@pytest.mark.parametrize("k", [-1, 129, 1 << 20])
def test_number_of_words_refused(lib, k):
    assert _top(lib, _head({}), k=k) == SHAPE and "128" in star.last_error()
    assert _top_grad(lib, _head({}), k=k) == SHAPE
    assert _distill(lib, _head({}), k=k) == SHAPE


def test_a_teacher_of_no_words_refused(lib):
    assert _distill(lib, _head({}), k=0) == SHAPE


def test_words_refused(lib):
    for ids, numbers, status in ((None, P, NULL), (P, None, NULL), (P + 4, P, SHAPE), (P, P + 2, SHAPE)):
        assert _top(lib, _head({}), ids=ids, top=numbers) == status
        assert _top_grad(lib, _head({}), ids=ids, dtop=numbers) == status
        assert _distill(lib, _head({}), ids=ids, teacher=numbers) == status


def test_what_needs_targets_refused_without(lib):
    h = _head(dict(targets=None))
    assert _top(lib, h) == NULL and "targets" in star.last_error()
    assert _top_grad(lib, h) == NULL and "targets" in star.last_error()
    assert _distill(lib, h, params=_params(ce=0.1)) == NULL and "targets" in star.last_error()


def test_outputs_refused(lib):
    assert _top(lib, _head({}), logp=P, entropy=P + 8) == SHAPE and "overlap" in star.last_error()      # 3 tokens, 12 bytes
    assert _top(lib, _head({}), logp=P, lse=P) == SHAPE
    assert _top(lib, _head({}), entropy=P, lse=P - 8, logp=None) == SHAPE
    assert _top_grad(lib, _head({}), out=None) == NULL
    assert _top_grad(lib, _head({}), out=P, ld=11) == SHAPE                                              # in place
    assert _top_grad(lib, _head({}), ld=9) == SHAPE
    assert _top_grad(lib, _head({}), out=2 * P + 1) == SHAPE
    assert _distill(lib, _head({}), stats=None) == NULL
    assert _distill(lib, _head({}), kl=P + 64, weights=P + 72) == SHAPE and "overlaps" in star.last_error()


def test_distill_params_and_workspace_refused(lib):
    inf, nan = float("inf"), float("nan")
    for bad in (dict(scale=inf), dict(scale=nan), dict(ce=-0.1), dict(ce=inf), dict(ce=nan)):
        assert _distill(lib, _head({}), params=_params(**bad)) == HPARAM
    assert lib.star_distill_loss(*_head({}), 4, P, P, None, None, None, 0, None, P, P, 1 << 30, 0) == NULL
    need = lib.star_distill_loss_workspace(BF16, 3, 10, 4)
    assert need > 0
    assert _distill(lib, _head({}), ws=None, size=0) == NULL
    assert _distill(lib, _head({}), size=need - 1) == SHAPE
    assert _distill(lib, _head({}), ws=P + 8) == SHAPE


NORM = dict(x=P, dtype=BF16, tokens=3, width=8, ld=8, residual=None, ld_residual=8, gain=P, gain_dtype=F32, eps=1e-6, sum=None, ld_sum=8, y=2 * P, ld_y=8,
            rstd=None, packed=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), NULL), (dict(y=None), NULL), (dict(dtype=2), DTYPE), (dict(gain_dtype=-1), DTYPE), (dict(tokens=-1), SHAPE),
    (dict(tokens=(1 << 30) + 1), SHAPE), (dict(width=0), SHAPE), (dict(width=-8), SHAPE), (dict(width=32769, ld=1 << 16, ld_y=1 << 16), SHAPE),
    (dict(ld=7), SHAPE), (dict(ld_y=7), SHAPE), (dict(ld=1 << 62), SHAPE), (dict(x=P + 1), SHAPE), (dict(y=P + 1), SHAPE), (dict(gain=P + 2), SHAPE),
    (dict(eps=0.0), HPARAM), (dict(eps=-1e-6), HPARAM), (dict(eps=float("inf")), HPARAM), (dict(eps=float("nan")), HPARAM),
    (dict(residual=3 * P), NULL), (dict(sum=3 * P), NULL), (dict(residual=3 * P, sum=4 * P, ld_residual=7), SHAPE),
    (dict(residual=3 * P, sum=4 * P, ld_sum=7), SHAPE), (dict(residual=3 * P, sum=2 * P), SHAPE), (dict(residual=3 * P + 1, sum=4 * P), SHAPE),
    (dict(y=P, ld_y=9), SHAPE), (dict(residual=3 * P, sum=P, ld_sum=9), SHAPE), (dict(residual=3 * P, sum=3 * P, ld_sum=9), SHAPE),
    (dict(residual=2 * P, sum=4 * P, ld_residual=9), SHAPE), (dict(packed=P + 8), SHAPE)])
def test_norm_refused(lib, change, status):
    a = {**NORM, **change}
    assert lib.star_rms_norm(a["x"], a["dtype"], a["tokens"], a["width"], a["ld"], a["residual"], a["ld_residual"], a["gain"], a["gain_dtype"], a["eps"],
                             a["sum"], a["ld_sum"], a["y"], a["ld_y"], a["rstd"], a["packed"], 0) == status
    assert star.last_error()


GRAD = dict(dy=P, dtype=BF16, tokens=3, width=8, ld_dy=8, h=2 * P, ld_h=8, gain=None, gain_dtype=F32, rstd=P, dres=None, ld_dres=8, dx=3 * P, ld_dx=8,
            dgain=P, dgain_dtype=F32, ws=P, size=1 << 30)


@pytest.mark.parametrize("change,status", [
    (dict(dy=None), NULL), (dict(h=None), NULL), (dict(dx=None), NULL), (dict(rstd=None), NULL), (dict(dtype=7), DTYPE), (dict(dgain_dtype=7), DTYPE),
    (dict(gain=P, gain_dtype=7), DTYPE), (dict(tokens=-2), SHAPE), (dict(width=0), SHAPE), (dict(width=32769), SHAPE), (dict(ld_dy=7), SHAPE),
    (dict(ld_h=7), SHAPE), (dict(ld_dx=7), SHAPE), (dict(dres=P, ld_dres=7), SHAPE), (dict(dy=P + 1), SHAPE), (dict(h=P + 1), SHAPE),
    (dict(dgain=P + 2), SHAPE), (dict(dx=P, ld_dx=9), SHAPE), (dict(dx=2 * P, ld_dx=9), SHAPE), (dict(dx=5 * P, dres=5 * P, ld_dres=9), SHAPE),
    (dict(ws=None, size=0), NULL), (dict(size=31), SHAPE), (dict(ws=P + 4), SHAPE)])
def test_norm_gradient_refused(lib, change, status):
    a = {**GRAD, **change}
    assert lib.star_rms_norm_grad(a["dy"], a["dtype"], a["tokens"], a["width"], a["ld_dy"], a["h"], a["ld_h"], a["gain"], a["gain_dtype"], a["rstd"],
                                  a["dres"], a["ld_dres"], a["dx"], a["ld_dx"], a["dgain"], a["dgain_dtype"], 0, a["ws"], a["size"], 0) == status
    assert star.last_error()


def test_empty_calls_need_nothing(lib):
    h = [None, BF16, 0, 10, 10, None]
    assert lib.star_top_logprobs(*h, 1.0, 4, None, None, None, None, None, None, 0, 0) == 0
    assert lib.star_top_logprobs_grad(*h, 1.0, None, None, 4, None, None, None, 10, 0) == 0
    assert lib.star_rms_norm(None, F32, 0, 8, 8, None, 0, None, F32, 1e-6, None, 0, None, 8, None, None, 0) == 0
    assert lib.star_rms_norm_grad(None, F32, 0, 8, 8, None, 8, None, F32, None, None, 0, None, 8, None, F32, 0, None, 0, 0) == 0


def test_workspaces_of_no_size(lib):
    assert lib.star_distill_loss_workspace(BF16, -1, 10, 4) == 0 and lib.star_distill_loss_workspace(7, 3, 10, 4) == 0
    assert lib.star_rms_norm_grad_workspace(BF16, 0, 8) == 0 and lib.star_rms_norm_grad_workspace(BF16, 8, 0) == 0
    assert lib.star_rms_norm_grad_workspace(9, 8, 8) == 0 and lib.star_rms_norm_grad_workspace(F32, 1 << 31, 8) == 0


def test_binding_refuses_tensors_of_other_kinds():
    T, V, K = 4, 10, 3
    x, y, f = torch.zeros(T, V), torch.zeros(T, dtype=torch.int64), torch.zeros(T)
    ids, t = torch.zeros(T, K, dtype=torch.int64), torch.zeros(T, K)
    with pytest.raises(ValueError):
        star.star_top_logprobs(x, y, f, top_ids=ids, stream=0)                    # no room for their log-probabilities
    with pytest.raises(ValueError):
        star.star_top_logprobs(x, y, f, top_ids=ids.int(), top_logp=t, stream=0)
    with pytest.raises(ValueError):
        star.star_top_logprobs(x, y, f, top_ids=ids, top_logp=t[:, :2], stream=0)
    with pytest.raises(ValueError):
        star.star_top_logprobs(x, y, f, top_ids=ids[:2], top_logp=t[:2], stream=0)
    with pytest.raises(star.StarError) as e:
        star.star_top_logprobs(x, None, f, stream=0)
    assert e.value.status == NULL
    with pytest.raises(ValueError):
        star.star_top_logprobs_grad(x, y, x.clone(), dlogp=f.double(), stream=0)
    with pytest.raises(TypeError):
        star.star_top_logprobs_grad(x, y, x.bfloat16(), stream=0)
    with pytest.raises(star.StarError):
        star.star_top_logprobs_grad(x, None, x.clone(), dlogp=f, stream=0)
    with pytest.raises(ValueError):
        star.star_distill_loss(x, ids, None, torch.zeros(4), stream=0)
    with pytest.raises(ValueError):
        star.star_distill_loss(x, ids, t.double(), torch.zeros(4), stream=0)
    with pytest.raises(ValueError):
        star.star_distill_loss(x, ids, t, torch.zeros(3), stream=0)
    with pytest.raises(star.StarError) as e:
        star.star_distill_loss(x, ids, t, torch.zeros(4), ce_coef=0.1, stream=0)
    assert e.value.status == NULL
    g = torch.ones(V)
    with pytest.raises(TypeError):
        star.star_rms_norm(x, g.half(), x.clone(), stream=0)
    with pytest.raises(TypeError):
        star.star_rms_norm(x, g, x.bfloat16(), stream=0)
    with pytest.raises(ValueError):
        star.star_rms_norm(x, g[:5], x.clone(), stream=0)
    with pytest.raises(ValueError):
        star.star_rms_norm(x, g, torch.zeros(T, V + 1), stream=0)
    with pytest.raises(star.StarError):
        star.star_rms_norm(x, g, x.clone(), residual=x, stream=0)
    with pytest.raises(ValueError):
        star.star_rms_norm(x, g, x.clone(), packed=torch.zeros(7, dtype=torch.uint8), stream=0)
    with pytest.raises(ValueError):
        star.star_rms_norm_grad(x, x[:2], g, f, x.clone(), stream=0)
    with pytest.raises(ValueError):
        star.star_rms_norm_grad(x, x, g, f[:2], x.clone(), stream=0)
    with pytest.raises(ValueError):
        star.star_rms_norm_grad(x, x, g, f, x.clone(), dgain=torch.zeros(2 * V)[::2], stream=0)


def test_binding_refuses_host_memory():
    T, V, K = 4, 10, 3
    x, y, f = torch.zeros(T, V), torch.zeros(T, dtype=torch.int64), torch.zeros(T)
    ids, t = torch.zeros(T, K, dtype=torch.int64), torch.zeros(T, K)
    for call in (lambda: star.star_top_logprobs(x, y, f, top_ids=ids, top_logp=t, stream=0),
                 lambda: star.star_top_logprobs_grad(x, y, x.clone(), dlogp=f, stream=0),
                 lambda: star.star_distill_loss(x, ids, t, torch.zeros(4), stream=0),
                 lambda: star.star_rms_norm(x, torch.ones(V), x.clone(), stream=0),
                 lambda: star.star_rms_norm_grad(x, x, torch.ones(V), f, x.clone(), stream=0)):
        with pytest.raises(ValueError, match="GPU memory"):
            call()


def _apart(names):
    return {name: 0x1000 * P + i * 0x10000 for i, name in enumerate(names)}


@pytest.mark.parametrize("k", [1, 4])
def test_outputs_over_one_another_or_the_targets_refused(lib, k):
    """Every pair, at both ends of the stretch in which they meet: 3 tokens, k words each."""
    size = dict(targets=24, logp=12, entropy=12, lse=12, ids=24 * k, top=12 * k)
    for a in size:
        for b in size:
            if a == b:
                continue
            at = _apart(size)
            grid = 8 if b in ("targets", "ids") else 4
            for off in (0, -grid, (size[a] - 1) // grid * grid):
                at[b] = at[a] + off
                args = {n: at[n] for n in size if n != "targets"}
                assert _top(lib, _head(dict(targets=at["targets"])), k=k, **args) == SHAPE, (a, b, off)
                assert "overlap" in star.last_error()


@pytest.mark.parametrize("k", [1, 4])
def test_divergences_over_an_input_or_the_sums_refused(lib, k):
    size = dict(targets=24, ids=24 * k, teacher=12 * k, weights=12, stats=16)
    for name in size:
        at = _apart(size)
        args = {n: at[n] for n in size if n != "targets"}
        for off in (0, -8, size[name] - 4):
            assert _distill(lib, _head(dict(targets=at["targets"])), k=k, kl=at[name] + off, **args) == SHAPE and "overlap" in star.last_error(), (name, off)
        # side by side: the next check's answer
        for off in (-12, size[name]):
            assert _distill(lib, _head(dict(targets=at["targets"])), k=k, kl=at[name] + off, ws=None, size=0, **args) == NULL
