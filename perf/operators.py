"""Measured cases of the worker-side operators: log-probabilities of taken tokens, the clipped policy loss and the
paired preference loss with their gradients, and activations saved in 8 bits with the weight gradient formed from them.

``own`` false: the plain form, elementary torch operations in 32 bits.  ``own`` true: the calls of the package.
"""
import math

import torch

own = False

_BF16, _F32 = "bf16", "f32"
_DTYPES = {_BF16: torch.bfloat16, _F32: torch.float32}
_BLOCK = 32          # tokens that share one scale in a saved activation
_E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------------------ cases
def _logits(op, name, tokens, vocab, dtype, *, pad=0, masked=0.0, temperature=1.0, **more):
    return dict(op=op, name=name, tokens=tokens, vocab=vocab, dtype=dtype, pad=pad, masked=masked,
                temperature=temperature, **more)


def _linear(name, tokens, out, inp, *, x="bf16", dy="bf16", dw="f32"):
    return dict(op="linear", name=name, tokens=tokens, out=out, inp=inp, x=x, dy=dy, dw=dw)


def listed():
    return [
        # one token just sampled: its log-probability is kept as old_logp (latency)
        _logits("logprobs", "logprobs one token", 1, 32000, _BF16),
        # the frozen reference model's log-probabilities over a batch
        _logits("logprobs", "logprobs reference batch", 4096, 131072, _BF16, masked=0.1),
        # a caller's own loss on the log-probabilities, fp32 logits of an odd vocabulary in padded rows: both directions
        _logits("logprobs_grad", "logprobs own loss fp32", 1023, 50021, _F32, pad=11, temperature=0.7),
        # the last few tokens of one rollout, a micro-batch that is all latency
        _logits("policy", "policy few tokens", 48, 32000, _BF16, kl=0.05, high=0.2),
        # a micro-batch of rollouts: prompts masked out, asymmetric clip range
        _logits("policy", "policy batch", 8192, 65536, _BF16, masked=0.25, kl=0.02, high=0.28),
        # fp32 logits of an odd vocabulary, no reference model
        _logits("policy", "policy odd fp32", 777, 50021, _F32, masked=0.1, kl=0.0, high=0.2, temperature=0.7),
        # two short pairs
        _logits("preference", "preference two pairs", 150, 32003, _BF16, pairs=2, smooth=0.0),
        # a batch of pairs of unequal lengths, prompts masked out
        _logits("preference", "preference batch", 12288, 32768, _BF16, masked=0.3, pairs=16, smooth=0.1),
        # a norm's input kept for the backward pass in 8 bits, brought back whole; ragged last block
        dict(op="save", name="save and restore", tokens=16381, inp=4096, x="bf16"),
        # the projections of a small layer over a short micro-batch
        _linear("weight gradient small", 250, 1024, 1000),
        # fp32 training: the row of the server is fp32, so are activations and gradients
        _linear("weight gradient fp32", 4096, 2048, 4096, x="f32", dy="f32"),
        # a wide layer over a long micro-batch, gradient row in bf16
        _linear("weight gradient wide", 16384, 8192, 8192, dw="bf16"),
    ]


def _between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs_grad", "policy", "policy", "preference", "preference", "save", "linear", "linear",
                     "linear"])
    if op == "linear":
        tokens, out, inp = _between(rng, 1, 32768), _between(rng, 16, 16384), _between(rng, 16, 16384)
        if rng.random() < 0.5:
            out, inp = -(-out // 64) * 64, -(-inp // 64) * 64
        tokens = max(1, min(tokens, int(16384 * 8192 * 8192 / (out * inp))))
        dy = rng.choice([_BF16, _BF16, _F32])
        case = _linear("", tokens, out, inp, x=rng.choice([_BF16, _F32]), dy=dy, dw=rng.choice([_F32, _BF16]))
    elif op == "save":
        tokens, inp = _between(rng, 1, 65536), _between(rng, 64, 16384)
        tokens = max(1, min(tokens, 16381 * 4096 // inp))
        case = dict(op=op, tokens=tokens, inp=inp, x=rng.choice([_BF16, _F32]))
    else:
        dtype = rng.choice([_BF16, _F32])
        tokens, vocab = _between(rng, 4 if op == "preference" else 1, 16384), _between(rng, 1000, 131072)
        if rng.random() < 0.5:
            vocab = -(-vocab // 64) * 64
        most = 2 ** 28 if op in ("logprobs", "preference") else 2 ** 27
        tokens = min(tokens, most // vocab)
        case = _logits(op, "", tokens, vocab, dtype, pad=rng.choice([0, 0, 3, 8]), masked=rng.choice([0.0, 0.25, 0.5]),
                       temperature=rng.choice([1.0, 0.7]))
        if op == "policy":
            case.update(kl=rng.choice([0.0, 0.05]), high=rng.choice([0.2, 0.28]))
        if op == "preference":
            case.update(pairs=rng.randint(1, max(1, min(32, tokens // 4))), smooth=rng.choice([0.0, 0.1]))
    case.pop("name", None)
    return case


# ----------------------------------------------------------------------------------------------------------- inputs
_LOW, _BETA = 0.2, 0.1


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _masked_count(case):
    return min(int(case["tokens"] * case["masked"]), case["tokens"] - 1)


def _pair_offsets(case):
    """Lengths of the 2 B sequences, chosen and rejected in turn: unequal, of at least one token."""
    n, T = 2 * case["pairs"], case["tokens"]
    share = [1.0 + 0.6 * math.sin(1.7 * i + 0.3) for i in range(n)]
    total, offsets, run = sum(share), [0], 0.0
    for s in share:
        run += s
        offsets.append(max(offsets[-1] + 1, min(T - (n - len(offsets)), int(round(T * run / total)))))
    offsets[-1] = T
    return offsets


def _logp64(logits, targets, temperature):
    z = logits.double() / temperature
    return z.gather(1, targets[:, None])[:, 0] - torch.logsumexp(z, dim=1)


def prepare(case, seed):
    g = _generator(seed)
    dev = "cuda"
    if case["op"] in ("save", "linear"):
        T, K = case["tokens"], case["inp"]
        # activations: a column's size differs from its neighbour's, a few columns are far larger than the rest
        x = torch.randn(T, K, generator=g, device=dev) * torch.exp(0.5 * torch.randn(K, generator=g, device=dev))
        x[:, ::97] *= 24.0
        state = dict(case=case, x=x.to(_DTYPES[case["x"]]))
        if case["op"] == "linear":
            dy = torch.randn(T, case["out"], generator=g, device=dev) * 1e-3
            state["dy"] = dy.to(_DTYPES[case["dy"]])
            state["dw"] = torch.empty(case["out"], K, dtype=_DTYPES[case["dw"]], device=dev)
        else:
            state["out"] = torch.empty_like(state["x"])
        return state
    T, V, dtype = case["tokens"], case["vocab"], _DTYPES[case["dtype"]]
    whole = torch.empty(T, V + case["pad"], dtype=dtype, device=dev)
    step = max(1, 2 ** 27 // (V + case["pad"]))
    for a in range(0, T, step):
        whole[a:a + step] = torch.randn(min(step, T - a), V + case["pad"], generator=g, device=dev) * 2.0
    logits = whole[:, :V]
    targets = torch.randint(0, V, (T,), generator=g, device=dev)
    # a model mostly takes tokens that it finds likely
    likely = torch.rand(T, generator=g, device=dev) < 0.7
    at = torch.arange(T, device=dev)
    logits[at, targets] = torch.where(likely, torch.full((T,), 10.0, device=dev),
                                      logits[at, targets].float()).to(dtype)
    taken = _logp64(logits, targets, case["temperature"])
    masked = torch.randperm(T, generator=g, device=dev)[:_masked_count(case)]
    targets[masked] = -100
    taken[masked] = 0.0
    state = dict(case=case, logits=logits, targets=targets,
                 logp=torch.empty(T, device=dev), lse=torch.empty(T, device=dev))
    if case["op"] == "logprobs":
        return state
    state["dlogits"] = torch.empty_like(whole)[:, :V]
    # another policy's log-probabilities: an older one's, or the reference's; steps of 0.01, none of which lies on a
    # border of the clip range (log 0.8, log 1.2, log 1.28 are 0.002 and more away)
    other = torch.round(torch.randn(T, generator=g, device=dev) * 16.0).double() * 0.01
    if case["op"] == "logprobs_grad":
        state["dlogp"] = torch.randn(T, generator=g, device=dev) / T
    elif case["op"] == "policy":
        state["old"] = (taken + other).float()
        state["adv"] = torch.randn(T, generator=g, device=dev)
        state["weights"] = torch.where(targets < 0, 0.0, 1.0 / max(1, T - _masked_count(case))).float()
        state["ref"] = (taken + 0.3 * torch.randn(T, generator=g, device=dev).double()).float() if case["kl"] else None
        state["stats"] = torch.empty(4, device=dev)
    else:
        state["ref"] = (taken + other).float()
        state["offsets"] = _pair_offsets(case)                                   # on the host, as the call takes them
        state["offsets_gpu"] = torch.tensor(state["offsets"], dtype=torch.int64, device=dev)
        state["margins"] = torch.empty(case["pairs"], device=dev)
        state["loss"] = torch.empty(1, device=dev)
    return state


# ------------------------------------------------------------------------------------------------------ plain forms
def _softmax_parts(logits, targets, temperature):
    z = logits.float() / temperature
    counts = targets >= 0
    m = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(dim=1, keepdim=True)
    picked = (z - m).gather(1, targets.clamp(min=0)[:, None])[:, 0]
    zero = torch.zeros((), device=z.device)
    logp = torch.where(counts, picked - torch.log(total[:, 0]), zero)
    lse = torch.where(counts, m[:, 0] + torch.log(total[:, 0]), zero)
    return e, total, logp, lse, counts


def _plain_dlogits(e, total, targets, counts, dlogp, temperature, out):
    c = torch.where(counts, dlogp, torch.zeros((), device=dlogp.device)) / temperature
    d = e * (-c[:, None] / total)
    at = torch.arange(d.shape[0], device=d.device)
    d[at, targets.clamp(min=0)] += c
    out.copy_(d)
    return out


def _plain_policy(s, case):
    e, total, logp, _, counts = _softmax_parts(s["logits"], s["targets"], case["temperature"])
    ratio = torch.exp(logp - s["old"])
    kept = ratio.clamp(1.0 - _LOW, 1.0 + case["high"])
    free, held = -s["adv"] * ratio, -s["adv"] * kept
    loss = torch.maximum(free, held)
    slope = torch.where(free >= held, free, torch.zeros_like(free))
    kl = torch.zeros_like(loss)
    if case["kl"]:
        away = s["ref"] - logp
        kl = torch.exp(away) - away - 1.0
        loss = loss + case["kl"] * kl
        slope = slope + case["kl"] * (1.0 - torch.exp(away))
    w = torch.where(counts, s["weights"], torch.zeros_like(s["weights"]))
    stats = torch.stack([(w.double() * loss.double()).sum(), (w.double() * kl.double()).sum(),
                         (w.double() * (free < held).double()).sum(), w.double().sum()]).float()
    _plain_dlogits(e, total, s["targets"], counts, w * slope, case["temperature"], s["dlogits"])
    return [stats, logp, s["dlogits"]]


def _plain_preference(s, case):
    e, total, logp, _, counts = _softmax_parts(s["logits"], s["targets"], case["temperature"])
    away = torch.where(counts, logp.double() - s["ref"].double(), torch.zeros((), device=logp.device, dtype=torch.float64))
    run = torch.cat([torch.zeros(1, dtype=torch.float64, device=away.device), away.cumsum(0)])
    sums = run[s["offsets_gpu"][1:]] - run[s["offsets_gpu"][:-1]]
    margin = _BETA * (sums[0::2] - sums[1::2])
    soft = lambda v: torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-v.abs()))  # noqa: E731
    eps, scale = case["smooth"], 1.0 / case["pairs"]
    loss = scale * ((1.0 - eps) * soft(-margin) + eps * soft(margin)).sum()
    slope = scale * _BETA * (1.0 / (1.0 + torch.exp(-margin)) - (1.0 - eps))
    sign = torch.stack([slope, -slope], dim=1).reshape(-1)
    lengths = s["offsets_gpu"][1:] - s["offsets_gpu"][:-1]
    dlogp = torch.repeat_interleave(sign, lengths, output_size=case["tokens"]).float()
    _plain_dlogits(e, total, s["targets"], counts, dlogp, case["temperature"], s["dlogits"])
    return [loss.float().reshape(1), margin.float(), logp, s["dlogits"]]


def _plain_saved(x):
    """The values that the 8-bit form stands for: blocks of 32 tokens of a column, e4m3 times a power of two."""
    T, K = x.shape
    blocks = -(-T // _BLOCK)
    full = torch.zeros(blocks * _BLOCK, K, device=x.device)
    full[:T] = x
    full = full.view(blocks, _BLOCK, K)
    most = full.abs().amax(dim=1, keepdim=True)
    mantissa, exponent = torch.frexp(most / _E4M3_MAX)       # the smallest e with most <= 448 * 2^e
    e = torch.where(mantissa == 0.5, exponent - 1, exponent).clamp(min=-117)
    scale = torch.ldexp(torch.ones_like(most), e)
    held = (full / scale).to(torch.float8_e4m3fn).float() * scale
    return held.view(blocks * _BLOCK, K)[:T]


# --------------------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    return _run_own(s, case) if own else _run_plain(s, case)


def _run_plain(s, case):
    op = case["op"]
    if op == "save":
        s["out"].copy_(_plain_saved(s["x"]))
        return s["out"]
    if op == "linear":
        s["dw"].copy_(s["dy"].float().t() @ _plain_saved(s["x"]))
        return s["dw"]
    if op == "policy":
        return _plain_policy(s, case)
    if op == "preference":
        return _plain_preference(s, case)
    e, total, logp, lse, counts = _softmax_parts(s["logits"], s["targets"], case["temperature"])
    if op == "logprobs":
        return [logp, lse]
    _plain_dlogits(e, total, s["targets"], counts, s["dlogp"], case["temperature"], s["dlogits"])
    return [logp, lse, s["dlogits"]]


def _run_own(s, case):
    import paper_2512_09685_amd as star

    op = case["op"]
    if op in ("save", "linear"):
        T, K = s["x"].shape
        packed = torch.empty(star.star_act_bytes(T, K), dtype=torch.uint8, device=s["x"].device)
        star.star_act_pack(s["x"], packed)
        if op == "save":
            star.star_act_unpack(packed, s["out"])
            return s["out"]
        star.star_act_weight_grad(s["dy"], packed, s["dw"])
        return s["dw"]
    t = case["temperature"]
    if op == "policy":
        star.star_policy_loss(s["logits"], s["targets"], s["old"], s["adv"], s["stats"], dlogits=s["dlogits"],
                              ref_logp=s["ref"], weights=s["weights"], scale=1.0, clip_low=_LOW, clip_high=case["high"],
                              kl_coef=case["kl"], temperature=t, logp_out=s["logp"])
        return [s["stats"], s["logp"], s["dlogits"]]
    if op == "preference":
        star.star_preference_loss(s["logits"], s["targets"], s["ref"], s["offsets"], s["loss"], dlogits=s["dlogits"],
                                  beta=_BETA, label_smoothing=case["smooth"], temperature=t,
                                  margins_out=s["margins"], logp_out=s["logp"])
        return [s["loss"], s["margins"], s["logp"], s["dlogits"]]
    star.star_token_logprobs(s["logits"], s["targets"], s["logp"], lse_out=s["lse"], temperature=t)
    if op == "logprobs":
        return [s["logp"], s["lse"]]
    star.star_token_logprobs_grad(s["logits"], s["targets"], s["lse"], s["dlogp"], s["dlogits"], temperature=t)
    return [s["logp"], s["lse"], s["dlogits"]]


# ------------------------------------------------------------------------------------------------------------- work
def work(case):
    size = {_BF16: 2, _F32: 4}
    T = case["tokens"]
    if case["op"] in ("save", "linear"):
        K = case["inp"]
        saved = -(-T // _BLOCK) * K * (_BLOCK + 1)
        if case["op"] == "save":
            return {"bytes": 2 * T * K * size[case["x"]] + 2 * saved, "flops": 0}
        N = case["out"]
        return {"bytes": T * K * size[case["x"]] + 2 * saved + T * N * size[case["dy"]] + N * K * size[case["dw"]],
                "flops": 2 * T * N * K}
    counted = T - _masked_count(case)
    row = case["vocab"] * size[case["dtype"]]
    small = {"logprobs": 16, "logprobs_grad": 20, "policy": 28, "preference": 16}[case["op"]] * T
    written = 0 if case["op"] == "logprobs" else T * row
    return {"bytes": counted * row + written + small, "flops": 4 * counted * case["vocab"]}


# ------------------------------------------------------------------------------------------------- from the definition
def _exact_saved(x):
    """Round-half-even on the grid of each value's own binade, 64 bits, straight from the definition of the format."""
    T, K = x.shape
    b = torch.nn.functional.pad(x.double(), (0, 0, 0, -T % _BLOCK)).unflatten(0, (-1, _BLOCK))
    most = b.abs().max(dim=1, keepdim=True).values
    e = torch.ceil(torch.log2(most.clamp(min=1e-300) / _E4M3_MAX))
    e = torch.where(most <= _E4M3_MAX * torch.exp2(e - 1.0), e - 1.0, e)      # (where log2 was rounded over a border)
    e = torch.where(most > _E4M3_MAX * torch.exp2(e), e + 1.0, e).clamp(min=-117.0)
    v = b * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return (torch.round(v / step) * step * torch.exp2(e)).flatten(0, 1)[:T]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "save":
        return _exact_saved(s["x"])
    if op == "linear":
        return torch.matmul(s["dy"].double().t().contiguous(), _exact_saved(s["x"]))
    T, V = s["logits"].shape
    beta = 1.0 / case["temperature"]
    y, counts = s["targets"].clamp(min=0), (s["targets"] >= 0).double()
    logp, lse = torch.empty(2, T, dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 26 // V)
    for a in range(0, T, step):
        z = s["logits"][a:a + step].double() * beta
        part = torch.logsumexp(z, dim=1)
        lse[a:a + step] = part * counts[a:a + step]
        logp[a:a + step] = (z[torch.arange(z.shape[0], device="cuda"), y[a:a + step]] - part) * counts[a:a + step]
    if op == "logprobs":
        return [logp, lse]
    if op == "logprobs_grad":
        first, slope = [logp, lse], s["dlogp"].double()
    elif op == "policy":
        A, w = s["adv"].double(), s["weights"].double() * counts
        r = torch.exp(logp - s["old"].double())
        clipped = torch.where(A >= 0, r > 1.0 + case["high"], r < 1.0 - _LOW)
        bound = torch.where(A >= 0, 1.0 + case["high"], 1.0 - _LOW)
        loss, slope = -A * torch.where(clipped, bound, r), torch.where(clipped, 0.0, -A * r)
        kl = torch.zeros_like(loss)
        if case["kl"]:
            q = torch.exp(s["ref"].double() - logp)
            kl = q - 1.0 - (s["ref"].double() - logp)
            loss, slope = loss + case["kl"] * kl, slope + case["kl"] * (1.0 - q)
        stats = torch.stack([(w * loss).sum(), (w * kl).sum(), (w * clipped).sum(), w.sum()])
        first, slope = [stats, logp], slope * w
    else:
        offsets = s["offsets"]
        away = (logp - s["ref"].double()) * counts
        sums = torch.stack([away[a:b].sum() for a, b in zip(offsets, offsets[1:])])
        margin = _BETA * (sums[0::2] - sums[1::2])
        eps = case["smooth"]
        loss = (-(1.0 - eps) * torch.nn.functional.logsigmoid(margin) -
                eps * torch.nn.functional.logsigmoid(-margin)).mean()
        d = _BETA * (eps * torch.sigmoid(margin) - (1.0 - eps) * torch.sigmoid(-margin)) / case["pairs"]
        slope = torch.zeros_like(logp)
        for i, (a, b) in enumerate(zip(offsets, offsets[1:])):
            slope[a:b] = d[i // 2] * (1.0 if i % 2 == 0 else -1.0)
        first = [loss.reshape(1), margin, logp]
    c = slope * counts * beta
    dlogits = torch.empty(T, V, dtype=torch.float64, device="cuda")
    for a in range(0, T, step):
        z = s["logits"][a:a + step].double() * beta
        p = torch.softmax(z, dim=1)
        dlogits[a:a + step] = -c[a:a + step, None] * p
        rows = torch.arange(z.shape[0], device="cuda")
        dlogits[a + rows, y[a:a + step]] += c[a:a + step]
    return first + [dlogits]
