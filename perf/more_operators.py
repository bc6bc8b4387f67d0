"""Performance cases of the operators around a block of refined layers in a training or serving step.

Each case is a dict of plain values; "op" names the operator:

  norm    the root-mean-square norm with the residual's addition: "y" is the norm alone, "i8"
          its result on 8 bits with a scale for each token (what an 8-bit layer takes),
          "train" the norm with its backward pass (gradients of the tokens and of the gain);
  linlog  log probabilities of given tokens from hidden states and the output layer's weights,
          without the logits; with "train" the gradients of the hidden states and of the weights;
  adamw   a step of AdamW over all tensors of a stack of gated blocks at once, the moments in
          32 bits or in 8 (e4m3 with a power of two for each 128 values).

`own` false computes a case in plain torch operations in 32 bits (64 where a power of two has
to be applied exactly), rounded once at the end; true calls the library.  Every input comes from
the seed.
"""

from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
_EPS = 1e-6                                          # of the norm
_LR, _B1, _B2, _ADAM_EPS, _DECAY = 3e-4, 0.9, 0.999, 1e-8, 0.1
_BLOCK = 128                                         # values that share a power of two


def listed():
    return [
        # one token between two layers in serving: latency
        {"name": "norm_token", "op": "norm", "form": "y", "tokens": 1, "d": 4096,
         "dtype": "bfloat16", "gain": "bfloat16", "residual": True},
        # prefill of two sequences of 2048 into an 8-bit layer
        {"name": "norm_prefill_i8", "op": "norm", "form": "i8", "tokens": 4096, "d": 4096,
         "dtype": "bfloat16", "gain": "bfloat16", "residual": True},
        # training: forward and backward in the middle of the residual stream
        {"name": "norm_train", "op": "norm", "form": "train", "tokens": 8192, "d": 4096,
         "dtype": "bfloat16", "gain": "bfloat16", "residual": True},
        # a small model's norm with odd sizes, fp32
        {"name": "norm_train_odd", "op": "norm", "form": "train", "tokens": 611, "d": 2501,
         "dtype": "float32", "gain": "float32", "residual": False},
        # the score of one token in serving: the output layer's weights are read once
        {"name": "linlog_token", "op": "linlog", "tokens": 1, "d": 4096, "vocab": 128000,
         "dtype": "bfloat16", "masked": False, "train": False},
        # perplexity of an evaluation sequence with padding
        {"name": "linlog_eval", "op": "linlog", "tokens": 2047, "d": 4096, "vocab": 32001,
         "dtype": "float16", "masked": True, "train": False},
        # a training step's loss over two sequences with its gradients
        {"name": "linlog_train", "op": "linlog", "tokens": 4096, "d": 4096, "vocab": 128000,
         "dtype": "bfloat16", "masked": False, "train": True},
        # a small model with odd sizes, prompts masked
        {"name": "linlog_train_odd", "op": "linlog", "tokens": 611, "d": 1000, "vocab": 50257,
         "dtype": "float16", "masked": True, "train": True},
        # one small block: latency
        {"name": "adamw_small", "op": "adamw", "layers": 1, "d": 256, "f": 1000,
         "dtype": "bfloat16", "bits": 8},
        # recovery training of one block of a 4096-wide model, the moments in 32 bits
        {"name": "adamw_block32", "op": "adamw", "layers": 1, "d": 4096, "f": 11008,
         "dtype": "bfloat16", "bits": 32},
        # the same with the moments in 8 bits
        {"name": "adamw_block8", "op": "adamw", "layers": 1, "d": 4096, "f": 11008,
         "dtype": "bfloat16", "bits": 8},
        # all tensors of a small model, odd sizes, fp32 parameters
        {"name": "adamw_many", "op": "adamw", "layers": 48, "d": 500, "f": 1375,
         "dtype": "float32", "bits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["norm", "linlog", "adamw"])
    dtype = rng.choice(["bfloat16", "float16", "float32"])
    if op == "norm":
        form = rng.choice(["y", "i8", "train"])
        d = 16 * _log(rng, 4, 1024) if form == "i8" or rng.random() < 0.5 else _log(rng, 64, 16384)
        most = 8192 * 4096 // d // (2 if dtype == "float32" else 1)
        return {"op": op, "form": form, "tokens": _log(rng, 1, min(16384, most)), "d": d,
                "dtype": dtype, "gain": rng.choice([dtype, "float32"]),
                "residual": rng.random() < 0.6}
    if op == "linlog":
        train = rng.random() < 0.5
        d, vocab = 8 * _log(rng, 16, 1024), _log(rng, 1000, 128000)
        most = 4096 * 4096 * 128000 // (d * vocab)
        return {"op": op, "tokens": _log(rng, 1, min(4096, most)), "d": d, "vocab": vocab,
                "dtype": rng.choice(["bfloat16", "bfloat16", "float16"]),
                "masked": rng.random() < 0.5, "train": train}
    d = _log(rng, 64, 4096)
    f = _log(rng, d, 3 * d)
    most = 4096 * 11008 * 2 // (d * f)
    return {"op": op, "layers": _log(rng, 1, max(1, min(48, most))), "d": d, "f": f,
            "dtype": dtype, "bits": rng.choice([8, 8, 32])}


# ---- inputs ----

def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _rand(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _tokens(gen, m, cols):
    """m hidden states: one channel in a hundred is an outlier, ten times the others."""
    return _randn(gen, m, cols) * torch.where(_rand(gen, cols) < 0.01, 10.0, 1.0)


def _tensors(case):
    """(shape, offset) of every parameter in the flat buffers, and the buffers' length.

    A tensor begins at a multiple of 128 values, as the moments' blocks do.
    """
    d, f = case["d"], case["f"]
    found, at = [], 0
    for _ in range(case["layers"]):
        for shape in ((d,), (f, d), (f, d), (d, f), (d,)):
            found.append((shape, at))
            at += -(-math.prod(shape) // _BLOCK) * _BLOCK
    return found, at


def _views(flat, tensors):
    return [flat[at:at + math.prod(shape)].view(shape) for shape, at in tensors]


def prepare(case, seed):
    gen = _gen(seed)
    s = {"case": dict(case)}
    dt = _DTYPES[case["dtype"]]
    if case["op"] == "norm":
        t, d = case["tokens"], case["d"]
        s["x"] = _tokens(gen, t, d).to(dt)
        s["residual"] = _tokens(gen, t, d).mul_(2.0).to(dt) if case["residual"] else None
        s["gain"] = _randn(gen, d).mul_(0.1).add_(1.0).to(_DTYPES[case["gain"]])
        if case["form"] == "train":
            s["dy"] = _randn(gen, t, d).mul_(0.05).to(dt)
            # what reaches the sum itself on the residual path
            s["dh"] = _randn(gen, t, d).mul_(0.05).to(dt) if case["residual"] else None
    elif case["op"] == "linlog":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        w = _randn(gen, v, d).mul_(2.0 / math.sqrt(d))
        s["targets"] = torch.randint(0, v, (t,), generator=gen, device="cuda")
        # half of the positions are predicted well: their token leads
        lead = _rand(gen, t).mul_(24.0).sub_(12.0).clamp_min_(0.0)
        s["x"] = (_tokens(gen, t, d) + w[s["targets"]] * (lead / 4.0)[:, None]).to(dt)
        s["w"] = w.to(dt)
        if case["masked"]:
            s["targets"] = torch.where(_rand(gen, t) < 0.2, -1, s["targets"])
        if case["train"]:
            s["d_logprob"] = _rand(gen, t).add_(0.5).neg_()
            s["d_lse"] = _rand(gen, t).mul_(0.02)   # keeps the normalisation near 1
    else:
        tensors, n = _tensors(case)
        live = torch.zeros(n, dtype=torch.bool, device="cuda")
        for view in _views(live, tensors):
            view.fill_(True)
        s["tensors"], s["step"], s["seed"] = tensors, 17, int(seed)
        # gradients over several orders of magnitude from one block to the next
        spread = torch.exp(_randn(gen, n // _BLOCK)).mul_(1e-3).repeat_interleave(_BLOCK)
        params = torch.where(live, _randn(gen, n).mul_(0.02), 0.0)
        s["grads"] = torch.where(live, _randn(gen, n).mul_(spread), 0.0).to(dt)
        s["params"] = params.to(dt)
        # 16-bit parameters are the rounded ones of 32 bits
        s["master"] = params if dt != torch.float32 else None
        m = torch.where(live, _randn(gen, n).mul_(spread).mul_(0.3), 0.0)
        v = torch.where(live, _rand(gen, n).add_(0.1).mul_(spread).mul_(spread), 0.0)
        if case["bits"] == 8:
            half = torch.full((n,), 1 << 19, dtype=torch.int32, device="cuda")
            s["m"], s["m_exp"] = _encode(m, half, False)
            s["v"], s["v_exp"] = _encode(torch.sqrt(v), half, True)
        else:
            s["m"], s["v"], s["m_exp"], s["v_exp"] = m, v, None, None
        for name in ("params", "master", "m", "v", "m_exp", "v_exp"):   # where the step goes
            s["new_" + name] = None if s[name] is None else torch.zeros_like(s[name])
        s["param_list"], s["grad_list"], s["new_list"] = (
            _views(s[k], tensors) for k in ("params", "grads", "new_params"))
    return s


# ---- one pass ----

def run(state):
    return _PATHS[state["case"]["op"]][1 if own else 0](state)


def _norm_plain(s):
    c, dt = s["case"], s["x"].dtype
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
    hf, gain = h.float(), s["gain"].float()
    r = 1.0 / torch.sqrt((hf * hf).mean(1, keepdim=True) + _EPS)
    out = {} if s["residual"] is None else {"h": h}
    if c["form"] == "i8":
        w = hf * gain
        amax = w.abs().amax(1, keepdim=True)
        live = amax >= 2.0 ** -100
        # (a quotient of tensors: a scalar's would be a product with the rounded reciprocal)
        mul = torch.full_like(amax, 127.0) / torch.where(live, amax, 1.0)
        out["q"] = torch.where(live, torch.round(w * mul), 0.0).to(torch.int8)
        out["scale"] = torch.where(live, amax / torch.full_like(amax, 127.0) * r, 0.0)
        return out
    out["y"] = (hf * r * gain).to(dt)
    if c["form"] == "train":
        dy = s["dy"].float()
        u = dy * gain
        dx = r * (u - hf * (r * r * (u * hf).mean(1, keepdim=True)))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        out["dx"] = dx.to(dt)
        out["dgain"] = (dy * (hf * r)).sum(0).to(s["gain"].dtype)
    return out


def _norm_own(s):
    from paper_2609_38599_amd import binding as jb
    c, x, res = s["case"], s["x"], s["residual"]
    if c["form"] == "i8":
        got = jb.rms_norm_i8(x, s["gain"], residual=res, eps=_EPS)
        out = {"q": got[0], "scale": got[1]}
        if res is not None:
            out["h"] = got[2]
        return out
    got = jb.rms_norm(x, s["gain"], residual=res, eps=_EPS)
    out = {"y": got} if res is None else {"y": got[0], "h": got[1]}
    if c["form"] == "train":
        out["dx"], out["dgain"] = jb.rms_norm_backward(out.get("h", x), s["gain"], s["dy"],
                                                       dH=s["dh"], eps=_EPS)
    return out


def _linlog_plain(s):
    c, t = s["case"], s["targets"]
    x, w = s["x"].float(), s["w"].float()
    logits = x @ w.t()
    m = logits.amax(1, keepdim=True)
    e = torch.exp(logits - m)
    z = e.sum(1, keepdim=True)
    lse = (m + torch.log(z))[:, 0]
    has, at = t >= 0, t.clamp_min(0)[:, None]
    out = {"logprob": torch.where(has, logits.gather(1, at)[:, 0] - lse, 0.0), "lse": lse}
    if c["train"]:
        g = torch.where(has, s["d_logprob"], 0.0)[:, None]
        d = e.mul_((s["d_lse"][:, None] - g) / z).scatter_add_(1, at, g)
        out["dx"], out["dw"] = (d @ w).to(s["x"].dtype), (d.t() @ x).to(s["w"].dtype)
    return out


def _linlog_own(s):
    from paper_2609_38599_amd import binding as jb
    r = jb.linear_logprobs(s["x"], s["w"], s["targets"])
    out = {"logprob": r.logprob, "lse": r.lse}
    if s["case"]["train"]:
        out["dx"], out["dw"] = jb.linear_logprobs_backward(s["x"], s["w"], s["targets"], r,
                                                           s["d_logprob"], d_lse=s["d_lse"])
    return out


def _two_to(exponent):
    """2^exponent in 64 bits for a tensor of whole numbers, exactly."""
    return ((exponent.long() + 1023) << 52).view(torch.float64)


def _encode(x, dither, positive):
    """(e4m3 values, exponents): x = value 2^(exponent - 134), in blocks of 128.

    The largest of a block lies in 2^7..2^8.  dither: 20 bits that are added below a value's
    last bit before it is cut off.  positive: what is above zero stays above zero.
    """
    blocks = x.view(-1, _BLOCK)
    field = (blocks.abs().amax(1).view(torch.int32) >> 23).clamp_min(1)
    # (the bits of value 2^-120 in 32 are e4m3's, 20 places further up)
    scaled = (blocks.abs().double() * _two_to(14 - field)[:, None]).float()
    code = (scaled.view(torch.int32).view(-1) + dither) >> 20
    if positive:
        code = torch.where((x > 0) & (code == 0), 1, code)
    code = torch.where(x < 0, code | 0x80, code)
    return code.to(torch.uint8).view(torch.float8_e4m3fn), field.to(torch.uint8)


def _decode(value, exponent):
    blocks = value.float().double().view(-1, _BLOCK)
    return (blocks * _two_to(exponent.int() - 134)[:, None]).float().view(-1)


def _mix(x):
    """32 bits of noise from 32 (held in 64)."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _noise(n, seed, step, device):
    """The dithers of m and of sqrt(v) of n values in a step."""
    key = _mix(((_mix((_mix(seed & 0xFFFFFFFF) + (seed >> 32)) & 0xFFFFFFFF)) + step) & 0xFFFFFFFF)
    r = _mix((torch.arange(n, device=device) + key) & 0xFFFFFFFF)   # n < 2^32
    return ((r & 0xFFFF) << 4).int(), ((r >> 16) << 4).int()


def _adamw_plain(s):
    c, t = s["case"], s["step"]
    g = s["grads"].float()
    if c["bits"] == 8:
        m, root = _decode(s["m"], s["m_exp"]), _decode(s["v"], s["v_exp"])
        v = root * root
    else:
        m, v = s["m"], s["v"]
    # each product and sum rounded by itself
    m = m * _B1 + g * (1.0 - _B1)
    v = v * _B2 + (g * (1.0 - _B2)) * g
    root = torch.sqrt(v)
    p = s["params"] if s["master"] is None else s["master"]
    denom = root * (1.0 / math.sqrt(1.0 - _B2 ** t)) + _ADAM_EPS
    p = p * (1.0 - _LR * _DECAY) - (m * (_LR / (1.0 - _B1 ** t))) / denom
    out = {"params": p.to(s["params"].dtype)}
    if s["master"] is not None:
        out["master"] = p
    if c["bits"] == 8:
        noise = _noise(len(g), s["seed"], t, g.device)
        out["m"], out["m_exp"] = _encode(m, noise[0], False)
        out["v"], out["v_exp"] = _encode(root, noise[1], True)
    else:
        out["m"], out["v"] = m, v
    return out


def _adamw_own(s):
    from paper_2609_38599_amd import binding as jb
    old, new = (jb.AdamWState(*(s[k + n] for n in ("master", "m", "v", "m_exp", "v_exp")))
                for k in ("", "new_"))
    jb.adamw_step(s["param_list"], s["grad_list"], old, s["step"], _LR, beta1=_B1, beta2=_B2,
                  eps=_ADAM_EPS, weight_decay=_DECAY, seed=s["seed"], out=(s["new_list"], new))
    return {n: s["new_" + n] for n in ("params", "master", "m", "v", "m_exp", "v_exp")
            if s["new_" + n] is not None}


_PATHS = {"norm": (_norm_plain, _norm_own), "linlog": (_linlog_plain, _linlog_own),
          "adamw": (_adamw_plain, _adamw_own)}


# ---- what a pass cannot do without ----

def work(case):
    e = torch.finfo(_DTYPES[case["dtype"]]).bits // 8
    if case["op"] == "norm":
        t, d = case["tokens"], case["d"]
        res = 2 if case["residual"] else 0
        gain = torch.finfo(_DTYPES[case["gain"]]).bits // 8
        n = t * d * e * (1 + res) + d * gain
        if case["form"] == "i8":
            return {"bytes": n + t * d + 4 * t, "flops": 6 * t * d}
        if case["form"] == "y":
            return {"bytes": n + t * d * e, "flops": 5 * t * d}
        # backward: dy and what reaches the sum in, the gradients out (the sum is at hand)
        return {"bytes": n + t * d * e * (3 + (1 if res else 0)) + d * gain, "flops": 14 * t * d}
    if case["op"] == "linlog":
        t, d, v = case["tokens"], case["d"], case["vocab"]
        times = 2 if case["train"] else 1
        return {"bytes": e * (t * d + v * d) * times + 16 * t,
                "flops": 2 * t * d * v * (3 if case["train"] else 1)}
    n = sum(math.prod(shape) for shape, _ in _tensors(case)[0])
    master = 8 if e == 2 else 0
    state = 16 if case["bits"] == 32 else 4 + 4 / _BLOCK
    return {"bytes": int(n * (3 * e - (e if e == 2 else 0) + master + state)), "flops": 14 * n}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "linlog": _linlog_exact, "adamw": _adamw_exact}[case["op"]](case, s)


def _norm_exact(case, s):
    x = s["x"].double()
    if s["residual"] is not None:   # the sum is defined by its rounding
        x = (x + s["residual"].double()).to(s["x"].dtype).double()
    x.requires_grad_(case["form"] == "train")
    gain = s["gain"].double().requires_grad_(case["form"] == "train")
    rms = (x.square().sum(1) / case["d"] + _EPS).sqrt()
    y = x / rms[:, None] * gain
    out = {} if s["residual"] is None else {"h": x.detach()}
    if case["form"] == "i8":
        out["q"] = None   # whole numbers: compared for equality elsewhere
        out["scale"] = y.abs().max(dim=1, keepdim=True).values / 127.0
        return out
    out["y"] = y.detach()
    if case["form"] == "train":
        total = (y * s["dy"].double()).sum()
        if s["dh"] is not None:
            total = total + (x * s["dh"].double()).sum()
        out["dx"], out["dgain"] = torch.autograd.grad(total, (x, gain))
    return out


def _linlog_exact(case, s):
    x, w, t = s["x"].double(), s["w"].double(), s["targets"]
    logp = torch.mm(x, w.t())
    lse = torch.logsumexp(logp, dim=1)
    logp -= lse[:, None]
    rows = torch.nonzero(t >= 0)[:, 0]
    logprob = torch.zeros_like(lse)
    logprob[rows] = logp[rows, t[rows]]
    out = {"logprob": logprob, "lse": lse}
    if case["train"]:
        g = torch.zeros_like(lse)
        g[rows] = s["d_logprob"].double()[rows]
        d = logp.exp_().mul_((s["d_lse"].double() - g)[:, None])
        d[rows, t[rows]] += g[rows]
        out["dx"], out["dw"] = torch.mm(d, w), torch.mm(d.t(), x)
    return out


def _adamw_exact(case, s):
    g, t = s["grads"].double(), s["step"]
    if case["bits"] == 8:
        m, v = (torch.ldexp(s[k].float().double().view(-1, _BLOCK), s[k + "_exp"].int()[:, None] - 134).view(-1)
                for k in ("m", "v"))
        v = v.square()
    else:
        m, v = s["m"].double(), s["v"].double()
    m = torch.lerp(g, m, _B1)
    v = torch.lerp(g.square(), v, _B2)
    p = (s["params"] if s["master"] is None else s["master"]).double()
    p = p - _LR * (_DECAY * p + m / (1 - _B1 ** t) / ((v / (1 - _B2 ** t)).sqrt() + _ADAM_EPS))
    out = {"params": p}
    if s["master"] is not None:
        out["master"] = p
    if case["bits"] == 32:
        out["m"], out["v"] = m, v
    else:   # rounded by the dither: compared by their types elsewhere
        out["m"] = out["v"] = out["m_exp"] = out["v_exp"] = None
    return out
