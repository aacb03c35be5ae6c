"""Cases, inputs and plain forms of the language-model operators, for timing and comparing them.

Three operators that stand next to the split FP32 product in a language model's FP32 path, each with
its gradient:

  linear    Y = act(X W + b) + R on the three-product kernel; gradients of X, W and b
  norm      layer normalisation with weight and bias; gradients of X, weight and bias
  logprobs  log probabilities of given tokens with entropy and top alternatives; gradient of the logits

`own` false: plain torch operations in 32 bits, rounded once at the end.  `own` true: the library's
entry points, as a program calls them.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_handles = []


def listed():
    return [
        # one token through a projection of a small model: latency decides
        _linear("linear_decode_one", 1, 4096, 1024, act="silu", packed=True),
        # a batch of 24 sequences, one token each, through an up-projection: the weight's bytes decide
        _linear("linear_decode_batch", 24, 16384, 4096, act="gelu", packed=True),
        # a short prompt, every size odd, weight stored inputs x outputs, down-projection with residual
        _linear("linear_prompt_ragged", 777, 2049, 1001, layout="kn", residual=True),
        # a long prompt through a square projection with residual
        _linear("linear_prompt", 4096, 4096, 4096, residual=True),
        # training step of a small up-projection, weight stored inputs x outputs
        _linear("linear_train_small", 1024, 4096, 1024, layout="kn", act="silu", residual=True, train=True),
        # training step of a large up-projection
        _linear("linear_train_large", 8192, 16384, 4096, act="gelu", train=True),
        # the norm in front of a layer, eight sequences, one token each
        _norm("norm_decode", 8, 4096, "f32"),
        # the same in training, FP32
        _norm("norm_train_f32", 8192, 4096, "f32", train=True),
        # 16-bit training with odd sizes: rows that start on odd addresses
        _norm("norm_train_bf16_ragged", 6001, 2047, "bf16", train=True),
        # sampling: four sequences, a large vocabulary of which a part is not allowed, 20 alternatives
        _logprobs("logprobs_decode", 4, 131072, "f32", top=20, masked=0.3),
        # scoring a text: 16-bit logits (many ties), odd vocabulary, eight alternatives
        _logprobs("logprobs_score_bf16", 1000, 50001, "bf16", top=8),
        # policy-gradient step: log probabilities and entropy of one long batch, and the gradient of both
        _logprobs("logprobs_train", 4096, 65536, "f32", train=True),
    ]


def _linear(name, m, n, k, layout="nk", act="none", bias=True, residual=False, packed=False, train=False):
    return {"name": name, "op": "linear", "m": m, "n": n, "k": k, "layout": layout, "act": act,
            "bias": bias, "residual": residual, "packed": packed, "train": train}


def _norm(name, rows, cols, dtype, train=False):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "dtype": dtype, "train": train}


def _logprobs(name, rows, vocab, dtype, top=0, masked=0.0, train=False):
    return {"name": name, "op": "logprobs", "rows": rows, "vocab": vocab, "dtype": dtype, "top": top,
            "masked": masked, "train": train}


def _log_size(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; three in four are left as they fall (odd
    ones among them), the others are made multiples of 64."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))
    if v >= 64 and rng.random() < 0.25:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["linear", "linear", "norm", "logprobs"])
    if op == "linear":
        n, k = _log_size(rng, 1000, 16384), _log_size(rng, 1000, 8192)
        train = rng.random() < 0.4
        m = _log_size(rng, 256, 4096) if train else _log_size(rng, 1, 4096)
        packed = not train and rng.random() < 0.5
        c = _linear("", m, n, k, layout=rng.choice(["nk", "kn"]), act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                    bias=rng.random() < 0.8, residual=rng.random() < 0.5, packed=packed, train=train)
    elif op == "norm":
        c = _norm("", _log_size(rng, 1, 16384), _log_size(rng, 256, 16384), rng.choice(["f32", "f16", "bf16"]),
                  train=rng.random() < 0.6)
        c["rows"] = min(c["rows"], (1 << 26) // c["cols"])
    else:
        train = rng.random() < 0.5
        c = _logprobs("", _log_size(rng, 1, 4096), _log_size(rng, 8192, 200000), rng.choice(["f32", "f16", "bf16"]),
                      top=0 if train else rng.choice([0, 1, 5, 20, 32]), masked=rng.choice([0.0, 0.0, 0.5]), train=train)
        c["rows"] = max(1, min(c["rows"], (1 << 27) // c["vocab"]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs


def _inputs(case, seed):
    """What both sides and the 64-bit form start from, made from the seed alone."""
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s = {"x": normal(m, k)}
        s["x"].mul_(torch.rand(k, generator=g, device=DEV).mul_(1.5).add_(0.25))    # channels of different size
        s["w"] = normal(n, k) if case["layout"] == "nk" else normal(k, n)
        s["w"].mul_(k ** -0.5)
        s["bias"] = normal(n).mul_(0.1) if case["bias"] else None
        s["residual"] = normal(m, n).mul_(2.0) if case["residual"] else None
        if case["train"]:
            s["dy"] = normal(m, n).mul_(1e-3 / m)                                   # a mean loss' gradient: small numbers
    elif case["op"] == "norm":
        r, c, t = case["rows"], case["cols"], TYPES[case["dtype"]]
        x = normal(r, c)
        x.mul_(torch.rand(r, 1, generator=g, device=DEV).mul_(4).add_(0.5))
        x.add_(normal(r, 1).mul_(0.5))
        x[:, :: max(1, c // 7)] *= 8.0                                             # a few channels stand out
        s = {"x": x.to(t), "weight": normal(c).mul_(0.2).add_(1.0), "bias": normal(c).mul_(0.2)}
        if case["train"]:
            s["dy"] = normal(r, c).mul_(1e-2).to(t)
    else:
        r, v, t = case["rows"], case["vocab"], TYPES[case["dtype"]]
        x = normal(r, v).mul_(2.0)
        peaks = torch.randint(0, v, (r, 16), generator=g, device=DEV)
        x.scatter_(1, peaks, 8.0 + 3.0 * normal(r, 16))                            # a few likely tokens a row
        if case["masked"]:
            x.masked_fill_(torch.rand(v, generator=g, device=DEV) < case["masked"], -math.inf)
        x = x.to(t)
        tokens = torch.where(torch.rand(r, generator=g, device=DEV) < 0.7, peaks[:, 0],
                             torch.randint(0, v, (r,), generator=g, device=DEV))
        if r >= 16:
            tokens[torch.rand(r, generator=g, device=DEV) < 0.1] = -1               # positions without a target
        s = {"logits": x, "tokens": tokens}
        if case["train"]:
            s["dlogp"], s["dentropy"] = normal(r).mul_(1.0 / r), normal(r).mul_(0.01 / r)
    return s


def _handle():
    """The library's handle, made once for the process."""
    if not _handles:
        from paper_2507_23387_b200 import binding
        _handles.append((binding.Handle(0), binding))
    return _handles[0]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if not own:
        return s
    h, binding = _handle()
    s["h"], s["binding"] = h, binding
    f32 = dict(dtype=torch.float32, device=DEV)
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["act"] = getattr(binding, "ACT_" + case["act"].upper())
        s["layout"] = binding.WEIGHT_NK if case["layout"] == "nk" else binding.WEIGHT_KN
        s["y"] = torch.empty(m, n, **f32)
        if case["packed"]:        # a server lays its weights out once, when it loads them
            s["wp"] = binding.PackedMatrix(*s["w"].shape)
            h.sgemm_cube_pack(s["w"], s["wp"])
        if case["train"]:         # buffers of a training loop; their contents are written in every pass
            s["xp"], s["wp"] = binding.PackedMatrix(m, k), binding.PackedMatrix(*s["w"].shape)
            s["z"] = torch.empty(m, n, **f32)
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["db"] = torch.empty(n, **f32) if case["bias"] else None
    elif case["op"] == "norm":
        r, c = case["rows"], case["cols"]
        s["y"] = torch.empty_like(s["x"])
        s["mean"], s["rstd"] = torch.empty(r, **f32), torch.empty(r, **f32)
        if case["train"]:
            s["dx"] = torch.empty_like(s["x"])
            s["dweight"], s["dbias"] = torch.empty(c, **f32), torch.empty(c, **f32)
    else:
        r = case["rows"]
        s["logp"], s["entropy"], s["stats"] = torch.empty(r, **f32), torch.empty(r, **f32), torch.empty(r, 2, **f32)
        if case["top"]:
            s["top_logp"] = torch.empty(r, case["top"], **f32)
            s["top_index"] = torch.empty(r, case["top"], dtype=torch.int64, device=DEV)
        if case["train"]:
            s["dlogits"] = torch.empty_like(s["logits"])
    return s


# ---------------------------------------------------------------------------------------- one pass


def run(state):
    op = state["case"]["op"]
    if own:
        return {"linear": _own_linear, "norm": _own_norm, "logprobs": _own_logprobs}[op](state)
    return {"linear": _plain_linear, "norm": _plain_norm, "logprobs": _plain_logprobs}[op](state)


def _own_linear(s):
    h = s["h"]
    if not s["case"]["train"]:
        h.sgemm_cube_linear(s["x"], s.get("wp", s["w"]), s["y"], bias=s["bias"], residual=s["residual"],
                            activation=s["act"], weight_layout=s["layout"])
        return {"y": s["y"]}
    # both operands are split once and serve the product and its two gradients
    h.sgemm_cube_pack(s["x"], s["xp"])
    h.sgemm_cube_pack(s["w"], s["wp"])
    h.sgemm_cube_linear(s["xp"], s["wp"], s["y"], bias=s["bias"], residual=s["residual"], activation=s["act"],
                        preact=s["z"], weight_layout=s["layout"])
    h.sgemm_cube_linear_backward(s["dy"], s["xp"], s["wp"], dX=s["dx"], dW=s["dw"], dbias=s["db"], preact=s["z"],
                                 activation=s["act"], weight_layout=s["layout"])
    return {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_norm(s):
    h = s["h"]
    h.sgemm_cube_layer_norm(s["x"], s["y"], weight=s["weight"], bias=s["bias"], eps=1e-5, mean=s["mean"], rstd=s["rstd"])
    if not s["case"]["train"]:
        return {"y": s["y"]}
    h.sgemm_cube_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["dx"], weight=s["weight"],
                                     dweight=s["dweight"], dbias=s["dbias"])
    return {"y": s["y"], "dx": s["dx"], "dweight": s["dweight"], "dbias": s["dbias"]}


def _own_logprobs(s):
    h = s["h"]
    h.sgemm_cube_token_logprobs(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], stats=s["stats"],
                                top_logp=s.get("top_logp"), top_index=s.get("top_index"))
    out = {"logp": s["logp"], "entropy": s["entropy"]}
    if s["case"]["top"]:
        out["top_logp"], out["top_index"] = s["top_logp"], s["top_index"]
    if s["case"]["train"]:
        h.sgemm_cube_token_logprobs_backward(s["logits"], s["tokens"], s["stats"], s["dlogits"], dlogp=s["dlogp"],
                                             entropy=s["entropy"], dentropy=s["dentropy"])
        out["dlogits"] = s["dlogits"]
    return out


def _plain_act(z, act):
    """act(z) and act'(z)."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).to(z.dtype)
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1 + z * (1 - p))
    return z, None


def _plain_linear(s):
    c = s["case"]
    w = s["w"].t() if c["layout"] == "nk" else s["w"]                # inputs x outputs
    z = s["x"] @ w
    if s["bias"] is not None:
        z = z + s["bias"]
    y, slope = _plain_act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"]
    if not c["train"]:
        return {"y": y}
    dz = s["dy"] if slope is None else s["dy"] * slope
    dw = dz.t() @ s["x"] if c["layout"] == "nk" else s["x"].t() @ dz
    return {"y": y, "dx": dz @ w.t(), "dw": dw, "db": dz.sum(0) if s["bias"] is not None else None}


def _plain_norm(s):
    t = s["x"].dtype
    x = s["x"].float()
    d = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + 1e-5)
    n = d * rstd
    y = (n * s["weight"] + s["bias"]).to(t)
    if not s["case"]["train"]:
        return {"y": y}
    dy = s["dy"].float()
    u = dy * s["weight"]
    dx = rstd * (u - u.mean(1, keepdim=True) - n * (u * n).mean(1, keepdim=True))
    return {"y": y, "dx": dx.to(t), "dweight": (dy * n).sum(0), "dbias": dy.sum(0)}


def _plain_logprobs(s):
    c, t = s["case"], s["logits"].dtype
    x = s["logits"].float()
    target = s["tokens"].clamp(min=0).unsqueeze(1)
    valid = s["tokens"] >= 0
    shifted = x - x.amax(1, keepdim=True)
    e = torch.exp(shifted)
    z = e.sum(1, keepdim=True)
    logz = torch.log(z)
    logp = torch.where(valid, (shifted.gather(1, target) - logz).squeeze(1), 0.0)
    p = e / z
    weighted = torch.where(p > 0, p * shifted, 0.0).sum(1)
    entropy = logz.squeeze(1) - weighted
    out = {"logp": logp, "entropy": entropy}
    if c["top"]:
        # value first, then the lower index: one whole number that orders both
        bits = (x + 0.0).view(torch.int32).long()
        bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        column = torch.arange(x.shape[1], device=x.device)
        key = (bits << 32) + (0x7FFFFFFF - column)
        index = 0x7FFFFFFF - (torch.topk(key, c["top"], dim=1).values & 0x7FFFFFFF)
        out["top_logp"], out["top_index"] = shifted.gather(1, index) - logz, index
    if c["train"]:
        g = torch.where(valid, s["dlogp"], 0.0).unsqueeze(1)
        logp_all = shifted - logz
        d = torch.where(p > 0, -p * (g + s["dentropy"].unsqueeze(1) * (logp_all + entropy.unsqueeze(1))), 0.0)
        out["dlogits"] = d.scatter_add_(1, target, g).to(t)
    return out


# -------------------------------------------------------------------------------- 64 bits, and work


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "linear":
        return _exact_linear(case, s)
    return _exact_norm(case, s) if case["op"] == "norm" else _exact_logprobs(case, s)


def _exact_linear(case, s):
    """The definition in FP64, its gradients by differentiation."""
    f = {k: v.double().requires_grad_(case["train"]) for k, v in s.items() if k in ("x", "w", "bias") and v is not None}
    z = torch.einsum("mk,nk->mn" if case["layout"] == "nk" else "mk,kn->mn", f["x"], f["w"])
    if "bias" in f:
        z = z + f["bias"]
    act = {"none": lambda v: v, "relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu,
           "gelu_tanh": lambda v: torch.nn.functional.gelu(v, approximate="tanh"),
           "silu": torch.nn.functional.silu}[case["act"]]
    y = act(z)
    if s["residual"] is not None:
        y = y + s["residual"].double()
    if not case["train"]:
        return {"y": y}
    names = [k for k in ("x", "w", "bias") if k in f]
    grads = dict(zip(names, torch.autograd.grad(y, [f[k] for k in names], s["dy"].double())))
    return {"y": y.detach(), "dx": grads["x"], "dw": grads["w"], "db": grads.get("bias")}


def _exact_norm(case, s):
    x, w, b = (s[k].double().requires_grad_(case["train"]) for k in ("x", "weight", "bias"))
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    y = (x - mean) / torch.sqrt(var + 1e-5) * w + b
    if not case["train"]:
        return {"y": y}
    dx, dw, db = torch.autograd.grad(y, [x, w, b], s["dy"].double())
    return {"y": y.detach(), "dx": dx, "dweight": dw, "dbias": db}


def _exact_logprobs(case, s):
    x = s["logits"].double()
    lse = torch.logsumexp(x, 1)
    at = s["tokens"].clamp(min=0)
    valid = s["tokens"] >= 0
    logp = torch.where(valid, x[torch.arange(len(at), device=x.device), at] - lse, 0.0)
    logq = x - lse[:, None]
    q = logq.exp()
    entropy = torch.special.entr(q).sum(1)
    out = {"logp": logp, "entropy": entropy}
    if case["top"]:
        out["top_logp"], out["top_index"] = torch.topk(logq, case["top"], dim=1).values, None
    if case["train"]:
        # d(log p_t)/dx = onehot - q;  dH/dx = -q log q - q H = entr(q) - q H
        g = torch.where(valid, s["dlogp"].double(), 0.0)[:, None]
        d = (torch.special.entr(q) - q * entropy[:, None]) * s["dentropy"].double()[:, None] - q * g
        d[torch.arange(len(at), device=x.device), at] += g[:, 0]
        out["dlogits"] = d
    return out


def work(case):
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        words = m * k + n * k + m * n * (2 if case["residual"] else 1) + (n if case["bias"] else 0)
        if case["train"]:          # dY in; dX, dW and db out
            words += m * n + m * k + n * k + (n if case["bias"] else 0)
        return {"bytes": 4 * words, "flops": 2 * m * n * k * (3 if case["train"] else 1)}
    e = TYPES[case["dtype"]].itemsize
    if case["op"] == "norm":
        r, c = case["rows"], case["cols"]
        nbytes = 2 * r * c * e + 2 * c * 4
        if case["train"]:          # dY in; dX and the two sums out
            nbytes += 2 * r * c * e + 2 * c * 4
        return {"bytes": nbytes, "flops": r * c * (20 if case["train"] else 8)}
    r, v = case["rows"], case["vocab"]
    nbytes = r * v * e + r * (8 + 4 + 4) + r * case["top"] * 12
    if case["train"]:              # the two gradients in, the logits' out
        nbytes += r * v * e + r * 8
    return {"bytes": nbytes, "flops": r * v * (16 if case["train"] else 6)}
