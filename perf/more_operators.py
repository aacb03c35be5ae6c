"""Cases, inputs and plain forms of what stands at the two ends of a language model's training step and behind it.

  embedding      rows of a table times a scale; the gradient of the table by sorted tokens
  loss           softmax cross entropy of X W + b over a large vocabulary without the logits; gradients of X, W and b
  orthogonalize  an update brought near the closest matrix with orthonormal rows (or columns) by Newton-Schulz
                 products, added to the weight that it updates

`own` false: plain torch operations in 32 bits, rounded once at the end.  `own` true: the library's entry
points, as a program calls them.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
QUINTIC = (3.4445, -4.7750, 2.0315)      # X <- a X + b (X X') X + c (X X')^2 X
EPS = 1e-7
_handles = []


def listed():
    return [
        # the next tokens of eight sequences enter the model: latency decides
        _embedding("embedding_decode", 8, 4096, 131072, "bf16"),
        # a batch of prompts enters the model
        _embedding("embedding_prompt", 16384, 4096, 131072, "bf16"),
        # 16-bit training with odd sizes: rows that start on odd addresses, frequent tokens in a third of the rows
        _embedding("embedding_train_ragged", 30001, 1001, 50001, "f16", train=True),
        # FP32 training, a large table of which few rows are met
        _embedding("embedding_train", 8192, 4096, 131072, "f32", train=True),
        # how likely four continuations are, the head packed once: its bytes decide
        _loss("loss_score_few", 4, 50001, 1024, packed=True),
        # scoring a text, every size odd, weight stored inputs x outputs
        _loss("loss_score_ragged", 1000, 50001, 1001, layout="kn"),
        # training step of a small model (the sizes that the example model trains with)
        _loss("loss_train_small", 1024, 8192, 512, train=True),
        # training step over a large vocabulary
        _loss("loss_train_large", 4096, 131072, 4096, train=True),
        # a small layer's update: a chain of small products
        _orthogonalize("orthogonalize_small", 128, 384, "f32"),
        # the example model's up-projection, outputs x inputs, taller than wide, added to the weight
        _orthogonalize("orthogonalize_tall", 2048, 512, "f32", residual=True),
        # a 16-bit gradient, every size odd
        _orthogonalize("orthogonalize_ragged", 1001, 2049, "bf16"),
        # a large model's projection, added to the weight
        _orthogonalize("orthogonalize_large", 4096, 16384, "f32", residual=True),
    ]


def _embedding(name, rows, cols, vocab, dtype, train=False):
    return {"name": name, "op": "embedding", "rows": rows, "cols": cols, "vocab": vocab, "dtype": dtype,
            "scale": 1.0 if train else math.sqrt(cols), "train": train}


def _loss(name, m, n, k, layout="nk", bias=True, packed=False, train=False):
    return {"name": name, "op": "loss", "m": m, "n": n, "k": k, "layout": layout, "bias": bias, "packed": packed,
            "train": train}


def _orthogonalize(name, rows, cols, dtype, steps=5, residual=False):
    return {"name": name, "op": "orthogonalize", "rows": rows, "cols": cols, "dtype": dtype, "steps": steps,
            "scale": -0.02 if residual else 1.0, "beta": 0.999, "residual": residual}


def _log_size(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm; three in four are left as they fall (odd
    ones among them), the others are made multiples of 64."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))
    if v >= 64 and rng.random() < 0.25:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["embedding", "loss", "loss", "orthogonalize", "orthogonalize"])
    if op == "embedding":
        cols = _log_size(rng, 128, 8192)
        vocab = min(_log_size(rng, 4096, 200000), (1 << 29) // cols)
        c = _embedding("", _log_size(rng, 1, 32768), cols, vocab, rng.choice(["f32", "f16", "bf16"]), train=rng.random() < 0.6)
    elif op == "loss":
        train = rng.random() < 0.5
        c = _loss("", _log_size(rng, 1, 4096), _log_size(rng, 4096, 131072), _log_size(rng, 128, 4096),
                  layout=rng.choice(["nk", "kn"]), bias=rng.random() < 0.7, packed=not train and rng.random() < 0.4, train=train)
        c["m"] = max(1, min(c["m"], (1 << 39) // (c["n"] * c["k"])))
    else:
        short = _log_size(rng, 32, 4096)
        long = max(short, _log_size(rng, 64, 16384))
        rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
        c = _orthogonalize("", rows, cols, rng.choice(["f32", "f32", "bf16", "f16"]), steps=rng.choice([3, 5, 5]),
                           residual=rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------ inputs


def _inputs(case, seed):
    """What both sides and the 64-bit form start from, made from the seed alone."""
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    if case["op"] == "embedding":
        r, c, v, t = case["rows"], case["cols"], case["vocab"], TYPES[case["dtype"]]
        table = torch.empty(v, c, dtype=t, device=DEV).normal_(0.0, 0.02, generator=g)
        # few tokens make up much of a text: token k has the probability ((k + 1)^1/4 - k^1/4) / vocab^1/4
        tokens = (torch.rand(r, generator=g, device=DEV, dtype=torch.float64) ** 4 * v).long().clamp_(max=v - 1)
        if r >= 16:
            tokens[torch.rand(r, generator=g, device=DEV) < 0.05] = -1             # padding
        s = {"table": table, "tokens": tokens}
        if case["train"]:
            s["dy"] = normal(r, c).mul_(1e-2).to(t)
    elif case["op"] == "loss":
        m, n, k = case["m"], case["n"], case["k"]
        s = {"w": normal(n, k) if case["layout"] == "nk" else normal(k, n)}
        s["w"].mul_(2.0 * k ** -0.5)
        s["bias"] = normal(n).mul_(0.5) if case["bias"] else None
        target = torch.randint(0, n, (m,), generator=g, device=DEV)
        # normalised features that point towards the target's weights, more or less
        rows = s["w"][target] if case["layout"] == "nk" else s["w"][:, target].t()
        s["x"] = normal(m, k).add_(rows * torch.rand(m, 1, generator=g, device=DEV).mul_(2.5))
        if m >= 16:
            target[torch.rand(m, generator=g, device=DEV) < 0.1] = -1               # positions without a target
        s["targets"] = target
        if case["train"]:                                                          # the mean loss over the others
            s["dloss"] = (target >= 0).float().div_((target >= 0).sum().clamp(min=1))
    else:
        r, c = case["rows"], case["cols"]
        u = normal(r, c).mul_(0.1)
        u.addmm_(normal(r, 16), normal(16, c), alpha=0.25)                         # a gradient has few strong directions
        s = {"g": u.mul_(1e-3).to(TYPES[case["dtype"]]), "w": normal(r, c).mul_(c ** -0.5) if case["residual"] else None}
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
    s["h"] = h
    f32 = dict(dtype=torch.float32, device=DEV)
    if case["op"] == "embedding":
        s["y"] = torch.empty(case["rows"], case["cols"], dtype=s["table"].dtype, device=DEV)
        if case["train"]:
            s["dtable"] = torch.empty(case["vocab"], case["cols"], **f32)
    elif case["op"] == "loss":
        s["layout"] = binding.WEIGHT_NK if case["layout"] == "nk" else binding.WEIGHT_KN
        s["loss"], s["lse"] = torch.empty(case["m"], **f32), torch.empty(case["m"], **f32)
        if case["packed"]:        # a server lays its weights out once, when it loads them
            s["wp"] = binding.PackedMatrix(*s["w"].shape)
            h.sgemm_cube_pack(s["w"], s["wp"])
        if case["train"]:
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
            s["db"] = torch.empty(case["n"], **f32) if case["bias"] else None
    else:
        s["o"] = torch.empty(case["rows"], case["cols"], **f32)
    return s


# ---------------------------------------------------------------------------------------- one pass


def run(state):
    op = state["case"]["op"]
    if own:
        return {"embedding": _own_embedding, "loss": _own_loss, "orthogonalize": _own_orthogonalize}[op](state)
    return {"embedding": _plain_embedding, "loss": _plain_loss, "orthogonalize": _plain_orthogonalize}[op](state)


def _own_embedding(s):
    h, c = s["h"], s["case"]
    h.sgemm_cube_embedding(s["tokens"], s["table"], s["y"], scale=c["scale"])
    if not c["train"]:
        return {"y": s["y"]}
    h.sgemm_cube_embedding_backward(s["tokens"], s["dy"], s["dtable"], scale=c["scale"])
    return {"y": s["y"], "dtable": s["dtable"]}


def _own_loss(s):
    h, c = s["h"], s["case"]
    if not c["train"]:
        h.sgemm_cube_cross_entropy(s["x"], s.get("wp", s["w"]), s["targets"], s["loss"], bias=s["bias"], lse=s["lse"],
                                   weight_layout=s["layout"])
        return {"loss": s["loss"], "lse": s["lse"]}
    h.sgemm_cube_cross_entropy_backward(s["x"], s["w"], s["targets"], s["dloss"], dX=s["dx"], dW=s["dw"], dbias=s["db"],
                                        bias=s["bias"], loss=s["loss"], lse=s["lse"], weight_layout=s["layout"])
    return {"loss": s["loss"], "lse": s["lse"], "dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_orthogonalize(s):
    c = s["case"]
    s["h"].sgemm_cube_orthogonalize(s["g"], s["o"], steps=c["steps"], coefficients=QUINTIC, eps=EPS, scale=c["scale"],
                                    residual=s["w"], beta=c["beta"])
    return {"o": s["o"]}


def _plain_embedding(s):
    c, t = s["case"], s["table"].dtype
    known = s["tokens"] >= 0
    at = s["tokens"].clamp(min=0)
    y = torch.where(known[:, None], s["table"][at].float() * c["scale"], 0.0).to(t)
    if not c["train"]:
        return {"y": y}
    dy = torch.where(known[:, None], s["dy"].float() * c["scale"], 0.0)
    return {"y": y, "dtable": torch.zeros(c["vocab"], c["cols"], device=dy.device).index_add_(0, at, dy)}


def _plain_loss(s):
    c = s["case"]
    w = s["w"].t() if c["layout"] == "nk" else s["w"]                # inputs x outputs
    z = s["x"] @ w
    if s["bias"] is not None:
        z = z + s["bias"]
    known = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    z = z - top
    log_sum = torch.log(torch.exp(z).sum(1, keepdim=True))
    out = {"loss": torch.where(known, (log_sum - z.gather(1, at))[:, 0], 0.0), "lse": (top + log_sum)[:, 0]}
    if not c["train"]:
        return out
    g = torch.where(known, s["dloss"], 0.0)[:, None]
    dz = torch.exp(z - log_sum) * g
    dz.scatter_add_(1, at, -g)
    out["dx"] = dz @ w.t()
    out["dw"] = dz.t() @ s["x"] if c["layout"] == "nk" else s["x"].t() @ dz
    out["db"] = dz.sum(0) if s["bias"] is not None else None
    return out


def _plain_orthogonalize(s):
    case = s["case"]
    a, b, c = QUINTIC
    x = s["g"].float()
    x = x / (x.double().square().sum().sqrt() + EPS).float()
    tall = case["rows"] > case["cols"]
    if tall:
        x = x.t()
    for _ in range(case["steps"]):
        gram = x @ x.t()
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    o = (x.t() if tall else x) * case["scale"]
    return {"o": o + case["beta"] * s["w"] if case["residual"] else o}


# -------------------------------------------------------------------------------- 64 bits, and work


def exact(case, seed):
    s = _inputs(case, seed)
    return {"embedding": _exact_embedding, "loss": _exact_loss, "orthogonalize": _exact_orthogonalize}[case["op"]](case, s)


def _exact_embedding(case, s):
    """Every token's row by itself: the runs of equal tokens in sorted order, summed as differences of nothing but
    their own rows."""
    keep = torch.nonzero(s["tokens"] >= 0)[:, 0]
    t = s["tokens"][keep]
    y = torch.zeros(case["rows"], case["cols"], dtype=torch.float64, device=t.device)
    y[keep] = torch.index_select(s["table"], 0, t).double() * case["scale"]
    if not case["train"]:
        return {"y": y}
    order = torch.argsort(t, stable=True)
    rows, lengths = torch.unique_consecutive(t[order], return_counts=True)
    sums = torch.segment_reduce(s["dy"][keep][order].double(), "sum", lengths=lengths, axis=0)
    d = torch.zeros(case["vocab"], case["cols"], dtype=torch.float64, device=t.device)
    d[rows] = sums * case["scale"]
    return {"y": y, "dtable": d}


def _exact_loss(case, s):
    """The definition in FP64, its gradients through the softmax's."""
    x, w = s["x"].double(), s["w"].double()
    z = torch.einsum("mk,nk->mn" if case["layout"] == "nk" else "mk,kn->mn", x, w)
    if s["bias"] is not None:
        z += s["bias"].double()
    lse = torch.logsumexp(z, 1)
    row = torch.nonzero(s["targets"] >= 0)[:, 0]
    t = s["targets"][row]
    loss = torch.zeros_like(lse)
    loss[row] = lse[row] - z[row, t]
    out = {"loss": loss, "lse": lse}
    if case["train"]:
        d = z.sub_(lse[:, None]).exp_()
        d[row, t] -= 1.0
        weight = torch.zeros_like(lse)
        weight[row] = s["dloss"].double()[row]
        d *= weight[:, None]
        out["dx"] = torch.einsum("mn,nk->mk" if case["layout"] == "nk" else "mn,kn->mk", d, w)
        out["dw"] = torch.einsum("mn,mk->nk" if case["layout"] == "nk" else "mn,mk->kn", d, x)
        out["db"] = d.sum(0) if s["bias"] is not None else None
    return out


def _exact_orthogonalize(case, s):
    """The polynomial from the other side: X <- X (a + b H + c H^2) with H = X' X on the shorter dimension."""
    a, b, c = QUINTIC
    x = s["g"].double()
    wide = case["cols"] > case["rows"]
    if wide:
        x = x.t().contiguous()
    x = x / (torch.linalg.vector_norm(x) + EPS)
    eye = torch.eye(x.shape[1], dtype=torch.float64, device=x.device)
    for _ in range(case["steps"]):
        h = x.t() @ x
        x = x @ torch.addmm(a * eye, h, b * eye + c * h)
    o = case["scale"] * (x.t() if wide else x)
    return {"o": o + case["beta"] * s["w"].double() if case["residual"] else o}


def work(case):
    if case["op"] == "embedding":
        r, c, v, e = case["rows"], case["cols"], case["vocab"], TYPES[case["dtype"]].itemsize
        k = torch.arange(v + 1, dtype=torch.float64).div_(v).pow_(0.25)
        distinct = float((1.0 - (1.0 - k.diff()).pow_(r)).sum())      # rows of the table that are met, on average
        nbytes = r * 8 + distinct * c * e + r * c * e
        if case["train"]:              # dY in; the table's gradient out, zeros among it
            nbytes += r * c * e + v * c * 4
        return {"bytes": int(nbytes), "flops": r * c * (2 if case["train"] else 1)}
    if case["op"] == "loss":
        m, n, k = case["m"], case["n"], case["k"]
        words = m * k + n * k + (n if case["bias"] else 0) + 4 * m
        if case["train"]:              # the loss' gradient in; dX, dW and db out
            words += m + m * k + n * k + (n if case["bias"] else 0)
        return {"bytes": 4 * words, "flops": 2 * m * n * k * (3 if case["train"] else 1)}
    short, long = sorted((case["rows"], case["cols"]))
    nbytes = short * long * (TYPES[case["dtype"]].itemsize + 4 + (4 if case["residual"] else 0))
    # X X' and its square are symmetric: half of each
    flops = case["steps"] * (short * (short + 1) * long + short * short * (short + 1) + 2 * short * short * long)
    return {"bytes": nbytes, "flops": flops}
