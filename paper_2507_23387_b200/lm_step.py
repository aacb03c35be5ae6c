"""A small next-token model trained and sampled through the library's language-model operators.

One residual block without attention, everything in FP32, every product on the three-product kernel:

    x  = E[token]                          rows of the embedding (a torch gather)
    n  = norm(x; g1, c1)                   sgemm_cube_layer_norm
    h  = gelu(n W1' + b1)                  sgemm_cube_linear, keeping Z = n W1' + b1
    y  = h W2' + b2 + x                    sgemm_cube_linear with the residual
    f  = norm(y; g2, c2)                   sgemm_cube_layer_norm
    l  = f H'                              sgemm_cube_linear
    logp, entropy of the next tokens       sgemm_cube_token_logprobs

The loss is -mean(logp) - entropy_weight * mean(entropy) over the rows whose next token is known
(negative: none).  `Model.gradients` walks the same list backwards through the `_backward` entry points;
`Model.step` adds plain gradient descent.  Every buffer is made once for the largest batch.  `Sampler` keeps the
weights packed and answers the most likely next tokens of a few sequences at a time.  `python -m` of this file
trains on a fixed random successor table and prints the loss, then what the sampler learned:

    python -m paper_2507_23387_b200.lm_step [--tokens 1024] [--width 512] [--hidden 2048] [--vocab 8192] [--steps 60]
"""
import argparse

import torch

from . import binding

NK, GELU = binding.WEIGHT_NK, binding.ACT_GELU


class Model:
    """Weights, gradients and the buffers of one training step of at most `tokens` rows."""

    def __init__(self, handle, tokens, width, hidden, vocab, seed=0):
        self.h, self.device = handle, torch.device("cuda", handle.device)
        g = torch.Generator(device=self.device).manual_seed(seed)

        def normal(rows, cols, scale):
            return torch.randn((rows, cols), generator=g, device=self.device).mul_(scale)

        def full(n, value):
            return torch.full((n,), value, device=self.device)

        self.weights = {
            "E": normal(vocab, width, 1.0), "H": normal(vocab, width, width ** -0.5),
            "W1": normal(hidden, width, width ** -0.5), "b1": full(hidden, 0.0),
            "W2": normal(width, hidden, hidden ** -0.5), "b2": full(width, 0.0),
            "g1": full(width, 1.0), "c1": full(width, 0.0), "g2": full(width, 1.0), "c2": full(width, 0.0),
        }
        self.grads = {k: torch.zeros_like(v) for k, v in self.weights.items()}

        def buffer(*shape):
            return torch.empty(shape, device=self.device)

        self.rows = {                                    # one row a token
            "x": buffer(tokens, width), "n": buffer(tokens, width), "y": buffer(tokens, width), "f": buffer(tokens, width),
            "z": buffer(tokens, hidden), "a": buffer(tokens, hidden), "l": buffer(tokens, vocab),
            "dx": buffer(tokens, width), "dy": buffer(tokens, width), "da": buffer(tokens, hidden),
            "mean1": buffer(tokens), "rstd1": buffer(tokens), "mean2": buffer(tokens), "rstd2": buffer(tokens),
            "logp": buffer(tokens), "entropy": buffer(tokens), "stats": buffer(tokens, 2),
        }

    def forward(self, tokens, targets):
        """Views of the buffers for these rows, filled up to logp, entropy and stats."""
        h, w = self.h, self.weights
        r = {k: v[:tokens.numel()] for k, v in self.rows.items()}
        torch.index_select(w["E"], 0, tokens, out=r["x"])
        h.sgemm_cube_layer_norm(r["x"], r["n"], w["g1"], w["c1"], mean=r["mean1"], rstd=r["rstd1"])
        h.sgemm_cube_linear(r["n"], w["W1"], r["a"], bias=w["b1"], activation=GELU, preact=r["z"], weight_layout=NK)
        h.sgemm_cube_linear(r["a"], w["W2"], r["y"], bias=w["b2"], residual=r["x"], weight_layout=NK)
        h.sgemm_cube_layer_norm(r["y"], r["f"], w["g2"], w["c2"], mean=r["mean2"], rstd=r["rstd2"])
        h.sgemm_cube_linear(r["f"], w["H"], r["l"], weight_layout=NK)
        h.sgemm_cube_token_logprobs(r["l"], targets, r["logp"], entropy=r["entropy"], stats=r["stats"])
        return r

    def gradients(self, tokens, targets, entropy_weight=0.0):
        """The loss (a tensor of one value); its gradients of all weights go to self.grads."""
        h, w, g = self.h, self.weights, self.grads
        r = self.forward(tokens, targets)
        known = (targets >= 0).float()
        share = known / known.sum().clamp(min=1.0)
        loss = -(share * (r["logp"] + entropy_weight * r["entropy"])).sum()
        h.sgemm_cube_token_logprobs_backward(r["l"], targets, r["stats"], r["l"], dlogp=-share, entropy=r["entropy"],
                                             dentropy=-entropy_weight * share)     # in the place of the logits
        h.sgemm_cube_linear_backward(r["l"], r["f"], w["H"], dX=r["dx"], dW=g["H"], weight_layout=NK)
        h.sgemm_cube_layer_norm_backward(r["dx"], r["y"], r["mean2"], r["rstd2"], r["dy"], w["g2"], g["g2"], g["c2"])
        h.sgemm_cube_linear_backward(r["dy"], r["a"], w["W2"], dX=r["da"], dW=g["W2"], dbias=g["b2"], weight_layout=NK)
        h.sgemm_cube_linear_backward(r["da"], r["n"], w["W1"], dX=r["dx"], dW=g["W1"], dbias=g["b1"], preact=r["z"],
                                     activation=GELU, weight_layout=NK)
        h.sgemm_cube_layer_norm_backward(r["dx"], r["x"], r["mean1"], r["rstd1"], r["dx"], w["g1"], g["g1"], g["c1"])
        r["dx"].add_(r["dy"])                                                      # the residual's path round the block
        g["E"].zero_().index_add_(0, tokens, r["dx"])
        return loss

    def step(self, tokens, targets, rate, entropy_weight=0.0):
        loss = self.gradients(tokens, targets, entropy_weight)
        for k, v in self.weights.items():
            v.sub_(self.grads[k], alpha=rate)
        return loss


class Sampler:
    """Next tokens of at most `sequences` sequences from a model's present weights, packed once."""

    def __init__(self, model, sequences, top=5):
        self.h, self.w, dev = model.h, model.weights, model.device
        self.packed = {}
        for k in ("W1", "W2", "H"):
            self.packed[k] = binding.PackedMatrix(*self.w[k].shape, device=dev)
            self.h.sgemm_cube_pack(self.w[k], self.packed[k])
        (vocab, width), hidden = self.w["H"].shape, self.w["b1"].numel()
        self.x, self.n = torch.empty((2, sequences, width), device=dev)
        self.a = torch.empty((sequences, hidden), device=dev)
        self.l = torch.empty((sequences, vocab), device=dev)
        self.none = torch.full((sequences,), -1, dtype=torch.int64, device=dev)
        self.logp = torch.empty(sequences, device=dev)
        self.top_logp = torch.empty((sequences, top), device=dev)
        self.top = torch.empty((sequences, top), dtype=torch.int64, device=dev)

    def next(self, tokens, temperature=1.0, allowed=None):
        """Log probabilities and indices of the most likely successors of each token; `allowed` is a mask over
        the vocabulary (a row with nothing allowed has log probabilities of -inf)."""
        h, w, p, s = self.h, self.w, self.packed, tokens.numel()
        x, n, a, l = self.x[:s], self.n[:s], self.a[:s], self.l[:s]
        torch.index_select(w["E"], 0, tokens, out=x)
        h.sgemm_cube_layer_norm(x, n, w["g1"], w["c1"])
        h.sgemm_cube_linear(n, p["W1"], a, bias=w["b1"], activation=GELU, weight_layout=NK)
        h.sgemm_cube_linear(a, p["W2"], x, bias=w["b2"], residual=x, weight_layout=NK)
        h.sgemm_cube_layer_norm(x, n, w["g2"], w["c2"])
        h.sgemm_cube_linear(n, p["H"], l, weight_layout=NK)
        if allowed is not None:
            l.masked_fill_(~allowed, float("-inf"))
        h.sgemm_cube_token_logprobs(l, self.none[:s], self.logp[:s], top_logp=self.top_logp[:s], top_index=self.top[:s],
                                    scale=1.0 / temperature)
        return self.top_logp[:s], self.top[:s]


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("tokens", 1024), ("width", 512), ("hidden", 2048), ("vocab", 8192), ("steps", 60)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--rate", type=float, default=4.0)
    args = ap.parse_args()
    h = binding.Handle(0)
    model = Model(h, args.tokens, args.width, args.hidden, args.vocab)
    gen = torch.Generator(device=model.device).manual_seed(1)
    successor = torch.randperm(args.vocab, generator=gen, device=model.device)
    tokens = torch.randint(0, args.vocab, (args.tokens,), generator=gen, device=model.device)
    for i in range(args.steps):
        loss = model.step(tokens, successor[tokens], args.rate)
        if i % 10 == 0 or i == args.steps - 1:
            print("step %4d  loss %.4f" % (i, float(loss)))
    logp, top = Sampler(model, 8).next(tokens[:8])
    print("token  successor  most likely (probability)")
    for t, s, row, lp in zip(tokens[:8].tolist(), successor[tokens[:8]].tolist(), top.tolist(), logp.exp().tolist()):
        print("%5d  %9d  %s" % (t, s, "  ".join("%d (%.3f)" % p for p in zip(row[:3], lp))))
    status, detail = h.sgemm_cube_check()
    h.destroy()
    return 0 if status == 0 else 1


if __name__ == "__main__":
    raise SystemExit(main())
