"""A small next-token model trained and sampled through the library's language-model operators.

One residual block without attention, everything in FP32, every product on the three-product kernel:

    x  = E[token]                          sgemm_cube_embedding
    n  = norm(x; g1, c1)                   sgemm_cube_layer_norm
    h  = gelu(n W1' + b1)                  sgemm_cube_linear, keeping Z = n W1' + b1
    y  = h W2' + b2 + x                    sgemm_cube_linear with the residual
    f  = norm(y; g2, c2)                   sgemm_cube_layer_norm
    l  = f H'                              sgemm_cube_linear
    logp, entropy of the next tokens       sgemm_cube_token_logprobs

The loss is -mean(logp) - entropy_weight * mean(entropy) over the rows whose next token is known
(negative: none).  `Model.gradients` walks the same list backwards through the `_backward` entry points;
`Model.step` adds plain gradient descent.  Every buffer is made once for the largest batch.  A model with keep_logits=False
keeps no l: the last two lines and their gradients are one call, sgemm_cube_cross_entropy_backward (no entropy then), whose workspace
holds the logits of a piece of the rows and the words of their gradient (8 bytes a logit, 2 GiB at the most).  `Model.loss` is
sgemm_cube_cross_entropy, which keeps logits of few rows only.  With orthogonal=... the step orthogonalises the updates of W1 and W2
(sgemm_cube_orthogonalize, into the weight).  `Sampler` keeps the
weights packed and answers the most likely next tokens of a few sequences at a time.  `python -m` of this file
trains on a fixed random successor table and prints the loss, then what the sampler learned:

    python -m paper_2507_23387_b200.lm_step [--tokens 1024] [--width 512] [--hidden 2048] [--vocab 8192] [--steps 60]
                                            [--no-logits] [--orthogonal 0.02]
"""
import argparse

import torch

from . import binding

NK, GELU = binding.WEIGHT_NK, binding.ACT_GELU


def _indices(tokens):
    """Tokens as the library reads them: 64 bits, next to each other (a view or a 32-bit tensor is copied)."""
    return tokens.long().contiguous()


class Model:
    """Weights, gradients and the buffers of one training step of at most `tokens` rows."""

    def __init__(self, handle, tokens, width, hidden, vocab, seed=0, keep_logits=True):
        self.keep_logits = keep_logits
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
            "z": buffer(tokens, hidden), "a": buffer(tokens, hidden),
            "dx": buffer(tokens, width), "dy": buffer(tokens, width), "da": buffer(tokens, hidden),
            "mean1": buffer(tokens), "rstd1": buffer(tokens), "mean2": buffer(tokens), "rstd2": buffer(tokens),
            "logp": buffer(tokens), "entropy": buffer(tokens), "stats": buffer(tokens, 2),
        }
        if keep_logits:
            self.rows["l"] = buffer(tokens, vocab)

    def features(self, tokens):
        """Views of the buffers for these rows, filled up to f."""
        h, w = self.h, self.weights
        r = {k: v[:tokens.numel()] for k, v in self.rows.items()}
        h.sgemm_cube_embedding(_indices(tokens), w["E"], r["x"])
        h.sgemm_cube_layer_norm(r["x"], r["n"], w["g1"], w["c1"], mean=r["mean1"], rstd=r["rstd1"])
        h.sgemm_cube_linear(r["n"], w["W1"], r["a"], bias=w["b1"], activation=GELU, preact=r["z"], weight_layout=NK)
        h.sgemm_cube_linear(r["a"], w["W2"], r["y"], bias=w["b2"], residual=r["x"], weight_layout=NK)
        h.sgemm_cube_layer_norm(r["y"], r["f"], w["g2"], w["c2"], mean=r["mean2"], rstd=r["rstd2"])
        return r

    def forward(self, tokens, targets):
        """The same up to logp, entropy and stats."""
        h, w, r = self.h, self.weights, self.features(tokens)
        h.sgemm_cube_linear(r["f"], w["H"], r["l"], weight_layout=NK)
        h.sgemm_cube_token_logprobs(r["l"], targets, r["logp"], entropy=r["entropy"], stats=r["stats"])
        return r

    def loss(self, tokens, targets):
        """The mean of -logp over the known targets (a tensor of one value), without logits or gradients."""
        r, known = self.features(tokens), (targets >= 0).float()
        self.h.sgemm_cube_cross_entropy(r["f"], self.weights["H"], targets, r["logp"], weight_layout=NK)
        return r["logp"].sum() / known.sum().clamp(min=1.0)

    def gradients(self, tokens, targets, entropy_weight=0.0):
        """The loss (a tensor of one value); its gradients of all weights go to self.grads."""
        h, w, g = self.h, self.weights, self.grads
        known = (targets >= 0).float()
        share = known / known.sum().clamp(min=1.0)
        if self.keep_logits:
            r = self.forward(tokens, targets)
            loss = -(share * (r["logp"] + entropy_weight * r["entropy"])).sum()
            h.sgemm_cube_token_logprobs_backward(r["l"], targets, r["stats"], r["l"], dlogp=-share, entropy=r["entropy"],
                                                 dentropy=-entropy_weight * share)     # in the place of the logits
            h.sgemm_cube_linear_backward(r["l"], r["f"], w["H"], dX=r["dx"], dW=g["H"], weight_layout=NK)
        else:
            assert entropy_weight == 0.0, "the entropy needs the logits"
            r = self.features(tokens)
            h.sgemm_cube_cross_entropy_backward(r["f"], w["H"], targets, share, dX=r["dx"], dW=g["H"], loss=r["logp"],
                                                weight_layout=NK)
            loss = (share * r["logp"]).sum()
        h.sgemm_cube_layer_norm_backward(r["dx"], r["y"], r["mean2"], r["rstd2"], r["dy"], w["g2"], g["g2"], g["c2"])
        h.sgemm_cube_linear_backward(r["dy"], r["a"], w["W2"], dX=r["da"], dW=g["W2"], dbias=g["b2"], weight_layout=NK)
        h.sgemm_cube_linear_backward(r["da"], r["n"], w["W1"], dX=r["dx"], dW=g["W1"], dbias=g["b1"], preact=r["z"],
                                     activation=GELU, weight_layout=NK)
        h.sgemm_cube_layer_norm_backward(r["dx"], r["x"], r["mean1"], r["rstd1"], r["dx"], w["g1"], g["g1"], g["c1"])
        r["dx"].add_(r["dy"])                                                      # the residual's path round the block
        h.sgemm_cube_embedding_backward(_indices(tokens), r["dx"], g["E"])
        return loss

    def step(self, tokens, targets, rate, entropy_weight=0.0, orthogonal=0.0, decay=0.0):
        """One step of gradient descent; with `orthogonal` > 0 the updates of W1 and W2 are that rate times the
        orthogonalised gradient, behind a decay of the weight."""
        loss = self.gradients(tokens, targets, entropy_weight)
        for k, v in self.weights.items():
            if orthogonal > 0.0 and k in ("W1", "W2"):
                # singular values of about one, so entries of about rows^-1/2 times this where rows > columns
                scale = orthogonal * max(1.0, v.shape[0] / v.shape[1]) ** 0.5
                self.h.sgemm_cube_orthogonalize(self.grads[k], v, scale=-scale, residual=v, beta=1.0 - orthogonal * decay)
            else:
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
        h.sgemm_cube_embedding(_indices(tokens), w["E"], x)
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
    ap.add_argument("--no-logits", action="store_true", help="the loss and its gradients in one call, no matrix of logits in the model")
    ap.add_argument("--orthogonal", type=float, default=0.0, help="rate of orthogonalised updates of W1 and W2")
    args = ap.parse_args()
    h = binding.Handle(0)
    model = Model(h, args.tokens, args.width, args.hidden, args.vocab, keep_logits=not args.no_logits)
    gen = torch.Generator(device=model.device).manual_seed(1)
    successor = torch.randperm(args.vocab, generator=gen, device=model.device)
    tokens = torch.randint(0, args.vocab, (args.tokens,), generator=gen, device=model.device)
    for i in range(args.steps):
        loss = model.step(tokens, successor[tokens], args.rate, orthogonal=args.orthogonal)
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
