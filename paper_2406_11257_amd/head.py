"""The output projection of a reconstructed checkpoint, answered with in 4 bits, scored and trained.

What the compression of a checkpoint costs shows in the log probabilities of its answers.  MxHead holds the projection
(vocabulary x width) in microscaled 4-bit floating point and takes hidden states to the log probabilities of given tokens,
and the gradient of those back to the hidden states and the weights.  Run as a command,

    python -m paper_2406_11257_amd.head [--config 0] [--tokens 256]

compresses the output embedding of one of the synthetic checkpoints (see synth.py), reconstructs it, and compares the
answers of the reconstruction with those of the weights it stands for.
"""
from __future__ import annotations

import contextlib

from . import binding as X


class MxHead:
    """logits = MX(hidden) MX(weight)^T.  weight: a (vocabulary x width) float32, float16 or bfloat16 tensor on the context's
    GPU, read once; with `train` it is kept quantised down its columns too, for the gradient of the hidden states.  Calls may
    be made from any stream: the context's waits for it, and it for the context's.  Results belong to the stream that a call
    is made from, as torch's own do; `codes` and `codes_t` to the context's, on which all calls read them."""

    def __init__(self, ctx: X.Context, weight, train: bool = False):
        self.ctx, (self.vocab, self.width) = ctx, weight.shape
        with self._on_stream(weight):
            self.codes = X.mx_empty(self.vocab, self.width, weight.device)
            self.codes_t = X.mx_empty(self.width, self.vocab, weight.device) if train else (None, None)
            ctx.excp_mx_quantize(weight, *self.codes, *self.codes_t)

    @contextlib.contextmanager
    def _on_stream(self, *read):
        """The context's stream as the current one, for work on the tensors `read` (None: none) and on what the caller's stream
        has allocated.  That memory goes back to the caller's stream when it is dropped, which waits for the context's, so
        that no other caller is given it while either may still use it.  (What is allocated on the context's stream inside
        goes back to that one, and is not for the caller.)"""
        import torch
        own, caller = self.ctx._stream, torch.cuda.current_stream(self.ctx.device)
        if own == caller:
            yield
            return
        own.wait_stream(caller)
        for t in read:
            if t is not None and t.is_cuda:
                t.record_stream(own)                         # whichever stream it was allocated on
        try:
            with torch.cuda.stream(own):
                yield
        finally:
            caller.wait_stream(own)                          # a refusal, too, may leave work that was queued before it

    def score(self, hidden, targets, ntop: int = 0) -> dict:
        """hidden: (tokens x width); targets: int64, -1 for a token without one.  Returns the logits (float32), the targets'
        log probabilities, the entropies, the log-sum-exps in two parts, and the ntop first alternatives of every token."""
        import torch
        tokens, device = hidden.shape[0], hidden.device

        def f32(*shape):
            return torch.empty(*shape, dtype=torch.float32, device=device)
        s = {"logits": f32(tokens, self.vocab), "logprob": f32(tokens), "entropy": f32(tokens), "lse": f32(tokens, 2),
             "top_logprob": f32(tokens, ntop) if ntop else None,
             "top_ids": torch.empty(tokens, ntop, dtype=torch.int64, device=device) if ntop else None}
        with self._on_stream(hidden, targets):
            self.ctx.excp_mx_linear(hidden, *self.codes, s["logits"], *X.mx_empty(tokens, self.width, device))
            self.ctx.excp_token_logprobs(s["logits"], targets, s["logprob"], s["entropy"], s["lse"], s["top_logprob"], s["top_ids"])
        return s

    def gradients(self, hidden, targets, scored: dict, g_logprob, g_entropy=None, g_top=None):
        """Of sum(g_logprob logprob) + sum(g_entropy entropy) + sum(g_top top_logprob): (over hidden, over the weight), both
        float32, from 4-bit products of what is quantised along and down.  The logits of `scored` become their gradient, so
        that it serves one call; another is refused."""
        import torch
        if self.codes_t[0] is None:
            raise ValueError("this head was not made to train")
        d = scored["logits"]
        if getattr(d, "holds_gradient", False):
            raise ValueError("the logits of these scores have become their gradient: score the hidden states again")
        if hidden.shape != (d.shape[0], self.width):
            raise ValueError("hidden is not of the shape that was scored")
        tokens, device, ctx = hidden.shape[0], hidden.device, self.ctx
        dhidden = torch.empty(tokens, self.width, dtype=torch.float32, device=device)
        dweight = torch.empty(self.vocab, self.width, dtype=torch.float32, device=device)
        with self._on_stream(hidden, targets, d, scored["lse"], scored["entropy"], scored["top_ids"], g_logprob, g_entropy, g_top):
            along, down = X.mx_empty(tokens, self.vocab, device), X.mx_empty(self.vocab, tokens, device)
            hidden_down = X.mx_empty(self.width, tokens, device)
            ctx.excp_mx_quantize(hidden, None, None, *hidden_down)
            ctx.excp_token_logprobs_backward(d, targets, scored["lse"], scored["entropy"], scored["top_ids"], g_logprob,
                                             g_entropy, g_top, d)
            d.holds_gradient = True
            ctx.excp_mx_quantize(d, *along, *down)
            ctx.excp_mx_matmul(*along, *self.codes_t, self.vocab, dhidden)
            ctx.excp_mx_matmul(*down, *hidden_down, tokens, dweight)
        return dhidden, dweight


def compare(config: int = 0, tokens: int = 256, ntop: int = 8) -> dict:
    """Answers of a synthetic checkpoint's output embedding before and after compression: the last tensor of that kind is
    compressed and reconstructed, and hidden states near the embeddings of random tokens are scored with both."""
    import torch
    from . import synth
    device = torch.device("cuda", torch.cuda.current_device())
    cfg = synth.config(config)
    idx, spec = [(i, t) for i, t in enumerate(cfg.tensors) if t.kind == "embed"][-1]
    vocab = {0: 50304, 1: 50304, 2: 50304, 3: 32000, 4: 50304}[config]
    width = spec.n // vocab
    Wp, W, m, v = synth.torch_draw_tensor(config, idx, spec, device)
    ctx = X.Context(spec.n, device=device)
    try:
        blob = torch.empty(X.excp_blob_bound(spec.n, synth.NBITS), dtype=torch.uint8, device=device)
        W_hat = torch.empty_like(W)
        _, nbytes, _ = ctx.excp_compress_step(Wp, W, m, v, blob, synth.ALPHA, synth.BETA, synth.NBITS, synth.LLOYD_ITERS)
        ctx.excp_decompress_step(Wp, blob, nbytes, W_hat)
        g = torch.Generator(device=device)
        g.manual_seed(synth.BASE_SEED)
        targets = torch.randint(0, vocab, (tokens,), device=device, generator=g)
        weight = W.view(vocab, width)
        hidden = weight[targets] * (12.0 / (0.02 ** 2 * width)) + torch.empty(tokens, width, device=device).normal_(0, 4.0, generator=g)
        out = {}
        for name, w in (("trained", weight), ("reconstructed", W_hat.view(vocab, width))):
            out[name] = MxHead(ctx, w).score(hidden, targets, ntop)
        torch.cuda.synchronize()
    finally:
        ctx.close()
    a, b = out["trained"], out["reconstructed"]
    return {"tensor": spec.name, "compressed": 12 * spec.n / nbytes, "logprob": (float(a["logprob"].mean()), float(b["logprob"].mean())),
            "entropy": (float(a["entropy"].mean()), float(b["entropy"].mean())),
            "largest_change": float((a["logprob"] - b["logprob"]).abs().max()),
            "same_first": float((a["top_ids"][:, 0] == b["top_ids"][:, 0]).float().mean())}


def main() -> None:
    import argparse
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--config", type=int, default=0, choices=(0, 1, 2, 3), help="synthetic checkpoint (see synth.py)")
    ap.add_argument("--tokens", type=int, default=256)
    a = ap.parse_args()
    r = compare(a.config, a.tokens)
    print(f"{r['tensor']} ({r['compressed']:.1f} times smaller with its moments), {a.tokens} tokens, 4-bit products\n"
          f"  mean log probability  trained {r['logprob'][0]:.4f}  reconstructed {r['logprob'][1]:.4f}  largest change {r['largest_change']:.4f}\n"
          f"  mean entropy          trained {r['entropy'][0]:.4f}  reconstructed {r['entropy'][1]:.4f}\n"
          f"  same first alternative for {100 * r['same_first']:.1f} % of the tokens")


if __name__ == "__main__":
    main()
