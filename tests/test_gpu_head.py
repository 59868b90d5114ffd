"""A reconstructed output projection answered with, scored and trained in 4 bits: the operators together, against the
oracle's reconstruction and plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import oracle as O
import paper_2406_11257_amd as X
from ops_util import f64, gradient_reference, mx_reference, mx_values, scores_reference
from paper_2406_11257_amd import head, synth

pytestmark = pytest.mark.gpu


def mx(a):
    return mx_values(*mx_reference(a), a.shape[1])


@pytest.mark.parametrize("tokens", [1, 16, 45])
def test_from_blob_to_log_probabilities_and_back(tokens):
    vocab, width, ntop = 517, 96, 5
    spec = synth.TensorSpec("embed_out.weight", vocab * width, "embed")
    Wp, W, m, v = synth.draw_tensor(0, 9, spec)
    blob = O.compress_step(Wp, W, m, v, synth.ALPHA, synth.BETA, synth.NBITS, synth.LLOYD_ITERS).blob
    W_ref, _, _ = O.decompress_step(Wp, blob)
    ctx = X.Context(spec.n)
    W_hat = torch.empty(spec.n, device="cuda")
    dev = torch.from_numpy(np.frombuffer(blob, dtype=np.uint8).copy()).cuda()
    ctx.excp_decompress_step(torch.from_numpy(Wp).cuda(), dev, len(blob), W_hat)
    g = np.random.default_rng(7)
    hidden = (g.standard_normal((tokens, width)) * 6.0).astype(np.float32)
    targets = g.integers(0, vocab, tokens)
    targets[tokens // 2] = -1 if tokens > 1 else targets[0]
    h, t = torch.from_numpy(hidden).cuda(), torch.from_numpy(targets).cuda()
    hd = head.MxHead(ctx, W_hat.view(vocab, width), train=True)
    s = hd.score(h, t, ntop)
    # the weights are the oracle's bit for bit, so the quantised ones are; logits are sums of exact products
    w = mx(W_ref.astype(np.float64).reshape(vocab, width))
    logits = mx(hidden.astype(np.float64)) @ w.T
    assert (np.abs(f64(s["logits"]) - logits) <= 2.0 ** -18 * (np.abs(mx(hidden.astype(np.float64))) @ np.abs(w).T)).all()
    x = f64(s["logits"])
    lse, lp, ent, top, ids = scores_reference(x, targets, ntop)
    for name, ref in (("logprob", lp), ("entropy", ent), ("top_logprob", top)):
        assert np.abs(f64(s[name]) - ref).max() < 2e-5, name
    assert np.array_equal(s["top_ids"].cpu().numpy(), ids)
    gl, ge, gt = g.standard_normal(tokens), 0.1 * g.standard_normal(tokens), g.standard_normal((tokens, ntop))
    gl, ge, gt = (a.astype(np.float32) for a in (gl, ge, gt))
    dh, dw = hd.gradients(h, t, s, *[torch.from_numpy(a).cuda() for a in (gl, ge, gt)])
    d = gradient_reference(x, targets, ids, gl, ge, gt)
    got = f64(s["logits"])
    assert np.abs(got - d).max() < 1e-4
    # the products of what the gradient's own values come to in 4 bits (an element beside a threshold may go either way)
    want_h, want_w = mx(got) @ mx(W_ref.astype(np.float64).reshape(vocab, width).T).T, mx(got.T) @ mx(hidden.astype(np.float64).T).T
    for a, b, c, e in ((dh, want_h, got, W_ref.reshape(vocab, width).T), (dw, want_w, got.T, hidden.T)):
        bound = 2.0 ** -18 * (np.abs(mx(c)) @ np.abs(mx(e.astype(np.float64))).T)
        assert (np.abs(f64(a) - b) <= bound + 1e-30).all()
    ctx.close()


def test_a_head_that_was_not_made_to_train():
    ctx = X.Context(4096)
    hd = head.MxHead(ctx, torch.zeros(64, 32, device="cuda"))
    s = hd.score(torch.ones(2, 32, device="cuda"), torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert np.allclose(f64(s["logprob"]), -np.log(64), atol=1e-6)
    with pytest.raises(ValueError):
        hd.gradients(None, None, s, None)
    ctx.close()


def test_a_context_on_another_stream():
    """Work queued before a call is waited for, and what follows a call waits for it, whatever stream each is on."""
    here, own = X.Context(4096), torch.cuda.Stream()
    own.wait_stream(torch.cuda.current_stream())
    there = X.Context(4096, stream=own)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w0, h0 = (torch.empty(n, 256, device="cuda").normal_(generator=g) for n in (4099, 300))
    t = torch.randint(0, 4099, (300,), device="cuda", generator=g)
    ones = torch.ones(300, device="cuda")
    big = torch.empty(4096, 8192, device="cuda")
    results = []
    for ctx in (here, there):
        for _ in range(20):
            big.normal_()                                    # keeps the caller's stream busy
        w, h = w0 * 0.5, h0 + 0.0
        hd = head.MxHead(ctx, w, train=True)
        del w
        torch.empty(4099, 256, device="cuda").fill_(7.0)
        s = hd.score(h, t, 3)
        scored = [s[k].clone() for k in ("logits", "logprob", "entropy", "top_ids")]
        dh, dw = hd.gradients(h, t, s, ones)
        results.append(scored + [dh + 0.0, dw + 0.0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    here.close()
    there.close()


def test_the_command():
    r = head.compare(0, 64)
    assert r["same_first"] > 0.9 and abs(r["logprob"][0] - r["logprob"][1]) < 0.1 and r["compressed"] > 8


@pytest.mark.parametrize("what", ["scores", "gradients"])
def test_two_callers_on_streams_of_their_own(what):
    """What one caller has dropped and its stream still reads is nobody else's, whoever calls the head meanwhile."""
    vocab, width, tokens = 5003, 256, 200
    own, one, two = (torch.cuda.Stream() for _ in range(3))
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    w = torch.empty(vocab, width, device="cuda").normal_(generator=g)
    hidden = [torch.empty(tokens, width, device="cuda").normal_(generator=g) for _ in range(2)]
    targets = torch.randint(0, vocab, (tokens,), device="cuda", generator=g)
    ones, big = torch.ones(tokens, device="cuda"), torch.empty(4096, 8192, device="cuda")
    torch.cuda.synchronize()

    def results(hd, h):
        s = hd.score(h, targets, 3)
        return [s[k] for k in ("logits", "logprob", "entropy", "lse", "top_logprob", "top_ids")] if what == "scores" else list(hd.gradients(h, targets, s, ones))
    ctx = X.Context(4096)
    want = [[t.clone() for t in results(head.MxHead(ctx, w, train=True), h)] for h in hidden]
    torch.cuda.synchronize()
    ctx.close()
    ctx = X.Context(4096, stream=own)
    hd = head.MxHead(ctx, w, train=True)
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        first = results(hd, hidden[0])
        places = {t.data_ptr() for t in first}
        for _ in range(60):
            big.normal_()                                    # the reads below are still to come when the others begin
        kept = [t + 0 for t in first]
        del first
    second = []
    with torch.cuda.stream(two):
        for _ in range(3):
            second.append(results(hd, hidden[1]))
            assert not places & {t.data_ptr() for t in second[-1]}
    with torch.cuda.stream(own):                             # nor that of another use of the context's stream
        other = [torch.zeros_like(t) for t in second[0]]
        assert not places & {t.data_ptr() for t in other}
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, want[0]))
    assert all(torch.equal(a, b) for s in second for a, b in zip(s, want[1]))
    ctx.close()
