"""Log probabilities of given tokens, entropy, alternatives and their gradient against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2406_11257_amd as X
from ops_util import DTYPES, HALF_ULP, SMALLEST, f64, gradient_reference, scores_reference, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = X.Context(4096)
    yield c
    c.close()


def case(rows, vocab, dtype, seed, masked=False):
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, vocab)) * 3.0
    t = g.integers(0, vocab, rows)
    x[np.arange(rows), t] += 4.0 * g.random(rows)
    if masked:
        hide = g.random((rows, vocab)) < 0.6
        lowest = float(torch.finfo(DTYPES[dtype]).min)
        x[(np.arange(rows) % 3 == 0)[:, None] & hide] = -np.inf
        x[(np.arange(rows) % 3 == 1)[:, None] & hide] = lowest
        x[rows // 2] = -np.inf
        x[rows // 3] = lowest
        t[::4] = g.choice([-1, vocab, -(1 << 40), 1 << 33], len(t[::4]))
    return torch.from_numpy(x).to(DTYPES[dtype]).double().numpy(), t


def outputs(rows, ntop):
    return dict(logprob=torch.full((rows,), 77.0, device="cuda"), entropy=torch.full((rows,), 77.0, device="cuda"),
                lse=torch.full((rows, 2), 77.0, device="cuda"),
                top_logprob=torch.full((rows, ntop), 77.0, device="cuda") if ntop else None,
                top_ids=torch.full((rows, ntop), 77, dtype=torch.int64, device="cuda") if ntop else None)


def close(got, ref, size):
    """Within `size` where the reference is finite, and the same infinities and NaN."""
    got = f64(got)
    fin = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    assert (np.abs(got - ref)[fin] <= np.broadcast_to(size, ref.shape)[fin]).all(), np.abs(got - ref)[fin].max()


def tolerance(x, vocab):
    """Of lse and log probabilities: the sum of exponentials is off by a relative 2^-20 at most -- an exponential by 4 units
    in the last place and 2^-24 of its argument (at most 32 where the term matters beside the others), fp32 sums over at
    most vocab / 64 + 64 additions that partly cancel: sqrt of their number -- and what is subtracted is rounded at its
    size.  The entropy adds the same again, times the spread of the logits that matter (at most 32)."""
    big = np.where(np.isfinite(x), np.abs(x), 0).max(1)
    big = np.where(big > 1e4, np.abs(np.where(np.isfinite(x) & (np.abs(x) < 1e4), x, 0)).max(1), big)
    t = 2.0 ** -20 + 2.0 ** -22 * big + 2.0 ** -24 * np.sqrt(vocab)
    return t


SIZES = [(1, 1), (1, 2), (3, 7), (1, 63), (2, 64), (5, 65), (4, 255), (3, 1000), (33, 513), (1, 5000), (2, 50304), (7, 32001), (1, 131073),
         (300, 700), (2, 300001), (9, 8192)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_scores_and_gradient(ctx, rows, vocab, dtype, masked):
    x, t = case(rows, vocab, dtype, rows + vocab, masked)
    targets = torch.from_numpy(t).cuda()
    g = np.random.default_rng(1)
    for ntop, gap, lead in ((0, 0, 0), (1, 3, 1), (5, 8, 8), (20, 0, 0), (64, 1, 3)):
        logits = strided(x, dtype, gap, lead)
        o = outputs(rows, ntop)
        ctx.excp_token_logprobs(logits, targets, **o)
        lse, lp, ent, top, ids = scores_reference(x, t, ntop)
        tol = tolerance(x, vocab)
        close(o["lse"].double().sum(1), lse, tol)
        # a log probability far below is rounded at its own size
        close(o["logprob"], lp, tol + 2.0 ** -23 * np.where(np.isfinite(lp), np.abs(lp), 0))
        close(o["entropy"], ent, 32.0 * tol)
        if ntop:
            assert np.array_equal(o["top_ids"].cpu().numpy(), ids)
            close(o["top_logprob"], top, tol[:, None] + 2.0 ** -23 * np.where(np.isfinite(top), np.abs(top), 0))
        gl, ge, gt = g.standard_normal(rows), g.standard_normal(rows) * 0.1, g.standard_normal((rows, ntop))
        gl, ge, gt = (a.astype(np.float32).astype(np.float64) for a in (gl, ge, gt))
        d = strided(np.full((rows, vocab), 5.0), dtype, gap + 2)
        dev = [torch.from_numpy(a).float().cuda() for a in (gl, ge, gt)]
        ctx.excp_token_logprobs_backward(logits, targets, o["lse"], o["entropy"], o["top_ids"], dev[0], dev[1], dev[2] if ntop else None, d)
        ref = gradient_reference(x, t, ids, gl, ge, gt if ntop else None)
        # p is off by a relative 2^-20 and lse's error; what multiplies it by the errors of the sums and of the entropy
        weight = np.abs(gl) + np.abs(gt).sum(1) + np.abs(ge) * 40.0
        rel = (64.0 * tol * weight)[:, None]
        p = np.exp(np.where(np.isfinite(x), x, -np.inf) - np.where(np.isfinite(lse), lse, 0.0)[:, None])
        bound = rel * np.minimum(p, 1.0) + 2.0 * HALF_ULP[dtype] * np.abs(ref) + 2.0 ** -22 * weight[:, None] * (ref != 0) + SMALLEST[dtype]
        close(d, ref, bound)
        if rows > 1:
            assert bool((torch.as_strided(d, (rows - 1, gap + 2), (d.stride(0), 1), vocab) == 7.0).all())
        # in place
        d2 = logits.clone() if not gap else logits
        ctx.excp_token_logprobs_backward(d2, targets, o["lse"], o["entropy"], o["top_ids"], dev[0], dev[1], dev[2] if ntop else None, d2)
        assert torch.equal(d2.contiguous().view(torch.uint8), d.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 70001])
def test_ties_and_what_is_no_number(ctx, dtype, vocab):
    g = np.random.default_rng(4)
    x = np.round(g.standard_normal((12, vocab)) * 2.0)                  # almost every alternative is tied
    x[1] = 0.0
    x[2], x[2, ::2] = 0.0, -0.0
    x[3, 17] = np.nan
    x[4, vocab - 1] = np.inf
    x[5, 3], x[5, 200] = np.inf, np.inf
    x[6] = np.nan
    x[7] = -np.inf
    x[7, 250] = -3.0
    x[8, 11], x[8, 12] = np.nan, np.inf
    x[9] = -np.inf
    x[9, ::100] = 1.0
    x[10] = np.inf
    x[11] = -np.inf
    t = np.array([5, 6, 7, 17, vocab - 1, 0, 1, 250, -1, 0, 3, 3])
    logits, targets = strided(x, dtype), torch.from_numpy(t).cuda()
    o = outputs(12, 9)
    ctx.excp_token_logprobs(logits, targets, **o)
    lse, lp, ent, top, ids = scores_reference(x, t, 9)
    assert np.array_equal(o["top_ids"].cpu().numpy(), ids)
    tol = 1e-5
    close(o["lse"].double().sum(1), lse, tol)
    close(o["logprob"], lp, tol)
    close(o["entropy"], ent, 32 * tol)
    close(o["top_logprob"], top, tol)
    ones = torch.ones(12, device="cuda")
    d = torch.empty_like(logits)
    ctx.excp_token_logprobs_backward(logits, targets, o["lse"], o["entropy"], o["top_ids"], ones, ones, torch.ones(12, 9, device="cuda"), d)
    ref = gradient_reference(x, t, ids, np.ones(12), np.ones(12), np.ones((12, 9)))
    assert np.array_equal(np.isnan(f64(d)), np.isnan(ref))
    fin = np.isfinite(ref)
    assert (np.abs(f64(d) - ref)[fin] <= 1e-4 + HALF_ULP[dtype] * np.abs(ref[fin])).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_with_masked_targets(ctx, dtype):
    """In place, whether a target is masked is found out before its logit is overwritten: long rows, several chunks."""
    rows, vocab = 600, 70001
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    logits = torch.empty(rows, vocab, device="cuda").normal_(0, 2, generator=g).to(DTYPES[dtype])
    targets = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    logits[torch.arange(rows, device="cuda")[::2], targets[::2]] = -float("inf")
    o = outputs(rows, 4)
    ctx.excp_token_logprobs(logits, targets, **o)
    gl, gt = torch.ones(rows, device="cuda"), torch.full((rows, 4), 0.5, device="cuda")
    d = torch.empty_like(logits)
    ctx.excp_token_logprobs_backward(logits, targets, o["lse"], None, o["top_ids"], gl, None, gt, d)
    ctx.excp_token_logprobs_backward(logits, targets, o["lse"], None, o["top_ids"], gl, None, gt, logits)
    assert torch.equal(d, logits)
    # the weights of a row sum to zero but for what a type rounds: 2^-8 of sum |d| < 2 (1 + 4 / 2)
    assert bool((d.double().sum(1).abs() < {"f32": 1e-4, "bf16": 6 * 2.0 ** -8}[dtype]).all())
    assert bool((o["logprob"][::2] == -float("inf")).all())
    at = d.gather(1, targets[:, None])[:, 0]
    assert bool((at[::2] == 0).all()) and bool((at[1::2] > 0.1).all())


@pytest.mark.parametrize("which", ["logprob", "entropy", "top"])
def test_gradient_against_differences(ctx, which):
    """Central differences of the fp32 outputs' 64-bit counterparts, in every direction of a small row."""
    rows, vocab, ntop = 3, 40, 4
    x, t = case(rows, vocab, "f32", 11)
    x[2, 5:9] = -np.inf
    t[2] = 20
    logits, targets = strided(x, "f32"), torch.from_numpy(t).cuda()
    o = outputs(rows, ntop)
    ctx.excp_token_logprobs(logits, targets, **o)
    g = {k: np.random.default_rng(2).standard_normal(s).astype(np.float32) for k, s in (("logprob", (rows,)), ("entropy", (rows,)), ("top", (rows, ntop)))}
    dev = {k: torch.from_numpy(v).cuda() if k == which else None for k, v in g.items()}
    d = torch.empty_like(logits)
    ctx.excp_token_logprobs_backward(logits, targets if which == "logprob" else None, o["lse"], o["entropy"] if which == "entropy" else None,
                                     o["top_ids"] if which == "top" else None, dev["logprob"], dev["entropy"], dev["top"], d)
    h = 1e-4
    ids = o["top_ids"].cpu().numpy()

    def loss(v):
        lse, lp, ent, _, _ = scores_reference(v, t, 0)
        if which == "top":
            return sum(g["top"][r, j] * (v[r, ids[r, j]] - lse[r]) for r in range(rows) for j in range(ntop))
        return float((g[which] * (lp if which == "logprob" else ent)).sum())
    for r in range(rows):
        for i in range(vocab):
            if not np.isfinite(x[r, i]):
                assert f64(d)[r, i] == 0
                continue
            up, down = x.copy(), x.copy()
            up[r, i] += h
            down[r, i] -= h
            # a central difference is off by h^2 / 6 of the third derivative (below 30 here), d by fp32's rounding
            assert abs((loss(up) - loss(down)) / (2 * h) - f64(d)[r, i]) < 5 * h * h + 1e-5


def test_outputs_left_out_and_empty_sizes(ctx):
    x, t = case(6, 500, "f32", 3)
    logits, targets = strided(x, "f32"), torch.from_numpy(t).cuda()
    full = outputs(6, 3)
    ctx.excp_token_logprobs(logits, targets, **full)
    for name in full:
        one = outputs(6, 3)
        ctx.excp_token_logprobs(logits, targets if name == "logprob" else None, **{name: one[name]})
        assert torch.equal(one[name], full[name]), name
    o = outputs(4, 2)
    ctx.excp_token_logprobs(torch.empty(4, 0, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), **o)
    assert bool((o["lse"][:, 0] == -np.inf).all() and (o["entropy"] == 0).all() and (o["logprob"] == 0).all() and (o["top_ids"] == -1).all())
    ctx.excp_token_logprobs(torch.empty(0, 9, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), lse=torch.empty(0, 2, device="cuda"))
    d = torch.full((6, 500), 4.0, device="cuda")
    ctx.excp_token_logprobs_backward(logits, None, full["lse"], None, None, None, None, None, d)
    assert bool((d == 0).all())


def test_rows_on_their_own_equal_rows_together(ctx):
    """A row's results do not depend on what is beside it beyond rounding: few rows are split over workgroups, many are not."""
    x, t = case(400, 30011, "bf16", 8)
    logits, targets = strided(x, "bf16"), torch.from_numpy(t).cuda()
    o = outputs(400, 6)
    ctx.excp_token_logprobs(logits, targets, **o)
    for r in (0, 17, 399):
        one = outputs(1, 6)
        ctx.excp_token_logprobs(logits[r:r + 1], targets[r:r + 1], **one)
        assert torch.equal(one["top_ids"][0], o["top_ids"][r])
        for name in ("logprob", "entropy", "lse", "top_logprob"):
            assert torch.allclose(one[name][0], o[name][r], rtol=0, atol=2e-5), name


def test_the_same_twice_and_in_a_captured_graph():
    st = torch.cuda.Stream()
    x, t = case(3, 60001, "f32", 9)
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        c = X.Context(4096, stream=st)
        logits, targets, o = strided(x, "f32"), torch.from_numpy(t).cuda(), outputs(3, 8)
        d = torch.empty_like(logits)
        ones = torch.ones(3, device="cuda")

        def both():
            c.excp_token_logprobs(logits, targets, **o)
            c.excp_token_logprobs_backward(logits, targets, o["lse"], o["entropy"], None, ones, ones, None, d)
        both()
    st.synchronize()
    first = [o[k].clone() for k in o] + [d.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        both()
    for _ in range(3):
        for k in o:
            o[k].zero_()
        d.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(first, [o[k] for k in o] + [d]):
            assert torch.equal(a, b)
    c.close()


def test_refusals(ctx):
    L, h = X.lib(), ctx._h
    x = torch.zeros(4, 100, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    v = torch.zeros(4, 8, device="cuda")
    ids = torch.zeros(4, 8, dtype=torch.int64, device="cuda")
    P = lambda a, off=0: a.data_ptr() + off

    def scores(p=P(x), kind=0, rows=4, vocab=100, ld=100, tg=P(t), ntop=8, lp=P(v), e=P(v), s=P(v), tl=P(v), ti=P(ids), ctx_=h):
        return L.excp_token_logprobs(ctx_, p, kind, rows, vocab, ld, tg, ntop, lp, e, s, tl, ti)
    assert scores() == X.EXCP_OK
    for bad in (dict(ctx_=None), dict(p=None), dict(p=P(x, 2)), dict(kind=5), dict(ld=99), dict(tg=None), dict(tg=P(t, 4)), dict(ntop=-1),
                dict(ntop=65), dict(lp=P(v, 2)), dict(e=P(v, 1)), dict(s=P(v, 3)), dict(tl=P(v, 2)), dict(ti=P(ids, 4)), dict(rows=1 << 31),
                dict(vocab=1 << 31)):
        assert scores(**bad) == X.EXCP_E_ARG, bad

    def grad(p=P(x), kind=0, rows=4, vocab=100, ld=100, tg=P(t), s=P(v), e=P(v), ti=P(ids), ntop=8, gl=P(v), ge=P(v), gt=P(v), d=P(x), ldd=100, ctx_=h):
        return L.excp_token_logprobs_backward(ctx_, p, kind, rows, vocab, ld, tg, s, e, ti, ntop, gl, ge, gt, d, ldd)
    assert grad() == X.EXCP_OK
    for bad in (dict(ctx_=None), dict(p=None), dict(kind=5), dict(ld=99), dict(ldd=99), dict(ldd=101), dict(tg=None), dict(s=None), dict(e=None),
                dict(ti=None), dict(ntop=65), dict(ntop=-1), dict(d=None), dict(d=P(x, 2)), dict(gl=P(v, 2)), dict(ge=P(v, 2)), dict(gt=P(v, 2)),
                dict(rows=1 << 31)):
        assert grad(**bad) == X.EXCP_E_ARG, bad
    for call in (lambda: ctx.excp_token_logprobs(x.double()), lambda: ctx.excp_token_logprobs(x, t.int(), logprob=v[:, 0].contiguous()),
                 lambda: ctx.excp_token_logprobs(x, t, logprob=v[:, 0]), lambda: ctx.excp_token_logprobs(x, top_ids=ids[:3]),
                 lambda: ctx.excp_token_logprobs(x, top_ids=ids, top_logprob=v[:, :3].contiguous()),
                 lambda: ctx.excp_token_logprobs_backward(x, t, v[:, :2].contiguous(), None, None, None, None, None, x.half())):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("parts", [False, True])
def test_small_probabilities_are_held_to_their_own_size(ctx, parts):
    """The gradient of improbable tokens, relative to itself: with x - max exact (logits are multiples of 2^-10), p is off by what
    the sum of exponentials is (2^-22), by what rounds its logarithm (2^-24 of that) and by half a unit of eight operations,
    however small it is."""
    rows, vocab = (3, 40001) if parts else (2500, 5003)
    g = np.random.default_rng(6)
    x = np.round(-80.0 * g.random((rows, vocab)) * 1024.0) / 1024.0
    x[:, 7] = 3.0
    x[1] = np.round(g.standard_normal(vocab) * 2048.0) / 1024.0
    x[1, 11] = -78.0
    t = np.full(rows, 7)
    logits, targets = strided(x, "f32"), torch.from_numpy(t).cuda()
    o = outputs(rows, 2)
    ctx.excp_token_logprobs(logits, targets, **o)
    ones, d = torch.full((rows,), 0.75, device="cuda"), torch.empty_like(logits)
    z = np.exp(x - x.max(1, keepdims=True))
    s = z.sum(1, keepdims=True)
    rel = 2.0 ** -22 + 2.0 ** -24 * (np.abs(np.log(s)) + 8.0)
    far = np.arange(vocab) != 7
    ctx.excp_token_logprobs_backward(logits, targets, o["lse"], None, None, ones, None, None, d)
    assert (np.abs(f64(d) + 0.75 * z / s) <= rel * 0.75 * z / s)[:, far].all()
    gt = torch.tensor([0.5, 0.25], device="cuda").repeat(rows, 1)
    ctx.excp_token_logprobs_backward(logits, None, o["lse"], None, o["top_ids"], None, None, gt, d)
    far = np.ones((rows, vocab), bool)
    far[np.arange(rows)[:, None], o["top_ids"].cpu().numpy()] = False
    assert (np.abs(f64(d) + 0.75 * z / s) <= rel * 0.75 * z / s)[far].all()
