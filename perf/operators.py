"""The operators a reconstructed checkpoint is answered and trained with, as measured cases.

Microscaled 4-bit floating point (blocks of 32 E2M1 elements under one power of two): quantisation of
weights and activations along their rows and down their columns, and the products of what was
quantised -- for a token, for a prompt, and for the three products of a training step.  And the log
probabilities of given tokens with the entropy and the top alternatives of every row of logits, with
their gradient.

`run` computes a case in plain torch operations, or, with `own`, through the library's entry points.
"""
import math

import torch

own = False

BLOCK = 32            # elements under one scale
GROUP = 128           # a row of codes is padded to whole groups of this many elements
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------
def quantize_case(rows, cols, dtype, both=False, gap=0):
    return {"op": "quantize", "rows": rows, "cols": cols, "type": dtype, "both": both, "gap": gap}


def linear_case(m, n, k, dtype, out):
    return {"op": "linear", "m": m, "n": n, "k": k, "type": dtype, "out": out}


def train_case(m, n, k, dtype):
    return {"op": "train", "m": m, "n": n, "k": k, "type": dtype}


def score_case(rows, vocab, dtype, top, grad=False, masked=False, gap=0):
    return {"op": "score", "rows": rows, "vocab": vocab, "type": dtype, "top": top, "grad": grad, "masked": masked,
            "gap": gap}


def listed():
    def named(name, case):
        return dict(case, name=name)
    return [
        # one hidden state of a small model goes to 4 bits: nothing but latency
        named("quantize_row", quantize_case(1, 1024, "f16")),
        # a slice of a wider odd matrix, for a training step: along the rows and down the columns at once
        named("quantize_both_odd", quantize_case(2047, 1031, "f32", both=True, gap=5)),
        # the largest weight of a 7B-shaped layer, reconstructed in bf16, is stored in 4 bits and read back
        named("quantize_weight", quantize_case(11008, 4096, "bf16")),
        # one new token through an attention projection of a 7B-shaped model
        named("linear_token", linear_case(1, 4096, 4096, "bf16", "bf16")),
        # sixteen sequences decoded together: their logits over a GPT-NeoX vocabulary
        named("linear_logits", linear_case(16, 50304, 2048, "bf16", "f32")),
        # sizes that fill no tile: a short prompt through a pruned layer
        named("linear_odd", linear_case(333, 1031, 1000, "f16", "f32")),
        # a batch of prompts through the widest product of a 7B-shaped layer
        named("linear_prompt", linear_case(8192, 11008, 4096, "bf16", "bf16")),
        # a training step of the widest layer of a 1.4B-shaped model: output, gradient of the input, of the weights
        named("train_layer", train_case(4096, 8192, 2048, "bf16")),
        # one generated token is reported with its twenty alternatives
        named("score_token", score_case(1, 50304, "f32", 20)),
        # answers of an evaluation are scored: every token with its entropy and a few alternatives
        named("score_batch", score_case(4096, 50304, "bf16", 8)),
        # constrained decoding with feedback: masked vocabularies, tokens without a target, a row with nothing left
        named("score_masked", score_case(77, 32001, "f16", 5, grad=True, masked=True, gap=3)),
        # the loss of a training step with an entropy bonus, and its gradient over the logits
        named("score_train", score_case(4096, 32000, "bf16", 0, grad=True)),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _size(rng, low, high):
    """Over the logarithm of the range; half of the sizes whole multiples of 64 where that fits, the rest as they come."""
    v = _log_int(rng, low, high)
    if rng.random() < 0.5 and v >= 64:
        v -= v % 64
    return v


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "train", "score", "score"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "quantize":
        cols = _size(rng, 32, 11008)
        rows = _size(rng, 1, min(50304, 11008 * 4096 // cols))
        return quantize_case(rows, cols, dtype, both=rng.random() < 0.4, gap=rng.choice([0, 0, 1, 8, 13]))
    if op == "linear":
        m = rng.choice([1, _size(rng, 1, 16), _size(rng, 1, 8192), _size(rng, 16, 8192)])
        k = _size(rng, 128, 11008)
        n = _size(rng, 128, 50304)
        while m * n * k > 8192 * 11008 * 4096 or m * n > 1 << 28:
            m = max(1, m // 2)
        return linear_case(m, n, k, dtype, rng.choice(["f32", dtype]))
    if op == "train":
        m, n, k = _size(rng, 32, 8192), _size(rng, 128, 11008), _size(rng, 128, 8192)
        while 3 * m * n * k > 8192 * 11008 * 4096:
            m = max(1, m // 2)
        return train_case(m, n, k, dtype)
    vocab = _size(rng, 512, 65536)
    rows = _size(rng, 1, 4096)
    grad = rng.random() < 0.5
    while rows * vocab * SIZES[dtype] > 4096 * 50304 * 2 // (2 if grad else 1):
        rows = max(1, rows // 2)
    return score_case(rows, vocab, dtype, rng.choice([0, 1, 5, 8, 20]), grad=grad, masked=rng.random() < 0.4,
                      gap=rng.choice([0, 0, 1, 8]))


def work(case):
    s = SIZES[case["type"]]
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        coded = n // 2 + n // BLOCK
        ways = 2 if case["both"] else 1
        return {"bytes": n * s + ways * (coded + n * s), "flops": 4 * n * ways}
    if case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k * s + n * k // 2 + n * k // BLOCK + m * n * SIZES[case["out"]], "flops": 2 * m * n * k}
    if case["op"] == "train":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * (m * k + n * k + m * n) * s - n * k * s + n * k * 4, "flops": 6 * m * n * k}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * s * (2 if case["grad"] else 1) + case["rows"] * (16 + 12 * case["top"]),
            "flops": n * (10 if case["grad"] else 5)}


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, rows, cols, scale, dtype, gap=0):
    """rows x cols of a matrix whose rows lie `gap` elements further apart than they are long."""
    base = torch.empty(rows, cols + gap, dtype=torch.float32, device="cuda").normal_(0.0, scale, generator=g).to(TYPES[dtype])
    return base[:, :cols]


def _activations(g, rows, cols, dtype):
    """Hidden states: about one in the scale, with a few channels that stand out, as trained models have them."""
    x = torch.empty(rows, cols, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=g)
    x *= torch.empty(cols, dtype=torch.float32, device="cuda").normal_(0.0, 0.7, generator=g).exp_()
    return x.to(TYPES[dtype])


def _inputs(case, seed):
    g = _gen(seed)
    dtype = case["type"]
    if case["op"] == "quantize":
        x = _normal(g, case["rows"], case["cols"], 0.02, dtype, case["gap"])
        return {"x": x}
    if case["op"] == "linear":
        w = _normal(g, case["n"], case["k"], 0.02, "f32")
        codes, scales = _pack(w)
        return {"x": _activations(g, case["m"], case["k"], dtype), "codes": codes, "scales": scales}
    if case["op"] == "train":
        return {"x": _activations(g, case["m"], case["k"], dtype), "w": _normal(g, case["n"], case["k"], 0.02, dtype),
                "dy": _normal(g, case["m"], case["n"], 1e-3, dtype)}
    rows, vocab = case["rows"], case["vocab"]
    x = _normal(g, rows, vocab, 2.5, dtype, case["gap"])
    peak = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
    line = torch.arange(rows, device="cuda")
    x[line, peak] += torch.empty(rows, dtype=torch.float32, device="cuda").uniform_(2.0, 14.0, generator=g).to(x.dtype)
    targets = torch.where(torch.rand(rows, device="cuda", generator=g) < 0.6, peak,
                          torch.randint(0, vocab, (rows,), device="cuda", generator=g))
    if case["masked"]:
        # two rows in three are masked: by minus infinity, or by the type's lowest value; one has nothing left
        lowest = torch.finfo(x.dtype).min
        hide = torch.rand(rows, vocab, device="cuda", generator=g) < 0.7
        hide[line, targets] &= torch.rand(rows, device="cuda", generator=g) < 0.2
        x[(line % 3 == 1)[:, None] & hide] = -math.inf
        x[(line % 3 == 2)[:, None] & hide] = lowest
        x[rows // 2] = -math.inf
        targets[line % 5 == 4] = -1
    st = {"x": x, "targets": targets}
    if case["grad"]:
        st["g_logprob"] = torch.empty(rows, device="cuda").normal_(-1.0, 0.3, generator=g) / rows
        st["g_entropy"] = torch.empty(rows, device="cuda").normal_(0.01, 0.003, generator=g) / rows
        st["g_top"] = torch.empty(rows, case["top"], device="cuda").normal_(0.0, 0.1, generator=g) / rows
    return st


def _pack(w):
    """Codes and scales of a float32 matrix, in the layout the library stores them in."""
    q, e = _blocks(w)
    rows = w.shape[0]
    mag = q.abs()
    code = ((mag > 0.25).to(torch.uint8) + (mag > 0.75) + (mag > 1.25) + (mag > 1.75) + (mag > 2.5) + (mag > 3.5)
            + (mag > 5.0) + 8 * torch.signbit(q))
    code = code.reshape(rows, -1, 2)
    return (code[:, :, 0] | (code[:, :, 1] << 4)).contiguous(), (e + 127).to(torch.uint8).contiguous()


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if own:
        _prepare_own(state, case)
    return state


# ---------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------
def _power(e):
    """2^e in float32, exactly, for whole e from -127 to 127."""
    e = e.int()
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).int().view(torch.float32)


def _blocks(x):
    """Elements (in units of their scale) and the scales' exponents of float32 rows in blocks of 32.

    exponent = floor(log2(largest magnitude)) - 2; element = x / 2^exponent to the nearest of 0, 0.5, 1, 1.5, 2, 3,
    4, 6, ties to the even code, beyond 6 to 6.
    """
    rows, cols = x.shape
    pad = -cols % GROUP
    if pad:
        x = torch.cat([x, x.new_zeros(rows, pad)], 1)
    x = x.reshape(rows, -1, BLOCK)
    peak = x.abs().amax(2)
    e = torch.where(peak > 0, (torch.frexp(peak).exponent - 3).clamp(-127, 127), -127)
    a = x * _power(-e)[:, :, None]
    mag = a.abs()
    q = (0.5 * ((mag > 0.25).float() + (mag >= 0.75) + (mag > 1.25) + (mag >= 1.75)) + (mag > 2.5).float()
         + (mag >= 3.5) + 2.0 * (mag > 5.0))
    return torch.copysign(q, a), e


def _round_trip(x):
    """The float32 values that the 4-bit form of float32 rows stands for."""
    rows, cols = x.shape
    q, e = _blocks(x)
    return (q * _power(e)[:, :, None]).reshape(rows, -1)[:, :cols]


GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _unpack(codes, scales, cols):
    table = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], 2)
    v = table[both.long()].reshape(codes.shape[0], -1, BLOCK)
    return (v * _power(scales.int() - 127)[:, :, None]).reshape(codes.shape[0], -1)[:, :cols]


def _run_plain(st, case):
    kind = TYPES[case["type"]]
    if case["op"] == "quantize":
        x = st["x"].float()
        out = [_round_trip(x).to(kind)]
        if case["both"]:
            out.append(_round_trip(x.t().contiguous()).to(kind))
        return out
    if case["op"] == "linear":
        w = _unpack(st["codes"], st["scales"], case["k"])
        return (_round_trip(st["x"].float()) @ w.t()).to(TYPES[case["out"]])
    if case["op"] == "train":
        x, w, dy = st["x"].float(), st["w"].float(), st["dy"].float()
        y = _round_trip(x) @ _round_trip(w).t()
        dx = _round_trip(dy) @ _round_trip(w.t().contiguous()).t()
        dw = _round_trip(dy.t().contiguous()) @ _round_trip(x.t().contiguous()).t()
        return [y.to(kind), dx.to(kind), dw]
    return _score_plain(st, case)


def _score_plain(st, case):
    x, t = st["x"].float(), st["targets"]
    rows, vocab = x.shape
    line = torch.arange(rows, device=x.device)
    peak = x.amax(1)
    some = peak > -math.inf                                # a row with nothing left has no distribution
    shift = torch.where(some, peak, torch.zeros_like(peak))
    e = torch.exp(x - shift[:, None])
    total = e.sum(1)
    lse = torch.where(some, shift + torch.log(total), torch.full_like(peak, -math.inf))
    p = e / torch.where(some, total, torch.ones_like(total))[:, None]
    logp = torch.where(p > 0, x - torch.where(some, lse, torch.zeros_like(lse))[:, None], torch.zeros_like(x))
    entropy = -(p * logp).sum(1)
    given = (t >= 0) & (t < vocab)
    at = t.clamp(0, vocab - 1)
    raw = x[line, at]
    lp = torch.where(raw > -math.inf, raw - lse, torch.full_like(raw, -math.inf))
    logprob = torch.where(given, lp, torch.zeros_like(lp))
    out = [logprob, entropy]
    ids = top = None
    if case["top"]:
        left = x.clone()
        index = torch.arange(vocab, device=x.device)
        ids, top = [], []
        for _ in range(case["top"]):
            best = left.amax(1)
            there = best > -math.inf
            first = torch.where(left == best[:, None], index, vocab).amin(1)
            ids.append(torch.where(there, first, -1))
            top.append(torch.where(there, best - lse, best))
            left[line, first] = -math.inf
        ids, top = torch.stack(ids, 1), torch.stack(top, 1)
        out += [top, ids]
    if case["grad"]:
        gl = torch.where(given & (raw > -math.inf), st["g_logprob"], torch.zeros_like(raw))
        weight = gl
        if case["top"]:
            gt = torch.where(ids >= 0, st["g_top"], torch.zeros_like(st["g_top"]))
            weight = weight + gt.sum(1)
        d = -p * (weight[:, None] + st["g_entropy"][:, None] * (logp + entropy[:, None]))
        d[line, at] += gl
        if case["top"]:
            for j in range(case["top"]):
                d[line, ids[:, j].clamp(min=0)] += gt[:, j]
        out.append(d.to(TYPES[case["type"]]))
    return out


# ---------------------------------------------------------------------------------------------------
# the library's operators
# ---------------------------------------------------------------------------------------------------
_context = None


def _ctx():
    """A program keeps one context for its stream."""
    global _context
    if _context is None:
        import paper_2406_11257_amd as X
        _context = X.Context(4096)
    return _context


def _prepare_own(st, case):
    """The context, and the arrays such a program keeps for what it computes."""
    import paper_2406_11257_amd as X
    st["ctx"] = _ctx()
    kind = TYPES[case["type"]]

    def coded(rows, cols):
        return X.mx_empty(rows, cols, "cuda")

    def like(rows, cols, dtype):
        return torch.empty(rows, cols, dtype=dtype, device="cuda")
    if case["op"] == "quantize":
        r, c = case["rows"], case["cols"]
        st["q"], st["back"] = coded(r, c), like(r, c, kind)
        if case["both"]:
            st["qt"], st["back_t"] = coded(c, r), like(c, r, kind)
    elif case["op"] == "linear":
        st["xq"] = coded(case["m"], case["k"])
        st["y"] = like(case["m"], case["n"], TYPES[case["out"]])
    elif case["op"] == "train":
        m, n, k = case["m"], case["n"], case["k"]
        st["xq"], st["xt"] = coded(m, k), coded(k, m)
        st["wq"], st["wt"] = coded(n, k), coded(k, n)
        st["dq"], st["dt"] = coded(m, n), coded(n, m)
        st["y"], st["dx"], st["dw"] = like(m, n, kind), like(m, k, kind), like(n, k, torch.float32)
    else:
        rows, top = case["rows"], case["top"]
        st["logprob"], st["entropy"] = (torch.empty(rows, device="cuda") for _ in range(2))
        st["lse"] = like(rows, 2, torch.float32)
        st["top_logprob"] = like(rows, top, torch.float32) if top else None
        st["top_ids"] = like(rows, top, torch.int64) if top else None
        if case["grad"]:
            st["d"] = like(rows, case["vocab"], kind)


def _run_own(st, case):
    ctx = st["ctx"]
    if case["op"] == "quantize":
        if case["both"]:
            ctx.excp_mx_quantize(st["x"], *st["q"], *st["qt"])
            ctx.excp_mx_dequantize(*st["q"], st["back"])
            ctx.excp_mx_dequantize(*st["qt"], st["back_t"])
            return [st["back"], st["back_t"]]
        ctx.excp_mx_quantize(st["x"], *st["q"])
        ctx.excp_mx_dequantize(*st["q"], st["back"])
        return [st["back"]]
    if case["op"] == "linear":
        ctx.excp_mx_linear(st["x"], st["codes"], st["scales"], st["y"], *st["xq"])
        return st["y"]
    if case["op"] == "train":
        m, n, k = case["m"], case["n"], case["k"]
        ctx.excp_mx_quantize(st["x"], *st["xq"], *st["xt"])
        ctx.excp_mx_quantize(st["w"], *st["wq"], *st["wt"])
        ctx.excp_mx_quantize(st["dy"], *st["dq"], *st["dt"])
        ctx.excp_mx_matmul(*st["xq"], *st["wq"], k, st["y"])
        ctx.excp_mx_matmul(*st["dq"], *st["wt"], n, st["dx"])
        ctx.excp_mx_matmul(*st["dt"], *st["xt"], m, st["dw"])
        return [st["y"], st["dx"], st["dw"]]
    ctx.excp_token_logprobs(st["x"], st["targets"], st["logprob"], st["entropy"], st["lse"], st["top_logprob"], st["top_ids"])
    out = [st["logprob"], st["entropy"]]
    if case["top"]:
        out += [st["top_logprob"], st["top_ids"]]
    if case["grad"]:
        ctx.excp_token_logprobs_backward(st["x"], st["targets"], st["lse"], st["entropy"], st["top_ids"], st["g_logprob"],
                                         st["g_entropy"], st["g_top"] if case["top"] else None, st["d"])
        out.append(st["d"])
    return out


def run(state):
    case = state["case"]
    return _run_own(state, case) if own else _run_plain(state, case)


# ---------------------------------------------------------------------------------------------------
# the definitions, in 64 bits
# ---------------------------------------------------------------------------------------------------
def _exact_values(x):
    """What the 4-bit form of the rows of x stands for: x over a power of two, to a grid whose step doubles with the octave."""
    x = x.double()
    rows, cols = x.shape
    out = torch.zeros_like(x)
    for first in range(0, cols, BLOCK):
        b = x[:, first:first + BLOCK]
        peak = b.abs().max(1, keepdim=True).values
        # the peak without its fraction bits is the power of two at or below it
        unit = 0.25 * (peak.clamp(min=2.0 ** -125).contiguous().view(torch.int64) >> 52 << 52).view(torch.float64)
        r = b / unit
        step = torch.where(r.abs() < 2, 0.5, torch.where(r.abs() < 4, 1.0, 2.0)).double()
        out[:, first:first + BLOCK] = (torch.round(r / step) * step).clamp(-6, 6) * unit
    return out


def exact(case, seed):
    st = _inputs(case, seed)
    if case["op"] == "quantize":
        out = [_exact_values(st["x"])]
        if case["both"]:
            out.append(_exact_values(st["x"].t()))
        return out
    if case["op"] == "linear":
        low, high = (st["codes"] & 15).long(), (st["codes"] >> 4).long()
        c = torch.stack([low, high], 2).reshape(case["n"], -1)
        size, neg = c & 7, c >= 8
        # one sign bit, two of the exponent (bias 1), one of the fraction; exponent 0: half the fraction bit
        half = (size & 1).double() * 0.5
        v = torch.where(size < 2, half, (1.0 + half) * (1 << (size >> 1)) * 0.5)
        w = torch.where(neg, -v, v) * (st["scales"].long() - 127 + 1023 << 52).view(torch.float64).repeat_interleave(BLOCK, 1)
        return _exact_values(st["x"]) @ w[:, :case["k"]].t()
    if case["op"] == "train":
        x, w, dy = st["x"], st["w"], st["dy"]
        return [_exact_values(x) @ _exact_values(w).t(), _exact_values(dy) @ _exact_values(w.t()).t(),
                _exact_values(dy.t()) @ _exact_values(x.t()).t()]
    return _exact_score(st, case)


def _exact_score(st, case):
    parts = []
    step = max(1, (1 << 26) // case["vocab"])
    for a in range(0, case["rows"], step):
        parts.append(_exact_score_rows({k: v[a:a + step] for k, v in st.items()}, case))
    return [torch.cat(p) for p in zip(*parts)]


def _exact_score_rows(st, case):
    x = st["x"].double()
    rows, vocab = x.shape
    empty = torch.isneginf(x).all(1)
    logp = torch.log_softmax(torch.where(empty[:, None], torch.zeros_like(x), x), 1)
    logp[empty] = -math.inf
    p = logp.exp()
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    entropy = -plogp.sum(1)
    t = st["targets"]
    given = (t >= 0) & (t < vocab)
    lp = logp.gather(1, t.clamp(0, vocab - 1)[:, None])[:, 0]
    out = [torch.where(given, lp, torch.zeros_like(lp)), entropy]
    use = given & ~torch.isneginf(lp)
    ids = None
    if case["top"]:
        # the logits are what is sorted: log probabilities of different logits may be equal
        order = torch.sort(x, dim=1, descending=True, stable=True)
        ids = order.indices[:, :case["top"]]
        top = logp.gather(1, ids)
        ids = torch.where(torch.isneginf(order.values[:, :case["top"]]), -1, ids)
        out += [top, ids]
    if case["grad"]:
        def along(weights, index, ok):
            """The gradient of sum_j weights_j * log p[index_j]: each hit less its share of p."""
            w = torch.where(ok, weights.double(), torch.zeros_like(weights, dtype=torch.float64))
            hit = torch.zeros_like(p).scatter_add_(1, index.clamp(0, vocab - 1), w)
            return hit - p * w.sum(1, keepdim=True)
        d = along(st["g_logprob"][:, None], t[:, None], use[:, None])
        if case["top"]:
            d += along(st["g_top"], ids, ids >= 0)
        d -= st["g_entropy"].double()[:, None] * (plogp + p * entropy[:, None])
        out.append(d)
    return out
