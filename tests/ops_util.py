"""Plain implementations in 64 bits of the operators on reconstructed weights, for the tests."""
import numpy as np
import torch

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}      # of a rounding to the type (bf16: 2^-9, rounded up)
SMALLEST = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx_reference(x):
    """(codes, scales) as stored, of the rows of a float64 matrix that holds values of a 32- or 16-bit type."""
    rows, cols = x.shape
    groups = -(-cols // 128)
    full = np.zeros((rows, groups * 128))
    full[:, :cols] = x
    blocks = full.reshape(rows, groups * 4, 32)
    bad = ~np.isfinite(blocks).all(2)
    peak = np.abs(np.where(np.isfinite(blocks), blocks, 0)).max(2)
    e = np.where(peak > 0, np.maximum(np.frexp(peak)[1] - 1 - 2, -127), -127)
    q = np.abs(np.where(bad[:, :, None], 0, blocks)) / np.ldexp(1.0, e)[:, :, None]
    # nearest of the grid, ties to the even code: the distance decides, and the code's last bit between equal ones
    dist = np.abs(q[..., None] - GRID)
    best = dist.min(-1, keepdims=True)
    code = np.where(dist == best, np.arange(8) + 8 * (np.arange(8) & 1), 99).min(-1) & 7
    code = code | (np.signbit(np.where(bad[:, :, None], 0, blocks)) * 8)
    code = code.reshape(rows, -1, 2).astype(np.uint8)
    return (code[:, :, 0] | code[:, :, 1] << 4), np.where(bad, 255, e + 127).astype(np.uint8)


def mx_values(codes, scales, cols):
    """float64 values of stored codes and scales."""
    both = np.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1)
    v = GRID[both & 7] * np.where(both & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (v.reshape(codes.shape[0], -1, 32) * s[:, :, None]).reshape(codes.shape[0], -1)[:, :cols]


def strided(a, dtype, gap=0, lead=0):
    """The float64 matrix a as a device matrix of `dtype` whose rows lie `gap` elements apart and begin `lead` elements
    into their storage."""
    rows, cols = a.shape
    base = torch.full((rows * (cols + gap) + lead,), 7.0, dtype=DTYPES[dtype], device="cuda")
    view = base[lead:lead + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    view.copy_(torch.from_numpy(a).to(DTYPES[dtype]))
    return view


def f64(t):
    return t.double().cpu().numpy()


def scores_reference(x, targets, ntop):
    """(lse, logprob, entropy, top values, top ids) of a float64 matrix of logits, by rows."""
    rows, vocab = x.shape
    lse, lp, ent = np.full(rows, -np.inf), np.zeros(rows), np.zeros(rows)
    top, ids = np.full((rows, ntop), -np.inf), np.full((rows, ntop), -1, dtype=np.int64)
    for r in range(rows):
        v = x[r]
        t = int(targets[r])
        given = 0 <= t < vocab
        left = np.flatnonzero(v > -np.inf)
        order = left[np.lexsort((left, -v[left]))][:ntop]
        ids[r, :len(order)] = order
        if np.isnan(v).any() or np.isposinf(v).any():
            lse[r] = ent[r] = np.nan
            lp[r] = np.nan if given else 0.0
            top[r] = np.nan
            continue
        if len(left) == 0:
            lp[r] = -np.inf if given else 0.0
            continue
        m = v.max()
        z = np.exp(v[left] - m)
        s = z.sum()
        lse[r] = m + np.log(s)
        p = z / s
        logp = v[left] - m - np.log(s)
        ent[r] = -(p[p > 0] * logp[p > 0]).sum()
        if given:
            lp[r] = v[t] - m - np.log(s)
        top[r, :len(order)] = v[order] - m - np.log(s)
    return lse, lp, ent, top, ids


def gradient_reference(x, targets, ids, g_logprob, g_entropy, g_top):
    """The gradient over the logits (float64); ids (rows x ntop) and each g may be None."""
    rows, vocab = x.shape
    d = np.zeros((rows, vocab))
    for r in range(rows):
        v = x[r]
        if np.isnan(v).any() or np.isposinf(v).any():
            d[r] = np.nan
            continue
        left = v > -np.inf
        if not left.any():
            continue
        m = v[left].max()
        z = np.where(left, np.exp(v - m), 0.0)
        p = z / z.sum()
        logp = np.where(p > 0, v - m - np.log(z.sum()), 0.0)
        pairs = []
        if g_logprob is not None and 0 <= targets[r] < vocab and left[targets[r]]:
            pairs.append((int(targets[r]), g_logprob[r]))
        if g_top is not None:
            pairs += [(int(i), g) for i, g in zip(ids[r], g_top[r]) if i >= 0]
        for i, g in pairs:
            d[r] -= g * p
            d[r, i] += g
        if g_entropy is not None:
            d[r] -= g_entropy[r] * p * (logp - (p * logp).sum())
    return d
