"""4-bit microscaled quantisation and products against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2406_11257_amd as X
from ops_util import DTYPES, HALF_ULP, SMALLEST, f64, mx_reference, mx_values, strided

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = X.Context(4096)
    yield c
    c.close()


def draw(rows, cols, dtype, seed, scale=0.02):
    g = np.random.default_rng(seed)
    a = g.standard_normal((rows, cols)) * scale
    a *= np.exp2(g.integers(-8, 8, (1, cols)) * (g.random((1, cols)) < 0.1))        # some columns stand out
    return f64_of_type(a, dtype)


def f64_of_type(a, dtype):
    return torch.from_numpy(a).to(DTYPES[dtype]).double().numpy()


def guarded(rows, cols):
    """Codes and scales inside larger arrays whose ends are checked."""
    groups = -(-cols // 128)
    room = [torch.full((rows * groups * w + 64,), 0xA5, dtype=torch.uint8, device="cuda") for w in (64, 4)]
    return room, [r[:rows * groups * w].view(rows, groups * w) for r, w in zip(room, (64, 4))]


def unharmed(room, views):
    return all(bool((r[v.numel():] == 0xA5).all()) for r, v in zip(room, views))


SHAPES = [(1, 1), (1, 31), (1, 32), (1, 33), (3, 127), (2, 128), (5, 129), (1, 1024), (64, 96), (127, 65), (128, 128), (129, 257),
          (31, 1000), (333, 37), (200, 640), (1031, 259), (77, 4097)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("gap,lead", [(0, 0), (3, 1), (8, 8)])
def test_quantize_both_ways_and_back(ctx, rows, cols, dtype, gap, lead):
    a = draw(rows, cols, dtype, rows * 1000 + cols)
    x = strided(a, dtype, gap, lead)
    room, q = guarded(rows, cols)
    room_t, qt = guarded(cols, rows)
    ctx.excp_mx_quantize(x, *q, *qt)
    one, only = X.mx_empty(rows, cols), X.mx_empty(cols, rows)
    ctx.excp_mx_quantize(x, *one)
    ctx.excp_mx_quantize(x, None, None, *only)
    back = strided(np.full((rows, cols), 9.0), dtype, gap, lead)
    ctx.excp_mx_dequantize(*q, back)
    for got, ref in ((q, mx_reference(a)), (one, mx_reference(a)), (qt, mx_reference(a.T)), (only, mx_reference(a.T))):
        assert np.array_equal(got[1].cpu().numpy(), ref[1])
        assert np.array_equal(got[0].cpu().numpy(), ref[0])
    assert unharmed(room, q) and unharmed(room_t, qt)
    want = torch.from_numpy(mx_values(*mx_reference(a), cols)).to(DTYPES[dtype])
    assert torch.equal(back.cpu(), want)
    if gap:
        outside = torch.as_strided(back, (rows - 1, gap), (back.stride(0), 1), back.storage_offset() + cols) if rows > 1 else None
        assert outside is None or bool((outside == 7.0).all())


@pytest.mark.parametrize("dtype,first", [("f32", -150), ("bf16", -134), ("f16", -25)])
def test_every_rounding_case(dtype, first):
    """Around every threshold of the grid, in every octave of the scale that the type has, and both signs."""
    edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, 7.75])
    near = np.concatenate([edges, edges * (1 - 2.0 ** {"f32": -20, "bf16": -7, "f16": -10}[dtype]), edges * (1 + 2.0 ** {"f32": -20, "bf16": -7, "f16": -10}[dtype])])
    rows = []
    for e in range(first, {"f32": 126, "bf16": 126, "f16": 14}[dtype]):
        for part in np.array_split(np.concatenate([near, -near]), 3):
            rows.append(np.concatenate([[4.0], part, [0.0, -0.0]])[:32] * 2.0 ** e)
            rows[-1] = np.pad(rows[-1], (0, 32 - len(rows[-1])))
    a = f64_of_type(np.array(rows), dtype)
    c = X.Context(4096)
    x = torch.from_numpy(a).to(DTYPES[dtype]).cuda()
    q = X.mx_empty(len(rows), 32)
    c.excp_mx_quantize(x, *q)
    back = torch.empty_like(x)
    c.excp_mx_dequantize(*q, back)
    codes, scales = mx_reference(a)
    assert np.array_equal(q[1].cpu().numpy(), scales)
    assert np.array_equal(q[0].cpu().numpy(), codes)
    assert torch.equal(back.cpu(), torch.from_numpy(mx_values(codes, scales, 32)).to(DTYPES[dtype]))
    c.close()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_smallest_largest_and_what_is_no_number(ctx, dtype):
    fi = torch.finfo(DTYPES[dtype])
    a = draw(40, 160, dtype, 5)
    a[0] = 0.0
    a[1, :32] = fi.max
    a[2, :32] = -fi.max
    a[3] = SMALLEST[dtype]
    a[4, ::2] = fi.tiny
    a[4, 1::2] = 0.0
    a[5, 7], a[6, 40], a[7, 159], a[8, 100] = np.nan, np.inf, -np.inf, np.nan
    a[9, 64:96] = 0.0
    x = strided(a, dtype)
    q, qt = X.mx_empty(40, 160), X.mx_empty(160, 40)
    ctx.excp_mx_quantize(x, *q, *qt)
    for got, src in ((q, a), (qt, a.T)):
        codes, scales = mx_reference(src)
        assert np.array_equal(got[1].cpu().numpy(), scales)
        fine = np.repeat(scales != 255, 16, axis=1)
        assert np.array_equal(got[0].cpu().numpy()[fine], codes[fine])
    back = torch.empty_like(x)
    ctx.excp_mx_dequantize(*q, back)
    codes, scales = mx_reference(a)
    want = torch.from_numpy(mx_values(codes, scales, 160)).to(DTYPES[dtype])
    assert torch.equal(torch.nan_to_num(back.cpu(), nan=123.0), torch.nan_to_num(want, nan=123.0))


def coded(a):
    codes, scales = mx_reference(a)
    return [torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()], mx_values(codes, scales, a.shape[1])


def product_bound(a, b, dtype):
    """What a product may be off: every group of 128 is one addition to an fp32 sum, joined sums a few more, an addition
    of the matrix units off by up to 2^-22 of what it adds; and one rounding to the type."""
    size = np.abs(a) @ np.abs(b).T
    return (-(-a.shape[1] // 128) + 16) * 2.0 ** -22 * size + HALF_ULP[dtype] * size + SMALLEST[dtype]


PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 17, 129), (2, 1000, 32), (15, 33, 1000), (16, 256, 512), (17, 65, 384), (33, 130, 130),
            (64, 64, 64), (128, 128, 128), (129, 127, 257), (200, 300, 640), (256, 256, 1024), (257, 511, 300), (333, 1031, 1000),
            (48, 2048, 4096), (1000, 24, 2500), (16, 100, 9000), (9, 70, 20001), (1, 40, 120000), (16, 9000, 700),
            (70, 200, 1152), (64, 64, 1280), (100, 90, 3000), (17, 40, 256), (128, 66, 128), (50, 4000, 2176)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_matmul(ctx, m, n, k, dtype):
    (ca, a), (cb, b) = coded(draw(m, k, "f32", m + k, 1.0)), coded(draw(n, k, "f32", n + k + 1, 0.02))
    y = strided(np.full((m, n), 9.0), dtype, 5, 1)
    ctx.excp_mx_matmul(*ca, *cb, k, y)
    err = np.abs(f64(y) - a @ b.T)
    assert (err <= product_bound(a, b, dtype)).all(), err.max()
    if m > 1:
        assert bool((torch.as_strided(y, (m - 1, 5), (n + 5, 1), 1 + n) == 7.0).all())
    again = torch.empty(m, n, dtype=DTYPES[dtype], device="cuda")
    ctx.excp_mx_matmul(*ca, *cb, k, again)
    assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(3500, 3700, 600), (4100, 3333, 1280), (2049, 8190, 384), (1500, 1700, 2944), (5000, 3900, 127), (50304, 300, 256)])
def test_matmul_of_many_tiles(ctx, m, n, k, dtype):
    """The same at sizes that fill the GPU with the larger tiles (compared in 64 bits on the GPU)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    (ca, cb), values = (X.mx_empty(m, k), X.mx_empty(n, k)), []
    for (codes, scales), rows, scale in ((ca, m, 1.0), (cb, n, 0.02)):
        a = torch.empty(rows, k, device="cuda").normal_(0, scale, generator=g)
        ctx.excp_mx_quantize(a, codes, scales)
        ctx.excp_mx_dequantize(codes, scales, a)
        values.append(a.double())
    y = torch.empty(m, n, dtype=DTYPES[dtype], device="cuda")
    ctx.excp_mx_matmul(*ca, *cb, k, y)
    want, size = values[0] @ values[1].t(), values[0].abs() @ values[1].abs().t()
    bound = (-(-k // 128) + 16) * 2.0 ** -22 * size + HALF_ULP[dtype] * size + SMALLEST[dtype]
    assert bool(((y.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("xtype,ytype", [("f32", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f16"), ("f32", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_linear_quantises_on_the_way(ctx, m, n, k, xtype, ytype):
    x = draw(m, k, xtype, m + k, 1.0)
    a = mx_values(*mx_reference(x), k)
    cb, b = coded(draw(n, k, "f32", n + k + 1, 0.02))
    for gap, lead in ((0, 0), (3, 1)):
        y = strided(np.full((m, n), 9.0), ytype, gap, 0)
        ctx.excp_mx_linear(strided(x, xtype, gap, lead), *cb, y, *X.mx_empty(m, k))
        err = np.abs(f64(y) - a @ b.T)
        assert (err <= product_bound(a, b, ytype)).all(), err.max()
        if m <= X.EXCP_MX_FEW_ROWS:
            again = torch.empty(m, n, dtype=DTYPES[ytype], device="cuda")
            ctx.excp_mx_linear(strided(x, xtype, gap, lead), *cb, again)
            assert torch.equal(again, y)


@pytest.mark.parametrize("m", [1, 3, 16, 40, 300])
def test_what_is_no_number_stays_in_its_row_and_column(ctx, m):
    n, k = 70, 500
    x, w = draw(m, k, "f32", 1, 1.0), draw(n, k, "f32", 2)
    x[m // 2, 77] = np.inf
    w[13, 499] = np.nan
    cb, b = coded(w)
    y = torch.empty(m, n, device="cuda")
    ctx.excp_mx_linear(strided(x, "f32"), *cb, y, *X.mx_empty(m, k))
    bad = np.zeros((m, n), bool)
    bad[m // 2], bad[:, 13] = True, True
    assert np.array_equal(np.isnan(f64(y)), bad)


def test_products_of_a_training_step(ctx):
    """Output, gradient of the input and of the weights are the three products of what is quantised both ways; and the
    gradients are those of the loss <dy, y> where nothing is lost to 4 bits."""
    m, n, k = 96, 160, 224
    g = np.random.default_rng(3)
    x, w, dy = (g.choice([-3.0, -1.0, 0.0, 0.5, 2.0, 6.0], size) for size in ((m, k), (n, k), (m, n)))
    mx = {}
    for name, a in (("x", x), ("w", w), ("dy", dy)):
        a[::32, :] = 6.0                                # every block has the same scale, so that every value is exact
        a[:, ::32] = 6.0
        mx[name] = X.mx_empty(*a.shape), X.mx_empty(*a.T.shape)
        ctx.excp_mx_quantize(strided(a, "bf16"), *mx[name][0], *mx[name][1])
    y, dx, dw = (torch.empty(s, device="cuda") for s in ((m, n), (m, k), (n, k)))
    ctx.excp_mx_matmul(*mx["x"][0], *mx["w"][0], k, y)
    ctx.excp_mx_matmul(*mx["dy"][0], *mx["w"][1], n, dx)
    ctx.excp_mx_matmul(*mx["dy"][1], *mx["x"][1], m, dw)
    assert np.array_equal(f64(y), x @ w.T)
    assert np.array_equal(f64(dx), dy @ w)
    assert np.array_equal(f64(dw), dy.T @ x)
    # differences: y is linear in one element of x and of w
    x2 = x.copy()
    x2[5, 7] += 0.25
    assert abs(((x2 @ w.T - x @ w.T) * dy).sum() / 0.25 - f64(dx)[5, 7]) < 1e-9
    w2 = w.copy()
    w2[11, 3] -= 0.5
    assert abs(((x @ w2.T - x @ w.T) * dy).sum() / -0.5 - f64(dw)[11, 3]) < 1e-9


def test_empty_sizes(ctx):
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        q, qt = X.mx_empty(rows, cols), X.mx_empty(cols, rows)
        x = torch.empty(rows, cols, device="cuda")
        ctx.excp_mx_quantize(x, *q, *qt)
        ctx.excp_mx_dequantize(*q, x)
    for m in (1, 40):
        y = torch.full((m, 33), 5.0, device="cuda")
        ctx.excp_mx_matmul(*X.mx_empty(m, 0), *X.mx_empty(33, 0), 0, y)
        assert bool((y == 0).all())
        y.fill_(5.0)
        ctx.excp_mx_linear(torch.empty(m, 0, device="cuda"), *X.mx_empty(33, 0), y, *X.mx_empty(m, 0))
        assert bool((y == 0).all())
    ctx.excp_mx_matmul(*X.mx_empty(0, 64), *X.mx_empty(33, 64), 64, torch.empty(0, 33, device="cuda"))
    ctx.excp_mx_linear(torch.empty(4, 64, device="cuda"), *X.mx_empty(0, 64), torch.empty(4, 0, device="cuda"))


def test_another_stream_and_a_captured_graph():
    """A context works on the stream it was made with; its operators can be recorded and replayed."""
    x, w = draw(8, 700, "bf16", 1, 1.0), draw(300, 700, "bf16", 2)
    a, (cb, b) = mx_values(*mx_reference(x), 700), coded(w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        c = X.Context(4096, stream=st)
        xd, y = strided(x, "bf16"), torch.zeros(8, 300, device="cuda")
        q = X.mx_empty(300, 700)
        wd = strided(w, "bf16")
        c.excp_mx_quantize(wd, *q)
        c.excp_mx_linear(xd, *q, y)
    st.synchronize()
    first = y.clone()
    assert (np.abs(f64(y) - a @ b.T) <= product_bound(a, b, "f32")).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        c.excp_mx_quantize(wd, *q)
        c.excp_mx_linear(xd, *q, y)
    for _ in range(3):
        y.zero_()
        q[0].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, first)
    c.close()


def test_refusals(ctx):
    L, h = X.lib(), ctx._h
    x = torch.zeros(64, 256, device="cuda")
    c, s = X.mx_empty(64, 256)
    y = torch.zeros(64, 64, device="cuda")
    P = lambda t, off=0: t.data_ptr() + off

    def quantize(p=P(x), kind=0, rows=64, cols=256, ld=256, c1=P(c), s1=P(s), c2=None, s2=None, ctx_=h):
        return L.excp_mx_quantize(ctx_, p, kind, rows, cols, ld, c1, s1, c2, s2)
    assert quantize() == X.EXCP_OK
    for bad in (dict(ctx_=None), dict(p=None), dict(p=P(x, 2)), dict(kind=3), dict(kind=-1), dict(ld=255), dict(c1=None), dict(s1=None),
                dict(c1=None, s1=None), dict(c1=P(c, 8)), dict(s1=P(s, 2)), dict(c2=P(c)), dict(s2=P(s)), dict(rows=1 << 31), dict(cols=1 << 31),
                dict(ld=1 << 40)):
        assert quantize(**bad) == X.EXCP_E_ARG, bad

    def dequantize(c1=P(c), s1=P(s), rows=64, cols=256, p=P(x), kind=0, ld=256, ctx_=h):
        return L.excp_mx_dequantize(ctx_, c1, s1, rows, cols, p, kind, ld)
    assert dequantize() == X.EXCP_OK
    for bad in (dict(ctx_=None), dict(p=None), dict(p=P(x, 2)), dict(kind=3), dict(ld=255), dict(c1=None), dict(s1=None), dict(c1=P(c, 8)),
                dict(s1=P(s, 1)), dict(rows=1 << 31)):
        assert dequantize(**bad) == X.EXCP_E_ARG, bad

    def matmul(a=P(c), sa=P(s), b=P(c), sb=P(s), m=64, n=64, k=256, p=P(y), kind=0, ld=64, ctx_=h):
        return L.excp_mx_matmul(ctx_, a, sa, b, sb, m, n, k, p, kind, ld)
    assert matmul() == X.EXCP_OK
    for bad in (dict(ctx_=None), dict(a=None), dict(sa=None), dict(b=None), dict(sb=None), dict(a=P(c, 4)), dict(sb=P(s, 2)), dict(p=None),
                dict(p=P(y, 1)), dict(kind=7), dict(ld=63), dict(m=1 << 31), dict(n=1 << 31), dict(k=1 << 31)):
        assert matmul(**bad) == X.EXCP_E_ARG, bad

    c2, s2 = X.mx_empty(64, 256)

    def linear(p=P(x), kind=0, ldx=256, b=P(c), sb=P(s), m=64, n=64, k=256, o=P(y), ok=0, ldy=64, xc=P(c2), xs=P(s2), ctx_=h):
        return L.excp_mx_linear(ctx_, p, kind, ldx, b, sb, m, n, k, o, ok, ldy, xc, xs)
    assert linear() == X.EXCP_OK and linear(m=16, xc=None, xs=None) == X.EXCP_OK
    for bad in (dict(ctx_=None), dict(p=None), dict(kind=9), dict(ok=-2), dict(ldx=255), dict(ldy=63), dict(b=None), dict(sb=None), dict(o=None),
                dict(xc=None, xs=None), dict(xc=None), dict(xs=None), dict(xc=P(c2, 8)), dict(m=17, xc=None, xs=None), dict(k=1 << 31)):
        assert linear(**bad) == X.EXCP_E_ARG, bad
    # the binding's own: types, shapes, devices
    for call in (lambda: ctx.excp_mx_quantize(x.double(), c, s), lambda: ctx.excp_mx_quantize(x.t(), *X.mx_empty(256, 64)),
                 lambda: ctx.excp_mx_quantize(x, c[:, :64], s), lambda: ctx.excp_mx_quantize(x.cpu(), c, s), lambda: ctx.excp_mx_quantize(x[0], c, s),
                 lambda: ctx.excp_mx_quantize(x, c, None), lambda: ctx.excp_mx_quantize(x, c.int(), s), lambda: ctx.excp_mx_dequantize(c, s[:1], x),
                 lambda: ctx.excp_mx_matmul(c, s, c, s, 512, y), lambda: ctx.excp_mx_linear(x, c, s, y, c2[:3], s2)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        ctx.excp_mx_linear(x, c, s, y[:3], c2, s2)
    with pytest.raises(X.ExcpError):
        ctx.excp_mx_quantize(x)
    with pytest.raises(X.ExcpError):
        ctx.excp_mx_linear(x, c, s, y)


def test_scales_without_codes_are_refused(ctx):
    x, y = torch.zeros(4, 256, device="cuda"), torch.zeros(4, 64, device="cuda")
    (c, s), (ct, st), (w, sw) = X.mx_empty(4, 256), X.mx_empty(256, 4), X.mx_empty(64, 256)
    for call in (lambda: ctx.excp_mx_quantize(x, None, s, ct, st), lambda: ctx.excp_mx_quantize(x, c, s, None, st),
                 lambda: ctx.excp_mx_linear(x, w, sw, y, None, s)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("dtype,gap", [("f32", 3), ("bf16", 0), ("f16", 8)])
@pytest.mark.parametrize("m,n,k", [(40, 16500, 4096), (64, 16449, 4200), (17, 20011, 5100), (1, 17000, 4224), (33, 16390, 8000), (63, 25000, 700),
                                   (16, 16400, 130), (100, 25001, 300), (128, 24700, 1000), (65, 24600, 4097), (129, 50000, 256)])
def test_matmul_of_few_rows_by_many(ctx, m, n, k, dtype, gap):
    """A few rows against so many that the GPU is full (compared in 64 bits on the GPU)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(m + n + k)
    (ca, cb), values = (X.mx_empty(m, k), X.mx_empty(n, k)), []
    for (codes, scales), rows, scale in ((ca, m, 1.0), (cb, n, 0.02)):
        a = torch.empty(rows, k, device="cuda").normal_(0, scale, generator=g)
        ctx.excp_mx_quantize(a, codes, scales)
        ctx.excp_mx_dequantize(codes, scales, a)
        values.append(a.double())
    whole = torch.full((m, n + gap), 9.0, dtype=DTYPES[dtype], device="cuda")
    y = whole[:, :n]
    ctx.excp_mx_matmul(*ca, *cb, k, y)
    want, size = values[0] @ values[1].t(), values[0].abs() @ values[1].abs().t()
    bound = (-(-k // 128) + 16) * 2.0 ** -22 * size + HALF_ULP[dtype] * size + SMALLEST[dtype]
    assert bool(((y.double() - want).abs() <= bound).all()) and bool((whole[:, n:] == 9.0).all())


@pytest.mark.parametrize("xtype,ytype", [("f32", "f32"), ("bf16", "f16")])
@pytest.mark.parametrize("m,n,k", [(16, 40, 6657), (16, 500, 11008), (12, 33, 9001), (5, 16500, 129), (16, 17000, 300), (4, 17000, 300), (9, 16384, 0),
                                   (16, 20, 63488), (16, 18, 63489), (13, 34, 90000), (7, 300, 33000)])
def test_few_rows_of_any_length(ctx, m, n, k, xtype, ytype):
    """One to sixteen rows that fit where they are quantised, or not, against few rows of W and many; with room given and without."""
    x = draw(m, k, xtype, m + k, 1.0)
    a = mx_values(*mx_reference(x), k) if k else x
    cb, b = coded(draw(n, k, "f32", n + k + 1, 0.02)) if k else (X.mx_empty(n, 0), np.zeros((n, 0)))
    y = strided(np.full((m, n), 9.0), ytype, 3, 0)
    ctx.excp_mx_linear(strided(x, xtype, 1, 1), *cb, y)
    assert (np.abs(f64(y) - a @ b.T) <= product_bound(a, b, ytype)).all()
    again = torch.full((m, n), 9.0, dtype=DTYPES[ytype], device="cuda")
    ctx.excp_mx_linear(strided(x, xtype), *cb, again, *X.mx_empty(m, k))
    assert torch.equal(again, y)
    # the room is that of rows of logits: neither harms the other
    logits = torch.linspace(-3, 3, 70001, device="cuda").repeat(2, 1)
    ids, lp = torch.empty(2, 4, dtype=torch.int64, device="cuda"), torch.empty(2, 4, device="cuda")
    for _ in range(3):
        ctx.excp_mx_linear(strided(x, xtype), *cb, again)
        ctx.excp_token_logprobs(logits, top_logprob=lp, top_ids=ids)
        assert torch.equal(again, y) and ids[1].tolist() == [70000, 69999, 69998, 69997]


@pytest.mark.parametrize("wide", [torch.int16, torch.int32, torch.int64])
def test_codes_in_a_wider_integer_type(ctx, wide):
    """Codes made by integer arithmetic, which promotes bytes: what reads them brings them back, on the context's stream."""
    (ca, _), (cb, _) = coded(draw(40, 700, "f32", 1, 1.0)), coded(draw(300, 700, "f32", 2))
    wa, wb = ([t.to(wide) for t in q] for q in (ca, cb))
    x = strided(draw(40, 700, "f32", 3, 1.0), "f32")
    y, z = torch.empty(40, 300, device="cuda"), torch.empty(40, 300, device="cuda")
    ctx.excp_mx_matmul(*ca, *cb, 700, y)
    for a, b in ((wa, wb), (ca, wb), ([wa[0], ca[1]], [cb[0], wb[1]])):
        ctx.excp_mx_matmul(*a, *b, 700, z.fill_(9.0))
        assert torch.equal(y, z)
    for rows in (1, 16, 40):
        ctx.excp_mx_linear(x[:rows], *cb, y[:rows], *X.mx_empty(rows, 700))
        ctx.excp_mx_linear(x[:rows], *wb, z[:rows].fill_(9.0), *X.mx_empty(rows, 700))
        assert torch.equal(y[:rows], z[:rows])
    v, w = torch.empty(300, 700, device="cuda"), torch.empty(300, 700, device="cuda")
    ctx.excp_mx_dequantize(*cb, v)
    ctx.excp_mx_dequantize(*wb, w)
    assert torch.equal(v, w)
    own, big, room, more = torch.cuda.Stream(), torch.empty(4096, 8192, device="cuda"), X.mx_empty(40, 700), X.mx_empty(40, 700)
    own.wait_stream(torch.cuda.current_stream())
    there = X.Context(4096, stream=own)
    with torch.cuda.stream(own):
        for _ in range(10):
            big.normal_()
        late = [t + 0 for t in wb]                           # not there yet when the call is made
    there.excp_mx_linear(x, *late, z, *room)
    ctx.excp_mx_linear(x, *cb, y, *more)
    torch.cuda.synchronize()
    assert torch.equal(y, z)
    there.close()


def test_codes_that_are_no_bytes_are_refused(ctx):
    x, y = torch.zeros(4, 256, device="cuda"), torch.zeros(4, 64, device="cuda")
    (w, sw), (c, s) = X.mx_empty(64, 256), X.mx_empty(4, 256)
    for call in (lambda: ctx.excp_mx_linear(x, w.float(), sw, y), lambda: ctx.excp_mx_linear(x, w.bool(), sw, y),
                 lambda: ctx.excp_mx_linear(x, w.long()[:63], sw, y), lambda: ctx.excp_mx_linear(x, w.long().cpu(), sw, y),
                 lambda: ctx.excp_mx_linear(x, w.long()[:, ::2], sw, y), lambda: ctx.excp_mx_linear(x, w, sw, y, c.long(), s),
                 lambda: ctx.excp_mx_quantize(x, c.long(), s), lambda: ctx.excp_mx_matmul(c.half(), s, w, sw, 256, y),
                 lambda: ctx.excp_mx_dequantize(c, s.float(), x)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("m,n,k", [(5, 16500, 129), (16, 17000, 300), (16, 40, 6657), (16, 20, 63488)])
def test_few_rows_work_in_the_room_they_are_given(ctx, m, n, k):
    """Where a few rows take two launches, the codes between them lie in the caller's room, if there is one."""
    x = draw(m, k, "f32", m + k, 1.0)
    cb, b = coded(draw(n, k, "f32", n + k + 1, 0.02))
    room, q = guarded(m, k)
    y, z = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    ctx.excp_mx_linear(strided(x, "f32"), *cb, y, *q)
    ctx.excp_mx_linear(strided(x, "f32"), *cb, z)
    codes, scales = mx_reference(x)
    assert np.array_equal(q[0].cpu().numpy(), codes) and np.array_equal(q[1].cpu().numpy(), scales) and unharmed(room, q)
    assert torch.equal(y, z)
    assert (np.abs(f64(y) - mx_values(codes, scales, k) @ b.T) <= product_bound(mx_values(codes, scales, k), b, "f32")).all()


def test_more_rows_than_a_launch_has_threads():
    """2^30 and some rows of W: sixteen million tiles of 256 threads would be more than a launch can have."""
    n = (1 << 30) + 5
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 80 GB")
    c = X.Context(4096)
    codes, scales = (t.zero_() for t in X.mx_empty(n, 1))
    at = torch.tensor([0, 63, 1 << 28, (1 << 28) + 77, (1 << 29) - 1, 1 << 30, n - 1], device="cuda")
    codes[at, 0] = 2                                         # 1.0 under 2^0, up to 2^6
    scales[at, 0] = 127 + torch.arange(7, dtype=torch.uint8, device="cuda")
    x = torch.ones(1, 1, device="cuda")
    q = X.mx_empty(1, 1)
    c.excp_mx_quantize(x, *q)
    for linear in (False, True):
        y = torch.full((1, n), 9.0, dtype=torch.float16, device="cuda")
        if linear:
            c.excp_mx_linear(x, codes, scales, y)
        else:
            c.excp_mx_matmul(*q, codes, scales, 1, y)
        assert y[0, at].tolist() == [2.0 ** i for i in range(7)]
        y[0, at] = 0
        assert not bool(y.any())
    c.close()
    del codes, scales, y
    torch.cuda.empty_cache()
