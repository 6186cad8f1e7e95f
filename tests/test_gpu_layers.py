"""The layer operators on the GPU against their definitions in 64 bits (layers_reference.py says how far off each may be), at the
sizes, strides, values and calls where they can go wrong."""
import pytest
import torch

import layers_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = ["f16", "bf16"]


@pytest.fixture(scope="module")
def T():
    import paper_2602_12630_amd as T

    assert torch.cuda.is_available(), "the GPU tests need a GPU"
    return T


@pytest.fixture(scope="module")
def ctx(T):
    c = T.Context(0)
    yield c
    c.close()


def rand(shape, seed, t, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(t)


def strided(m, left=0, right=0, sentinel=7):
    """the same values as columns of a wider buffer"""
    buf = torch.full((m.shape[0], left + m.shape[1] + right), sentinel, dtype=m.dtype, device=m.device)
    view = buf[:, left:left + m.shape[1]]
    view.copy_(m)
    return buf, view


def empty(rows, cols, t, pad=(0, 0)):
    """an output of rows x cols inside a wider buffer of sevens, the whole of it one row longer"""
    buf = torch.full((rows + 1, pad[0] + cols + pad[1]), 7, dtype=t, device="cuda")
    return buf, buf[:rows, pad[0]:pad[0] + cols]


def untouched(buf, rows, cols, pad=(0, 0)):
    return bool((buf[rows:] == 7).all() and (buf[:, :pad[0]] == 7).all() and (buf[:, pad[0] + cols:] == 7).all())


def rows8(x):
    q, s = ref.encode(x)
    return q, s


def space(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def ok(got, want, bound):
    w = ref.worst(got, want, bound)
    assert w <= 1.0, "off by %.3g bounds" % w


# ---- checkpoints ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, (0, 0)), (3, 7, (0, 0)), (5, 8, (8, 8)), (9, 512, (0, 0)), (4, 513, (0, 3)), (2, 2048, (1, 0)), (7, 4096, (0, 0)),
                                           (3, 4104, (0, 0)), (2, 11008, (0, 0)), (2, 16384, (0, 8)), (2, 16385, (0, 0)), (2, 40000, (0, 0)), (1000, 64, (0, 0)),
                                           (3, 9, (0, 0)), (2, 2049, (0, 0)), (2, 4101, (5, 0)), (2, 8199, (0, 0)), (3, 1, (0, 2)), (2, 18433, (0, 0))])
def test_checkpoints(T, ctx, dtype, rows, cols, pad):
    t = ref.DT[dtype]
    _, x = strided(rand((rows, cols), rows * cols, t, 3.0), *pad)
    qbuf, q = empty(rows, cols, torch.int8, pad)
    s = torch.full((rows + 1,), 7.0, device="cuda")
    ctx.checkpoint_encode(T.Matrix(x), T.Matrix(q, s[:rows]))
    bbuf, back = empty(rows, cols, t, pad)
    ctx.checkpoint_decode(T.Matrix(q, s[:rows]), T.Matrix(back))
    ctx.sync()
    want, scale = ref.encode(x)
    assert torch.equal(q, want) and torch.equal(s[:rows], scale) and s[rows] == 7
    v = ref.value(want, scale)
    ok(back, v, (ref.u(t) + 2 * ref.E) * v.abs() + ref.tiny(t))
    assert untouched(qbuf, rows, cols, pad) and untouched(bbuf, rows, cols, pad)


@pytest.mark.parametrize("dtype", DTYPES)
def test_checkpoint_values_at_the_edges(T, ctx, dtype):
    """infinities, NaNs, zeros of both signs, the type's largest and smallest values, and every tie: rows whose largest value is k over all
    values of that type up to k in steps of k / 254"""
    t = ref.DT[dtype]
    inf, nan = float("inf"), float("nan")
    big, small = torch.finfo(t).max, torch.finfo(t).smallest_normal * torch.finfo(t).eps
    rows = [[inf, -inf, nan, 1, -2, 0, -0.0, 0.5], [nan] * 8, [inf] * 8, [0.0, -0.0] * 4, [big, -big, big / 2, 1, small, -small, 0, nan],
            [small, -small, 0, small * 2, small * 3, 0, 0, 0], [big, inf, -inf, nan, 0, 1, -1, 2], [-127.0, 63.5, 0.5, 1.5, 2.5, -0.5, -1.5, 126.5]]
    x = torch.tensor(rows, device="cuda").to(t)
    q, s = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(rows), device="cuda")
    ctx.checkpoint_encode(T.Matrix(x), T.Matrix(q, s))
    ctx.sync()
    want, scale = ref.encode(x)
    assert torch.equal(q, want) and torch.equal(s, scale)
    k = torch.arange(1, 255, device="cuda", dtype=torch.float64)
    ties = (torch.arange(-254, 255, device="cuda", dtype=torch.float64)[None, :] * k[:, None] / 254).to(t)      # those that the type can hold are exact ties
    ties[:, 0] = k.to(t)
    q, s = torch.empty(ties.shape, dtype=torch.int8, device="cuda"), torch.empty(254, device="cuda")
    ctx.checkpoint_encode(T.Matrix(ties), T.Matrix(q, s))
    ctx.sync()
    want, scale = ref.encode(ties)
    assert torch.equal(q, want) and torch.equal(s, scale)


# ---- norms ---------------------------------------------------------------------------------------------------------
NORM_SIZES = [(1, 1, (0, 0)), (1, 4096, (0, 0)), (3, 7, (0, 0)), (6, 512, (8, 0)), (5, 520, (0, 0)), (33, 1027, (0, 2)), (4, 2056, (0, 0)), (17, 4096, (0, 0)),
              (3, 8192, (0, 0)), (2, 11008, (0, 0)), (2, 16392, (0, 0)), (2, 32768, (0, 0)), (2, 32767, (0, 0)), (1500, 256, (0, 0)), (700, 1024, (0, 0)),
              (2, 9, (0, 0)), (3, 515, (0, 0)), (2, 2049, (1, 0)), (1100, 4099, (0, 0)), (2, 8197, (0, 0)), (1030, 7, (0, 0)), (2, 16390, (0, 0))]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("rows,cols,pad", NORM_SIZES)
def test_norm_and_its_gradient(T, ctx, dtype, kind, rows, cols, pad):
    t = ref.DT[dtype]
    centred = kind == "layer"
    k = T.TC_NORM_LAYER if centred else T.TC_NORM_RMS
    seed = rows * 7 + cols
    x = rand((rows, cols), seed, t) + (0.5 if centred else 0.0)
    x = x.to(t)
    gamma, beta = rand((cols,), seed + 1, t, 0.2) + 1, rand((cols,), seed + 2, t, 0.2)
    gamma = gamma.to(t)
    if not centred:
        beta = None
    eight = rows8(x)
    _, xs = strided(x, *pad)
    for data, scale in ((xs, None), eight):
        v = ref.value(data, scale)
        ybuf, y = empty(rows, cols, t, pad)
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        mx = T.Matrix(data, scale) if scale is not None else T.Matrix(data)
        ctx.norm(k, mx, gamma, beta, 1e-5, T.Matrix(y), mean, rstd)
        ctx.sync()
        g64, b64 = gamma.double(), beta.double() if beta is not None else None
        want, wmean, wrstd = ref.norm(v, g64, b64, 1e-5, centred)
        ok(y, want, ref.norm_bound(v, g64, b64, want, wrstd, t, centred))
        ok(mean, wmean, 64 * ref.E * v.abs().mean(1) + 1e-30)
        off = 66 * ref.E * v.abs().mean(1) + 2 * ref.E * v.abs().square().mean(1).sqrt()
        ok(rstd, wrstd, wrstd * (64 * ref.E + (off * wrstd if centred else 0)))
        assert untouched(ybuf, rows, cols, pad)
        # the gradient, from the statistics that the pass has left
        _, dy = strided(rand((rows, cols), seed + 3, t), *pad)
        dbuf, dx = empty(rows, cols, t, pad)
        dg, db = torch.full((cols + 1,), 7.0, device="cuda"), torch.full((cols + 1,), 7.0, device="cuda")
        ctx.norm_backward(k, T.Matrix(dy), mx, gamma, mean, rstd, T.Matrix(dx), dg[:cols], db[:cols], space(ctx.norm_backward_workspace(rows, cols)))
        ctx.sync()
        m64, r64 = mean.double(), rstd.double()
        wdx, wdg, wdb = ref.norm_backward(dy.double(), v, g64, m64, r64, centred)
        e_dx, e_dg, e_db = ref.norm_backward_bounds(dy.double(), v, g64, m64, r64, wdx, t, centred)
        ok(dx, wdx, e_dx)
        ok(dg[:cols], wdg, e_dg + 1e-30)
        ok(db[:cols], wdb, e_db + 1e-30)
        assert untouched(dbuf, rows, cols, pad) and dg[cols] == 7 and db[cols] == 7


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_arguments_that_may_be_left_out_or_shared(T, ctx, dtype):
    t = ref.DT[dtype]
    x, dy = rand((9, 264), 1, t), rand((9, 264), 2, t)
    y, mean, rstd = torch.empty_like(x), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
    ctx.norm(0, T.Matrix(x), None, None, 1e-5, T.Matrix(y), mean, rstd)
    want, m64, r64 = ref.norm(x.double(), None, None, 1e-5, True)
    ctx.sync()
    ok(y, want, ref.norm_bound(x.double(), None, None, want, r64, t, True))
    same = x.clone()
    ctx.norm(0, T.Matrix(same), None, None, 1e-5, T.Matrix(same))
    ctx.sync()
    assert torch.equal(same, y)
    w = space(ctx.norm_backward_workspace(9, 264))
    dx, dg, db = torch.empty_like(x), torch.empty(264, device="cuda"), torch.empty(264, device="cuda")
    ctx.norm_backward(0, T.Matrix(dy), T.Matrix(x), None, mean, rstd, T.Matrix(dx), dg, db, w)
    alone, dg2, db2 = torch.empty_like(x), torch.zeros_like(dg), torch.zeros_like(db)
    ctx.norm_backward(0, T.Matrix(dy), T.Matrix(x), None, mean, rstd, T.Matrix(alone), None, None, None)
    ctx.norm_backward(0, T.Matrix(dy), T.Matrix(x), None, mean, rstd, None, dg2, None, w)
    ctx.norm_backward(0, T.Matrix(dy), T.Matrix(x), None, mean, rstd, None, None, db2, w)
    ctx.sync()
    assert torch.equal(alone, dx) and torch.equal(dg, dg2) and torch.equal(db, db2)
    ctx.norm_backward(0, T.Matrix(dy), T.Matrix(x), None, mean, rstd, T.Matrix(dy), None, None, None)
    ctx.sync()
    assert torch.equal(dy, dx)


@pytest.mark.parametrize("dtype", DTYPES)
def test_norm_of_rows_that_are_not_numbers(T, ctx, dtype):
    """a NaN or an infinity spoils its own row and no other; a constant row has y = beta"""
    t = ref.DT[dtype]
    x = rand((6, 1024), 4, t)
    x[1, 5], x[2, 9], x[3] = float("nan"), float("inf"), 2.0
    beta = rand((1024,), 5, t)
    y = torch.empty_like(x)
    ctx.norm(0, T.Matrix(x), None, beta, 1e-5, T.Matrix(y))
    ctx.sync()
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all() and torch.equal(y[3], beta)
    assert torch.isfinite(y[[0, 4, 5]]).all()


# ---- products ------------------------------------------------------------------------------------------------------
LINEAR_SIZES = [(1, 1, 1, (0, 0)), (1, 64, 128, (0, 0)), (1, 4096, 264, (0, 0)), (2, 65, 7, (0, 0)), (3, 63, 130, (1, 0)), (15, 1000, 48, (0, 0)), (16, 512, 96, (8, 8)),
                (17, 72, 129, (0, 0)), (33, 256, 1000, (0, 0)), (64, 200, 64, (0, 0)), (65, 1027, 33, (0, 0)), (100, 8, 8, (0, 0)), (127, 128, 256, (0, 0)),
                (129, 640, 264, (0, 0)), (257, 64, 520, (0, 5)), (300, 328, 392, (0, 0)), (512, 1024, 512, (0, 0)),
                # a strip of 512 columns, a tile, a chunk or a piece with one to seven entries in it
                (9, 24, 515, (0, 0)), (5, 1025, 1030, (0, 0)), (70, 129, 513, (3, 0)), (3, 9, 1031, (0, 0)), (131, 519, 65, (0, 1))]


def linear_inputs(T, t, rows, k, n, w8, seed, pad):
    x = strided(rand((rows, k), seed, t), *pad)[1]
    w = rand((n, k), seed + 1, t, k ** -0.5)
    if w8:
        q, s = rows8(w)
        q = strided(q, *pad)[1]
        return x, T.Matrix(q, s), ref.value(q, s)
    w = strided(w, *pad)[1]
    return x, T.Matrix(w), ref.value(w)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("w8", [False, True])
@pytest.mark.parametrize("rows,k,n,pad", LINEAR_SIZES)
def test_linear(T, ctx, dtype, w8, rows, k, n, pad):
    t = ref.DT[dtype]
    seed = rows + k + n
    x, mw, w64 = linear_inputs(T, t, rows, k, n, w8, seed, pad)
    bias, residual = rand((n,), seed + 2, t), strided(rand((rows, n), seed + 3, t), *pad)[1]
    work = space(ctx.linear_workspace(rows, k, n))
    z64 = x.double() @ w64.t() + bias.double()
    ez = ref.product_error(x.double().abs() @ w64.abs().t() + bias.double().abs(), k + 2)
    for act, code in ref.ACTS.items():
        ybuf, y = empty(rows, n, t, pad)
        zbuf, z = empty(rows, n, t, pad)
        ctx.linear(T.Matrix(x), mw, T.Matrix(y), bias=bias, activation=code, residual=T.Matrix(residual), z=T.Matrix(z), workspace=work)
        ctx.sync()
        y64 = ref.activate(z64, act) + residual.double()
        ok(z, z64, ez + ref.u(t) * (z64.abs() + ez) + ref.tiny(t))
        ey = 1.13 * ez + ref.activation_error(z64, act) + ref.E * y64.abs()      # no activation is steeper than 1.13
        ok(y, y64, ey + ref.u(t) * (y64.abs() + ey) + ref.tiny(t))
        assert untouched(ybuf, rows, n, pad) and untouched(zbuf, rows, n, pad)
    # without anything in the epilogue, and with y in the place of the residual
    bare, again = torch.empty(rows, n, dtype=t, device="cuda"), residual.clone()
    ctx.linear(T.Matrix(x), mw, T.Matrix(bare), workspace=work)
    ctx.linear(T.Matrix(x), mw, T.Matrix(again), residual=T.Matrix(again), workspace=work)
    ctx.sync()
    z64 = z64 - bias.double()
    ok(bare, z64, ez + ref.u(t) * (z64.abs() + ez) + ref.tiny(t))
    y64 = z64 + residual.double()
    ok(again, y64, ez + ref.E * y64.abs() + ref.u(t) * (y64.abs() + ez) + ref.tiny(t))


def backward_bounds(dy, z64, act, t, w64, x64, m_w, m_x, qw, qx, dx64, dw64):
    d = (dy * ref.slope(z64, act)).abs()
    e = dy.abs() * ref.slope_error(z64, act) + 2 * ref.E * d                # the unrounded gradient
    rows, n = d.shape
    bounds = {"dz": e + ref.u(t) * (d + e) + ref.tiny(t), "dbias": (e + (rows + 64) * ref.E * d).sum(0) + 1e-30}
    rounded = act != "none"
    for name, m, q, left, other, terms, want in (("dx", m_w, qw, lambda v: v, w64, n, dx64), ("dw", m_x, qx, lambda v: v.t(), x64, rows, dw64)):
        if want is None:
            continue
        r = (ref.u(t) + 3 * ref.E) * (d + e) + e if rounded or m is not None else torch.zeros_like(d)
        err = left(r) @ other.abs()
        # a factor under float16's normal range is off by half its smallest step, in units of m
        if m is not None:
            err = err + left(torch.full_like(d, ref.tiny(t) * m)) @ q.abs()
        elif rounded:
            err = err + left(torch.full_like(d, ref.tiny(t))) @ other.abs()
        err = err + ref.product_error(left(d + r) @ other.abs(), terms)
        bounds[name] = err + ref.u(t) * (want.abs() + err) + ref.tiny(t)
    return bounds


def power_above(s):
    return 2.0 ** (torch.floor(torch.log2(s.max())).item() + 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act,w8,x8,z8", [("none", False, False, False), ("none", True, True, False), ("gelu", False, True, True), ("silu", True, False, True),
                                          ("relu", True, True, False), ("gelu", False, False, False)])
@pytest.mark.parametrize("rows,k,n,pad", LINEAR_SIZES)
def test_linear_gradients(T, ctx, dtype, act, w8, x8, z8, rows, k, n, pad):
    t = ref.DT[dtype]
    seed = rows + 2 * k + 3 * n
    x, mw, w64 = linear_inputs(T, t, rows, k, n, w8, seed, pad)
    mx, x64, qx, m_x = T.Matrix(x), ref.value(x), None, None
    if x8:
        q, s = rows8(x)
        q = strided(q, *pad)[1]
        mx, x64, qx, m_x = T.Matrix(q, s), ref.value(q, s), q.double(), power_above(s)
    m_w, qw = (power_above(mw.scale), mw.tensor.double()) if w8 else (None, None)
    dy = strided(rand((rows, n), seed + 5, t), *pad)[1]
    z64, mz, dz, mdz = torch.zeros(rows, n, device="cuda", dtype=torch.float64), None, None, None
    if act != "none":
        z = strided(rand((rows, n), seed + 6, t, 2.0), *pad)[1]
        mz, z64 = T.Matrix(z), ref.value(z)
        if z8:
            q, s = rows8(z)
            q = strided(q, *pad)[1]
            mz, z64 = T.Matrix(q, s), ref.value(q, s)
        dzbuf, dz = empty(rows, n, t, pad)
        mdz = T.Matrix(dz)
    dxbuf, dx = empty(rows, k, t, pad)
    dwbuf, dw = empty(n, k, t, pad)
    db = torch.full((n + 1,), 7.0, device="cuda")
    work = space(ctx.linear_backward_workspace(rows, k, n))
    ctx.linear_backward(T.Matrix(dy), mx, mw, ref.ACTS[act], mz, mdz, T.Matrix(dx), T.Matrix(dw), db[:n], work)
    ctx.sync()
    d64 = dy.double() * ref.slope(z64, act)
    dx64, dw64 = d64 @ w64, d64.t() @ x64
    e = backward_bounds(dy.double(), z64, act, t, w64, x64, m_w, m_x, qw, qx, dx64, dw64)
    if dz is not None:
        ok(dz, d64, e["dz"])
        assert untouched(dzbuf, rows, n, pad)
    ok(dx, dx64, e["dx"])
    ok(dw, dw64, e["dw"])
    ok(db[:n], d64.sum(0), e["dbias"])
    assert untouched(dxbuf, rows, k, pad) and untouched(dwbuf, n, k, pad) and db[n] == 7
    # each gradient asked for alone is the same
    one, two, three = torch.empty(rows, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda"), torch.empty(n, device="cuda")
    mdz2 = T.Matrix(torch.empty(rows, n, dtype=t, device="cuda")) if act != "none" else None
    ctx.linear_backward(T.Matrix(dy), None, mw, ref.ACTS[act], mz, mdz2, dx=T.Matrix(one), workspace=work)
    ctx.linear_backward(T.Matrix(dy), mx, None, ref.ACTS[act], mz, mdz2, dw=T.Matrix(two), workspace=work)
    ctx.linear_backward(T.Matrix(dy), None, None, ref.ACTS[act], mz, mdz2, dbias=three, workspace=work)
    ctx.sync()
    assert torch.equal(one, dx) and torch.equal(two, dw) and torch.equal(three, db[:n])
    if act != "none":                                       # dz in the place of dy
        ctx.linear_backward(T.Matrix(dy), mx, mw, ref.ACTS[act], mz, T.Matrix(dy), T.Matrix(one), workspace=work)
        ctx.sync()
        assert torch.equal(dy, dz) and torch.equal(one, dx)


@pytest.mark.parametrize("dtype", DTYPES)
def test_values_before_the_activation_that_overflowed(T, ctx, dtype):
    """activations and slopes at infinities, far values and NaN, through the identity as weights"""
    t = ref.DT[dtype]
    inf, nan = float("inf"), float("nan")
    vals = torch.tensor([inf, -inf, 1e4, -1e4, 90.0, -90.0, 20.0, -20.0, 0.0, -0.0, nan, 1.0, -1.0, 5.0, -5.0, 0.25], device="cuda").to(t)
    eye = torch.eye(16, device="cuda").to(t)
    zero = torch.zeros(16, 16, device="cuda").to(t)
    for act, code in ref.ACTS.items():
        y = torch.empty(16, 16, dtype=t, device="cuda")
        ctx.linear(T.Matrix(zero), T.Matrix(eye), T.Matrix(y), bias=vals, activation=code)
        dz = torch.empty_like(y)
        if act != "none":
            ctx.linear_backward(T.Matrix(torch.ones_like(y)), None, None, code, T.Matrix(vals.repeat(16, 1)), T.Matrix(dz),
                                workspace=space(ctx.linear_backward_workspace(16, 1, 16)))
        ctx.sync()
        far = {"none": [inf, -inf], "relu": [inf, 0.0], "gelu": [inf, 0.0], "silu": [inf, 0.0]}[act]
        assert y[3, :2].tolist() == far and torch.isnan(y[3, 10])
        keep = [i for i in range(2, 16) if i != 10]
        v = vals[keep].double()
        want = ref.activate(v, act)
        ok(y[5][keep], want, ref.u(t) * want.abs() + ref.activation_error(v, act) + ref.tiny(t))
        if act != "none":
            assert dz[0, :2].tolist() == [1.0, 0.0] and torch.isnan(dz[0, 10])
            want = ref.slope(v, act)
            ok(dz[2][keep], want, ref.u(t) * want.abs() + ref.slope_error(v, act) + ref.tiny(t))


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_row_that_is_not_a_number_stays_alone(T, ctx, dtype):
    """rows and weights beside a NaN, and what lies behind the last column of a row, do not reach other results"""
    t = ref.DT[dtype]
    for rows, k, n in ((5, 72, 40), (70, 100, 200), (150, 264, 136)):
        buf = torch.full((rows, k + 8), float("nan"), device="cuda", dtype=t)
        x = buf[:, :k]
        x.copy_(rand((rows, k), 1, t))
        wbuf = torch.full((n, k + 8), float("nan"), device="cuda", dtype=t)
        w = wbuf[:, :k]
        w.copy_(rand((n, k), 2, t))
        y = torch.empty(rows, n, dtype=t, device="cuda")
        work = space(ctx.linear_workspace(rows, k, n))
        ctx.linear(T.Matrix(x), T.Matrix(w), T.Matrix(y), workspace=work)
        ctx.sync()
        assert torch.isfinite(y).all()
        x[3, 1], w[7, 2] = float("nan"), float("inf")
        ctx.linear(T.Matrix(x), T.Matrix(w), T.Matrix(y), workspace=work)
        ctx.sync()
        bad = ~torch.isfinite(y)
        assert bad[3].all() and bad[:, 7].all() and bad.sum() == n + rows - 1
        gbuf = torch.full((rows, n + 8), float("nan"), device="cuda", dtype=t)
        dy = gbuf[:, :n]
        dy.copy_(rand((rows, n), 3, t))
        x.copy_(rand((rows, k), 1, t))
        w.copy_(rand((n, k), 2, t))
        dx, dw = torch.empty(rows, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda")
        work = space(ctx.linear_backward_workspace(rows, k, n))
        ctx.linear_backward(T.Matrix(dy), T.Matrix(x), T.Matrix(w), dx=T.Matrix(dx), dw=T.Matrix(dw), workspace=work)
        ctx.sync()
        assert torch.isfinite(dx).all() and torch.isfinite(dw).all()
        dy[4, 9] = float("nan")
        ctx.linear_backward(T.Matrix(dy), T.Matrix(x), T.Matrix(w), dx=T.Matrix(dx), dw=T.Matrix(dw), workspace=work)
        ctx.sync()
        assert torch.isnan(dx[4]).all() and torch.isnan(dx).sum() == k and torch.isnan(dw[9]).all() and torch.isnan(dw).sum() == k


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,n", [(3, 64, 48), (70, 72, 65), (3, 65, 33)])
def test_the_smallest_values_are_not_lost(T, ctx, dtype, rows, k, n):
    """entries below the type's normal range, in products by one: the results are they themselves"""
    t = ref.DT[dtype]
    least = torch.finfo(t).smallest_normal * torch.finfo(t).eps
    x = (torch.arange(rows * k, device="cuda").reshape(rows, k) % 15 - 7).double() * least
    x = x.to(t)
    w = torch.eye(n, k, device="cuda").to(t)
    y = torch.empty(rows, n, dtype=t, device="cuda")
    ctx.linear(T.Matrix(x), T.Matrix(w), T.Matrix(y), workspace=space(ctx.linear_workspace(rows, k, n)))
    ctx.sync()
    m = min(k, n)
    assert torch.equal(y[:, :m], x[:, :m]) and not y[:, m:].any()


def test_small_gradients_of_float16_through_scales(T, ctx):
    """scales of 2^-20 and gradients of 2^-10: their product alone would be lost in float16"""
    t = torch.float16
    rows, k, n = 40, 64, 48
    q, s = rows8(rand((n, k), 1, t))
    s = s * 2.0 ** -14
    dy = rand((rows, n), 2, t, 2.0 ** -10)
    x8 = rows8(rand((rows, k), 3, t))
    sx = x8[1] * 2.0 ** -10
    dx, dw = torch.empty(rows, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda")
    big = torch.full((rows, n), 2.0 ** 12, device="cuda").to(t)
    ctx.linear_backward(T.Matrix(dy * big), T.Matrix(x8[0], sx), T.Matrix(q, s), dx=T.Matrix(dx), dw=T.Matrix(dw), workspace=space(ctx.linear_backward_workspace(rows, k, n)))
    ctx.sync()
    d = (dy * big).double()
    w64, x64 = ref.value(q, s), ref.value(x8[0], sx)
    e = backward_bounds(d, d * 0, "none", t, w64, x64, power_above(s), power_above(sx), q.double(), x8[0].double(), d @ w64, d.t() @ x64)
    ok(dx, d @ w64, e["dx"])
    ok(dw, d.t() @ x64, e["dw"])
    rel = ((dw.double() - d.t() @ x64).norm() / (d.t() @ x64).norm()).item()
    assert rel < 2.0 ** -11


# ---- used together -------------------------------------------------------------------------------------------------
class Block:
    """A feed-forward block as a program runs it: norm, up product with its activation, down product added to the residual stream; what
    the backward pass needs is kept in 8 bits."""

    def __init__(self, T, ctx, t, rows, d, f, seed):
        self.T, self.ctx, self.t = T, ctx, t
        self.gamma, self.beta = (rand((d,), seed, t, 0.1) + 1).to(t), rand((d,), seed + 1, t, 0.1)
        self.w1, self.b1, self.w2 = rand((f, d), seed + 2, t, d ** -0.5), rand((f,), seed + 3, t, 0.1), rand((d, f), seed + 4, t, f ** -0.5)
        e = lambda *s, dt=t: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        f32, i8 = torch.float32, torch.int8
        self.h, self.z, self.a, self.y = e(rows, d), e(rows, f), e(rows, f), e(rows, d)
        self.mean, self.rstd = e(rows, dt=f32), e(rows, dt=f32)
        self.x8, self.h8, self.z8, self.a8 = [(e(rows, c, dt=i8), e(rows, dt=f32)) for c in (d, d, f, f)]
        self.da, self.dz, self.dh, self.dx = e(rows, f), e(rows, f), e(rows, d), e(rows, d)
        self.dw1, self.dw2, self.db1 = e(f, d), e(d, f), e(f, dt=f32)
        self.dgamma, self.dbeta = e(d, dt=f32), e(d, dt=f32)
        need = max(ctx.linear_workspace(rows, d, f), ctx.linear_workspace(rows, f, d), ctx.linear_backward_workspace(rows, d, f),
                   ctx.linear_backward_workspace(rows, f, d), ctx.norm_backward_workspace(rows, d))
        self.work = space(need)

    def forward(self, x):
        M, c = self.T.Matrix, self.ctx
        c.checkpoint_encode(M(x), M(*self.x8))
        c.norm(0, M(x), self.gamma, self.beta, 1e-5, M(self.h), self.mean, self.rstd)
        c.checkpoint_encode(M(self.h), M(*self.h8))
        c.linear(M(self.h), M(self.w1), M(self.a), bias=self.b1, activation=2, z=M(self.z), workspace=self.work)
        c.checkpoint_encode(M(self.z), M(*self.z8))
        c.checkpoint_encode(M(self.a), M(*self.a8))
        c.linear(M(self.a), M(self.w2), M(self.y), residual=M(x), workspace=self.work)

    def backward(self, dy):
        M, c = self.T.Matrix, self.ctx
        c.linear_backward(M(dy), M(*self.a8), M(self.w2), dx=M(self.da), dw=M(self.dw2), workspace=self.work)
        c.linear_backward(M(self.da), M(*self.h8), M(self.w1), 2, M(*self.z8), M(self.dz), M(self.dh), M(self.dw1), self.db1, self.work)
        c.norm_backward(0, M(self.dh), M(*self.x8), self.gamma, self.mean, self.rstd, M(self.dx), self.dgamma, self.dbeta, self.work)

    def outputs(self):
        return [self.y, self.dx, self.dw1, self.dw2, self.db1, self.dgamma, self.dbeta, *self.x8, *self.h8, *self.z8, *self.a8]


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_block_its_gradients_and_its_commitments(T, ctx, dtype):
    """Forward and backward of a block; the gradients are those of the 64-bit definitions at the values that the checkpoints stand
    for, and the checkpoints are committed as they lie and opened to the bytes that the gradients were taken from."""
    from gpu_util import TAU_BYTES, pps
    from oracle import bls12_381 as ec
    from oracle import cbind

    t = ref.DT[dtype]
    rows, d, f = 37, 64, 176
    b = Block(T, ctx, t, rows, d, f, 40)
    x, dy = rand((rows, d), 50, t), rand((rows, d), 51, t)
    b.forward(x)
    b.backward(dy)
    ctx.sync()
    v = [ref.value(*e) for e in (b.x8, b.h8, b.z8, b.a8)]
    da = dy.double() @ b.w2.double()
    dz = da * ref.slope(v[2], "gelu")
    dh = dz @ b.w1.double()
    dx, dg, db = ref.norm_backward(dh, v[0], b.gamma.double(), b.mean.double(), b.rstd.double(), True)
    want = {"dw2": dy.double().t() @ v[3], "dw1": dz.t() @ v[1], "db1": dz.sum(0), "dx": dx, "dgamma": dg, "dbeta": db}
    for name, w in want.items():
        rel = ((getattr(b, name).double() - w).norm() / w.norm()).item()
        assert rel < 4 * ref.u(t), (name, rel)              # at most four roundings to the type on the longest way
    y = ref.value(x) + ref.activate(ref.norm(ref.value(x), b.gamma.double(), b.beta.double(), 1e-5, True)[0] @ b.w1.double().t() + b.b1.double(), "gelu") @ b.w2.double().t()
    assert ((b.y.double() - y).norm() / y.norm()).item() < 4 * ref.u(t)
    for q, _ in (b.x8, b.z8):
        srs = ctx.setup_from_trapdoor(TAU_BYTES, tuple(q.shape), T.TC_SRS_SUFFIX)
        C = ctx.commit(srs, q, T.TC_I8)
        assert C == ec.g1_to_bytes(cbind.commit(pps(tuple(q.shape)), q.cpu().numpy()))
        value, _ = ctx.open(srs, q, T.TC_I8, (3, 5))
        assert value == ec.fr_to_bytes(int(q[3, 5].item()) % ec.R)
        srs.close()


def test_equal_calls_give_equal_bytes(T, ctx):
    t = torch.bfloat16
    b = Block(T, ctx, t, 300, 512, 1408, 60)
    x, dy = rand((300, 512), 61, t), rand((300, 512), 62, t)
    seen = None
    for _ in range(3):
        b.forward(x)
        b.backward(dy)
        ctx.sync()
        got = [o.clone() for o in b.outputs()]
        assert seen is None or all(torch.equal(p, q) for p, q in zip(seen, got))
        seen = got
        b.work.fill_(0xFF)                                  # what a workspace held before does not matter


def test_captured_and_replayed(T):
    """the block captured into a graph on a stream of its own, replayed on new inputs between eager runs, each replay against the eager result"""
    t = torch.float16
    stream = torch.cuda.Stream()
    c = T.Context(0, stream.cuda_stream)
    x, dy = rand((130, 256), 1, t), rand((130, 256), 2, t)
    torch.cuda.synchronize()
    b = Block(T, c, t, 130, 256, 704, 70)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        b.forward(x)
        b.backward(dy)
    stream.synchronize()
    before = c.alloc_calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.forward(x)
        b.backward(dy)
    assert c.alloc_calls() == before
    for i in range(4):
        x.copy_(rand((130, 256), 10 + i, t))
        dy.copy_(rand((130, 256), 20 + i, t))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            b.forward(x)
            b.backward(dy)
        stream.synchronize()
        want = [o.clone() for o in b.outputs()]
        for o in b.outputs():
            o.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, b.outputs())), i
    c.close()


def test_two_streams_at_once(T):
    """two contexts on streams of their own, a workspace each, work that overlaps"""
    t = torch.bfloat16
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    ctxs = [T.Context(0, s.cuda_stream) for s in streams]
    blocks = [Block(T, c, t, 260, 512, 1024, 80 + i) for i, c in enumerate(ctxs)]
    xs, dys = [rand((260, 512), 90 + i, t) for i in range(2)], [rand((260, 512), 92 + i, t) for i in range(2)]
    torch.cuda.synchronize()
    want = []
    for b, x, dy in zip(blocks, xs, dys):
        b.forward(x)
        b.backward(dy)
        torch.cuda.synchronize()
        want.append([o.clone() for o in b.outputs()])
    for _ in range(3):
        for b in blocks:
            for o in b.outputs():
                o.fill_(3)
        torch.cuda.synchronize()
        for b, x in zip(blocks, xs):
            b.forward(x)
        for b, dy in zip(blocks, dys):
            b.backward(dy)
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            assert all(torch.equal(p, q) for p, q in zip(w, b.outputs()))
    for c in ctxs:
        c.close()


def test_offsets_past_32_bits(T, ctx):
    """rows that start more than 2^32 elements into a buffer: views of a few rows with a wide stride"""
    t = torch.float16
    ld = 1 << 30
    rows, k, n = 6, 64, 40
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 26 GB of device memory")
    buf = torch.empty(rows * ld, dtype=t, device="cuda").view(rows, ld)
    x, y, z = buf[:, :k], buf[:, 128:128 + k], buf[:, 256:256 + n]
    x.copy_(rand((rows, k), 1, t))
    w = rand((n, k), 2, t)
    ctx.norm(0, T.Matrix(x), None, None, 1e-5, T.Matrix(y))
    ctx.linear(T.Matrix(x), T.Matrix(w), T.Matrix(z), workspace=space(ctx.linear_workspace(rows, k, n)))
    dx, dw = buf[:, 384:384 + k], torch.empty_like(w)
    ctx.linear_backward(T.Matrix(z), T.Matrix(x), T.Matrix(w), dx=T.Matrix(dx), dw=T.Matrix(dw), workspace=space(ctx.linear_backward_workspace(rows, k, n)))
    q8 = torch.empty(rows * ld, dtype=torch.int8, device="cuda").view(rows, ld)
    q, s = q8[:, 8:8 + k], torch.empty(rows, device="cuda")
    ctx.checkpoint_encode(T.Matrix(x), T.Matrix(q, s))
    ctx.sync()
    x64, w64 = x.double(), w.double()
    want, _, rstd = ref.norm(x64, None, None, 1e-5, True)
    ok(y, want, ref.norm_bound(x64, None, None, want, rstd, t, True))
    z64 = x64 @ w64.t()
    ez = ref.product_error(x64.abs() @ w64.abs().t(), k)
    ok(z, z64, ez + ref.u(t) * (z64.abs() + ez) + ref.tiny(t))
    d = z.double()
    e = backward_bounds(d, d * 0, "none", t, w64, x64, None, None, None, None, d @ w64, d.t() @ x64)
    ok(dx, d @ w64, e["dx"])
    ok(dw, d.t() @ x64, e["dw"])
    assert torch.equal(q, ref.encode(x)[0])


# every layout of a product and every way of splitting it: sizes at which each of them is the cheapest for one of the three products
LARGE = [(8200, 136, 8456), (8200, 8456, 136), (136, 8456, 8200), (487, 4104, 4104), (4104, 1040, 1040), (300, 4104, 520), (200, 200, 4104), (1100, 2056, 520),
         # whole rounds of the largest tiles and the rest by others: cut along either axis, in each of the three products
         (8456, 520, 8200), (10248, 520, 8200), (8456, 8200, 520), (10248, 8200, 520), (520, 8200, 8456), (520, 8200, 10248)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("rows,k,n", LARGE)
def test_products_of_every_layout(T, ctx, dtype, eight, rows, k, n):
    t = ref.DT[dtype]
    seed = rows + 5 * k + 7 * n
    x, mw, w64 = linear_inputs(T, t, rows, k, n, eight, seed, (0, 0))
    work = space(ctx.linear_workspace(rows, k, n))
    work.fill_(0xFF)
    bias, residual = rand((n,), seed + 2, t), rand((rows, n), seed + 3, t)
    ybuf, y = empty(rows, n, t)
    z = torch.empty(rows, n, dtype=t, device="cuda")
    ctx.linear(T.Matrix(x), mw, T.Matrix(y), bias=bias, activation=T.TC_ACT_GELU, residual=T.Matrix(residual), z=T.Matrix(z), workspace=work)
    ctx.sync()
    z64 = x.double() @ w64.t() + bias.double()
    ez = ref.product_error(x.double().abs() @ w64.abs().t() + bias.double().abs(), k + 2)
    ok(z, z64, ez + ref.u(t) * (z64.abs() + ez) + ref.tiny(t))
    y64 = ref.activate(z64, "gelu") + residual.double()
    ey = 1.13 * ez + ref.activation_error(z64, "gelu") + ref.E * y64.abs()
    ok(y, y64, ey + ref.u(t) * (y64.abs() + ey) + ref.tiny(t))
    assert untouched(ybuf, rows, n)
    del z64, ez, y64, ey
    mx, x64, qx, m_x = T.Matrix(x), ref.value(x), None, None
    if eight:
        q, s = rows8(x)
        mx, x64, qx, m_x = T.Matrix(q, s), ref.value(q, s), q.double(), power_above(s)
    m_w, qw = (power_above(mw.scale), mw.tensor.double()) if eight else (None, None)
    dy = rand((rows, n), seed + 5, t)
    dxbuf, dx = empty(rows, k, t)
    dwbuf, dw = empty(n, k, t)
    db = torch.empty(n, device="cuda")
    work = space(ctx.linear_backward_workspace(rows, k, n))
    work.fill_(0xFF)
    ctx.linear_backward(T.Matrix(dy), mx, mw, dx=T.Matrix(dx), dw=T.Matrix(dw), dbias=db, workspace=work)
    ctx.sync()
    d64 = dy.double()
    dx64, dw64 = d64 @ w64, d64.t() @ x64
    e = backward_bounds(d64, torch.zeros_like(d64), "none", t, w64, x64, m_w, m_x, qw, qx, dx64, dw64)
    ok(dx, dx64, e["dx"])
    ok(dw, dw64, e["dw"])
    ok(db, d64.sum(0), e["dbias"])
    assert untouched(dxbuf, rows, k) and untouched(dwbuf, n, k)


def test_more_rows_than_a_launch_has_workgroups(T, ctx):
    t = torch.float16
    rows = (1 << 24) + 77
    x = rand((rows, 8), 1, t)
    q, s, back, y = torch.empty(rows, 8, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x), torch.empty_like(x)
    ctx.checkpoint_encode(T.Matrix(x), T.Matrix(q, s))
    ctx.checkpoint_decode(T.Matrix(q, s), T.Matrix(back))
    ctx.norm(1, T.Matrix(x), None, None, 1e-5, T.Matrix(y))
    ctx.sync()
    want, scale = ref.encode(x)
    assert torch.equal(q, want) and torch.equal(s, scale)
    v = ref.value(want, scale)
    ok(back, v, (ref.u(t) + 2 * ref.E) * v.abs() + ref.tiny(t))
    del v
    x64 = x.double()
    want, _, rstd = ref.norm(x64, None, None, 1e-5, False)
    ok(y, want, ref.norm_bound(x64, None, None, want, rstd, t, False))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_the_greatest_length(T, ctx, dtype):
    most = 1 << 20
    test_checkpoints(T, ctx, dtype, 2, most, (0, 0))
    for rows, k, n in [(3, most, 16), (3, 16, most), (16, most - 1, 5), (17, 5, most - 1)]:
        for w8 in (False, True):
            test_linear(T, ctx, dtype, w8, rows, k, n, (0, 0))
        test_linear_gradients(T, ctx, dtype, "none", False, False, False, rows, k, n, (0, 0))
        test_linear_gradients(T, ctx, dtype, "gelu", True, True, True, rows, k, n, (0, 0))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad", [(8, 8), (16, 0), (1, 2)])
@pytest.mark.parametrize("rows,k,n", [(1, 64, 96), (3, 7, 5), (5, 8, 9), (37, 72, 40), (65, 200, 264), (130, 1027, 513), (300, 4104, 520), (1100, 2056, 520)])
def test_what_lies_between_the_rows_does_not_matter(T, ctx, dtype, rows, k, n, pad):
    """the same bytes from buffers whose other columns hold sevens, NaNs and infinities"""
    t = ref.DT[dtype]
    x, w, dy, z = rand((rows, k), 1, t), rand((n, k), 2, t, k ** -0.5), rand((rows, n), 3, t), rand((rows, n), 4, t)
    x8, w8, z8 = rows8(x), rows8(w), rows8(z)
    work = space(max(ctx.linear_workspace(rows, k, n), ctx.linear_backward_workspace(rows, k, n), ctx.norm_backward_workspace(rows, k)))
    seen = None
    for between, between8 in ((7, 7), (float("nan"), -128), (float("inf"), 127)):
        M = lambda m: T.Matrix(strided(m, *pad, sentinel=between)[1])  # noqa: E731
        M8 = lambda m: T.Matrix(strided(m[0], *pad, sentinel=between8)[1], m[1])  # noqa: E731
        e = lambda *s, dt=t: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
        got = []
        for mx, mw, mz in ((M(x), M(w), M(z)), (M8(x8), M8(w8), M8(z8))):
            mean, rstd, h, dh, dg, db = e(rows, dt=torch.float32), e(rows, dt=torch.float32), e(rows, k), e(rows, k), e(k, dt=torch.float32), e(k, dt=torch.float32)
            ctx.norm(0, mx, None, None, 1e-5, T.Matrix(h), mean, rstd)
            ctx.norm_backward(0, M(x), mx, None, mean, rstd, T.Matrix(dh), dg, db, work)
            y, dz, dx, dw, dbias = e(rows, n), e(rows, n), e(rows, k), e(n, k), e(n, dt=torch.float32)
            ctx.linear(M(x), mw, T.Matrix(y), residual=M(dy), workspace=work)
            ctx.linear_backward(M(dy), mx, mw, 2, mz, T.Matrix(dz), T.Matrix(dx), T.Matrix(dw), dbias, work)
            bare, dw2 = e(rows, k), e(n, k)
            ctx.linear_backward(M(dy), mx, mw, dx=T.Matrix(bare), dw=T.Matrix(dw2), workspace=work)
            q, s, back = e(rows, k, dt=torch.int8), e(rows, dt=torch.float32), e(rows, k)
            ctx.checkpoint_encode(M(x), T.Matrix(q, s))
            ctx.checkpoint_decode(M8(x8), T.Matrix(back))
            ctx.sync()
            got += [mean, rstd, h, dh, dg, db, y, dz, dx, dw, dbias, bare, dw2, q, s, back]
        assert all(bool(torch.isfinite(g.float()).all()) for g in got)
        assert seen is None or [i for i, (p, q) in enumerate(zip(seen, got)) if not torch.equal(p, q)] == []
        seen = got


def test_tensors_that_are_elsewhere_are_refused(T, ctx):
    t = torch.float16
    x, far = torch.zeros(4, 8, dtype=t, device="cuda"), torch.zeros(4, 8, dtype=t)
    m, bad = T.Matrix(x), T.Matrix(far)
    square, v = T.Matrix(torch.zeros(8, 8, dtype=t, device="cuda")), torch.zeros(8)
    for call in (lambda: ctx.norm(0, bad, None, None, 1e-5, m), lambda: ctx.norm(0, m, None, None, 1e-5, bad),
                 lambda: ctx.norm(0, m, v.to(t), None, 1e-5, m), lambda: ctx.norm(0, m, None, None, 1e-5, m, v, None),
                 lambda: ctx.checkpoint_encode(bad, m), lambda: ctx.checkpoint_decode(m, bad),
                 lambda: ctx.linear(bad, square, m), lambda: ctx.linear(m, square, m, residual=bad), lambda: ctx.linear(m, square, m, bias=v.to(t)),
                 lambda: ctx.linear(m, square, m, workspace=torch.zeros(1 << 16, dtype=torch.uint8)),
                 lambda: ctx.linear_backward(m, None, square, dx=bad, workspace=space(1 << 20)),
                 lambda: ctx.linear_backward(m, None, square, dbias=v, workspace=space(1 << 20)),
                 lambda: ctx.norm_backward(1, m, m, None, None, v, m, None, None, None)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [4096, 4101])
def test_outputs_larger_than_the_caches_keep(T, ctx, dtype, width):
    """outputs of 128 MB and more, which are written past the caches, with rows at any alignment"""
    test_checkpoints(T, ctx, dtype, 16400, width, (0, 0))
    test_norm_and_its_gradient(T, ctx, dtype, "layer", 16400, width, (1, 2))
    test_linear(T, ctx, dtype, True, 16400, 40, width, (1, 2))
    test_linear_gradients(T, ctx, dtype, "none", True, False, False, 16400, width, 40, (1, 2))
    test_linear_gradients(T, ctx, dtype, "gelu", False, True, True, 40, 16400, width, (0, 0))


def spread_inputs(t, rows, k, n, spread, size, quiet, act, seed):
    """x and w as int8 rows of which some stand out by `spread` (one large entry, as a first token has), gradients of the given size, zero for those rows
    and outputs where `quiet`"""
    x, w, dy = rand((rows, k), seed, t), rand((n, k), seed + 1, t, k ** -0.5), rand((rows, n), seed + 2, t, size)
    loud_x, loud_w = torch.arange(0, rows, 37, device="cuda"), torch.arange(0, n, 41, device="cuda")
    x[loud_x, loud_x % k], w[loud_w, loud_w % k] = 3.0 * spread, 3.0 * k ** -0.5 * spread
    if quiet:
        dy[loud_x], dy[:, loud_w] = 0, 0
    z = rand((rows, n), seed + 3, t) if act != "none" else None
    return rows8(x), rows8(w), dy, z


# a wave's worth, rows of fewer than eight entries and of no whole pieces, sums in several parts, and each kind of tile
SPREAD = [(40, 64, 48), (9, 5, 7), (70, 65, 33), (300, 200, 520), (487, 1032, 1096), (520, 8200, 8456), (8456, 520, 8200)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,n", SPREAD)
@pytest.mark.parametrize("act,spread,size,quiet", [("none", 2.0 ** 4, 1e-2, False), ("none", 2.0 ** 9, 1e-3, True), ("gelu", 2.0 ** 12, 1e-3, False), ("none", 2.0 ** 14, 1e-4, True)])
def test_gradients_through_scales_that_differ_widely(T, ctx, dtype, rows, k, n, act, spread, size, quiet):
    """A row whose scale stands out costs the others nothing.  The gradient times what its scale has beside a power of two, a number from 1/2 to 1, is rounded to the
    type: half a step of it, and below the normal range half the smallest step, which is at most a whole one in units of the gradient."""
    t = ref.DT[dtype]
    qx, qw, dy, z = spread_inputs(t, rows, k, n, spread, size, quiet, act, rows + k + n)
    mz, mdz = (T.Matrix(z), T.Matrix(torch.empty_like(dy))) if z is not None else (None, None)
    dx, dw = torch.empty(rows, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda")
    work = space(ctx.linear_backward_workspace(rows, k, n))
    work.fill_(0xFF)
    ctx.linear_backward(T.Matrix(dy), T.Matrix(*qx), T.Matrix(*qw), ref.ACTS[act], mz, mdz, T.Matrix(dx), T.Matrix(dw), workspace=work)
    ctx.sync()
    x64, w64, d64 = ref.value(*qx), ref.value(*qw), dy.double()
    e = torch.zeros_like(d64)
    if z is not None:
        s = ref.slope(z.double(), act)
        e = d64.abs() * ref.slope_error(z.double(), act) + 2 * ref.E * (d64 * s).abs()
        d64 = d64 * s
    off = (ref.u(t) + 3 * ref.E) * (d64.abs() + e) + e + 2 * ref.tiny(t)
    for got, left, right, terms in ((dx, (d64, off), w64, n), (dw, (d64.t(), off.t()), x64, rows)):
        want = left[0] @ right
        err = left[1] @ right.abs()
        err = err + ref.product_error((left[0].abs() + left[1]) @ right.abs(), terms)
        ok(got, want, err + ref.u(t) * (want.abs() + err) + ref.tiny(t))
        if quiet:                                           # the rows that stand out add nothing: what the others give is as exact as ever
            # (a rounding of the gradient and one of the result, each at most half a step; below the normal range a step of it against its size)
            rel = (got.double() - want).norm() / want.norm()
            assert rel < 2 * ref.u(t) + 4 * ref.tiny(t) / size + ref.tiny(t) * want.numel() ** 0.5 / want.norm(), rel


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,n", [(40, 64, 48), (70, 65, 33), (520, 8200, 8456)])
def test_gradients_through_scales_of_every_kind(T, ctx, dtype, rows, k, n):
    """scales of zero, below zero, below the normal range, and so far below the largest that their rows show only because its gradient is zero"""
    t = ref.DT[dtype]
    (qx, sx), (qw, sw) = rows8(rand((rows, k), 1, t)), rows8(rand((n, k), 2, t))
    dy = rand((rows, n), 3, t)
    top = torch.tensor([1.0, 0.0, -1.0, 2.0 ** -31, -2.0 ** -33, 2.0 ** -38, 1e-40, 2.0 ** -32], device="cuda")
    sx = (2.0 ** 31 * top[torch.arange(rows, device="cuda") % 8]) * (sx / sx.max())
    sw = (2.0 ** 28 * top[torch.arange(n, device="cuda") % 8]) * (sw / sw.max())
    dy[sx.abs() > 2.0 ** 10], dy[:, sw.abs() > 2.0 ** 10] = 0, 0
    dx, dw = torch.empty(rows, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda")
    ctx.linear_backward(T.Matrix(dy), T.Matrix(qx, sx), T.Matrix(qw, sw), dx=T.Matrix(dx), dw=T.Matrix(dw), workspace=space(ctx.linear_backward_workspace(rows, k, n)))
    ctx.sync()
    d64, x64, w64 = dy.double(), ref.value(qx, sx), ref.value(qw, sw)
    for got, left, right, scale, terms in ((dx, d64, w64, sw[None, :], n), (dw, d64.t(), x64, sx[None, :], rows)):
        # beyond 2^32 below the largest a scale's rest is with the gradient, whose smallest step counts for that much more
        size = scale.double().abs()
        below = torch.where(size == 0, torch.ones_like(size), size.max() / size * 2.0 ** -31).clamp(min=1)
        off = (ref.u(t) + 3 * ref.E) * left.abs() + 2 * ref.tiny(t) * below
        want = left @ right
        err = off @ right.abs()
        err = err + ref.product_error((left.abs() + off) @ right.abs(), terms)
        ok(got, want, err + ref.u(t) * (want.abs() + err) + ref.tiny(t))
        assert got.any()
    for bad in (float("nan"), float("inf")):                # not a number in, none out: in its own sum over the rows, which is every one of dw
        sx[3] = bad
        dy[3] = 1
        ctx.linear_backward(T.Matrix(dy), T.Matrix(qx, sx), None, dw=T.Matrix(dw), workspace=space(ctx.linear_backward_workspace(rows, k, n)))
        ctx.sync()
        assert not torch.isfinite(dw).any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act,least", [("gelu", 13.0), ("silu", 80.0)])
def test_activations_far_below_zero_are_rounded_once(T, ctx, dtype, act, least):
    """Every number of the type from -least to 0, against a bound relative to the result.  The exponential's argument has three roundings (two for silu), so it is
    off by 1.5 z^2 (2 |z|) half steps of float32; 24 (8) more for the tail's fit, its terms, the reciprocal and the products."""
    t = ref.DT[dtype]
    z = torch.arange(0, 1 << 15, device="cuda").to(torch.int16).view(t)
    z = -z[torch.isfinite(z) & (z <= least)]
    n, zero = z.numel(), torch.zeros(1, 8, device="cuda", dtype=t)
    y, dz = torch.empty(1, n, dtype=t, device="cuda"), torch.empty(1, n, dtype=t, device="cuda")
    w = torch.zeros(n, 8, device="cuda", dtype=t)
    ctx.linear(T.Matrix(zero), T.Matrix(w), T.Matrix(y), bias=z, activation=ref.ACTS[act], workspace=space(ctx.linear_workspace(1, 8, n)))
    ctx.linear_backward(T.Matrix(torch.ones_like(y)), None, None, ref.ACTS[act], T.Matrix(z[None, :]), T.Matrix(dz), workspace=space(ctx.linear_backward_workspace(1, 8, n)))
    ctx.sync()
    v = z.double()
    rel = ((1.5 * v * v + 24) if act == "gelu" else (2 * v.abs() + 8)) * ref.E
    want = ref.activate(v, act)
    ok(y[0], want, rel * want.abs() + ref.u(t) * (1 + rel) * want.abs() + ref.tiny(t))
    # the slope is a sum of two terms with that error each
    terms = ref.phi(v) + v.abs() * torch.exp(-0.5 * v * v) / (2.0 * torch.pi) ** 0.5 if act == "gelu" else torch.sigmoid(v) * (1 + v.abs())
    want, e = ref.slope(v, act), rel * terms
    ok(dz[0], want, e + ref.u(t) * (want.abs() + e) + ref.tiny(t))


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("most,rows,k,n", [(8192, 5370, 11008, 4096), (8192, 4096, 4096, 1024), (16384, 64, 2048, 8), (8192, 300, 1027, 513), (20000, 4096, 4096, 11008), (1, 2100, 1024, 4096)])
def test_a_workspace_of_other_rows(T, ctx, eight, most, rows, k, n):
    """Calls in the workspace of a larger call (tc_linear: also of a smaller one, and none), which may be less than their own would be: results within the
    bounds, nothing written behind it; in a larger one than their own the same bytes."""
    t = torch.float16
    seed = rows + k + n

    def room(size):
        buf = torch.full((size + 256,), 0xAB, dtype=torch.uint8, device="cuda")
        return buf, buf[:size]

    x, mw, w64 = linear_inputs(T, t, rows, k, n, eight, seed, (0, 0))
    x64, d64 = x.double(), None
    z64 = x64 @ w64.t()
    ez = ref.product_error(x64.abs() @ w64.abs().t(), k)
    y = torch.empty(rows, n, dtype=t, device="cuda")
    own = ctx.linear_workspace(rows, k, n)
    seen = None
    for size in (0, ctx.linear_workspace(most, k, n), own, own + 4096):
        buf, work = room(size)
        ctx.linear(T.Matrix(x), mw, T.Matrix(y), workspace=work if size else None)
        ctx.sync()
        ok(y, z64, ez + ref.u(t) * (z64.abs() + ez) + ref.tiny(t))
        assert (buf[size:] == 0xAB).all()
        if size >= own:
            assert seen is None or torch.equal(seen, y)
            seen = y.clone()
    del z64, ez
    if most < rows:
        return
    dy = rand((rows, n), seed + 5, t)
    mx = T.Matrix(x)
    if eight:
        q, s = rows8(x)
        mx, x64 = T.Matrix(q, s), ref.value(q, s)
    d64 = dy.double()
    off = (ref.u(t) + 3 * ref.E) * d64.abs() + 2 * ref.tiny(t) if eight else torch.zeros_like(d64)
    dx, dw = torch.empty(rows, k, dtype=t, device="cuda"), torch.empty(n, k, dtype=t, device="cuda")
    own = ctx.linear_backward_workspace(rows, k, n)
    seen = None
    for size in (ctx.linear_backward_workspace(most, k, n), ctx.linear_backward_workspace(rows, 1, n), own, own + 4096):
        buf, work = room(size)
        ctx.linear_backward(T.Matrix(dy), mx, mw, dx=T.Matrix(dx), dw=T.Matrix(dw), workspace=work)
        ctx.sync()
        assert (buf[size:] == 0xAB).all()
        for got, left, e, right, terms in ((dx, d64, off, w64, n), (dw, d64.t(), off.t(), x64, rows)):
            want, err = left @ right, e @ right.abs()
            err = err + ref.product_error((left.abs() + e) @ right.abs(), terms)
            ok(got, want, err + ref.u(t) * (want.abs() + err) + ref.tiny(t))
        if size >= own:
            assert seen is None or (torch.equal(seen[0], dx) and torch.equal(seen[1], dw))
            seen = dx.clone(), dw.clone()


def test_calls_of_the_binding_without_a_matrix(T, ctx):
    """None, or a tc_matrix by reference, where a Matrix is expected: what the library says of them"""
    import ctypes

    t = torch.float16
    x, q, s = rand((4, 8), 1, t), torch.empty(4, 8, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    m, m8, w = T.Matrix(x), T.Matrix(q, s), T.Matrix(rand((8, 8), 2, t))
    v, work = torch.ones(8, device="cuda"), space(1 << 20)
    for call in (lambda: ctx.checkpoint_encode(None, m8), lambda: ctx.checkpoint_encode(m, None), lambda: ctx.checkpoint_decode(None, m), lambda: ctx.checkpoint_decode(m8, None),
                 lambda: ctx.norm(0, None, None, None, 1e-5, m), lambda: ctx.norm(0, m, v.to(t), None, 1e-5, None), lambda: ctx.norm_backward(1, None, m, None, None, v, m, None, None, None),
                 lambda: ctx.norm_backward(1, m, None, None, None, v, m, None, None, None), lambda: ctx.linear(None, w, m), lambda: ctx.linear(m, None, m),
                 lambda: ctx.linear(m, w, None), lambda: ctx.linear_backward(None, m, w, dx=m, workspace=work), lambda: ctx.linear_backward(m, m, None, dx=m, workspace=work)):
        with pytest.raises(T.TcError) as e:
            call()
        assert e.value.code == T.binding.TC_ERR_ARG
    by = lambda a: ctypes.byref(a.view)  # noqa: E731
    ctx.checkpoint_encode(by(m), by(m8))
    y, back = torch.empty_like(x), torch.empty_like(x)
    ctx.norm(1, by(m), None, None, 1e-5, by(T.Matrix(y)))
    ctx.checkpoint_decode(by(m8), by(T.Matrix(back)))
    ctx.sync()
    want, scale = ref.encode(x)
    assert torch.equal(q, want) and torch.equal(s, scale)
    v64 = ref.value(want, scale)
    ok(back, v64, (ref.u(t) + 2 * ref.E) * v64.abs() + ref.tiny(t))
    y64, _, rstd = ref.norm(x.double(), None, None, 1e-5, False)
    ok(y, y64, ref.norm_bound(x.double(), None, None, y64, rstd, t, False))


def test_a_library_that_is_named_is_checked_too(T):
    c = T.Context(0, None, T.load_library(T.binding.library_path()))
    near, far = (T.Matrix(torch.zeros(4, 8, dtype=torch.float16, device=d)) for d in ("cuda", "cpu"))
    for call in (lambda: c.norm(1, far, None, None, 1e-5, near), lambda: c.norm(1, near, None, None, 1e-5, far), lambda: c.norm(1, near, torch.ones(8, dtype=torch.float16), None, 1e-5, near),
                 lambda: c.linear(near, T.Matrix(torch.zeros(8, 8, dtype=torch.float16, device="cuda")), near, workspace=torch.zeros(64, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call()
    c.close()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols", [(5, 7), (300, 515), (1100, 2051), (40, 4099), (1030, 8190), (9, 12295), (6, 32767), (1500, 16392)])
def test_norms_in_the_place_of_their_input(T, ctx, dtype, rows, cols):
    t = ref.DT[dtype]
    for kind in (T.TC_NORM_LAYER, T.TC_NORM_RMS):
        x, dy, y, dx = (strided(rand((rows, cols), 3 + i, t), 1, 2)[1] for i in range(4))
        mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        ctx.norm(kind, T.Matrix(x), None, None, 1e-5, T.Matrix(y), mean, rstd)
        ctx.norm_backward(kind, T.Matrix(dy), T.Matrix(x), None, mean, rstd, T.Matrix(dx), None, None, None)
        ctx.norm_backward(kind, T.Matrix(dy), T.Matrix(x), None, mean, rstd, T.Matrix(dy), None, None, None)
        ctx.norm(kind, T.Matrix(x), None, None, 1e-5, T.Matrix(x))
        ctx.sync()
        assert torch.equal(x, y) and torch.equal(dy, dx)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,n", [(5, 64, 40), (70, 65, 33), (487, 4104, 4104), (8200, 136, 8456), (8456, 520, 8200), (10248, 8200, 520)])
def test_products_in_the_place_of_their_input(T, ctx, dtype, rows, k, n):
    t = ref.DT[dtype]
    x, w, residual, y = rand((rows, k), 1, t), rand((n, k), 2, t, k ** -0.5), rand((rows, n), 3, t), torch.empty(rows, n, dtype=t, device="cuda")
    work = space(max(ctx.linear_workspace(rows, k, n), ctx.linear_backward_workspace(rows, k, n)))
    ctx.linear(T.Matrix(x), T.Matrix(w), T.Matrix(y), activation=3, residual=T.Matrix(residual), workspace=work)
    ctx.linear(T.Matrix(x), T.Matrix(w), T.Matrix(residual), activation=3, residual=T.Matrix(residual), workspace=work)
    ctx.sync()
    assert torch.equal(residual, y)
    z8, w8, dy, dz = rows8(rand((rows, n), 4, t)), rows8(w), rand((rows, n), 5, t), torch.empty_like(y)
    dx, again = torch.empty_like(x), torch.empty_like(x)
    ctx.linear_backward(T.Matrix(dy), None, T.Matrix(*w8), 2, T.Matrix(*z8), T.Matrix(dz), T.Matrix(dx), workspace=work)
    ctx.linear_backward(T.Matrix(dy), None, T.Matrix(*w8), 2, T.Matrix(*z8), T.Matrix(dy), T.Matrix(again), workspace=work)
    ctx.sync()
    assert torch.equal(dy, dz) and torch.equal(dx, again)


def test_large_products_captured_and_replayed(T):
    """the kernels of the largest tiles, int8 operands widened, in a graph that is replayed on new inputs between eager calls"""
    t = torch.bfloat16
    stream = torch.cuda.Stream()
    c = T.Context(0, stream.cuda_stream)
    rows, k, n = 4096, 2048, 4104
    x, w8, dy = rand((rows, k), 1, t), rows8(rand((n, k), 2, t, k ** -0.5)), rand((rows, n), 3, t)
    x8 = rows8(x)
    y, dx, dw = (torch.empty(*s, dtype=t, device="cuda") for s in ((rows, n), (rows, k), (n, k)))
    work = space(max(c.linear_workspace(rows, k, n), c.linear_backward_workspace(rows, k, n)))
    mx, mw, my, mdy, mx8, mdx, mdw = T.Matrix(x), T.Matrix(*w8), T.Matrix(y), T.Matrix(dy), T.Matrix(*x8), T.Matrix(dx), T.Matrix(dw)

    def calls():
        c.linear(mx, mw, my, activation=2, workspace=work)
        c.linear_backward(mdy, mx8, mw, dx=mdx, dw=mdw, workspace=work)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        calls()
    for i in range(3):
        x.copy_(rand((rows, k), 10 + i, t))
        dy.copy_(rand((rows, n), 20 + i, t))
        torch.cuda.synchronize()
        calls()
        torch.cuda.synchronize()
        want = [o.clone() for o in (y, dx, dw)]
        for o in (y, dx, dw, work):
            o.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(want, (y, dx, dw))), i
    c.close()


def test_the_scales_of_a_checkpoint_are_committed_as_their_bytes(T, ctx):
    """a commitment of the rows binds the whole numbers alone; one of the scales' bytes binds what they stand for"""
    from gpu_util import TAU_BYTES, pps
    from oracle import bls12_381 as ec
    from oracle import cbind

    rows, cols = 12, 40
    x = rand((rows, cols), 1, torch.float16)
    q, s = torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, device="cuda")
    ctx.checkpoint_encode(T.Matrix(x), T.Matrix(q, s))
    ctx.sync()
    q2, s2 = torch.empty_like(q), torch.empty_like(s)
    ctx.checkpoint_encode(T.Matrix(x * 2), T.Matrix(q2, s2))
    ctx.sync()
    commitments = []
    for tensor in (q, q2, s.view(torch.int8).view(rows, 4), s2.view(torch.int8).view(rows, 4)):
        srs = ctx.setup_from_trapdoor(TAU_BYTES, tuple(tensor.shape), T.TC_SRS_SUFFIX)
        commitments.append(ctx.commit(srs, tensor, T.TC_I8))
        assert commitments[-1] == ec.g1_to_bytes(cbind.commit(pps(tuple(tensor.shape)), tensor.cpu().numpy()))
        srs.close()
    assert commitments[0] == commitments[1] and commitments[2] != commitments[3]
