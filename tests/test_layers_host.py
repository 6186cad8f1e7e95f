"""The layer operators on the CPU: what their entry points refuse, the views they take, and the 64-bit definitions that the GPU tests
compare with (gradients against differences), through the host build of the library's checks."""
import ctypes
import os

import pytest
import torch

import layers_reference as ref
import paper_2602_12630_amd as T
from test_host_logic import EMU, ROOT, entry

B = T.binding


@pytest.fixture(scope="module")
def emu():
    csrc = os.path.join(ROOT, "paper_2602_12630_amd", "csrc")
    src = [os.path.join(csrc, f) for f in os.listdir(csrc)] + [os.path.join(ROOT, "include", "tc.h")]
    if not os.path.exists(EMU) or os.path.getmtime(EMU) < max(os.path.getmtime(f) for f in src):
        entry.build_host_emulation(EMU)
    ctx = T.Context(0, None, T.load_library(EMU))
    yield ctx
    ctx.close()


def refused(code, call, *args, **kw):
    with pytest.raises(T.TcError) as e:
        call(*args, **kw)
    assert e.value.code == code, str(e.value)


def mat(rows, cols, dtype=torch.float16, ld=None):
    m = torch.zeros(rows, ld or cols, dtype=dtype)[:, :cols]
    return T.Matrix(m, torch.zeros(rows)) if dtype == torch.int8 else T.Matrix(m)


def changed(m, **fields):
    """the same view with fields of the C structure changed"""
    v = B.tc_matrix.from_buffer_copy(m.view)
    for k, x in fields.items():
        setattr(v, k, x)
    v.keep = m
    return ctypes.byref(v)


def ws(n):
    return torch.zeros(n, dtype=torch.uint8)


# ---- refusals ------------------------------------------------------------------------------------------------------
BAD_VIEWS = [(B.TC_ERR_SHAPE, {"cols": 0}), (B.TC_ERR_SHAPE, {"ld": 7}), (B.TC_ERR_SHAPE, {"ld": 2 ** 31 + 1}), (B.TC_ERR_SHAPE, {"rows": 2 ** 31}),
             (B.TC_ERR_SHAPE, {"cols": 2 ** 20 + 1, "ld": 2 ** 21}), (B.TC_ERR_ARG, {"d_data": None}), (B.TC_ERR_ARG, {"dtype": T.TC_I16}),
             (B.TC_ERR_ARG, {"dtype": 0}), (B.TC_ERR_ARG, {"dtype": T.TC_I8})]


@pytest.mark.parametrize("code,fields", BAD_VIEWS)
def test_bad_views_are_refused_everywhere(emu, code, fields):
    m, q = mat(4, 8), mat(4, 8, torch.int8)
    bad = changed(m, **fields)
    v = torch.zeros(8)
    refused(code, emu.checkpoint_encode, bad, q)
    refused(code, emu.checkpoint_decode, q, bad)
    refused(code, emu.norm, 0, bad, None, None, 1e-5, m)
    refused(code, emu.norm, 0, m, None, None, 1e-5, bad)
    refused(code, emu.norm_backward, 0, bad, m, None, v, v, m, None, None, None)
    refused(code, emu.norm_backward, 0, m, bad, None, v, v, m, None, None, None)
    refused(code, emu.norm_backward, 0, m, m, None, v, v, bad, None, None, None)
    w = mat(8, 8)
    big = ws(1 << 20)
    refused(code, emu.linear, bad, w, m)
    refused(code, emu.linear, m, w, bad)
    refused(code, emu.linear, m, w, m, residual=bad)
    refused(code, emu.linear, m, w, m, z=bad)
    for name in ("z", "dz", "dx"):
        args = {"z": m, "dz": m, "dx": m, name: bad}
        refused(code, emu.linear_backward, m, m, w, 2, workspace=big, **args)
    refused(code, emu.linear_backward, bad, m, w, 0, dx=m, workspace=big)
    refused(code, emu.linear_backward, m, bad, w, 0, dw=w, workspace=big)


def test_views_of_torch_tensors_are_checked():
    for bad in (torch.zeros(3), torch.zeros(2, 2), torch.zeros(2, 4, dtype=torch.float16).t(), torch.zeros(2, 2, dtype=torch.int8)):
        with pytest.raises(ValueError):
            T.Matrix(bad)
    with pytest.raises(ValueError):
        T.Matrix(torch.zeros(2, 2, dtype=torch.float16), torch.zeros(2))
    q = torch.zeros(2, 2, dtype=torch.int8)
    for scale in (torch.zeros(3), torch.zeros(2, dtype=torch.float64), torch.zeros(4)[::2], torch.zeros(2, 1)):
        with pytest.raises(ValueError):
            T.Matrix(q, scale)
    v = T.Matrix(torch.zeros(5, 12, dtype=torch.bfloat16)[1:4, 2:9])
    assert (v.view.rows, v.view.cols, v.view.ld, v.view.dtype) == (3, 7, 12, T.TC_BF16)


def test_checkpoint_refusals(emu):
    m, q = mat(4, 8), mat(4, 8, torch.int8)
    refused(B.TC_ERR_ARG, emu.checkpoint_encode, m, m)
    refused(B.TC_ERR_ARG, emu.checkpoint_encode, q, q)
    refused(B.TC_ERR_ARG, emu.checkpoint_decode, m, m)
    refused(B.TC_ERR_ARG, emu.checkpoint_encode, None, q)
    refused(B.TC_ERR_ARG, emu.checkpoint_encode, m, None)
    refused(B.TC_ERR_SHAPE, emu.checkpoint_encode, m, mat(5, 8, torch.int8))
    refused(B.TC_ERR_SHAPE, emu.checkpoint_decode, q, mat(4, 9))
    refused(B.TC_ERR_ARG, emu.checkpoint_encode, m, changed(q, d_scale=None))
    refused(B.TC_ERR_ARG, emu.checkpoint_decode, changed(q, d_scale=q.view.d_scale + 2), m)
    refused(B.TC_ERR_ARG, emu.checkpoint_encode, changed(m, d_data=m.view.d_data + 1), q)
    assert emu.lib.tc_checkpoint_encode(None, m, q) == B.TC_ERR_ARG


def test_norm_refusals(emu):
    m, q, b = mat(4, 8), mat(4, 8, torch.int8), mat(4, 8, torch.bfloat16)
    v = torch.zeros(8)
    for eps in (0.0, -1.0, 1.0, float("nan"), float("inf")):
        refused(B.TC_ERR_ARG, emu.norm, 0, m, None, None, eps, m)
    refused(B.TC_ERR_ARG, emu.norm, 2, m, None, None, 1e-5, m)
    refused(B.TC_ERR_ARG, emu.norm, 0, m, None, None, 1e-5, b)
    refused(B.TC_ERR_ARG, emu.norm, 0, m, None, None, 1e-5, q)
    refused(B.TC_ERR_SHAPE, emu.norm, 0, m, None, None, 1e-5, mat(4, 9))
    refused(B.TC_ERR_ARG, emu.norm, 0, m, v.data_ptr() + 1, None, 1e-5, m)
    refused(B.TC_ERR_ARG, emu.norm, 0, m, None, None, 1e-5, m, mean=v.data_ptr() + 2)
    long = mat(1, 2 ** 15 + 1)
    refused(B.TC_ERR_SHAPE, emu.norm, 0, long, None, None, 1e-5, long)
    refused(B.TC_ERR_SHAPE, emu.norm_backward, 0, long, long, None, v, v, long, None, None, None)
    refused(B.TC_ERR_SHAPE, emu.norm_backward_workspace, 4, 2 ** 15 + 1)
    refused(B.TC_ERR_SHAPE, emu.norm_backward_workspace, 4, 0)
    assert emu.lib.tc_norm_backward_workspace(4, 8, None) == B.TC_ERR_ARG
    refused(B.TC_ERR_ARG, emu.norm_backward, 0, m, m, None, None, v, m, None, None, None)
    refused(B.TC_ERR_ARG, emu.norm_backward, 1, m, m, None, None, None, m, None, None, None)
    refused(B.TC_ERR_ARG, emu.norm_backward, 0, m, b, None, v, v, m, None, None, None)
    refused(B.TC_ERR_ARG, emu.norm_backward, 0, m, m, None, v, v, b, None, None, None)
    need = emu.norm_backward_workspace(4, 8)
    refused(B.TC_ERR_ARG, emu.norm_backward, 0, m, m, None, v, v, m, v, v, None)
    refused(B.TC_ERR_ARG, emu.norm_backward, 0, m, m, None, v, v, m, v, v, ws(need - 1))
    refused(B.TC_ERR_ARG, emu.norm_backward, 0, m, m, None, v, v, m, v, v, ws(need + 16)[8:])
    emu.norm_backward(0, m, m, None, v, v, m, None, None, None)              # without sums no workspace is needed


def test_linear_refusals(emu):
    m, w, b, q = mat(4, 8), mat(8, 8), mat(4, 8, torch.bfloat16), mat(4, 8, torch.int8)
    v = torch.zeros(8)
    big = ws(1 << 20)
    for act in (-1, 4):
        refused(B.TC_ERR_ARG, emu.linear, m, w, m, activation=act)
        refused(B.TC_ERR_ARG, emu.linear_backward, m, m, w, act, z=m, dz=m, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, emu.linear, q, w, m)
    refused(B.TC_ERR_ARG, emu.linear, m, mat(8, 8, torch.bfloat16), m)
    refused(B.TC_ERR_ARG, emu.linear, m, w, b)
    refused(B.TC_ERR_ARG, emu.linear, m, w, m, residual=b)
    refused(B.TC_ERR_ARG, emu.linear, m, w, m, z=q)
    refused(B.TC_ERR_ARG, emu.linear, m, w, m, bias=v.data_ptr() + 1)
    refused(B.TC_ERR_SHAPE, emu.linear, m, mat(8, 9), m)
    refused(B.TC_ERR_SHAPE, emu.linear, m, mat(9, 8), m)
    refused(B.TC_ERR_SHAPE, emu.linear, m, mat(0, 8), m)
    refused(B.TC_ERR_SHAPE, emu.linear, m, w, m, residual=mat(3, 8))
    back = emu.linear_backward
    refused(B.TC_ERR_ARG, back, m, m, w, 0, z=m, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, w, 0, dz=m, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, w, 2, dz=m, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, w, 2, z=m, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, w, 2, z=b, dz=m, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, None, 0, dx=m, workspace=big)
    refused(B.TC_ERR_ARG, back, m, None, w, 0, dw=w, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, w, 0, dx=b, workspace=big)
    refused(B.TC_ERR_ARG, back, m, m, w, 0, dw=mat(8, 8, torch.int8), workspace=big)
    refused(B.TC_ERR_SHAPE, back, m, m, w, 0, dx=mat(3, 8), workspace=big)
    refused(B.TC_ERR_SHAPE, back, m, m, w, 0, dx=mat(4, 9), workspace=big)
    refused(B.TC_ERR_SHAPE, back, m, m, w, 0, dx=m, dw=mat(8, 9), workspace=big)
    refused(B.TC_ERR_SHAPE, back, m, mat(5, 8), w, 0, dw=w, workspace=big)
    need = emu.linear_backward_workspace(4, 8, 8)
    for bad in (None, ws(need - 1), ws(need + 16)[8:]):
        refused(B.TC_ERR_ARG, back, m, m, w, 0, dx=m, workspace=bad)
    for sizes in ((2 ** 31, 8, 8), (4, 0, 8), (4, 8, 0), (4, 2 ** 20 + 1, 8), (4, 8, 2 ** 20 + 1)):
        refused(B.TC_ERR_SHAPE, emu.linear_workspace, *sizes)
        refused(B.TC_ERR_SHAPE, emu.linear_backward_workspace, *sizes)
    assert emu.lib.tc_linear_workspace(4, 8, 8, None) == B.TC_ERR_ARG


def test_a_workspace_for_the_sizes_serves_every_call_of_them(emu):
    """also a call that asks for fewer gradients, whose inner width the library then cannot see"""
    for rows, k, n in ((1, 1, 1), (5, 4096, 7), (300, 33, 1000), (4096, 64, 64)):
        w = ws(emu.linear_backward_workspace(rows, k, n))
        emu.linear_backward(mat(0, n), mat(0, k), mat(n, k), 0, dx=mat(0, k), workspace=w)
        if rows * n <= 4096:
            emu.linear_backward(mat(rows, n), None, None, 0, dbias=torch.zeros(n), workspace=w)


def test_empty_inputs(emu):
    m, q = mat(0, 8), mat(0, 8, torch.int8)
    emu.checkpoint_encode(m, q)
    emu.checkpoint_decode(q, m)
    emu.norm(0, m, None, None, 1e-5, m)
    emu.linear(m, mat(3, 8), mat(0, 3))
    dg, db = torch.ones(8), torch.ones(8)
    emu.norm_backward(0, m, m, None, None, None, m, dg, db, ws(emu.norm_backward_workspace(0, 8)))
    assert not dg.any() and not db.any()
    dw, dbias = torch.ones(3, 10, dtype=torch.float16), torch.ones(3)
    emu.linear_backward(mat(0, 3), m, mat(3, 8), 0, dx=m, dw=T.Matrix(dw[:, :8]), dbias=dbias, workspace=ws(emu.linear_backward_workspace(0, 8, 3)))
    assert not dw[:, :8].any() and not dbias.any() and (dw[:, 8:] == 1).all()


# ---- the definitions -----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_checkpoint_on_the_host(emu, dtype):
    t = ref.DT[dtype]
    gen = torch.Generator().manual_seed(3)
    x = torch.randn(6, 37, generator=gen).to(t)
    x[0] = 0
    x[1, 3], x[1, 4], x[1, 5] = float("inf"), float("-inf"), float("nan")
    x[2] = float("inf")
    x[3] = (torch.arange(37) - 18).to(t)                  # amax 18: ties at 254 x = odd * 18
    x[4] *= 1e-7
    q, s = torch.full((6, 37), 99, dtype=torch.int8), torch.full((6,), -1.0)
    emu.checkpoint_encode(T.Matrix(x), T.Matrix(q, s))
    want, scale = ref.encode(x)
    assert torch.equal(q, want) and torch.equal(s, scale)
    back = torch.empty_like(x)
    emu.checkpoint_decode(T.Matrix(q, s), T.Matrix(back))
    v = ref.value(want, scale)
    assert ref.worst(back, v, (ref.u(t) + 2 * ref.E) * v.abs() + ref.tiny(t)) <= 1


@pytest.mark.parametrize("act", list(ref.ACTS))
def test_the_gradients_of_the_definitions_are_their_differences(act):
    """central differences of the 64-bit forward definitions against the 64-bit gradients: step 1e-6, so an error of 1e-9 or so"""
    gen = torch.Generator().manual_seed(5)
    x, w, b, dy = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((3, 5), (4, 5), (4,), (3, 4)))

    def loss(x, w, b):
        return (ref.activate(x @ w.t() + b, act) * dy).sum().item()

    dz = dy * ref.slope(x @ w.t() + b, act)
    for arg, grad in ((0, dz @ w), (1, dz.t() @ x), (2, dz.sum(0))):
        for i in range(grad.numel()):
            ts = [[v.clone() for v in (x, w, b)] for _ in range(2)]
            ts[0][arg].view(-1)[i] += 1e-6
            ts[1][arg].view(-1)[i] -= 1e-6
            d = (loss(*ts[0]) - loss(*ts[1])) / 2e-6
            assert abs(d - grad.reshape(-1)[i].item()) < 1e-7


@pytest.mark.parametrize("centred", [True, False])
def test_the_norms_gradients_are_differences(centred):
    gen = torch.Generator().manual_seed(6)
    x, g, b, dy = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((3, 7), (7,), (7,), (3, 7)))

    def loss(x, g, b):
        return (ref.norm(x, g, b, 1e-2, centred)[0] * dy).sum().item()

    _, mean, rstd = ref.norm(x, g, b, 1e-2, centred)
    grads = ref.norm_backward(dy, x, g, mean, rstd, centred)
    for arg, grad in enumerate(grads):
        for i in range(grad.numel()):
            ts = [[v.clone() for v in (x, g, b)] for _ in range(2)]
            ts[0][arg].view(-1)[i] += 1e-6
            ts[1][arg].view(-1)[i] -= 1e-6
            d = (loss(*ts[0]) - loss(*ts[1])) / 2e-6
            assert abs(d - grad.reshape(-1)[i].item()) < 1e-7


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("eight", [False, True])
def test_norm_and_linear_on_the_host(emu, dtype, eight):
    """the host build keeps to the views: strides, rows with scales, columns that are not its own"""
    t = ref.DT[dtype]
    gen = torch.Generator().manual_seed(8)
    rows, k, n = 5, 11, 6
    xs = torch.randn(rows, k + 3, generator=gen).to(t)
    x, w = xs[:, 1:1 + k], torch.randn(n, k, generator=gen).to(t)
    qx, qw = ref.encode(x), ref.encode(w)
    mx = T.Matrix(*qx) if eight else T.Matrix(x)
    vx = ref.value(*qx) if eight else ref.value(x)
    y = torch.full((rows, k + 2), 7.0).to(t)
    mean, rstd = torch.empty(rows), torch.empty(rows)
    emu.norm(0, mx, None, None, 1e-5, T.Matrix(y[:, :k]), mean, rstd)
    want, wmean, wrstd = ref.norm(vx, None, None, 1e-5, True)
    assert ref.worst(y[:, :k], want, (ref.u(t) + ref.E) * want.abs() + ref.tiny(t) + 1e-12) <= 1 and (y[:, k:] == 7).all()
    out, z = torch.full((rows, n + 1), 7.0).to(t), torch.empty(rows, n, dtype=t)
    mw = T.Matrix(*qw) if eight else T.Matrix(w)
    vw = ref.value(*qw) if eight else ref.value(w)
    emu.linear(T.Matrix(x), mw, T.Matrix(out[:, :n]), activation=2, z=T.Matrix(z))
    wz = ref.value(x) @ vw.t()
    wy = ref.activate(wz, "gelu")
    assert ref.worst(z, wz, (ref.u(t) + ref.E) * wz.abs() + ref.tiny(t) + 1e-12) <= 1
    assert ref.worst(out[:, :n], wy, (ref.u(t) + ref.E) * wy.abs() + ref.tiny(t) + 1e-12) <= 1 and (out[:, n:] == 7).all()
    dy = torch.randn(rows, n, generator=gen).to(t)
    dz, dx, dw, db = torch.empty(rows, n, dtype=t), torch.empty(rows, k, dtype=t), torch.empty(n, k, dtype=t), torch.empty(n)
    emu.linear_backward(T.Matrix(dy), mx, mw, 2, T.Matrix(z), T.Matrix(dz), T.Matrix(dx), T.Matrix(dw), db, ws(emu.linear_backward_workspace(rows, k, n)))
    d = ref.value(dy) * ref.slope(ref.value(z), "gelu")
    for got, w64 in ((dz, d), (dx, d @ vw), (dw, d.t() @ vx)):
        assert ref.worst(got, w64, (ref.u(t) + ref.E) * w64.abs() + ref.tiny(t) + 1e-12) <= 1
    assert ref.worst(db, d.sum(0), 2 * ref.E * d.sum(0).abs() + 1e-12) <= 1


def test_vectors_of_torch_are_checked(emu):
    """too short, of another type, with gaps"""
    m, w = mat(4, 8), mat(8, 8)
    h, f = torch.zeros(8, dtype=torch.float16), torch.zeros(8)
    big = ws(1 << 20)
    emu.norm(0, m, h, h, 1e-5, m, f[:4], f[:4])
    emu.linear_backward(m, None, w, dx=mat(4, 8), dbias=f, workspace=big)
    for bad in (h[:7], f, h.bfloat16(), torch.zeros(16, dtype=torch.float16)[::2]):
        for call in (lambda: emu.norm(0, m, bad, None, 1e-5, m), lambda: emu.norm(0, m, None, bad, 1e-5, m),
                     lambda: emu.norm_backward(0, m, m, bad, f, f, m, None, None, None), lambda: emu.linear(m, w, m, bias=bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (f[:3], h, f.double(), torch.zeros(16)[::2]):
        for call in (lambda: emu.norm(0, m, None, None, 1e-5, m, bad, None), lambda: emu.norm(0, m, None, None, 1e-5, m, None, bad),
                     lambda: emu.norm_backward(0, m, m, None, f, f, m, bad, None, big), lambda: emu.norm_backward(0, m, m, None, f, bad, m, None, None, big),
                     lambda: emu.linear_backward(m, None, w, dx=m, dbias=bad, workspace=big)):
            with pytest.raises(ValueError):
                call()
