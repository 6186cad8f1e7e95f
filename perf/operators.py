"""What the performance of the layer operators is measured on: the passes that make the tensors which a prover commits, and the
gradients that are taken from their stored 8-bit rows.

    checkpoint     16-bit activations -> int8 rows with a scale each, and back
    norm           layer norm or root-mean-square norm, one pass over the rows
    norm_backward  its gradient, the input given in 16 bits or as a checkpoint, with the sums for gamma and beta
    linear         y = act(x W^T + bias) + residual, the weights in 16 bits or int8 with a scale for each row
    linear_backward  dz = dy act'(z), dx = dz W, dW = dz^T x, dbias = sum dz; x and z in 16 bits or as checkpoints

Values: activations N(0, 1) with a few large channels, as residual streams have them; weights N(0, 1 / in), or int8 uniform in
[-127, 127]; gradients N(0, 1) times a loss scale that keeps them well inside the type.  Everything comes from the seed.
"""
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
EPS_RMS = 1e-6


def listed():
    return [
        # one token's activation kept: launches are all of it
        {"name": "checkpoint_token", "kind": "checkpoint", "dtype": "f16", "rows": 1, "cols": 4096},
        # the MLP intermediate of a training batch, kept for the backward pass
        {"name": "checkpoint_mlp", "kind": "checkpoint", "dtype": "bf16", "rows": 8192, "cols": 11008},
        # a token being decoded
        {"name": "norm_token", "kind": "norm", "dtype": "f16", "norm": "rms", "rows": 1, "cols": 4096},
        # a prompt whose length is no round number
        {"name": "norm_prompt", "kind": "norm", "dtype": "bf16", "norm": "layer", "rows": 487, "cols": 4096},
        # a training batch, its input kept in 8 bits
        {"name": "norm_backward_train", "kind": "norm_backward", "dtype": "bf16", "norm": "layer", "rows": 16384, "cols": 4096, "x8": True},
        # a short batch at an odd width
        {"name": "norm_backward_odd", "kind": "norm_backward", "dtype": "f16", "norm": "rms", "rows": 333, "cols": 1027, "x8": False},
        # a token through the gate projection of a model whose committed int8 weights are served
        {"name": "linear_token_w8", "kind": "linear", "dtype": "f16", "act": "silu", "rows": 1, "in": 4096, "out": 11008, "w8": True,
         "bias": False, "residual": False, "keep_z": False},
        # the down projection of a prompt of ragged length, added to the residual stream
        {"name": "linear_prompt_ragged", "kind": "linear", "dtype": "f16", "act": "none", "rows": 487, "in": 11008, "out": 4096, "w8": False,
         "bias": False, "residual": True, "keep_z": False},
        # the up projection of a training batch; the value before the activation is kept
        {"name": "linear_train", "kind": "linear", "dtype": "bf16", "act": "gelu", "rows": 8192, "in": 4096, "out": 11008, "w8": False,
         "bias": True, "residual": False, "keep_z": True},
        # gradients of that projection for one sequence, from 8-bit checkpoints
        {"name": "linear_backward_train", "kind": "linear_backward", "dtype": "bf16", "act": "gelu", "rows": 4096, "in": 4096, "out": 11008,
         "x8": True, "z8": True, "w8": False, "dw": True},
        # an output projection's gradients, 16-bit inputs, ragged length
        {"name": "linear_backward_ragged", "kind": "linear_backward", "dtype": "f16", "act": "none", "rows": 501, "in": 4096, "out": 4096,
         "x8": False, "z8": False, "w8": False, "dw": True},
        # gradients through committed int8 weights that stay as they are
        {"name": "linear_backward_frozen", "kind": "linear_backward", "dtype": "bf16", "act": "silu", "rows": 512, "in": 4096, "out": 11008,
         "x8": True, "z8": True, "w8": True, "dw": False},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _width(rng, hi=11008):
    """a model's width, or any other"""
    return rng.choice([512, 1024, 2048, 4096, 11008, _log_int(rng, 64, hi), _log_int(rng, 64, hi), 8 * _log_int(rng, 8, hi // 8)])


def draw(rng):
    kind = rng.choice(["checkpoint", "norm", "norm_backward", "linear", "linear", "linear", "linear_backward", "linear_backward"])
    case = {"kind": kind, "dtype": rng.choice(["f16", "bf16"])}
    if kind in ("checkpoint", "norm", "norm_backward"):
        case["cols"] = _width(rng)
        case["rows"] = _log_int(rng, 1, min(16384, (16384 * 4096 if kind != "checkpoint" else 8192 * 11008) // case["cols"]))
        if kind != "checkpoint":
            case["norm"] = rng.choice(["layer", "rms"])
        if kind == "norm_backward":
            case["x8"] = rng.random() < 0.5
        return case
    case["in"], case["out"] = _width(rng), _width(rng)
    case["act"] = rng.choice(["none", "relu", "gelu", "silu"])
    case["w8"] = rng.random() < 0.4
    if kind == "linear":
        largest = 8192 * 4096 * 11008
        case["rows"] = _log_int(rng, 1, min(8192, largest // (case["in"] * case["out"])))
        case["bias"] = rng.random() < 0.5
        case["residual"] = rng.random() < 0.5
        case["keep_z"] = case["act"] != "none" and rng.random() < 0.5
    else:
        largest = 4096 * 4096 * 11008
        case["rows"] = _log_int(rng, 1, min(4096, largest // (case["in"] * case["out"])))
        case["x8"] = rng.random() < 0.5
        case["z8"] = case["act"] != "none" and rng.random() < 0.5
        case["dw"] = not case["w8"]
    return case


# ---- what the cases are made of ------------------------------------------------------------------------------------
class State:
    pass


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _activation(gen, rows, cols):
    x = _normal(gen, rows, cols)
    loud = torch.randint(0, cols, (max(1, cols // 1024),), generator=gen, device="cuda")
    x[:, loud] *= 8.0
    return x


def _rows8(x):
    """int8 rows and their scales, as a program holds them that has kept them: the rule of the checkpoint operator"""
    amax = x.double().abs().amax(dim=1, keepdim=True)
    q = torch.round(x.double() * 127.0 / torch.where(amax > 0, amax, torch.ones_like(amax)))
    return q.to(torch.int8), (amax / 127.0).float().reshape(-1).contiguous()


def _inputs(case, seed):
    st = State()
    st.case = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t = DTYPES[case["dtype"]]
    kind = case["kind"]
    st.t = t
    st.x8 = st.z8 = st.w8 = None
    if kind in ("checkpoint", "norm", "norm_backward"):
        rows, cols = case["rows"], case["cols"]
        st.x = _activation(gen, rows, cols).to(t)
        if kind == "checkpoint":
            return st
        st.gamma = (1.0 + 0.1 * _normal(gen, cols)).to(t)
        st.beta = (0.1 * _normal(gen, cols)).to(t) if case["norm"] == "layer" else None
        if kind == "norm_backward":
            st.dy = _normal(gen, rows, cols).to(t)
            # the statistics of the true input, kept by the forward pass; the input itself kept in 8 bits or as it was
            x = st.x.double()
            mean = x.mean(dim=1) if case["norm"] == "layer" else torch.zeros(rows, device="cuda", dtype=torch.float64)
            var = (x - mean[:, None]).square().mean(dim=1)
            st.mean = mean.float()
            st.rstd = (var + (EPS if case["norm"] == "layer" else EPS_RMS)).rsqrt().float()
            if case["x8"]:
                st.x8 = _rows8(st.x)
                st.x = None
        return st
    rows, k, n = case["rows"], case["in"], case["out"]
    if case["w8"]:
        st.w8 = (torch.randint(-127, 128, (n, k), generator=gen, device="cuda", dtype=torch.int8),
                 ((0.75 + 0.5 * torch.rand(n, generator=gen, device="cuda")) / (73.0 * k ** 0.5)).float())
        st.w = None
    else:
        st.w = (_normal(gen, n, k) * k ** -0.5).to(t)
    st.x = _activation(gen, rows, k).to(t)
    if kind == "linear":
        st.bias = (0.1 * _normal(gen, n)).to(t) if case["bias"] else None
        st.residual = _activation(gen, rows, n).to(t) if case["residual"] else None
        return st
    st.dy = _normal(gen, rows, n).to(t)
    st.z = _normal(gen, rows, n).to(t) if case["act"] != "none" else None
    if case["z8"]:
        st.z8 = _rows8(st.z)
        st.z = None
    if case["x8"]:
        st.x8 = _rows8(st.x)
        st.x = None
    return st


def _own_buffers(st):
    """what a program of this library keeps: a context, views of its tensors, output buffers and workspace"""
    import paper_2602_12630_amd as T

    case, t, kind = st.case, st.t, st.case["kind"]
    st.T = T
    st.ctx = T.Context(torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream)

    def matrix(tensor, eight=None):
        if eight is not None:
            return T.Matrix(*eight)
        return T.Matrix(tensor) if tensor is not None else None

    def out(rows, cols, dtype=t):
        return torch.empty(rows, cols, device="cuda", dtype=dtype)

    if kind == "checkpoint":
        rows, cols = case["rows"], case["cols"]
        st.q, st.scale = out(rows, cols, torch.int8), torch.empty(rows, device="cuda", dtype=torch.float32)
        st.back = out(rows, cols)
        st.mx, st.mq, st.mback = T.Matrix(st.x), T.Matrix(st.q, st.scale), T.Matrix(st.back)
        return
    st.mx = matrix(st.x, st.x8)
    if kind in ("norm", "norm_backward"):
        rows, cols = case["rows"], case["cols"]
        st.kind = T.TC_NORM_LAYER if case["norm"] == "layer" else T.TC_NORM_RMS
        st.y = out(rows, cols)
        st.my = T.Matrix(st.y)
        if kind == "norm_backward":
            st.mdy = T.Matrix(st.dy)
            st.dgamma = torch.empty(cols, device="cuda", dtype=torch.float32)
            st.dbeta = torch.empty_like(st.dgamma) if case["norm"] == "layer" else None
            st.workspace = torch.empty(st.ctx.norm_backward_workspace(rows, cols), device="cuda", dtype=torch.uint8)
        return
    rows, k, n = case["rows"], case["in"], case["out"]
    st.act = {"none": T.TC_ACT_NONE, "relu": T.TC_ACT_RELU, "gelu": T.TC_ACT_GELU, "silu": T.TC_ACT_SILU}[case["act"]]
    st.mw = matrix(st.w, st.w8)
    if kind == "linear":
        st.y = out(rows, n)
        st.my = T.Matrix(st.y)
        st.z = out(rows, n) if case["keep_z"] else None
        st.mz, st.mresidual = matrix(st.z), matrix(st.residual)
        st.workspace = torch.empty(st.ctx.linear_workspace(rows, k, n), device="cuda", dtype=torch.uint8)
    else:
        st.mdy, st.mz = T.Matrix(st.dy), matrix(st.z, st.z8)
        st.dz = out(rows, n) if case["act"] != "none" else None
        st.dx = out(rows, k)
        st.dw = out(n, k) if case["dw"] else None
        st.dbias = torch.empty(n, device="cuda", dtype=torch.float32)
        st.mdz, st.mdx, st.mdw = matrix(st.dz), T.Matrix(st.dx), matrix(st.dw)
        st.workspace = torch.empty(st.ctx.linear_backward_workspace(rows, k, n), device="cuda", dtype=torch.uint8)


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _own_buffers(st)
    torch.cuda.synchronize()
    return st


# ---- plain forms ---------------------------------------------------------------------------------------------------
def _value(tensor, eight):
    return tensor.float() if eight is None else eight[0].float() * eight[1][:, None]


def _activate(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.5 ** 0.5))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain(st):
    case, t, kind = st.case, st.t, st.case["kind"]
    if kind == "checkpoint":
        # which whole number is nearest is settled in 64 bits: the products are exact there
        x = st.x.double()
        amax = x.abs().amax(dim=1, keepdim=True)
        q = torch.round(x * 127.0 / torch.where(amax > 0, amax, torch.ones_like(amax))).float()
        scale = (amax / 127.0).float()
        return {"values": (q * scale).to(t), "scale": scale.reshape(-1)}
    if kind == "norm":
        x = st.x.float()
        if case["norm"] == "layer":
            d = x - x.mean(dim=1, keepdim=True)
            y = d * torch.rsqrt(d.square().mean(dim=1, keepdim=True) + EPS) * st.gamma.float() + st.beta.float()
        else:
            y = x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + EPS_RMS) * st.gamma.float()
        return y.to(t)
    if kind == "norm_backward":
        dy, x = st.dy.float(), _value(st.x, st.x8)
        xh = (x - st.mean[:, None]) * st.rstd[:, None]
        g = dy * st.gamma.float()
        dx = g - xh * (g * xh).mean(dim=1, keepdim=True)
        if case["norm"] == "layer":
            dx = dx - g.mean(dim=1, keepdim=True)
        grads = {"dx": (dx * st.rstd[:, None]).to(t), "dgamma": (dy * xh).sum(dim=0)}
        if case["norm"] == "layer":
            grads["dbeta"] = dy.sum(dim=0)
        return grads
    if kind == "linear":
        z = st.x.float() @ _value(st.w, st.w8).t()
        if st.bias is not None:
            z = z + st.bias.float()
        y = _activate(z, case["act"])
        if st.residual is not None:
            y = y + st.residual.float()
        return {"y": y.to(t), "z": z.to(t)} if case["keep_z"] else {"y": y.to(t)}
    dz = st.dy.float()
    grads = {}
    if case["act"] != "none":
        dz = dz * _slope(_value(st.z, st.z8), case["act"])
        grads["dz"] = dz.to(t)
    grads["dx"] = (dz @ _value(st.w, st.w8)).to(t)
    if case["dw"]:
        grads["dw"] = (dz.t() @ _value(st.x, st.x8)).to(t)
    grads["dbias"] = dz.sum(dim=0)
    return grads


def _own(st):
    case, ctx, kind = st.case, st.ctx, st.case["kind"]
    if kind == "checkpoint":
        ctx.checkpoint_encode(st.mx, st.mq)
        ctx.checkpoint_decode(st.mq, st.mback)
        return {"values": st.back, "scale": st.scale}
    if kind == "norm":
        ctx.norm(st.kind, st.mx, st.gamma, st.beta, EPS if case["norm"] == "layer" else EPS_RMS, st.my)
        return st.y
    if kind == "norm_backward":
        ctx.norm_backward(st.kind, st.mdy, st.mx, st.gamma, st.mean, st.rstd, st.my, st.dgamma, st.dbeta, st.workspace)
        grads = {"dx": st.y, "dgamma": st.dgamma}
        if case["norm"] == "layer":
            grads["dbeta"] = st.dbeta
        return grads
    if kind == "linear":
        ctx.linear(st.mx, st.mw, st.my, bias=st.bias, activation=st.act, residual=st.mresidual, z=st.mz, workspace=st.workspace)
        return {"y": st.y, "z": st.z} if case["keep_z"] else {"y": st.y}
    ctx.linear_backward(st.mdy, st.mx, st.mw, activation=st.act, z=st.mz, dz=st.mdz, dx=st.mdx, dw=st.mdw, dbias=st.dbias,
                        workspace=st.workspace)
    grads = {}
    if case["act"] != "none":
        grads["dz"] = st.dz
    grads["dx"] = st.dx
    if case["dw"]:
        grads["dw"] = st.dw
    grads["dbias"] = st.dbias
    return grads


def run(st):
    return _own(st) if own else _plain(st)


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------
def _exact_value(tensor, eight):
    if eight is None:
        return tensor.to(torch.float64)
    q, scale = eight
    return torch.mul(q.to(torch.float64).t(), scale.to(torch.float64)).t()


def exact(case, seed):
    st = _inputs(case, seed)
    kind = case["kind"]
    f64 = torch.float64
    if kind == "checkpoint":
        # floor of (2 * 127 x + amax) / (2 amax) is the nearest whole number, the upper one of two; an upper one that is odd
        # and exactly half a step away gives way to the even one below
        x = st.x.to(f64)
        top = x.abs().max(dim=1).values.unsqueeze(1)
        safe = top.clamp(min=2.0 ** -1000)
        up = torch.floor((254.0 * x + safe) / (2.0 * safe))
        half = (2.0 * up - 1.0) * safe == 254.0 * x
        q = up - (half & (torch.remainder(up, 2.0) == 1.0)).to(f64)
        scale = top / 127.0
        return {"values": q * scale, "scale": scale.squeeze(1)}
    if kind == "norm":
        x = st.x.to(f64)
        n = x.shape[1]
        if case["norm"] == "layer":
            x = x - (x.sum(1) / n).unsqueeze(1)
        length = (torch.linalg.vector_norm(x, dim=1) ** 2 / n + (EPS if case["norm"] == "layer" else EPS_RMS)).sqrt()
        y = x / length.unsqueeze(1) * st.gamma.to(f64)
        return y + st.beta.to(f64) if st.beta is not None else y
    if kind == "norm_backward":
        n = case["cols"]
        rstd = st.rstd.to(f64).unsqueeze(1)
        c = _exact_value(st.x, st.x8).sub_(st.mean.to(f64).unsqueeze(1))
        dy = st.dy.to(f64)
        out = {"dgamma": torch.mul(dy, c).mul_(rstd).sum(0)}
        g = torch.mul(dy, st.gamma.to(f64))
        along = torch.mul(g, c).sum(1).unsqueeze(1) * rstd ** 3 / n
        dx = g * rstd - c * along
        if case["norm"] == "layer":
            dx -= g.sum(1).unsqueeze(1) * rstd / n
            out["dbeta"] = dy.sum(0)
        out["dx"] = dx
        return out
    if kind == "linear":
        z = torch.mm(st.x.to(f64), _exact_value(st.w, st.w8).t())
        if st.bias is not None:
            z += st.bias.to(f64)
        if case["act"] == "relu":
            y = torch.clamp(z, min=0.0)
        elif case["act"] == "gelu":
            y = z * torch.special.erfc(-z / 2.0 ** 0.5) / 2.0
        elif case["act"] == "silu":
            y = z * torch.sigmoid(z)
        else:
            y = z.clone()
        if st.residual is not None:
            y += st.residual.to(f64)
        return {"y": y, "z": z} if case["keep_z"] else {"y": y}
    out = {}
    dz = st.dy.to(f64)
    if case["act"] != "none":
        z = _exact_value(st.z, st.z8)
        if case["act"] == "relu":
            dz = torch.where(z > 0, dz, torch.zeros((), dtype=f64, device=z.device))
        elif case["act"] == "gelu":
            dz = dz * (torch.special.erfc(-z / 2.0 ** 0.5) / 2.0 + z * torch.exp(-z.square() / 2.0) / (2.0 * torch.pi) ** 0.5)
        else:
            dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        out["dz"] = dz
    out["dx"] = torch.mm(dz, _exact_value(st.w, st.w8))
    if case["dw"]:
        out["dw"] = torch.mm(dz.t(), _exact_value(st.x, st.x8))
    out["dbias"] = dz.sum(0)
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "checkpoint":
        n = case["rows"] * case["cols"]
        # the 16-bit rows once, the int8 rows and scales and the restored rows
        return {"bytes": 5 * n + 4 * case["rows"], "flops": 4 * n}
    if kind == "norm":
        n = case["rows"] * case["cols"]
        return {"bytes": 4 * n + (4 if case["norm"] == "layer" else 2) * case["cols"], "flops": 8 * n}
    if kind == "norm_backward":
        n = case["rows"] * case["cols"]
        return {"bytes": (5 if case["x8"] else 6) * n + (12 if case["x8"] else 8) * case["rows"]
                + (10 if case["norm"] == "layer" else 6) * case["cols"], "flops": 14 * n}
    m, k, n = case["rows"], case["in"], case["out"]
    w = n * k * (1 if case["w8"] else 2) + (4 * n if case["w8"] else 0)
    if kind == "linear":
        outs = 1 + case["residual"] + case["keep_z"]
        return {"bytes": w + 2 * m * k + 2 * m * n * outs + (2 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    bent = case["act"] != "none"
    moved = w + 2 * m * n + 2 * m * k + 4 * n
    moved += (1 if case["z8"] else 2) * m * n + 2 * m * n if bent else 0
    moved += ((1 if case["x8"] else 2) * m * k + 2 * n * k) if case["dw"] else 0
    return {"bytes": moved, "flops": 2 * m * n * k * (2 if case["dw"] else 1)}
