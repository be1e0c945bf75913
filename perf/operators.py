"""The dense sublayer's operators, as a program calls them: the linear with its
epilogue, layer norm, both with their backward passes, and the 8-bit
checkpoints of activations that the backward passes read.

    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, s)    what a program holds before the call
    run(state)          one pass, and its outputs (``own``: by the library's
                        calls; else in plain torch operations)
    work(case)          bytes and flops the pass cannot do without
    exact(case, s)      the same outputs from the definitions, in 64 bits

A checkpoint is returned as the values that it stands for (read back in the
same pass).  "pad" adds so many elements to every row's stride.
"""

import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 32            # columns that share one scale of a checkpoint
EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "silu")

FWD = dict(op="linear", dtype="bf16", act="none", bias=True, residual=False, save_z="none",
           save_out=False, pad=0)
BWD = dict(op="linear_backward", dtype="bf16", act="none", bias=True, saved="rows", pad=0)
NORM = dict(op="norm", dtype="bf16", center=True, beta=True, add=True, save=False, pad=0)
NORM_BWD = dict(op="norm_backward", dtype="bf16", center=True, beta=True, saved="rows", dres=True,
                pad=0)
CKPT = dict(op="checkpoint", dtype="bf16", pad=0)


def listed():
    return [
        # single-stream generation: one token through a projection of the
        # DeepSeek-V3-shaped hidden size; the weight is read once
        dict(FWD, name="linear_one_token", m=1, n=2048, k=7168, act="silu"),
        # a serving step of 64 tokens, added into the residual stream
        dict(FWD, name="linear_decode", m=64, n=7168, k=2048, residual=True),
        # ragged tokens, widths that no vector or tile divides, odd strides
        dict(FWD, name="linear_odd", m=777, n=1001, k=1409, act="gelu", residual=True),
        # forward of a training step at the Llama-4-Scout-shaped widths, the
        # pre-activation kept in 8 bits
        dict(FWD, name="linear_train", m=8192, n=8192, k=5120, act="silu", save_z="codes"),
        # fp32 training (numerics checks)
        dict(BWD, name="linear_backward_f32", m=512, n=1408, k=2048, act="relu", dtype="f32"),
        # a training step's backward at the DeepSeek-V2-Lite-shaped widths
        # (two shared experts of 1408 twice over), everything saved in 8 bits
        dict(BWD, name="linear_backward_8bit", m=4096, n=5632, k=2048, act="gelu", saved="codes"),
        # the largest backward, saved rows
        dict(BWD, name="linear_backward_train", m=8192, n=8192, k=5120, act="silu"),
        # the deferred add and the norm before a serving step's block
        dict(NORM, name="norm_decode", m=64, n=7168),
        # the same in training: sum, normalised rows, statistics, and the
        # norm's input kept in 8 bits
        dict(NORM, name="norm_train", m=8192, n=5120, save=True),
        # its backward from the 8-bit input, the residual's gradient added
        dict(NORM_BWD, name="norm_backward_train", m=8192, n=5120, saved="codes"),
        # an activation with ragged rows and columns into 8 bits and back
        dict(CKPT, name="checkpoint_odd", m=1001, n=1409, dtype="f32"),
        # a layer's widest activation into 8 bits and back
        dict(CKPT, name="checkpoint_train", m=8192, n=8192),
    ]


def draw(rng):
    def size(lo, hi):
        n = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        step = rng.choice((1, 1, 8, 64))
        return min(hi, max(lo, n // step * step))

    op = rng.choice(("linear", "linear", "linear", "linear_backward", "linear_backward", "norm",
                     "norm_backward", "checkpoint"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    pad = rng.choice((0, 0, 0, 1, 8))
    if op in ("linear", "linear_backward"):
        most = 2 ** 38 if dtype == "bf16" else 2 ** 35
        m, n, k = size(1, 8192), size(16, 8192), size(16, 8192)
        while m * n * k > most:
            m = max(1, m // 2)
        c = dict(dtype=dtype, m=m, n=n, k=k, act=rng.choice(ACTS), bias=rng.random() < 0.7, pad=pad)
        if op == "linear":
            return dict(FWD, **{**c, "residual": rng.random() < 0.5,
                                "save_z": rng.choice(("none", "none", "rows", "codes")),
                                "save_out": rng.random() < 0.2})
        return dict(BWD, **{**c, "saved": rng.choice(("rows", "codes"))})
    c = dict(dtype=dtype, m=size(1, 16384), n=size(32, 16384), pad=pad)
    while c["m"] * c["n"] > 2 ** 26:
        c["m"] = max(1, c["m"] // 2)
    if op == "checkpoint":
        return dict(CKPT, **c)
    c.update(center=rng.random() < 0.7, beta=rng.random() < 0.7)
    if op == "norm":
        return dict(NORM, **{**c, "add": rng.random() < 0.6, "save": rng.random() < 0.5})
    return dict(NORM_BWD, **{**c, "saved": rng.choice(("rows", "codes")), "dres": rng.random() < 0.5})


# ------------------------------------------------------------------ inputs
def _rows(gen, m, n, case, scale=1.0):
    """[m, n] of N(0, scale^2) with the case's type and row stride."""
    full = torch.empty((m, n + case["pad"]), dtype=DTYPES[case["dtype"]], device=DEV)
    full.normal_(0.0, scale, generator=gen)
    return full[:, :n]


def _stream(gen, m, n, case):
    """Rows of a residual stream: a few channels are much larger than the
    rest, and rows differ in size."""
    x = torch.randn((m, n), generator=gen, device=DEV)
    chan = torch.rand((n,), generator=gen, device=DEV)
    x *= torch.where(chan < 0.005, 20.0, 1.0) * (0.3 + chan)
    x *= 0.5 + 2.0 * torch.rand((m, 1), generator=gen, device=DEV)
    out = _rows(gen, m, n, case)
    out.copy_(x)
    return out


def _vec(gen, n, mid, spread):
    return mid + spread * torch.randn((n,), generator=gen, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    m, n = case["m"], case["n"]
    op = case["op"]
    s = {"case": case, "keep": {}}
    if op in ("linear", "linear_backward"):
        k = case["k"]
        s["a"] = _rows(gen, m, k, case)
        s["w"] = _rows(gen, n, k, case, 1.0 / math.sqrt(k))
        s["bias"] = _vec(gen, n, 0.0, 0.2) if case["bias"] else None
        if op == "linear":
            s["residual"] = _stream(gen, m, n, case) if case["residual"] else None
        else:
            s["z"] = _rows(gen, m, n, case, 1.2)
            s["dout"] = _rows(gen, m, n, case, 0.05)
    else:
        s["x"] = _stream(gen, m, n, case)
        if op != "checkpoint":
            s["gamma"] = _vec(gen, n, 1.0, 0.2)
            s["beta"] = _vec(gen, n, 0.0, 0.2) if case["beta"] else None
        if op == "norm":
            s["add"] = _rows(gen, m, n, case, 0.5) if case["add"] else None
        if op == "norm_backward":
            s["dy"] = _rows(gen, m, n, case, 0.05)
            s["dres"] = _rows(gen, m, n, case, 0.05) if case["dres"] else None
            x = s["x"].float()
            s["mean"] = x.mean(1) if case["center"] else torch.zeros((m,), device=DEV)
            var = (x - s["mean"][:, None]).square().mean(1)
            s["rstd"] = torch.rsqrt(var + EPS)
    if case.get("saved") == "codes":
        # what the forward pass kept: codes and scale bytes in place of rows
        for name in ("a", "z") if op == "linear_backward" else ("x",):
            s[name] = _encode(s[name])
    return s


# -------------------------------------------------------------- plain form
def _pow2(e):
    """2^e in fp32, exactly, by its exponent field."""
    return ((e + 127).int() << 23).view(torch.float32)


def _encode(x):
    """Codes [m, n] and scale bytes [m, ceil(n / 32)] of a checkpoint."""
    m, n = x.shape
    nb = (n + BLOCK - 1) // BLOCK
    v = torch.zeros((m, nb * BLOCK), dtype=torch.float32, device=x.device)
    v[:, :n] = x
    v = v.view(m, nb, BLOCK)
    frac, exp = torch.frexp(v.abs().amax(2))
    e = torch.clamp_min(exp - torch.where(frac <= 0.875, 9, 8), -117)
    codes = (v * _pow2(-e)[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.view(m, nb * BLOCK)[:, :n].contiguous(), (e + 127).to(torch.uint8)


def _decode(codes, scales):
    """The fp32 values that a checkpoint stands for (exact)."""
    m, n = codes.shape
    v = codes.view(torch.float8_e4m3fn).float()
    return v * _pow2(scales.int() - 127).repeat_interleave(BLOCK, dim=1)[:, :n]


def _values(t):
    return _decode(*t) if isinstance(t, tuple) else t.float()


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        g = 1.0 / (1.0 + torch.exp(-z))
        return g * (1.0 + z * (1.0 - g))
    return torch.ones_like(z)


def _plain(s):
    c = s["case"]
    dt = DTYPES[c["dtype"]]
    op = c["op"]
    out = {}
    if op == "linear":
        z = s["a"].float() @ s["w"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(z, c["act"])
        if s["residual"] is not None:
            y = y + s["residual"].float()
        out["out"] = y.to(dt)
        if c["save_z"] == "rows":
            out["z"] = z.to(dt)
        elif c["save_z"] == "codes":
            out["z"] = _decode(*_encode(z.to(dt))).to(dt)
        if c["save_out"]:
            out["saved_out"] = _decode(*_encode(out["out"])).to(dt)
    elif op == "linear_backward":
        dz = s["dout"].float()
        if c["act"] != "none":
            dz = dz * _act_grad(_values(s["z"]), c["act"])
        out["da"] = (dz @ s["w"].float()).to(dt)
        out["dw"] = (dz.t() @ _values(s["a"])).to(dt)
        if s["bias"] is not None:
            out["dbias"] = dz.sum(0)
    elif op == "norm":
        x = s["x"]
        if s["add"] is not None:
            x = (x.float() + s["add"].float()).to(dt)
            out["sum"] = x
        v = x.float()
        mean = v.mean(1, keepdim=True) if c["center"] else torch.zeros((c["m"], 1), device=DEV)
        rstd = torch.rsqrt((v - mean).square().mean(1, keepdim=True) + EPS)
        y = (v - mean) * rstd * s["gamma"]
        if s["beta"] is not None:
            y = y + s["beta"]
        out.update(y=y.to(dt), rstd=rstd[:, 0])
        if c["center"]:
            out["mean"] = mean[:, 0]
        if c["save"]:
            out["saved"] = _decode(*_encode(x)).to(dt)
    elif op == "norm_backward":
        dy = s["dy"].float()
        h = (_values(s["x"]) - s["mean"][:, None]) * s["rstd"][:, None]
        u = dy * s["gamma"]
        g = u - h * (u * h).mean(1, keepdim=True)
        if c["center"]:
            g = g - u.mean(1, keepdim=True)
        g = g * s["rstd"][:, None]
        if s["dres"] is not None:
            g = g + s["dres"].float()
        out.update(dx=g.to(dt), dgamma=(dy * h).sum(0))
        if s["beta"] is not None:
            out["dbeta"] = dy.sum(0)
    else:
        out["saved"] = _decode(*_encode(s["x"])).to(dt)
    return out


# ------------------------------------------------------- the library's calls
def _kept(s, name, make):
    """What the program keeps from pass to pass: workspace, descriptor, outputs."""
    if name not in s["keep"]:
        s["keep"][name] = make()
    return s["keep"][name]


def _call(s):
    import paper_2511_11505_amd as fs

    c = s["case"]
    dt = DTYPES[c["dtype"]]
    dtype = fs.FS_BF16 if c["dtype"] == "bf16" else fs.FS_F32
    op, m, n = c["op"], c["m"], c["n"]

    def rows(name, r=m, cols=n):
        return _kept(s, name, lambda: torch.empty((r, cols), dtype=dt, device=DEV))

    def vec(name, size):
        return _kept(s, name, lambda: torch.empty((size,), dtype=torch.float32, device=DEV))

    def codes(name):
        return _kept(s, name, lambda: fs.checkpoint_buffers(m, n, DEV))

    def space(nbytes):
        return _kept(s, "ws", lambda: torch.empty((max(256, nbytes()),), dtype=torch.uint8, device=DEV))

    def values(name, saved):
        fs.fs_checkpoint_restore(dtype, m, n, *saved, rows(name))
        return rows(name)

    out = {}
    if op == "linear":
        desc = _kept(s, "desc", lambda: fs.linear_desc(m, n, c["k"], c["dtype"], c["act"]))
        ws = space(lambda: fs.fs_linear_workspace(desc, fs.FS_OP_LINEAR))
        out["out"] = rows("out")
        save_z = {"none": lambda: None, "rows": lambda: rows("z"), "codes": lambda: codes("zc")}[c["save_z"]]()
        save_out = codes("oc") if c["save_out"] else None
        fs.fs_linear(desc, s["a"], s["w"], s["bias"], s["residual"], out["out"], ws, save_z=save_z,
                     save_out=save_out)
        if save_z is not None:
            out["z"] = save_z if c["save_z"] == "rows" else values("z", save_z)
        if save_out is not None:
            out["saved_out"] = values("so", save_out)
    elif op == "linear_backward":
        k = c["k"]
        desc = _kept(s, "desc", lambda: fs.linear_desc(m, n, k, c["dtype"], c["act"]))
        ws = space(lambda: fs.fs_linear_workspace(desc, fs.FS_OP_LINEAR_BACKWARD))
        out["da"], out["dw"] = rows("da", m, k), rows("dw", n, k)
        if s["bias"] is not None:
            out["dbias"] = vec("dbias", n)
        z = None if c["act"] == "none" else s["z"]
        fs.fs_linear_backward(desc, s["dout"], s["a"], s["w"], z, out["da"], out["dw"],
                              out.get("dbias"), ws)
    elif op == "norm":
        desc = _kept(s, "desc", lambda: fs.norm_desc(m, n, c["dtype"], c["center"], EPS))
        out["y"], out["rstd"] = rows("y"), vec("rstd", m)
        if c["center"]:
            out["mean"] = vec("mean", m)
        if c["add"]:
            out["sum"] = rows("sum")
        save = codes("xc") if c["save"] else None
        fs.fs_layer_norm(desc, s["x"], s["add"], s["gamma"], s["beta"], out.get("sum"), out["y"],
                         out.get("mean"), out["rstd"], save_in=save)
        if c["save"]:
            out["saved"] = values("saved", save)
    elif op == "norm_backward":
        desc = _kept(s, "desc", lambda: fs.norm_desc(m, n, c["dtype"], c["center"], EPS))
        ws = space(lambda: fs.fs_layer_norm_workspace(desc))
        out["dx"], out["dgamma"] = rows("dx"), vec("dgamma", n)
        if s["beta"] is not None:
            out["dbeta"] = vec("dbeta", n)
        fs.fs_layer_norm_backward(desc, s["dy"], s["x"], s["mean"] if c["center"] else None, s["rstd"],
                                  s["gamma"], s["dres"], out["dx"], out["dgamma"], out.get("dbeta"), ws)
    else:
        saved = codes("xc")
        fs.fs_checkpoint_fp8(dtype, m, n, s["x"], *saved)
        out["saved"] = values("saved", saved)
    return out


def run(state):
    if own:
        return _call(state)
    return _plain(state)


# ----------------------------------------------------------- work and oracle
def work(case):
    m, n, op = case["m"], case["n"], case["op"]
    e = 2 if case["dtype"] == "bf16" else 4
    coded = m * n + m * ((n + BLOCK - 1) // BLOCK)
    if op == "linear":
        k = case["k"]
        b = e * (m * k + n * k + m * n * (2 if case["residual"] else 1)) + (4 * n if case["bias"] else 0)
        b += {"none": 0, "rows": e * m * n, "codes": 2 * coded + e * m * n}[case["save_z"]]
        b += 2 * coded + e * m * n if case["save_out"] else 0
        return {"bytes": b, "flops": 2.0 * m * n * k}
    if op == "linear_backward":
        k = case["k"]
        ck = m * k + m * ((k + BLOCK - 1) // BLOCK)
        b = e * (m * n + n * k + m * k + n * k) + (4 * n if case["bias"] else 0)
        b += ck if case["saved"] == "codes" else e * m * k
        if case["act"] != "none":
            b += coded if case["saved"] == "codes" else e * m * n
        return {"bytes": b, "flops": 4.0 * m * n * k}
    if op == "norm":
        b = e * m * n * (4 if case["add"] else 2) + 8 * m + 8 * n
        b += 2 * coded + e * m * n if case["save"] else 0
        return {"bytes": b, "flops": 8.0 * m * n}
    if op == "norm_backward":
        b = e * m * n * (3 if case["dres"] else 2) + 8 * m + 12 * n
        b += coded if case["saved"] == "codes" else e * m * n
        return {"bytes": b, "flops": 16.0 * m * n}
    return {"bytes": 2 * e * m * n + 2 * coded, "flops": 4.0 * m * n}


def _f64_saved(t):
    """Values of a saved activation, each code decoded from its bits."""
    if not isinstance(t, tuple):
        return t.double()
    codes, scales = t
    c = codes.long()
    field, man = (c >> 3) & 15, (c & 7).double()
    mag = torch.where(field == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * 2.0 ** (field.double() - 7))
    col = torch.arange(codes.shape[1], device=codes.device) // BLOCK
    return torch.where(c >= 128, -mag, mag) * 2.0 ** (scales.double()[:, col] - 127)


def _f64_rounded(x, dt):
    return x.to(dt).double()


def _f64_coded(x):
    """x (64 bits, already of the stored type's values) through a checkpoint,
    by arithmetic on the code's grid."""
    m, n = x.shape
    pad = (-n) % BLOCK
    v = torch.nn.functional.pad(x, (0, pad)).reshape(m, -1, BLOCK)
    top = v.abs().amax(2, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp_min(top, 1e-300) / 448))
    e = torch.where(top > 448 * 2.0 ** e, e + 1, e)
    e = torch.where(top <= 448 * 2.0 ** (e - 1), e - 1, e).clamp_min(-117)
    q = v * 2.0 ** -e
    grid = 2.0 ** (torch.floor(torch.log2(torch.clamp_min(q.abs(), 2.0 ** -6))) - 3)
    return (torch.round(q / grid) * grid * 2.0 ** e).reshape(m, n + pad)[:, :n]


def exact(case, seed):
    s = prepare(case, seed)
    dt = DTYPES[case["dtype"]]
    op = case["op"]
    if op == "linear":
        z = torch.mm(s["a"].double(), s["w"].double().t().contiguous())
        if s["bias"] is not None:
            z += s["bias"].double()
        act = case["act"]
        y = {"none": lambda: z.clone(), "relu": lambda: z.clamp_min(0),
             "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[act]()
        if s["residual"] is not None:
            y += s["residual"].double()
        out = {"out": y}
        if case["save_z"] == "rows":
            out["z"] = z
        elif case["save_z"] == "codes":
            out["z"] = _f64_coded(_f64_rounded(z, dt))
        if case["save_out"]:
            out["saved_out"] = _f64_coded(_f64_rounded(y, dt))
        return out
    if op == "linear_backward":
        dz = s["dout"].double()
        z = _f64_saved(s["z"])
        act = case["act"]
        if act == "relu":
            dz = torch.where(z > 0, dz, torch.zeros_like(dz))
        elif act == "gelu":
            dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
        elif act == "silu":
            dz = dz * torch.sigmoid(z) * (1 + z * torch.sigmoid(-z))
        out = {"da": torch.mm(dz, s["w"].double()),
               "dw": torch.mm(dz.t().contiguous(), _f64_saved(s["a"]))}
        if s["bias"] is not None:
            out["dbias"] = dz.sum(0)
        return out
    if op == "norm":
        x = s["x"].double()
        out = {}
        if s["add"] is not None:
            out["sum"] = x + s["add"].double()
            x = _f64_rounded(out["sum"], dt)
        var, mean = torch.var_mean(x, 1, correction=0)
        if not case["center"]:
            var, mean = x.pow(2).mean(1), torch.zeros_like(mean)
        out["rstd"] = (var + EPS) ** -0.5
        y = s["gamma"].double() * (x - mean[:, None]) * out["rstd"][:, None]
        out["y"] = y if s["beta"] is None else y + s["beta"].double()
        if case["center"]:
            out["mean"] = mean
        if case["save"]:
            out["saved"] = _f64_coded(x)
        return out
    if op == "norm_backward":
        dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
        h = (_f64_saved(s["x"]) - s["mean"].double()[:, None]) * rstd
        u = dy * s["gamma"].double()
        dx = u - h * torch.mean(h * u, 1, keepdim=True)
        if case["center"]:
            dx -= torch.mean(u, 1, keepdim=True)
        dx *= rstd
        if s["dres"] is not None:
            dx += s["dres"].double()
        out = {"dx": dx, "dgamma": torch.einsum("mn,mn->n", dy, h)}
        if s["beta"] is not None:
            out["dbeta"] = torch.sum(dy, 0)
        return out
    return {"saved": _f64_coded(s["x"].double())}
