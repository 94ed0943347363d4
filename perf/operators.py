"""The operators of an 8-bit feed-forward path, as measurable cases.

Kinds of a case:
  norm_fwd   niti.rmsnorm_fwd: residual addition, root-mean-square norm, int8 rows with a scale each
  norm_bwd   niti.rmsnorm_bwd: the gradients of its input and of its gain
  quant      niti.quantize_rows: a float matrix as int8 rows with a scale each
  lin_fwd    niti.linear_fwd: product of int8 rows with bias, activation and residual in its epilogue
  lin_bwd    niti.linear_bwd: the gradients of its operands and its bias, by int8 products
  adamw      niti.adamw_step over many tensors at once, with states in 32 or in 8 bits

Int8 results come back as the values they stand for: the norm and the
quantisation write these themselves (their output y), the optimiser's states
are read by niti.adamw_read.  A step of a quantisation is near 1% of a row's
largest value, and the last bit of a sum decides ties: such values are in the
tensor's own 16-bit type, and 32-bit cases go without int8 results.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = 2.0 ** -100     # the least row maximum that a scale is formed from
EPS = 1e-6
BLOCK = 256            # elements that share a scale in an 8-bit state
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01

# The weights of the networks of this repository, in elements.
NETS = {
    "lenet5": [150, 2400, 48000, 10080, 840],
    "alexnet": [96 * 121 * 4, 256 * 25 * 96, 384 * 9 * 256, 384 * 9 * 384, 256 * 9 * 384, 9216 * 4096, 4096 * 4096,
                4096 * 1000],
}


def norm_fwd(m, d, dtype, res, quant):
    return {"kind": "norm_fwd", "m": m, "d": d, "dtype": dtype, "res": res, "quant": quant}


def norm_bwd(m, d, dtype, dh):
    return {"kind": "norm_bwd", "m": m, "d": d, "dtype": dtype, "dh": dh}


def quant(m, d, dtype, mode):
    return {"kind": "quant", "m": m, "d": d, "dtype": dtype, "mode": mode}


def lin_fwd(m, n, k, dtype, act, bias, res, keep):
    return {"kind": "lin_fwd", "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "bias": bias, "res": res, "keep": keep}


def lin_bwd(m, n, k, dtype, act, mode):
    return {"kind": "lin_bwd", "m": m, "n": n, "k": k, "dtype": dtype, "act": act, "mode": mode}


def adamw(bits, grad, mode, net=None, count=0, total=0):
    d = {"kind": "adamw", "bits": bits, "grad": grad, "mode": mode}
    return dict(d, net=net) if net else dict(d, count=count, total=total)


def listed():
    return [
        # serving, one token: the norm before a product; a call's latency
        dict(norm_fwd(1, 4096, "bf16", True, True), name="norm_1x4096"),
        # training or reading a prompt of 4096 tokens at that width
        dict(norm_fwd(4096, 4096, "bf16", True, True), name="norm_4096x4096"),
        # its backward pass, with the gradient that arrives by the residual stream
        dict(norm_bwd(4096, 4096, "bf16", True), name="norm_bwd_4096x4096"),
        # an odd width and an odd number of rows, in 32 bits
        dict(norm_bwd(1777, 1111, "f32", False), name="norm_bwd_1777x1111_f32"),
        # a layer's weights laid out as int8 rows after an update
        dict(quant(4096, 9216, "bf16", "rtn"), name="quant_4096x9216"),
        # a small ragged batch of errors, rounded stochastically
        dict(quant(321, 1000, "f16", "sr"), name="quant_321x1000_sr"),
        # serving, one token through a 4096 x 4096 layer: the weights are the traffic
        dict(lin_fwd(1, 4096, 4096, "bf16", "silu", True, False, False), name="lin_1x4096x4096"),
        # a ragged prompt: no size is a multiple of 16 but one
        dict(lin_fwd(1000, 1500, 1111, "f32", "gelu", True, True, True), name="lin_1000x1500x1111_f32"),
        # the large square product, with bias and residual
        dict(lin_fwd(8192, 8192, 8192, "bf16", "none", True, True, False), name="lin_8192"),
        # the backward pass of a hidden layer on 2048 tokens
        dict(lin_bwd(2048, 4096, 4096, "bf16", "silu", "rtn"), name="lin_bwd_2048x4096x4096"),
        # a small network's step: five tensors of 61470 weights in all
        dict(adamw(32, "f32", "rtn", net="lenet5"), name="adamw32_lenet5"),
        # a large network's step: eight tensors of 62.4M weights, states in 8 bits with stochastic rounding
        dict(adamw(8, "bf16", "sr", net="alexnet"), name="adamw8_alexnet"),
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of lo..hi."""
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi):
    """A size as layers have them: mostly whole 64s or 16s, else any."""
    v, unit = _log(rng, lo, hi), rng.choice([64, 64, 16, 1])
    return max(unit, v // unit * unit)


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_bwd", "quant", "lin_fwd", "lin_fwd", "lin_bwd", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    half = "bf16" if dtype == "f32" else dtype
    if kind in ("norm_fwd", "norm_bwd", "quant"):
        while True:
            m, d = _log(rng, 1, 16384), _size(rng, 64, 16384)
            if m * d <= 4096 * 9216:
                break
        if kind == "norm_fwd":
            return norm_fwd(m, d, dtype, rng.random() < 0.7, dtype != "f32")
        if kind == "norm_bwd":
            return norm_bwd(m, d, dtype, rng.random() < 0.5)
        return quant(m, d, half, rng.choice(["rtn", "sr"]))
    if kind in ("lin_fwd", "lin_bwd"):
        while True:
            m, n, k = _log(rng, 1, 8192), _size(rng, 32, 9216), _size(rng, 32, 9216)
            if m * n * k <= (8192 ** 3 if kind == "lin_fwd" else 8192 ** 3 // 2):
                break
        act = rng.choice(["none", "relu", "gelu", "silu"])
        if kind == "lin_fwd":
            return lin_fwd(m, n, k, dtype, act, rng.random() < 0.6, rng.random() < 0.5, rng.random() < 0.3)
        return lin_bwd(m, n, k, half, act, rng.choice(["rtn", "sr"]))
    return adamw(rng.choice([8, 32]), rng.choice(["f32", "bf16"]), rng.choice(["rtn", "sr"]),
                 count=_log(rng, 1, 160), total=_log(rng, 2000, 60_000_000))


def _sizes(case):
    """Elements of each tensor of an optimiser's case: a network's, or large and small ones in turn, odd sizes among them."""
    if case.get("net"):
        return NETS[case["net"]]
    weights = [1.0 / (1 + (7 * i) % 13) ** 2 for i in range(case["count"])]
    return [max(1, int(case["total"] * w / sum(weights))) for w in weights]


# ------------------------------------------------------------------ inputs
def _quantised(x):
    """A float matrix as int8 rows and their scales."""
    top = x.abs().amax(dim=1, keepdim=True).clamp(min=TINY)
    return (x * (127.0 / top)).round().clamp(-127, 127).to(torch.int8), (top / 127.0).squeeze(1)


def prepare(case, seed):
    """Inputs, and the buffers, workspaces and plans that a program keeps.

    A plan or workspace is the package's own: only where it is used are they
    made.  All else is the same on both sides."""
    if own:
        from paper_2009_13108_amd import niti
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def stream(m, d):
        """Activations of a residual stream: normal, a few channels far larger."""
        return randn(m, d) * (1 + 9 * (torch.rand(d, generator=g, device="cuda") < 0.005))

    def errors(m, d):
        """Errors: small, of another size in each row."""
        return randn(m, d) * 1e-3 * torch.exp(randn(m, 1))

    s = {"case": case, "seed": int(seed)}
    kind = case["kind"]
    t = TYPES[case["dtype"]] if "dtype" in case else None
    if kind == "norm_fwd":
        m, d = case["m"], case["d"]
        s.update(x=stream(m, d).to(t), res=stream(m, d).to(t) if case["res"] else None, gain=(1 + 0.1 * randn(d)).to(t),
                 h=empty(m, d, dtype=t) if case["res"] else None, y=empty(m, d, dtype=t), rstd=empty(m),
                 q=empty(m, d, dtype=torch.int8) if case["quant"] else None, scale=empty(m) if case["quant"] else None)
    elif kind == "norm_bwd":
        m, d = case["m"], case["d"]
        h = stream(m, d).to(t)
        s.update(dy=errors(m, d).to(t), h=h, gain=(1 + 0.1 * randn(d)).to(t), dh=errors(m, d).to(t) if case["dh"] else None,
                 rstd=torch.rsqrt(h.float().square().mean(dim=1) + EPS), dx=empty(m, d, dtype=t), dgain=empty(d))
        if own:
            s["ws"] = niti.new_workspace(niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, m, d))
    elif kind == "quant":
        m, d = case["m"], case["d"]
        s.update(x=(errors(m, d) if case["mode"] == "sr" else randn(m, d) * 0.02).to(t), q=empty(m, d, dtype=torch.int8),
                 scale=empty(m), y=empty(m, d, dtype=t))
    elif kind in ("lin_fwd", "lin_bwd"):
        m, n, k = case["m"], case["n"], case["k"]
        a, s_a = _quantised(stream(m, k))
        b, s_b = _quantised(randn(n, k) / math.sqrt(k))
        s.update(a=a, s_a=s_a, b=b, s_b=s_b)
        if kind == "lin_fwd":
            s.update(bias=(0.1 * randn(n)).to(t) if case["bias"] else None, res=randn(m, n).to(t) if case["res"] else None,
                     out=empty(m, n, dtype=t), z=empty(m, n, dtype=t) if case["keep"] else None)
        else:
            s.update(dy=errors(m, n).to(t), z=(1.5 * randn(m, n)).to(t) if case["act"] != "none" else None,
                     da=empty(m, k, dtype=t), db=empty(n, k, dtype=t), dbias=empty(n))
        if own:
            op = niti.OP_LINEAR_FWD if kind == "lin_fwd" else niti.OP_LINEAR_BWD
            s["ws"] = niti.new_workspace(niti.workspace_bytes(op, None, m, n, k))
    else:
        # Every tensor begins a block of 256 elements of one arena, so that
        # the plain form can take them all at once; what lies between is zero.
        sizes = _sizes(case)
        starts, at = [], 0
        for v in sizes:
            starts.append(at)
            at += -(-v // BLOCK) * BLOCK
        used = torch.zeros(at, dtype=torch.bool, device="cuda")
        for v, o in zip(sizes, starts):
            used[o:o + v] = True
        p, gr = 0.02 * randn(at) * used, (1e-3 * randn(at) * used).to(TYPES[case["grad"]])
        mom, var = 3e-4 * randn(at) * used, 1e-6 * (0.05 + randn(at).square()) * used
        s.update(p=p, g=gr, used=used, gscale=torch.tensor(0.75, device="cuda"), step=100)
        if case["bits"] == 8:
            mb, vb = mom.view(-1, BLOCK), var.view(-1, BLOCK)
            ms, vs = mb.abs().amax(dim=1) / 16129.0, vb.amax(dim=1) / 255.0 ** 4
            s.update(m=((mb.abs() / ms[:, None]).sqrt().round().clamp(max=127) * mb.sign()).view(-1).to(torch.int8),
                     v=torch.where(vb > 0, (vb / vs[:, None]).sqrt().sqrt().round().clamp(1, 255),
                                   torch.zeros_like(vb)).view(-1).to(torch.uint8), ms=ms, vs=vs,
                     m_read=torch.zeros(at, dtype=torch.bfloat16, device="cuda"),
                     v_read=torch.zeros(at, dtype=torch.bfloat16, device="cuda"))
        else:
            s.update(m=mom, v=var)
        if own:
            def parts(x, unit=1):
                return [x[o // unit:o // unit + -(-v // unit)] for v, o in zip(sizes, starts)]
            more = {}
            if case["bits"] == 8:
                more = dict(m_scale=parts(s["ms"], BLOCK), v_scale=parts(s["vs"], BLOCK), m_read=parts(s["m_read"]),
                            v_read=parts(s["v_read"]))
            s["plan"] = niti.adamw_plan(parts(p), parts(gr), parts(s["m"]), parts(s["v"]), **more)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return PLAIN[kind](s)
    from paper_2009_13108_amd import niti
    if kind == "norm_fwd":
        niti.rmsnorm_fwd(s["x"], s["gain"], res=s["res"], h=s["h"], y=s["y"], q=s["q"], scale=s["scale"], rstd=s["rstd"],
                         eps=EPS)
        return {"h": s["h"], "y": s["y"], "scale": s["scale"], "rstd": s["rstd"]}
    if kind == "norm_bwd":
        niti.rmsnorm_bwd(s["dy"], s["h"], s["gain"], s["rstd"], s["dx"], s["dgain"], s["ws"], dh=s["dh"])
        return {"dx": s["dx"], "dgain": s["dgain"]}
    mode = (niti.SR if case["mode"] == "sr" else niti.RTN) if "mode" in case else None
    if kind == "quant":
        niti.quantize_rows(s["x"], s["q"], s["scale"], y=s["y"], mode=mode, seed=s["seed"], call=7)
        return {"y": s["y"], "scale": s["scale"]}
    act = getattr(niti, "ACT_" + case["act"].upper()) if "act" in case else None
    if kind == "lin_fwd":
        niti.linear_fwd(s["a"], s["b"], s["out"], s["s_a"], s["s_b"], bias=s["bias"], act=act, res=s["res"], z=s["z"],
                        ws=s["ws"])
        return {"out": s["out"], "z": s["z"]}
    if kind == "lin_bwd":
        niti.linear_bwd(s["dy"], s["a"], s["b"], s["s_a"], s["s_b"], s["ws"], z=s["z"], act=act, da=s["da"], db=s["db"],
                        dbias=s["dbias"], mode=mode, seed=s["seed"], call=7)
        return {"da": s["da"], "db": s["db"], "dbias": s["dbias"]}
    s["step"] += 1
    niti.adamw_step(s["plan"], s["step"], LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, weight_decay=DECAY,
                    grad_scale=s["gscale"], mode=mode, seed=s["seed"])
    if case["bits"] == 8:
        niti.adamw_read(s["plan"])
        return {"p": s["p"], "m": s["m_read"], "v": s["v_read"]}
    return {"p": s["p"], "m": s["m"], "v": s["v"]}


# ------------------------------------------------------------------ plain forms, in 32 bits
GOLDEN, MIX1, MIX2 = (v - (1 << 64) for v in (0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB))


def _shift(z, n):
    """Logical right shift of 64-bit words that are held as signed."""
    return (z >> n) & ((1 << (64 - n)) - 1)


def _signed(v):
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _draws(seed, call, n):
    """SplitMix64 outputs call 2^40 + 1 ... call 2^40 + n of the stream of seed."""
    z = torch.arange(1, n + 1, device="cuda", dtype=torch.int64) * GOLDEN + _signed(seed + (call << 40) * GOLDEN)
    z = (z ^ _shift(z, 30)) * MIX1
    z = (z ^ _shift(z, 27)) * MIX2
    return z ^ _shift(z, 31)


def _codes(x, dim, u):
    """Codes of x with one scale along dim, and the scales; u: the draws of stochastic rounding, or None."""
    top = x.abs().amax(dim=dim, keepdim=True).clamp(min=TINY)
    r = x * (127.0 / top)
    return (r.round() if u is None else (r + u).floor()).clamp(-127, 127), top / 127.0


def _activation(name, z):
    if name == "relu":
        return z.clamp(min=0)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(name, z):
    if name == "relu":
        return (z > 0).float()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    sg = 1 / (1 + torch.exp(-z))
    return sg * (1 + z * (1 - sg))


def _plain_norm_fwd(s):
    t = s["x"].dtype
    h = s["x"].float()
    if s["res"] is not None:
        h = h + s["res"].float()
    rstd = 1 / torch.sqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    y = h * rstd * s["gain"].float()
    scale = None
    if s["case"]["quant"]:
        c, scale = _codes(y, 1, None)
        y, scale = c * scale, scale.squeeze(1)
    return {"h": h.to(t) if s["res"] is not None else None, "y": y.to(t), "scale": scale, "rstd": rstd.squeeze(1)}


def _plain_norm_bwd(s):
    dy, xh = s["dy"].float(), s["h"].float() * s["rstd"][:, None]
    t = dy * s["gain"].float()
    dx = s["rstd"][:, None] * (t - xh * (t * xh).mean(dim=1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(s["dy"].dtype), "dgain": (dy * xh).sum(dim=0)}


def _plain_quant(s):
    x = s["x"].float()
    u = None
    if s["case"]["mode"] == "sr":
        u = _shift(_draws(s["seed"], 7, x.numel()), 40).float().view(x.shape) * 2.0 ** -24
    c, scale = _codes(x, 1, u)
    return {"y": (c * scale).to(s["x"].dtype), "scale": scale.squeeze(1)}


def _plain_lin_fwd(s):
    t = s["out"].dtype
    z = (s["a"].float() @ s["b"].float().t()) * (s["s_a"][:, None] * s["s_b"])
    if s["bias"] is not None:
        z = z + s["bias"].float()
    out = _activation(s["case"]["act"], z)
    if s["res"] is not None:
        out = out + s["res"].float()
    return {"out": out.to(t), "z": z.to(t) if s["case"]["keep"] else None}


def _plain_lin_bwd(s):
    t = s["dy"].dtype
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _slope(s["case"]["act"], s["z"].float())
    u = v = None
    if s["case"]["mode"] == "sr":
        r = _draws(s["seed"], 7, dz.numel()).view(dz.shape)
        u, v = _shift(r, 40).float() * 2.0 ** -24, (_shift(r, 8) & 0xFFFFFF).float() * 2.0 ** -24
    c, sc = _codes(dz * s["s_b"], 1, u)
    da = (c @ s["b"].float()) * sc
    c, sc = _codes(dz * s["s_a"][:, None], 0, v)
    db = (c.t() @ s["a"].float()) * sc.t()
    return {"da": da.to(t), "db": db.to(t), "dbias": dz.sum(dim=0)}


def _plain_adamw(s):
    """In place, as the step is: the arena's parameters and states are the new ones afterwards."""
    case = s["case"]
    s["step"] += 1
    bits8 = case["bits"] == 8
    if bits8:
        c = s["m"].view(-1, BLOCK).float()
        m = (c * c.abs() * s["ms"][:, None]).view(-1)
        c = s["v"].view(-1, BLOCK).float()
        v = ((c * c) * (c * c) * s["vs"][:, None]).view(-1)
    else:
        m, v = s["m"], s["v"]
    g = s["g"].float() * s["gscale"]
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    up = m / (torch.sqrt(v) * (1 / math.sqrt(1 - BETA2 ** s["step"])) + ADAM_EPS)
    s["p"].mul_(1 - LR * DECAY).sub_(up * (LR / (1 - BETA1 ** s["step"])))
    if not bits8:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {"p": s["p"], "m": s["m"], "v": s["v"]}
    mb, vb = m.view(-1, BLOCK), v.view(-1, BLOCK)
    ms, vs = mb.abs().amax(dim=1, keepdim=True), vb.amax(dim=1, keepdim=True)
    ms, vs = (torch.where(top < TINY, 0.0, top) for top in (ms, vs))
    rm, rv = (x / top.clamp(min=TINY) for x, top in ((mb.abs(), ms), (vb, vs)))
    rm, rv = 127 * rm.sqrt(), 255 * rv.sqrt().sqrt()
    if case["mode"] == "sr":
        r = _draws(s["seed"], s["step"], -(-m.numel() // 2))
        u = torch.stack([_shift(r, k) & 0xFFFF for k in (0, 16, 32, 48)], dim=1).float() * 2.0 ** -16
        rm = (rm + u[:, 0::2].reshape(rm.shape)).floor()
        rv = (rv + u[:, 1::2].reshape(rv.shape)).floor()
    else:
        rm, rv = rm.round(), rv.round()
    cm = torch.where(ms > 0, rm.clamp(max=127) * mb.sign(), 0.0)
    cv = torch.where((vs > 0) & (vb > 0), rv.clamp(1, 255), 0.0)
    ms, vs = ms * (1 / 16129.0), vs * (1 / 255.0 ** 4)
    s["m"].copy_(cm.view(-1))
    s["v"].copy_(cv.view(-1))
    s["ms"].copy_(ms.view(-1))
    s["vs"].copy_(vs.view(-1))
    return {"p": s["p"], "m": (cm * cm.abs() * ms).view(-1).bfloat16(), "v": ((cv * cv) * (cv * cv) * vs).view(-1).bfloat16()}


PLAIN = {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "quant": _plain_quant, "lin_fwd": _plain_lin_fwd,
         "lin_bwd": _plain_lin_bwd, "adamw": _plain_adamw}


# ------------------------------------------------------------------ work, and the results in 64 bits
def work(case):
    """Each input read once, each output written once; two operations per multiply-add."""
    kind = case["kind"]
    t = {"f32": 4, "bf16": 2, "f16": 2}.get(case.get("dtype"), 0)
    if kind == "norm_fwd":
        m, d = case["m"], case["d"]
        return {"bytes": m * d * (t * (4 if case["res"] else 2) + (1 if case["quant"] else 0)) + 8 * m + t * d, "flops": 8 * m * d}
    if kind == "norm_bwd":
        m, d = case["m"], case["d"]
        return {"bytes": m * d * t * (4 if case["dh"] else 3) + 4 * m + (t + 4) * d, "flops": 10 * m * d}
    if kind == "quant":
        m, d = case["m"], case["d"]
        return {"bytes": m * d * (2 * t + 1) + 4 * m, "flops": 4 * m * d}
    if kind == "lin_fwd":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * (k + 4) + m * n * t * (1 + case["res"] + case["keep"]) + (t * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    if kind == "lin_bwd":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": (m + n) * (k * (1 + t) + 4) + m * n * t * (1 if case["act"] == "none" else 2) + 4 * n,
                "flops": 4 * m * n * k}
    n, gb = sum(_sizes(case)), {"f32": 4, "bf16": 2}[case["grad"]]
    if case["bits"] == 8:   # codes read and written, scales of blocks; the states' values read for the caller
        return {"bytes": n * (8 + gb + 4 + 4) + 16 * n // BLOCK, "flops": 20 * n}
    return {"bytes": n * (8 + gb + 16), "flops": 15 * n}


def _draws64(seed, call, n):
    """The same SplitMix64 outputs, in the machine's unsigned words on the host."""
    import numpy as np
    u = np.uint64
    with np.errstate(over="ignore"):
        z = u(seed) + (u(call << 40) + np.arange(1, n + 1, dtype=u)) * u(0x9E3779B97F4A7C15)
        z ^= z >> u(30)
        z *= u(0xBF58476D1CE4E5B9)
        z ^= z >> u(27)
        z *= u(0x94D049BB133111EB)
        z ^= z >> u(31)
    return z


def _field(z, low, bits, shape):
    """Bits low .. low + bits - 1 of the draws, as fractions in 64 bits."""
    import numpy as np
    f = ((z >> np.uint64(low)) & np.uint64((1 << bits) - 1)).astype(np.float64) / 2.0 ** bits
    return torch.from_numpy(f).cuda().reshape(shape)


def _row_values(x, u=None):
    """(values that the codes of the rows of x stand for, codes, scales), all in 64 bits."""
    scale = torch.maximum(x.abs().max(dim=1).values, torch.tensor(TINY, dtype=x.dtype, device=x.device)) / 127
    steps = x / scale[:, None]
    codes = torch.clamp(torch.round(steps) if u is None else torch.floor(steps + u), -127, 127)
    return codes * scale[:, None], codes, scale


def exact(case, seed):
    """The first pass of run() from the definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and k not in ("h", "out") or k == "h" and kind == "norm_bwd"}
    if kind == "norm_fwd":
        h = f["x"] + f["res"] if case["res"] else f["x"]
        rms = torch.sqrt((h * h).sum(dim=1) / case["d"] + EPS)
        y, scale = h / rms[:, None] * f["gain"][None, :], None
        if case["quant"]:
            y, _, scale = _row_values(y)
        return {"h": h if case["res"] else None, "y": y, "scale": scale, "rstd": 1 / rms}
    if kind == "norm_bwd":
        # with the norm's reciprocal r: d(h_i r)/dh_j = r (i = j) - h_i h_j r^3 / D
        r = f["rstd"][:, None]
        t = f["dy"] * f["gain"][None, :]
        dx = t * r - f["h"] * r ** 3 * (t * f["h"]).sum(dim=1, keepdim=True) / case["d"]
        return {"dx": dx + f["dh"] if case["dh"] else dx, "dgain": torch.einsum("md,md->d", f["dy"], f["h"] * r)}
    if kind == "quant":
        u = _field(_draws64(seed, 7, case["m"] * case["d"]), 40, 24, s["x"].shape) if case["mode"] == "sr" else None
        y, _, scale = _row_values(f["x"], u)
        return {"y": y, "scale": scale}
    root2 = math.sqrt(2.0)
    if kind == "lin_fwd":
        z = (f["a"] * f["s_a"][:, None]) @ (f["b"] * f["s_b"][:, None]).t()
        if case["bias"]:
            z += f["bias"][None, :]
        out = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)),
               "gelu": lambda: z * torch.erfc(-z / root2) / 2, "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        return {"out": out + f["res"] if case["res"] else out, "z": z if case["keep"] else None}
    if kind == "lin_bwd":
        dz = f["dy"]
        if case["act"] != "none":
            z = f["z"]
            sg = torch.sigmoid(z)
            dz = dz * {"relu": lambda: (z > 0).double(), "silu": lambda: sg + z * sg * torch.sigmoid(-z),
                       "gelu": lambda: torch.erfc(-z / root2) / 2 + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[case["act"]]()
        rows = cols = None
        if case["mode"] == "sr":
            r = _draws64(seed, 7, dz.numel())
            rows, cols = _field(r, 40, 24, dz.shape), _field(r, 8, 24, dz.shape).t()
        by_row, _, _ = _row_values(dz * f["s_b"][None, :], rows)
        by_col, _, _ = _row_values((dz * f["s_a"][:, None]).t().contiguous(), cols)
        return {"da": by_row @ f["b"], "db": by_col @ f["a"], "dbias": dz.sum(dim=0)}
    t = s["step"] + 1
    m, v = f["m"], f["v"]
    if case["bits"] == 8:
        wide = lambda x: x.repeat_interleave(BLOCK)  # noqa: E731
        m, v = m.sign() * m ** 2 * wide(f["ms"]), v ** 4 * wide(f["vs"])
    g = f["g"] * f["gscale"]
    m, v = m + (1 - BETA1) * (g - m), v + (1 - BETA2) * (g ** 2 - v)
    p = f["p"] - LR * (DECAY * f["p"] + m / (1 - BETA1 ** t) / (torch.sqrt(v / (1 - BETA2 ** t)) + ADAM_EPS))
    if case["bits"] == 8:
        r = _draws64(seed, t, m.numel() // 2) if case["mode"] == "sr" else None

        def coded(x, top_code, power, low):
            top = wide(x.view(-1, BLOCK).abs().max(dim=1).values)
            top = torch.where(top < TINY, torch.zeros_like(top), top)
            steps = torch.where(top > 0, (x.abs() / top) ** (1 / power) * top_code, torch.zeros_like(x))
            if r is None:
                codes = torch.round(steps)
            else:
                u = torch.stack([_field(r, low, 16, -1), _field(r, 32 + low, 16, -1)], dim=1).view(-1)
                codes = torch.floor(steps + u)
            codes = torch.clamp(codes, max=top_code)
            if power == 4:
                codes = torch.where((x > 0) & (top > 0), torch.clamp(codes, min=1), torch.zeros_like(codes))
            else:
                codes = torch.where(top > 0, codes, torch.zeros_like(codes))
            return x.sign() * (codes / top_code) ** power * top
        m, v = coded(m, 127, 2, 0), coded(v, 255, 4, 16)
    return {"p": p, "m": m, "v": v}
