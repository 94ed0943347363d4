"""The operators around an 8-bit feed-forward path, from tokens to a loss, as measurable cases.

Kinds of a case:
  emb_fwd   niti.embedding_fwd: rows of a table for given tokens, scaled; the table in a float type or as int8 rows
  emb_bwd   niti.embedding_bwd: the table's gradient, written whole or added to what is there
  gate_fwd  niti.gated_fwd: act(a Wg) * (a Wu) of int8 rows, both projections in one call
  gate_bwd  niti.gated_bwd: the gradients of its operands and its bias, by int8 products
  logprobs  niti.token_logprobs: log probabilities of given tokens, entropy and the top alternatives
  distill   niti.distill_fwd with the gradient in the same call: divergence from a teacher's top logits
  dist_bwd  niti.distill_bwd: the gradient alone, from what the forward call kept
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = 2.0 ** -100     # the least row maximum that a scale is formed from


def emb_fwd(m, v, d, table, dtype):
    return {"kind": "emb_fwd", "m": m, "v": v, "d": d, "table": table, "dtype": dtype}


def emb_bwd(m, v, d, dtype, grad, add):
    return {"kind": "emb_bwd", "m": m, "v": v, "d": d, "dtype": dtype, "grad": grad, "add": add}


def gate_fwd(m, f, k, dtype, act, bias, keep):
    return {"kind": "gate_fwd", "m": m, "f": f, "k": k, "dtype": dtype, "act": act, "bias": bias, "keep": keep}


def gate_bwd(m, f, k, dtype, act, mode):
    return {"kind": "gate_bwd", "m": m, "f": f, "k": k, "dtype": dtype, "act": act, "mode": mode}


def logprobs(m, v, dtype, top, scale):
    return {"kind": "logprobs", "m": m, "v": v, "dtype": dtype, "top": top, "scale": scale}


def distill(m, v, dtype, top, scale, kind="distill"):
    return {"kind": kind, "m": m, "v": v, "dtype": dtype, "top": top, "scale": scale}


def listed():
    return [
        # serving: the rows of eight sequences' last tokens, from int8 rows
        dict(emb_fwd(8, 32000, 4096, "i8", "bf16"), name="emb_8x4096_i8"),
        # training: 8192 tokens' gradients into a whole gradient of the table
        dict(emb_bwd(8192, 32000, 4096, "bf16", "bf16", False), name="emb_bwd_8192x4096"),
        # a table shared with the output layer: added to that one's gradient, ragged sizes, 32 bits
        dict(emb_bwd(4111, 50001, 1111, "f32", "f32", True), name="emb_bwd_4111x1111_add"),
        # serving, one token: the weights of both projections are the traffic
        dict(gate_fwd(1, 9216, 4096, "bf16", "silu", False, False), name="gate_1x9216x4096"),
        # a prompt or a training batch of 4096 tokens, as a training step needs it
        dict(gate_fwd(4096, 8192, 4096, "bf16", "silu", False, True), name="gate_4096x8192x4096"),
        # a ragged prompt: no size is a multiple of 16
        dict(gate_fwd(1000, 1500, 1111, "f32", "gelu", True, False), name="gate_1000x1500x1111_f32"),
        # the backward pass of a hidden layer on 2048 tokens
        dict(gate_bwd(2048, 4096, 4096, "bf16", "silu", "rtn"), name="gate_bwd_2048x4096x4096"),
        # serving, one token: its log probability and twenty alternatives
        dict(logprobs(1, 32000, "bf16", 20, 1.0), name="logprobs_1x32000"),
        # scoring a batch of 4096 tokens
        dict(logprobs(4096, 32000, "bf16", 5, 1.0), name="logprobs_4096x32000"),
        # an odd vocabulary, in 32 bits, at a temperature
        dict(logprobs(77, 128001, "f32", 20, 1 / 0.7), name="logprobs_77x128001_f32"),
        # training a small network by a large one's 64 top logits, loss and gradient
        dict(distill(4096, 32000, "bf16", 64, 0.5), name="distill_4096x32000"),
        # the gradient alone, a ragged batch in 32 bits
        dict(distill(333, 50001, "f32", 20, 1.0, "dist_bwd"), name="dist_bwd_333x50001_f32"),
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of lo..hi."""
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi):
    """A size as layers have them: mostly whole 64s or 16s, else any."""
    v, unit = _log(rng, lo, hi), rng.choice([64, 64, 16, 1])
    return max(unit, v // unit * unit)


def draw(rng):
    kind = rng.choice(["emb_fwd", "emb_bwd", "gate_fwd", "gate_fwd", "gate_bwd", "logprobs", "logprobs", "distill", "dist_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    half = "bf16" if dtype == "f32" else dtype
    if kind == "emb_fwd":
        while True:
            m, v, d = _log(rng, 1, 16384), _size(rng, 256, 131072), _size(rng, 64, 8192)
            if m * d <= 8192 * 4096 and v * d <= 32000 * 4096:
                return emb_fwd(m, v, d, rng.choice(["i8", dtype, dtype]), dtype)
    if kind == "emb_bwd":
        while True:
            m, v, d = _log(rng, 1, 16384), _size(rng, 256, 131072), _size(rng, 64, 8192)
            if m * d <= 8192 * 4096 and v * d <= 32000 * 2048:
                return emb_bwd(m, v, d, dtype, rng.choice(["f32", dtype]), rng.random() < 0.5)
    if kind in ("gate_fwd", "gate_bwd"):
        while True:
            m, f, k = _log(rng, 1, 8192), _size(rng, 32, 9216), _size(rng, 32, 9216)
            if m * f * k <= (4096 * 8192 * 4096 if kind == "gate_fwd" else 2048 * 4096 * 4096):
                break
        act = rng.choice(["relu", "gelu", "silu", "silu"])
        if kind == "gate_fwd":
            return gate_fwd(m, f, k, dtype, act, rng.random() < 0.4, rng.random() < 0.4)
        return gate_bwd(m, f, k, half, act, rng.choice(["rtn", "sr"]))
    while True:
        m, v = _log(rng, 1, 8192), _size(rng, 300, 200000)
        if m * v <= 4096 * 32000 // (2 if dtype == "f32" else 1):
            break
    scale = rng.choice([1.0, 1.0, 0.5, 1 / 0.7])
    if kind == "logprobs":
        return logprobs(m, v, dtype, rng.choice([0, 1, 5, 20, 64]), scale)
    return distill(m, v, dtype, _log(rng, 1, 256), scale, kind)


# ------------------------------------------------------------------ inputs
def _quantised(x):
    """A float matrix as int8 rows and their scales."""
    top = x.abs().amax(dim=1, keepdim=True).clamp(min=TINY)
    return (x * (127.0 / top)).round().clamp(-127, 127).to(torch.int8), (top / 127.0).squeeze(1)


def prepare(case, seed):
    """Inputs, and the buffers and workspaces that a program keeps.  A workspace
    is the package's own: only where it is used is it made.  All else is the
    same on both sides."""
    if own:
        from paper_2009_13108_amd import niti
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def stream(m, d):
        """Activations of a residual stream: normal, a few channels far larger."""
        return randn(m, d) * (1 + 9 * (rand(d) < 0.005))

    def errors(m, d):
        """Errors: small, of another size in each row."""
        return randn(m, d) * 1e-3 * torch.exp(randn(m, 1))

    def words(m, v):
        """Tokens as texts have them: the r-th most frequent with a share of 1/r; frequent ones lie anywhere."""
        rank = (torch.exp(rand(m) * math.log(v + 1.0)) - 1).long().clamp(0, v - 1)
        return torch.randperm(v, generator=g, device="cuda")[rank].to(torch.int32)

    def logits(m, v):
        """Logits of a trained network: a wide body and a few tokens far above it."""
        x = 2 * randn(m, v)
        x.scatter_add_(1, (rand(m, 8) * v).long().clamp(max=v - 1), 6 + 3 * randn(m, 8))
        return x

    s = {"case": case}
    kind = case["kind"]
    t = TYPES[case["dtype"]]
    m = case["m"]
    if kind == "emb_fwd":
        v, d = case["v"], case["d"]
        s.update(tokens=words(m, v), out=empty(m, d, dtype=t), table_scale=None, alpha=math.sqrt(d))
        if case["table"] == "i8":
            s["table"], s["table_scale"] = _quantised(0.02 * randn(v, d))
        else:
            s["table"] = (0.02 * randn(v, d)).to(TYPES[case["table"]])
    elif kind == "emb_bwd":
        v, d = case["v"], case["d"]
        s.update(tokens=words(m, v), dy=errors(m, d).to(t), alpha=math.sqrt(d))
        s["dtable"] = errors(v, d).to(TYPES[case["grad"]]) if case["add"] else empty(v, d, dtype=TYPES[case["grad"]])
        if own:
            s["ws"] = niti.new_workspace(niti.workspace_bytes(niti.OP_EMBEDDING_BWD, None, m, v, d))
    elif kind in ("gate_fwd", "gate_bwd"):
        f, k = case["f"], case["k"]
        a, s_a = _quantised(stream(m, k))
        b, s_b = _quantised(randn(2 * f, k) / math.sqrt(k))
        s.update(a=a, s_a=s_a, b=b, s_b=s_b)
        if kind == "gate_fwd":
            s.update(bias=(0.1 * randn(2 * f)).to(t) if case["bias"] else None, out=empty(m, f, dtype=t),
                     z=empty(m, 2 * f, dtype=t) if case["keep"] else None)
        else:
            s.update(dy=errors(m, f).to(t), z=(1.5 * randn(m, 2 * f)).to(t), da=empty(m, k, dtype=t),
                     db=empty(2 * f, k, dtype=t), dbias=empty(2 * f), seed=int(seed))
        if own:
            op = niti.OP_GATED_FWD if kind == "gate_fwd" else niti.OP_GATED_BWD
            s["ws"] = niti.new_workspace(niti.workspace_bytes(op, None, m, f, k))
    elif kind == "logprobs":
        v, top = case["v"], case["top"]
        s.update(x=logits(m, v).to(t), tokens=words(m, v), logp=empty(m), lse=empty(m), entropy=empty(m),
                 top_logp=empty(m, top) if top else None, top_idx=empty(m, top, dtype=torch.int32) if top else None)
        if own:
            s["ws"] = niti.new_workspace(niti.workspace_bytes(niti.OP_TOKEN_LOGPROBS, None, m, v, top))
    else:
        v, top = case["v"], case["top"]
        x = logits(m, v)
        val, idx = torch.topk(x + randn(m, v), top, dim=1)
        s.update(x=x.to(t), t_val=val.to(t), t_idx=idx.to(torch.int32), dloss=rand(m) / m, dx=empty(m, v, dtype=t))
        if kind == "distill":
            s.update(loss=empty(m), lse=empty(m))
            if own:
                s["ws"] = niti.new_workspace(niti.workspace_bytes(niti.OP_DISTILL_FWD, None, m, v, top))
        else:
            s["lse"] = torch.logsumexp(s["x"].double() * case["scale"], dim=1).float()
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        return PLAIN[kind](s)
    from paper_2009_13108_amd import niti
    if kind == "emb_fwd":
        niti.embedding_fwd(s["table"], s["tokens"], s["out"], table_scale=s["table_scale"], alpha=s["alpha"])
        return s["out"]
    if kind == "emb_bwd":
        niti.embedding_bwd(s["dy"], s["tokens"], s["dtable"], s["ws"], alpha=s["alpha"], accumulate=case["add"])
        return s["dtable"]
    if kind == "logprobs":
        niti.token_logprobs(s["x"], tokens=s["tokens"], logp=s["logp"], lse=s["lse"], entropy=s["entropy"],
                            top_logp=s["top_logp"], top_idx=s["top_idx"], scale=case["scale"], ws=s["ws"])
        return {k: s[k] for k in ("logp", "lse", "entropy", "top_logp", "top_idx")}
    if kind == "distill":
        niti.distill_fwd(s["x"], s["t_val"], s["t_idx"], s["loss"], lse=s["lse"], dlogits=s["dx"], dloss=s["dloss"],
                         scale=case["scale"], ws=s["ws"])
        return {"loss": s["loss"], "lse": s["lse"], "dx": s["dx"]}
    if kind == "dist_bwd":
        niti.distill_bwd(s["x"], s["t_val"], s["t_idx"], s["lse"], s["dloss"], s["dx"], scale=case["scale"])
        return {"dx": s["dx"]}
    act = getattr(niti, "ACT_" + case["act"].upper())
    if kind == "gate_fwd":
        niti.gated_fwd(s["a"], s["b"], s["out"], s["s_a"], s["s_b"], act=act, bias=s["bias"], z=s["z"], ws=s["ws"])
        return {"out": s["out"], "z": s["z"]}
    niti.gated_bwd(s["dy"], s["z"], s["a"], s["b"], s["s_a"], s["s_b"], s["ws"], act=act, da=s["da"], db=s["db"],
                   dbias=s["dbias"], mode=niti.SR if case["mode"] == "sr" else niti.RTN, seed=s["seed"], call=7)
    return {"da": s["da"], "db": s["db"], "dbias": s["dbias"]}


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
    return z / (1 + torch.exp(-z))


def _slope(name, z):
    if name == "relu":
        return (z > 0).float()
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    sg = 1 / (1 + torch.exp(-z))
    return sg * (1 + z * (1 - sg))


def _plain_emb_fwd(s):
    rows = s["table"][s["tokens"].long()].float()
    if s["table_scale"] is not None:
        rows = rows * s["table_scale"][s["tokens"].long()][:, None]
    s["out"].copy_(rows * s["alpha"])
    return s["out"]


def _plain_emb_bwd(s):
    sums = torch.zeros(s["dtable"].shape, device="cuda").index_add_(0, s["tokens"], s["dy"].float()) * s["alpha"]
    s["dtable"].copy_(sums + s["dtable"].float() if s["case"]["add"] else sums)
    return s["dtable"]


def _plain_gate_fwd(s):
    t, f = s["out"].dtype, s["case"]["f"]
    z = (s["a"].float() @ s["b"].float().t()) * (s["s_a"][:, None] * s["s_b"])
    if s["bias"] is not None:
        z = z + s["bias"].float()
    out = _activation(s["case"]["act"], z[:, :f]) * z[:, f:]
    return {"out": out.to(t), "z": z.to(t) if s["case"]["keep"] else None}


def _plain_gate_bwd(s):
    t, f, act = s["dy"].dtype, s["case"]["f"], s["case"]["act"]
    dy, zg, zu = s["dy"].float(), s["z"][:, :f].float(), s["z"][:, f:].float()
    dz = torch.cat([dy * zu * _slope(act, zg), dy * _activation(act, zg)], dim=1)
    u = v = None
    if s["case"]["mode"] == "sr":
        r = _draws(s["seed"], 7, dz.numel()).view(dz.shape)
        u, v = _shift(r, 40).float() * 2.0 ** -24, (_shift(r, 8) & 0xFFFFFF).float() * 2.0 ** -24
    c, sc = _codes(dz * s["s_b"], 1, u)
    da = (c @ s["b"].float()) * sc
    c, sc = _codes(dz * s["s_a"][:, None], 0, v)
    db = (c.t() @ s["a"].float()) * sc.t()
    return {"da": da.to(t), "db": db.to(t), "dbias": dz.sum(dim=0)}


def _softmax(x):
    """Shifted logits, their exponentials, and the sums of those."""
    x = x - x.amax(dim=1, keepdim=True)
    e = torch.exp(x)
    return x, e, e.sum(dim=1)


def _plain_logprobs(s):
    case = s["case"]
    raw = s["x"].float()
    x = raw * case["scale"]
    t, e, total = _softmax(x)
    log = torch.log(total)
    out = {"logp": t.gather(1, s["tokens"].long()[:, None]).squeeze(1) - log, "lse": x.amax(dim=1) + log,
           "entropy": log - (e * t).sum(dim=1) / total, "top_logp": None, "top_idx": None}
    if case["top"]:
        # one integer for each logit: its order above, its column below, lower columns first
        bits = (raw + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -2147483648 - bits, bits) * (1 << 32) + (case["v"] - 1 - torch.arange(case["v"], device="cuda"))
        idx = torch.topk(key, case["top"], dim=1).indices
        out["top_logp"], out["top_idx"] = t.gather(1, idx) - log[:, None], idx.to(torch.int32)
    return out


def _teacher(s):
    """Probabilities of the listed tokens, and their logarithms."""
    t, e, total = _softmax(s["t_val"].float() * s["case"]["scale"])
    return e / total[:, None], t - torch.log(total)[:, None]


def _plain_distill(s):
    case, idx = s["case"], s["t_idx"].long()
    x = s["x"].float() * case["scale"]
    t, e, total = _softmax(x)
    log = torch.log(total)
    p, logp = _teacher(s)
    loss = (p * (logp - (t.gather(1, idx) - log[:, None]))).sum(dim=1)
    dx = ((e / total[:, None]).scatter_add_(1, idx, -p)) * (s["dloss"] * case["scale"])[:, None]
    return {"loss": loss, "lse": x.amax(dim=1) + log, "dx": dx.to(s["x"].dtype)}


def _plain_dist_bwd(s):
    case = s["case"]
    q = torch.exp(s["x"].float() * case["scale"] - s["lse"][:, None])
    dx = q.scatter_add_(1, s["t_idx"].long(), -_teacher(s)[0]) * (s["dloss"] * case["scale"])[:, None]
    return {"dx": dx.to(s["x"].dtype)}


PLAIN = {"emb_fwd": _plain_emb_fwd, "emb_bwd": _plain_emb_bwd, "gate_fwd": _plain_gate_fwd, "gate_bwd": _plain_gate_bwd,
         "logprobs": _plain_logprobs, "distill": _plain_distill, "dist_bwd": _plain_dist_bwd}


# ------------------------------------------------------------------ work, and the results in 64 bits
def work(case):
    """Each input read once, each output written once; two operations per multiply-add."""
    kind, m = case["kind"], case["m"]
    size = {"f32": 4, "bf16": 2, "f16": 2, "i8": 1}
    t = size[case["dtype"]]
    if kind in ("emb_fwd", "emb_bwd"):
        v, d = case["v"], case["d"]
        # distinct tokens of m with shares 1 / rank, in the mean
        norm = math.log(v + 1.0)
        rows = sum(1 - math.exp(m * math.log1p(-min(0.999999, math.log1p(1.0 / r) / norm))) for r in range(1, v + 1))
        if kind == "emb_fwd":
            return {"bytes": int(rows * d * size[case["table"]]) + m * (d * t + 4) + (int(rows) * 4 if case["table"] == "i8" else 0),
                    "flops": m * d}
        g = size[case["grad"]]
        return {"bytes": m * (d * t + 4) + (int(2 * rows * d * g) if case["add"] else v * d * g), "flops": 2 * m * d}
    if kind in ("gate_fwd", "gate_bwd"):
        f, k = case["f"], case["k"]
        if kind == "gate_fwd":
            return {"bytes": (m + 2 * f) * (k + 4) + m * f * t * (3 if case["keep"] else 1) + (2 * f * t if case["bias"] else 0),
                    "flops": 4 * m * f * k}
        return {"bytes": (m + 2 * f) * (k * (1 + t) + 4) + 3 * m * f * t + 8 * f, "flops": 8 * m * f * k}
    v, top = case["v"], case["top"]
    if kind == "logprobs":
        return {"bytes": m * (v * t + 16 + 8 * top), "flops": 6 * m * v}
    return {"bytes": m * (2 * v * t + top * (t + 4) + (12 if kind == "distill" else 8)), "flops": (8 if kind == "distill" else 4) * m * v}


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
    """The values that the codes of the rows of x stand for, in 64 bits."""
    scale = torch.maximum(x.abs().max(dim=1).values, torch.tensor(TINY, dtype=x.dtype, device=x.device)) / 127
    steps = x / scale[:, None]
    return torch.clamp(torch.round(steps) if u is None else torch.floor(steps + u), -127, 127) * scale[:, None]


def exact(case, seed):
    """The first pass of run() from the definitions in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "emb_fwd":
        one_hot_rows = torch.index_select(s["table"], 0, s["tokens"])
        out = one_hot_rows.double() * s["alpha"]
        return out if s["table_scale"] is None else out * torch.index_select(s["table_scale"], 0, s["tokens"]).double()[:, None]
    if kind == "emb_bwd":
        order = torch.argsort(s["tokens"], stable=True)
        tok, count = torch.unique_consecutive(s["tokens"][order], return_counts=True)
        ends = torch.cumsum(count, 0)
        run_sums = torch.cumsum(torch.cat([torch.zeros(1, case["d"], dtype=torch.float64, device="cuda"),
                                           s["dy"].double()[order]]), 0)
        out = s["dtable"].double() if case["add"] else torch.zeros(s["dtable"].shape, dtype=torch.float64, device="cuda")
        out[tok.long()] += (run_sums[ends] - run_sums[ends - count]) * s["alpha"]
        return out
    if kind in ("gate_fwd", "gate_bwd"):
        f, root2 = case["f"], math.sqrt(2.0)

        def act(z):
            return {"relu": lambda: torch.where(z > 0, z, torch.zeros_like(z)), "gelu": lambda: z * torch.erfc(-z / root2) / 2,
                    "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        a, b = s["a"].double(), s["b"].double()
        if kind == "gate_fwd":
            z = (a * s["s_a"].double()[:, None]) @ (b * s["s_b"].double()[:, None]).t()
            if case["bias"]:
                z += s["bias"].double()[None, :]
            return {"out": act(z[:, :f]) * z[:, f:], "z": z if case["keep"] else None}
        gate, up, dy = s["z"][:, :f].double(), s["z"][:, f:].double(), s["dy"].double()
        sg = torch.sigmoid(gate)
        slope = {"relu": lambda: (gate > 0).double(), "silu": lambda: sg + gate * sg * torch.sigmoid(-gate),
                 "gelu": lambda: torch.erfc(-gate / root2) / 2 + gate * torch.exp(-gate * gate / 2) / math.sqrt(2 * math.pi)}[case["act"]]()
        dz = torch.cat([dy * slope * up, dy * act(gate)], dim=1)
        rows = cols = None
        if case["mode"] == "sr":
            r = _draws64(seed, 7, dz.numel())
            rows, cols = _field(r, 40, 24, dz.shape), _field(r, 8, 24, dz.shape).t()
        da = _row_values(dz * s["s_b"].double()[None, :], rows) @ b
        db = _row_values((dz * s["s_a"].double()[:, None]).t().contiguous(), cols) @ a
        return {"da": da, "db": db, "dbias": dz.sum(dim=0)}
    x = s["x"].double() * case["scale"]
    lse = torch.logsumexp(x, dim=1) if kind != "dist_bwd" else s["lse"].double()
    if kind == "logprobs":
        logq = x - lse[:, None]
        out = {"logp": logq[torch.arange(case["m"], device="cuda"), s["tokens"].long()], "lse": lse,
               "entropy": -(torch.exp(logq) * logq).sum(dim=1), "top_logp": None, "top_idx": None}
        if case["top"]:
            out["top_idx"] = torch.stack([torch.argsort(row.float(), descending=True, stable=True)[:case["top"]]
                                          for row in s["x"]]).to(torch.int32)
            out["top_logp"] = torch.gather(logq, 1, out["top_idx"].long())
        return out
    lt = torch.log_softmax(s["t_val"].double() * case["scale"], dim=1)
    at = torch.arange(case["m"], device="cuda")[:, None]
    q = torch.exp(x - lse[:, None])
    listed_q = x[at, s["t_idx"].long()] - lse[:, None]
    q[at, s["t_idx"].long()] -= torch.exp(lt)          # (a list's indices are distinct)
    dx = q * (s["dloss"].double() * case["scale"])[:, None]
    if kind == "dist_bwd":
        return {"dx": dx}
    return {"loss": (torch.exp(lt) * (lt - listed_q)).sum(dim=1), "lse": lse, "dx": dx}
