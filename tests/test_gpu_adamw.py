"""AdamW over many tensors, states in 32 and in 8 bits, against 64-bit forms."""
import pytest
import torch

import scaled_ref as R
from helpers import say
from paper_2009_13108_amd import niti

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
SIZES = [1, 0, 7, 255, 256, 257, 2047, 2048, 2049, 5000, 61470]
MANY = [(i * 37) % 700 for i in range(150)] + [100_000]


def make(sizes, p_dt, g_dt, seed=1):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda n, s: torch.randn(n, generator=g) * s  # noqa: E731
    p = [rnd(n, 0.1).to(p_dt).cuda() for n in sizes]
    gr = [rnd(n, 1e-2).to(g_dt).cuda() for n in sizes]
    m = [rnd(n, 3e-3) for n in sizes]
    v = [(rnd(n, 1e-2)) ** 2 + 1e-7 for n in sizes]
    return p, gr, m, v


def step64(p, g, m, v, step, gs):
    """New (p, m, v) and their bounds."""
    h = HYPER
    g = g.double().cpu() * gs
    p, m, v = p.double().cpu(), m.double().cpu(), v.double().cpu()
    m2 = h["beta1"] * m + (1 - h["beta1"]) * g
    v2 = h["beta2"] * v + (1 - h["beta2"]) * g * g
    # each term: the rate's rounding, the gradient's (squared) and the operations'
    mb = 4 * R.U32 * (m.abs() * h["beta1"] + (1 - h["beta1"]) * g.abs())
    vb = 6 * R.U32 * (v * h["beta2"] + (1 - h["beta2"]) * g * g)
    root = torch.sqrt(v2 / (1 - h["beta2"] ** step)) + h["eps"]
    up = h["lr"] / (1 - h["beta1"] ** step) * m2 / root
    p2 = p - h["lr"] * h["weight_decay"] * p - up
    pb = 3 * R.U32 * (p.abs() + up.abs()) + 12 * R.U32 * up.abs() + h["lr"] / (1 - h["beta1"] ** step) * mb / root
    return p2, pb, m2, mb, v2, vb


@pytest.mark.parametrize("p_dt", [F32, BF16, F16])
@pytest.mark.parametrize("g_dt", [F32, BF16, F16])
def test_states_of_32_bits(p_dt, g_dt):
    say("adamw 32", p_dt, g_dt)
    p, g, m, v = make(SIZES, p_dt, g_dt)
    m, v = [t.cuda() for t in m], [t.cuda() for t in v]
    plan = niti.adamw_plan(p, g, m, v)
    gs = torch.tensor(0.5, device="cuda")
    for step in (1, 2, 1000):
        old = [[t.clone() for t in x] for x in (p, m, v)]
        niti.adamw_step(plan, step, grad_scale=gs, **HYPER)
        for i in range(len(SIZES)):
            p2, pb, m2, mb, v2, vb = step64(old[0][i], g[i], old[1][i], old[2][i], step, 0.5)
            R.close(p[i], p2, pb, p_dt, "p %d" % i)
            R.close(m[i], m2, mb, what="m %d" % i)
            R.close(v[i], v2, vb, what="v %d" % i)


def test_many_tensors_and_unaligned_views():
    """More tensors than one launch's table, at odd addresses."""
    p, g, m, v = make(MANY, F32, BF16, seed=3)
    shift = lambda ts: [torch.cat([t.new_zeros(1), t]).cuda()[1:] for t in ts]  # noqa: E731
    p, g, m, v = shift(p), shift(g), shift(m), shift(v)
    old = [[t.clone() for t in x] for x in (p, m, v)]
    niti.adamw_step(niti.adamw_plan(p, g, m, v), 3, **HYPER)
    for i in range(len(MANY)):
        p2, pb, m2, mb, v2, vb = step64(old[0][i], g[i], old[1][i], old[2][i], 3, 1.0)
        R.close(p[i], p2, pb, what="p %d" % i)
        R.close(m[i], m2, mb, what="m %d" % i)
        R.close(v[i], v2, vb, what="v %d" % i)


def eight(sizes, m, v):
    """8-bit states and scales of given values (any codes will do to start from)."""
    B = niti.ADAMW_BLOCK
    cm, cv, sm, sv = [], [], [], []
    for n, a, b in zip(sizes, m, v):
        k = -(-n // B)
        pad = lambda t: torch.cat([t, t.new_zeros(k * B - n)]).view(k, B)  # noqa: E731
        a, b = pad(a), pad(b)
        s1, s2 = a.abs().amax(dim=1) / 127 ** 2 if k else a.new_zeros(0), b.amax(dim=1) / 255.0 ** 4 if k else b.new_zeros(0)
        cm.append(((a.abs() / s1[:, None].clamp(min=1e-30)).sqrt().round().clamp(max=127) * a.sign()).reshape(-1)[:n].to(torch.int8).cuda())
        cv.append((b / s2[:, None].clamp(min=1e-30)).sqrt().sqrt().round().clamp(0, 255).reshape(-1)[:n].to(torch.uint8).cuda())
        sm.append(s1.cuda())
        sv.append(s2.cuda())
    return cm, cv, sm, sv


def decoded(c, s, power):
    c, s = c.double().cpu(), s.double().cpu().repeat_interleave(niti.ADAMW_BLOCK)[: c.numel()]
    return c.sign() * c.abs() ** power * s


def check_states(x, bound, code, scale, power, top_code, u):
    """Codes and scales of a tensor's new state x (64 bits)."""
    B, n = niti.ADAMW_BLOCK, x.numel()
    k = -(-n // B)
    pad = torch.cat([x, x.new_zeros(k * B - n)]).view(k, B)
    top = pad.abs().amax(dim=1)
    slack = torch.cat([bound, bound.new_zeros(k * B - n)]).view(k, B).amax(dim=1)
    R.close(scale, torch.where(top < R.TINY, torch.zeros_like(top), top / float(top_code) ** power), (slack + 3 * R.U32 * top) / float(top_code) ** power,
            what="scale")
    wide = top.repeat_interleave(B)[:n]
    r = top_code * (x.abs() / wide.clamp(min=1e-300)) ** (1 / power)
    c = code.double().cpu().abs()
    # r's own error: 1/power of the value's and the maximum's, the roots' and the product's, relative to itself
    room = r * ((bound / x.abs().clamp(min=1e-300) + (slack / top.clamp(min=1e-300)).repeat_interleave(B)[:n]) / power + 8 * R.U32) + 1e-6
    arg = r if u is None else r + u
    low, high = (torch.round(arg - room), torch.round(arg + room)) if u is None else (torch.floor(arg - room), torch.floor(arg + room))
    low, high = low.clamp(max=top_code), high.clamp(max=top_code)
    if power == 4:
        low = torch.where(x > 0, low.clamp(min=1), low)
        high = torch.where(x > 0, high.clamp(min=1), high)
    assert ((c >= low) & (c <= high))[wide >= R.TINY].all()
    assert (c[wide < R.TINY] == 0).all()
    if power == 2:
        s = code.double().cpu().sign()
        assert ((s == x.sign()) | (s == 0) | (x.abs() <= bound)).all()


@pytest.mark.parametrize("mode", [niti.RTN, niti.SR])
@pytest.mark.parametrize("p_dt,g_dt", [(F32, BF16), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("sizes", [SIZES, MANY])
def test_states_of_8_bits(sizes, p_dt, g_dt, mode):
    say("adamw 8", p_dt, g_dt, mode, len(sizes))
    p, g, m, v = make(sizes, p_dt, g_dt, seed=5)
    cm, cv, sm, sv = eight(sizes, m, v)
    mr, vr = ([torch.full((n,), 9.0, device="cuda") for n in sizes] for _ in range(2))
    plan = niti.adamw_plan(p, g, cm, cv, sm, sv, mr, vr)
    for step in (1, 50):
        old = [[t.clone() for t in x] for x in (p, cm, cv, sm, sv)]
        niti.adamw_step(plan, step, mode=mode, seed=11, **HYPER)
        niti.adamw_read(plan)
        blocks = 0
        for i, n in enumerate(sizes):
            k = -(-n // niti.ADAMW_BLOCK)
            if n:
                m0, v0 = decoded(old[1][i], old[3][i], 2), decoded(old[2][i], old[4][i], 4)
                p2, pb, m2, mb, v2, vb = step64(old[0][i], g[i], m0, v0, step, 1.0)
                mb, vb = mb + 3 * R.U32 * m0.abs(), vb + 4 * R.U32 * v0
                R.close(p[i], p2, pb + 12 * R.U32 * (p2 - old[0][i].double().cpu()).abs(), p_dt, "p %d" % i)
                um = uv = None
                if mode == niti.SR:
                    z = R.draws(11, step, blocks * 128 + k * 128)[blocks * 128:]
                    um = torch.stack([R.field(z, 0, 16), R.field(z, 32, 16)], dim=1).reshape(-1)[:n]
                    uv = torch.stack([R.field(z, 16, 16), R.field(z, 48, 16)], dim=1).reshape(-1)[:n]
                check_states(m2, mb, cm[i], sm[i], 2, 127, um)
                check_states(v2, vb, cv[i], sv[i], 4, 255, uv)
                assert (cv[i] > 0).all()        # no v above 0 is rounded away
                # the values that the codes stand for: three products
                mw, vw = decoded(cm[i], sm[i], 2), decoded(cv[i], sv[i], 4)
                R.close(mr[i], mw, 3 * R.U32 * mw.abs(), what="m_read")
                R.close(vr[i], vw, 4 * R.U32 * vw, what="v_read")
            blocks += k


def test_blocks_that_are_empty_or_not_finite():
    n = 1024
    p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    g[300] = float("nan")
    g[600] = float("inf")
    g[800:1024] = 1e-3
    z = lambda t, k=n: torch.zeros(k, dtype=t, device="cuda")  # noqa: E731
    m, v, sm, sv = z(torch.int8), z(torch.uint8), z(F32, 4), z(F32, 4)
    plan = niti.adamw_plan([p], [g], [m], [v], [sm], [sv])
    niti.adamw_step(plan, 1, 1e-2, mode=niti.SR)
    assert (p[:256] == 1).all() and float(sm[0]) == 0 and float(sv[0]) == 0 and (m[:256] == 0).all() and (v[:256] == 0).all()
    assert torch.isnan(sm[1:3]).all() and torch.isnan(sv[1:3]).all() and (m[256:768] == 0).all() and (v[256:768] == 0).all()
    assert torch.isnan(p[300]) and torch.isfinite(sm[3]) and torch.isfinite(sv[3]) and torch.isfinite(p[768:]).all()
    assert (v[800:] > 0).all() and (v[768:800] == 0).all()
    g.fill_(1e-3)
    niti.adamw_step(plan, 2, 1e-2)
    assert torch.isnan(p[256:768]).all() and torch.isfinite(p[:256]).all() and torch.isfinite(p[768:]).all()
    # 32-bit states: only the element itself
    p, g = torch.ones(n, device="cuda"), torch.zeros(n, device="cuda")
    g[300] = float("nan")
    niti.adamw_step(niti.adamw_plan([p], [g], [z(F32)], [z(F32)]), 1, 1e-2)
    assert torch.isnan(p[300]) and int(torch.isnan(p).sum()) == 1


def test_eight_bits_follow_thirty_two():
    """A quadratic's descent with 8-bit states ends where the one with 32-bit states does."""
    g = torch.Generator().manual_seed(0)
    target, curve = torch.randn(3000, generator=g).cuda(), (0.1 + torch.rand(3000, generator=g)).cuda()
    ends = []
    for bits in (32, 8):
        p, gr = torch.zeros(3000, device="cuda"), torch.zeros(3000, device="cuda")
        if bits == 32:
            plan = niti.adamw_plan([p], [gr], [torch.zeros_like(p)], [torch.zeros_like(p)])
        else:
            z = lambda t, k=3000: torch.zeros(k, dtype=t, device="cuda")  # noqa: E731
            plan = niti.adamw_plan([p], [gr], [z(torch.int8)], [z(torch.uint8)], [z(F32, 12)], [z(F32, 12)])
        for t in range(1, 401):
            gr.copy_(curve * (p - target))
            niti.adamw_step(plan, t, 0.02, mode=niti.SR, seed=3)
        ends.append(float((0.5 * curve * (p - target) ** 2).mean()))
    start = float((0.5 * curve * target ** 2).mean())
    assert ends[0] < 1e-3 * start and ends[1] < 1e-2 * start


def test_refusals():
    p, h = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda", dtype=F16)
    with pytest.raises(ValueError):
        niti.adamw_plan([p], [p, p], [p], [p])
    with pytest.raises(ValueError):
        niti.adamw_plan([p], [p[:7]], [p], [p])
    with pytest.raises(TypeError):
        niti.adamw_plan([p], [p], [h], [p])
    with pytest.raises(TypeError):
        niti.adamw_plan([p, h], [p, p], [p, p], [p, p])
    with pytest.raises(ValueError):
        niti.adamw_plan([p], [p], [p], [p], m_read=[p])
    plan = niti.adamw_plan([p], [p], [p.clone()], [p.clone()])
    for bad in (dict(step=0), dict(step=1, beta1=1.0), dict(step=1, eps=-1.0), dict(step=1, mode=niti.PSR), dict(step=1, lr=float("nan"))):
        with pytest.raises(niti.NitiError):
            niti.adamw_step(plan, bad.pop("step"), bad.pop("lr", 1e-3), **bad)
    with pytest.raises(ValueError):
        niti.adamw_read(plan)
    niti.adamw_step(niti.adamw_plan([], [], [], []), 1, 1e-3)     # nothing to do
