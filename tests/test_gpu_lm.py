"""Lookup, gated product, log probabilities and distillation together, as a
model uses them: gradients against 64 bits, another stream, a captured graph, recorded calls."""
import pytest
import torch

import scaled_ref as R
from paper_2009_13108_amd import lm, niti

pytestmark = pytest.mark.gpu
V, D, F, M, TOP = 300, 96, 104, 130, 12


def inputs(seed=4):
    g = torch.Generator().manual_seed(seed)
    tok = torch.randint(0, V, (M,), generator=g).to(torch.int32)
    tok[::7] = 5                                   # one token again and again
    tok[3], tok[4] = -1, V                         # padding
    val, idx = torch.topk(2 * torch.randn(M, V, generator=g), TOP, dim=1)
    idx[10, 4:] = -1
    return tok.cuda(), val.cuda(), idx.to(torch.int32).cuda()


def model(dtype=torch.bfloat16, **kw):
    return lm.TokenModel(V, D, F, M, dtype, TOP, **kw)


def outputs(net):
    return [net.loss, net.logits, net.dx] + list(net.dw.values()) + list(net.dvec.values())


def one_step(net, tok, val, idx):
    net.forward(tok)
    net.teach(tok, val, idx)
    got = [t.clone() for t in outputs(net)]
    net.step()
    return got + [w.clone() for w in net.w.values()] + [net.score(tok, tok).clone(), net.entropy.clone(), net.top_idx.clone()]


def test_gradients():
    """The model in 64 bits on the values that the codes stand for, which pass gradients straight through.  A product's error codes
    are off by half a step: at most (largest / rms) / 254 of a row, below 0.04 for rows of up to 300 whose largest is within ten
    rms.  Three such products lie behind a gradient at most, and their errors add up to less than 0.12 of it."""
    tok, val, idx = inputs()
    net = model(torch.float32, mode=niti.RTN, state_bits=32)
    net.forward(tok)
    value = {k: (q.double() * s.double()[:, None]).cpu() for k, (q, s) in list(net.wq.items()) + list(net.rows.items())}
    net.teach(tok, val, idx)
    w = {k: value[k].clone().requires_grad_() for k in net.w}
    vec = {k: t.double().cpu().requires_grad_() for k, t in net.vec.items()}
    through = lambda x, v: x + (v - x).detach()  # noqa: E731
    at = tok.long().cpu()
    inside = ((at >= 0) & (at < V)).double()[:, None]
    x = w["table"][at.clamp(0, V - 1)] * inside * net.alpha
    norm = lambda t, g: t / torch.sqrt((t * t).mean(dim=1, keepdim=True) + 1e-6) * g  # noqa: E731
    z = through(norm(x, vec["gain"]), value["n"]) @ w["gated"].t()
    u = through(z[:, :F] * torch.sigmoid(z[:, :F]) * z[:, F:], value["u"])
    logits = through(norm(u @ w["down"].t() + x, vec["last"]), value["last"]) @ w["table"].t()
    listed = idx.long().cpu()
    t = torch.where(listed >= 0, val.double().cpu(), torch.full((), float("-inf"), dtype=torch.float64))
    p, logq = torch.softmax(t, dim=1), torch.log_softmax(logits, dim=1).gather(1, listed.clamp(min=0))
    loss = (p * (torch.log_softmax(t, dim=1).nan_to_num(neginf=0) - logq)).sum(dim=1)
    assert (net.loss.double().cpu() - loss).abs().max() < 1e-4
    loss.mean().backward()
    for name, want in [(k, w[k].grad) for k in w] + [(k, vec[k].grad) for k in vec]:
        got = (net.dw if name in net.dw else net.dvec)[name].double().cpu()
        assert float((got - want).norm() / want.norm()) < 0.12, name


def test_scores_agree_with_the_loss():
    """The divergence from a list of one token is its negative log probability."""
    tok, _, _ = inputs()
    net = model(torch.float32)
    want = torch.arange(M, dtype=torch.int32, device="cuda") % V
    logp = net.score(tok, want).clone()
    niti.distill_fwd(net.logits, torch.zeros(M, 1, device="cuda"), want.view(M, 1), net.loss)
    room = 64 * R.U32 * (1 + logp.abs().max())      # both are differences of numbers of that size, of a few roundings each
    assert (net.loss + logp).abs().max() <= room
    order = torch.sort(net.logits.cpu(), dim=1, descending=True, stable=True).indices[:, :TOP]
    assert torch.equal(net.top_idx.long().cpu(), order)


def test_another_stream_gives_the_same():
    data = inputs()
    want = one_step(model(), *data)
    net = model()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = one_step(net, *data)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graph_replays_match_plain_calls():
    """A forward pass, its loss and gradients and a scoring, captured once; inputs and weights change between the replays."""
    tok, val, idx = inputs()
    net = model()

    def work():
        net.forward(tok)
        net.teach(tok, val, idx)
        net.score(tok, tok)
    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for i in range(4):
        for a, b in zip((tok, val, idx), inputs(10 + i)):
            a.copy_(b)
        work()
        want = [t.clone() for t in outputs(net) + [net.logp, net.entropy, net.top_logp, net.top_idx]]
        for t in outputs(net):
            t.zero_()
        net.ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        got = outputs(net) + [net.logp, net.entropy, net.top_logp, net.top_idx]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        net.w["gated"].mul_(0.9)
        net.lay_out()


def test_recorded_calls_replay():
    tok, val, idx = inputs()
    net = model()
    with niti.recording() as calls:
        net.forward(tok)
        net.teach(tok, val, idx)
    want = [t.clone() for t in outputs(net)]
    for t in outputs(net):
        t.zero_()
    niti.replay(calls)
    assert all(torch.equal(a, b) for a, b in zip(outputs(net), want))


@pytest.mark.parametrize("dtype,bits", [(torch.bfloat16, 8), (torch.float32, 32), (torch.float16, 8)])
def test_training_runs(dtype, bits):
    losses, net = lm.train(steps=5, v=200, d=64, f=96, tokens=64, dtype=dtype, state_bits=bits)
    assert all(x == x and 0 <= x < 100 for x in losses)
    assert all(torch.isfinite(w).all() for w in net.w.values())
