"""A residual feed-forward block on int8 rows, trained by the library's calls.

    h = x + res,  n = norm(h),  u = act(n Wu^T + bu),  out = u Wd^T + bd + h

n, u and both weight matrices are int8 rows with a scale each wherever they
are multiplied, forwards and backwards; the weights' 32-bit masters are what
AdamW updates (states in 8 or 32 bits), and they are laid out as int8 rows
again after each step.  All memory is taken once: a pass allocates nothing
and never waits for the device.

    python -m paper_2009_13108_amd.ffn    trains one on a synthetic target
"""
from __future__ import annotations

from . import niti


class FeedForward:
    """A block of width d and hidden width f for `tokens` rows of type dtype."""

    def __init__(self, d, f, tokens, dtype, act=niti.ACT_SILU, state_bits=8, mode=niti.SR, seed=1, device="cuda"):
        import torch
        self.d, self.f, self.tokens, self.act, self.mode, self.seed, self.steps = d, f, tokens, act, mode, seed, 0
        # the optimiser counts its draws by steps, the gradients by calls: under one seed they would meet
        self.state_seed = seed ^ 1 << 63
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        new = lambda *shape, t=dtype: torch.zeros(shape, dtype=t, device=device)  # noqa: E731
        f32, i8 = torch.float32, torch.int8
        # masters: matrices, and vectors (whose gradients are 32-bit whatever dtype is)
        self.w = {"up": torch.randn(f, d, generator=g, device=device) / d ** 0.5,
                  "down": torch.randn(d, f, generator=g, device=device) / f ** 0.5}
        self.vec = {"gain": torch.ones(d, device=device), "bu": new(f, t=f32), "bd": new(d, t=f32)}
        self.dw = {k: new(*v.shape) for k, v in self.w.items()}
        self.dvec = {k: torch.zeros_like(v) for k, v in self.vec.items()}
        self.wq = {k: (new(*v.shape, t=i8), new(v.shape[0], t=f32)) for k, v in self.w.items()}
        # a forward pass and its gradients
        self.h, self.rstd = new(tokens, d), new(tokens, t=f32)
        self.nq, self.ns = new(tokens, d, t=i8), new(tokens, t=f32)
        self.z, self.u = new(tokens, f), new(tokens, f)
        self.uq, self.us = new(tokens, f, t=i8), new(tokens, t=f32)
        self.out, self.du, self.dn, self.dx = new(tokens, d), new(tokens, f), new(tokens, d), new(tokens, d)
        ws = max(niti.workspace_bytes(niti.OP_LINEAR_FWD, None, tokens, f, d),
                 niti.workspace_bytes(niti.OP_LINEAR_FWD, None, tokens, d, f),
                 niti.workspace_bytes(niti.OP_LINEAR_BWD, None, tokens, f, d),
                 niti.workspace_bytes(niti.OP_LINEAR_BWD, None, tokens, d, f),
                 niti.workspace_bytes(niti.OP_RMSNORM_BWD, None, tokens, d))
        self.ws = niti.new_workspace(ws, device)
        self.plans = [self._plan(list(self.w.values()), list(self.dw.values()), state_bits, device),
                      self._plan(list(self.vec.values()), list(self.dvec.values()), 32, device)]
        self.lay_out()

    @staticmethod
    def _plan(params, grads, bits, device):
        import torch
        like = lambda t: [torch.zeros(p.numel(), dtype=t, device=device) for p in params]  # noqa: E731
        if bits == 32:
            return niti.adamw_plan(params, grads, like(torch.float32), like(torch.float32))
        scales = lambda: [torch.zeros(-(-p.numel() // niti.ADAMW_BLOCK), device=device) for p in params]  # noqa: E731
        return niti.adamw_plan(params, grads, like(torch.int8), like(torch.uint8), scales(), scales())

    def lay_out(self):
        """The weights as int8 rows, one scale for each output channel."""
        for k, w in self.w.items():
            niti.quantize_rows(w, *self.wq[k])

    def forward(self, x, res=None):
        """out [tokens][d]; x (and res) stay the caller's."""
        niti.rmsnorm_fwd(x, self.vec["gain"], res=res, h=self.h, q=self.nq, scale=self.ns, rstd=self.rstd)
        (wu, su), (wd, sd) = self.wq["up"], self.wq["down"]
        niti.linear_fwd(self.nq, wu, self.u, self.ns, su, bias=self.vec["bu"], act=self.act, z=self.z, ws=self.ws)
        niti.quantize_rows(self.u, self.uq, self.us)
        niti.linear_fwd(self.uq, wd, self.out, self.us, sd, bias=self.vec["bd"], res=self.h, ws=self.ws)
        return self.out

    def backward(self, dout):
        """Gradients of the last forward pass; returns that of x (and of res).  Their
        stochastic draws go by the number of steps taken: repeated before the next, it
        gives the same again."""
        (wu, su), (wd, sd) = self.wq["up"], self.wq["down"]
        kw = dict(mode=self.mode, seed=self.seed)
        niti.linear_bwd(dout, self.uq, wd, self.us, sd, self.ws, da=self.du, db=self.dw["down"], dbias=self.dvec["bd"],
                        call=2 * self.steps, **kw)
        niti.linear_bwd(self.du, self.nq, wu, self.ns, su, self.ws, z=self.z, act=self.act, da=self.dn, db=self.dw["up"],
                        dbias=self.dvec["bu"], call=2 * self.steps + 1, **kw)
        niti.rmsnorm_bwd(self.dn, self.h, self.vec["gain"], self.rstd, self.dx, self.dvec["gain"], self.ws, dh=dout)
        return self.dx

    def step(self, lr=1e-3, weight_decay=0.01, grad_scale=None):
        """AdamW on all weights, and their int8 rows again."""
        self.steps += 1
        for plan in self.plans:
            niti.adamw_step(plan, self.steps, lr, weight_decay=weight_decay, grad_scale=grad_scale, mode=self.mode,
                            seed=self.state_seed)
        self.lay_out()


def train(steps=200, d=256, f=1024, tokens=512, dtype=None, state_bits=8, seed=1, lr=2e-3, say=None):
    """Fits the block to a fixed random map of fixed tokens; returns the mean squared errors by step."""
    import torch
    dtype = dtype or torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    x = torch.randn(tokens, d, generator=g, device="cuda").to(dtype)
    target = x.float() + torch.tanh(x.float() @ torch.randn(d, d, generator=g, device="cuda") / d ** 0.5)
    net = FeedForward(d, f, tokens, dtype, state_bits=state_bits, seed=seed)
    losses = []
    for i in range(steps):
        diff = net.forward(x).float() - target
        losses.append(diff.square().mean())
        net.backward((diff * (2.0 / d)).to(dtype))
        net.step(lr=lr, weight_decay=0.0)
        if say and (i % 50 == 0 or i == steps - 1):
            say("step %d: mean squared error %.5f" % (i, float(losses[-1])))
    return [float(v) for v in losses]


if __name__ == "__main__":
    train(say=print)
