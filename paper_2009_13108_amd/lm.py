"""From tokens to a loss on int8 rows, by the library's calls: a model that
predicts a token's successor from the token, taught by another model's top logits.

    x = alpha E[token],  h = x + (act(n Wg^T) * (n Wu^T)) Wd^T  with n = norm(x),  logits = norm(h) E^T

E, the table and the output layer in one, and the weights are int8 rows with a
scale each wherever they are read or multiplied; their 32-bit masters are what
AdamW updates.  E's gradient is the output layer's, to which the lookup's is
added.  All memory is taken once: a pass allocates nothing and never waits for the device.

    python -m paper_2009_13108_amd.lm    teaches one a synthetic successor table and scores it
"""
from __future__ import annotations

from . import ffn, niti


class TokenModel:
    """A model of a vocabulary of v, width d and hidden width f, for `tokens` tokens at a time."""

    def __init__(self, v, d, f, tokens, dtype, top, act=niti.ACT_SILU, scale=1.0, state_bits=8, mode=niti.SR, seed=1, device="cuda"):
        import torch
        self.v, self.d, self.f, self.tokens, self.act, self.scale = v, d, f, tokens, act, scale
        self.mode, self.seed, self.steps, self.alpha = mode, seed, 0, d ** 0.5
        # the optimiser counts its draws by steps, the gradients by calls: under one seed they would meet
        self.state_seed = seed ^ 1 << 63
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        new = lambda *shape, t=dtype: torch.zeros(shape, dtype=t, device=device)  # noqa: E731
        f32, i8 = torch.float32, torch.int8
        normal = lambda rows, cols: torch.randn(rows, cols, generator=g, device=device) / cols ** 0.5  # noqa: E731
        self.w = {"table": normal(v, d), "gated": normal(2 * f, d), "down": normal(d, f)}
        self.vec = {"gain": torch.ones(d, device=device), "last": torch.ones(d, device=device)}
        self.dw = {k: new(*w.shape) for k, w in self.w.items()}
        self.dvec = {k: torch.zeros_like(w) for k, w in self.vec.items()}
        self.wq = {k: (new(*w.shape, t=i8), new(w.shape[0], t=f32)) for k, w in self.w.items()}
        # a forward pass, its loss and its gradients
        m = tokens
        self.x, self.out = new(m, d), new(m, d)
        self.rows = {k: (new(m, c, t=i8), new(m, t=f32)) for k, c in (("n", d), ("u", f), ("last", d))}
        self.rstd = {k: new(m, t=f32) for k in ("n", "last")}
        self.z, self.u, self.logits = new(m, 2 * f), new(m, f), new(m, v)
        self.loss, self.lse, self.weight = new(m, t=f32), new(m, t=f32), torch.full((1,), 1.0 / m, device=device)
        self.dn, self.dout, self.du, self.dx = new(m, d), new(m, d), new(m, f), new(m, d)
        self.logp, self.entropy = new(m, t=f32), new(m, t=f32)
        self.top_logp, self.top_idx = new(m, top, t=f32), new(m, top, t=torch.int32)
        ws = max(niti.workspace_bytes(op, None, *sizes) for op, sizes in (
            (niti.OP_GATED_FWD, (m, f, d)), (niti.OP_GATED_BWD, (m, f, d)), (niti.OP_LINEAR_FWD, (m, d, f)), (niti.OP_LINEAR_BWD, (m, d, f)),
            (niti.OP_LINEAR_FWD, (m, v, d)), (niti.OP_LINEAR_BWD, (m, v, d)), (niti.OP_RMSNORM_BWD, (m, d)), (niti.OP_EMBEDDING_BWD, (m, v, d)),
            (niti.OP_DISTILL_FWD, (m, v)), (niti.OP_TOKEN_LOGPROBS, (m, v, top))))
        self.ws = niti.new_workspace(ws, device)
        self.plans = [ffn.FeedForward._plan(list(self.w.values()), list(self.dw.values()), state_bits, device),
                      ffn.FeedForward._plan(list(self.vec.values()), list(self.dvec.values()), 32, device)]
        self.lay_out()

    def lay_out(self):
        """The weights as int8 rows, one scale for each output channel or token."""
        for k, w in self.w.items():
            niti.quantize_rows(w, *self.wq[k])

    def forward(self, tokens):
        """Logits [tokens][v] of the tokens' successors."""
        (e, se), (w, sw), (wd, sd) = (self.wq[k] for k in ("table", "gated", "down"))
        (n, sn), (u, su), (last, sl) = (self.rows[k] for k in ("n", "u", "last"))
        niti.embedding_fwd(e, tokens, self.x, table_scale=se, alpha=self.alpha)
        niti.rmsnorm_fwd(self.x, self.vec["gain"], q=n, scale=sn, rstd=self.rstd["n"])
        niti.gated_fwd(n, w, self.u, sn, sw, act=self.act, z=self.z, ws=self.ws)
        niti.quantize_rows(self.u, u, su)
        niti.linear_fwd(u, wd, self.out, su, sd, res=self.x, ws=self.ws)
        niti.rmsnorm_fwd(self.out, self.vec["last"], q=last, scale=sl, rstd=self.rstd["last"])
        niti.linear_fwd(last, e, self.logits, sl, se, ws=self.ws)
        return self.logits

    def teach(self, tokens, t_val, t_idx):
        """Losses [tokens] of the last forward pass against a teacher's top logits, and the gradients of their mean; the
        logits are their own gradient afterwards.  Stochastic draws go by the number of steps taken: repeated before the
        next, after another forward pass, it gives the same again."""
        (e, se), (w, sw), (wd, sd) = (self.wq[k] for k in ("table", "gated", "down"))
        (n, sn), (u, su), (last, sl) = (self.rows[k] for k in ("n", "u", "last"))
        draws = lambda i: dict(mode=self.mode, seed=self.seed, call=3 * self.steps + i)  # noqa: E731
        niti.distill_fwd(self.logits, t_val, t_idx, self.loss, lse=self.lse, dlogits=self.logits, dloss=self.weight, scale=self.scale,
                         ws=self.ws)
        niti.linear_bwd(self.logits, last, e, sl, se, self.ws, da=self.dn, db=self.dw["table"], **draws(0))
        niti.rmsnorm_bwd(self.dn, self.out, self.vec["last"], self.rstd["last"], self.dout, self.dvec["last"], self.ws)
        niti.linear_bwd(self.dout, u, wd, su, sd, self.ws, da=self.du, db=self.dw["down"], **draws(1))
        niti.gated_bwd(self.du, self.z, n, w, sn, sw, self.ws, act=self.act, da=self.dn, db=self.dw["gated"], **draws(2))
        niti.rmsnorm_bwd(self.dn, self.x, self.vec["gain"], self.rstd["n"], self.dx, self.dvec["gain"], self.ws, dh=self.dout)
        niti.embedding_bwd(self.dx, tokens, self.dw["table"], self.ws, alpha=self.alpha, accumulate=True)
        return self.loss

    def step(self, lr=1e-3, weight_decay=0.01):
        """AdamW on all weights, and their int8 rows again."""
        self.steps += 1
        for plan in self.plans:
            niti.adamw_step(plan, self.steps, lr, weight_decay=weight_decay, mode=self.mode, seed=self.state_seed)
        self.lay_out()

    def score(self, tokens, successors):
        """Log probabilities of given successors; entropies and top alternatives are in entropy, top_logp and top_idx."""
        niti.token_logprobs(self.forward(tokens), tokens=successors, logp=self.logp, lse=self.lse, entropy=self.entropy,
                            top_logp=self.top_logp, top_idx=self.top_idx, scale=self.scale, ws=self.ws)
        return self.logp


def train(steps=200, v=1000, d=256, f=512, tokens=512, dtype=None, top=8, state_bits=8, seed=1, lr=3e-3, say=None):
    """Teaches a model a random table of successors; returns the mean losses by step and the model."""
    import torch
    dtype = dtype or torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    val, idx = torch.topk(3 * torch.randn(v, v, generator=g, device="cuda"), top, dim=1)
    idx = idx.to(torch.int32)
    net = TokenModel(v, d, f, tokens, dtype, top, state_bits=state_bits, seed=seed)
    losses = []
    for i in range(steps):
        tok = torch.randint(0, v, (tokens,), generator=g, device="cuda").to(torch.int32)
        net.forward(tok)
        losses.append(net.teach(tok, val[tok.long()], idx[tok.long()]).mean())
        net.step(lr=lr, weight_decay=0.0)
        if say and (i % 50 == 0 or i == steps - 1):
            say("step %d: divergence from the teacher %.4f" % (i, float(losses[-1])))
    if say:
        tok = torch.arange(tokens, device="cuda", dtype=torch.int32) % v
        logp = net.score(tok, idx[tok.long(), 0].contiguous())
        say("mean log probability of the teacher's first choice %.3f, mean entropy %.3f" % (float(logp.mean()), float(net.entropy.mean())))
    return [float(x) for x in losses], net


if __name__ == "__main__":
    train(say=print)
