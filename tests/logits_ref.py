"""64-bit forms of the operators on logits, and what their evaluation in 32
bits may be off by.

With u = x - max x an exponential's argument is off by 3 U32 scale |u| (the difference, the factor, their
product), its value by one step of the hardware's exponential (2 U32) more, and a sum of them by U32 for each level:
up to 128 terms of a thread one after the other, 6 levels in a wave, 16 waves, 6 for the parts of a row."""
import torch

from scaled_ref import U32

DEPTH = 128 + 6 + 16 + 6


class Rows:
    """Softmax statistics of scale * x by rows; masked values are minus infinity."""

    def __init__(self, x, scale):
        x = x.double().cpu()
        top = x.amax(dim=1, keepdim=True)
        self.empty = (top == float("-inf")).squeeze(1)
        base = torch.where(top == float("-inf"), torch.zeros_like(top), top)
        self.x, self.scale, self.base = x, scale, base
        self.u = x - base
        e = torch.exp(scale * self.u)
        self.s = e.sum(dim=1)
        eu = torch.where(e > 0, e * self.u, torch.zeros_like(e))
        euu = torch.where(e > 0, eu * self.u, torch.zeros_like(e))
        self.log = torch.log(self.s)
        self.q = torch.where(self.empty[:, None], torch.zeros_like(e), e / self.s[:, None])
        self.mean = torch.where(self.empty, torch.zeros_like(self.s), -scale * eu.sum(dim=1) / self.s)     # of scale |u|
        square = torch.where(self.empty, torch.zeros_like(self.s), scale * scale * euu.sum(dim=1) / self.s)
        self.lse = scale * base.squeeze(1) + self.log
        self.entropy = torch.where(self.empty, torch.zeros_like(self.s), self.log + self.mean)
        # relative error of S, in U32, and the bounds of what is formed from it
        self.rel = DEPTH + 2 + 3 * self.mean
        log = self.log.abs().nan_to_num(posinf=0)
        self.log_off = U32 * (self.rel + 2 * log)
        self.lse_off = self.log_off + U32 * ((scale * base).abs().squeeze(1) + self.lse.abs().nan_to_num(posinf=0))
        self.entropy_off = self.log_off + U32 * ((DEPTH + 6) * self.mean + 3 * square + self.rel * self.mean + 2 * self.entropy)

    def logp(self, cols):
        """Log probabilities of columns [M][n] and their bounds."""
        u = torch.gather(self.u, 1, cols)
        v = self.scale * u - self.log[:, None]
        v = torch.where(self.empty[:, None], torch.full_like(v, float("-inf")), v)
        off = self.log_off[:, None] + U32 * (2 * (self.scale * u).abs() + v.abs())
        return v, off.nan_to_num(posinf=0, nan=0)

    def top(self, k):
        """Columns of the k largest, equal ones by column."""
        return torch.sort(self.x, dim=1, descending=True, stable=True).indices[:, :k]


class Teacher:
    """The distribution over listed columns; columns outside 0..v-1 are no part of it."""

    def __init__(self, t_val, t_idx, v, scale):
        t = t_val.double().cpu()
        idx = t_idx.long().cpu()
        inside = (idx >= 0) & (idx < v)
        self.col = idx.clamp(0, v - 1)
        rows = Rows(torch.where(inside, t, torch.full_like(t, float("-inf"))), scale)
        self.p, self.empty = rows.q, rows.empty
        at = torch.arange(t.shape[1]).expand(t.shape)
        self.logp, self.logp_off = rows.logp(at)
        # p = exp / sum: as an exponential, the sum and two roundings more
        self.p_rel = U32 * (3 * (scale * rows.u).abs().nan_to_num(posinf=0) + 2 + rows.rel[:, None] + 2)


def loss64(rows, teacher):
    logq, logq_off = rows.logp(teacher.col)
    live = teacher.p > 0
    d = torch.where(live, teacher.logp - logq, torch.zeros_like(logq))
    loss = (teacher.p * d).nan_to_num(posinf=float("inf")).sum(dim=1)
    fine = d.nan_to_num(posinf=0).abs()
    off = (teacher.p * (teacher.logp_off + logq_off) + teacher.p * fine * (teacher.p_rel + 30 * U32)).sum(dim=1)
    return loss, off


def listed(rows, teacher):
    """Sum of p by column, and of its bounds."""
    zero = torch.zeros_like(rows.x)
    return zero.scatter_add(1, teacher.col, teacher.p), zero.scatter_add(1, teacher.col, teacher.p * teacher.p_rel)


def grad64(rows, teacher, dloss, lse=None):
    """dx and its bound: from the row's own statistics, or from a given lse."""
    g = (dloss.double().cpu() * rows.scale).view(-1, 1)
    if lse is None:
        q = rows.q
        q_off = q * U32 * (3 * (rows.scale * rows.u).abs() + 2 + rows.rel[:, None] + 2).nan_to_num(posinf=0)
    else:
        d = rows.scale * rows.x - lse.double().cpu()[:, None]
        q = torch.where(lse.double().cpu()[:, None] == float("-inf"), torch.zeros_like(d), torch.exp(d))
        q_off = q * U32 * (3 * d.abs() + 2).nan_to_num(posinf=0, nan=0)
    p, p_off = listed(rows, teacher)
    dx = g * (q - p)
    dx = torch.where(teacher.empty[:, None], torch.zeros_like(dx), dx)
    # the list's sum has up to 256 terms, where columns are listed more than once; three products
    off = g.abs() * (1.01 * q_off + p_off + 256 * U32 * p) + 4 * U32 * (dx.abs() + g.abs() * q)
    return dx, off
