"""The losses of a linear head over many classes in 64 bits, from their formulas, and how far fp32 arithmetic may be off.

u = 2^-24 is fp32's rounding, K the width, S = sum |x| |w| + |bias| of a logit.  A matrix instruction adds 16 products to a
sum; each may be off by two roundings (it drops instead of rounding), so a 16-bit logit is off by at most (K / 8 + 16) u S.
fp32 operands are six times as many products, of which those left out are below 2^-24 of theirs: (K + 24) u S.  A logit of an
entry is a sum of K / 64 products a lane and six more: within the same bound.  The same holds for the
sums over classes and over rows.
"""
import torch

U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def gamma(n, dtype):
    return ((n + 24) if dtype == torch.float32 else (n / 8 + 16)) * U


def shares(index, teacher, classes, tau):
    """(entries that count, t, log t with 0 where t is 0) of [rows, top]."""
    there = (index >= 0) & (index < classes)
    if teacher is None:
        return there, there.double(), torch.zeros(index.shape, dtype=torch.float64, device=index.device)
    l = (teacher.double() / tau).masked_fill(~there, float("-inf"))
    some = (l > float("-inf")).any(1, keepdim=True)
    t = torch.softmax(l.masked_fill(~some, 0.0), 1).masked_fill(~some | ~there, 0.0)
    return there & some, t, torch.where(t > 0, t, 1.0).log()


class Head:
    """z / tau and its error's bound, of rows [rows, width]; index [rows, top]."""

    def __init__(self, x, weight, bias, index, teacher=None, tau=1.0):
        self.dtype, self.tau = x.dtype, tau
        self.x, self.w, self.index = x.double(), weight.double(), index
        classes = len(weight)
        self.there, self.t, self.logt = shares(index, teacher, classes, tau)
        self.row = self.there.any(1)
        self.x = torch.where(self.row[:, None], self.x, 0.0)
        self.pick = index.clamp(0, classes - 1)
        z, size = self.x @ self.w.T, self.x.abs() @ self.w.abs().T
        if bias is not None:
            z, size = z + bias.double(), size + bias.double().abs().nan_to_num(posinf=0.0)
        self.z = z / tau
        # z, and its division (a product with a rounded quotient)
        self.ez = gamma(x.shape[1], x.dtype) * size / tau + 3 * U * self.z.abs().nan_to_num(posinf=0.0)

    def forward(self):
        """loss, lse, logq, and their bounds."""
        lse = torch.logsumexp(self.z, 1)
        q = torch.exp(self.z - lse[:, None])
        off = (lse[:, None] - self.z).nan_to_num(posinf=0.0)
        # each term by its logit's error, its exponential (|argument| + 4 roundings) and a sum in a tree; then a logarithm
        elementwise = self.ez + (2 * off + 200) * U
        elementwise = torch.where(q > 0, elementwise, 0.0)
        else_ = (q * elementwise).sum(1) + 4 * U * lse.abs() + 4 * U
        logq = self.z.gather(1, self.pick) - lse[:, None]
        elogq = self.ez.gather(1, self.pick) + else_[:, None] + 2 * U * (logq.abs() + lse.abs()[:, None])
        logq, elogq = (torch.where(self.there, v, 0.0) for v in (logq, elogq))
        cross = torch.where(self.t > 0, self.t * (self.logt - logq), 0.0)
        # shares: an exponential and a quotient, with the teacher's logits' division before
        et = (8 + 2 * self.logt.abs()) * 4 * U * self.t
        size = torch.where(self.t > 0, self.t * (self.logt.abs() + logq.abs()), 0.0)
        eloss = torch.where(self.t > 0, et * (1 + self.logt.abs() + logq.abs()) + self.t * elogq, 0.0) + 40 * U * size
        tau2 = self.tau ** 2
        loss, eloss = tau2 * cross.sum(1), tau2 * eloss.sum(1) * (1 + 4 * U)
        zero = torch.zeros_like(lse)
        return (torch.where(self.row, loss, zero), torch.where(self.row, lse, zero), logq, torch.where(self.row, eloss, zero),
                torch.where(self.row, else_, zero), elogq)

    def backward(self, lse, logq, dloss):
        """dx, dweight, dbias from given lse and logq, and their bounds."""
        lse, logq = lse.double()[:, None], logq.double()
        coef = torch.where(self.row, dloss.double().expand(len(lse)) * self.tau, 0.0)[:, None]
        arg = self.z - lse
        q = torch.exp(arg)
        eq = q * (self.ez + (2 * arg.abs().nan_to_num(posinf=0.0) + 8) * U + 2 * U * lse.abs())
        at = torch.exp(logq)
        n = torch.arange(len(q), device=q.device)[:, None].expand(self.pick.shape)
        q, eq = q.clone(), eq.clone()
        q[n[self.there], self.pick[self.there]] = at[self.there]
        eq[n[self.there], self.pick[self.there]] = ((2 * logq.abs() + 8) * U * at)[self.there]
        t = torch.zeros_like(q).index_put_((n[self.there], self.pick[self.there]), self.t[self.there], accumulate=True)
        et = torch.zeros_like(q).index_put_((n[self.there], self.pick[self.there]),
                                            ((8 + 2 * self.logt.abs()) * 4 * U * self.t)[self.there], accumulate=True)
        g = torch.where(self.row[:, None], coef * (q - t), 0.0)
        eg = torch.where(self.row[:, None], coef.abs() * (eq + et) + 4 * U * coef.abs() * (q + t), 0.0)
        # the bias's gradient is taken before the rounding: sums of 64 rows, then of tiles in 64 bits; shares as whole 2^-24 of 2^-13
        whole = 2.0 ** -37 * coef.abs().max()
        dbias, edbias = g.sum(0), (eg + 80 * U * (coef * q).abs() + whole).sum(0) + 2 * U * g.sum(0).abs()
        low = 2.0 ** -38 * coef.abs().max() if self.dtype == torch.float16 else 0.0  # (fp16's smallest step, scaled)
        # up to 256 rows or classes in 16 bits: a rounding and that of what it leaves over, and sums of twice as many products
        terms = 2 if min(q.shape) <= 256 and self.dtype in (torch.bfloat16, torch.float16) else 1
        eg = eg + HALF[self.dtype] ** terms * (g.abs() + eg) + torch.where(self.row[:, None], low, 0.0)
        dx, dw = g @ self.w, g.T @ self.x
        edx = eg @ self.w.abs() + gamma(terms * q.shape[1], self.dtype) * (g.abs() @ self.w.abs())
        edw = eg.T @ self.x.abs() + gamma(terms * len(q), self.dtype) * (g.abs().T @ self.x.abs())

        def stored(v, e):
            return e + HALF[self.dtype] * (v.abs() + e) + TINY[self.dtype]

        return dx, dw, dbias, stored(dx, edx), stored(dw, edw), edbias + 1e-37
