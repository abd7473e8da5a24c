"""The losses over the vocabulary and the embedding in 64 bits, from their formulas, with the error that their kernels are
allowed.

Allowed errors, from the arithmetic (u = 2^-24, half an fp32 step; a bf16 half step is 2^-8 of the value):
  a logit     Products of bf16 values are exact in fp32; fp32 operands are three bf16 parts each, whose dropped partial products
              are under 3 * 2^-26 of a product. A piece of a sum is at most 512 deep, 32 MMAs (of three parts 256, 16 at the
              full size of its terms and 80 at 2^-8 of it), each of which truncates its products' sum and the accumulator's, at
              most 2 * 2^-23 of the sum of the terms' absolute values S; pieces are added in fp32. So
              dz = (M 2^-22 + (d / 128 + 4) u) S with M = 32 (17 of three parts); the
              truncations hardly ever all have one sign, and 16 is what is asked of both.
  lse         A weighted mean of the logits' errors (over tau), the exponentials' (2^-21 each with its argument's rounding of
              u |z|), and the sums' of positive terms: 128 a thread in four sums, the slots' and their join: under 2^-17.
  loss        lse's and the target's logit's, the final operations' u of their operands.
  dz          p's relative error e = dz + lse's + 2^-20 + u |z| and the multiplication's; stored in bf16 (2^-8 |dz|), in two
              parts for up to 16 tokens (2^-16 |dz|), or in three (2^-24 |dz|).
  dX, dW      a sum over `depth` of products with those errors, truncated in every MMA of 16 (bf16: depth / 16 of them in one
              accumulator; fp32: in pieces, as for a logit), and the output's rounding."""
import torch

U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def _acc(depth, f32):
    """Error of a sum of products over `depth`, of the sum of the terms' absolute values"""
    return 16 * 2.0 ** -22 + (depth / 128 + 4) * U if f32 else (depth / 16 + 2) * 2.0 ** -22


class Loss:
    """goal: (T, V) weights of a token's targets in 64 bits; self_entropy (T): sum q log q"""

    def __init__(self, X, W, goal, self_entropy, has, tau=1.0):
        self.X, self.W, self.goal, self.has, self.tau = X.double(), W.double(), goal, has, tau
        self.f32 = X.dtype == torch.float32
        d = X.shape[1]
        self.X = torch.where(has[:, None], self.X, 0.0)   # what a token without a target holds reaches nothing
        S = self.X.abs() @ self.W.abs().t()
        self.z = self.X @ self.W.t()
        self.dz_err = S * (16 * 2.0 ** -22 + (d / 128 + 4) * U)
        zt = self.z / tau
        self.lse = torch.logsumexp(zt, dim=1)
        self.p = torch.exp(zt - self.lse[:, None])
        top = zt.abs().amax(dim=1)
        self.lse_err = self.dz_err.amax(dim=1) / tau + 2.0 ** -17 + 8 * U * (top + self.lse.abs())
        self.loss = tau * tau * (self_entropy + self.lse - (goal * zt).sum(dim=1))
        self.loss_err = tau * tau * (2 * self.lse_err + 2.0 ** -20 * (self_entropy.abs() + (goal * zt.abs()).sum(dim=1)))
        self.loss = torch.where(has, self.loss, 0.0)
        self.lse = torch.where(has, self.lse, 0.0)

    def check_fwd(self, loss, lse):
        for name, got, want, err in (("lse", lse, self.lse, self.lse_err), ("loss", loss, self.loss, self.loss_err)):
            off = (got.double() - want).abs()
            assert bool((off <= torch.where(self.has, err, 0.0)).all()), (name, float((off / err).max()), float(off.max()))

    def grads(self, dloss):
        g = torch.where(self.has, dloss.double() * self.tau, 0.0)[:, None]
        dz = (self.p - self.goal) * g
        zt = (self.z / self.tau).abs()
        e = self.dz_err / self.tau + self.lse_err[:, None] + 2.0 ** -20 + 4 * U * (zt + self.lse.abs()[:, None])
        err = g.abs() * (self.p * e + 4 * U * self.goal) + dz.abs() * (3 * U if self.f32 else 2.0 ** -16 if dz.shape[0] <= 16 else 2.0 ** -8)
        return dz, err

    def check_bwd(self, dloss, dX, dW):
        dz, err = self.grads(dloss)
        half = 2.0 ** -8 if not self.f32 else U
        out = {}
        for name, got, a, ae, b in (("dX", dX, dz, err, self.W), ("dW", dW, dz.t(), err.t(), self.X)):
            if got is None:
                continue
            want = a @ b
            tol = (ae + _acc(a.shape[1], self.f32) * (a.abs() + ae)) @ b.abs()
            tol = (tol + half * (want.abs() + tol)) * 1.001 + 1e-37
            off = (got.double() - want).abs()
            assert bool((off <= tol).all()), (name, float((off / tol).max()))
            norm = float(want.norm())
            out[name] = float(off.norm()) / norm if norm else 0.0
        return out


def ce(X, W, labels):
    T, V = X.shape[0], W.shape[0]
    has = labels >= 0
    goal = torch.zeros(T, V, dtype=torch.float64, device=X.device)
    goal[has, labels[has]] = 1.0
    return Loss(X, W, goal, torch.zeros(T, dtype=torch.float64, device=X.device), has)


def distill(X, W, index, teacher, tau):
    T, V = X.shape[0], W.shape[0]
    there = index >= 0
    has = there.any(dim=1)
    q = torch.softmax(torch.where(there, teacher.double() / tau, -torch.inf), dim=1)
    q = torch.where(has[:, None], q, 0.0)
    goal = torch.zeros(T, V, dtype=torch.float64, device=X.device).scatter_add_(1, index.clamp_min(0), q)
    return Loss(X, W, goal, torch.xlogy(q, q).sum(dim=1), has, tau)


def inputs(T, V, d, dtype="bf16", seed=0, pad=0, ignored=0.1, wpad=0):
    """Hidden states (a slice of a wider buffer), a head, labels: logits of about one, some far above"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")
    W = normal(V, d + wpad) / d ** 0.5
    labels = torch.randint(0, V, (T,), generator=g, device="cuda")
    X = normal(T, d + pad)
    X[:, :d] += W[labels][:, :d] * (12 * torch.rand(T, 1, generator=g, device="cuda"))
    labels[torch.rand(T, generator=g, device="cuda") < ignored] = -100
    return X.to(DT[dtype])[:, :d], W.to(DT[dtype])[:, :d], labels


def entries(T, V, K, dtype="bf16", seed=0, missing=0.1, empty=0.1):
    """K words a token in no order, and a teacher's logits there"""
    g = torch.Generator(device="cuda").manual_seed(seed + 1000)
    index = torch.rand(T, V, generator=g, device="cuda").argsort(dim=1)[:, :K].contiguous()
    teacher = (2 * torch.randn(T, K, generator=g, device="cuda") + 5).to(DT[dtype])
    index[torch.rand(T, K, generator=g, device="cuda") < missing] = -1
    index[torch.rand(T, generator=g, device="cuda") < empty] = -1
    return index, teacher
