"""Definitions in 64 bits of rotary positions and exact cross attention, and bounds on what the roundings may change."""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # largest relative error of one rounding


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original=0, slow=1.0, fast=32.0):
    out = []
    for j in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "ntk" else base
        t = b ** (-2.0 * j / rot)
        if scaling == "linear":
            t /= factor
        if scaling == "parts":
            keep = min(1.0, max(0.0, (original * t / (2 * math.pi) - slow) / (fast - slow)))
            t = t * (keep + (1 - keep) / factor)
        out.append(t)
    return torch.tensor(out, dtype=torch.float64)


def rotated(X, pos, theta, layout="half", gain=1.0, transpose=False):
    """X [B,H,L,d] by positions [B,L], in 64 bits on X's device; only the pairs' features are computed."""
    x = X.double().clone()
    rot = 2 * len(theta)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    angle = (pos.double()[:, None, :, None] * theta.to(x.device)) * (-1 if transpose else 1)
    u, v = X.double()[..., a], X.double()[..., b]
    x[..., a], x[..., b] = gain * (u * angle.cos() - v * angle.sin()), gain * (v * angle.cos() + u * angle.sin())
    return x


def seen_of(B, Lk, key_len=None, key_mask=None):
    s = torch.ones(B, Lk, dtype=torch.bool)
    if key_len is not None:
        s &= torch.arange(Lk)[None] < key_len.cpu().long().clamp(0, Lk)[:, None]
    if key_mask is not None:
        s &= key_mask.cpu().bool().expand(B, Lk)
    return s


class Cross:
    """Cross attention and its gradients from the definition in 64 bits on the CPU, with sums of magnitudes for bounds."""

    def __init__(self, Q, K, V, scale, key_len=None, key_mask=None):
        q, k, v = (t.detach().cpu().double() for t in (Q, K, V))
        B, H, Lq, d = q.shape
        self.seen = seen_of(B, k.shape[2], key_len, key_mask)
        hide = ~self.seen[:, None, :, None]
        self.g, self.scale = H // k.shape[1], scale
        k, v = (t.masked_fill(hide, 0.0).repeat_interleave(self.g, 1) for t in (k, v))
        self.q, self.k, self.v = q, k, v
        S = (q @ k.transpose(2, 3)) * scale
        S = S.masked_fill(~self.seen[:, None, None], -math.inf)
        self.lse = torch.logsumexp(S, 3) if k.shape[2] else torch.full((B, H, Lq), -math.inf, dtype=torch.float64)
        some = self.lse > -math.inf
        self.P = (S - torch.where(some, self.lse, 0.0)[..., None]).exp()
        self.Y = self.P @ v
        self.Yabs = self.P @ v.abs()
        self.Sabs = (q.abs() @ k.abs().transpose(2, 3)) * scale          # sums of magnitudes behind each score

    def grads(self, dY):
        g = dY.detach().cpu().double()
        fold = lambda t: t.unflatten(1, (-1, self.g)).sum(2)             # noqa: E731  (heads that share keys)
        dP = g @ self.v.transpose(2, 3)
        D = (g * self.Y).sum(3, keepdim=True)
        self.dS = self.P * (dP - D) * self.scale
        return self.dS @ self.k, fold(self.dS.transpose(2, 3) @ self.q), fold(self.P.transpose(2, 3) @ g)

    def score_error(self, d):
        """Largest absolute error of a score summed in fp32 from d products (exact ones of bf16, rounded ones of fp32), the
        factor applied to Q or to the sum, in nats: (d + 4) half steps of the sum of magnitudes."""
        return (d + 4) * 2.0 ** -24 * self.Sabs

    def bound_Y(self, dtype):
        """|error of Y|.  A score off by e changes its weight by the factor exp(e), and the normaliser's error is at most as
        large: 2 max e; one more for the exponential and the sums (a 2^-20 covers 2^x to 2 ulp and sums over tiles).  bf16:
        weights rounded once (or their 2^x from a cubic of relative error 8.6e-5 first), the result once."""
        e = 2 * self.score_error(self.q.shape[3]).amax(3, keepdim=True) if self.P.shape[3] else 0.0
        h = HALF_STEP[dtype]
        w = 2.0 ** -20 + e + (h + 2e-4 if dtype == torch.bfloat16 else 0.0)
        return 1.02 * (w * self.Yabs + h * (self.Y.abs() + w * self.Yabs)) + 1e-30

    def bound_grads(self, dY, dtype):
        """|error| of dQ, dK, dV, given Y of the forward call (bound_Y off).  dP sums dv products in fp32; D sums dY times an
        inexact Y; dS is rounded to the products' type; results are rounded once; P as above."""
        h, g = HALF_STEP[dtype], dY.detach().cpu().double()
        fold = lambda t: t.unflatten(1, (-1, self.g)).sum(2)             # noqa: E731
        dQ, dK, dV = self.grads(dY)
        lse_off = 2.0 ** -22 * (1 + self.lse.abs().nan_to_num(0, 0, 0))[..., None]      # lse rounded, times log2(e) rounded
        e = self.score_error(self.q.shape[3]) + lse_off + 2.0 ** -20 + (2e-4 if dtype == torch.bfloat16 else 0.0)
        dP = g @ self.v.transpose(2, 3)
        D = (g * self.Y).sum(3, keepdim=True)
        dv = self.v.shape[3]
        off = (dv + 2) * 2.0 ** -24 * (g.abs() @ self.v.abs().transpose(2, 3)) + \
            ((g.abs() * (self.bound_Y(dtype) + (dv + 2) * 2.0 ** -24 * self.Y.abs())).sum(3, keepdim=True))
        hs = h if dtype == torch.bfloat16 else 2.0 ** -23
        ds = self.scale * self.P * (off + (e + hs) * (dP - D).abs()) * 1.02
        p = self.P * (e + hs)
        n = (self.P.shape[2] * self.g + self.P.shape[3]) * 2.0 ** -24    # sums in fp32
        bQ = ds @ self.k.abs() + n * (self.dS.abs() @ self.k.abs()) + h * dQ.abs()
        bK = fold(ds.transpose(2, 3) @ self.q.abs() + n * (self.dS.abs().transpose(2, 3) @ self.q.abs())) + h * dK.abs()
        bV = fold(p.transpose(2, 3) @ g.abs() + n * (self.P.transpose(2, 3) @ g.abs())) + h * dV.abs()
        return tuple(1.05 * b + 1e-30 for b in (bQ, bK, bV))


def inside(got, ref, bound, what=""):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() / bound
    assert float(over.max() if over.numel() else 0.0) <= 1.0, (what, float(over.max()), int(over.argmax()))
