"""How far the exact cross attention is off as a whole: the 2-norm of a head's error relative to its result's.  An element's bound has to
allow for the worst signs of all roundings; a norm need not, so it sees a seen key that a kernel has left out.

bf16: relative rounding errors of 2^-8 at most are 2^-8 / sqrt(3) sqrt(0.541) = 0.00166 in the root mean square (significands spread over their
logarithm).  Y and dV have two of them (P, the result), independent of each other: 0.0024; so have dQ and dK (dS, the result), and D from the Y that was
rounded, 0.0024 / sqrt(keys that count) more.  0.004 is over 1.5 times that, and a norm over N values varies by 1 / sqrt(2 N) of itself.
fp32: scores off by some 2^-25 sqrt(d) of their size (up to 4e-7), the exponential by 2 ulp, its argument and lse by 2^-20 half steps where
they are 8 to 32 (3e-7 each), sums over up to 2000 values by 2^-25 sqrt(2000) at most (1.3e-6 if nothing is summed by tiles first; a tenth of that on the
tensor cores, whose sums are made by tiles): 2e-6."""
import math

import pytest
import torch

from paper_2302_00787_b200 import binding as fb
from tests.layer_util import Cross

F32, BF16 = torch.float32, torch.bfloat16
MOST = {BF16: 0.004, F32: 2e-6}


def off_by(got, ref):
    """The largest relative 2-norm of a (batch, head)'s error; a result that is zero has to be it exactly."""
    got, ref = got.detach().cpu().double(), ref.double()
    e, n = (got - ref).flatten(2).norm(dim=2), ref.flatten(2).norm(dim=2)
    assert torch.isfinite(got).all() and (e[n == 0] == 0).all()
    return float((e / n.clamp_min(1e-300))[n > 0].max()) if (n > 0).any() else 0.0


CASES = [
    # B, H, Hk, Lq, Lk, d, dv, mask: at least 16 seen keys, so that dS is not a difference of equal numbers
    (2, 4, 2, 20, 1500, 64, 64, ""),
    (2, 4, 4, 100, 2001, 64, 64, "len"),
    (1, 4, 1, 130, 700, 128, 128, "bytes"),
    (3, 6, 3, 1, 900, 64, 64, "len"),
    (3, 6, 6, 1, 900, 128, 64, "len+bytes"),
    (2, 8, 2, 1, 1100, 128, 128, "len+bytes"),
    (2, 4, 2, 300, 257, 32, 32, "len"),
    (1, 2, 2, 513, 1030, 16, 64, "bytes"),
    (20, 8, 8, 20, 1500, 64, 64, "len"),
    (20, 8, 4, 60, 600, 128, 128, "len+bytes"),
    (2, 2, 1, 1000, 300, 64, 128, "len"),
]
NAMES = ["x".join(map(str, c[:7])) + c[7] for c in CASES]


def make(case, dtype, seed=0):
    B, H, Hk, Lq, Lk, d, dv, mask = case
    gen = torch.Generator().manual_seed(seed)
    Q, K, V, dY = (torch.randn(B, *s, generator=gen).to(dtype) for s in ((H, Lq, d), (Hk, Lk, d), (Hk, Lk, dv), (H, Lq, dv)))
    key_len = torch.randint(100, Lk + 1, (B,), generator=gen).int() if "len" in mask else None
    key_mask = torch.rand(B, Lk, generator=gen) < 0.7 if "bytes" in mask else None
    return Q, K, V, dY, key_len, key_mask, Cross(Q, K, V, d ** -0.5, key_len, key_mask)


@pytest.mark.parametrize("case", CASES[:4], ids=NAMES[:4])
def test_a_key_left_out_shows(case):
    """The mistake is planted in the definition: one seen key of one head without its V (Y), without its K (dQ); one row missing (dK, dV)."""
    Q, K, V, dY, _, _, ref = make(case, BF16)
    dQ, dK, dV = ref.grads(dY)
    assert off_by(ref.Y, ref.Y) == off_by(dQ, dQ) == 0.0
    # the worst places a test can have: the key and the row that matter least among the upper half of them
    weight = torch.where(ref.seen[0], (ref.P[0, 0] ** 2).sum(0), -1.0)
    j = int(weight.argsort(descending=True)[int(ref.seen[0].sum()) // 2])
    Y = ref.Y.clone()
    Y[0, 0] -= ref.P[0, 0, :, j: j + 1] * ref.v[0, 0, j]
    assert off_by(Y, ref.Y) > MOST[BF16]
    wrong = dQ.clone()
    wrong[0, 0] -= ref.dS[0, 0, :, j: j + 1] * ref.k[0, 0, j]
    assert off_by(wrong, dQ) > MOST[BF16]
    i = ref.P.shape[2] // 2
    wrong = dV.clone()
    wrong[0, 0] -= ref.P[0, 0, i][:, None] * dY[0, 0, i].double()
    assert off_by(wrong, dV) > MOST[BF16]
    wrong = dK.clone()
    wrong[0, 0] -= ref.dS[0, 0, i][:, None] * ref.q[0, 0, i]
    assert off_by(wrong, dK) > MOST[BF16]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("impl", (fb.IMPL_AUTO, fb.IMPL_SIMT), ids=("auto", "simt"))
@pytest.mark.parametrize("case", CASES, ids=NAMES)
def test_norms_of_errors(case, impl, dtype):
    Q, K, V, dY, key_len, key_mask, ref = make(case, dtype)
    junk = torch.tensor(math.nan, dtype=dtype)
    K, V = (torch.where(ref.seen[:, None, :, None], t, junk) for t in (K, V))
    Q, K, V, dY = (t.cuda() for t in (Q, K, V, dY))
    kw = {"key_len": None if key_len is None else key_len.cuda(), "key_mask": None if key_mask is None else key_mask.cuda()}
    ctx = fb.Context(0)
    ctx.set_impl(impl)
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
    got = (Y,) + ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
    off = {n: off_by(g, r) for n, g, r in zip(("Y", "dQ", "dK", "dV"), got, (ref.Y,) + ref.grads(dY))}
    assert max(off.values()) <= MOST[dtype], off
    # lse is an fp32 number whatever the tensors' type: the scores' error, the exponentials' (3e-6 by the quartic, 2 ulp otherwise), the sum's
    # additions, and the roundings of the logarithm and of the factor
    bound = ref.score_error(case[5]).amax(3) + (4e-6 if dtype == BF16 else 2.0 ** -22) + case[4] * 2.0 ** -24 + 2.0 ** -22 * (1 + ref.lse.abs())
    assert ((lse.cpu().double() - ref.lse).abs() <= bound).all()
    assert ctx.status() == 0
    ctx.close()
