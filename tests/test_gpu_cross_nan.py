"""NaNs and infinities among what the gradients of the exact cross attention see: a gradient is NaN where the definition in
64 bits is, whatever the place of the bad row in a tile, and what does not depend on it stays as it was, bit for bit."""
import math

import pytest
import torch

from paper_2302_00787_b200 import binding as fb
from tests.layer_util import Cross

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    c.close()


def gradients(ctx, Q, K, V, dY, **kw):
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
    return (Y, lse) + ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("impl", (fb.IMPL_AUTO, fb.IMPL_SIMT), ids=("auto", "simt"))
@pytest.mark.parametrize("d,dv", ((64, 64), (128, 128), (32, 128)))
@pytest.mark.parametrize("bad", (math.nan, math.inf, -math.inf))
def test_bad_query_row_at_every_place(ctx, dtype, impl, d, dv, bad):
    """One entry of one query row, at each place of eight neighbouring rows and of both halves of a tile."""
    B, H, Hk, Lq, Lk = 2, 4, 2, 70, 150
    gen = torch.Generator().manual_seed(0)
    Q, dY = (torch.randn(B, H, Lq, n, generator=gen).to(dtype) for n in (d, dv))
    K, V = (torch.randn(B, Hk, Lk, n, generator=gen).to(dtype) for n in (d, dv))
    key_len = torch.tensor([Lk - 9, Lk], dtype=torch.int32)
    ctx.set_impl(impl)
    try:
        clean = gradients(ctx, Q.cuda(), K.cuda(), V.cuda(), dY.cuda(), key_len=key_len.cuda())
        for row in [*range(8), *range(30, 38), *range(62, 70)]:
            q = Q.clone()
            q[0, 1, row, 5] = bad
            got = gradients(ctx, q.cuda(), K.cuda(), V.cuda(), dY.cuda(), key_len=key_len.cuda())
            ref = Cross(q, K, V, d ** -0.5, key_len)
            want = (ref.Y, None) + ref.grads(dY.double())
            for name, g, c, r in zip(("Y", "lse", "dQ", "dK", "dV"), got, clean, want):
                g, c = g.cpu(), c.cpu()
                if r is not None:
                    lost = torch.isnan(r) & ~torch.isnan(g)
                    if name in ("dK", "dV"):
                        lost &= ref.seen[:, None, :, None]          # (zeros at hidden keys, whatever else is NaN)
                    assert not lost.any(), (name, row, int(lost.sum()))
                # the bad row itself, and the keys that it shares with its key head, may be anything else
                same = torch.ones_like(g, dtype=torch.bool)
                if name in ("dK", "dV"):
                    same[0, 0, : Lk - 9] = False
                else:
                    same[0, 1, row] = False
                assert torch.equal(g[same], c[same]), (name, row)
    finally:
        ctx.set_impl(fb.IMPL_AUTO)
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("d", (64, 128))
def test_rows_of_nan_at_hidden_keys_and_of_empty_sequences(ctx, dtype, d):
    """NaN queries and cotangents of a sequence without keys reach nobody; NaN cotangents of one head stay with its key head."""
    B, H, Lq, Lk = 3, 2, 133, 140
    gen = torch.Generator().manual_seed(1)
    Q, K, V, dY = (torch.randn(B, H, n, d, generator=gen).to(dtype).cuda() for n in (Lq, Lk, Lk, Lq))
    key_len = torch.tensor([Lk, 0, 77], dtype=torch.int32).cuda()
    clean = gradients(ctx, Q, K, V, dY, key_len=key_len)
    Q, dY = Q.clone(), dY.clone()
    Q[1], dY[1], dY[2, 0] = math.nan, math.nan, math.nan
    got = gradients(ctx, Q, K, V, dY, key_len=key_len)
    for name, g, c in zip(("Y", "lse", "dQ", "dK", "dV"), got, clean):
        same = torch.ones_like(g, dtype=torch.bool)
        if name in ("dQ", "dK", "dV"):
            same[2, 0] = False
        assert torch.equal(g[same], c[same]), name
    assert torch.isnan(got[2][2, 0]).all() and torch.isnan(got[3][2, 0, :77]).all() and torch.isnan(got[4][2, 0, :77]).all()
    assert (got[3][2, 0, 77:] == 0).all() and (got[4][2, 0, 77:] == 0).all()
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("impl", (fb.IMPL_AUTO, fb.IMPL_SIMT), ids=("auto", "simt"))
@pytest.mark.parametrize("d", (64, 128))
def test_scale_of_zero(ctx, dtype, impl, d):
    """All scores are zero; dQ and dK are zero times their sums, NaN where those are."""
    gen = torch.Generator().manual_seed(2)
    Q, K, V, dY = (torch.randn(1, 2, n, d, generator=gen).to(dtype) for n in (70, 150, 150, 70))
    Q[0, 0, 9, 3] = math.nan
    ctx.set_impl(impl)
    try:
        got = gradients(ctx, Q.cuda(), K.cuda(), V.cuda(), dY.cuda(), scale=0.0)
    finally:
        ctx.set_impl(fb.IMPL_AUTO)
    ref = Cross(Q, K, V, 0.0)
    for name, g, r in zip(("Y", "dQ", "dK", "dV"), (got[0],) + got[2:], (ref.Y,) + ref.grads(dY.double())):
        assert torch.equal(torch.isnan(g.cpu()), torch.isnan(r)), name
        if name in ("dQ", "dK"):
            assert (g.cpu()[~torch.isnan(r)] == 0).all(), name
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("Lq", (1, 3))
def test_as_many_units_as_there_may_be(ctx, dtype, Lq):
    """B Hk = 65535, against the formulas in fp32 on the same device (sums over two keys and 16 features: 2e-6, and bf16's roundings)."""
    B, Hk, g, Lk, d = 21845, 3, 2, 2, 16
    gen = torch.Generator(device="cuda").manual_seed(3)
    Q, K, V, dY = (torch.randn(B, *s, d, generator=gen, device="cuda").to(dtype) for s in ((Hk * g, Lq), (Hk, Lk), (Hk, Lk), (Hk * g, Lq)))
    key_len = torch.randint(0, Lk + 1, (B,), generator=gen, device="cuda").int()
    got = gradients(ctx, Q, K, V, dY, key_len=key_len)
    seen = (torch.arange(Lk, device="cuda") < key_len[:, None])[:, None, None]
    q, k, v, y = Q.float(), K.float().repeat_interleave(g, 1), V.float().repeat_interleave(g, 1), dY.float()
    S = (q @ k.transpose(2, 3) * d ** -0.5).masked_fill(~seen, -math.inf)
    P = S.softmax(3).nan_to_num(0.0)
    Y = P @ v
    dS = P * (y @ v.transpose(2, 3) - (y * Y).sum(3, keepdim=True)) * d ** -0.5
    fold = lambda t: t.unflatten(1, (Hk, g)).sum(2)                   # noqa: E731
    want = (Y, S.logsumexp(3), dS @ k, fold(dS.transpose(2, 3) @ q), fold(P.transpose(2, 3) @ y))
    for name, a, b in zip(("Y", "lse", "dQ", "dK", "dV"), got, want):
        if name == "lse":
            assert torch.equal(a == -math.inf, b == -math.inf)
            assert (a - b)[b > -math.inf].abs().max() <= 1e-5
        else:
            # bf16: 0.0045 of dQ and dK by P, dS, Y (in D: all of dS where one key is seen) and the results rounded, made in 64 bits
            assert torch.isfinite(a).all()
            off, size = (a.float() - b).norm(), b.norm()
            assert off <= (0.006 if dtype == BF16 else 4e-6) * size, (name, float(off / size))
    assert ctx.status() == 0
