"""A decoder layer's attention as its pieces are used together: rotary positions on q and k, causal FAVOR# self attention, exact
cross attention of its outputs to a padded encoding; and the gradients back through all three.  fp32, against the chain of
the definitions in 64 bits; every stage is held by the tolerances of its own tests (attention 1e-4 per stage, in the metric
max|error| / max|value| per (batch, head)), a chain of three by three times that."""
import numpy as np
import pytest
import torch

from oracle import favor_sharp as fs
from paper_2302_00787_b200 import binding as fb
from paper_2302_00787_b200 import workloads as wl
from tests.layer_util import Cross, frequencies, rotated

pytestmark = pytest.mark.gpu
TOL = 3e-4


def close(got, ref):
    got, ref = got.detach().cpu().double(), torch.as_tensor(ref)
    for b in range(ref.shape[0]):
        for h in range(ref.shape[1]):
            assert (got[b, h] - ref[b, h]).abs().max() <= TOL * ref[b, h].abs().max()


def test_layer_and_its_gradients():
    B, H, L, Le, d, M = 2, 2, 128, 77, 64, 64
    gen = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(B, L, H, d, generator=gen).mul(d ** -0.25).cuda().permute(0, 2, 1, 3) for _ in range(3))
    Ke, Ve = (torch.randn(B, 1, Le, d, generator=gen).cuda() for _ in range(2))
    dY = torch.randn(B, H, L, d, generator=gen).cuda()
    key_len = torch.tensor([Le, 40], dtype=torch.int32).cuda()
    Om = torch.from_numpy(wl.orthogonal_omega(M, d, 7)).cuda()
    ctx = fb.Context(0)
    rope = fb.make_rope(d)
    qr, kr = ctx.fsharp_rotate(q, k, rope)
    params = ctx.fsharp_fit_params(ctx.fsharp_stats(qr, kr), d, "saderf")
    at = {"causal": True, "chunk": 64}
    S = ctx.fsharp_attend(qr, kr, v, Om, params, **at)
    Y, lse = ctx.fsharp_cross_attend(S, Ke, Ve, key_len=key_len, want_lse=True)
    dS, dKe, dVe = ctx.fsharp_cross_attend_backward(S, Ke, Ve, Y, lse, dY, key_len=key_len)
    dqr, dkr, dv = ctx.fsharp_attend_backward(qr, kr, v, dS, Om, params, **at)
    dq, dk = ctx.fsharp_rotate(dqr, dkr, rope, transpose=True)
    assert ctx.status() == 0

    # the same chain in 64 bits
    pos, theta = torch.arange(L).expand(B, L), frequencies(d)
    Q, K = (rotated(t.cpu(), pos, theta).numpy() for t in (q, k))
    V, om = v.cpu().double().numpy(), Om.cpu().numpy()
    p = [[fb.unpack_params(params.cpu().numpy()[b * H + h], d) for h in range(H)] for b in range(B)]
    S64 = np.array([[fs.favor_sharp_attention(Q[b, h], K[b, h], V[b, h], om, p[b][h], causal=True) for h in range(H)] for b in range(B)])
    ref = Cross(torch.from_numpy(S64), Ke, Ve, d ** -0.5, key_len)
    close(Y, ref.Y)
    rS, rK, rV = ref.grads(dY)
    close(dKe, rK)
    close(dVe, rV)
    back = np.array([[fs.favor_sharp_attention_vjp(Q[b, h], K[b, h], V[b, h], rS[b, h].numpy(), om, p[b][h], causal=True)
                      for h in range(H)] for b in range(B)])
    close(dv, back[:, :, 2])
    close(dq, rotated(torch.from_numpy(back[:, :, 0]), pos, theta, transpose=True))
    close(dk, rotated(torch.from_numpy(back[:, :, 1]), pos, theta, transpose=True))
    # a decoding step at the last position: the same row of the layer's cross attention
    step = ctx.fsharp_cross_attend(S[:, :, -1:], Ke, Ve, key_len=key_len)
    close(step, ref.Y[:, :, -1:])
    ctx.close()
