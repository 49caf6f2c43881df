"""Layouts of Q, K, V, Y and dY that a forward call of the exact cross attention takes: the backward call takes them too, and writes its
gradients to places that the library can address."""
import ctypes as C

import pytest
import torch

from paper_2302_00787_b200 import binding as fb
from tests.layer_util import Cross, inside

F32, BF16 = torch.float32, torch.bfloat16

# How [B,H,L,d] values may lie in storage
LAYOUTS = {
    "dense": lambda x: x,
    "transposed": lambda x: x.transpose(2, 3).contiguous().transpose(2, 3),                  # [B,H,d,L], a cache of transposed keys
    "tokens_last": lambda x: x.permute(0, 3, 1, 2).contiguous().permute(0, 2, 3, 1),         # [B,d,H,L]
    "batch_last": lambda x: x.permute(1, 2, 3, 0).contiguous().permute(3, 0, 1, 2),          # [H,L,d,B]
    "tokens_first": lambda x: x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3),        # [L,B,H,d]
    "slice_of_transposed": lambda x: torch.cat([x, x], 3).transpose(2, 3).contiguous().transpose(2, 3)[..., : x.shape[3]],
    "every_second": lambda x: torch.stack([x, x], 4).flatten(3)[..., ::2],
    "one_for_all": lambda x: x[..., :1].expand(x.shape),                                     # last dimension of stride zero
}


class Recorder:
    """In the library's place: takes the sizes and strides of a call and answers success."""

    def fsharp_cross_scratch_bytes(self, *_):
        return 0

    def fsharp_cross_attend_backward(self, *args):
        self.dims = fb._CROSS_DIMS.unpack(args[9])
        self.written = args[12:15]
        return 0


def backward_on_cpu(ctx, Q, K, V, Y, lse, dY, **kw):
    """The call on tensors that are on no device that the context could check."""
    real = torch.Tensor.get_device
    torch.Tensor.get_device = lambda self: ctx.device if not self.is_cuda else real(self)
    try:
        return ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
    finally:
        torch.Tensor.get_device = real


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("name", LAYOUTS)
def test_gradients_have_places_that_the_library_takes(name, dtype):
    ctx = object.__new__(fb.Context)
    ctx.lib, ctx.device, ctx._h = Recorder(), 0, C.c_void_p()
    ctx._mine = lambda **named: None
    ctx._stream = None
    B, H, Hk, Lq, Lk, d, dv = 2, 6, 3, 5, 10, 16, 32
    lay = LAYOUTS[name]
    Q, K, V = lay(torch.zeros(B, H, Lq, d, dtype=dtype)), lay(torch.zeros(B, Hk, Lk, d, dtype=dtype)), lay(torch.zeros(B, Hk, Lk, dv, dtype=dtype))
    Y = lay(torch.zeros(B, H, Lq, dv, dtype=dtype))
    got = backward_on_cpu(ctx, Q, K, V, Y, torch.zeros(B, H, Lq), Y)
    strides = ctx.lib.dims[7:]
    for g, x, at, s in zip(got, (Q, K, V), ctx.lib.written, (strides[15:18], strides[18:21], strides[21:24])):
        assert g.shape == x.shape and g.dtype == x.dtype and g.data_ptr() == at
        assert g.stride() == (*s, 1)
        assert all(n * g.element_size() % 16 == 0 for n in s)
        # a place for every value
        at = sum(torch.arange(n).view([-1 if k == i else 1 for k in range(4)]) * g.stride(i) for i, n in enumerate(g.shape))
        assert at.unique().numel() == g.numel()
    if name in ("dense", "tokens_first"):
        assert all(g.stride() == x.stride() for g, x in zip(got, (Q, K, V)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("name", LAYOUTS)
def test_there_and_back(name, dtype):
    B, H, Hk, Lq, Lk, d, dv = 2, 6, 3, 33, 90, 64, 32
    gen = torch.Generator().manual_seed(2)
    lay = LAYOUTS[name]
    Q, K, V, dY = (lay(torch.randn(B, *s, generator=gen).to(dtype).cuda()) for s in ((H, Lq, d), (Hk, Lk, d), (Hk, Lk, dv), (H, Lq, dv)))
    key_len = torch.tensor([Lk, 41], dtype=torch.int32).cuda()
    ctx = fb.Context(0)
    ref = Cross(Q, K, V, d ** -0.5, key_len)
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, key_len=key_len, want_lse=True)
    inside(Y, ref.Y, ref.bound_Y(dtype), "Y")
    got = ctx.fsharp_cross_attend_backward(Q, K, V, lay(Y) if name != "one_for_all" else Y, lse, dY, key_len=key_len)
    for what, g, r, b in zip(("dQ", "dK", "dV"), got, ref.grads(dY), ref.bound_grads(dY, dtype)):
        inside(g, r, b, what)
    assert ctx.status() == 0
    ctx.close()
