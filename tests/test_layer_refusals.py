"""Arguments that fsharp_rotate and the cross attention refuse.  The library checks them before it touches the device or the
context's contents, so a blank block of memory stands in for a context here and every call must end at its check."""
import ctypes as C

import pytest
import torch

from paper_2302_00787_b200 import binding as fb

BADARG, SHAPE, ALIGN, DTYPE, NOMEM = -1, -2, -3, -4, -5
P = 1 << 20        # an aligned address that nothing reads


@pytest.fixture(scope="module")
def lib():
    import __graft_entry__ as ge
    ge.build()
    return fb.load_library()


@pytest.fixture(scope="module")
def blank():
    return C.create_string_buffer(4096)


def rotate(lib, ctx, rope=None, q=P, k=P, qo=P, ko=P, dtype=0, pos_stride=0, ctx_null=False, no_rope=False, **dims):
    r = fb.make_rope(**{**dict(rot=32), **(rope or {})}) if not isinstance(rope, fb.fsharp_rope) else rope
    dm = fb.fsharp_rotate_dims()
    for n, v in {**dict(B=1, L=4, H=2, Hk=2, d=32), **dims}.items():
        setattr(dm, n, (C.c_int64 * 3)(*v) if n.endswith("stride") else v)
    return lib.fsharp_rotate(None if ctx_null else ctx, q, k, None, pos_stride, 0, None if no_rope else C.byref(r), C.byref(dm), dtype, 0,
                             qo, ko)


def test_rotate(lib, blank):
    go = lambda **kw: rotate(lib, blank, **kw)                       # noqa: E731
    assert go(ctx_null=True) == BADARG and go(no_rope=True) == BADARG
    for bad in (dict(B=-1), dict(L=-1), dict(H=-1), dict(Hk=-1), dict(d=48), dict(d=0), dict(d=256)):
        assert go(**bad) == SHAPE, bad
    for rot in (0, 1, 3, 34, -2):
        assert go(rope=dict(rot=rot)) == SHAPE, rot
    assert go(rope=dict(rot=2, scaling="ntk", factor=2.0)) == SHAPE
    assert go(dtype=2) == DTYPE
    for bad in (dict(base=0.0), dict(base=-1.0), dict(base=float("nan")), dict(gain=float("inf")),
                dict(scaling="linear", factor=0.0), dict(scaling="parts", factor=2.0, original=0),
                dict(scaling="parts", factor=2.0, original=100, slow=4.0, fast=4.0)):
        assert go(rope=dict(rot=32, **bad)) == BADARG, bad
    r = fb.make_rope(32)
    r.layout = 2
    assert go(rope=r) == BADARG
    r.layout, r.scaling = 0, 4
    assert go(rope=r) == BADARG
    assert go(pos_stride=-1) == BADARG
    assert go(q=None) == BADARG and go(ko=None) == BADARG
    assert go(q=P + 4) == ALIGN and go(ko=P + 8) == ALIGN
    assert go(q_stride=(256, 128, 33)) == ALIGN and go(ko_stride=(-256, 128, 32)) == ALIGN
    assert go(q_stride=(256, 128, 36), dtype=1) == ALIGN             # 72 bytes
    assert go(B=0, q=None) == 0 and go(L=0, q=None) == 0 and go(H=0, Hk=0, q=None, k=None) == 0


def cross(lib, ctx, backward=False, dtype=0, scale=1.0, scratch=P, nbytes=1 << 40, null=(), move=(), ctx_null=False, **dims):
    dm = fb.fsharp_cross_dims()
    for n, v in {**dict(B=2, H=4, Hk=2, Lq=8, Lk=100, d=32, dv=64), **dims}.items():
        setattr(dm, n, (C.c_int64 * 3)(*v) if n.endswith("stride") and n != "mask_stride" else v)
    at = lambda n: None if n in null else P + (8 if n in move else 0)    # noqa: E731
    c = None if ctx_null else ctx
    if backward:
        return lib.fsharp_cross_attend_backward(c, at("q"), at("k"), at("v"), at("y"), at("lse"), at("dy"), None, None, C.byref(dm),
                                                dtype, scale, at("dq"), at("dk"), at("dv"), scratch, nbytes)
    return lib.fsharp_cross_attend(c, at("q"), at("k"), at("v"), None, None, C.byref(dm), dtype, scale, at("y"), at("lse"), scratch,
                                   nbytes)


@pytest.mark.parametrize("backward", (False, True))
def test_cross(lib, blank, backward):
    go = lambda **kw: cross(lib, blank, backward, **kw)              # noqa: E731
    assert go(ctx_null=True) == BADARG
    for bad in (dict(B=-1), dict(H=3), dict(Hk=0), dict(Lq=-1), dict(Lk=-1), dict(d=48), dict(dv=8), dict(B=70000, Hk=1, H=1),
                dict(Lq=0x7fffffff), dict(Lk=0x7fffffff)):
        assert go(**bad) == SHAPE, bad
    assert go(dtype=2) == DTYPE
    for s in (-1.0, float("nan"), float("inf")):
        assert go(scale=s) == BADARG
    assert go(mask_stride=-1) == BADARG
    for n in ("q", "k", "v", "y") + (("dy", "dq", "dk", "dv") if backward else ()):
        assert go(null=(n,)) == BADARG, n
        assert go(move=(n,)) == ALIGN, n
        assert go(**{n + "_stride": (6400, 3200, 33)}) == ALIGN, n
    for n in ("k", "v") + (("q", "dy") if backward else ()):
        assert go(**{n + "_stride": (6400, 3200, 0)}) == SHAPE
    if backward:
        assert go(null=("lse",)) == BADARG
        assert go(scratch=None) == BADARG and go(scratch=P + 4) == ALIGN and go(nbytes=16) == NOMEM
        assert go(Lq=0) == SHAPE
    assert go(B=0, null=("q",)) == 0 and go(H=0, Hk=0, null=("q",)) == 0
    assert go(Lq=0, Lk=0 if backward else 100, null=("q",)) == 0


def test_cross_scratch(lib, blank):
    dm = fb.fsharp_cross_dims()
    dm.B, dm.H, dm.Hk, dm.Lq, dm.Lk, dm.d, dm.dv = 2, 4, 2, 8, 100, 32, 64
    assert lib.fsharp_cross_scratch_bytes(None, C.byref(dm), 0, 0) == BADARG
    assert lib.fsharp_cross_scratch_bytes(blank, None, 0, 0) == BADARG
    assert lib.fsharp_cross_scratch_bytes(blank, C.byref(dm), 7, 0) == DTYPE
    assert lib.fsharp_cross_scratch_bytes(blank, C.byref(dm), 0, 1) >= 2 * 4 * 8 * 8
    dm.Lq = 0
    assert lib.fsharp_cross_scratch_bytes(blank, C.byref(dm), 0, 1) == 0


def test_binding_refuses_what_the_kernels_would_overrun(lib, blank):
    ctx = object.__new__(fb.Context)
    ctx.lib, ctx.device, ctx._h = lib, 0, C.c_void_p()
    x = torch.zeros(2, 4, 8, 32)
    with pytest.raises(ValueError):                                   # not on the context's device
        ctx.fsharp_rotate(x, x, fb.make_rope(32))
    with pytest.raises(ValueError):
        ctx.fsharp_cross_attend(x, x, x)
    ctx._mine = lambda **named: None                                  # (what stands behind the check of the device)
    with pytest.raises(ValueError):
        ctx.fsharp_rotate(x, x[:, :, :4], fb.make_rope(32))
    with pytest.raises(ValueError):
        ctx.fsharp_rotate(x, x.bfloat16(), fb.make_rope(32))
    with pytest.raises(ValueError):
        ctx.fsharp_rotate(x, None, fb.make_rope(32), pos=torch.zeros(2, 8, dtype=torch.int32))
    with pytest.raises(ValueError):
        ctx.fsharp_rotate(x, None, fb.make_rope(32), pos=torch.zeros(2, 7, dtype=torch.int64))
    with pytest.raises(ValueError):
        ctx.fsharp_rotate(x, None, fb.make_rope(32), out=(x[:, :2], None))
    for k, v in ((x[:1], x[:1]), (x, x[:, :, :4]), (x[..., :16], x), (x.bfloat16(), x)):
        with pytest.raises(ValueError):
            ctx.fsharp_cross_attend(x, k, v)
    for kw in (dict(key_len=torch.zeros(2, dtype=torch.int64)), dict(key_len=torch.zeros(3, dtype=torch.int32)),
               dict(key_mask=torch.zeros(2, 7, dtype=torch.bool)), dict(key_mask=torch.zeros(2, 8)),
               dict(out=x[:, :2]), dict(out=x[:, :1].expand(2, 4, 8, 32))):
        with pytest.raises(ValueError):
            ctx.fsharp_cross_attend(x, x, x, **kw)
    with pytest.raises(TypeError):
        ctx.fsharp_cross_attend(x.double(), x.double(), x.double())
    lse = torch.zeros(2, 4, 8)
    for y, s, g in ((x[:, :2], lse, x), (x, lse[:1], x), (x, lse.double(), x), (x, lse, x[..., :16])):
        with pytest.raises(ValueError):
            ctx.fsharp_cross_attend_backward(x, x, x, y, s, g)


def test_no_query_with_keys_has_no_gradient(lib, blank):
    """dK and dV would have to be written: the call must not report success and leave them as they were."""
    assert cross(lib, blank, True, H=0) == SHAPE and cross(lib, blank, True, Lq=0) == SHAPE
    assert cross(lib, blank, True, H=0, Lk=0) == 0 and cross(lib, blank, False, H=0) == 0


def test_rotation_into_the_other_tensor(lib, blank):
    for at in (dict(qo=2 * P, ko=P, q=P, k=2 * P), dict(qo=2 * P, ko=3 * P, q=P, k=2 * P), dict(qo=3 * P, ko=P, q=P, k=2 * P),
               dict(qo=3 * P, ko=3 * P, q=P, k=2 * P)):
        assert rotate(lib, blank, **at) == BADARG, at
