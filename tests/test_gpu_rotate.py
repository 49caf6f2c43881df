"""Rotary positions (fsharp_rotate) against the definition in 64 bits, element by element: an output is a rounded sum of
two products whose sine and cosine are fp32 values of an angle that is off by 2^-24 turns at most."""
import math

import pytest
import torch

from paper_2302_00787_b200 import binding as fb
from tests.layer_util import HALF_STEP, frequencies, rotated

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    c.close()


def tensors(B, H, Hk, L, d, dtype, store, seed=0):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for h in (H, Hk):
        x = torch.randn((B, L, h, d) if store == "blhd" else (B, h, L, d), generator=gen).to(dtype).cuda()
        out.append(x.permute(0, 2, 1, 3) if store == "blhd" else x)
    return out


def check(got, X, pos, theta, layout, gain, transpose):
    rot, dt = 2 * len(theta), X.dtype
    ref = rotated(X, pos.to(X.device), theta, layout, gain, transpose)
    x = X.double()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    size = abs(gain) * (x[..., a].abs() + x[..., b].abs())
    # sine and cosine: 2^-24 turns of angle (4e-7), 2 ulp of their own and the gain's product (3 half steps); products and sum
    off = size * (2 * math.pi * 2.0 ** -24 + 8 * 2.0 ** -24)
    for part in (a, b):
        bound = off + HALF_STEP[dt] * (ref[..., part].abs() + off) + 1e-38
        assert ((got.double()[..., part] - ref[..., part]).abs() <= bound).all()
    assert torch.equal(got[..., rot:], X[..., rot:])


CASES = [
    # B, H, Hk, L, d, rot, layout, dtype, store, scaling, far, gain, transpose
    (1, 1, 1, 1, 16, 2, "half", "f32", "bhld", {}, 0, 1.0, False),
    (2, 3, 1, 5, 16, 16, "interleaved", "bf16", "bhld", {}, 100, 1.0, False),
    (3, 4, 2, 37, 32, 20, "half", "bf16", "blhd", {}, 5000, 1.0, False),            # halves of 10: 4-byte vectors
    (3, 4, 2, 37, 32, 18, "half", "bf16", "blhd", {}, 5000, 1.0, True),             # halves of 9: single values
    (2, 12, 12, 129, 64, 64, "half", "bf16", "blhd", {}, 1 << 20, 1.0, False),
    (2, 9, 3, 63, 64, 24, "interleaved", "bf16", "blhd", {"scaling": "linear", "factor": 4.0}, 1 << 20, 1.0, True),
    (1, 16, 4, 300, 128, 64, "interleaved", "bf16", "bhld",
     {"scaling": "parts", "factor": 8.0, "original": 8192}, 1 << 20, 1.2079, False),
    (1, 5, 5, 77, 128, 128, "half", "f32", "blhd", {"scaling": "parts", "factor": 32.0, "original": 2048, "slow": 1.0,
                                                    "fast": 4.0}, (1 << 31) - 100, 1.0, False),
    (2, 3, 2, 41, 64, 48, "half", "f32", "bhld", {"scaling": "ntk", "factor": 8.0}, 100000, 0.9, True),
    (2, 3, 2, 41, 64, 10, "half", "f32", "bhld", {}, 100000, 1.0, True),            # halves of 5
    (64, 12, 12, 1, 64, 64, "half", "bf16", "bhld", {}, 8000, 1.0, False),          # a decoding step
    (1, 1, 1, 40001, 16, 12, "interleaved", "f32", "bhld", {}, 0, 1.0, False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[5]}of{c[4]}_{c[6]}_{c[7]}_{c[3]}")
def test_against_definition(ctx, case):
    B, H, Hk, L, d, rot, layout, dtype, store, scaling, far, gain, transpose = case
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    Q, K = tensors(B, H, Hk, L, d, dt, store)
    base = 500000.0 if far > 1 << 19 else 10000.0
    rope = fb.make_rope(rot, layout=layout, base=base, gain=gain, **scaling)
    theta = frequencies(rot, base, **scaling)
    pos = torch.arange(L)[None].repeat(B, 1)
    if far:
        pos = pos + torch.randint(0, far, (B, 1), generator=torch.Generator().manual_seed(1))
    Qo, Ko = ctx.fsharp_rotate(Q, K, rope, pos=pos.cuda() if far else None, transpose=transpose)
    check(Qo, Q, pos, theta, layout, gain, transpose)
    check(Ko, K, pos, theta, layout, gain, transpose)
    assert ctx.status() == 0


def test_positions_in_every_form(ctx):
    Q, K = tensors(3, 2, 2, 9, 32, torch.float32, "bhld")
    rope, theta = fb.make_rope(32), frequencies(32)
    shared = torch.tensor([5, 0, 7, -3, 1 << 20, 2, 2, 11, 40])
    for pos, pos0 in ((None, 0), (None, 17), (shared, 0), (shared, -2), (shared + torch.arange(3)[:, None], 4)):
        got, _ = ctx.fsharp_rotate(Q, K, rope, pos=None if pos is None else pos.cuda(), pos0=pos0)
        at = (torch.arange(9) if pos is None else pos).expand(3, 9) + pos0
        check(got, Q, at, theta, "half", 1.0, False)


def test_in_place_and_transpose_undoes(ctx):
    Q, K = tensors(2, 4, 2, 100, 64, torch.float32, "blhd")
    q, k = Q.clone(memory_format=torch.preserve_format), K.clone(memory_format=torch.preserve_format)
    rope = fb.make_rope(32, layout="interleaved")
    want = ctx.fsharp_rotate(Q, K, rope, pos0=1000)
    got = ctx.fsharp_rotate(q, k, rope, pos0=1000, out=(q, k))
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1])
    ctx.fsharp_rotate(q, k, rope, pos0=1000, transpose=True, out=(q, k))
    assert (q - Q).abs().max() < 4e-6 and (k - K).abs().max() < 4e-6


def test_features_that_pass_keep_their_bits(ctx):
    X = torch.full((1, 2, 8, 64), float("nan"), device="cuda", dtype=torch.bfloat16)
    X[..., :16] = 1.0
    X[..., 20], X[..., 21] = float("inf"), -0.0
    for layout in ("half", "interleaved"):
        got, none = ctx.fsharp_rotate(X, None, fb.make_rope(16, layout=layout))
        assert none is None
        assert torch.equal(got[..., 16:].view(torch.int16), X[..., 16:].view(torch.int16))
        assert torch.isfinite(got[..., :16]).all()


def test_nothing_is_written_beside_the_output(ctx):
    Q, _ = tensors(2, 3, 1, 21, 32, torch.bfloat16, "bhld")
    room = torch.full((2, 3, 23, 48), 7.0, device="cuda", dtype=torch.bfloat16)
    out = room[:, :, 1:22, :32]
    out = room.as_strided((2, 3, 21, 32), room.stride(), 8)        # a start that is 16 bytes in
    ctx.fsharp_rotate(Q, None, fb.make_rope(20), out=(out, None))
    check(out, Q, torch.arange(21).expand(2, 21), frequencies(20), "half", 1.0, False)
    left = torch.ones_like(room, dtype=torch.bool)
    left.as_strided((2, 3, 21, 32), room.stride(), 8).fill_(False)
    assert (room[left] == 7.0).all()


def test_broadcast_and_unaligned_inputs(ctx):
    one = torch.randn(32, device="cuda")
    X = one.expand(2, 3, 5, 32)                                    # three zero strides: not a dense tensor
    got, _ = ctx.fsharp_rotate(X, None, fb.make_rope(32))
    check(got, X, torch.arange(5).expand(2, 5), frequencies(32), "half", 1.0, False)
    Y = torch.randn(2, 3, 5, 33, device="cuda")[..., 1:]           # rows that start anywhere
    got, _ = ctx.fsharp_rotate(Y, None, fb.make_rope(32))
    check(got, Y, torch.arange(5).expand(2, 5), frequencies(32), "half", 1.0, False)
    with pytest.raises(ValueError):
        ctx.fsharp_rotate(X, None, fb.make_rope(32), out=(X, None))


def test_captured_and_replayed(ctx):
    Q, K = tensors(4, 8, 8, 1, 64, torch.bfloat16, "bhld")
    pos = torch.arange(4, device="cuda")[:, None] * 100
    rope, out = fb.make_rope(64), (torch.empty_like(Q), torch.empty_like(K))
    stream = torch.cuda.Stream()
    mine = fb.Context(0, stream)
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        mine.fsharp_rotate(Q, K, rope, pos=pos, out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        mine.fsharp_rotate(Q, K, rope, pos=pos, out=out)
    for step in range(3):
        pos.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        check(out[0], Q, pos.cpu(), frequencies(64), "half", 1.0, False)
    mine.close()
