"""Rotary positions far out: sine and cosine of positions up to 2^31 in magnitude against 64 bits of mantissa (a 53-bit frequency
alone is off by 2^-23 radians there), read from pairs (1, 0) and (0, 1) that no product rounds."""
import numpy as np
import pytest
import torch

from paper_2302_00787_b200 import binding as fb

pytestmark = pytest.mark.gpu

LD = np.longdouble
# A turn's fraction, at most 1/2, rounded to fp32: off by 2^-26 turns.  sincospif: 2 ulp of a value up to 1, each 2^-24.
BOUND = 1.02 * (2 * np.pi * 2.0 ** -26 + 2 * 2.0 ** -24)

needs_long = pytest.mark.skipif(np.finfo(LD).nmant < 63, reason="no 64-bit mantissa here")


def frequencies(rot, base, scaling="none", factor=1.0, original=0, slow=1.0, fast=32.0):
    j = np.arange(rot // 2).astype(LD)
    b = LD(base) * LD(factor) ** (LD(rot) / LD(rot - 2)) if scaling == "ntk" else LD(base)
    t = np.exp2(-np.log2(b) * 2 * j / rot)
    if scaling == "linear":
        t = t / LD(factor)
    if scaling == "parts":
        pi = LD("3.14159265358979323846264338327950288")
        keep = np.clip((LD(original) * t / (2 * pi) - LD(slow)) / (LD(fast) - LD(slow)), LD(0), LD(1))
        t = t * (keep + (1 - keep) / LD(factor))
    return t


@needs_long
@pytest.mark.parametrize("rot", (2, 24, 64))
@pytest.mark.parametrize("scaling", ({}, {"scaling": "linear", "factor": 0.25}, {"scaling": "linear", "factor": 3.0},
                                     {"scaling": "ntk", "factor": 8.0}, {"scaling": "parts", "factor": 32.0, "original": 8192}),
                         ids=lambda s: "_".join(map(str, s.values())) or "plain")
@pytest.mark.parametrize("layout", ("half", "interleaved"))
def test_sines_of_far_positions(rot, scaling, layout):
    if rot == 2 and scaling.get("scaling") == "ntk":
        pytest.skip("one pair has no such base")
    base, L, d = 500000.0, 3000, 64
    gen = torch.Generator().manual_seed(0)
    near = torch.randint(0, 1 << 31, (L,), generator=gen)
    near[:1000] = (1 << 31) - torch.arange(1000)
    near[1000:1200] = torch.arange(200)
    pos = near * torch.where(torch.rand(L, generator=gen) < 0.3, -1, 1)
    if scaling.get("factor", 1.0) < 1.0:
        pos = pos // 4                                                # (theta / factor: the same angles)
    one = torch.zeros(1, 2, L, d)
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    one[0, 0, :, a], one[0, 1, :, b] = 1.0, 1.0
    ctx = fb.Context(0)
    got, _ = ctx.fsharp_rotate(one.cuda(), None, fb.make_rope(rot, layout=layout, base=base, **scaling), pos=pos[None].cuda())
    got = got.cpu().numpy()[0]
    angle = pos.numpy().astype(LD)[:, None] * frequencies(rot, base, **scaling)
    # (reduced by the turn in the 64-bit mantissa's own pi would lose what is tested: the library's reduction of a long double is exact)
    cos, sin = np.cos(angle), np.sin(angle)
    for g, want, what in ((got[0, :, a], cos, "cos"), (got[0, :, b], sin, "sin"), (got[1, :, a], -sin, "-sin"), (got[1, :, b], cos, "cos")):
        off = np.abs(g.astype(LD) - want)
        assert off.max() <= BOUND, (what, float(off.max() * 2 ** 24), np.unravel_index(off.argmax(), off.shape))
    assert ctx.status() == 0
    ctx.close()
