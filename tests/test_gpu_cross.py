"""Exact cross attention (fsharp_cross_attend and its backward pass) against the definition in 64 bits, element by element, with the
bounds of layer_util: sizes at the edges of tiles and pieces, shared heads, lengths and masks that leave rows without keys,
anything at all at hidden keys, every layout; graphs, streams and repeatability."""
import math

import pytest
import torch

from paper_2302_00787_b200 import binding as fb
from tests.layer_util import Cross, inside

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = fb.Context(0)
    yield c
    c.close()


def tensor(gen, B, H, L, d, dtype, store, size=1.0):
    x = (torch.randn((B, L, H, d) if store == "blhd" else (B, H, L, d), generator=gen) * size).to(dtype).cuda()
    return x.permute(0, 2, 1, 3) if store == "blhd" else x


def masks(B, Lk, kind, gen):
    key_len = key_mask = None
    if "len" in kind:
        key_len = torch.tensor([Lk, 0, Lk // 2, 1, Lk + 9, -3][:B] + [max(1, Lk - 5)] * max(0, B - 6), dtype=torch.int32).cuda()
    if "bytes" in kind:
        key_mask = (torch.rand(B, Lk, generator=gen) < 0.6).cuda()
        key_mask[-1, : Lk // 2] = False
    return key_len, key_mask


def spoil(t, seen, gen):
    """Whatever hidden keys may hold."""
    junk = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(t.dtype).min, 0.0])
    pick = junk[torch.randint(0, 5, t.shape, generator=gen)].to(t.dtype).to(t.device)
    return torch.where(seen[:, None, :, None].to(t.device), t, pick)


CASES = [
    # B, H, Hk, Lq, Lk, d, dv, mask, store
    (1, 1, 1, 1, 1, 16, 16, "", "bhld"),
    (2, 4, 2, 1, 257, 64, 64, "len", "bhld"),                  # decoding steps: two rows per key head, an empty slot
    (6, 12, 12, 1, 700, 64, 64, "len", "blhd"),
    (2, 3, 1, 1, 1111, 32, 32, "bytes", "bhld"),               # three rows
    (1, 8, 2, 1, 4099, 128, 128, "", "bhld"),                  # four rows, pieces
    (1, 4, 1, 1, 33, 16, 128, "len+bytes", "bhld"),
    (2, 2, 2, 3, 65, 128, 32, "", "blhd"),
    (3, 6, 2, 1, 100, 128, 64, "bytes", "bhld"),
    (2, 8, 1, 1, 333, 32, 128, "bytes", "bhld"),               # eight rows
    (4, 2, 2, 65, 130, 64, 64, "len", "blhd"),
    (2, 5, 5, 16, 64, 16, 32, "", "bhld"),
    (2, 1, 1, 17, 63, 32, 16, "len", "bhld"),
    (1, 4, 4, 128, 128, 128, 128, "", "bhld"),
    (1, 3, 1, 43, 700, 64, 64, "len+bytes", "bhld"),           # 129 rows of three heads
    (3, 6, 3, 200, 129, 128, 128, "len", "blhd"),
    (1, 1, 1, 300, 2500, 64, 64, "bytes", "bhld"),
    (1, 2, 1, 513, 1030, 128, 64, "bytes", "bhld"),
    (1, 2, 2, 257, 385, 64, 128, "", "blhd"),
    (2, 16, 2, 5, 1, 64, 64, "", "bhld"),                      # one key
    (1, 2, 2, 1000, 5, 64, 64, "", "bhld"),
    (2, 7, 7, 5, 200, 64, 64, "len+bytes", "blhd"),
]
NAMES = ["x".join(map(str, c[:7])) + c[7] for c in CASES]


def make(case, dtype, seed=0):
    B, H, Hk, Lq, Lk, d, dv, mask, store = case
    gen = torch.Generator().manual_seed(seed)
    Q, K, V = (tensor(gen, B, *s, dtype, store) for s in ((H, Lq, d), (Hk, Lk, d), (Hk, Lk, dv)))
    key_len, key_mask = masks(B, Lk, mask, gen)
    ref = Cross(Q, K, V, d ** -0.5 * 1.5, key_len, key_mask)
    if mask:
        K, V = spoil(K, ref.seen, gen), spoil(V, ref.seen, gen)
    dY = tensor(gen, B, H, Lq, dv, dtype, store)
    return Q, K, V, dY, {"scale": ref.scale, "key_len": key_len, "key_mask": key_mask}, ref


def check_lse(lse, ref, d):
    lse = lse.cpu().double()
    empty = ref.lse == -math.inf
    assert torch.equal(lse == -math.inf, empty)
    e = ref.score_error(d).amax(3) if ref.P.shape[3] else 0.0
    # the scores' error, the sum's (2^-20, the cubic exponential's 8.6e-5 in bf16 kernels), log2 and the factor's roundings
    bound = e + 2e-4 + 2.0 ** -22 * (1 + ref.lse.abs())
    off = (lse - ref.lse).abs()[~empty]
    assert (off <= bound[~empty]).all(), float(off.max())


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("impl", (fb.IMPL_AUTO, fb.IMPL_SIMT), ids=("auto", "simt"))
@pytest.mark.parametrize("case", CASES, ids=NAMES)
def test_forward(ctx, case, dtype, impl):
    Q, K, V, _, kw, ref = make(case, dtype)
    ctx.set_impl(impl)
    try:
        Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
        alone = ctx.fsharp_cross_attend(Q, K, V, **kw)
    finally:
        ctx.set_impl(fb.IMPL_AUTO)
    inside(Y, ref.Y, ref.bound_Y(dtype), "Y")
    check_lse(lse, ref, case[5])
    assert torch.equal(Y, alone)
    hidden = ref.lse == -math.inf
    assert (Y.cpu()[hidden] == 0).all()
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("impl", (fb.IMPL_AUTO, fb.IMPL_SIMT), ids=("auto", "simt"))
@pytest.mark.parametrize("case", CASES, ids=NAMES)
def test_backward(ctx, case, dtype, impl):
    Q, K, V, dY, kw, ref = make(case, dtype, 1)
    ctx.set_impl(impl)
    try:
        Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
        got = ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
        again = ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
    finally:
        ctx.set_impl(fb.IMPL_AUTO)
    for name, g, h, r, b, like in zip(("dQ", "dK", "dV"), got, again, ref.grads(dY), ref.bound_grads(dY, dtype), (Q, K, V)):
        inside(g, r, b, name)
        assert torch.equal(g, h) and g.stride() == torch.empty_like(like).stride()
    off = ~ref.seen[:, None].expand(-1, K.shape[1], -1)
    assert (got[1].cpu()[off] == 0).all() and (got[2].cpu()[off] == 0).all()
    assert (got[0].cpu()[ref.lse == -math.inf] == 0).all()
    assert ctx.status() == 0


def test_gradients_against_differences(ctx):
    """sum(dY Y) along a direction U, central differences with two steps and Richardson's combination (error of the fourth
    order in the step); fp32 outputs carry some 2^-22 of their size each, divided by the step 2^-5."""
    Q, K, V, dY, kw, ref = make((2, 4, 2, 33, 150, 32, 32, "len", "bhld"), F32)
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
    grads = ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
    K, V = (t.where(ref.seen[:, None, :, None].cuda(), 0.0) for t in (K, V))
    gen = torch.Generator().manual_seed(5)
    for k, (name, x, g) in enumerate(zip("QKV", (Q, K, V), grads)):
        U = torch.randn(x.shape, generator=gen).cuda()
        U /= U.norm(dim=3, keepdim=True)

        def slope(step):
            ends = []
            for s in (step, -step):
                args = [Q, K, V]
                args[k] = x + s * U
                ends.append((ctx.fsharp_cross_attend(*args, **kw).double() * dY).sum())
            return float((ends[0] - ends[1]) / (2 * step))
        got, want = (4 * slope(2.0 ** -5) - slope(2.0 ** -4)) / 3, float((g.double() * U).sum())
        size = float((g.double().abs() * U.abs()).sum())
        noise = 2.0 ** -22 * float((Y.double().abs() * dY.abs()).sum()) / 2.0 ** -5
        assert abs(got - want) <= noise + 1e-3 * size, (name, got, want, noise, size)


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
def test_no_key_at_all(ctx, dtype):
    gen = torch.Generator().manual_seed(0)
    Q, K = tensor(gen, 2, 4, 9, 64, dtype, "bhld"), tensor(gen, 2, 2, 0, 64, dtype, "bhld")
    Y, lse = ctx.fsharp_cross_attend(Q, K, K, want_lse=True)
    assert (Y == 0).all() and (lse == -math.inf).all()
    dQ, dK, dV = ctx.fsharp_cross_attend_backward(Q, K, K, Y, lse, Y + 1)
    assert (dQ == 0).all() and dK.shape == K.shape
    K = tensor(gen, 2, 2, 70, 64, dtype, "bhld")
    K[:] = math.nan
    none = torch.zeros(2, dtype=torch.int32, device="cuda")
    Y, lse = ctx.fsharp_cross_attend(Q, K, K, want_lse=True, key_len=none)
    assert (Y == 0).all() and (lse == -math.inf).all()
    grads = ctx.fsharp_cross_attend_backward(Q, K, K, Y, lse, Y + 1, key_len=none)
    assert all((g == 0).all() for g in grads)


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("Lq", (1, 150))
def test_scores_of_every_size(ctx, dtype, Lq):
    """Scores of some hundreds (weights of one key) beside rows of equal scores; scale 0."""
    gen = torch.Generator().manual_seed(3)
    Q, K, V = (tensor(gen, 1, 2, n, 64, dtype, "bhld") for n in (Lq, 300, 300))
    Q[:, 0] *= 30.0
    for scale in (1.0, 0.125, 0.0):
        ref = Cross(Q, K, V, scale)
        Y, lse = ctx.fsharp_cross_attend(Q, K, V, scale=scale, want_lse=True)
        inside(Y, ref.Y, ref.bound_Y(dtype), scale)
        check_lse(lse, ref, 64)


def test_nan_where_it_is_seen_is_not_lost(ctx):
    gen = torch.Generator().manual_seed(4)
    for Lq in (1, 140):
        for bad in (math.nan, math.inf):
            Q, K, V = (tensor(gen, 1, 1, n, 64, BF16, "bhld") for n in (Lq, 400, 400))
            for j in (0, 131, 255, 399):
                k = K.clone()
                k[0, 0, j, 7] = bad
                Y = ctx.fsharp_cross_attend(Q, k, V)
                hit = torch.ones(Lq, dtype=torch.bool) if bad != bad else (Q[0, 0, :, 7] > 0).cpu()
                assert torch.isnan(Y[0, 0].cpu()[hit]).all(), (Lq, bad, j)
                assert torch.isfinite(Y[0, 0].cpu()[~hit]).all()


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
def test_broadcast_and_strided_inputs(ctx, dtype):
    """Keys shared by the batch, queries that repeat, slices of a wider projection; gradients come as tensors of their own."""
    gen = torch.Generator().manual_seed(6)
    Q = tensor(gen, 1, 1, 1, 64, dtype, "bhld").expand(2, 4, 70, 64)
    K = tensor(gen, 1, 2, 90, 64, dtype, "bhld").expand(2, 2, 90, 64)
    wide = tensor(gen, 2, 2, 90, 256, dtype, "blhd")
    V = wide[..., 64:128]
    dY = tensor(gen, 2, 4, 70, 1, dtype, "bhld").expand(2, 4, 70, 64)
    ref = Cross(Q, K, V, 0.125)
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True)
    inside(Y, ref.Y, ref.bound_Y(dtype))
    for g, r, b in zip(ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY), ref.grads(dY), ref.bound_grads(dY, dtype)):
        inside(g, r, b)
    room = torch.full((2, 4, 72, 80), 3.0, dtype=dtype, device="cuda")
    out = room.as_strided((2, 4, 70, 64), room.stride(), 80)
    assert ctx.fsharp_cross_attend(Q, K, V, out=out) is out
    assert torch.equal(out, Y)
    room.as_strided((2, 4, 70, 64), room.stride(), 80).fill_(3.0)
    assert (room == 3.0).all()                                      # nothing beside the output was written
    shared = (torch.rand(90, generator=gen) < 0.5).cuda()
    ref = Cross(Q, K, V, 0.125, key_mask=shared)
    inside(ctx.fsharp_cross_attend(Q, K, V, key_mask=shared), ref.Y, ref.bound_Y(dtype))


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
def test_two_graphs_and_an_eager_call(ctx, dtype):
    """Two captured training steps and an eager one, each with scratch of its own, on streams of their own at the same time."""
    cases = [make((2, 4, 2, 40, 600, 64, 64, "len", "bhld"), dtype, s) for s in (0, 1, 2)]
    runs = []
    for Q, K, V, dY, kw, ref in cases[:2]:
        stream = torch.cuda.Stream()
        mine = fb.Context(0, stream)

        def step(mine=mine, Q=Q, K=K, V=V, dY=dY, kw=kw):
            Y, lse = mine.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
            return (Y,) + mine.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            want = step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
        runs.append((graph, stream, got, want, mine))
    Q, K, V, dY, kw, ref = cases[2]
    Y0 = ctx.fsharp_cross_attend(Q, K, V, **kw)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, stream, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        assert torch.equal(ctx.fsharp_cross_attend(Q, K, V, **kw), Y0)
    torch.cuda.synchronize()
    for graph, stream, got, want, mine in runs:
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    del runs


def test_piece_boundaries(ctx):
    """Lengths around the pieces of one long sequence: few units, so that keys and rows are split."""
    gen = torch.Generator().manual_seed(8)
    Q, K, V, dY = (tensor(gen, 1, 2, n, 64, BF16, "bhld") for n in (20, 3000, 3000, 20))
    for n in (0, 1, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1024, 2999, 3000):
        key_len = torch.tensor([n], dtype=torch.int32, device="cuda")
        ref = Cross(Q, K, V, 0.125, key_len)
        Y, lse = ctx.fsharp_cross_attend(Q, K, V, key_len=key_len, want_lse=True)
        inside(Y, ref.Y, ref.bound_Y(BF16), n)
        for g, r, b in zip(ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, key_len=key_len), ref.grads(dY),
                           ref.bound_grads(dY, BF16)):
            inside(g, r, b, n)
        step = Q[:, :, :1].contiguous()
        ref = Cross(step, K, V, 0.125, key_len)
        inside(ctx.fsharp_cross_attend(step, K, V, key_len=key_len), ref.Y, ref.bound_Y(BF16), n)


def test_offsets_past_32_bits(ctx):
    """Keys of one sequence that lie 2^32 elements apart in storage."""
    if torch.cuda.mem_get_info()[0] < 14 << 30:
        pytest.skip("needs 13 GB")
    gen = torch.Generator().manual_seed(9)
    L, row = 70, 1 << 26
    store = torch.empty(L * row + 64, dtype=BF16, device="cuda")
    K = store.as_strided((1, 1, L, 64), (row * L, row * L, row, 1))
    K.copy_(tensor(gen, 1, 1, L, 64, BF16, "bhld"))
    V = tensor(gen, 1, 1, L, 64, BF16, "bhld")
    for Lq in (1, 40):
        Q, dY = (tensor(gen, 1, 1, Lq, 64, BF16, "bhld") for _ in range(2))
        ref = Cross(Q, K, V, 0.125)
        Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True)
        inside(Y, ref.Y, ref.bound_Y(BF16))
        for g, r, b in zip(ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY), ref.grads(dY), ref.bound_grads(dY, BF16)):
            inside(g, r, b)


BATCHES = [
    # B, H, Hk, Lq, Lk, d: several turns of every persistent block, sequences that are sorted by length or too many for it
    (40, 8, 8, 130, 300, 64),
    (24, 8, 4, 130, 300, 128),
    (40, 12, 4, 43, 200, 32),
    (260, 2, 2, 40, 70, 64),
]


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("kind", ("", "len", "bytes", "len+bytes"), ids=("full", "len", "bytes", "both"))
@pytest.mark.parametrize("case", BATCHES, ids=["x".join(map(str, c)) for c in BATCHES])
def test_more_tiles_than_blocks(ctx, case, kind, dtype):
    B, H, Hk, Lq, Lk, d = case
    gen = torch.Generator().manual_seed(11)
    Q, K, V = (tensor(gen, B, *s, dtype, "blhd") for s in ((H, Lq, d), (Hk, Lk, d), (Hk, Lk, d)))
    key_len = key_mask = None
    if "len" in kind:
        n = torch.randint(0, Lk + 1, (B,), generator=gen)
        n[::7], n[3::11], n[-1] = 0, Lk, 1
        key_len = n.int().cuda()
    if "bytes" in kind:
        key_mask = (torch.rand(B, Lk, generator=gen) < 0.5).cuda()
        key_mask[5] = False
    kw = {"scale": d ** -0.5, "key_len": key_len, "key_mask": key_mask}
    ref = Cross(Q, K, V, d ** -0.5, key_len, key_mask)
    K, V = spoil(K, ref.seen, gen), spoil(V, ref.seen, gen)
    dY = tensor(gen, B, H, Lq, d, dtype, "blhd")
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw)
    inside(Y, ref.Y, ref.bound_Y(dtype), "Y")
    check_lse(lse, ref, d)
    got = ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)
    for name, g, r, b in zip(("dQ", "dK", "dV"), got, ref.grads(dY), ref.bound_grads(dY, dtype)):
        inside(g, r, b, name)
    off = ~ref.seen[:, None].expand(-1, Hk, -1)
    assert (got[1].cpu()[off] == 0).all() and (got[2].cpu()[off] == 0).all()
    assert all(torch.equal(a, b) for a, b in zip(got, ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY, **kw)))
    assert ctx.status() == 0


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
def test_keys_shared_by_all_heads(ctx, dtype):
    """One key head stored once and broadcast over the heads; every head's gradient is its own."""
    gen = torch.Generator().manual_seed(12)
    Q, dY = (tensor(gen, 2, 4, 150, 64, dtype, "bhld") for _ in range(2))
    K, V = (tensor(gen, 2, 1, 170, 64, dtype, "bhld").expand(2, 4, 170, 64) for _ in range(2))
    ref = Cross(Q, K, V, 0.125)
    Y, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True)
    inside(Y, ref.Y, ref.bound_Y(dtype))
    for g, r, b in zip(ctx.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY), ref.grads(dY), ref.bound_grads(dY, dtype)):
        inside(g, r, b)


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
def test_context_on_another_stream(ctx, dtype):
    """The current stream is busy: copies that a call makes of its inputs, and its scratch, belong to the context's stream."""
    gen = torch.Generator().manual_seed(13)
    Q, dY = (tensor(gen, 2, 4, 70, 64, dtype, "bhld") for _ in range(2))
    K, V = (tensor(gen, 2, 4, 900, 66, dtype, "bhld")[..., 1:65] for _ in range(2))      # rows that have to be copied
    rope = fb.make_rope(64)

    def step(c):
        Y, lse = c.fsharp_cross_attend(Q, K, V, want_lse=True)
        return (Y,) + c.fsharp_cross_attend_backward(Q, K, V, Y, lse, dY) + c.fsharp_rotate(K, V, rope)
    want = step(ctx)
    side = torch.cuda.Stream()
    mine = fb.Context(0, side)
    for c in (mine, fb.Context(0)):                                  # (the second was made on the default stream)
        c.set_stream(side)
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        got = step(c)
        side.synchronize()
        with torch.cuda.stream(side):
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()
    with torch.cuda.stream(side):                                    # and back: the default stream's context, another one current
        torch.cuda._sleep(20_000_000)
        got = step(ctx)
    torch.cuda.current_stream().synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", (F32, BF16), ids=("f32", "bf16"))
@pytest.mark.parametrize("kind", ("len", "bytes", "len+bytes"))
@pytest.mark.parametrize("Lq,Lk,d", ((20, 1500, 64), (20, 1500, 32), (270, 1237, 64), (40, 1111, 128), (100, 2001, 64)))
def test_few_rows_and_many_tiles(ctx, Lq, Lk, d, kind, dtype):
    """Blocks of up to 128 rows, whose warpgroups take the tiles in turn, over many tiles in one piece, most of a block's warps
    without rows: every tile's hidden keys are cleared in the tile itself.  The same bits in every run."""
    B, H = 20, 8                                                     # (more units than SMs: one piece each)
    gen = torch.Generator().manual_seed(14)
    Q, K, V, dY = (tensor(gen, B, H, n, d, dtype, "blhd") for n in (Lq, Lk, Lk, Lq))
    key_len = key_mask = None
    if "len" in kind:
        key_len = torch.randint(Lk // 2, Lk + 1, (B,), generator=gen).int().cuda()
    if "bytes" in kind:
        key_mask = (torch.rand(B, Lk, generator=gen) < 0.7).cuda()
    kw = {"scale": d ** -0.5, "key_len": key_len, "key_mask": key_mask}
    ref = Cross(Q, K, V, d ** -0.5, key_len, key_mask)
    K, V = spoil(K, ref.seen, gen), spoil(V, ref.seen, gen)
    runs = [ctx.fsharp_cross_attend(Q, K, V, want_lse=True, **kw) for _ in range(8)]
    inside(runs[0][0], ref.Y, ref.bound_Y(dtype), "Y")
    check_lse(runs[0][1], ref, d)
    assert all(torch.equal(Y, runs[0][0]) and torch.equal(lse, runs[0][1]) for Y, lse in runs)
    got = ctx.fsharp_cross_attend_backward(Q, K, V, *runs[0], dY, **kw)
    for name, g, r, b in zip(("dQ", "dK", "dV"), got, ref.grads(dY), ref.bound_grads(dY, dtype)):
        inside(g, r, b, name)
    assert ctx.status() == 0


@pytest.mark.parametrize("Lq,Lk,d", ((207, 31, 64), (300, 46, 64), (130, 1500, 64), (260, 700, 128), (50, 75, 32), (200, 3, 16)))
def test_log_sum_exp_of_bf16_tensors_is_an_fp32_number(ctx, Lq, Lk, d):
    """Off by the scores' error, the exponentials' 3e-6 at most, the sum's additions and the roundings of lse: nothing of bf16's."""
    gen = torch.Generator().manual_seed(15)
    Q, K, V = (tensor(gen, 2, 4, n, d, BF16, "bhld") for n in (Lq, Lk, Lk))
    ref = Cross(Q, K, V, d ** -0.5)
    _, lse = ctx.fsharp_cross_attend(Q, K, V, want_lse=True)
    bound = ref.score_error(d).amax(3) + 4e-6 + Lk * 2.0 ** -24 + 2.0 ** -22 * (1 + ref.lse.abs())
    assert ((lse.cpu().double() - ref.lse).abs() <= bound).all()
