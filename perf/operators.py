"""Performance cases of what a decoder layer needs next to FAVOR# attention: rotary positions on queries and keys, and
exact softmax cross attention to an encoder's states of another length, for training, prompts and single tokens.

A case is a plain dict.  `kind` says which calls one pass makes:

  rotate   rotary positions on Q and K in one call (transpose: the gradient, the rotation by the negative angle)
  attend   cross attention, forward (Lq = 1: a decoding step)
  train    cross attention forward with the rows' log-sum-exp, then its backward pass for a cotangent dY

Head sizes and counts are those of the package's workloads (8, 12, 16 heads; d = 32, 64, 128), lengths theirs and ragged
ones around them.  `store` "blhd" is what a projection layer hands over: [B, L, H, d] storage seen as [B, H, L, d].
`mask` "len" gives every sequence a length of its own (padding behind it; one slot of a larger batch is empty), "bytes"
a mask with a quarter of the keys hidden anywhere.
"""
import functools
import math

import torch

own = False          # False: the plain forms below; True: the library's calls


def _rotate(name, B, H, Hk, L, d, dtype, rot=None, layout="half", scaling="none", base=10000.0, factor=1.0, original=0,
            gain=1.0, far=0, store="bhld", transpose=False):
    c = {"kind": "rotate", "B": B, "H": H, "Hk": Hk, "L": L, "d": d, "dtype": dtype, "rot": rot or d, "layout": layout,
         "scaling": scaling, "base": base, "factor": factor, "original": original, "gain": gain, "far": far, "store": store,
         "transpose": transpose}
    return dict(c, name=name) if name else c


def _cross(name, kind, B, H, Lq, Lk, d, dtype, Hk=None, dv=None, mask="none", store="bhld"):
    c = {"kind": kind, "B": B, "H": H, "Hk": Hk or H, "Lq": Lq, "Lk": Lk, "d": d, "dv": dv or d, "dtype": dtype, "mask": mask,
         "store": store}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of a batch of 64 sequences, each at a position of its own: latency
        _rotate("rotate_step_bf16", 64, 12, 12, 1, 64, "bf16", far=8000),
        # queries and keys of the causal 8192-token layer as its projection hands them over
        _rotate("rotate_layer_bf16", 4, 12, 12, 8192, 64, "bf16", store="blhd"),
        # one very long document, wide heads, half of each head rotated, frequencies scaled by parts beyond the trained length
        _rotate("rotate_long_bf16", 1, 16, 4, 65536, 128, "bf16", rot=64, layout="interleaved", scaling="parts", factor=8.0,
                original=8192, gain=0.1 * math.log(8.0) + 1.0, far=1 << 20),
        # the gradient on its way back through the positions of a small fp32 encoder
        _rotate("rotate_grad_f32", 4, 8, 8, 1501, 32, "f32", transpose=True),
        # one decoding step of one sequence against a short encoding: the smallest call
        _cross("step_small_bf16", "attend", 1, 8, 1, 512, 64, "bf16"),
        # one decoding step of a batch of 64 sequences with 1500 frames at most, ragged
        _cross("step_ragged_bf16", "attend", 64, 12, 1, 1500, 64, "bf16", mask="len"),
        # one decoding step against long encodings, wide heads that share keys and values
        _cross("step_long_gqa_bf16", "attend", 16, 16, 1, 16384, 128, "bf16", Hk=4, mask="len"),
        # a decoder's 4096 tokens against 8192 encoder states
        _cross("prompt_8k_bf16", "attend", 4, 12, 4096, 8192, 64, "bf16", store="blhd"),
        # wide shared heads, keys hidden by a byte mask, ragged lengths
        _cross("prompt_gqa_mask_bf16", "attend", 1, 16, 2049, 10007, 128, "bf16", Hk=4, mask="bytes"),
        # a training step of an encoder-decoder of 12 heads on a padded batch
        _cross("train_bf16", "train", 16, 12, 512, 1500, 64, "bf16", mask="len", store="blhd"),
        # a training step with wide shared heads and longer sequences
        _cross("train_gqa_d128_bf16", "train", 2, 16, 2048, 4096, 128, "bf16", Hk=8),
        # fp32 training of a small encoder-decoder (ragged, narrow heads)
        _cross("train_f32", "train", 4, 8, 701, 1501, 32, "f32", mask="len"),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, at most about half of the largest listed case's work."""
    while True:
        kind = rng.choice(["rotate"] * 3 + ["step"] * 3 + ["attend"] * 3 + ["train"] * 3)
        d, dtype, store = rng.choice([16, 32, 64, 64, 128]), rng.choice(["bf16", "bf16", "f32"]), rng.choice(["bhld", "blhd"])
        Hk, g, B = rng.choice([1, 2, 4, 8, 12]), rng.choice([1, 1, 2, 3, 4, 8]), _logint(rng, 1, 64)
        if kind == "rotate":
            step = rng.random() < 0.3
            scaling = rng.choice(["none", "none", "linear", "ntk", "parts"])
            c = _rotate(None, B, Hk * g, Hk, 1 if step else _logint(rng, 2, 65536), d, dtype,
                        rng.choice([d, d, d // 2, 2 * rng.randint(2, d // 2)]), rng.choice(["half", "interleaved"]), scaling,
                        rng.choice([10000.0, 500000.0]), 1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                        rng.choice([2048, 8192]), rng.choice([1.0, 1.0, 1.2]), rng.choice([0, 1 << 13, 1 << 20]), store,
                        rng.random() < 0.4)
        else:
            Lq = 1 if kind == "step" else _logint(rng, 1, 8192)
            least = 16 if kind == "train" else 1     # (the scores' gradient of a row that sees one key is zero: nothing to compare)
            c = _cross(None, "train" if kind == "train" else "attend", B, Hk * g, Lq, _logint(rng, least, 32768), d, dtype, Hk,
                       d if rng.random() < 0.7 else rng.choice([16, 32, 64, 128]), rng.choice(["none", "len", "len", "bytes"]), store)
        w = work(c)
        scores = 0 if kind == "rotate" else c["B"] * c["H"] * c["Lq"] * c["Lk"]
        if w["flops"] <= 2.5e11 and w["bytes"] <= 5e8 and scores <= 1e9 and w["bytes"] > 0:
            return c


# ---- inputs ----------------------------------------------------------------------------------------------------

def _tensor(c, gen, H, L, width):
    B = c["B"]
    shape = (B, L, H, width) if c["store"] == "blhd" else (B, H, L, width)
    x = torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16 if c["dtype"] == "bf16" else torch.float32)
    return x.permute(0, 2, 1, 3) if c["store"] == "blhd" else x


def _lengths(c):
    """The visible keys of the batch's sequences, in no order: the same numbers for every seed."""
    B, Lk = c["B"], c["Lk"]
    if c["mask"] == "none":
        return [Lk] * B
    if c["mask"] == "bytes":
        return [max(1, Lk - Lk // 4)] * B
    got = [max(1, Lk - (Lk - Lk // 4) * i // max(1, B - 1)) for i in range(B)]
    if B >= 8:
        got[-1] = 0
    return got


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if c["kind"] == "rotate":
        s = {"c": c, "Q": _tensor(c, gen, c["H"], c["L"], c["d"]), "K": _tensor(c, gen, c["Hk"], c["L"], c["d"]), "pos": None}
        if c["far"]:      # each sequence continues from a place of its own
            start = torch.randint(0, c["far"], (c["B"], 1), generator=gen, device="cuda")
            s["pos"] = start + torch.arange(c["L"], device="cuda")
        return s
    s = {"c": c, "Q": _tensor(c, gen, c["H"], c["Lq"], c["d"]), "K": _tensor(c, gen, c["Hk"], c["Lk"], c["d"]),
         "V": _tensor(c, gen, c["Hk"], c["Lk"], c["dv"]), "scale": c["d"] ** -0.5, "len": None, "mask": None}
    if c["mask"] == "len":
        n = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
        s["len"] = n[torch.randperm(c["B"], generator=gen, device="cuda")].contiguous()
    elif c["mask"] == "bytes":
        order = torch.rand(c["B"], c["Lk"], generator=gen, device="cuda").argsort(1).argsort(1)
        s["mask"] = order < _lengths(c)[0]
    if c["kind"] == "train":
        s["dY"] = _tensor(c, gen, c["H"], c["Lq"], c["dv"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

@functools.lru_cache(maxsize=None)
def _library():
    """The binding, and the one context that a program keeps."""
    from paper_2302_00787_b200 import binding as fb
    return fb, fb.Context(0)


def _own_pass(s):
    c = s["c"]
    fb, ctx = _library()
    if c["kind"] == "rotate":
        rope = fb.make_rope(c["rot"], layout=c["layout"], base=c["base"], scaling=c["scaling"], factor=c["factor"],
                            original=c["original"], gain=c["gain"])
        return ctx.fsharp_rotate(s["Q"], s["K"], rope, pos=s["pos"], transpose=c["transpose"])
    at = {"scale": s["scale"], "key_len": s["len"], "key_mask": s["mask"]}
    if c["kind"] == "attend":
        return ctx.fsharp_cross_attend(s["Q"], s["K"], s["V"], **at)
    Y, lse = ctx.fsharp_cross_attend(s["Q"], s["K"], s["V"], want_lse=True, **at)
    return (Y, lse) + ctx.fsharp_cross_attend_backward(s["Q"], s["K"], s["V"], Y, lse, s["dY"], **at)


def _frequencies(c):
    """Radians per position of the head's pairs, in 64 bits."""
    rot, s = c["rot"], c["factor"]
    base = c["base"]
    if c["scaling"] == "ntk":
        base *= s ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if c["scaling"] == "linear":
        f = f / s
    if c["scaling"] == "parts":      # pairs with under one turn in the trained length are stretched, with over 32 turns kept
        keep = ((c["original"] * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        f = f / s * (1 - keep) + f * keep
    return f


def _plain_rotate(s):
    c, rot = s["c"], s["c"]["rot"]
    pos = torch.arange(c["L"], device="cuda")[None] if s["pos"] is None else s["pos"]
    angle = pos[:, None, :, None].double() * _frequencies(c)
    cos, sin = (c["gain"] * angle.cos()).float(), (c["gain"] * angle.sin()).float()
    if c["transpose"]:
        sin = -sin

    def turned(X):
        x = X.float()
        if c["layout"] == "half":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        else:
            a, b = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([y, x[..., rot:]], -1).to(X.dtype)
    return turned(s["Q"]), turned(s["K"])


def _plain_pass(s):
    c = s["c"]
    if c["kind"] == "rotate":
        return _plain_rotate(s)
    B, H, Hk, Lq, Lk, dv, dt = c["B"], c["H"], c["Hk"], c["Lq"], c["Lk"], c["dv"], s["Q"].dtype
    q = s["Q"].float().reshape(B, Hk, -1, c["d"])                  # the rows of the heads that share keys, one after the other
    k, v = s["K"].float(), s["V"].float()
    S = (q * s["scale"]) @ k.transpose(2, 3)
    if s["len"] is not None or s["mask"] is not None:
        seen = s["mask"] if s["mask"] is not None else torch.arange(Lk, device="cuda") < s["len"][:, None]
        S.masked_fill_(~seen[:, None, None], -math.inf)
    top = S.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)                  # a row that sees nothing: all its exponentials are zero
    P = (S - top).exp_()
    total = P.sum(3, keepdim=True)
    some = total > 0
    P = P / torch.where(some, total, 1.0)
    y = P @ v
    Y = y.to(dt).reshape(B, H, Lq, dv)
    if c["kind"] == "attend":
        return Y
    lse = torch.where(some, top + total.log(), -math.inf).reshape(B, H, Lq)
    g = s["dY"].float().reshape(B, Hk, -1, dv)
    dV = P.transpose(2, 3) @ g
    dS = P * (g @ v.transpose(2, 3) - (g * y).sum(3, keepdim=True)) * s["scale"]
    dQ, dK = dS @ k, dS.transpose(2, 3) @ q
    return Y, lse, dQ.to(dt).reshape(B, H, Lq, c["d"]), dK.to(dt), dV.to(dt)


def run(state):
    return _own_pass(state) if own else _plain_pass(state)


# ---- the same from the definition, in 64 bits ----------------------------------------------------------------------

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rotate":
        j = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
        stretch = torch.full_like(j, c["factor"])
        theta = torch.exp(-2.0 * j / c["rot"] * math.log(c["base"]))
        if c["scaling"] == "none":
            stretch = torch.ones_like(j)
        if c["scaling"] == "ntk":                                  # a larger base is a stretch that grows with the pair's number
            stretch = c["factor"] ** (2.0 * j / (c["rot"] - 2))
        if c["scaling"] == "parts":
            turns = c["original"] * theta / (2 * math.pi)
            keep = torch.clamp((turns - 1.0) / (32.0 - 1.0), min=0.0, max=1.0)
            stretch = 1.0 / (keep + (1.0 - keep) / c["factor"])
        p = s["pos"] if s["pos"] is not None else torch.arange(c["L"], device="cuda").expand(c["B"], -1)
        angle = p.double()[:, :, None] * (theta / stretch) * (-1.0 if c["transpose"] else 1.0)
        z = torch.polar(torch.full_like(angle, c["gain"]), angle)[:, None]
        out = []
        for X in (s["Q"], s["K"]):
            y = X.double().contiguous()
            n = c["rot"]
            first, second = (slice(0, n // 2), slice(n // 2, n)) if c["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
            t = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * z
            y[..., first], y[..., second] = t.real, t.imag
            out.append(y)
        return tuple(out)
    g, train = c["H"] // c["Hk"], c["kind"] == "train"
    shape = (c["B"], c["H"], c["Lq"])
    Y = torch.zeros(*shape, c["dv"], dtype=torch.float64, device="cuda")
    lse = torch.full(shape, -math.inf, dtype=torch.float64, device="cuda")
    grads = [torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("Q", "K", "V")]
    for b in range(c["B"]):
        see = torch.arange(c["Lk"], device="cuda")                 # the keys that this sequence has, and no others
        if s["len"] is not None:
            see = see[:int(s["len"][b])]
        if s["mask"] is not None:
            see = see[s["mask"][b]]
        if not len(see):
            continue
        for h in range(c["Hk"]):
            of = slice(h * g, (h + 1) * g)
            q, k, v = (t.double().detach().requires_grad_(train) for t in (s["Q"][b, of], s["K"][b, h, see], s["V"][b, h, see]))
            logits = torch.einsum("hid,jd->hij", q, k) * s["scale"]
            total = torch.logsumexp(logits, 2)
            y = torch.einsum("hij,jd->hid", (logits - total[..., None]).exp(), v)
            Y[b, of], lse[b, of] = y.detach(), total.detach()
            if train:
                for into, at, grad in zip(grads, ((b, of), (b, h, see), (b, h, see)),
                                          torch.autograd.grad((y * s["dY"][b, of].double()).sum(), (q, k, v))):
                    into[at] = grad
    return (Y, lse, *grads) if train else Y


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    B, H, Hk, d = c["B"], c["H"], c["Hk"], c["d"]
    if c["kind"] == "rotate":
        rows = B * (H + Hk) * c["L"]
        return {"bytes": 2 * rows * d * e + (8 * B * c["L"] if c["far"] else 0), "flops": 3 * rows * c["rot"]}
    dv, Lq, Lk = c["dv"], c["Lq"], c["Lk"]
    keys = sum(_lengths(c))                                        # those that are seen: the others need not be read
    pairs = H * Lq * keys
    read = e * (B * H * Lq * d + Hk * keys * (d + dv)) + (4 * B if c["mask"] == "len" else B * Lk if c["mask"] == "bytes" else 0)
    wrote = e * B * H * Lq * dv
    flops = 2 * pairs * (d + dv)                                   # q k, p v
    if c["kind"] == "train":                                       # the log-sum-exp and dY; dQ, dK, dV whole
        read += e * B * H * Lq * dv
        wrote += 4 * B * H * Lq + e * (B * H * Lq * d + B * Hk * Lk * (d + dv))
        flops += 2 * pairs * (3 * d + 2 * dv)                      # q k again, dy v, p dy, ds k, ds q
    return {"bytes": read + wrote, "flops": flops}
