"""Performance cases of the operators around the hybrid attention: what stands before it, behind it and behind its
gradient in a distillation step or in generation.

  rope   rotary positions of queries and keys, and their gradient (the inverse rotation)
  loss   the distillation loss sum w |y_hat - y| and its gradient
  adamw  one AdamW step over all feature-map parameters, moments in 32 or in 8 bits

With `own` false a case runs in elementary torch operations, otherwise through the library's binding.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}

# name: what it stands for
_LISTED = [
    # queries and keys of one layer at 480x832 (21 x 30 x 52 latent), as the projections leave them (token-major), into
    # the head-major operands of the attention
    dict(name="rope_480p", op="rope", dtype="bf16", layout="interleaved", B=1, N=32760, Hq=12, Hk=12, d=128, rot=128,
         axes=3, rows=30, cols=52, start=0, inverse=False, token_major=True, scaling="none", factor=1.0),
    # the gradient of the same for a guidance pair: head-major gradients back to token-major ones
    dict(name="rope_480p_pair_gradient", op="rope", dtype="bf16", layout="interleaved", B=2, N=32760, Hq=12, Hk=12,
         d=128, rot=128, axes=3, rows=30, cols=52, start=0, inverse=True, token_major=True, scaling="none", factor=1.0),
    # a long token sequence: half layout, half of the head, fewer key heads, far positions of its own for each sequence,
    # frequencies scaled by parts; an odd length
    dict(name="rope_scaled_partial", op="rope", dtype="fp16", layout="half", B=3, N=4097, Hq=16, Hk=4, d=128, rot=64,
         axes=1, rows=0, cols=0, start=100000, inverse=False, token_major=True, scaling="parts", factor=8.0),
    # one new token for each of 16 sequences, each at its own position: latency
    dict(name="rope_token", op="rope", dtype="bf16", layout="half", B=16, N=1, Hq=24, Hk=24, d=64, rot=64,
         axes=1, rows=0, cols=0, start=5000, inverse=False, token_major=True, scaling="none", factor=1.0),
    # one layer at 480x832, teacher in bf16
    dict(name="loss_480p", op="loss", teacher="bf16", B=1, H=12, N=32760, d=128, weighted=False),
    # a padded batch of 320x480 clips, teacher in fp32, a weight for each token
    dict(name="loss_320p_padded", op="loss", teacher="fp32", B=2, H=12, N=24600, d=128, weighted=True),
    # the smallest configuration (4 frames of 8 x 8 tokens, 2 heads of 64): latency
    dict(name="loss_tiny", op="loss", teacher="bf16", B=1, H=2, N=256, d=64, weighted=False),
    # the eight tensors of one block's feature maps (12 heads of 128)
    dict(name="adamw_block", op="adamw", bits=32, param="bf16", master=True, grad="fp32", blocks=1, H=12, d=128, trim=0),
    # all 25 converted blocks at once, 200 tensors
    dict(name="adamw_25_blocks", op="adamw", bits=32, param="bf16", master=True, grad="fp32", blocks=25, H=12, d=128,
         trim=0),
    # the same with moments in 8 bits, which are read back as for a checkpoint
    dict(name="adamw_25_blocks_8bit", op="adamw", bits=8, param="bf16", master=True, grad="fp32", blocks=25, H=12, d=128,
         trim=0),
    # odd sizes: tensors that end inside a group of 32, no copy of the weights in 32 bits, gradients in bf16
    dict(name="adamw_odd_8bit", op="adamw", bits=8, param="bf16", master=False, grad="bf16", blocks=7, H=3, d=64,
         trim=37),
    # the smallest configuration's maps (2 heads of 64): latency
    dict(name="adamw_tiny", op="adamw", bits=32, param="bf16", master=True, grad="fp32", blocks=1, H=2, d=64, trim=0),
]

_LR, _B1, _B2, _EPS, _WD = 1e-3, 0.9, 0.999, 1e-8, 0.01   # of the paper's distillation, and the usual others
_STEP = 40                                                 # updates made before the one that is measured
_ALIGN, _GROUP = 256, 32


def _f32(x):
    return float(torch.tensor(x, dtype=torch.float32))


def listed():
    return [dict(c) for c in _LISTED]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    while True:
        op = rng.choice(("rope", "rope", "loss", "adamw", "adamw"))
        if op == "rope":
            d = rng.choice((64, 128, 128, 80, 96, 256))
            rot = rng.choice((d, d, d // 2, 2 * rng.randint(4, d // 2)))
            axes = rng.choice((1, 1, 2, 3, 3)) if rot >= 16 else 1
            rows, cols = rng.randint(3, 60), rng.randint(3, 80)
            hk = _log_int(rng, 1, 24)
            c = dict(op=op, dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")), layout=rng.choice(("interleaved", "half")),
                     B=_log_int(rng, 1, 16), N=_log_int(rng, 1, 75600), Hq=hk * rng.choice((1, 1, 2, 4)), Hk=hk, d=d,
                     rot=rot, axes=axes, rows=rows if axes == 3 else 0, cols=cols if axes > 1 else 0,
                     start=rng.choice((0, _log_int(rng, 1, 1000000))) if axes == 1 else rng.choice((0, rng.randint(1, 200))),
                     inverse=rng.random() < 0.4, token_major=rng.random() < 0.7,
                     scaling=rng.choice(("none", "none", "linear", "base", "parts")), factor=1.0)
            if c["scaling"] != "none":
                c["factor"] = rng.choice((2.0, 4.0, 8.0, 2.5))
        elif op == "loss":
            c = dict(op=op, teacher=rng.choice(("bf16", "bf16", "fp16", "fp32")), B=rng.choice((1, 1, 2, 3)),
                     H=_log_int(rng, 1, 24), N=_log_int(rng, 1, 75600), d=rng.choice((64, 128)),
                     weighted=rng.random() < 0.5)
        else:
            p = rng.choice(("bf16", "bf16", "fp16", "fp32"))
            c = dict(op=op, bits=rng.choice((32, 8)), param=p, master=p != "fp32" and rng.random() < 0.7,
                     grad=rng.choice(("fp32", "fp32", "bf16")), blocks=_log_int(rng, 1, 30), H=_log_int(rng, 1, 24),
                     d=rng.choice((64, 128)), trim=rng.choice((0, rng.randint(1, 255))))
        if work(c)["bytes"] <= max(work(x)["bytes"] for x in _LISTED if x["op"] == op):
            return c


# ---- inputs ---------------------------------------------------------------------------------------------------------


def _sections(c):
    """Pairs of a head for each axis: a third each, the first axis takes what is left over."""
    pairs, n = c["rot"] // 2, c["axes"]
    return [pairs - (n - 1) * (pairs // n)] + [pairs // n] * (n - 1)


def _frequencies(c):
    """Radians a position of each pair in 64 bits, and the factor on the rotated values: scaling of the first axis
    "linear" (positions divided), "base" (a larger base), "parts" (slow pairs divided, fast ones kept, between them a
    ramp over the turns that a pair makes in 4,096 positions, from 1 to 32)."""
    out, mu = [], 1.0
    for axis, n in enumerate(_sections(c)):
        base, s = 10000.0, c["factor"] if axis == 0 else 1.0
        kind = c["scaling"] if axis == 0 else "none"
        if kind == "base":
            base *= s ** (n / (n - 1)) if n > 1 else 1.0
        f = base ** (-torch.arange(n, dtype=torch.float64) / n)
        if kind == "linear":
            f = f / s
        elif kind == "parts":
            keep = ((4096 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
            f = f * keep + f / s * (1.0 - keep)
            mu = 0.1 * math.log(s) + 1.0
        out.append(f)
    return torch.cat(out), mu


def _tensors(c):
    """Element counts of one set of parameters, weights first, and how many of them are weights."""
    H, d, w = c["H"], c["d"], 2 * c["d"]
    weights = [H * w * d, H * w * w] * 2 * c["blocks"]
    biases = [H * w] * 4 * c["blocks"]
    return [n - min(c["trim"], n - 1) for n in weights], [n - min(c["trim"], n - 1) for n in biases]


def _offsets(sizes):
    """Each tensor begins at a multiple of 256 elements of one buffer."""
    out, at = [], 0
    for n in sizes:
        out.append(at)
        at += -(-n // _ALIGN) * _ALIGN
    return out, at


def _pack_m(m):
    """Groups of 32 as e4m3 and the group's exponent (biased; at least 8; 255: not finite)."""
    x = m.view(-1, _GROUP)
    e = (x.abs().amax(1).view(torch.int32) >> 23).clamp(min=8)
    codes = (x * ((261 - e) << 23).view(torch.float32)[:, None]).to(torch.float8_e4m3fn)
    return codes.view(-1), torch.where(e >= 254, 255, e).to(torch.uint8)


def _unpack_m(codes, e):
    e = e.to(torch.int32)
    x = codes.view(-1, _GROUP).float() * ((e - 7) << 23).view(torch.float32)[:, None]
    return torch.where(e[:, None] == 255, math.nan, x).view(-1)


def _pack_v(v):
    """Groups of 32 as unsigned floats of 5 exponent and 3 mantissa bits under the group's exponent; what is not zero
    keeps a code of at least 1."""
    x = v.view(-1, _GROUP)
    e = (x.amax(1).view(torch.int32) >> 23).clamp(min=31)
    bits = x.view(torch.int32)
    codes = ((bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20) - ((e - 30) << 3)[:, None]
    codes = torch.where(x == 0, 0, codes.clamp(1, 255))
    return codes.to(torch.uint8).view(-1), torch.where(e >= 254, 255, e).to(torch.uint8)


def _unpack_v(codes, e):
    e, k = e.to(torch.int32)[:, None], codes.view(-1, _GROUP).to(torch.int32)
    x = torch.where(k == 0, 0.0, ((k + ((e - 30) << 3)) << 20).view(torch.float32))
    return torch.where(e == 255, math.nan, x).view(-1)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    st = dict(case=dict(c))
    if c["op"] == "rope":
        dt = _DTYPES[c["dtype"]]

        def operand(H, token_major):   # logically [B, H, N, d]
            if token_major:
                return normal(c["B"], c["N"], H, c["d"]).to(dt).transpose(1, 2)
            return normal(c["B"], H, c["N"], c["d"]).to(dt)

        token_major = c["token_major"] and not c["inverse"]   # gradients arrive head-major
        st["q"], st["k"] = operand(c["Hq"], token_major), operand(c["Hk"], token_major)
        if c["axes"] == 1:   # positions of each sequence in a buffer of the caller, as with sequences of different lengths
            first = torch.randint(0, c["start"] + 1, (c["B"], 1), generator=g, device="cuda")
            st["positions"] = first + torch.arange(c["N"], device="cuda")
        st["freqs"], st["mu"] = _frequencies(c)
        if own:
            from paper_2601_04342_amd import binding
            scaling = None if c["scaling"] == "none" else dict(kind=c["scaling"], factor=c["factor"], original=4096)
            st["plan"] = binding.Rope(c["d"], rot=c["rot"], layout=c["layout"], sections=_sections(c), scaling=scaling)
        else:
            st["freqs"] = st["freqs"].cuda()
        return st
    if c["op"] == "loss":
        y = normal(c["B"], c["H"], c["N"], c["d"])
        st["y_hat"] = (y + 0.1 * normal(c["B"], c["H"], c["N"], c["d"])).to(torch.bfloat16)
        st["y"] = y.to(_DTYPES[c["teacher"]])
        st["scale"] = 1.0 / y.numel()
        if c["weighted"]:   # the clips of a batch end at different tokens; behind them stands whatever was there
            ends = torch.randint((c["N"] + 1) // 2, c["N"] + 1, (c["B"], 1), generator=g, device="cuda")
            pad = torch.arange(c["N"], device="cuda") >= ends
            st["weight"] = torch.where(pad, 0.0, 0.5 + torch.rand(c["B"], c["N"], generator=g, device="cuda"))
            st["y_hat"].masked_fill_(pad[:, None, :, None], math.nan)
        return st
    weights, biases = _tensors(c)
    off, n = _offsets(weights + biases)
    nw = off[len(weights)]
    live = torch.zeros(n, device="cuda", dtype=torch.bool)
    for o, k in zip(off, weights + biases):
        live[o:o + k] = True

    def flat(x):
        return torch.where(live, x, 0.0)

    dt = _DTYPES[c["param"]]
    p = flat(0.02 * normal(n))
    grad = flat(1e-3 * normal(n)).to(_DTYPES[c["grad"]])
    m = flat(3e-4 * normal(n))
    v = flat((1e-3 * normal(n)).square() + 1e-9)
    st["w"] = p[:nw].to(dt)
    st["b"] = p[nw:].clone()                      # biases are kept in 32 bits, as the library has them
    st["master"] = st["w"].float() if c["master"] else None
    st["grad"], st["step"], st["live"] = grad, _STEP, live
    if c["bits"] == 8:
        (st["m"], st["me"]), (st["v"], st["ve"]) = _pack_m(m), _pack_v(v)
    else:
        st["m"], st["v"] = m, v
    if own:
        from paper_2601_04342_amd import binding
        at = list(zip(off, weights + biases))
        params = [st["w"][o:o + k] for o, k in at[:len(weights)]] + [st["b"][o - nw:o - nw + k] for o, k in at[len(weights):]]
        st["opt"] = binding.AdamW(params, lr=_LR, betas=(_B1, _B2), eps=_EPS, weight_decay=_WD, state_bits=c["bits"],
                                  master=c["master"], grads=[grad[o:o + k] for o, k in at])
        st["opt"].load_state(st["m"], st["v"], _STEP, m_exp=st.get("me"), v_exp=st.get("ve"))
        st["opt"].nearest_steps = 1 << 62   # codes as the plain form rounds them; by default this update's are rounded at random
        if c["bits"] == 8:
            st["values"] = [torch.empty(n, device="cuda") for _ in range(2)]
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------


def _rope_plain(st):
    c = st["case"]
    if c["axes"] == 1:
        pos = st["positions"][:, :, None].double()
    else:
        n = torch.arange(c["N"], device="cuda")
        hw, w = max(c["rows"], 1) * c["cols"], c["cols"]
        at = [n // hw, n % hw // w, n % w] if c["axes"] == 3 else [n // w, n % w]
        at[0] = at[0] + c["start"]
        pos = torch.stack(at, 1).double()[None]
    axis = torch.repeat_interleave(torch.arange(c["axes"]), torch.tensor(_sections(c))).cuda()
    angle = pos[..., axis] * st["freqs"]                                # [B or 1, N, rot / 2], 64 bits: far positions
    cos = (angle.cos() * st["mu"]).float()[:, None]
    sin = (angle.sin() * (-st["mu"] if c["inverse"] else st["mu"])).float()[:, None]
    rot = c["rot"]

    def turn(x):
        out = torch.empty(x.shape, device="cuda", dtype=x.dtype)
        if c["inverse"] and c["token_major"]:
            out = torch.empty(x.transpose(1, 2).shape, device="cuda", dtype=x.dtype).transpose(1, 2)
        if c["layout"] == "interleaved":
            first, second = slice(0, rot, 2), slice(1, rot, 2)
        else:
            first, second = slice(0, rot // 2), slice(rot // 2, rot)
        a, b = x[..., first].float(), x[..., second].float()
        out[..., first] = a * cos - b * sin
        out[..., second] = b * cos + a * sin
        out[..., rot:] = x[..., rot:]
        return out

    return turn(st["q"]), turn(st["k"])


def _loss_plain(st):
    diff = st["y_hat"].float() - st["y"].float()
    scale = torch.full((), st["scale"], device="cuda", dtype=torch.float32)
    sign = (diff > 0).float() - (diff < 0).float()
    sign = torch.where(diff.isnan(), diff, sign)
    if not st["case"]["weighted"]:
        return (diff.abs().sum(dtype=torch.float64) * st["scale"]).float(), (sign * scale).to(torch.bfloat16)
    w = st["weight"][:, None, :, None]
    diff = torch.where(w == 0, 0.0, diff)
    sign = torch.where(w == 0, 0.0, sign)
    return ((diff.abs() * w).sum(dtype=torch.float64) * st["scale"]).float(), (sign * (w * scale)).to(torch.bfloat16)


def _adamw_plain(st):
    c = st["case"]
    st["step"] += 1
    nw = st["w"].numel()
    p = torch.cat([st["master"] if c["master"] else st["w"].float(), st["b"]])
    if c["bits"] == 8:   # in 64 bits: the moments are rounded once, to 32 bits, before they are rounded to 8
        g = st["grad"].double()
        m = (_unpack_m(st["m"], st["me"]).double() * _f32(_B1) + g * _f32(1.0 - _B1)).float()
        v = (_unpack_v(st["v"], st["ve"]).double() * _f32(_B2) + g * g * _f32(1.0 - _B2)).float()
    else:
        g = st["grad"].float()
        m = st["m"] * _B1 + g * (1.0 - _B1)
        v = st["v"] * _B2 + g * g * (1.0 - _B2)
    denom = v.sqrt() / math.sqrt(1.0 - _B2 ** st["step"]) + _EPS
    p = p * (1.0 - _LR * _WD) - m / denom * (_LR / (1.0 - _B1 ** st["step"]))
    st["w"].copy_(p[:nw])
    st["b"].copy_(p[nw:])
    if c["master"]:
        st["master"].copy_(p[:nw])
    if c["bits"] == 8:
        (st["m"], st["me"]), (st["v"], st["ve"]) = _pack_m(m), _pack_v(v)
        m, v = _unpack_m(st["m"], st["me"]), _unpack_v(st["v"], st["ve"])
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
    out = dict(w=st["w"], b=st["b"], m=m, v=v)
    return dict(out, master=st["master"]) if c["master"] and c["param"] != "fp32" else out


def _run_own(st):
    from paper_2601_04342_amd import binding
    c = st["case"]
    if c["op"] == "rope":
        q, k = st["q"], st["k"]
        if c["axes"] == 1:
            where = dict(positions=st["positions"])
        else:
            where = dict(grid=(c["rows"], c["cols"]) if c["axes"] == 3 else (c["cols"],), start=c["start"])
        if c["inverse"] and c["token_major"]:
            where["out"] = tuple(torch.empty(x.transpose(1, 2).shape, device="cuda", dtype=x.dtype).transpose(1, 2)
                                 for x in (q, k))
        return binding.rope(q, k, st["plan"], inverse=c["inverse"], **where)
    if c["op"] == "loss":
        return binding.distill_loss(st["y_hat"], st["y"], scale=st["scale"], weight=st.get("weight"))
    opt = st["opt"]
    opt.step()
    m, v = opt.moments(out=st["values"]) if c["bits"] == 8 else (opt.m, opt.v)
    out = dict(w=st["w"], b=st["b"], m=m, v=v)
    return dict(out, master=opt.master) if c["master"] and c["param"] != "fp32" else out


def run(state):
    if own:
        return _run_own(state)
    if state["case"]["op"] == "rope":
        return _rope_plain(state)
    return _loss_plain(state) if state["case"]["op"] == "loss" else _adamw_plain(state)


# ---- the same in 64 bits ----------------------------------------------------------------------------------------------


def _rope_exact(st):
    c = st["case"]
    B, N, n = c["B"], c["N"], c["axes"]
    tokens = torch.arange(N, dtype=torch.float64, device="cuda")
    if n == 1:
        where = [st["positions"].double()]
    elif n == 2:
        row = torch.div(tokens, c["cols"], rounding_mode="floor")
        where = [row + c["start"], tokens - row * c["cols"]]
    else:
        line = torch.div(tokens, c["cols"], rounding_mode="floor")
        frame = torch.div(line, c["rows"], rounding_mode="floor")
        where = [frame + c["start"], line - frame * c["rows"], tokens - line * c["cols"]]
    freqs = _frequencies(c)[0].cuda().split(_sections(c))
    turns = torch.cat([torch.polar(torch.full((), st["mu"], dtype=torch.float64, device="cuda").expand(x.shape + f.shape),
                                   x[..., None] * f) for x, f in zip(where, freqs)], -1)
    turns = (turns.conj() if c["inverse"] else turns).expand(B, N, -1)
    outs = []
    for x in (st["q"], st["k"]):
        out = x.double()
        for b in range(B):
            z, t = out[b, :, :, :c["rot"]], turns[b]
            if c["layout"] == "interleaved":
                z = torch.view_as_complex(z.unflatten(-1, (-1, 2)).contiguous()) * t
                out[b, :, :, :c["rot"]] = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(*z.contiguous().chunk(2, -1)) * t
                out[b, :, :, :c["rot"]] = torch.cat([z.real, z.imag], -1)
        outs.append(out)
    return tuple(outs)


def _loss_exact(st):
    diff = st["y_hat"].double().sub_(st["y"].double())
    if "weight" not in st:
        return diff.abs().sum() * st["scale"], diff.sign() * st["scale"]
    w = st["weight"].double()[:, None, :, None].expand_as(diff)
    diff[w == 0] = 0.0
    return (diff.abs() * w).sum() * st["scale"], diff.sign() * w * st["scale"]


def _two_to(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _value_m(m):
    """What stands for m, a number of 32 bits: e4m3 multiples of a power of two for each 32 (at 128 to 256 for the largest)."""
    x = m.view(-1, _GROUP)
    top = torch.frexp(x.abs().amax(1, keepdim=True))[1].clamp(min=-118)       # largest value in [2^(top-1), 2^top)
    x = x * _two_to(8 - top)
    step = _two_to(torch.frexp(x)[1].clamp(min=-5) - 4)                       # the least e4m3 exponent is 2^-6
    return ((x / step).round() * step * _two_to(top - 8)).view(-1)


def _value_v(v):
    """What stands for v: three bits behind the leading one, 30 binades below the group's largest and what is less at
    the least of them."""
    x = v.view(-1, _GROUP)
    top = torch.frexp(x.amax(1, keepdim=True))[1].clamp(min=-95)
    step = _two_to(torch.frexp(x)[1] - 4)
    least = 1.125 * _two_to(top - 31)
    return torch.where(x > 0, torch.maximum((x / step).round() * step, least), 0.0).view(-1)


def _adamw_exact(st):
    c, t = st["case"], st["step"] + 1
    nw = st["w"].numel()
    p = torch.cat([(st["master"] if c["master"] else st["w"]).double(), st["b"].double()])
    g = st["grad"].double()
    if c["bits"] == 8:   # coefficients and new moments are numbers of 32 bits, and those are what is kept in 8
        m, v = _unpack_m(st["m"], st["me"]).double(), _unpack_v(st["v"], st["ve"]).double()
        m = torch.add(_f32(_B1) * m, g, alpha=_f32(1 - _B1)).float().double()
        v = torch.addcmul(_f32(_B2) * v, g, g, value=_f32(1 - _B2)).float().double()
    else:
        m = torch.lerp(g, st["m"].double(), _B1)
        v = torch.lerp(g.square(), st["v"].double(), _B2)
    p = p - _LR * _WD * p - _LR * (m / (1 - _B1 ** t)) / ((v / (1 - _B2 ** t)).sqrt() + _EPS)
    out = dict(w=p[:nw], b=p[nw:], m=_value_m(m) if c["bits"] == 8 else m, v=_value_v(v) if c["bits"] == 8 else v)
    return dict(out, master=p[:nw]) if c["master"] and c["param"] != "fp32" else out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "rope":
        return _rope_exact(st)
    return _loss_exact(st) if case["op"] == "loss" else _adamw_exact(st)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------


def work(case):
    c = case
    if c["op"] == "rope":
        rows = c["B"] * c["N"] * (c["Hq"] + c["Hk"])
        return dict(bytes=2 * rows * c["d"] * _SIZE[c["dtype"]] + (8 * c["B"] * c["N"] if c["axes"] == 1 else 0),
                    flops=3 * rows * c["rot"])
    if c["op"] == "loss":
        n = c["B"] * c["H"] * c["N"] * c["d"]
        return dict(bytes=n * (4 + _SIZE[c["teacher"]]) + (4 * c["B"] * c["N"] if c["weighted"] else 0), flops=3 * n)
    weights, biases = (sum(x) for x in _tensors(c))
    n, size = weights + biases, _SIZE[c["param"]]
    p = weights * (size + 8 if c["master"] else 2 * size) + biases * 8
    # 8 bits: both moments and an exponent for 32 of each, read, written, and read again for their values in 32 bits
    state = n * (3 * 2 + 3 * 2 / 32 + 8) if c["bits"] == 8 else n * 16
    return dict(bytes=int(p + state + n * _SIZE[c["grad"]]), flops=16 * n)
