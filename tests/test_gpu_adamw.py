"""AdamW over many tensors (rehyat_adamw_*) against its formulas in 64 bits, and its 8-bit moments code for code against
a search through all values of the formats."""
import math

import numpy as np
import pytest
import torch

from paper_2601_04342_amd import binding, synth

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
SIZES = [1, 3, 31, 32, 33, 255, 256, 257, 1000, 4095, 4096, 4097, 10001]


def f32(x):
    return float(np.float32(x))


def make(sizes, dtype, grad_dtype, bits, master=True, seed=0, gap=0, scale=1e-3, **kw):
    """Parameters and gradients (in buffers of their own with `gap` elements around each) and an optimiser with a state
    of some updates."""
    g = torch.Generator().manual_seed(seed)

    def views(dt, spread):
        flat = torch.full((sum(sizes) + gap * (len(sizes) + 1),), 7.0, dtype=dt)
        out, at = [], gap
        for n in sizes:
            flat[at:at + n] = (torch.randn(n, generator=g) * spread).to(dt)
            out.append((at, n))
            at += n + gap
        flat = flat.cuda()
        return flat, [flat[a:a + n] for a, n in out]

    pf, params = views(dtype, 0.02)
    gf, grads = views(grad_dtype, scale)
    opt = binding.AdamW(params, grads=grads, state_bits=bits, master=master, **kw)
    return opt, pf, gf


def fill_state(opt, seed=1, scale=1e-3, step=9):
    """Random moments: of 32 bits directly, of 8 bits by some updates."""
    g = torch.Generator().manual_seed(seed)
    n = opt.m.numel()
    if opt.state_bits == 32:
        opt.load_state(torch.randn(n, generator=g) * 0.3 * scale, (torch.randn(n, generator=g) * scale).square(), step)
        return
    keep = [t.clone() for t in opt._grads]
    for _ in range(3):
        for t in opt._grads:
            t.copy_((torch.randn(t.shape, generator=g) * scale).to(t.dtype))
        opt.step(lr=0.0)
    for t, k in zip(opt._grads, keep):
        t.copy_(k)
    opt.step_count.fill_(step)


def state_of(opt):
    """p, g, m, v of every tensor in 64 bits on the CPU."""
    torch.cuda.synchronize()
    m, v = (t.cpu().double() for t in opt.moments())
    master = None if opt.master is None else opt.master.cpu().double()
    out = []
    for p, g, o, mo in zip(opt.params, opt._grads, opt.offsets, opt.master_offsets):
        n = p.numel()
        weight = p.cpu().double().view(-1) if mo is None else master[mo:mo + n]
        out.append((weight, g.cpu().double().view(-1), m[o:o + n], v[o:o + n]))
    return out


def check_step(opt, lr=None, label=""):
    """One step against the formulas from the state before it."""
    before, t = state_of(opt), int(opt.step_count.item()) + 1
    opt.step() if lr is None else opt.step(lr=lr)
    rate = opt.lr if lr is None else float(lr)
    (b1, b2), eps, wd = opt.betas, opt.eps, opt.weight_decay
    u = 2.0**-24
    assert int(opt.step_count.item()) == t
    for i, ((p, g, m, v), (p2, _, m2, v2)) in enumerate(zip(before, state_of(opt))):
        dt = opt.params[i].dtype
        # moments: a coefficient, a product and a sum are rounded (g^2 once more)
        wm, wv = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        em, ev = 4 * u * (b1 * m.abs() + (1 - b1) * g.abs()) + 2.0**-148, 5 * u * wv + 2.0**-147
        if opt.state_bits == 32:
            assert ((m2 - wm).abs() <= em).all() and ((v2 - wv).abs() <= ev).all(), (label, i)
        # update: what the moments are off by (a root halves it), then at most 12 roundings of factors, root, sum and
        # quotient; the weight: two roundings of the decay, one of the sum
        denom = wv.sqrt() / math.sqrt(1 - b2**t) + eps
        step = rate / (1 - b1**t) * wm / denom
        off = rate / (1 - b1**t) * em / denom + step.abs() * (ev / wv.clamp(min=1e-300) / 2 + 12 * u)
        want = p * (1 - rate * wd) - step
        most = off + u * (3 * p.abs() + 2 * step.abs()) + 2.0**-149
        if opt.master_offsets[i] is not None:
            assert ((p2 - want).abs() <= most).all(), (label, i, ((p2 - want).abs() / most).max())
            assert torch.equal(opt.params[i].cpu().view(-1), p2.to(dt)), (label, i)
        else:
            half = torch.finfo(dt).eps / 2
            tiny = 2.0**-25 if dt == FP16 else 0.0
            err = (p2 - want).abs()
            assert (err <= most * (1 + 2 * half) + (half * (want.abs() + most) + tiny if dt != FP32 else 0)).all(), (label, i)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [FP32, BF16, FP16])
@pytest.mark.parametrize("dtype,master", [(BF16, True), (FP16, True), (FP32, False), (BF16, False), (FP16, False)])
def test_types_and_sizes(dtype, master, grad, bits):
    opt, _, _ = make(SIZES, dtype, grad, bits, master, seed=3)
    fill_state(opt)
    for i in range(3):
        check_step(opt, label=str(i))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gap", [1, 3, 8])
def test_tensors_at_any_place_of_a_buffer(gap, bits):
    """Views that begin at any element; what stands between them is left alone."""
    opt, pf, gf = make([5, 33, 4097, 64, 1], BF16, BF16, bits, seed=4, gap=gap)
    fill_state(opt)
    was, state = gf.clone(), [opt.m.float().cpu(), opt.v.float().cpu()]
    check_step(opt)
    live = torch.zeros_like(pf, dtype=torch.bool)
    for p in opt.params:
        at = (p.data_ptr() - pf.data_ptr()) // 2
        live[at:at + p.numel()] = True
    assert (pf[~live] == 7).all() and torch.equal(gf, was)
    used = torch.zeros(opt.m.numel(), dtype=torch.bool)
    for o, p in zip(opt.offsets, opt.params):
        used[o:o + p.numel()] = True
    for now, then in zip((opt.m, opt.v), state):
        assert torch.equal(now.float().cpu()[~used], then[~used])


def test_more_tensors_than_a_launch_describes():
    """Types and sizes mixed, empty ones among them; a list of dicts, as the feature maps of many blocks are."""
    g = torch.Generator().manual_seed(5)
    blocks = []
    for i in range(60):
        n = int(torch.randint(1, 6000, (1,), generator=g))
        blocks.append({"w": (torch.randn(n, generator=g) * 0.02).to("cuda", (BF16, FP16, FP32)[i % 3]),
                       "b": (torch.randn(i % 5, 3, generator=g) * 0.02).cuda(), "s": torch.ones((), device="cuda")})
    opt = binding.AdamW(blocks, weight_decay=0.1)
    assert len(opt.params) == 180 and opt.grads[7]["b"].shape == (2, 3) and opt.grads[7]["w"].dtype == FP32
    for b in opt.grads:
        for t in b.values():
            t.copy_(torch.randn(t.shape, generator=g) * 1e-2)
    for _ in range(3):
        check_step(opt)


@pytest.mark.parametrize("bits", [32, 8])
def test_offsets_beyond_32_bits(bits):
    n = 2**31 + 4099 if bits == 8 else 2**30 + 4099        # 2^32 bytes and more of each buffer
    dt = BF16 if bits == 8 else FP32
    p, g = torch.zeros(n, device="cuda", dtype=dt), torch.zeros(n, device="cuda", dtype=dt)
    g[-5000:] = (torch.randn(5000, generator=torch.Generator().manual_seed(6)) * 1e-3).to("cuda", dt)
    p[:100] = 1.0
    opt = binding.AdamW([p], grads=[g], state_bits=bits, master=False, lr=0.5, weight_decay=0.25)
    opt.step()
    assert (p[:100] == 0.875).all() and (p[100:-5000] == 0).all()
    want = -0.5 * g[-5000:].double() / (g[-5000:].double().abs() + 1e-8)
    assert ((p[-5000:].double() - want).abs() <= (2.0**-8 + 2.0**-18) * 0.5).all()   # one rounding, to bf16 at most
    assert (opt.m[:4096].float() == 0).all() and (opt.m[-1:].float() == 0).all()      # the buffer's own padding
    del opt, p, g
    torch.cuda.empty_cache()


# ---- moments in 8 bits -------------------------------------------------------------------------------------------------


def e4m3_values():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    return v


def nearest(values, x):
    """Index of the nearest of the sorted `values`, ties to the even index."""
    i = np.searchsorted(values, x)
    lo, hi = max(i - 1, 0), min(i, len(values) - 1)
    a, b = x - values[lo], values[hi] - x
    return lo if a < b or (a == b and lo % 2 == 0) else hi


def encode(m, v):
    """Codes and exponents of one group from its fp32 moments, by search."""
    top = max(abs(float(x)) for x in m)
    em = max(8, (int(np.float32(top).view(np.int32)) >> 23))
    half = e4m3_values()[:127]                     # 0 and up, in order; 127 is NaN
    cm = []
    for x in m:
        c = nearest(half, abs(float(x)) * 2.0**(134 - em))
        cm.append(int(c) | (0x80 if np.signbit(x) else 0))
    ev = max(31, int(np.float32(max(v)).view(np.int32)) >> 23)
    # code c: the number without sign of leading bits c + 8 (ev - 30); code 0 stands for 0 instead
    codes = (np.arange(256) + 8 * (ev - 30)).astype(np.int64) << 20
    values = codes.astype(np.int32).view(np.float32).astype(np.float64)
    cv = [0 if x == 0 else max(1, int(nearest(values, float(x)))) for x in v]
    return cm, em, cv, ev


def decode(cm, em, cv, ev):
    m = e4m3_values()[cm] * 2.0**(max(em, 8) - 134)
    v = ((np.asarray(cv, np.int64) + 8 * (max(ev, 31) - 30)) << 20).astype(np.int32).view(np.float32).astype(np.float64)
    return m, np.where(np.asarray(cv) == 0, 0.0, v)


def moments_after(m, v, g, b1=0.9, b2=0.999):
    """The new moments in fp32: products of 24-bit numbers are exact in 64 bits, and so is what they add up to but for
    one rounding far below the fp32 one."""
    with np.errstate(all="ignore"):
        nm = (f32(b1) * m + f32(1 - b1) * g).astype(np.float32)
        nv = (f32(b2) * v + f32(1 - b2) * (g * g)).astype(np.float32)
    return nm, nv


@pytest.mark.parametrize("kind", ["normal", "bf16", "wide", "tiny", "huge", "sparse", "equal"])
def test_codes_are_the_nearest_values(kind):
    """bf16 gradients beside 4-bit moments fall half way between two codes often; "wide" spans 40 binades in a group."""
    g = torch.Generator().manual_seed(len(kind))
    n = 32 * 24 + 5
    draw = {"normal": lambda: torch.randn(n, generator=g) * 1e-3,
            "bf16": lambda: (torch.randn(n, generator=g) * 1e-3).to(BF16).float(),
            "wide": lambda: torch.randn(n, generator=g) * 2.0**-torch.randint(0, 40, (n,), generator=g),
            "tiny": lambda: torch.randn(n, generator=g) * 2.0**-torch.randint(55, 80, (n,), generator=g),
            "huge": lambda: torch.randn(n, generator=g) * 2.0**torch.randint(50, 62, (n,), generator=g),
            "sparse": lambda: torch.randn(n, generator=g) * (torch.rand(n, generator=g) < 0.05),
            "equal": lambda: torch.full((n,), 0.125)}[kind]
    p = torch.zeros(n, device="cuda")
    opt = binding.AdamW([p], state_bits=8)
    pad = -(-n // 32) * 32
    cm, cv = np.zeros(pad, np.int64), np.zeros(pad, np.int64)
    em, ev = np.zeros(pad // 32, np.int64), np.zeros(pad // 32, np.int64)
    for step in range(6):
        grad = draw()
        opt._grads[0].copy_(grad)
        opt.step()
        gg = np.concatenate([grad.double().numpy(), np.zeros(pad - n)])
        for k in range(pad // 32):
            s = slice(32 * k, 32 * k + 32)
            m, v = decode(cm[s], em[k], cv[s], ev[k])
            nm, nv = moments_after(m, v, gg[s])
            cm[s], em[k], cv[s], ev[k] = encode(nm, nv)
        got_m = opt.m.view(torch.uint8).cpu().numpy().astype(np.int64)[:pad]
        got_v = opt.v.cpu().numpy().astype(np.int64)[:pad]
        assert (opt.m_exp.cpu().numpy()[:pad // 32] == em).all() and (opt.v_exp.cpu().numpy()[:pad // 32] == ev).all(), step
        assert ((got_m == cm) | ((got_m & 127 == 0) & (cm & 127 == 0))).all(), (step, np.nonzero(got_m != cm))
        assert (got_v == cv).all(), (step, np.nonzero(got_v != cv))
        mv = [t.cpu().double().numpy() for t in opt.moments()]
        for k in range(pad // 32):
            s = slice(32 * k, 32 * k + 32)
            m, v = decode(cm[s], em[k], cv[s], ev[k])
            assert (mv[0][s] == m).all() and (mv[1][s] == v).all()
        assert ((got_v[:n] > 0) | (cv[:n] == 0)).all()


def test_a_gradient_that_is_no_number():
    """With 32 bits its element alone, with 8 bits its group of 32 is lost; everything else goes on as before."""
    for bad in (float("nan"), float("inf"), float("-inf")):
        for bits in (32, 8):
            opt, _, _ = make([100, 64], FP32, FP32, bits, master=False, seed=7)
            ref, _, _ = make([100, 64], FP32, FP32, bits, master=False, seed=7)
            fill_state(opt), fill_state(ref)
            opt._grads[0][40] = bad
            for _ in range(2):
                opt.step(), ref.step()
                opt._grads[0][40] = 0.0
                ref._grads[0][40] = 0.0
            lost = torch.zeros(100, dtype=torch.bool)
            lost[32:64] = True if bits == 8 else False
            lost[40] = True
            a, b = opt.params[0].cpu(), ref.params[0].cpu()
            assert torch.isnan(a[lost]).all() and torch.equal(a[~lost], b[~lost]), (bad, bits)
            assert torch.equal(opt.params[1], ref.params[1])
            m, v = opt.moments()
            assert torch.equal(torch.isnan(m[:100].cpu()) | torch.isinf(v[:100].cpu()) | torch.isnan(v[:100].cpu()), lost)


# ---- how it is called -----------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(betas=(0.0, 0.0)), dict(betas=(0.0, 0.999), weight_decay=0.0), dict(eps=1e-3),
                                dict(betas=(0.95, 0.5), lr=1.0), dict(lr=0.0), dict(weight_decay=0.5, lr=0.1)])
def test_parameters_of_the_method(kw, bits):
    opt, _, _ = make([777, 32], BF16, FP32, bits, seed=9, **kw)
    if kw.get("betas") != (0.0, 0.0):
        fill_state(opt)
    for _ in range(2):
        check_step(opt)


def test_first_and_late_steps():
    for step in (0, 1, 10**6, 2**40):
        opt, _, _ = make([100], FP32, FP32, 32, master=False, seed=10)
        fill_state(opt, step=step)
        check_step(opt)
        assert int(opt.step_count.item()) == step + 1


def test_two_runs_agree():
    for bits in (32, 8):
        ends = []
        for _ in range(2):
            opt, _, _ = make(SIZES * 5, BF16, FP32, bits, seed=11)
            for _ in range(4):
                opt.step()
            ends.append([p.clone() for p in opt.params] + [opt.master.clone(), *opt.moments()])
        assert all(torch.equal(a, b) for a, b in zip(*ends))


@pytest.mark.parametrize("bits", [32, 8])
def test_graph_replays_count_and_follow_a_schedule(bits):
    opt, pf, gf = make([3000, 77], BF16, FP32, bits, seed=12)
    ref, rf, _ = make([3000, 77], BF16, FP32, bits, seed=12)
    lr = torch.full((1,), 1e-3, device="cuda")
    opt.step(lr=lr), ref.step(lr=1e-3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(lr=lr)
    for i in range(4):
        rate = f32(1e-3 * (i + 1))
        lr.fill_(rate)
        graph.replay()
        torch.cuda.synchronize()
        ref.step(lr=rate)
        assert torch.equal(pf, rf) and int(opt.step_count.item()) == i + 2
        gf.mul_(-0.5), ref._grads[0].mul_(-0.5), ref._grads[1].mul_(-0.5)
        if i == 1:                                   # an eager step between replays
            opt.step(lr=lr), ref.step(lr=rate)
            ref.step_count.sub_(1), opt.step_count.sub_(1)
    assert all(torch.equal(a, b) for a, b in zip(opt.moments(), ref.moments()))


def test_another_stream():
    opt, pf, _ = make(SIZES, BF16, FP32, 8, seed=13)
    ref, rf, _ = make(SIZES, BF16, FP32, 8, seed=13)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        opt.step(stream=side)
        ref.step()
    m, v = opt.moments(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(pf, rf) and torch.equal(m, ref.moments()[0]) and torch.equal(v, ref.moments()[1])


@pytest.mark.parametrize("bits", [32, 8])
def test_state_moves_to_another_optimiser(bits):
    opt, _, _ = make([500, 33], BF16, FP32, bits, seed=14)
    for _ in range(3):
        opt.step()
    other, _, _ = make([500, 33], BF16, FP32, bits, seed=14)
    for p, q in zip(other.params, opt.params):
        p.copy_(q)
    other.load_state(opt.m, opt.v, opt.step_count, m_exp=opt.m_exp, v_exp=opt.v_exp, master=opt.master)
    opt.step(), other.step()
    assert all(torch.equal(p, q) for p, q in zip(other.params, opt.params)) and torch.equal(opt.master, other.master)
    with pytest.raises(ValueError):
        other.load_state(opt.m[:-1], opt.v, 3, m_exp=opt.m_exp, v_exp=opt.v_exp)
    wrong, _, _ = make([500, 33], BF16, FP32, 40 - bits, seed=14)
    with pytest.raises(ValueError):
        wrong.load_state(opt.m, opt.v, 3, m_exp=opt.m_exp, v_exp=opt.v_exp)


def test_parameters_changed_from_elsewhere():
    opt, _, _ = make([100], BF16, FP32, 32, seed=15)
    opt.params[0].fill_(1.0)
    opt.reset_master()
    check_step(opt)
    assert (opt.params[0].float() - 1).abs().max() < 0.01


def test_refusals():
    p = torch.zeros(64, device="cuda")
    for bad in ([p, p], [p, p[10:20]], [p[:40], p[30:]]):     # the same numbers twice
        with pytest.raises(binding.RehyatError) as e:
            binding.AdamW(bad)
        assert e.value.code == binding.E_SHAPE
    with pytest.raises(binding.RehyatError):                   # a gradient that the step itself would overwrite
        binding.AdamW([p], grads=[p])
    with pytest.raises(TypeError):
        binding.AdamW([p.cpu()])
    with pytest.raises(TypeError):
        binding.AdamW([p.double()])
    with pytest.raises(TypeError):
        binding.AdamW([p[::2]])
    with pytest.raises(TypeError):
        binding.AdamW([p], grads=[p[:32].clone()])
    with pytest.raises(ValueError):
        binding.AdamW([p], grads=[p.clone(), p.clone()])
    with pytest.raises(ValueError):
        binding.AdamW([p], state_bits=16)
    with pytest.raises(ValueError):
        binding.AdamW([])
    with pytest.raises(binding.RehyatError):                   # nothing to update
        binding.AdamW([p[:0]])
    opt = binding.AdamW([p])
    for name, v in (("betas", (1.0, 0.9)), ("betas", (0.9, -0.1)), ("eps", 0.0), ("eps", 1e-50), ("lr", -1.0),
                    ("lr", math.nan), ("weight_decay", -1.0), ("weight_decay", math.inf)):
        keep = getattr(opt, name)
        setattr(opt, name, v)
        with pytest.raises(binding.RehyatError) as e:
            opt.step()
        assert e.value.code == binding.E_SHAPE, name
        setattr(opt, name, keep)
    with pytest.raises(TypeError):
        opt.step(lr=torch.ones(1))
    assert int(opt.step_count.item()) == 0


def test_feature_maps_of_a_block():
    """The dict that phi_backward takes and gives: its gradients are written where the step reads them."""
    B, H, T, HW, d = 1, 2, 4, 60, 64
    q, k, v = (t.to("cuda", BF16) for t in synth.make_qkv(B, H, T * HW, d, seed=16))
    phi = binding.phi_to_device(synth.make_phi(H, d, seed=17, gain=4.0))
    opt = binding.AdamW(phi)
    G = synth.make_grad_out(B, H, T * HW, d).to("cuda", BF16)
    want, _ = binding.phi_backward(q, k, v, phi, G, T, HW, 1)
    grads, _ = binding.phi_backward(q, k, v, phi, G, T, HW, 1, grads=opt.grads)
    assert all(torch.equal(grads[n], want[n]) and grads[n] is opt.grads[n] for n in phi)
    check_step(opt)


@pytest.mark.parametrize("bits", [32, 8])
def test_two_graphs_of_one_optimiser(bits):
    """Steps at two rates, captured apart, replayed in turn: one state, one count."""
    opt, pf, _ = make([5000, 33], BF16, FP32, bits, seed=20)
    ref, rf, _ = make([5000, 33], BF16, FP32, bits, seed=20)
    opt.step(), ref.step()
    torch.cuda.synchronize()
    graphs = []
    for lr in (1e-3, 3e-3):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            opt.step(lr=lr)
    for i in range(6):
        graphs[i % 2].replay()
        ref.step(lr=(1e-3, 3e-3)[i % 2])
        torch.cuda.synchronize()
        assert torch.equal(pf, rf) and int(opt.step_count.item()) == i + 2


def test_two_optimisers_at_once():
    sizes = [3000, 100000, 77]
    pairs = [(make(sizes, BF16, FP32, bits, seed=21), make(sizes, BF16, FP32, bits, seed=21)) for bits in (32, 8)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pairs]
    for _ in range(10):
        for s, (mine, _) in zip(streams, pairs):
            mine[0].step(stream=s)
        for _, ref in pairs:
            ref[0].step()
    torch.cuda.synchronize()
    for mine, ref in pairs:
        assert torch.equal(mine[1], ref[1]) and int(mine[0].step_count.item()) == 10
        assert all(torch.equal(a, b) for a, b in zip(mine[0].moments(), ref[0].moments()))
