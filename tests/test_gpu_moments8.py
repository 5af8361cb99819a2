"""8-bit moments of AdamW rounded at random: codes one for one against the formats' model, and thousands of updates beside an
optimiser with 32 bits."""
import numpy as np
import pytest
import torch

from paper_2601_04342_amd import binding
from tests import moments8
from tests.test_moments8_cpu import MEAN, MEDIAN, RMS

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("kind,steps", [("normal", 1500), ("constant", 1500), ("around", 1000), ("fall", 6000)])
def test_a_long_run_follows_32_bits(kind, steps):
    """The bounds are those of the model on the CPU, whose derivations stand there."""
    n = 2048 + 37
    g = torch.Generator(device="cuda").manual_seed(3)
    p = [torch.zeros(n, device="cuda") for _ in range(2)]
    grad = torch.zeros(n, device="cuda")
    mine, ref = (binding.AdamW([t], grads=[grad], state_bits=bits, lr=1.0, weight_decay=0.0) for t, bits in zip(p, (8, 32)))
    draw = {"normal": lambda t: torch.randn(n, generator=g, device="cuda") * 1e-3,
            "constant": lambda t: torch.full((n,), 1e-3, device="cuda"),
            "around": lambda t: (1 + 0.3 * torch.randn(n, generator=g, device="cuda")) * 1e-3,
            "fall": lambda t: torch.randn(n, generator=g, device="cuda") * (1e-3 if t <= 1000 else 1e-4)}[kind]
    for t in range(1, steps + 1):
        grad.copy_(draw(t))
        for x in p:
            x.zero_()
        mine.step(), ref.step()
        if t not in (100, 1000, 1500, 4000, 6000):
            continue
        v, want = (o.moments()[1][:n].double().cpu() for o in (mine, ref))
        rms = (p[0].double().square().mean() / p[1].double().square().mean()).sqrt().item()
        mean, median = (v / want).mean().item(), (v / want).median().item()
        if kind == "fall" and t > 1000:
            assert abs(mean - 1) <= 4 * 0.5 / n**0.5 and abs(rms - 1) <= (0.15 if t < 6000 else 0.1), (t, mean, rms)
        else:
            assert abs(mean - 1) <= MEAN and abs(median - 1) <= MEDIAN and abs(rms - 1) <= RMS, (t, mean, median, rms)


def padded(x):
    return np.concatenate([x, np.zeros(-len(x) % 32, x.dtype)])


@pytest.mark.parametrize("kind", ["normal", "wide", "small", "large", "sparse", "equal"])
@pytest.mark.parametrize("nearest_steps", [0, 2])
def test_codes_are_those_of_the_model(kind, nearest_steps):
    """Products of bf16 gradients, 4-bit moments and these betas are exact in fp32 and sums are rounded once, however they are
    contracted: codes are equal.  Several tensors, of odd sizes: each begins at a place of its own."""
    g = torch.Generator().manual_seed(len(kind))
    sizes = [32 * 40 + 5, 7, 1024, 3000]
    n = sum(sizes)
    draw = {"normal": lambda: torch.randn(n, generator=g) * 1e-3,
            "wide": lambda: torch.randn(n, generator=g) * 2.0**-torch.randint(0, 25, (n,), generator=g),
            "small": lambda: torch.randn(n, generator=g) * 2.0**-40,
            "large": lambda: torch.randn(n, generator=g) * 2.0**50,
            "sparse": lambda: torch.randn(n, generator=g) * (torch.rand(n, generator=g) < 0.05),
            "equal": lambda: torch.full((n,), 0.125)}[kind]
    b1, b2 = 1 - 2.0**-4, 1 - 2.0**-10
    opt = binding.AdamW([torch.zeros(k, device="cuda") for k in sizes], betas=(b1, b2), state_bits=8,
                        grads=[torch.zeros(k, device="cuda", dtype=BF16) for k in sizes], nearest_steps=nearest_steps)
    first = np.cumsum([0] + [-(-k // 1024) * 1024 for k in sizes])
    codes = [moments8.encode(padded(np.zeros(k, np.float32)), padded(np.zeros(k, np.float32))) for k in sizes]
    for t in (1, 2, 3, 4, 2**33 + 7, 2**33 + 8):
        grads = draw().to(BF16).split(sizes)
        for dst, src in zip(opt._grads, grads):
            dst.copy_(src)
        opt.step_count.fill_(t - 1)
        opt.step()
        for i, k in enumerate(sizes):
            x = padded(grads[i].float().numpy())
            m, v = (y.astype(np.float32) for y in moments8.decode(*codes[i]))
            m = np.float32(b1) * m + np.float32(1 - b1) * x
            v = np.float32(b2) * v + np.float32(1 - b2) * (x * x)
            bits = None if t <= nearest_steps else moments8.random_bits(t, int(first[i]) + np.arange(len(x)))
            codes[i] = moments8.encode(m, v, bits)
            o, pad = opt.offsets[i], len(x)
            got = [opt.m.view(torch.uint8)[o:o + pad], opt.m_exp[o // 32:(o + pad) // 32], opt.v[o:o + pad],
                   opt.v_exp[o // 32:(o + pad) // 32]]
            for name, a, b in zip(("m", "m_exp", "v", "v_exp"), got, codes[i]):
                assert np.array_equal(a.cpu().numpy(), b), (name, t, i, np.nonzero(a.cpu().numpy() != b)[0][:10])


def test_what_is_not_a_number_loses_its_group_alone():
    for bad in (float("nan"), float("inf"), -float("inf")):
        opt = binding.AdamW([torch.zeros(100, device="cuda")], state_bits=8, nearest_steps=0)
        opt._grads[0].fill_(1e-3)
        opt._grads[0][40] = bad
        opt.step()
        opt._grads[0][40] = 1e-3
        opt.step()
        m, v = (x[:100].cpu() for x in opt.moments())
        lost = torch.zeros(100, dtype=torch.bool)
        lost[32:64] = True
        assert torch.equal(torch.isnan(m), lost) and torch.equal(torch.isnan(v), lost)
        assert torch.equal(torch.isnan(opt.params[0].cpu()), lost)


def test_steps_to_the_nearest_are_checked_and_may_be_set():
    p = [torch.zeros(3000, device="cuda") for _ in range(3)]
    opts = [binding.AdamW([t], state_bits=8, nearest_steps=k) for t, k in zip(p, (0, 2, 2))]
    g = torch.randn(3000, generator=torch.Generator().manual_seed(1))
    for t in range(1, 5):
        if t == 3:
            opts[2].nearest_steps = 4
        for o in opts:
            o._grads[0].copy_(g)
            o.step()
        same = [torch.equal(opts[0].v, opts[1].v), torch.equal(opts[1].v, opts[2].v)]
        assert same == [False, t < 3]
    opts[0].nearest_steps = -1
    with pytest.raises(binding.RehyatError) as e:
        opts[0].step()
    assert e.value.code == binding.E_SHAPE


def test_replays_and_moved_states_are_rounded_alike():
    """The random bits go by the count on the device: a captured step rounds every replay by its own number, as eager steps
    and those of an optimiser that took over the state do."""
    def fresh():
        g = torch.Generator().manual_seed(9)
        opt = binding.AdamW([torch.zeros(k, device="cuda") for k in (5000, 33)], state_bits=8, nearest_steps=1)
        for t in opt._grads:
            t.copy_(torch.randn(t.shape, generator=g) * 1e-3)
        opt.step()
        return opt

    opt, ref, other = fresh(), fresh(), fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    codes = []
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        ref.step()
        if i == 3:
            other.load_state(ref.m, ref.v, ref.step_count, m_exp=ref.m_exp, v_exp=ref.v_exp)
            for a, b in zip(other.params, ref.params):
                a.copy_(b)
        elif i > 3:
            other.step()
        for o in (ref,) if i < 3 else (ref, other):
            assert torch.equal(opt.v, o.v) and torch.equal(opt.m.view(torch.uint8), o.m.view(torch.uint8)), i
            assert all(torch.equal(a, b) for a, b in zip(opt.params, o.params)), i
        codes.append(opt.v.clone())
    assert not any(torch.equal(a, b) for a, b in zip(codes, codes[1:]))
