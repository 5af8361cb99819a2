"""The loss and AdamW past the size (256 MB) from which they go past the caches: oddly placed tensors of mixed types, and
buffers of 8-bit moments beyond 2^32 bytes."""
import numpy as np
import pytest
import torch

from paper_2601_04342_amd import binding
from tests import moments8
from tests.test_gpu_adamw import check_step

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
PAST = 256 << 20


@pytest.mark.parametrize("N,d,weighted", [(24571, 127, False), (24571, 127, True), (24571, 128, True)])
@pytest.mark.parametrize("teacher", [BF16, FP16, FP32])
def test_loss(teacher, N, d, weighted):
    """Tolerances: those of the tests at smaller sizes (differences and products of 24 bits, eight added in 32 bits; one
    rounding of the gradient to bf16)."""
    B, H = 3, 7
    g = torch.Generator(device="cuda").manual_seed(d)
    y = torch.randn(B, H, N, d, generator=g, device="cuda").to(teacher)
    y_hat = (y.float() + 0.1 * torch.randn(B, H, N, d, generator=g, device="cuda")).to(BF16)
    assert y.numel() * (4 + y.element_size()) > PAST
    weight = None
    if weighted:
        weight = torch.rand(B, N, generator=g, device="cuda") * (torch.rand(B, N, generator=g, device="cuda") < 0.7)
    scale = 2.0**-25
    loss, grad = binding.distill_loss(y_hat, y, scale=scale, weight=weight)
    want = torch.zeros((), device="cuda", dtype=torch.float64)
    for b in range(B):
        diff = y_hat[b].double() - y[b].double()
        w = (torch.ones(1, N, 1, device="cuda") if weight is None else weight[b][None, :, None]).double()
        want += (w * diff.abs()).sum()
        ref = scale * w * diff.sign()
        got = grad[b].double()
        assert ((got - ref).abs() <= (2.0**-8 + 2 * 2.0**-24) * (1 + 2.0**-8) * ref.abs()).all(), b
        assert torch.equal(got == 0, ref == 0), b
    assert abs(loss.item() - want.item() * scale) <= (2 + 7 + 2) * 2.0**-24 * want.item() * scale


def decode(opt):
    """(m, v) of 8 bits from their definition."""
    em, ev = (e.to(torch.int32).repeat_interleave(32) for e in (opt.m_exp, opt.v_exp))
    m = opt.m.float() * torch.ldexp(torch.ones((), device="cuda"), em.clamp(min=8) - 134)
    c = opt.v.to(torch.int32)
    return m, torch.where(c == 0, 0.0, ((c + 8 * (ev.clamp(min=31) - 30)) << 20).view(torch.float32))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    sizes = [13_000_001, 5, 9_000_017, 4097, 7_000_033]
    kinds = [(BF16, FP32), (FP32, BF16), (FP32, FP16), (FP16, FP32), (BF16, FP16)]
    g = torch.Generator(device="cuda").manual_seed(bits)

    def odd(n, dtype, spread):                       # begins one element into its buffer
        return (torch.randn(n + 1, generator=g, device="cuda") * spread).to(dtype)[1:]

    params = [odd(n, dt, 0.02) for n, (dt, _) in zip(sizes, kinds)]
    opt = binding.AdamW(params, grads=[odd(n, dt, 1e-3) for n, (_, dt) in zip(sizes, kinds)], state_bits=bits, nearest_steps=1)
    assert opt.m.numel() * 10 > PAST
    opt.step()
    for _ in range(2):
        for t in opt._grads:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda") * 1e-3)
        before = None if bits == 32 else [t.clone() for t in (opt.m, opt.m_exp, opt.v, opt.v_exp)]
        check_step(opt)
    m, v = opt.moments()
    if bits == 32:
        return
    want = decode(opt)
    assert torch.equal(m, want[0]) and torch.equal(v, want[1])
    # codes of the last step, of pieces of every tensor, by what the moments before it and the gradients bound them to
    opt.m, opt.m_exp, opt.v, opt.v_exp, now = *before, (m, v)
    old = decode(opt)
    for o, n, t in zip(opt.offsets, sizes, opt._grads):
        gr = t.double()
        for x, was, beta, term in ((now[0], old[0], 0.9, gr), (now[1], old[1], 0.999, gr * gr)):
            new = beta * was[o:o + n].double() + (1 - beta) * term
            # a step of the codes is at most 1/8 of the value, or 2^-9 of e4m3's least power of two under the group's 2^8
            top = torch.nn.functional.pad(new.abs(), (0, -n % 32)).view(-1, 32).amax(1).repeat_interleave(32)[:n]
            assert ((x[o:o + n].double() - new).abs() <= new.abs() * (1 / 8 + 1e-6) + top * 2.0**-16).all()


def test_codes_beyond_32_bits():
    n, tail = 2**32 + 4099, 4096 + 3                 # the last whole groups of 32, and what is left
    g = (torch.randn(tail, generator=torch.Generator().manual_seed(6)) * 1e-3).to(BF16)
    p, grad = torch.zeros(n, device="cuda", dtype=BF16), torch.zeros(n, device="cuda", dtype=BF16)
    grad[-tail:] = g.cuda()
    b1, b2 = 1 - 2.0**-4, 1 - 2.0**-10               # products of these are exact, see the tests of codes
    opt = binding.AdamW([p], grads=[grad], betas=(b1, b2), state_bits=8, master=False, weight_decay=0.0, nearest_steps=0)
    for _ in range(2):
        opt.step()
    x = np.concatenate([g.float().numpy(), np.zeros(-tail % 32, np.float32)])
    at = n - tail
    assert at % 32 == 0 and at == 2**32
    codes = moments8.encode(np.zeros_like(x), np.zeros_like(x))
    for t in (1, 2):
        m, v = (y.astype(np.float32) for y in moments8.decode(*codes))
        m = np.float32(b1) * m + np.float32(1 - b1) * x
        v = np.float32(b2) * v + np.float32(1 - b2) * (x * x)
        codes = moments8.encode(m, v, moments8.random_bits(t, at + np.arange(len(x))))
    got = [opt.m.view(torch.uint8)[at:at + len(x)], opt.m_exp[at // 32:(at + len(x)) // 32], opt.v[at:at + len(x)],
           opt.v_exp[at // 32:(at + len(x)) // 32]]
    for a, b in zip(got, codes):
        assert np.array_equal(a.cpu().numpy(), b)
    assert (p[-tail:] != 0).sum() == (g != 0).sum() and not p[:4096].any() and not p[at - 4096:at].any()
    m, v = opt.moments()
    for a, b in zip((m, v), moments8.decode(*codes)):
        assert np.array_equal(a[at:at + len(x)].cpu().double().numpy(), b) and not a[at - 4096:at].any()
    del opt, p, grad, m, v
    torch.cuda.empty_cache()
