"""Buffers of 8-bit moments beyond 2^32 bytes."""
import numpy as np
import pytest
import torch

from paper_2601_04342_amd import binding
from tests import moments8

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


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
