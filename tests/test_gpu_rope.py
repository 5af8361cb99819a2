"""Rotary positions (rehyat_rope) against the rotation written out in 64 bits: layouts, part of the head, types, axes and
kinds of positions, strides, single tokens, far positions, the inverse as transpose and as gradient, streams and graphs."""
import math

import pytest
import torch

from paper_2601_04342_amd import binding

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def reference(x, freqs, sections, pos, layout, mu=1.0, inverse=False):
    """x: [B, H, N, d] on any device; pos: integers [B, N, axes] -> (rotated in 64 bits on the CPU, sum of the absolute
    values that enter each element)."""
    x = x.detach().cpu().double()
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    # the angle modulo a turn, from whole positions: exact products of a 53-bit and a 31-bit number need more than 64
    # bits, so positions are split at 2^20
    p = pos.cpu()[..., axis]
    hi, lo = p // 2**20, p % 2**20
    turn = freqs / (2 * math.pi)
    step = torch.remainder(turn * 2**20, 1.0)
    angle = 2 * math.pi * torch.remainder(torch.remainder(hi.double() * step, 1.0) + torch.remainder(lo.double() * turn, 1.0), 1.0)
    c, s = (f(angle)[:, None] * mu for f in (torch.cos, torch.sin))
    s = -s if inverse else s
    r = 2 * len(freqs)
    out, size = x.clone(), x.abs()
    i, j = (slice(0, r, 2), slice(1, r, 2)) if layout == "interleaved" else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., i], x[..., j]
    out[..., i], out[..., j] = a * c - b * s, b * c + a * s
    size[..., i] = size[..., j] = a.abs() + b.abs()
    return out, size


def check(got, want, size, mu=1.0, label=""):
    """cos and sin are each off by at most 2^-22 (the angle's rounding to 24 bits, of at most 0.79: 2^-24.3; 2^-32 turns
    cut off; two roundings of the series), each of the two products and their sum rounds by 2^-24 of the terms: together
    below 2^-21 mu (|a| + |b|), and one rounding to the type (half a step; in fp16 at least half of 2^-24)."""
    eps = torch.finfo(got.dtype).eps
    tiny = 2.0**-25 if got.dtype == FP16 else 2.0**-134
    err = (got.detach().cpu().double() - want).abs()
    most = (1 + eps) * (eps / 2 * want.abs() + tiny) + 2.0**-21 * mu * size
    worst = (err / most).max().item()
    assert worst <= 1, (label, worst)


def grid_positions(N, grid, start, B=1):
    n = torch.arange(N)
    if len(grid) == 0:
        p = (n + start)[:, None]
    elif len(grid) == 1:
        p = torch.stack([n // grid[0] + start, n % grid[0]], 1)
    else:
        p = torch.stack([n // (grid[0] * grid[1]) + start, n // grid[1] % grid[0], n % grid[1]], 1)
    return p[None].expand(B, -1, -1)


def operand(B, H, N, d, dtype, seed, token_major=True):
    g = torch.Generator().manual_seed(seed)
    if token_major:
        return torch.randn(B, N, H, d, generator=g).to("cuda", dtype).transpose(1, 2)
    return torch.randn(B, H, N, d, generator=g).to("cuda", dtype)


def nan_out(x):
    return torch.full(x.shape, float("nan"), device=x.device, dtype=x.dtype)


def run(plan, B, Hq, Hk, N, dtype, grid=(), start=0, inverse=False, token_major=True, seed=0):
    q, k = (operand(B, H, N, plan.d, dtype, seed + i, token_major) for i, H in enumerate((Hq, Hk)))
    out = binding.rope(q, k, plan, grid=grid or None, start=start, inverse=inverse, out=(nan_out(q), nan_out(k)))
    pos = grid_positions(N, grid, start, B)
    for x, y in zip((q, k), out):
        assert y.shape == x.shape and y.dtype == x.dtype
        want, size = reference(x, plan.freqs, plan.sections, pos, plan.layout, plan.scale, inverse)
        check(y, want, size, plan.scale, (plan.layout, dtype))
        assert torch.equal(y[..., plan.rot:], x[..., plan.rot:])
    return q, k, out


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("d,rot", [(128, 128), (64, 64), (128, 64), (96, 40), (80, 46), (2, 2), (6, 4), (256, 256),
                                   (512, 512), (512, 2), (72, 66), (64, 16), (10, 6), (34, 32)])
def test_layouts_types_and_parts_of_the_head(d, rot, layout, dtype, inverse):
    run(binding.Rope(d, rot=rot, layout=layout), 2, 3, 2, 37, dtype, start=11, inverse=inverse, seed=d + rot)


@pytest.mark.parametrize("B,Hq,Hk,N", [(1, 1, 1, 1), (16, 24, 24, 1), (3, 5, 1, 2), (1, 12, 12, 257), (5, 17, 3, 63),
                                       (1, 1, 40, 1000), (300, 2, 1, 3), (2, 40, 8, 64), (1, 9, 9, 4097)])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_sizes(B, Hq, Hk, N, layout):
    for d, token_major in ((128, True), (64, False)):
        run(binding.Rope(d, layout=layout), B, Hq, Hk, N, BF16, token_major=token_major, seed=N)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("N,grid,start", [(4 * 7 * 9, (7, 9), 0), (250, (7, 9), 13), (1, (30, 52), 20), (100, (64, 64), 3),
                                          (333, (1, 1), 5), (77, (5, 1), 0)])
def test_three_axes(N, grid, start, layout, d):
    """Frames, rows and columns, also where the last frame is not full or the frame is larger than what is there."""
    run(binding.Rope.video(d, layout=layout), 2, 3, 3, N, BF16, grid=grid, start=start, seed=N)


def test_two_axes():
    run(binding.Rope(64, sections=(9, 23)), 2, 2, 3, 130, FP32, grid=(12,), start=4)


@pytest.mark.parametrize("scaling,changed", [
    (dict(kind="linear", factor=4.0), lambda f, n: f / 4),
    (dict(kind="base", factor=4.0), lambda f, n: (10000.0 * 4 ** (n / (n - 1))) ** (-torch.arange(n, dtype=torch.float64) / n)),
    (dict(kind="parts", factor=8.0, original=4096), None),
])
def test_scaled_frequencies(scaling, changed):
    plain = binding.Rope(128).freqs
    plan = binding.Rope(128, scaling=scaling, layout="half")
    if changed is not None:
        assert torch.allclose(plan.freqs, changed(plain, 64), rtol=1e-14) and plan.scale == 1.0
    else:
        turns = 4096 * plain / (2 * math.pi)
        for i in range(64):
            part = min(max((turns[i].item() - 1) / 31, 0.0), 1.0)
            assert math.isclose(plan.freqs[i].item(), plain[i].item() * part + plain[i].item() / 8 * (1 - part), rel_tol=1e-13)
        assert plan.freqs[0] == plain[0] and plan.freqs[-1] == plain[-1] / 8
        assert math.isclose(plan.scale, 0.1 * math.log(8.0) + 1)
    run(plan, 1, 2, 2, 100, FP32, start=30000)


def test_base_scaling_keeps_the_fastest_pair_and_divides_the_slowest():
    plain, scaled = binding.Rope(128).freqs, binding.Rope(128, scaling=dict(kind="base", factor=4.0)).freqs
    assert scaled[0] == plain[0] and math.isclose(scaled[-1].item(), plain[-1].item() / 4, rel_tol=1e-12)


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("axes", [1, 2, 3])
def test_explicit_positions(dtype, shared, axes):
    B, N, d = 3, 45, 64
    sections = {1: (32,), 2: (10, 22), 3: (12, 10, 10)}[axes]
    plan = binding.Rope(d, sections=sections, layout="half")
    g = torch.Generator().manual_seed(axes)
    pos = torch.randint(-5000, 2**31 - 1, (N, axes) if shared else (B, N, axes), generator=g)
    pos[..., 0, :] = 0
    dev = pos.to("cuda", dtype)
    q, k = operand(B, 4, N, d, FP32, 1), operand(B, 2, N, d, FP32, 2, token_major=False)
    out = binding.rope(q, k, plan, positions=dev[..., 0] if axes == 1 else dev)
    full = pos[None].expand(B, -1, -1) if shared else pos
    for x, y in zip((q, k), out):
        want, size = reference(x, plan.freqs, sections, full, "half")
        check(y, want, size)
    assert torch.equal(out[0][:, :, 0], q[:, :, 0])   # position 0 turns nothing


def test_strided_positions_and_expanded_inputs():
    """Every second entry of a position buffer that all sequences share; a gradient that is one row for all heads."""
    B, N, d = 2, 33, 64
    plan = binding.Rope(d)
    store = torch.arange(2 * N, device="cuda", dtype=torch.int32)
    x = operand(1, 1, N, d, FP32, 3).expand(B, 5, N, d)
    y = binding.rope(x, None, plan, positions=store[::2].expand(B, N), inverse=True)
    want, size = reference(x, plan.freqs, plan.sections, 2 * grid_positions(N, (), 0, B), "interleaved", inverse=True)
    check(y, want, size)


def test_far_positions_lose_nothing():
    """The angle is a product modulo a turn: at positions near 2^40 results are as exact as at 0."""
    plan = binding.Rope(64)
    N = 50
    start = 2**40 + 12345
    x = operand(1, 2, N, 64, FP32, 4)
    y = binding.rope(x, None, plan, start=start)
    z = binding.rope(x, None, plan, positions=torch.arange(start, start + N, device="cuda"))
    assert torch.equal(y, z)
    # the frequencies' own 53 bits are 2^-53 of a turn, 1e-4 of a turn at 2^40: the kernel and a calculation in whole
    # numbers of the same 2^-64 parts have to agree far closer
    turns = [int(t) % 2**64 for t in plan.turns.tolist()]
    angle = torch.tensor([[(p * t % 2**64) / 2**64 * 2 * math.pi for t in turns] for p in range(start, start + N)],
                         dtype=torch.float64)
    a, b = x.cpu().double()[..., 0::2], x.cpu().double()[..., 1::2]
    want = torch.stack([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1).flatten(-2)
    check(y, want, torch.stack([a.abs() + b.abs()] * 2, -1).flatten(-2))


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (80, 46)])
def test_in_place(layout, d, rot):
    plan = binding.Rope(d, rot=rot, layout=layout)
    q, k = operand(2, 3, 70, d, BF16, 5), operand(2, 2, 70, d, BF16, 6, token_major=False)
    want = binding.rope(q, k, plan, start=9)
    out = binding.rope(q, k, plan, start=9, out=(q, k))
    assert out[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("offset", [0, 1, 3, 4])
def test_parts_of_larger_buffers(offset, dtype):
    """q, k and v in one projection, out into rows of a K window at any element offset: nothing else is written."""
    B, H, N, d, win = 2, 3, 29, 64, 50
    plan = binding.Rope(d, layout="half")
    g = torch.Generator().manual_seed(7)
    flat = torch.randn(B * N * 3 * H * d + 8, generator=g).to("cuda", dtype)
    qkv = flat[offset:offset + B * N * 3 * H * d].view(B, N, 3, H, d)
    q, k = qkv[:, :, 0].transpose(1, 2), qkv[:, :, 1].transpose(1, 2)
    store = torch.full((B * H * win * d + 8,), 7.0, device="cuda", dtype=dtype)
    window = store[offset:offset + B * H * win * d].view(B, H, win, d)
    q_out = nan_out(q)
    binding.rope(q, k, plan, start=100, out=(q_out, window[:, :, 13:13 + N]))
    pos = grid_positions(N, (), 100, B)
    for x, y in ((q, q_out), (k, window[:, :, 13:13 + N])):
        want, size = reference(x, plan.freqs, plan.sections, pos, "half")
        check(y, want, size)
    assert (window[:, :, :13] == 7).all() and (window[:, :, 13 + N:] == 7).all()
    assert (store[:offset] == 7).all() and (store[offset + B * H * win * d:] == 7).all()


def test_long_cache_rows_beyond_32_bit_offsets():
    """Rows of a window that stand more than 2^32 bytes apart."""
    B, H, N, d = 2, 2, 3, 64
    plan = binding.Rope(d)
    far = 2**31 + 8 * d                                # elements between sequences: 2^32 bytes and more
    store = torch.empty(far + 64 * d, device="cuda", dtype=BF16)
    window = store.as_strided((B, H, N, d), (far, 16 * d, d, 1))
    store[:64 * d] = 0
    store[far:] = 0
    q = operand(B, H, N, d, BF16, 8)
    binding.rope(q, None, plan, start=3, out=window)
    want, size = reference(q, plan.freqs, plan.sections, grid_positions(N, (), 3, B), "interleaved")
    check(window, want, size)
    back = binding.rope(window, None, plan, start=3, inverse=True)
    check(back, *reference(window, plan.freqs, plan.sections, grid_positions(N, (), 3, B), "interleaved", inverse=True))


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_infinities_and_nan_stay_in_their_pair(layout):
    d, rot = 64, 48
    plan = binding.Rope(d, rot=rot, layout=layout)
    q = operand(1, 2, 20, d, BF16, 9).contiguous()
    clean = binding.rope(q, None, plan, start=1)
    q[0, 0, 4, 6] = float("nan")
    q[0, 1, 7, rot + 3] = float("inf")
    q[0, 1, 9, 5] = float("-inf")
    got = binding.rope(q, None, plan, start=1)
    i, j = (6, 7) if layout == "interleaved" else (6, 6 + rot // 2)
    m, n = (4, 5) if layout == "interleaved" else (5, 5 + rot // 2)
    assert torch.isnan(got[0, 0, 4, [i, j]]).all() and torch.isinf(got[0, 1, 9, [m, n]]).all()
    assert got[0, 1, 7, rot + 3] == float("inf")
    touched = torch.zeros_like(got, dtype=torch.bool)
    for h, t, cols in ((0, 4, (i, j)), (1, 7, (rot + 3,)), (1, 9, (m, n))):
        touched[0, h, t, list(cols)] = True
    assert torch.equal(got[~touched], clean[~touched])


@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_inverse_is_the_gradient(layout):
    """Against differences of the rotation itself (it is linear, so a step of any size will do) and as its transpose."""
    plan = binding.Rope(32, rot=20, layout=layout, scaling=dict(kind="parts", factor=4.0, original=100))
    x, g = operand(1, 2, 9, 32, FP32, 10), operand(1, 2, 9, 32, FP32, 11)
    grad = binding.rope(g, None, plan, start=50, inverse=True).double()
    y = binding.rope(x, None, plan, start=50).double()
    left, right = (g.double() * y).sum().item(), (grad * x.double()).sum().item()
    assert abs(left - right) <= 2.0**-20 * (g.double().abs() * y.abs()).sum().item()
    for h, n, c in ((0, 0, 0), (1, 8, 19), (0, 3, 10), (1, 5, 25), (0, 7, 1)):
        e = x.clone()
        e[0, h, n, c] += 1.0
        d = (binding.rope(e, None, plan, start=50).double() - y) / (e[0, h, n, c] - x[0, h, n, c]).item()
        want = (g.double() * d).sum().item()
        assert abs(want - grad[0, h, n, c].item()) <= 2.0**-17, (h, n, c)   # 32 elements of about 1, 2^-22 each


def test_turning_back_gives_the_input():
    plan = binding.Rope.video(128)
    q = operand(2, 3, 200, 128, FP32, 12)
    y = binding.rope(q, None, plan, grid=(5, 8), start=2)
    z = binding.rope(y, None, plan, grid=(5, 8), start=2, inverse=True)
    size = q.abs()[..., 0::2] + q.abs()[..., 1::2]
    size = torch.stack([size, size], -1).flatten(-2)
    assert ((z - q).abs() <= 2.0**-19 * size + 2.0**-23 * q.abs()).all()   # twice the bound of one rotation


def test_another_stream_and_back():
    plan = binding.Rope(128)
    q = operand(1, 4, 500, 128, BF16, 13)
    want = binding.rope(q, None, plan)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [binding.rope(q, None, plan, stream=side) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(x, want) for x in got)


def test_graph_replays_with_new_positions():
    """A captured step for single tokens reads its positions from device memory at every replay."""
    B, H, d = 4, 6, 64
    plan = binding.Rope(d, layout="half")
    q, k = operand(B, H, 1, d, BF16, 14), operand(B, 2, 1, d, BF16, 15)
    pos = torch.zeros(B, 1, device="cuda", dtype=torch.int64)
    out = (nan_out(q), nan_out(k))
    step = lambda: binding.rope(q, k, plan, positions=pos, out=out)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        pos.copy_(torch.tensor([[5], [70000 + i], [i], [2**33 + i]]))
        for t in out:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = binding.rope(q, k, plan, positions=pos.clone())
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]), i


def test_refusals_on_the_device_side_of_the_binding():
    plan = binding.Rope(64)
    q = operand(2, 3, 8, 64, BF16, 16)
    for bad in (dict(out=q[:, :, :4]), dict(out=torch.empty_like(q, dtype=FP32))):
        with pytest.raises(TypeError):
            binding.rope(q, None, plan, **bad)
    with pytest.raises(TypeError):
        binding.rope(q.transpose(2, 3), None, plan)
    with pytest.raises(ValueError):
        binding.rope(q[..., :32], None, plan)
    with pytest.raises(ValueError):
        binding.rope(q, q[:, :, :4], plan)
    with pytest.raises(ValueError):
        binding.rope(q, None, plan, positions=torch.zeros(3, 8, device="cuda", dtype=torch.int64))
    with pytest.raises(TypeError):
        binding.rope(q, None, plan, positions=torch.zeros(8, device="cuda"))
    with pytest.raises(TypeError):
        binding.rope(q, None, plan, positions=torch.zeros(8, dtype=torch.int64))
    with pytest.raises(ValueError):
        binding.rope(q, None, binding.Rope(64, device="cpu"))
    with pytest.raises(binding.RehyatError) as e:      # every head into the same row
        binding.rope(q, None, plan, out=torch.empty(2, 1, 8, 64, device="cuda", dtype=BF16).expand(2, 3, 8, 64))
    assert e.value.code == binding.E_SHAPE
    torch.cuda.synchronize()


def test_queries_and_keys_of_one_projection_in_place():
    """Each in place, between the other's rows; the values beside them stay."""
    B, H, N, d = 2, 3, 40, 64
    plan = binding.Rope(d)
    qkv = operand(B, 3 * H, N, d, BF16, 17).transpose(1, 2).reshape(B, N, 3, H, d).contiguous()
    was = qkv.clone()
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    want = binding.rope(q, k, plan, start=7)
    binding.rope(q, k, plan, start=7, out=(q, k))
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, 2], was[:, :, 2])
    for out in ((k, q), (q, q), (v, q)):     # exchanged, one for both, onto what the other reads
        with pytest.raises(binding.RehyatError) as e:
            binding.rope(q, k, plan, out=out)
        assert e.value.code == binding.E_SHAPE
    torch.cuda.synchronize()


def test_queries_and_keys_that_are_one_tensor():
    plan = binding.Rope(64)
    x = operand(1, 2, 30, 64, BF16, 18)
    a, b = binding.rope(x, x, plan, start=2)
    assert torch.equal(a, b) and torch.equal(a, binding.rope(x, None, plan, start=2))


def test_nothing_to_rotate_is_refused():
    plan = binding.Rope(64)
    x = operand(2, 3, 8, 64, BF16, 19)
    for empty in (x[:0], x[:, :0], x[:, :, :0]):
        with pytest.raises(binding.RehyatError):
            binding.rope(empty, None, plan)
    with pytest.raises(ValueError):
        binding.rope(x, None, plan, start=2**63)
