"""A distillation step as it is used: rotary positions, forward pass, loss, gradients of the feature maps, AdamW, and
rotary positions in front of the streaming step.  Each operator has tests of its own; here they run together."""
import numpy as np
import pytest
import torch

from oracle import grad as ograd
from paper_2601_04342_amd import binding, synth
from tests import parity
from tests.test_gpu_backward import check_grads

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def setup(B=1, H=2, T=4, rows=6, cols=11, d=64, seed=0):
    """Token-major projections, head-major values, the teacher's output (plain softmax attention on the rotated
    queries and keys) and feature maps."""
    HW = rows * cols
    q, k, v = synth.make_qkv(B, H, T * HW, d, seed=seed)
    phi = binding.phi_to_device(synth.make_phi(H, d, seed=seed + 1, gain=6.0))
    qt, kt = (x.transpose(1, 2).contiguous().to("cuda", BF16).transpose(1, 2) for x in (q, k))
    dv = v.to("cuda", BF16)
    plan = binding.Rope.video(d)
    qr, kr = binding.rope(qt, kt, plan, grid=(rows, cols))
    y = binding.forward(qr, kr, dv, phi, T, HW, T)
    return dict(q=qt, k=kt, v=dv, y=y, phi=phi, T=T, HW=HW, plan=plan, grid=(rows, cols), qr=qr, kr=kr)


def copy_phi(phi):
    return {n: t.clone() for n, t in phi.items()}


@pytest.mark.parametrize("overlap", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_the_whole_chain(d, overlap):
    """Against the gradient oracle on the rotated inputs, with the loss's own gradient (its signs are of differences of
    bf16 outputs, which the oracle's 64-bit ones need not share)."""
    s = setup(B=2, d=d, seed=3)
    T, HW = s["T"], s["HW"]
    grads = {n: torch.full(t.shape, float("nan"), device="cuda") for n, t in s["phi"].items()}
    loss = binding.distill_gradients(s["q"], s["k"], s["v"], s["y"], s["phi"], grads, T, HW, 1, overlap=overlap,
                                     rope_plan=s["plan"], grid=s["grid"], scale=1.0 / 65536)
    out = binding.forward(s["qr"], s["kr"], s["v"], s["phi"], T, HW, 1, overlap=overlap)
    want, g = binding.distill_loss(out, s["y"], scale=1.0 / 65536)
    assert torch.equal(loss, want) and loss.item() > 0
    n64 = lambda t: t.float().cpu().double().numpy()
    ref, y_ref = ograd.phi_backward(n64(s["qr"]), n64(s["kr"]), n64(s["v"]), {n: n64(t) for n, t in s["phi"].items()},
                                    n64(g), T, HW, 1, overlap, hidden_round="bf16")
    assert np.abs(n64(out) - y_ref).max() <= parity.OUT_MAX_ABS
    check_grads(grads, ref, f"d{d} overlap{overlap}")


@pytest.mark.parametrize("bits", [32, 8])
def test_step_is_its_parts(bits):
    s = setup(seed=5)
    T, HW = s["T"], s["HW"]
    phi, mine = copy_phi(s["phi"]), copy_phi(s["phi"])
    opt, ref = binding.AdamW(phi, state_bits=bits), binding.AdamW(mine, state_bits=bits)
    losses = []
    for i in range(4):
        loss = binding.distill_step(s["q"], s["k"], s["v"], s["y"], phi, opt, T, HW, 1, overlap=1, rope_plan=s["plan"],
                                    grid=s["grid"], scale=1e-2)
        qr, kr = binding.rope(s["q"], s["k"], s["plan"], grid=s["grid"])
        out, comps = binding.forward(qr, kr, s["v"], mine, T, HW, 1, overlap=1, debug=True)
        want, g = binding.distill_loss(out, s["y"], scale=1e-2)
        binding.phi_backward(qr, kr, s["v"], mine, g, T, HW, 1, overlap=1, saved=(out, comps["nS"], comps["nL"]),
                             grads=ref.grads)
        ref.step()
        losses.append(loss.item())
        assert torch.equal(loss, want) and all(torch.equal(phi[n], mine[n]) for n in phi), i
    assert all(not torch.equal(phi[n], s["phi"][n]) for n in phi)
    assert int(opt.step_count.item()) == 4 and all(np.isfinite(losses))


def test_blocks_share_an_optimiser():
    """Three blocks, one launch of the update; the same as an optimiser for each."""
    parts = [setup(seed=10 + i) for i in range(3)]
    T, HW = parts[0]["T"], parts[0]["HW"]
    shared, alone = ([copy_phi(p["phi"]) for p in parts] for _ in range(2))
    opt, opts = binding.AdamW(shared), [binding.AdamW(phi) for phi in alone]
    for _ in range(2):
        for i, p in enumerate(parts):
            args = (p["qr"], p["kr"], p["v"], p["y"])
            binding.distill_gradients(*args, shared[i], opt.grads[i], T, HW, 1)
            binding.distill_step(*args, alone[i], opts[i], T, HW, 1)
        opt.step()
    assert all(torch.equal(a[n], b[n]) for a, b in zip(shared, alone) for n in a)


def test_padded_clips_do_not_count():
    """A clip shorter than its batch: what its padding tokens' outputs are does not reach loss or gradients."""
    s = setup(B=2, seed=7)
    T, HW = s["T"], s["HW"]
    weight = torch.ones(2, T * HW, device="cuda")
    weight[1, 2 * HW:] = 0
    got = []
    for fill in (0.0, float("nan")):
        y = s["y"].clone()
        y[1, :, 2 * HW:] = fill
        grads = {n: torch.empty(t.shape, device="cuda") for n, t in s["phi"].items()}
        loss = binding.distill_gradients(s["qr"], s["kr"], s["v"], y, s["phi"], grads, T, HW, 1, weight=weight)
        got.append((loss, grads))
    assert torch.isfinite(got[0][0]) and torch.equal(got[0][0], got[1][0])
    assert all(torch.equal(got[0][1][n], got[1][1][n]) and torch.isfinite(got[0][1][n]).all() for n in s["phi"])


@pytest.mark.parametrize("bits", [32, 8])
def test_step_replays_from_a_graph(bits):
    """A captured step goes on learning with every replay, beside eager work, as eager steps do."""
    s = setup(seed=8)
    T, HW = s["T"], s["HW"]
    phi, mine = copy_phi(s["phi"]), copy_phi(s["phi"])
    opt, ref = binding.AdamW(phi, state_bits=bits), binding.AdamW(mine, state_bits=bits)
    step = lambda p, o: binding.distill_step(s["q"], s["k"], s["v"], s["y"], p, o, T, HW, 1, rope_plan=s["plan"],
                                             grid=s["grid"], scale=1e-2)
    step(phi, opt), step(mine, ref)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = step(phi, opt)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = step(mine, ref)
        assert torch.equal(loss, want) and all(torch.equal(phi[n], mine[n]) for n in phi), i
        binding.forward(s["qr"], s["kr"], s["v"], mine, T, HW, 2)     # the same library workspace
        torch.cuda.synchronize()
    assert int(opt.step_count.item()) == 5


def test_step_on_another_stream():
    s = setup(seed=9)
    T, HW = s["T"], s["HW"]
    phi, mine = copy_phi(s["phi"]), copy_phi(s["phi"])
    opt, ref = binding.AdamW(phi), binding.AdamW(mine)
    args = (s["q"], s["k"], s["v"], s["y"])
    kw = dict(rope_plan=s["plan"], grid=s["grid"])
    side = torch.cuda.Stream()
    want = [binding.distill_step(*args, mine, ref, T, HW, 1, **kw) for _ in range(3)]
    side.wait_stream(torch.cuda.current_stream())
    got = [binding.distill_step(*args, phi, opt, T, HW, 1, stream=side, **kw) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(phi[n], mine[n]) for n in phi)


@pytest.mark.parametrize("overlap", [0, 1])
def test_streaming_with_rotated_windows(overlap):
    """Generation frame by frame: each frame's queries and keys are rotated at its own place, the keys straight into the
    window that slides over them; the same as the whole video at once."""
    s = setup(T=5, rows=7, cols=9, seed=12)
    T, HW, d = s["T"], s["HW"], 64
    B, H = s["q"].shape[:2]
    whole = binding.forward(s["qr"], s["kr"], s["v"], s["phi"], T, HW, 1, overlap=overlap)
    S, z = torch.zeros(B, H, 2 * d, d, device="cuda"), torch.zeros(B, H, 2 * d, device="cuda")
    plan = binding.chunk_plan(T, HW, 1, overlap).tolist()
    last = None
    for t, (lo, hi, s_lo, s_hi, _) in enumerate(plan):
        kw = torch.empty(B, H, s_hi - s_lo, d, device="cuda", dtype=BF16)
        if lo > s_lo:
            kw[:, :, :lo - s_lo] = last
        q_t = torch.empty(B, H, HW, d, device="cuda", dtype=BF16)
        binding.rope(s["q"][:, :, lo:hi], s["k"][:, :, lo:hi], s["plan"], grid=s["grid"], start=t,
                     out=(q_t, kw[:, :, lo - s_lo:]))
        absorb = plan[t + 1][2] - s_lo if t + 1 < T else 0
        y = binding.step(q_t, kw, s["v"][:, :, s_lo:s_hi].contiguous(), s["phi"], S, z, absorb)
        assert torch.equal(q_t, s["qr"][:, :, lo:hi]) and torch.equal(kw, s["kr"][:, :, s_lo:s_hi])
        err = (y.float() - whole[:, :, lo:hi].float()).abs()
        assert err.max().item() <= parity.OUT_MAX_ABS and err.mean().item() <= parity.OUT_MEAN_ABS
        last = kw[:, :, kw.shape[2] - HW * overlap:] if overlap else None


def test_refusals():
    s = setup(seed=13)
    T, HW = s["T"], s["HW"]
    phi, opt = s["phi"], binding.AdamW(copy_phi(s["phi"]))
    args = (s["q"], s["k"], s["v"], s["y"])
    with pytest.raises(ValueError):                                  # an optimiser over other tensors
        binding.distill_step(*args, phi, opt, T, HW, 1, rope_plan=s["plan"], grid=s["grid"])
    with pytest.raises(ValueError):
        binding.distill_step(*args, phi, binding.AdamW([phi]), T, HW, 1)
    grads = opt.grads
    mine = copy_phi(s["phi"])
    moved = binding.AdamW(mine)
    moved.grads["w1_q"] = moved.grads["w1_q"].clone()                # a gradient that the update would not read
    with pytest.raises(ValueError):
        binding.distill_step(*args, mine, moved, T, HW, 1, rope_plan=s["plan"], grid=s["grid"])
    with pytest.raises(TypeError):                                   # token-major without a rotation
        binding.distill_gradients(*args, phi, grads, T, HW, 1)
    with pytest.raises(ValueError):
        binding.distill_gradients(*args, phi, grads, T, HW, 1, rope_plan=s["plan"], grid=(HW, 2))
    with pytest.raises(ValueError):
        binding.distill_gradients(s["qr"], s["kr"], s["v"], s["y"], phi, grads, T, HW, 1, start=3)
    with pytest.raises(ValueError):
        binding.distill_gradients(s["qr"], s["kr"], s["v"], s["y"], phi, grads, T + 1, HW, 1)
    assert int(opt.step_count.item()) == 0
