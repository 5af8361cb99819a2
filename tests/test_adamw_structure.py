"""Which gradient belongs to which parameter of an AdamW, and what a state that is loaded replaces."""
import pytest
import torch

from paper_2601_04342_amd import binding, synth


def test_gradients_are_found_by_their_keys():
    t = [torch.zeros(1) for _ in range(8)]
    params = {"a": t[0], "b": [t[1], {"x": t[2], "y": t[3]}]}
    grads = {"b": (t[5], {"y": t[7], "x": t[6]}), "a": t[4]}
    got = binding._leaves_like(params, grads)
    assert len(got) == 4 and all(a is b for a, b in zip(got, t[4:]))
    for bad in ({"a": t[4]}, {"a": t[4], "b": (t[5],)}, {"a": t[4], "c": grads["b"]}, [t[4], grads["b"]], t[4],
                {"a": [t[4]], "b": grads["b"]}, {"a": t[4], "b": (t[5], t[6])}, {**grads, "c": t[7]}):
        with pytest.raises(ValueError):
            binding._leaves_like(params, bad)


def turned(x):
    """The same dict with queries' and keys' entries in each other's places, which fit in shape."""
    return {m: x[m] for m in (n[:-1] + {"q": "k", "k": "q"}[n[-1]] for n in x)}


@pytest.mark.gpu
def test_a_dict_of_gradients_in_another_order():
    start = binding.phi_to_device(synth.make_phi(2, 64, seed=1))
    want, phi = ({n: t.clone() for n, t in start.items()} for _ in range(2))
    ref = binding.AdamW(want)
    grads = {n: torch.randn(t.shape, generator=torch.Generator().manual_seed(i)).cuda() for i, (n, t) in enumerate(phi.items())}
    for n, g in grads.items():
        ref.grads[n].copy_(g)
    opt = binding.AdamW(phi, grads=turned(grads))
    opt.step(), ref.step()
    assert all(torch.equal(phi[n], want[n]) and not torch.equal(phi[n], start[n]) for n in start)
    with pytest.raises(ValueError):
        binding.AdamW(phi, grads={n: g for n, g in grads.items() if n != "b2_k"})


@pytest.mark.gpu
def test_a_step_of_distillation_goes_by_names():
    B, H, T, HW, d = 1, 2, 4, 60, 64
    q, k, v = (t.to("cuda", torch.bfloat16) for t in synth.make_qkv(B, H, T * HW, d, seed=2))
    start = binding.phi_to_device(synth.make_phi(H, d, seed=3, gain=4.0))
    y = binding.forward(q, k, v, start, T, HW, T)
    want, phi = ({n: t.clone() for n, t in start.items()} for _ in range(2))
    ref = binding.AdamW(want)
    opt = binding.AdamW(phi, grads=turned({n: torch.zeros(t.shape, device="cuda") for n, t in phi.items()}))
    for _ in range(2):
        a = binding.distill_step(q, k, v, y, want, ref, T, HW, 1)
        b = binding.distill_step(q, k, v, y, turned(phi), opt, T, HW, 1)
        assert torch.equal(a, b) and all(torch.equal(phi[n], want[n]) for n in phi)
    swapped = {**phi, "w1_q": phi["w1_k"], "w1_k": phi["w1_q"]}
    with pytest.raises(ValueError):
        binding.distill_step(q, k, v, y, swapped, opt, T, HW, 1)
    opt.grads["w1_q"], opt.grads["w1_k"] = opt.grads["w1_k"], opt.grads["w1_q"]
    with pytest.raises(ValueError):
        binding.distill_step(q, k, v, y, phi, opt, T, HW, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_a_state_without_fp32_copies(bits):
    """A checkpoint's weights are copied into the parameters, its moments loaded: the next step starts from those weights."""
    g = torch.Generator().manual_seed(4)
    weights = (torch.randn(700, generator=g) * 0.02).to("cuda", torch.bfloat16)
    grad = torch.randn(700, generator=g).cuda() * 1e-3
    fresh = binding.AdamW([weights.clone()], state_bits=bits)
    resumed = binding.AdamW([torch.zeros_like(weights)], state_bits=bits)
    resumed.params[0].copy_(weights)
    resumed.load_state(fresh.m, fresh.v, 0, m_exp=fresh.m_exp, v_exp=fresh.v_exp)
    for o in (fresh, resumed):
        o._grads[0].copy_(grad)
        o.step()
    assert torch.equal(fresh.master, resumed.master) and torch.equal(fresh.params[0], resumed.params[0])


def test_a_step_that_is_no_count_is_refused_before_anything_is_copied():
    opt = binding.AdamW.__new__(binding.AdamW)      # its buffers on the host
    opt.m, opt.v, opt.m_exp, opt.v_exp, opt.master = torch.zeros(4), torch.zeros(4), None, None, None
    opt.params, opt.master_offsets, opt.step_count = [], [], torch.zeros((), dtype=torch.int64)
    for bad in (-1, 2**63):
        with pytest.raises(ValueError):
            opt.load_state(torch.ones(4), torch.ones(4), bad)
        assert (opt.m == 0).all() and (opt.v == 0).all()
    opt.load_state(torch.ones(4), torch.ones(4), 2**63 - 1)
    assert (opt.m == 1).all() and opt.step_count.item() == 2**63 - 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_copies_of_leaves_are_no_part_of_their_graphs(dtype):
    g = torch.Generator().manual_seed(5)
    start = [(torch.randn(3, 70, generator=g) * 0.02).to("cuda", dtype), torch.ones((), device="cuda", dtype=dtype),
             torch.randn(5, generator=g).cuda(), torch.zeros(0, 4, device="cuda", dtype=dtype)]
    opt = binding.AdamW([torch.nn.Parameter(t.clone()) for t in start])
    plain = binding.AdamW([t.clone() for t in start])
    for o in (opt, plain):
        for i, t in enumerate(o._grads):
            t.fill_(1e-3 * (i + 1))
        o.step()
        o.reset_master()
        o.load_state(o.m.clone(), o.v.clone(), 1)
        o.step()
        assert not any(t.requires_grad for t in (o.master, o.m, o.v))
    assert torch.equal(opt.master, plain.master) and all(torch.equal(a, b) for a, b in zip(opt.params, plain.params))
