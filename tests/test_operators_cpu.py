"""Refusals and host arithmetic of the operators around the attention, without a GPU: every rejected call returns before
it touches the device (the pointers below are fake and never dereferenced)."""
import ctypes
import math

import pytest
import torch

from paper_2601_04342_amd import binding

A = 0x1000


# ---- rotary positions ---------------------------------------------------------------------------------------------


def rope_call(n_ops=1, B=2, N=8, type_=0, inverse=0, heads=3, x=A, out=2 * A, xs=None, os_=None, plan=None, pos=None,
              second=None, **fields):
    d = fields.get("d", 64)
    p = binding.RopePlan(A, d, d, 0, 1, (ctypes.c_int32 * 3)(d // 2, 0, 0), 1.0)
    if "d" in fields:
        p.section[0] = fields.get("rot", d) // 2
    for name, v in fields.items():
        if name == "section":
            p.section = (ctypes.c_int32 * 3)(*v)
        else:
            setattr(p, name, v)
    ops = (binding.RopeOperand * 2)()
    for i in range(2):
        ops[i] = binding.RopeOperand(x, out + i * A, *(xs or (heads * N * d, N * d, d)), *(os_ or (heads * N * d, N * d, d)),
                                     heads)
    if second is not None:
        for name, v in second.items():
            setattr(ops[1], name, v)
    return binding.library().rehyat_rope(ops, n_ops, ctypes.byref(p) if plan is None else plan,
                                         ctypes.byref(binding.RopePositions() if pos is None else pos), B, N, type_,
                                         inverse, None)


@pytest.mark.parametrize("bad", [
    dict(n_ops=0), dict(n_ops=3), dict(B=0), dict(N=0), dict(type_=3), dict(type_=-1), dict(inverse=2),
    dict(d=1, rot=2), dict(d=514), dict(d=65, rot=64), dict(rot=66), dict(rot=0), dict(rot=31), dict(layout=2), dict(axes=0), dict(axes=4),
    dict(section=(31, 0, 0)), dict(axes=2, section=(32, 0, 0)), dict(axes=2, section=(33, -1, 0)), dict(scale=math.inf),
    dict(scale=math.nan), dict(turns=A + 4), dict(x=A + 1), dict(out=A + 1), dict(type_=2, x=A + 2), dict(heads=0),
    dict(heads=65536), dict(xs=(-1, 512, 64)), dict(xs=(1536, 512, 1 << 40)), dict(os_=(1536, 512, 32)),
    dict(os_=(1536, 0, 64)), dict(os_=(0, 512, 64)), dict(os_=(1500, 512, 64)), dict(B=1 << 16, N=1 << 15),
    dict(B=1 << 15, N=1 << 10), dict(n_ops=2, second=dict(out=2 * A)), dict(n_ops=2, second=dict(heads=0)),
])
def test_rope_rejects(bad):
    assert rope_call(**bad) == binding.E_SHAPE


def test_rope_rejects_null_and_bad_positions():
    lib = binding.library()
    assert rope_call(turns=None) == binding.E_NULL
    assert rope_call(x=None) == binding.E_NULL
    assert rope_call(n_ops=2, second=dict(out=None)) == binding.E_NULL
    assert lib.rehyat_rope(None, 1, None, None, 1, 1, 0, 0, None) == binding.E_NULL
    P = binding.RopePositions
    three = dict(axes=3, section=(12, 10, 10))
    for pos in (P(rows=3), P(cols=4), P(rows=-1, cols=4)):
        assert rope_call(pos=pos, **three) == binding.E_SHAPE
    assert rope_call(pos=P(cols=0), axes=2, section=(16, 16, 0)) == binding.E_SHAPE
    for pos in (P(data=A, bits=16), P(data=A + 4, bits=64), P(data=A + 2, bits=32), P(data=A, bits=32, stride_b=-1),
                P(data=A, bits=32, stride_n=-1)):
        assert rope_call(pos=pos) == binding.E_SHAPE


def test_turns_are_the_frequencies_modulo_a_turn():
    lib = binding.library()

    def turns(*radians):
        f = (ctypes.c_double * len(radians))(*radians)
        t = (ctypes.c_uint64 * len(radians))()
        return lib.rehyat_rope_turns(f, len(radians), t), list(t)

    rc, t = turns(0.0, 1.0, -1.0, math.pi, 2 * math.pi, 100.0, 1e-12)
    assert rc == binding.OK
    # an x87 quotient is off by at most half of 2^-63 of itself; math.pi as a double is 1.2e-16 off pi
    one = 2**64 / (2 * math.pi)
    assert t[0] == 0 and abs(t[1] - one) <= 2**64 * 2.0**-53 and t[1] + t[2] in (2**64 - 1, 2**64, 2**64 + 1)
    assert abs(t[3] - 2**63) <= 2**64 * 2.0**-53 and min(t[4], 2**64 - t[4]) <= 2**64 * 2.0**-52
    assert abs(t[5] - (100 / (2 * math.pi) % 1) * 2**64) <= 2**64 * 2.0**-47 and abs(t[6] - 1e-12 * one) <= 1
    assert turns(math.nan)[0] == binding.E_SHAPE and turns(1.0, math.inf)[0] == binding.E_SHAPE
    assert lib.rehyat_rope_turns(None, 1, (ctypes.c_uint64 * 1)()) == binding.E_NULL
    assert lib.rehyat_rope_turns((ctypes.c_double * 1)(), 0, (ctypes.c_uint64 * 1)()) == binding.E_SHAPE


@pytest.mark.parametrize("bad", [
    dict(rot=3), dict(rot=0), dict(rot=130), dict(d=129, rot=128), dict(layout="other"), dict(sections=(32, 31)), dict(sections=(64, 0)),
    dict(sections=(16, 16, 16, 16)), dict(scaling=dict(kind="no", factor=2.0)), dict(scaling=dict(kind="linear", factor=0.0)),
    dict(scaling=dict(kind="parts", factor=2.0, original=100, low=2, high=2)), dict(freqs=[1.0]),
    dict(freqs=[1.0] * 64, scaling=dict(kind="linear", factor=2.0)),
])
def test_rope_plan_rejects(bad):
    with pytest.raises(ValueError):
        binding.Rope(**{"d": 128, "device": "cpu", **bad})


def test_video_plan_splits_the_pairs():
    for d, want in ((128, (22, 21, 21)), (64, (12, 10, 10)), (6, (1, 1, 1))):
        assert binding.Rope.video(d, device="cpu").sections == want


def test_rope_binding_rejects_host_tensors_and_missing_grids():
    plan = binding.Rope(64, device="cpu")
    with pytest.raises(TypeError):
        binding.rope(torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16), None, plan)


# ---- distillation loss --------------------------------------------------------------------------------------------


def loss_call(y_hat=A, y=2 * A, type_=0, weight=None, scale=1.0, grad=3 * A, loss=A, B=1, H=2, N=8, d=64, ws=A, bytes_=1 << 20):
    return binding.library().rehyat_distill_loss(y_hat, y, type_, weight, scale, grad, loss, B, H, N, d, ws, bytes_, None)


@pytest.mark.parametrize("bad,code", [
    (dict(y_hat=None), "NULL"), (dict(y=None), "NULL"), (dict(grad=None), "NULL"), (dict(loss=None), "NULL"),
    (dict(ws=None), "NULL"), (dict(type_=3), "SHAPE"), (dict(scale=math.nan), "SHAPE"), (dict(scale=math.inf), "SHAPE"),
    (dict(y_hat=A + 8), "SHAPE"), (dict(y=A + 2), "SHAPE"), (dict(grad=A + 4), "SHAPE"), (dict(loss=A + 2), "SHAPE"),
    (dict(weight=A + 1), "SHAPE"), (dict(B=0), "SHAPE"), (dict(H=0), "SHAPE"), (dict(N=0), "SHAPE"), (dict(d=0), "SHAPE"),
    (dict(B=256, H=256), "SHAPE"), (dict(N=1 << 24, d=128), "SHAPE"), (dict(ws=A + 16), "WORKSPACE"),
    (dict(bytes_=0), "WORKSPACE"),
])
def test_distill_loss_rejects(bad, code):
    assert loss_call(**bad) == getattr(binding, "E_" + code)


def test_distill_loss_workspace():
    size = binding.distill_loss_workspace_bytes
    for shape in ((1, 1, 1, 1), (1, 12, 32760, 128), (65535, 1, 1, 1), (2, 12, 75600, 128), (255, 257, 3000, 64)):
        need = size(*shape)
        assert need % 256 == 0 and 0 < need <= 1 << 20
        assert loss_call(B=shape[0], H=shape[1], N=shape[2], d=shape[3], bytes_=need - 1) == binding.E_WORKSPACE
    assert size(0, 1, 1, 1) == size(1, 1, 1 << 24, 128) == size(256, 256, 1, 1) == 0


def test_distill_loss_binding_rejects_host_tensors():
    y = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        binding.distill_loss(y, y)


# ---- AdamW --------------------------------------------------------------------------------------------------------


def adamw_tensors(count=2, **fields):
    t = (binding.AdamWTensor * count)()
    for i in range(count):
        at = A * 0x100 * (i + 1)
        t[i] = binding.AdamWTensor(at, at + 0x10000, at + 0x20000, at + 0x30000, at + 0x40000, at + 0x50000, at + 0x60000,
                                   1000, 0, 2)
    for name, v in fields.items():
        setattr(t[count - 1], name, v)
    return t


def prepare(t, bits=32, step=0, table=A, bytes_=1 << 20, n=None):
    plan = binding.AdamWPlan()
    return binding.library().rehyat_adamw_prepare(t, len(t) if n is None else n, bits, step, table, bytes_,
                                                  ctypes.byref(plan), None)


SECOND = 2 * A * 0x100


@pytest.mark.parametrize("bits,bad,code", [
    (32, dict(param=None), "NULL"), (32, dict(grad=None), "NULL"), (32, dict(m=None), "NULL"), (32, dict(v=None), "NULL"),
    (8, dict(m_exp=None), "NULL"), (8, dict(v_exp=None), "NULL"), (32, dict(n=-1), "SHAPE"), (32, dict(n=1 << 40), "SHAPE"),
    (32, dict(param_type=3), "SHAPE"), (32, dict(grad_type=-1), "SHAPE"), (32, dict(param=SECOND + 1), "SHAPE"),
    (32, dict(grad=SECOND + 0x20002), "SHAPE"), (32, dict(m=SECOND + 0x30008), "SHAPE"), (32, dict(v=SECOND + 0x40004), "SHAPE"),
    (32, dict(master=SECOND + 0x10002), "SHAPE"),
    # ranges that overlap: of two tensors, of one, and of the table
    (32, dict(param=A * 0x100 + 1998), "SHAPE"), (32, dict(m=A * 0x100 + 0x30000 + 3984), "SHAPE"),
    (32, dict(v=SECOND + 0x30000), "SHAPE"), (32, dict(grad=SECOND + 0x10f9c), "SHAPE"),
    (8, dict(m_exp=SECOND + 0x3001f), "SHAPE"), (32, dict(param=A + 64), "SHAPE"), (32, dict(n=1 << 39), "WORKSPACE"),
])
def test_adamw_prepare_rejects(bits, bad, code):
    assert prepare(adamw_tensors(**bad), bits) == getattr(binding, "E_" + code)


def test_adamw_prepare_rejects_sizes_and_tables():
    t = adamw_tensors()
    assert prepare(t, n=0) == prepare(t, bits=16) == prepare(t, step=-1) == binding.E_SHAPE
    assert prepare(t, table=A + 64) == binding.E_WORKSPACE and prepare(t, table=None) == binding.E_NULL
    size = binding.library().rehyat_adamw_table_bytes
    need = size((ctypes.c_int64 * 2)(1000, 1000), 2)
    assert need % 256 == 0 and prepare(t, bytes_=need - 1) == binding.E_WORKSPACE
    assert size((ctypes.c_int64 * 1)(-1), 1) == size((ctypes.c_int64 * 1)(1 << 40), 1) == size(None, 1) == 0
    assert prepare(adamw_tensors(1, n=0)) == binding.E_SHAPE          # nothing to update
    assert binding.library().rehyat_adamw_prepare(None, 1, 32, 0, A, 1 << 20, None, None) == binding.E_NULL


@pytest.mark.parametrize("bad", [
    dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.5),
    dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-60), dict(weight_decay=-0.1), dict(lr_device=A + 1),
])
def test_adamw_step_rejects(bad):
    plan = binding.AdamWPlan(A, 5, 2, 32)
    h = binding.AdamWHyper(1e-3, 0.9, 0.999, 1e-8, 0.01)
    for name, v in bad.items():
        setattr(h, name, v)
    assert binding.library().rehyat_adamw_step(ctypes.byref(plan), ctypes.byref(h), None) == binding.E_SHAPE


def test_adamw_step_and_moments_reject_plans_and_pointers():
    lib = binding.library()
    h = binding.AdamWHyper(1e-3, 0.9, 0.999, 1e-8, 0.01)
    P = ctypes.byref
    assert lib.rehyat_adamw_step(None, P(h), None) == lib.rehyat_adamw_step(P(binding.AdamWPlan(A, 5, 2, 32)), None, None) \
        == lib.rehyat_adamw_step(P(binding.AdamWPlan()), P(h), None) == binding.E_NULL
    for plan in ((A, 0, 2, 32), (A, 5, 0, 32), (A, 5, 2, 16)):
        assert lib.rehyat_adamw_step(P(binding.AdamWPlan(*plan)), P(h), None) == binding.E_SHAPE
    assert lib.rehyat_adamw_step(P(binding.AdamWPlan(A + 8, 5, 2, 32)), P(h), None) == binding.E_WORKSPACE
    ok = [A, A, A, A, A, A, 64, None]
    for i in range(6):
        assert lib.rehyat_adamw_moments(*ok[:i], None, *ok[i + 1:]) == binding.E_NULL
    for i in (0, 2, 4, 5):
        assert lib.rehyat_adamw_moments(*ok[:i], A + 8, *ok[i + 1:]) == binding.E_SHAPE
    assert lib.rehyat_adamw_moments(*ok[:6], 0, None) == binding.E_SHAPE


def test_adamw_binding_rejects_host_tensors():
    with pytest.raises(TypeError):
        binding.AdamW([torch.zeros(4)])
