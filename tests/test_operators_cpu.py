"""Refusals and host arithmetic of the operators around the attention, without a GPU: every rejected call returns before
it touches the device (the pointers below are fake and never dereferenced)."""
import ctypes
import math
import os
import shutil
import subprocess
import types

import pytest
import torch

from paper_2601_04342_amd import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x1000


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    """run("rope" | "loss" | "adamw", ...) -> (status, launches) of a call whose launches are recorded, not made."""
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    binding.library()
    exe = str(tmp_path_factory.mktemp("host") / "record_operators")
    subprocess.run(["gcc", "-O1", "-rdynamic", os.path.join(ROOT, "tests", "host", "record_operators.c"), "-o", exe, "-ldl"],
                   check=True, capture_output=True, text=True)

    def run(*args):
        r = subprocess.run([exe, build.LIB, *map(str, args)], capture_output=True, text=True, timeout=120, check=True)
        *lines, status = r.stdout.splitlines()
        grids = [line.split() for line in lines if not line.startswith("items")]
        return int(status.split()[1]), [(int(x), int(y), int(z), name) for x, y, z, name in grids]

    return run


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
    dict(heads=65536), dict(xs=(-1, 512, 64)), dict(xs=(1536, 512, 1 << 44)), dict(os_=((1 << 63) - 1, 512, 64)), dict(os_=(1536, 512, 32)),
    dict(os_=(1536, 0, 64)), dict(os_=(0, 512, 64)), dict(os_=(1500, 512, 64)), dict(B=1 << 16, N=1 << 15),
    dict(B=1 << 15, N=1 << 10), dict(n_ops=2, second=dict(out=2 * A)), dict(n_ops=2, second=dict(heads=0)),
])
def test_rope_rejects(bad):
    assert rope_call(**bad) == binding.E_SHAPE


HEAD, TOKEN = (1536, 512, 64), (1536, 64, 192)   # B = 2, N = 8, 3 heads of 64: head-major and token-major
FUSED = (8 * 384, 64, 384)                        # [B, N, 2, 3, 64]: queries and keys of one projection
FAR = 1 << 32


@pytest.mark.parametrize("ops,taken", [
    ([(A, FAR, HEAD, HEAD)], True), ([(A, FAR, TOKEN, HEAD)], True), ([(A, A, TOKEN, TOKEN)], True),
    ([(A, A + 6144, HEAD, HEAD)], True),                # right behind what is read (2 x 1536 elements of two bytes)
    ([(A + 6144, A, HEAD, HEAD)], True),
    ([(A, A + 6142, HEAD, HEAD)], False),               # the last element
    ([(A, A + 128, HEAD, HEAD)], False), ([(A + 128, A, HEAD, HEAD)], False),       # shifted by a token
    ([(A, A + 64, HEAD, HEAD)], False),                 # by half a row
    ([(A, A + 1024, HEAD, HEAD)], False), ([(A, A + 3072, HEAD, HEAD)], False),     # onto the next head, sequence
    ([(A, A, HEAD, TOKEN)], False),                     # transposed in place
    ([(A, A + 128, (0, 0, 64), HEAD)], False),          # one row for all heads, over which the first would be written
    ([(A, A, (0, 0, 64), HEAD)], False),
    ([(A, A, FUSED, FUSED), (A + 384, A + 384, FUSED, FUSED)], True),               # each in place, between the other's rows
    ([(A, A, FUSED, FUSED), (A + 256, A + 256, FUSED, FUSED)], False),              # begins within the first's heads
    ([(A, A, FUSED, FUSED), (A + 382, A + 382, FUSED, FUSED)], False),
    ([(A, FAR, FUSED, HEAD), (A + 384, 2 * FAR, FUSED, HEAD)], True),
    ([(A, FAR, HEAD, HEAD), (2 * FAR, FAR, HEAD, HEAD)], False),                    # one output
    ([(A, FAR, HEAD, HEAD), (2 * FAR, FAR + 128, HEAD, HEAD)], False),
    ([(A, FAR, HEAD, HEAD), (FAR, A, HEAD, HEAD)], False),                          # exchanged
    ([(A, FAR, HEAD, HEAD), (FAR + 6000, 2 * FAR, HEAD, HEAD)], False),             # the second reads what the first writes
    ([(A, FAR, HEAD, HEAD), (A, 2 * FAR, HEAD, HEAD)], True),                       # both read the same
])
def test_rope_outputs_overlap_nothing(record, ops, taken):
    args = [v for x, out, xs, os_ in ops for v in (x, out, 3, *xs, *os_)]
    status, launches = record("rope", 0, 0, 2, 8, 64, 64, len(ops), *args)
    assert (status, len(launches)) == ((binding.OK, 1) if taken else (binding.E_SHAPE, 0))


def rows_meet(delta, out, other, d):
    """Whether two rows share an element, by going through all of them: (strides, extents) of both, `delta` between them."""
    rows = [{b * s[0] + h * s[1] + n * s[2] + at for b in range(e[0]) for h in range(e[1]) for n in range(e[2])}
            for (s, e), at in ((out, 0), (other, delta))]
    cells = [{r + c for r in part for c in range(d)} for part in rows]
    return bool(cells[0] & cells[1])


def test_rope_overlap_against_all_elements(record):
    """Both tensors in one layout, anywhere near each other, with different numbers of heads."""
    d, N, B = 4, 3, 2
    strides = (100, 4, 20)                              # token-major with room for five heads, sequences 100 apart
    for heads in ((2, 3), (3, 2), (5, 1)):
        for delta in list(range(-24, 25, 2)) + [-100, -96, 76, 100, 104, 116, 180, 190]:
            at = 1 << 20
            x = [at, at + 2 * delta]
            args = [v for i in range(2) for v in (x[i], x[i], heads[i], *strides, *strides)]
            status, _ = record("rope", 0, 0, B, N, d, d, 2, *args)
            meet = rows_meet(delta, (strides, (B, heads[0], N)), (strides, (B, heads[1], N)), d)
            assert (status == binding.E_SHAPE) == meet, (heads, delta)


@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("B,N,H,d", [(1, 1, 65535, 64), (1, 1, 1, 2), (1, 4194303, 1, 512), (65536, 1, 3, 64), (1, 32760, 12, 128)])
def test_rope_grids_stay_in_bounds(record, B, N, H, d, layout):
    s = (N * H * d, N * d, d)
    args = [v for i in range(2) for v in (FAR << 10, (FAR << 12) * (i + 1), H, *s, *s)]
    status, launches = record("rope", 0, layout, B, N, d, d, 2, *args)
    assert status == binding.OK and len(launches) == 1
    for x, y, z, _ in launches:
        assert 1 <= x < 2**31 // 256 and 1 <= y <= 65535 and z == 1


@pytest.mark.parametrize("weighted", [0, 1])
@pytest.mark.parametrize("B,H,N,d", [(1, 1, 1, 1), (65535, 1, 1, 1), (255, 257, 3000, 64), (2, 12, 75600, 128), (1, 2, 256, 64)])
def test_loss_grids_and_workspaces_stay_in_bounds(record, B, H, N, d, weighted):
    status, launches = record("loss", 0, weighted, B, H, N, d)
    assert status == binding.OK and len(launches) == (1 if B * H * N * d <= 32768 and (B * H <= 4 or not weighted) else 2)
    x, y, z, _ = launches[0]
    assert 1 <= x <= 16384 and 1 <= y <= 65535 and z == 1
    if len(launches) == 2:
        assert 8 * x * y <= binding.distill_loss_workspace_bytes(B, H, N, d)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("tensors,elements", [(1, 1), (8, 100000), (200, 300000), (1, 1 << 34), (1000, 5)])
def test_adamw_grids_stay_in_bounds(record, tensors, elements, bits):
    status, launches = record("adamw", bits, tensors, elements)
    assert status == binding.OK
    *tables, (x, y, z, name) = launches
    assert "adamw_kernel" in name and 1 <= x <= min(-(-elements // 1024) * tensors, 256 * 8) and y == z == 1
    assert sum(g[0] for g in tables) == tensors


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
                P(data=A, bits=32, stride_n=-1), P(data=A, bits=32, stride_b=1 << 62),
                P(data=A, bits=32, stride_n=1 << 46)):
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
    dict(sections=(16, 16, 16, 16)), dict(scaling=dict(kind="no", factor=2.0)), dict(scaling=dict(kind="linear")), dict(scaling=dict(factor=2.0)),
    dict(scaling=dict(kind="parts", factor=2.0)), dict(scaling=dict(kind="base", factor=math.inf)), dict(scaling=dict(kind="linear", factor=0.0)),
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
    (dict(bytes_=0), "WORKSPACE"), (dict(grad=A), "SHAPE"), (dict(grad=2 * A + 2032), "SHAPE"),
    (dict(y=3 * A + 2032), "SHAPE"), (dict(y=4 * A - 32, type_=2, grad=3 * A + 2000 + 32), "SHAPE"),
    (dict(weight=3 * A + 4), "SHAPE"), (dict(y_hat=3 * A - 16), "SHAPE"),
])
def test_distill_loss_rejects(bad, code):
    assert loss_call(**bad) == getattr(binding, "E_" + code)


def test_distill_loss_workspace():
    size = binding.distill_loss_workspace_bytes
    for shape in ((1, 1, 1, 1), (1, 12, 32760, 128), (65535, 1, 1, 1), (2, 12, 75600, 128), (255, 257, 3000, 64)):
        need = size(*shape)
        assert need % 256 == 0 and 0 < need <= 1 << 20
        far = dict(y_hat=1 << 40, y=2 << 40, grad=3 << 40)
        assert loss_call(B=shape[0], H=shape[1], N=shape[2], d=shape[3], bytes_=need - 1, **far) == binding.E_WORKSPACE
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
    dict(beta2=math.nan), dict(lr=1e39), dict(eps=1e39), dict(weight_decay=math.nan),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-60), dict(weight_decay=-0.1), dict(lr_device=A + 1),
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
    ok = [A, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 64, None]
    for i, j in ((4, 5), (4, 0), (4, 1), (5, 2), (5, 3)):            # a value onto what is read, or onto the other
        assert lib.rehyat_adamw_moments(*ok[:i], ok[j], *ok[i + 1:]) == binding.E_SHAPE
    for i in range(6):
        assert lib.rehyat_adamw_moments(*ok[:i], None, *ok[i + 1:]) == binding.E_NULL
    for i in (0, 2, 4, 5):
        assert lib.rehyat_adamw_moments(*ok[:i], A + 8, *ok[i + 1:]) == binding.E_SHAPE
    assert lib.rehyat_adamw_moments(*ok[:6], 0, None) == binding.E_SHAPE


def test_adamw_binding_rejects_host_tensors():
    with pytest.raises(TypeError):
        binding.AdamW([torch.zeros(4)])


# ---- all of them under the sanitizers -----------------------------------------------------------------------------


def test_host_layers_under_asan_ubsan(tmp_path):
    """Every call of the program is rejected, or answered, before the first HIP call; device code is compiled as usual."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "operators_san")
    host = []
    for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined"):
        host += ["-Xarch_host", f]
    flags = [f for f in build.FLAGS if f not in ("-O3", "-fPIC")]
    subprocess.run([build.HIPCC, *flags, "-O1", "-g", *host,
                    *(os.path.join(build.CSRC, s) for s in build.SOURCES),
                    os.path.join(ROOT, "tests", "sanitize", "operators_driver.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True, timeout=900)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "operators sanitize ok" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr


def test_work_belongs_to_the_tensors_device_and_stream(monkeypatch):
    """Another current device is left for the tensors'; a stream of another device is refused."""
    t = types.SimpleNamespace(device=torch.device("cuda:1"), get_device=lambda: 1)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    ctx = binding._elsewhere(t, None)
    assert isinstance(ctx, torch.cuda.device) and ctx.idx == 1
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    assert binding._elsewhere(t, None) is None
    with pytest.raises(ValueError):
        binding._elsewhere(t, types.SimpleNamespace(device=torch.device("cuda:0")))
