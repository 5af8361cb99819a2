"""Sizes and places at which calls of the operators around the attention are refused, or are cut into launches that the
runtime takes: without a GPU, the pointers are fake."""
import ctypes
import os
import random
import shutil
import subprocess
from fractions import Fraction

import pytest

from paper_2601_04342_amd import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    """run("moments" | "positions" | "loss", ...) -> (status, grids) of a call whose launches are recorded, not made."""
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    binding.library()
    exe = str(tmp_path_factory.mktemp("host") / "record_places")
    subprocess.run(["gcc", "-O1", "-rdynamic", os.path.join(ROOT, "tests", "host", "record_places.c"), "-o", exe, "-ldl"],
                   check=True, capture_output=True, text=True)

    def run(*args):
        r = subprocess.run([exe, build.LIB, *map(str, args)], capture_output=True, text=True, timeout=120, check=True)
        *lines, status = r.stdout.splitlines()
        return int(status.split()[1]), [line.split()[:3] for line in lines]

    return run


@pytest.mark.parametrize("n", [1, 1024, 1025, 10**6, 2**33, 2**33 + 1, 2**34 - 1, 2**34 + 5, 2**38 - 1])
def test_moments_of_any_size_fit_the_runtimes_grids(record, n):
    """A grid's threads, and the elements of a launch, are counted in 32 bits."""
    status, launches = record("moments", n)
    assert status == binding.OK
    assert all(0 < int(x) * 256 < 2**32 and int(x) * 1024 <= 2**32 and y == z == "1" for x, y, z in launches)
    assert sum(int(x) for x, _, _ in launches) == -(-n // 1024)


def test_moments_beyond_what_is_supported(record):
    assert record("moments", 2**38) == (binding.E_SHAPE, [])


OUT, SECOND, OUT_BYTES = 1 << 40, 2 << 40, 2 * 3 * 8 * 64 * 2      # B = 2, 3 heads, N = 8, 64 elements of two bytes


@pytest.mark.parametrize("bits,axes,strides,size", [
    (32, 1, (0, 1), 32), (64, 1, (8, 1), 128), (32, 3, (24, 3), 192), (64, 2, (0, 2), 128), (32, 1, (100, 4), 4 * (100 + 28 + 1)),
    (64, 1, (0, 0), 8),
])
@pytest.mark.parametrize("out", [OUT, SECOND])
def test_rope_positions_are_not_written_over(record, bits, axes, strides, size, out):
    """A workgroup would read what another has turned already."""
    word = bits // 8
    for at, taken in ((out + OUT_BYTES, True), (out + OUT_BYTES - word, False), (out - size, True), (out - size + word, False),
                      (out + 2048, False)):
        status, launches = record("positions", bits, axes, 2, 8, *strides, at, OUT, SECOND)
        assert (status, len(launches)) == ((binding.OK, 1) if taken else (binding.E_SHAPE, 0)), at - out


GB = 1 << 30
LARGE, SMALL = (2, 3, 4001, 64), (1, 2, 100, 64)                   # two launches, one launch


@pytest.mark.parametrize("B,H,N,d", [LARGE, SMALL])
@pytest.mark.parametrize("type_", [0, 2])
def test_loss_and_workspace_overlap_nothing_that_is_read_or_written(record, B, H, N, d, type_):
    n = B * H * N * d
    room = binding.distill_loss_workspace_bytes(B, H, N, d)
    far = dict(y_hat=GB, y=2 * GB, weight=0, grad=3 * GB, loss=4 * GB, workspace=5 * GB)
    run = lambda **at: record("loss", type_, B, H, N, d, *{**far, **at}.values())
    launches = 1 if (B, H, N, d) == SMALL else 2
    assert run() == (binding.OK, run()[1]) and len(run()[1]) == launches
    assert len(run(weight=6 * GB)[1]) == launches
    for name, size in (("y_hat", 2 * n), ("y", (4 if type_ == 2 else 2) * n), ("grad", 2 * n)):
        for at in (far[name], far[name] + size - 4, far[name] + size // 2 // 4 * 4):
            assert run(loss=at) == (binding.E_SHAPE, []), (name, at)
        last = far[name] + (size - 1) // 256 * 256
        for at in (far[name], last, far[name] - room + 256):
            assert run(workspace=at) == (binding.E_SHAPE, []), (name, at)
        assert run(loss=far[name] + size)[0] == run(loss=far[name] - 4)[0] == binding.OK
        assert run(workspace=far[name] - room)[0] == run(workspace=last + 256)[0] == binding.OK
    # the sum of the pieces' sums is written when all of them have been read
    assert run(loss=far["workspace"])[0] == binding.OK


@pytest.mark.parametrize("source", ["rehyat_rope.hip", "rehyat_loss.hip", "rehyat_adamw.hip"])
def test_sources_that_meet_numbers_that_are_none_are_compiled_for_them(source):
    """What such an element becomes is stated and tested: nothing of it may be taken to be impossible."""
    flags = [f for f in build.FLAGS + build.EXTRA_FLAGS.get(source, []) if f.endswith("honor-nans")]
    assert flags[-1] == "-fhonor-nans"
    assert not [f for f in build.FLAGS if "fast-math" in f or "finite" in f or f == "-fno-honor-infinities"]


# 1 / (2 pi) to 120 places, from a series for pi in whole numbers: pi = 16 atan(1/5) - 4 atan(1/239)
def _turns_of(radians):
    one = 10**140
    atan = lambda k: sum((-1)**i * (one // k**(2 * i + 1)) // (2 * i + 1) for i in range(110))
    pi = Fraction(16 * atan(5) - 4 * atan(239), one)
    return Fraction(radians) / (2 * pi) * 2**64


@pytest.mark.parametrize("scale", [1e-6, 1e-3, 1.0, 100.0, 1e6])
def test_turns_are_rounded_to_the_nearest(scale):
    """Half a unit, and what the quotient in 64 bits is off by: its own rounding and that of 2 pi, each 2^-64 of it."""
    rng = random.Random(int(scale * 1e6))
    f = [rng.choice((-1, 1)) * scale * rng.uniform(0.1, 1) for _ in range(64)]
    t = (ctypes.c_uint64 * 64)()
    assert binding.library().rehyat_rope_turns((ctypes.c_double * 64)(*f), 64, t) == binding.OK
    for x, got in zip(f, t):
        want = _turns_of(x)
        off = (got - want) % 2**64
        assert min(off, 2**64 - off) <= Fraction(1, 2) + abs(want) / 2**63 + Fraction(1, 10**6), x
