"""The 8-bit moments of AdamW from their definition in include/rehyat.h: values, and codes by search through all of them, in
64 bits, where everything below is exact.  Arrays are whole groups of 32."""
import numpy as np

GROUP = 32


def _e4m3():
    c = np.arange(127)
    return np.where(c >> 3 == 0, c * 2.0**-9, (8 + (c & 7)) * 2.0**((c >> 3) - 10.0))


M_VALUES = _e4m3()                                          # codes 0 .. 126
_V = (np.arange(256) + 8 * 70) << 20                        # codes under the exponent 100
V_VALUES = _V.astype(np.int32).view(np.float32).astype(np.float64)


def _exponents(x, least):
    top = np.abs(x).reshape(-1, GROUP).max(1).astype(np.float32)
    return np.maximum(top.view(np.int32) >> 23, least).astype(np.int64)


def _up(values, x, least, rises):
    """Index of the value below x or of the one above it, by `rises` (how far x is on its way, its index below)."""
    lo = np.clip(np.searchsorted(values, x, side="right") - 1, 0, len(values) - 2)
    way = np.clip((x - values[lo]) / (values[lo + 1] - values[lo]), 0.0, 1.0)
    return np.maximum(lo + rises(way, lo), least)


def _nearest(way, lo):
    return (way > 0.5) | ((way == 0.5) & (lo % 2 == 1))


def encode(m, v, random=None):
    """(codes of m, exponents, codes of v, exponents) of fp32 moments; `random`: 32 bits for each element, None: nearest.
    m takes the lower 16, in the middle of their steps, v the upper 20."""
    em, ev = _exponents(m, 8), _exponents(v, 31)
    rises_m = rises_v = _nearest
    if random is not None:
        r = random.astype(np.int64)
        rises_m = lambda way, _: way + ((r & 0xFFFF) + 0.5) / 2**16 >= 1
        rises_v = lambda way, _: way + (r >> 12) / 2**20 >= 1
    xm = np.abs(m.astype(np.float64)) * 2.0**(134.0 - np.repeat(em, GROUP))
    xv = v.astype(np.float64) * 2.0**(100.0 - np.repeat(ev, GROUP))
    cm = _up(M_VALUES, xm, 0, rises_m) | np.where(np.signbit(m), 0x80, 0)
    cv = np.where(v == 0, 0, _up(V_VALUES, xv, 1, rises_v))
    return cm, em, cv, ev


def decode(cm, em, cv, ev):
    sign = np.where(cm & 0x80, -1.0, 1.0)
    m = sign * M_VALUES[cm & 0x7F] * 2.0**(np.maximum(np.repeat(em, GROUP), 8) - 134.0)
    v = np.where(cv == 0, 0.0, V_VALUES[cv] * 2.0**(np.maximum(np.repeat(ev, GROUP), 31) - 100.0))
    return m, v


def _scatter(x):
    x = x.astype(np.uint64)
    for shift, factor in ((16, 0x6A09E667), (15, 0xBB67AE85)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(factor)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(step, places):
    """The hash of an update's number and of the places of four elements each (a tensor begins at a multiple of 1,024
    elements), of which each element has the bits from another byte on."""
    step, golden, mask = int(step), 0x9E3779B9, 0xFFFFFFFF
    places, left = np.divmod(np.asarray(places, np.uint64), np.uint64(4))
    left *= np.uint64(8)
    key = int(_scatter(np.array([(step * golden + (step >> 32)) & mask], np.uint64))[0])
    mix = (np.uint64(key) + (places >> np.uint64(32)) * np.uint64(golden)) & np.uint64(mask)
    h = _scatter((places & np.uint64(mask)) ^ mix)
    return ((h << left) | (h >> (np.uint64(32) - left))) & np.uint64(mask)
