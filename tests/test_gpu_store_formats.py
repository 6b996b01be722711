"""The conversions of the two block formats over their whole range: every 16-bit number at every scale into codes, fp32 numbers on both sides
of every tie, every code at every scale byte back into numbers."""
import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
import workloads
from oracle import store
from gpu_util import TORCH_DTYPE, dev, to_device, to_float64

pytestmark = pytest.mark.gpu
DTYPES = ["f32", "f16", "bf16"]
# codes' values, scale exponents by type, the first magnitude at scale 1 that needs a larger one, the largest code's value
FORMATS = {4: (store.VALUES4, store.BOUNDS4, np.nextafter(7.0, 0.0), 6.0), 8: (store.VALUES8, store.BOUNDS8, 464.0, 448.0)}


def _all_numbers(dtype):
    """Every finite number of a 16-bit type, in float64."""
    bits = np.arange(1 << 16, dtype=np.uint16)
    with np.errstate(invalid="ignore"):
        x = workloads.to_float64(bits.view(np.float16) if dtype == "f16" else bits, dtype)
    return x[np.isfinite(x)]


def _blocks(x, pin):
    """Rows of 32: 31 of the numbers and, at a place that moves on, the number that sets the scale."""
    rows = -(-len(x) // 31)
    wide = np.zeros(rows * 31)
    wide[:len(x)] = x
    out = np.empty((rows, 32))
    at = np.arange(rows) % 32
    rest = np.arange(32)[None] != at[:, None]
    out[rest] = wide
    out[~rest] = pin * np.where(np.arange(rows) % 2, -1.0, 1.0)
    return out


def _storage(x, dtype):
    """Float64 numbers of the type in its storage."""
    s = x.astype(np.float32) if dtype == "f32" else workloads.to_storage(x.astype(np.float32), dtype)
    assert np.array_equal(workloads.to_float64(s, dtype) if dtype != "f32" else s.astype(np.float64), x)
    return s


def _check_codes(bits, dtype, x, e):
    """Blocks x, whose scale is 2^e, against the nearest codes."""
    values, bounds, _, _ = FORMATS[bits]
    t = to_device(_storage(x, dtype), dtype)
    if bits == 4:
        codes, scales = lrbi.quant_pack(lrbi.Desc(len(x), 32, len(x), 32, 1), t)
        got = store.nibbles(codes.cpu().numpy())
    else:
        codes, scales = lrbi.checkpoint_pack(t)
        got = codes.cpu().numpy()
        x = np.clip(x, -store.MOST8[dtype], store.MOST8[dtype])
    assert (scales[:, 0] == e + 127).all()
    sign = 8 if bits == 4 else 128
    want = np.minimum(store.nearest(x / 2.0 ** e, values), len(values) - 1)
    assert np.array_equal(got & (sign - 1), want)
    zero = want == 0  # of either sign
    assert np.array_equal((got & sign != 0)[~zero], np.signbit(x)[~zero])


def _pin(bits, dtype, e):
    """A number that takes scale 2^e, and the largest magnitude that does."""
    _, bounds, limit, most = FORMATS[bits]
    largest = float(torch.finfo(TORCH_DTYPE[dtype]).max)
    if e == bounds[dtype][1]:
        return min(most * 2.0 ** e, store.MOST8[dtype] if bits == 8 else np.inf), largest
    return most * 2.0 ** e, limit * 2.0 ** e


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_every_number_at_every_scale(dtype, bits):
    print("store formats, numbers", dtype, bits, flush=True)
    x = _all_numbers(dtype)
    lo, hi = FORMATS[bits][1][dtype]
    for e in range(lo, hi + 1):
        pin, limit = _pin(bits, dtype, e)
        _check_codes(bits, dtype, _blocks(x[np.abs(x) <= limit], pin), e)


@pytest.mark.parametrize("bits", [4, 8])
def test_fp32_beside_every_tie(bits):
    """Ties and codes' own values, the fp32 numbers just above and below them, both signs, at scales over the whole range (below the normal
    numbers at the lowest)."""
    print("store formats, ties", bits, flush=True)
    values, bounds, _, _ = FORMATS[bits]
    lo, hi = bounds["f32"]
    points = np.concatenate((values, (values[:-1] + values[1:]) / 2))
    for e in (lo, lo + 1, -60, -1, 0, 1, 60, hi - 1, hi):
        pin, limit = _pin(bits, "f32", e)
        at = (points * 2.0 ** e)[points * 2.0 ** e <= limit].astype(np.float32)
        assert e == hi or len(at) == len(points)
        x = np.concatenate((at, np.nextafter(at, np.float32(np.inf)), np.nextafter(at, np.float32(0)))).astype(np.float64)
        x = np.concatenate((x, -x))
        _check_codes(bits, "f32", _blocks(x[np.abs(x) <= limit], pin), e)
    # the border between two scales: the last number of one, the first of the next
    last = np.float32(np.nextafter(np.float32(7), np.float32(0)) if bits == 4 else 464)
    for e in (lo + 1, 0, hi - 1):
        for v, s in ((last, e), (np.nextafter(last, np.float32(np.inf)), e + 1)):
            _check_codes(bits, "f32", np.full((1, 32), float(np.ldexp(v, e))), s)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_code_at_every_scale(dtype, bits):
    """Scales that packing writes for the type: exact.  Others: rounded to the type, to an infinity beyond it.  255: NaN."""
    print("store formats, codes", dtype, bits, flush=True)
    n = 32 if bits == 4 else 256
    codes = np.tile((np.arange(n) % (1 << bits)).astype(np.uint8), (256, 1))
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 8, axis=1)
    if bits == 4:
        got = lrbi.quant_unpack(torch.from_numpy(store.packed_nibbles(codes)).to(dev()), torch.from_numpy(scales[:, :4].copy()).to(dev()), n, TORCH_DTYPE[dtype])
        exact = store.unpack4(codes, scales[:, :1], n)
    else:
        got = lrbi.checkpoint_unpack(torch.from_numpy(codes).to(dev()), torch.from_numpy(scales).to(dev()), n, TORCH_DTYPE[dtype])
        exact = store.unpack8(codes, scales, n)
        exact[255] = np.nan
    want = to_float64(torch.from_numpy(exact).to(TORCH_DTYPE[dtype]))  # at most four bits at 2^-136 and more: numbers of fp32 on the way
    lo, hi = (store.BOUNDS4 if bits == 4 else store.BOUNDS8)[dtype]
    inside = slice(lo + 127, hi + 127 + (1 if bits == 4 else 0))  # 8 bits: half of the codes of the last scale stand for numbers beyond the type
    assert np.array_equal(want[inside], exact[inside], equal_nan=True)
    assert np.array_equal(to_float64(got), want, equal_nan=True)
