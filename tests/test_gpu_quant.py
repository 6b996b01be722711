"""4-bit weights on the GPU against the oracle: packing bit for bit, values bit for bit, the product within the roundings of
its sums."""
import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
import workloads
from oracle import lrbi_oracle as orc
from oracle import store
from gpu_util import TORCH_DTYPE, dev, device_factors, to_device, to_float64

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
DTYPES = ["f32", "f16", "bf16"]


def _weights(m, n, dtype, seed, spread=1.0):
    """Rows of very different size, zeros among them, in the storage type."""
    rng = np.random.default_rng(seed)
    W = rng.standard_normal((m, n)) * 0.05 * np.exp(spread * rng.standard_normal((m, 1)))
    W[rng.random((m, n)) < 0.1] = 0
    return workloads.to_storage(W.astype(np.float32), dtype)


def _packed(codes, scales, n):
    """Device codes and scales -> one code a byte, scale bytes, without what lies behind the last block."""
    blocks = -(-n // 32)
    return store.nibbles(codes.cpu().numpy()[:, :16 * blocks]), scales.cpu().numpy()[:, :blocks]


def _same_values(t, want):
    got = to_float64(t)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(want)], want[~np.isnan(want)])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,r,c,k", [(1, 1, 1, 1, 1), (3, 31, 2, 7, 3), (17, 64, 8, 64, 5), (40, 200, 16, 33, 40), (5, 1000, 5, 1000, 8),
                                       (130, 257, 64, 128, 70)])
def test_pack_and_unpack(dtype, m, n, r, c, k):
    print("quant pack", dtype, m, n, r, c, k, flush=True)
    W = _weights(m, n, dtype, m + n)
    rng = np.random.default_rng(n)
    d = lrbi.Desc(m, n, r, c, k)
    Ip01, Iz01 = workloads.make_factors(rng, d.tiles, r, c, k, 0.4 if k < 10 else 0.15)
    dIp, dIz = device_factors(d, Ip01, Iz01)
    M = orc.decode_mask(Ip01, Iz01, m, n, r, c, k)
    W64 = workloads.to_float64(W, dtype)
    for factors, mask in (((dIp, dIz), M), ((), None)):
        codes, scales = lrbi.quant_pack(d, to_device(W, dtype), *factors)
        want, exps = store.pack4(W64, mask, dtype)
        got, gexps = _packed(codes, scales, n)
        assert np.array_equal(gexps, exps)
        # a zero has either sign's code
        assert np.array_equal(np.where(got == 8, 0, got), np.where(want == 8, 0, want))
        _same_values(lrbi.quant_unpack(codes, scales, n, TORCH_DTYPE[dtype]), store.unpack4(want, exps, n))
    assert np.all(want[:, n:] == 0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_pack_at_the_ends_of_the_range(dtype):
    """Ties, values that round past the largest code, the smallest and largest numbers of the type, infinities and NaN kept and pruned."""
    print("quant pack, range", dtype, flush=True)
    fi = torch.finfo(TORCH_DTYPE[dtype])
    rows = [[6.0], [7.0], [6.99], [5.0, 2.5, 3.5, 1.75, 0.25, 0.75, 6.0], [fi.max], [fi.max / 2, 1.0], [fi.tiny], [fi.smallest_normal, fi.tiny * 0.5],
            [fi.smallest_normal * fi.eps, fi.smallest_normal * fi.eps * 3], [0.0], [np.inf, 1.0], [np.nan, 1.0], [-np.inf], [1e-30 if dtype != "f16" else 1e-6, 1.0]]
    W = np.zeros((len(rows), 64), dtype=np.float32)
    for i, v in enumerate(rows):
        W[i, 5:5 + len(v)] = v
        W[i, 32] = 0.3
    W = workloads.to_storage(W, dtype)
    W64 = workloads.to_float64(W, dtype)
    d = lrbi.Desc(len(rows), 64, len(rows), 64, 1)
    codes, scales = lrbi.quant_pack(d, to_device(W, dtype))
    want, exps = store.pack4(W64, None, dtype)
    got, gexps = _packed(codes, scales, 64)
    assert np.array_equal(gexps, exps)
    assert np.array_equal(np.where(got == 8, 0, got), np.where(want == 8, 0, want))
    _same_values(lrbi.quant_unpack(codes, scales, 64, TORCH_DTYPE[dtype]), store.unpack4(want, exps, 64))
    # everything but one column pruned: what lies under the mask, infinities and NaN included, leaves no trace
    Ip01 = np.ones((1, len(rows), 1), dtype=np.uint8)
    Iz01 = np.zeros((1, 1, 64), dtype=np.uint8)
    Iz01[0, 0, 32] = 1
    codes, scales = lrbi.quant_pack(d, to_device(W, dtype), *device_factors(d, Ip01, Iz01))
    back = to_float64(lrbi.quant_unpack(codes, scales, 64, TORCH_DTYPE[dtype]))
    want = np.zeros_like(back)
    want[:, 32] = store.unpack4(*store.pack4(W64[:, 32:33], None, dtype), 1)[:, 0]
    assert np.array_equal(back, want)


def test_strided_buffers_and_untouched_bytes():
    print("quant strides", flush=True)
    m, n = 37, 130
    W = torch.randn(m, n + 11, device=dev()).half()[:, 3:3 + n]  # rows that are no 16-byte pieces
    d = lrbi.Desc(m, n, 16, 16, 4)
    codes = torch.full((m, 16 * 5 + 32), 0xAB, dtype=torch.uint8, device=dev())
    scales = torch.full((m, 12), 0xCD, dtype=torch.uint8, device=dev())
    lrbi.quant_pack(d, W, out=(codes, scales))
    plain = lrbi.quant_pack(d, W.contiguous())
    assert torch.equal(codes[:, :80], plain[0]) and torch.equal(scales[:, :5], plain[1][:, :5])
    assert (codes[:, 80:] == 0xAB).all() and (scales[:, 5:] == 0xCD).all()
    out = torch.full((m, n + 5), 7.0, dtype=torch.float16, device=dev())
    lrbi.quant_unpack(codes, scales, n, torch.float16, out=out[:, 1:1 + n])
    assert torch.equal(out[:, 1:1 + n], lrbi.quant_unpack(*plain, n, torch.float16))
    assert (out[:, 0] == 7).all() and (out[:, 1 + n:] == 7).all()
    X = torch.randn(n, 9, device=dev()).half()
    y = torch.full((m, 14), 7.0, dtype=torch.float16, device=dev())
    lrbi.quant_matvec(codes, scales, X[:, 2:7], out=y[:, 4:9])
    assert torch.equal(y[:, 4:9], lrbi.quant_matvec(*plain, X[:, 2:7].contiguous()))
    assert (y[:, :4] == 7).all() and (y[:, 9:] == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,N", [(1, 1, 1), (1, 33, 1), (16, 32, 1), (17, 100, 1), (500, 800, 1), (300, 2048, 1), (33, 2049, 1), (100, 6000, 1),
                                   (31, 70, 2), (64, 512, 5), (50, 300, 6), (40, 2100, 10), (65, 257, 16), (20, 96, 17), (48, 4200, 20),
                                   (30, 130, 33), (16, 64, 70), (40, 4100, 31), (40, 4100, 32), (33, 2600, 67), (50, 2000, 35), (20000, 70, 33), (2000, 1500, 1), (70, 20000, 3)])
def test_matvec(dtype, m, n, N):
    print("quant matvec", dtype, m, n, N, flush=True)
    rng = np.random.default_rng(m + n + N)
    codes = rng.integers(0, 16, (m, -(-n // 32) * 32)).astype(np.uint8)
    codes[:, n:] = 0
    scales = rng.integers(118, 125, (m, -(-n // 32))).astype(np.uint8)
    scales[m // 2] = 104 if dtype == "f16" else 3  # a row at the smallest scales of the type
    X = workloads.to_storage(rng.standard_normal((n, N)).astype(np.float32), dtype)
    pad = np.zeros((m, -(-scales.shape[1] // 4) * 4), dtype=np.uint8)
    pad[:, :scales.shape[1]] = scales
    dc, ds = torch.from_numpy(store.packed_nibbles(codes)).to(dev()), torch.from_numpy(pad).to(dev())
    x = to_device(X, dtype)
    Y = lrbi.quant_matvec(dc, ds, x if N > 1 else x[:, 0])
    Y = to_float64(Y).reshape(m, N)
    W64, X64 = store.unpack4(codes, scales, n), workloads.to_float64(X, dtype)
    want, size = W64 @ X64, np.abs(W64) @ np.abs(X64)
    # Exact products.  A wavefront adds them up 32 a matrix instruction (their order inside is the hardware's: at most 32
    # roundings), an eighth of them one after the other, the eight wavefronts (fp32: three parts of each) in the end; one
    # rounding on store, to a subnormal number at worst by half the smallest one.
    chain = n / 8 + 128 * 4 + 32
    tiny = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}[dtype]
    assert np.all(np.abs(Y - want) <= HALF[dtype] * np.abs(want) + min(chain, n + 40) * 2.0 ** -24 * size + tiny)


@pytest.mark.parametrize("dtype", DTYPES)
def test_matvec_of_unusual_values(dtype):
    """NaN scales reach their row alone; large and small numbers of X go through whole (fp32: in three parts)."""
    print("quant matvec, values", dtype, flush=True)
    m, n = 40, 160
    rng = np.random.default_rng(5)
    codes = rng.integers(0, 16, (m, n)).astype(np.uint8)
    scales = np.full((m, 8), 127, dtype=np.uint8)
    scales[7, 2] = 255
    fi = torch.finfo(TORCH_DTYPE[dtype])
    X = np.zeros((n, 3), dtype=np.float32)
    X[:, 0] = rng.standard_normal(n)
    X[3, 1] = fi.max / 16
    X[50:60, 2] = fi.smallest_normal * np.arange(1, 11) * 16
    X = workloads.to_storage(X, dtype)
    x = to_device(X, dtype)
    Y = to_float64(lrbi.quant_matvec(torch.from_numpy(store.packed_nibbles(codes)).to(dev()), torch.from_numpy(scales).to(dev()), x))
    assert np.isnan(Y[7]).all() and not np.isnan(np.delete(Y, 7, axis=0)).any()
    scales[7, 2] = 127
    W64, X64 = store.unpack4(codes, scales[:, :5], n), workloads.to_float64(X, dtype)
    want, size = np.delete(W64 @ X64, 7, axis=0), np.delete(np.abs(W64) @ np.abs(X64), 7, axis=0)
    tiny = {"f32": 2.0 ** -140, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}[dtype]
    assert np.all(np.abs(np.delete(Y, 7, axis=0) - want) <= HALF[dtype] * np.abs(want) + (n + 40) * 2.0 ** -24 * size + tiny)


def test_matvec_infinite_input():
    """fp32: an infinity or a NaN in X is one in the result, as IEEE arithmetic has it, not an artefact of the parts."""
    print("quant matvec, infinities", flush=True)
    codes = np.full((2, 32), 2, dtype=np.uint8)  # ones
    X = torch.zeros(32, 3, device=dev())
    X[4, 0], X[5, 1], X[6, 2] = float("inf"), float("-inf"), float("nan")
    X += 1
    Y = lrbi.quant_matvec(torch.from_numpy(store.packed_nibbles(codes)).to(dev()), torch.full((2, 4), 127, dtype=torch.uint8, device=dev()), X)
    assert torch.equal(Y[:, 0], torch.full((2,), float("inf"), device=dev())) and torch.equal(Y[:, 1], -Y[:, 0]) and torch.isnan(Y[:, 2]).all()
