"""Activation checkpoints on the GPU against the oracle: packing and values bit for bit, the weight gradient from them within
the roundings of its sums."""
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


def _inputs(n, N, dtype, seed):
    rng = np.random.default_rng(seed)
    X = rng.standard_normal((n, N)) * np.exp(2 * rng.standard_normal((n, 1)))
    X[rng.random((n, N)) < 0.2] = 0
    return workloads.to_storage(X.astype(np.float32), dtype)


def _check_packed(codes, scales, X64, dtype, N):
    blocks = -(-N // 32)
    want, exps = store.pack8(X64, dtype)
    assert np.array_equal(scales.cpu().numpy()[:, :blocks], exps)
    got = codes.cpu().numpy()[:, :32 * blocks]
    nan = (want & 127) == 127
    assert np.array_equal((got & 127) == 127, nan)
    zero = (want & 127) == 0  # of either sign
    assert np.array_equal(np.where(nan | zero, got & 127, got), np.where(nan | zero, want & 127, want))
    return want, exps


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,N", [(1, 1), (3, 7), (5, 31), (4, 32), (9, 33), (70, 64), (33, 100), (6, 1000)])
def test_pack_and_unpack(dtype, n, N):
    print("checkpoint", dtype, n, N, flush=True)
    X = _inputs(n, N, dtype, n + N)
    codes, scales = lrbi.checkpoint_pack(to_device(X, dtype))
    want, exps = _check_packed(codes, scales, workloads.to_float64(X, dtype), dtype, N)
    assert np.all(codes.cpu().numpy()[:, N:] == 0)
    back = lrbi.checkpoint_unpack(codes, scales, N, TORCH_DTYPE[dtype])
    assert np.array_equal(to_float64(back), store.unpack8(want, exps, N))


@pytest.mark.parametrize("dtype", DTYPES)
def test_pack_at_the_ends_of_the_range(dtype):
    print("checkpoint, range", dtype, flush=True)
    fi = torch.finfo(TORCH_DTYPE[dtype])
    rows = [[448.0], [464.0], [465.0], [17.0, 19.0, 256.0, 2.0 ** -10, 3 * 2.0 ** -10], [fi.max], [-fi.max, 1.0], [fi.max / 4], [fi.smallest_normal],
            [fi.smallest_normal * fi.eps, fi.smallest_normal * fi.eps * 5], [0.0], [np.inf, 1.0], [np.nan, -2.0, -np.inf], [np.inf], [1e4, 1e-4]]
    X = np.zeros((len(rows), 40), dtype=np.float32)
    for i, v in enumerate(rows):
        X[i, 3:3 + len(v)] = v
    X[:, 35] = 0.7
    X = workloads.to_storage(X, dtype)
    codes, scales = lrbi.checkpoint_pack(to_device(X, dtype))
    want, exps = _check_packed(codes, scales, workloads.to_float64(X, dtype), dtype, 40)
    back, ref = to_float64(lrbi.checkpoint_unpack(codes, scales, 40, TORCH_DTYPE[dtype])), store.unpack8(want, exps, 40)
    nan = np.isnan(ref)
    assert np.array_equal(np.isnan(back), nan) and np.array_equal(back[~nan], ref[~nan])


def test_strided_buffers_and_untouched_bytes():
    print("checkpoint strides", flush=True)
    n, N = 21, 45
    for off in (0, 1, 8):
        X = torch.randn(n, N + 19, device=dev()).bfloat16()[:, off:off + N]
        plain = lrbi.checkpoint_pack(X.contiguous())
        codes = torch.full((n, 96), 0xAB, dtype=torch.uint8, device=dev())
        scales = torch.full((n, 8), 0xCD, dtype=torch.uint8, device=dev())
        lrbi.checkpoint_pack(X, out=(codes, scales))
        assert torch.equal(codes[:, :64], plain[0]) and torch.equal(scales[:, :2], plain[1][:, :2])
        assert (codes[:, 64:] == 0xAB).all() and (scales[:, 2:] == 0xCD).all()
        out = torch.full((n, N + 16), 7.0, dtype=torch.bfloat16, device=dev())
        lrbi.checkpoint_unpack(codes, scales, N, torch.bfloat16, out=out[:, off:off + N])
        assert torch.equal(out[:, off:off + N], lrbi.checkpoint_unpack(*plain, N, torch.bfloat16))
        assert (out[:, :off] == 7).all() and (out[:, off + N:] == 7).all()


# shapes of every route: whole 128 x 128 and 256 x 256 blocks, cut-off tiles, ranks above 64, tile widths that line up with
# nothing, batches that end inside a block, one column
GRADS = [(1, 1, 1, 1, 1, 1), (20, 30, 7, 11, 3, 5), (130, 200, 64, 64, 8, 33), (256, 512, 128, 128, 8, 64), (300, 260, 100, 100, 70, 100),
         (128, 192, 128, 64, 16, 40), (256, 576, 256, 192, 32, 96), (512, 384, 256, 128, 12, 31), (129, 257, 128, 128, 4, 128)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,r,c,k,N", GRADS)
def test_grad(dtype, m, n, r, c, k, N):
    print("checkpoint grad", dtype, m, n, r, c, k, N, flush=True)
    _grad(dtype, m, n, r, c, k, N)


def _grad(dtype, m, n, r, c, k, N, dY_pad=0, dW_pad=0):
    rng = np.random.default_rng(m + n + N)
    d = lrbi.Desc(m, n, r, c, k)
    Ip01, Iz01 = workloads.make_factors(rng, d.tiles, r, c, k, 0.4 if k < 10 else 0.2)
    dIp, dIz = device_factors(d, Ip01, Iz01)
    M = orc.decode_mask(Ip01, Iz01, m, n, r, c, k)
    X64 = workloads.to_float64(_inputs(n, N, dtype, n + N), dtype)
    codes8, exps = store.pack8(X64, dtype)
    Xq = store.unpack8(codes8, exps, N)
    codes, scales = lrbi.checkpoint_pack(to_device(_inputs(n, N, dtype, n + N), dtype))
    dY = workloads.to_storage(rng.standard_normal((m, N)).astype(np.float32), dtype)
    dYd = to_device(dY, dtype)
    if dY_pad:
        wide = torch.full((m, N + dY_pad), float("nan"), dtype=dYd.dtype, device=dev())
        wide[:, :N] = dYd
        dYd = wide[:, :N]
    out = torch.full((m, n + dW_pad), 7.0, dtype=dYd.dtype, device=dev())
    lrbi.checkpoint_grad(d, dYd, codes, scales, dIp, dIz, out=out[:, :n])
    assert (out[:, n:] == 7).all()
    got = to_float64(out[:, :n])
    dY64 = workloads.to_float64(dY, dtype)
    want, size = orc.masked_grad(dY64, Xq, M), np.abs(dY64) @ np.abs(Xq).T
    assert np.all(got[M == 0] == 0)
    # exact operands; at most N additions, in fp32, and one rounding on store
    tiny = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}[dtype]
    assert np.all(np.abs(got - want) <= HALF[dtype] * np.abs(want) + N * 2.0 ** -24 * size + tiny)


@pytest.mark.parametrize("dtype", DTYPES)
def test_grad_of_strided_operands(dtype):
    print("checkpoint grad, strides", dtype, flush=True)
    _grad(dtype, 140, 200, 64, 64, 8, 50, dY_pad=3, dW_pad=1)
    _grad(dtype, 256, 256, 128, 128, 8, 64, dY_pad=8, dW_pad=8)


def test_grad_is_the_difference_of_a_linear_loss():
    """L(W) = sum(dY * ((W o I_a) Xq)) is linear in W: its difference along any direction is the gradient's product with it."""
    print("checkpoint grad, differences", flush=True)
    m, n, r, c, k, N = 96, 128, 32, 64, 6, 48
    rng = np.random.default_rng(9)
    d = lrbi.Desc(m, n, r, c, k)
    Ip01, Iz01 = workloads.make_factors(rng, d.tiles, r, c, k, 0.4)
    M = orc.decode_mask(Ip01, Iz01, m, n, r, c, k)
    codes, scales = lrbi.checkpoint_pack(to_device(_inputs(n, N, "f32", 1), "f32"))
    Xq = to_float64(lrbi.checkpoint_unpack(codes, scales, N, torch.float32))
    dY = rng.standard_normal((m, N)).astype(np.float32)
    dW = to_float64(lrbi.checkpoint_grad(d, to_device(dY, "f32"), codes, scales, *device_factors(d, Ip01, Iz01)))
    for seed in range(4):
        D = np.random.default_rng(seed).standard_normal((m, n))
        diff = (dY.astype(np.float64) * orc.masked_gemm(D, M, Xq)).sum()  # L(W + D) - L(W)
        size = ((np.abs(dY).astype(np.float64) @ np.abs(Xq).T) * M * np.abs(D)).sum()
        assert abs((dW * D).sum() - diff) <= (N + 1) * 2.0 ** -24 * size


def test_nan_codes_reach_their_weights():
    print("checkpoint grad, NaN", flush=True)
    X = torch.ones(64, 40, device=dev()).half()
    X[5, 33] = float("nan")
    codes, scales = lrbi.checkpoint_pack(X)
    d = lrbi.Desc(32, 64, 32, 64, 1)
    Ip01, Iz01 = np.ones((1, 32, 1), dtype=np.uint8), np.ones((1, 1, 64), dtype=np.uint8)
    Ip01[0, 3] = 0
    for t in (torch.float16, torch.float32):
        dW = lrbi.checkpoint_grad(d, torch.ones(32, 40, device=dev(), dtype=t), codes, scales, *device_factors(d, Ip01, Iz01))
        bad = torch.isnan(dW)
        assert bad[:, 5].sum() == 31 and bad.sum() == 31 and not bad[3, 5] and (dW[3] == 0).all()


def test_gradient_of_tiny_numbers():
    """fp32 dY of 2^-100 to below the normal numbers: three bf16 parts hold each to 2^-133."""
    print("checkpoint grad, tiny", flush=True)
    m, n, N = 64, 96, 40
    d = lrbi.Desc(m, n, 64, 96, 1)
    ip, iz = device_factors(d, np.ones((1, m, 1), dtype=np.uint8), np.ones((1, 1, n), dtype=np.uint8))
    gen = torch.Generator().manual_seed(5)
    X = torch.randn(n, N, generator=gen).mul_(2.0 ** 60).to(dev())
    dY = torch.ldexp(torch.randn(m, N, generator=gen), torch.arange(-140, -100).repeat_interleave(N * m // 40).reshape(m, N)).to(dev())
    kept = lrbi.checkpoint_pack(X)
    Xq = lrbi.checkpoint_unpack(*kept, N, torch.float32).double()
    got, want, size = lrbi.checkpoint_grad(d, dY, *kept, ip, iz).double(), dY.double() @ Xq.T, dY.double().abs() @ Xq.abs().T
    # parts: 2^-133 a product; sums: N roundings; the store: half a step
    assert ((got - want).abs() <= 2.0 ** -133 * Xq.abs().sum(1)[None] + N * 2.0 ** -24 * size + 2.0 ** -24 * want.abs()).all()


# large enough for 256 x 256 blocks; batches of few slabs of 32 columns, of eight and one more, of odd numbers of them
@pytest.mark.parametrize("dtype,m,n,r,c,k,N", [("bf16", 4096, 4096, 512, 512, 32, 128), ("f16", 4096, 4096, 256, 256, 16, 288), ("bf16", 4096, 4096, 128, 64, 40, 544),
                                               ("f16", 2304, 4096, 256, 256, 16, 1024), ("bf16", 4096, 9216, 256, 256, 16, 96)])
def test_grad_of_large_layers(dtype, m, n, r, c, k, N):
    print("checkpoint grad, large", dtype, m, n, r, c, k, N, flush=True)
    _large(dtype, m, n, r, c, k, N)


# more 128 x 128 blocks than half the compute units, and more than are resident at once; rows that no alignment holds for
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,r,c,k,N", [(1500, 1603, 100, 100, 12, 77), (2000, 1500, 128, 64, 40, 130), (1666, 2500, 250, 300, 70, 3),
                                         (64, 20001, 64, 64, 64, 200), (4000, 4001, 250, 250, 16, 65)])
def test_grad_of_many_blocks(dtype, m, n, r, c, k, N):
    print("checkpoint grad, many blocks", dtype, m, n, r, c, k, N, flush=True)
    _large(dtype, m, n, r, c, k, N)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n", [(100, 130), (1700, 1500)])
def test_codes_behind_the_batch_do_not_count(dtype, m, n):
    """The first 70 of a checkpoint's 128 columns; what stands behind them in their last block, NaN too, is left alone."""
    print("checkpoint grad, columns behind", dtype, m, n, flush=True)
    d = lrbi.Desc(m, n, 100, 128, 8)
    ip, iz = device_factors(d, *workloads.make_factors(np.random.default_rng(3), d.tiles, 100, 128, 8, 0.3))
    gen = torch.Generator(device=dev()).manual_seed(m)
    X = torch.randn(n, 128, device=dev(), generator=gen).to(TORCH_DTYPE[dtype])
    dY = torch.randn(m, 70, device=dev(), generator=gen).to(TORCH_DTYPE[dtype])
    codes, scales = lrbi.checkpoint_pack(X)
    cut = codes.clone()
    cut[:, 70:] = 0
    want = lrbi.checkpoint_grad(d, dY, cut[:, :96], scales[:, :3], ip, iz)
    codes[:, 70:72] = 0x7F
    codes[::3, 79:96] = 0xFF
    assert torch.isfinite(want).all() and torch.equal(lrbi.checkpoint_grad(d, dY, codes[:, :96], scales[:, :3], ip, iz), want)


def _large(dtype, m, n, r, c, k, N):
    rng = np.random.default_rng(N)
    d = lrbi.Desc(m, n, r, c, k)
    ip, iz = device_factors(d, *workloads.make_factors(rng, d.tiles, r, c, k, 0.15))
    gen = torch.Generator(device=dev()).manual_seed(N)
    X = (torch.randn(n, N, device=dev(), generator=gen) * torch.exp(torch.randn(n, 1, device=dev(), generator=gen))).to(TORCH_DTYPE[dtype])
    dY = torch.randn(m, N, device=dev(), generator=gen).to(TORCH_DTYPE[dtype])
    codes, scales = lrbi.checkpoint_pack(X)
    Xq = lrbi.checkpoint_unpack(codes, scales, N, TORCH_DTYPE[dtype]).double()
    got = lrbi.checkpoint_grad(d, dY, codes, scales, ip, iz).double()
    bits = lrbi.decode_mask(d, ip, iz)
    M = ((bits[:, :, None] >> torch.arange(8, device=dev(), dtype=torch.uint8)) & 1).reshape(m, -1)[:, :n].bool()
    want, size = dY.double() @ Xq.T, dY.double().abs() @ Xq.abs().T
    want[~M] = 0
    assert (got[~M] == 0).all()
    assert ((got - want).abs() <= HALF[dtype] * want.abs() + N * 2.0 ** -24 * size + 2.0 ** -25).all()
