"""Tensors of more than 256 MB, which are read or written past the last-level cache: the same bits as parts of them, or as the same rows at an
alignment that goes through it."""
import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
import workloads
from gpu_util import TORCH_DTYPE, dev, device_factors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n", [("f16", 12003), ("bf16", 12032), ("f32", 6001)])
def test_weights_and_checkpoints(dtype, n):
    print("past the cache, weights", dtype, n, flush=True)
    m, r, c, k, t = 12000, 500, 300, 6, TORCH_DTYPE[dtype]
    gen = torch.Generator(device=dev()).manual_seed(n)
    W = torch.randn(m, n, device=dev(), generator=gen).to(t)
    d, half = lrbi.Desc(m, n, r, c, k), lrbi.Desc(m // 2, n, r, c, k)
    ip, iz = device_factors(d, *workloads.make_factors(np.random.default_rng(n), d.tiles, r, c, k, 0.3))
    codes, scales = lrbi.quant_pack(d, W, ip, iz)
    values = lrbi.quant_unpack(codes, scales, n, t)
    kept = lrbi.checkpoint_pack(W)
    back = lrbi.checkpoint_unpack(*kept, n, t)
    blocks = -(-n // 32)
    for i, rows in enumerate((slice(0, m // 2), slice(m // 2, m))):
        x, y = ip.chunk(2)[i].contiguous(), iz.chunk(2)[i].contiguous()
        part = lrbi.quant_pack(half, W[rows], x, y)
        assert torch.equal(part[0], codes[rows]) and torch.equal(part[1][:, :blocks], scales[rows, :blocks])
        assert torch.equal(lrbi.quant_unpack(*part, n, t), values[rows])
        part = lrbi.checkpoint_pack(W[rows])
        assert torch.equal(part[0], kept[0][rows]) and torch.equal(part[1][:, :blocks], kept[1][rows, :blocks])
        assert torch.equal(lrbi.checkpoint_unpack(*part, n, t), back[rows])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits(dtype):
    print("past the cache, logits", dtype, flush=True)
    V, N = 70000, 2048
    wide = torch.empty(V, N + 8, device=dev(), dtype=TORCH_DTYPE[dtype])
    logits = torch.randn(V, N, device=dev(), generator=torch.Generator(device=dev()).manual_seed(V)).mul_(3).to(TORCH_DTYPE[dtype])
    wide[:, :N] = logits
    tokens = torch.randint(0, V, (N,), device=dev())
    for a, b in zip(lrbi.token_logprobs(logits, tokens), lrbi.token_logprobs(wide[:, :N], tokens)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,m,n", [("f16", 11990, 12032), ("bf16", 12100, 12288), ("f32", 8200, 8224)])
def test_weight_gradient(dtype, m, n):
    print("past the cache, gradient", dtype, m, n, flush=True)
    t, N = TORCH_DTYPE[dtype], 40
    d = lrbi.Desc(m, n, 256, 64, 8)
    ip, iz = device_factors(d, *workloads.make_factors(np.random.default_rng(m), d.tiles, 256, 64, 8, 0.3))
    X, dY = torch.randn(n, N, device=dev()).to(t), torch.randn(m, N, device=dev()).to(t)
    kept = lrbi.checkpoint_pack(X)
    wide = torch.full((m, n + 8), 7.0, device=dev(), dtype=t)
    lrbi.checkpoint_grad(d, dY, *kept, ip, iz, out=wide[:, :n])
    assert torch.equal(lrbi.checkpoint_grad(d, dY, *kept, ip, iz), wide[:, :n]) and (wide[:, n:] == 7).all()
