"""Rows whose byte and element offsets pass 2^32: the language-model operators on buffers with very long pitches against the same call
on small ones, bit for bit."""
import torch

import paper_1905_05686_amd as lrbi
import pytest
import workloads
import numpy as np
from gpu_util import dev, device_factors

pytestmark = pytest.mark.gpu


def test_logits_far_apart():
    print("far offsets, logits", flush=True)
    V, N, pitch = 70000, 24, 70016  # 4.9e9 elements
    small = (torch.randn(V, N, device=dev()) * 3).bfloat16()
    wide = torch.empty((V, pitch), dtype=torch.bfloat16, device=dev())
    far = wide[:, pitch - N:]
    far.copy_(small)
    tokens = torch.randint(0, V, (N,), device=dev())
    a, b = lrbi.token_logprobs(small, tokens, top=7), lrbi.token_logprobs(far, tokens, top=7)
    for x, y in zip(a, b):
        assert torch.equal(x, y)
    one = torch.ones(N, device=dev())
    want = lrbi.token_logprobs_grad(small, tokens, a, one, one)
    assert torch.equal(lrbi.token_logprobs_grad(far, tokens, b, one, one, out=far), want)


def test_codes_far_apart():
    print("far offsets, codes", flush=True)
    m, n, pitch = 70000, 256, 65536  # 4.6e9 bytes
    W = torch.randn(m, n, device=dev()).half()
    d = lrbi.Desc(m, n, 100, 64, 3)
    codes, scales = lrbi.quant_pack(d, W)
    far = torch.empty((m, pitch), dtype=torch.uint8, device=dev())[:, :128]
    lrbi.quant_pack(d, W, out=(far, scales))
    assert torch.equal(far, codes)
    x = torch.randn(n, 2, device=dev()).half()
    assert torch.equal(lrbi.quant_matvec(far, scales, x), lrbi.quant_matvec(codes, scales, x))
    assert torch.equal(lrbi.quant_unpack(far, scales, n, torch.float16), lrbi.quant_unpack(codes, scales, n, torch.float16))


def test_checkpoint_far_apart():
    print("far offsets, checkpoint", flush=True)
    n, N, m, pitch = 70016, 64, 128, 65536  # 4.6e9 bytes of codes
    X = torch.randn(n, N, device=dev()).half()
    codes, scales = lrbi.checkpoint_pack(X)
    far = torch.empty((n, pitch), dtype=torch.uint8, device=dev())[:, :N]
    lrbi.checkpoint_pack(X, out=(far, scales))
    assert torch.equal(far, codes)
    assert torch.equal(lrbi.checkpoint_unpack(far, scales, N, torch.float16), lrbi.checkpoint_unpack(codes, scales, N, torch.float16))
    d = lrbi.Desc(m, n, 128, 128, 4)
    rng = np.random.default_rng(1)
    ip, iz = device_factors(d, *workloads.make_factors(rng, d.tiles, 128, 128, 4, 0.4))
    dY = torch.randn(m, N, device=dev())
    for t in (torch.float16, torch.float32):
        want = lrbi.checkpoint_grad(d, dY.to(t), codes, scales, ip, iz)
        assert torch.equal(lrbi.checkpoint_grad(d, dY.to(t), far, scales, ip, iz), want)
