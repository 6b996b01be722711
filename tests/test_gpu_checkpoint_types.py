"""The weight gradient from a checkpoint of another type than dY's: values that are numbers of dY's type go in exactly, others rounded to it."""
import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
import workloads
from gpu_util import TORCH_DTYPE, dev, device_factors

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


# shapes of the three kernels: few blocks, 128 x 128 blocks, 256 x 256 blocks
@pytest.mark.parametrize("kept,dtype", [("f32", "f16"), ("bf16", "f16"), ("f16", "bf16"), ("f32", "bf16"), ("f16", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("m,n,r,c,k,N", [(96, 160, 32, 64, 6, 48), (1700, 1500, 100, 128, 8, 70), (4096, 4096, 256, 256, 16, 128)])
def test_checkpoint_of_another_type(kept, dtype, m, n, r, c, k, N):
    print("checkpoint grad, types", kept, dtype, m, n, N, flush=True)
    d = lrbi.Desc(m, n, r, c, k)
    ip, iz = device_factors(d, *workloads.make_factors(np.random.default_rng(m), d.tiles, r, c, k, 0.3))
    gen = torch.Generator(device=dev()).manual_seed(n)
    X = torch.randn(n, N, device=dev(), generator=gen)
    if kept != "f16":  # rows from far below f16's smallest number to beyond its largest
        X *= torch.exp2(torch.arange(n, device=dev()) % 52 - 32.0)[:, None]
    codes, scales = lrbi.checkpoint_pack(X.to(TORCH_DTYPE[kept]))
    Xq = lrbi.checkpoint_unpack(codes, scales, N, TORCH_DTYPE[kept])
    Xq = Xq.float().to(TORCH_DTYPE[dtype]).double()
    finite = torch.isfinite(Xq).all(dim=1)
    assert finite.all() == (dtype != "f16")
    dY = torch.rand(m, N, device=dev(), generator=gen).add_(0.25).to(TORCH_DTYPE[dtype])  # positive
    got = lrbi.checkpoint_grad(d, dY, codes, scales, ip, iz).double()
    bits = lrbi.decode_mask(d, ip, iz)
    M = ((bits[:, :, None] >> torch.arange(8, device=dev(), dtype=torch.uint8)) & 1).reshape(m, -1)[:, :n].bool()
    assert (got[~M] == 0).all()
    want, size = dY.double() @ Xq[finite].T, dY.double().abs() @ Xq[finite].abs().T
    # exact products, at most N additions in fp32, one rounding on store
    tol = HALF[dtype] * want.abs() + N * 2.0 ** -24 * size + (2.0 ** -25 if dtype == "f16" else 2.0 ** -134)
    inside, part = M[:, finite], got[:, finite]
    large = inside & (want.abs() > torch.finfo(TORCH_DTYPE[dtype]).max * (1 - HALF[dtype]))  # (f16) at or beyond the type's end
    assert ((part - want).abs() <= tol)[inside & ~large].all()
    assert (part[large].isinf() | ((part - want).abs() <= tol)[large]).all()
    # rows with an infinity of one sign: that infinity; of both: NaN
    beyond = Xq[~finite]
    total = torch.where((beyond == torch.inf).any(1), torch.inf, 0.0) + torch.where((beyond == -torch.inf).any(1), -torch.inf, 0.0)
    rest, kept_rows = got[:, ~finite], M[:, ~finite]
    assert (torch.where(kept_rows, rest, total) == total).logical_or(total.isnan() & torch.where(kept_rows, rest, total).isnan()).all()
