"""The 4-bit product of layers with many rows against a product in 64 bits: workgroups that keep X and go over several blocks of rows with
two sets of sums in turn, wavefronts on two and four blocks of rows, the last block cut off."""
import pytest
import torch

import paper_1905_05686_amd as lrbi
from oracle import store
from gpu_util import TORCH_DTYPE, dev

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
DTYPES = ["f32", "f16", "bf16"]


def _matvec(dtype, m, n, N, off=0):
    gen = torch.Generator(device=dev()).manual_seed(m + n + N)
    blocks = -(-n // 32)
    codes = torch.randint(0, 256, (m, 16 * blocks), dtype=torch.uint8, device=dev(), generator=gen)
    scales = torch.randint(118, 125, (m, -(-blocks // 4) * 4), dtype=torch.uint8, device=dev(), generator=gen)
    nibbles = torch.stack((codes & 15, codes >> 4), dim=2).reshape(m, -1)[:, :n].long()
    values = torch.tensor(store.VALUES4, device=dev())
    table = torch.cat((values, -values))
    W = table[nibbles] * torch.exp2(scales[:, :blocks].double() - 127).repeat_interleave(32, dim=1)[:, :n]
    whole = torch.randn(n, N + off, device=dev(), generator=gen).to(TORCH_DTYPE[dtype])
    X = whole[:, off:]
    Y = lrbi.quant_matvec(codes, scales, X if N > 1 or off else X[:, 0]).double().reshape(m, N)
    want, size = W @ X.double(), W.abs() @ X.double().abs()
    # Products are exact.  However they are split among wavefronts, a sum has at most n additions and 40 more of the wavefronts' and parts'
    # sums; the second and third part of fp32 X (2^-8 and 2^-16 of the first) add n roundings of that size each.  One rounding on store.
    tol = HALF[dtype] * want.abs() + (n * (1 + 2.0 ** -7) + 40) * 2.0 ** -24 * size + 2.0 ** -25
    assert ((Y - want).abs() <= tol).all()
    # a wrong set of sums, stale X or a block of rows left out would be off by about its size: far beyond the tolerance
    assert (tol < 0.02 * size).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,N", [(8300, 4200, 1), (16500, 4200, 1), (33000, 2100, 1), (33000, 2100, 3), (33000, 2100, 5), (33000, 700, 20), (70001, 1100, 2),
                                   (66000, 70, 16)])
def test_many_rows(dtype, m, n, N):
    print("quant matvec, many rows", dtype, m, n, N, flush=True)
    _matvec(dtype, m, n, N)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [8300, 16500, 33000])
def test_column_of_a_matrix(dtype, m):
    """One column that is not contiguous: the other loads of X."""
    print("quant matvec, many rows, strided column", dtype, m, flush=True)
    _matvec(dtype, m, 1300, 1, off=3)
