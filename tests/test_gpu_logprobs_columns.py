"""Token log probabilities of one contiguous column of a large vocabulary: every sweep of the single launch (up to 32768 words), the run
numbers across its sweeps, and the two launches that read a column in 16-byte pieces beyond that."""
import math

import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
from gpu_util import TORCH_DTYPE, dev
from test_gpu_logprobs import DTYPES, _check, _grad_check

pytestmark = pytest.mark.gpu
SIZES = [8192, 8193, 10000, 16385, 24577, 32767, 32768, 32769, 65537, 131073]


def _column(x, dtype, off):
    """x as a contiguous [V, 1] of the type that begins `off` elements behind a 16-byte aligned address."""
    whole = torch.empty(len(x) + 8, dtype=TORCH_DTYPE[dtype], device=dev())
    assert whole.data_ptr() % 16 == 0
    column = whole[off:off + len(x)].unsqueeze(1)
    column[:, 0] = x.to(column.dtype)
    assert column.stride() == (1, 1)
    return column


# Tolerances: those of _check, whose count holds here: a lane of the single launch adds at most 32 terms at one maximum, then ten joins.
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", SIZES)
def test_one_column(dtype, V):
    print("logprobs, one column", dtype, V, flush=True)
    gen = torch.Generator().manual_seed(V)
    x = torch.randn(V, generator=gen) * 3
    x[torch.rand(V, generator=gen) < 0.2] = -math.inf
    for off, top, word in ((0, 20, V - 1), (1, 64, V // 2), (3, 0, 8191), (0, 1, -1)):
        logits, tokens = _column(x, dtype, off), torch.tensor([word], device=dev())
        r = _check(logits, tokens, top, dtype)
        one = torch.full((1,), 0.75, device=dev())
        _grad_check(logits, tokens, r, one, -one, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", SIZES)
def test_order_of_one_column(dtype, V):
    """Equal logits by the lower word, rising and falling columns, the largest in the last word of a run and of a sweep."""
    print("logprobs, order of one column", dtype, V, flush=True)
    v = torch.arange(V)
    rising = (v - V).mul(2.0 ** -4).clamp(min=-2000.0)
    ends = torch.where((v % 32 == 31) | (v == V - 1), 2.0, 0.0)
    sweeps = torch.where(v % 8192 == 8191, 3.0, ends)
    few = torch.randint(0, 4, (V,), generator=torch.Generator().manual_seed(V)).float()
    for x in (torch.zeros(V), rising, -rising, ends, sweeps, few):
        for off in (0, 1):
            logits = _column(x, dtype, off)
            order = torch.sort(logits, dim=0, descending=True, stable=True)
            for top in (1, 20, 64):
                r = lrbi.token_logprobs(logits, top=top)
                assert torch.equal(r.top_ids, order.indices[:top])
                # as in _check: one maximum, equal terms exactly equal
                lp = torch.log_softmax(logits.double(), 0)
                want = lp.gather(0, r.top_ids)
                assert ((r.top_logp - want).abs() <= 1e-5 + 2.0 ** -22 * want.abs()).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [10000, 32768, 40000])
def test_masked_and_bad_columns(dtype, V):
    """Sweeps without a word, one word in the last place, no word at all, the type's lowest value; a NaN and +infinity in a late sweep."""
    print("logprobs, masks of one column", dtype, V, flush=True)
    low = torch.finfo(TORCH_DTYPE[dtype]).min
    last = torch.full((V,), -math.inf)
    last[V - 1] = 1.5
    late = torch.full((V,), -math.inf)
    late[8192:] = torch.randn(V - 8192, generator=torch.Generator().manual_seed(V))
    lows = torch.full((V,), low)
    some = lows.clone()
    some[9000::7] = 0.5
    for x, word in ((last, V - 1), (late, 5), (late, 9000), (torch.full((V,), -math.inf), 3), (lows, 9999), (some, 9007)):
        logits, tokens = _column(x, dtype, 0), torch.tensor([word], device=dev())
        r = _check(logits, tokens, 30, dtype)
        one = torch.ones(1, device=dev())
        _grad_check(logits, tokens, r, one, one, dtype)
    for bad in (math.nan, math.inf):
        x = late.clone()
        x[9500] = bad
        r = lrbi.token_logprobs(_column(x, dtype, 1), torch.tensor([9100], device=dev()), top=6)
        assert torch.isnan(r.logp).all() and torch.isnan(r.entropy).all() and torch.isnan(r.top_logp).all()
        words = np.array([v for v in torch.sort(late.to(TORCH_DTYPE[dtype]).float(), descending=True, stable=True).indices.tolist() if v != 9500][:6])
        want = words if math.isnan(bad) else np.append(9500, words[:5])
        assert np.array_equal(r.top_ids.cpu().numpy()[:, 0], want)
    r = lrbi.token_logprobs(_column(late, dtype, 0), torch.tensor([V], device=dev()))
    assert torch.isnan(r.logp).all() and torch.isfinite(r.entropy).all()
