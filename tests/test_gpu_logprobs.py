"""Token log probabilities on the GPU against the fp64 oracle, and their gradient."""
import math

import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
from oracle import logprobs as orc
from gpu_util import TORCH_DTYPE, dev, to_float64

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -150, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}
DTYPES = ["f32", "f16", "bf16"]


def _near(got, want, tol):
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want))
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf])
    fine = np.isfinite(want)
    assert np.all(np.abs(got[fine] - want[fine]) <= np.broadcast_to(tol, want.shape)[fine]), np.max(np.abs(got[fine] - want[fine]))


def _check(logits, tokens, top, dtype, result=None):
    """Tolerances.  log s: 32 additions a lane and run of rows, a rescaling every 16 rows, at most 9 joins in a workgroup and
    14 more of its partial sums, each join a product, a sum and two exponentials of 2 units in the last place: below 120
    roundings of 2^-24 on a sum of positive terms, 7e-6; a term e^d is off by at most 25 * 2^-24 of itself (1.5e-6) for all d
    that count: 1e-5 together.  log p adds a rounding of its own size.  t / s has terms of one sign too: 1e-5 of its size,
    which is at most log V."""
    V, N = logits.shape
    r = lrbi.token_logprobs(logits, tokens, top=top) if result is None else result
    x = to_float64(logits)
    lp = orc.log_probs(x)
    lse_tol = 1e-5 * (1 + 2 * (V * N > 2 ** 24))
    if tokens is not None:
        want = orc.of_tokens(lp, tokens.cpu().numpy())
        _near(to_float64(r.logp), want, lse_tol + 2.0 ** -22 * np.where(np.isfinite(want), np.abs(want), 0))
    H = orc.entropy(lp)
    _near(to_float64(r.entropy), H, lse_tol * (1 + math.log(V)))
    if top:
        ids = orc.top(x, top)
        assert np.array_equal(r.top_ids.cpu().numpy(), ids)
        want = np.where(ids < 0, -np.inf, np.take_along_axis(lp, np.maximum(ids, 0), axis=0))
        _near(to_float64(r.top_logp), want, lse_tol + 2.0 ** -22 * np.where(np.isfinite(want), np.abs(want), 0))
    else:
        assert r.top_ids.shape == (0, N) and r.top_logp.shape == (0, N)
    stats = to_float64(r.stats)
    fine = np.isfinite(x).any(axis=0) & ~np.isnan(lp).any(axis=0)
    with np.errstate(invalid="ignore"):
        m = x.max(axis=0)
        assert np.array_equal(stats[0][fine], m[fine])
        lse = np.log(np.exp(x - m).sum(axis=0))
    assert np.all(np.abs(stats[1] * math.log(2) - lse)[fine] <= lse_tol + 2.0 ** -23 * np.abs(m[fine]))
    return r


def _grad_check(logits, tokens, r, gl, gh, dtype, out=None):
    """p is off by 1e-5 of itself at most (above), log p + H by 1e-5 (2 + log V); the result is rounded once."""
    V, N = logits.shape
    x = to_float64(logits)
    got = to_float64(lrbi.token_logprobs_grad(logits, tokens, r, gl, gh, out=out))
    gl64 = None if gl is None else to_float64(gl)
    gh64 = None if gh is None else to_float64(gh)
    want = orc.grad(x, None if tokens is None else tokens.cpu().numpy(), gl64, gh64)
    lp = orc.log_probs(x)
    p, l = np.exp(lp), np.where(np.isneginf(lp), 0, lp)
    a = np.zeros(N) if gl is None else np.abs(gl64)
    b = np.zeros(N) if gh is None else np.abs(gh64)
    tol = HALF[dtype] * np.abs(want) + 2e-5 * p * (a + b * (np.abs(l) + orc.entropy(lp) + 2 + math.log(V))) + TINY[dtype]
    _near(got, want, np.where(np.isnan(tol), 0, tol))


def _logits(V, N, dtype, seed, sigma=3.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(V, N, generator=gen) * sigma).to(TORCH_DTYPE[dtype]).to(dev())


def _tokens(V, N, seed):
    return torch.randint(-1, V, (N,), generator=torch.Generator().manual_seed(seed)).to(dev())


SHAPES = [(1, 1, 1), (1, 3, 2), (2, 1, 5), (31, 4, 3), (33, 7, 40), (64, 2, 64), (100, 1, 8), (1000, 20, 8), (1000, 33, 1), (5000, 1, 20), (10000, 6, 64),
          (257, 129, 4), (40, 600, 5), (70000, 3, 20), (3000, 64, 0), (2049, 512, 2)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,N,top", SHAPES)
def test_forward_and_gradient(dtype, V, N, top):
    print("logprobs", dtype, V, N, top, flush=True)
    logits, tokens = _logits(V, N, dtype, V + N), _tokens(V, N, V)
    r = _check(logits, tokens, top, dtype)
    gen = torch.Generator().manual_seed(N)
    gl, gh = (torch.randn(N, generator=gen).to(dev()) for _ in range(2))
    _grad_check(logits, tokens, r, gl, gh, dtype)
    _grad_check(logits, tokens, r, gl, None, dtype)
    _grad_check(logits, None, r, None, gh, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,N,top", [(20000, 431, 0), (39000, 431, 3), (131071, 301, 20), (2000, 4097, 0)])
def test_many_odd_columns(dtype, V, N, top):
    """Rows that no piece of several columns divides: what stands beside them stays, and the gradient may take the logits' place."""
    print("logprobs, odd columns", dtype, V, N, top, flush=True)
    gen = torch.Generator(device=dev()).manual_seed(V + N)
    whole = torch.randn(V, N + 2, device=dev(), generator=gen).mul_(3).to(TORCH_DTYPE[dtype])
    logits, tokens = whole[:, 1:1 + N], torch.randint(-1, V, (N,), device=dev(), generator=gen)
    r = lrbi.token_logprobs(logits, tokens, top=top)
    x = logits.double()
    lp = torch.log_softmax(x, 0)
    p = lp.exp()
    H = -(p * lp).sum(0)
    own = torch.where(tokens < 0, 0, lp.gather(0, tokens.clamp(min=0)[None])[0])
    tol = 3e-5 + 2.0 ** -22 * lp.abs().max()  # as in _check
    assert ((r.logp - own).abs() <= tol).all() and ((r.entropy - H).abs() <= 3e-5 * (1 + math.log(V))).all()
    assert torch.equal(r.stats[0].double(), x.max(0).values)
    if top:
        order = torch.sort(x, dim=0, descending=True, stable=True)
        assert torch.equal(r.top_ids, order.indices[:top]) and ((r.top_logp - lp.gather(0, r.top_ids)).abs() <= tol).all()
        del order
    gl, gh = (torch.randn(N, device=dev(), generator=gen) for _ in range(2))
    want = torch.zeros_like(lp).scatter_(0, tokens.clamp(min=0)[None], torch.where(tokens < 0, 0.0, gl).double()[None])
    gl64, gh64 = torch.where(tokens < 0, 0.0, gl).double(), gh.double()
    want -= p * (gl64 + gh64 * (lp + H))
    tol = HALF[dtype] * want.abs() + 2e-5 * p * (gl64.abs() + gh64.abs() * (lp.abs() + H + 2 + math.log(V))) + TINY[dtype]  # as in _grad_check
    out = torch.full((V, N + 2), 7.0, device=dev()).to(TORCH_DTYPE[dtype])
    lrbi.token_logprobs_grad(logits, tokens, r, gl, gh, out=out[:, 1:1 + N])
    assert ((out[:, 1:1 + N].double() - want).abs() <= tol).all()
    assert (out[:, 0] == 7).all() and (out[:, -1] == 7).all()
    before = whole[:, [0, -1]].clone()
    lrbi.token_logprobs_grad(logits, tokens, r, gl, gh, out=logits)
    assert torch.equal(whole[:, 1:1 + N], out[:, 1:1 + N]) and torch.equal(whole[:, [0, -1]], before)


@pytest.mark.parametrize("V", [20000, 32769, 65537, 131072, 150000])
def test_top_words_of_large_vocabularies(V):
    """Several rounds of runs, every run in the list, the top words at the end of the last round."""
    print("logprobs, large vocabulary", V, flush=True)
    x = torch.zeros(V, 3, device=dev(), dtype=torch.float16)  # all equal: the lowest words
    x[:, 1] = torch.arange(V, device=dev()).sub(V).mul(2.0 ** -4).clamp(min=-2000.0).half()  # towards the end larger, in groups
    x[:, 2] = torch.randn(V, generator=torch.Generator().manual_seed(V)).half().to(dev())
    for N in (1, 3):
        r = lrbi.token_logprobs(x[:, 3 - N:], None, top=64)
        assert torch.equal(r.top_ids, torch.sort(x[:, 3 - N:], dim=0, descending=True, stable=True).indices[:64])


@pytest.mark.parametrize("dtype", DTYPES)
def test_strided_logits(dtype):
    """Row pitches and first columns of every alignment; the gradient in the logits' own place."""
    print("logprobs, strides", dtype, flush=True)
    V, N = 300, 24
    for off, wide in ((0, 32), (1, 33), (2, 40), (4, 28), (8, 64)):
        whole = _logits(V, wide + 8, dtype, off)
        logits, tokens = whole[:, off:off + N], _tokens(V, N, 1)
        r = _check(logits, tokens, 6, dtype)
        gl = torch.ones(N, device=dev())
        _grad_check(logits, tokens, r, gl, gl, dtype)
        before = whole.clone()
        want = lrbi.token_logprobs_grad(logits, tokens, r, gl, gl)
        lrbi.token_logprobs_grad(logits, tokens, r, gl, gl, out=logits)
        assert torch.equal(logits, want)
        before[:, off:off + N] = want
        assert torch.equal(whole, before)


@pytest.mark.parametrize("dtype", DTYPES)
def test_ties_and_order(dtype):
    """Equal logits by the lower word: constant columns, two values, runs that end in the largest, zeros of both signs, rising and falling columns."""
    print("logprobs, ties", dtype, flush=True)
    V = 3000
    x = torch.zeros(V, 8)
    x[:, 1] = torch.arange(V) % 2
    x[:, 2] = (torch.arange(V) % 32 == 31).float()
    x[::3, 3] = -0.0
    x[:, 4] = torch.arange(V) / V
    x[:, 5] = -torch.arange(V) / V
    x[:, 6] = torch.arange(V) // 300
    x[:, 7] = (torch.randint(0, 4, (V,), generator=torch.Generator().manual_seed(2))).float()
    for top in (1, 20, 64):
        _check(x.to(TORCH_DTYPE[dtype]).to(dev()), None, top, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_masked_words(dtype):
    """Words at -infinity and at the type's lowest value, columns with few, one or no words left, ranges of words."""
    print("logprobs, masks", dtype, flush=True)
    V, N = 2000, 12
    x = _logits(V, N, dtype, 4)
    low = torch.finfo(x.dtype).min
    x[torch.rand(V, N, device=dev()) < 0.5] = -math.inf
    x[:, 1] = -math.inf
    x[:, 2] = -math.inf
    x[77, 2] = 1.5
    x[:, 3] = low
    x[:, 4] = low
    x[1234, 4] = 0.25
    x[:, 5] = -math.inf
    x[100:700, 5] = 1.0
    x[:, 6] = -math.inf
    x[::500, 6] = low
    x[:, 7] = low
    x[3, 7] = -torch.finfo(x.dtype).max / 2
    x[:, 8] = -math.inf
    x[1990:, 8] = torch.arange(10, device=dev()).to(x.dtype)
    x[:, 9] = torch.finfo(x.dtype).max
    x[5, 9] = 0
    tokens = torch.tensor([0, 5, 77, 9, 1234, 300, 500, 3, 1995, 5, -1, 0], device=dev())
    for top in (3, 30):
        r = _check(x, tokens, top, dtype)
    one = torch.ones(N, device=dev())
    _grad_check(x, tokens, r, one, None, dtype)
    _grad_check(x, tokens, r, one, -one, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
def test_bad_logits_and_words(dtype):
    print("logprobs, NaN", dtype, flush=True)
    V, N = 500, 6
    x = _logits(V, N, dtype, 5)
    x[17, 1] = math.nan
    x[400, 2] = math.inf
    tokens = torch.tensor([3, 3, 3, V, -5, 2 ** 40], device=dev())
    r = lrbi.token_logprobs(x, tokens, top=4)
    logp, H = to_float64(r.logp), to_float64(r.entropy)
    assert np.isnan(logp[[1, 2, 3, 5]]).all() and np.isfinite(logp[[0, 4]]).all() and logp[4] == 0
    assert np.isnan(H[[1, 2]]).all() and np.isfinite(H[[0, 3, 4, 5]]).all()
    assert np.array_equal(r.top_ids.cpu().numpy(), orc.top(to_float64(x), 4)) and r.top_ids[0, 2] == 400
    assert torch.isnan(r.top_logp[:, 1:3]).all() and torch.isfinite(r.top_logp[:, 3:]).all()
    one = torch.ones(N, device=dev())
    g = to_float64(lrbi.token_logprobs_grad(x, tokens, r, one))
    assert np.isnan(g[:, [1, 2, 3, 5]]).all() and np.isfinite(g[:, 0]).all() and (g[:, 4] == 0).all()
    # no gradient comes in: none goes out, whatever the logits
    none = torch.zeros(N, device=dev())
    assert (lrbi.token_logprobs_grad(x, tokens.clamp(max=V - 1), r, none, none) == 0).all()


def test_no_tokens_and_reused_outputs():
    print("logprobs, outputs", flush=True)
    x = _logits(777, 9, "f16", 6)
    r = lrbi.token_logprobs(x, top=5)
    assert r.logp is None
    ws = torch.full((lrbi.token_logprobs_workspace_bytes(lrbi.F16, 777, 9, 5),), 0xFF, dtype=torch.uint8, device=dev())
    for t in r[1:]:
        t.fill_(-7)
    again = lrbi.token_logprobs(x, top=5, out=r, workspace=ws)
    assert again.top_ids is r.top_ids
    _check(x, None, 5, "f16", result=r)
    with pytest.raises(ValueError):
        lrbi.token_logprobs(x, top=4, out=r)
    with pytest.raises(ValueError):
        lrbi.token_logprobs(x, _tokens(777, 9, 1), top=5, out=r)


def test_gradient_against_differences():
    """Forward differences of the GPU's own fp32 results, in steps large enough for their rounding: (L(x + h) - L(x - h)) / 2h with
    h = 2^-5 is off by h^2 / 6 of a third derivative (at most 1 for log p, 4 + 2 log V for the entropy) and 2e-5 / h."""
    print("logprobs, differences", flush=True)
    V, N, h = 50, 4, 2.0 ** -5
    x, tokens = _logits(V, N, "f32", 8, sigma=1.0), torch.tensor([3, 49, 0, -1], device=dev())
    gl, gh = torch.tensor([1.0, -0.5, 0.25, 1.0], device=dev()), torch.tensor([0.5, 1.0, -1.0, 0.25], device=dev())
    g = to_float64(lrbi.token_logprobs_grad(x, tokens, lrbi.token_logprobs(x, tokens), gl, gh))
    for v in (0, 3, 17, 49):
        up, down = x.clone(), x.clone()
        up[v] += h
        down[v] -= h
        a, b = lrbi.token_logprobs(up, tokens), lrbi.token_logprobs(down, tokens)
        loss = [to_float64(gl) * to_float64(r.logp) + to_float64(gh) * to_float64(r.entropy) for r in (a, b)]
        assert np.all(np.abs((loss[0] - loss[1]) / (2 * h) - g[v]) <= h * h / 6 * (5 + 2 * math.log(V)) + 2e-5 * (2 + math.log(V)) / h)


def test_many_rows_of_many_columns():
    """Several runs of rows a lane, several blocks of columns."""
    print("logprobs, large", flush=True)
    V, N = 20000, 1160
    x, tokens = _logits(V, N, "bf16", 9), _tokens(V, N, 2)
    r = lrbi.token_logprobs(x, tokens, top=3)
    xd = x.double()
    lp = torch.log_softmax(xd, dim=0)
    want = torch.where(tokens < 0, 0.0, lp.gather(0, tokens.clamp(min=0)[None])[0])
    assert (r.logp.double() - want).abs().max() <= 3e-5
    H = -(lp.exp() * lp).sum(dim=0)
    assert (r.entropy.double() - H).abs().max() <= 3e-5 * (1 + math.log(V))
    order = torch.sort(xd, dim=0, descending=True, stable=True)[1][:3]
    assert torch.equal(r.top_ids, order)
    g = lrbi.token_logprobs_grad(x, tokens, r, torch.ones(N, device=dev()))
    want = -lp.exp()
    want.scatter_add_(0, tokens.clamp(min=0)[None], torch.ones((1, N), dtype=torch.float64, device=dev()))
    want[:, tokens < 0] = 0
    assert ((g.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2e-5 * lp.exp() + 2.0 ** -134).all()
