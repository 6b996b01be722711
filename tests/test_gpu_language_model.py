"""The token log probabilities, the 4-bit weights and the activation checkpoints together, as a pruned language model uses them:
a served word and a training step, eager, on another stream and replayed as a graph."""
import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
import workloads
from oracle import logprobs
from oracle import lrbi_oracle as orc
from oracle import store
from gpu_util import TORCH_DTYPE, dev, device_factors, to_device, to_float64

pytestmark = pytest.mark.gpu
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _layer(dtype, V=700, n=300, r=100, c=60, k=6, N=40, seed=0):
    """The output layer of a language model: V words, n hidden units, N tokens."""
    rng = np.random.default_rng(seed)
    d = lrbi.Desc(V, n, r, c, k)
    Ip01, Iz01 = workloads.make_factors(rng, d.tiles, r, c, k, 0.35)
    W = workloads.to_storage((rng.standard_normal((V, n)) * 0.2).astype(np.float32), dtype)
    X = workloads.to_storage(rng.standard_normal((n, N)).astype(np.float32), dtype)
    tokens = torch.from_numpy(rng.integers(-1, V, N)).to(dev())
    return d, orc.decode_mask(Ip01, Iz01, V, n, r, c, k), device_factors(d, Ip01, Iz01), W, X, tokens


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_served_word(dtype):
    print("language model, served", dtype, flush=True)
    d, M, (ip, iz), W, X, tokens = _layer(dtype)
    W64 = workloads.to_float64(W, dtype)
    codes, scales = lrbi.quant_pack(d, to_device(W, dtype), ip, iz)
    x = to_device(X, dtype)
    for N in (1, 7):
        logits = lrbi.quant_matvec(codes, scales, x[:, :N].contiguous())
        res = lrbi.token_logprobs(logits, tokens[:N].contiguous(), top=5)
        Wq = store.unpack4(*store.pack4(W64, M, dtype), d.n)
        X64 = workloads.to_float64(X, dtype)[:, :N]
        want, size = Wq @ X64, np.abs(Wq) @ np.abs(X64)
        got = to_float64(logits)
        assert np.all(np.abs(got - want) <= HALF[dtype] * np.abs(want) + (d.n + 40) * 2.0 ** -24 * size + 2.0 ** -25)
        lp = logprobs.log_probs(got)  # of the logits as stored
        ids = logprobs.top(got, 5)
        assert np.array_equal(res.top_ids.cpu().numpy(), ids)
        assert np.abs(to_float64(res.top_logp) - np.take_along_axis(lp, ids, axis=0)).max() <= 2e-5
        assert np.abs(to_float64(res.logp) - logprobs.of_tokens(lp, tokens[:N].cpu().numpy())).max() <= 2e-5
        assert np.abs(to_float64(res.entropy) - logprobs.entropy(lp)).max() <= 1e-4


class Step:
    """One training step of the output layer with its input kept in 8 bits."""

    def __init__(self, dtype, **kw):
        self.d, self.M, (self.ip, self.iz), W, X, self.tokens = _layer(dtype, **kw)
        self.W, self.X = to_device(W, dtype), to_device(X, dtype)
        self.W64, self.X64 = workloads.to_float64(W, dtype), workloads.to_float64(X, dtype)
        V, n, N = self.d.m, self.d.n, X.shape[1]
        new = lambda *shape: torch.zeros(shape, dtype=TORCH_DTYPE[dtype], device=dev())  # noqa: E731
        self.Y, self.dY, self.dX, self.dW = new(V, N), new(V, N), new(n, N), new(V, n)
        code = {"f32": lrbi.F32, "f16": lrbi.F16, "bf16": lrbi.BF16}[dtype]
        some = lambda b: torch.empty(max(16, b), dtype=torch.uint8, device=dev())  # noqa: E731
        self.ws = some(lrbi.masked_gemm_workspace_bytes(self.d, code, N))
        self.ws_t = some(lrbi.masked_gemm_t_workspace_bytes(self.d, code, N))
        self.ws_l = some(lrbi.token_logprobs_workspace_bytes(code, V, N))
        self.gl = torch.full((N,), -1.0, device=dev())
        self.gh = torch.full((N,), -0.05, device=dev())
        self.packed = self.res = None

    def run(self):
        self.packed = lrbi.checkpoint_pack(self.X, out=self.packed)
        lrbi.masked_gemm(self.d, self.W, self.ip, self.iz, self.X, out=self.Y, workspace=self.ws)
        self.res = lrbi.token_logprobs(self.Y, self.tokens, out=self.res, workspace=self.ws_l)
        lrbi.token_logprobs_grad(self.Y, self.tokens, self.res, self.gl, self.gh, out=self.dY)
        lrbi.masked_gemm_t(self.d, self.W, self.ip, self.iz, self.dY, out=self.dX, workspace=self.ws_t)
        lrbi.checkpoint_grad(self.d, self.dY, *self.packed, self.ip, self.iz, out=self.dW)

    def outputs(self):
        codes, scales = self.packed
        return [self.Y, self.res.logp, self.res.entropy, self.res.stats, self.dY, self.dX, self.dW, codes, scales[:, :-(-self.X.shape[1] // 32)]]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_training_step(dtype):
    print("language model, training", dtype, flush=True)
    s = Step(dtype)
    s.run()
    Y, dY = to_float64(s.Y), to_float64(s.dY)
    tokens, gl, gh = s.tokens.cpu().numpy(), to_float64(s.gl), to_float64(s.gh)
    want = logprobs.grad(Y, tokens, gl, gh)
    lp = logprobs.log_probs(Y)
    p = np.exp(lp)
    tol = HALF[dtype] * np.abs(want) + 2e-5 * p * (np.abs(gl) + np.abs(gh) * (np.abs(lp) + logprobs.entropy(lp) + 9)) + 2.0 ** -25
    assert np.all(np.abs(dY - want) <= tol)
    Xq = store.unpack8(*store.pack8(s.X64, dtype), s.X64.shape[1])
    N, V = Y.shape[1], Y.shape[0]
    want, size = orc.masked_grad(dY, Xq, s.M), np.abs(dY) @ np.abs(Xq).T
    assert np.all(np.abs(to_float64(s.dW) - want) <= HALF[dtype] * np.abs(want) + N * 2.0 ** -24 * size + 2.0 ** -25)
    want, size = orc.masked_gemm_t(s.W64, s.M, dY), np.abs(s.W64).T @ np.abs(dY)
    assert np.all(np.abs(to_float64(s.dX) - want) <= HALF[dtype] * np.abs(want) + V * 2.0 ** -24 * size + 2.0 ** -25)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_on_another_stream_and_replayed(dtype):
    print("language model, graph", dtype, flush=True)
    s = Step(dtype, V=1024, n=512, r=256, c=128, k=8, N=64)
    s.run()
    torch.cuda.synchronize()
    ref = [t.clone() for t in s.outputs()]

    def same():
        for a, b in zip(s.outputs(), ref):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))

    def spoil():
        for t in s.outputs() + [s.ws, s.ws_t, s.ws_l]:
            t.view(torch.uint8).fill_(0x5A)

    side = torch.cuda.Stream()
    spoil()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for _ in range(3):
        spoil()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same()


def test_top_words_and_matvec_in_a_graph():
    print("language model, served in a graph", flush=True)
    d, _, (ip, iz), W, X, tokens = _layer("f16", V=3000, n=500)
    codes, scales = lrbi.quant_pack(d, to_device(W, "f16"), ip, iz)
    x = to_device(X, "f16")[:, :3].contiguous()
    tok = tokens[:3].contiguous()
    ws = torch.empty(lrbi.token_logprobs_workspace_bytes(lrbi.F16, d.m, 3, 10), dtype=torch.uint8, device=dev())
    Y = lrbi.quant_matvec(codes, scales, x)
    res = lrbi.token_logprobs(Y, tok, top=10, workspace=ws)
    ref = [t.clone() for t in (Y, *res)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lrbi.quant_matvec(codes, scales, x, out=Y)
        lrbi.token_logprobs(Y, tok, top=10, out=res, workspace=ws)
    for _ in range(3):
        for t in (Y, ws, *res):
            t.view(torch.uint8).fill_(0x5A)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((Y, *res), ref):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
