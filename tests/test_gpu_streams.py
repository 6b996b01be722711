"""Calls on another stream than the current one: the same bits as on it, and no tensor that they make lies where the current stream has just
freed one, which its queued kernels may still read."""
import types

import numpy as np
import pytest
import torch

import paper_1905_05686_amd as lrbi
import workloads
from gpu_util import dev, device_factors

pytestmark = pytest.mark.gpu
M, N_IN, BATCH = 640, 512, 96


@pytest.fixture(scope="module")
def calls():
    d = lrbi.Desc(M, N_IN, 128, 64, 6)
    ip, iz = device_factors(d, *workloads.make_factors(np.random.default_rng(4), d.tiles, 128, 64, 6, 0.3))
    gen = torch.Generator(device=dev()).manual_seed(8)
    W, X, Y = (torch.randn(shape, device=dev(), generator=gen).half() for shape in ((M, N_IN), (N_IN, BATCH), (M, BATCH)))
    codes4, codes8 = lrbi.quant_pack(d, W, ip, iz), lrbi.checkpoint_pack(X)
    tokens = torch.randint(0, M, (BATCH,), device=dev(), generator=gen)
    r, one = lrbi.token_logprobs(Y, tokens), torch.ones(BATCH, device=dev())
    Mp, Mz = (torch.rand(shape, device=dev(), generator=gen) + 0.1 for shape in ((d.tiles, 128, 6), (d.tiles, 6, 64)))
    search = lambda s: lrbi.search_thresholds(d, W, 0.1, Mp, Mz, 0.8, [0.5, 0.7], 4, 100, want_factors=True, stream=s)  # noqa: E731
    return {
        "decode_mask": lambda s: (lrbi.decode_mask(d, ip, iz, stream=s),),
        "masked_gemm": lambda s: (lrbi.masked_gemm(d, W, ip, iz, X, stream=s),),
        "decode_and_gemm": lambda s: lrbi.decode_and_gemm(d, W, ip, iz, X, stream=s),
        "masked_gemm_t": lambda s: (lrbi.masked_gemm_t(d, W, ip, iz, Y, stream=s),),
        "masked_grad": lambda s: (lrbi.masked_grad(d, Y, X, ip, iz, stream=s),),
        "search_thresholds": search,
        "quant_pack": lambda s: lrbi.quant_pack(d, W, ip, iz, stream=s),
        "quant_unpack": lambda s: (lrbi.quant_unpack(*codes4, N_IN, torch.float16, stream=s),),
        "quant_matvec": lambda s: (lrbi.quant_matvec(*codes4, X, stream=s),),
        "checkpoint_pack": lambda s: lrbi.checkpoint_pack(X, stream=s),
        "checkpoint_unpack": lambda s: (lrbi.checkpoint_unpack(*codes8, BATCH, torch.float16, stream=s),),
        "checkpoint_grad": lambda s: (lrbi.checkpoint_grad(d, Y, *codes8, ip, iz, stream=s),),
        "token_logprobs": lambda s: tuple(lrbi.token_logprobs(Y, tokens, top=5, stream=s)),
        "token_logprobs_grad": lambda s: (lrbi.token_logprobs_grad(Y, tokens, r, one, one, stream=s),),
    }


@pytest.mark.parametrize("name", ["decode_mask", "masked_gemm", "decode_and_gemm", "masked_gemm_t", "masked_grad", "search_thresholds",
                                  "quant_pack", "quant_unpack", "quant_matvec", "checkpoint_pack", "checkpoint_unpack", "checkpoint_grad", "token_logprobs",
                                  "token_logprobs_grad"])
def test_call_on_another_stream(calls, name):
    print("streams", name, flush=True)
    call, side = calls[name], torch.cuda.Stream()
    want = call(None)
    torch.cuda.synchronize()
    # tensors of the same sizes, freed on the current stream: the first that an allocation on it would take
    freed = [torch.empty_like(t) for t in want]
    where = [(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()) for t in freed]
    del freed
    got = call(side)
    for t in got:
        begin, end = t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()
        assert all(end <= a or b <= begin for a, b in where)
    torch.cuda.current_stream().wait_stream(side)
    if name == "checkpoint_pack":  # three blocks a row: the fourth scale byte is left as it is
        got, want = (got[0], got[1][:, :3]), (want[0], want[1][:, :3])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["quant_matvec", "checkpoint_grad", "token_logprobs", "masked_gemm", "search_thresholds"])
def test_another_stream_in_a_graph(calls, name):
    """Captured on a stream that forks from the captured one and joins it again; the first call's tensors are freed under capture."""
    print("streams, graph", name, flush=True)
    call, side = calls[name], torch.cuda.Stream()
    want = call(None)
    call(side)  # the kernels' first launch is outside the graph
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        call(side)
        got = call(side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        for t in got:
            t.view(torch.uint8).fill_(0x5A)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.equal(a, b) for a, b in zip(call(None), want))  # the program's own work between the replays


@pytest.mark.parametrize("name", ["decode_mask", "quant_pack", "token_logprobs", "search_thresholds"])
def test_a_streams_handle_alone(calls, name):
    """Streams of other libraries: objects with a handle, the default stream's among them."""
    print("streams, handles", name, flush=True)
    call, side = calls[name], torch.cuda.Stream()
    want = call(None)
    torch.cuda.synchronize()
    for handle in (side.cuda_stream, torch.cuda.default_stream().cuda_stream):
        got = call(types.SimpleNamespace(cuda_stream=handle))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
