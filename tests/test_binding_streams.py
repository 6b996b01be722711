"""Calls with `stream=`: the tensors that a call makes come from that stream's memory, so that its kernels do not write over what the current
stream still reads, and what is handed out is marked as used by the current stream.  Without a GPU: torch's allocation and streams are
stood in for."""
import contextlib
import types

import pytest
import torch

import paper_1905_05686_amd as lrbi
from paper_1905_05686_amd import binding


class _Stream:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


class _Made(torch.Tensor):
    """A tensor that knows the stream its memory belongs to and those it was marked for."""

    def record_stream(self, stream):
        self.marked.append(stream)


class _Library:
    def __getattr__(self, name):
        return lambda *args: 0


@pytest.fixture
def torch_stand_in(monkeypatch):
    here, side, made = _Stream(5), _Stream(6), []
    on = [here]
    empty = torch.empty

    def make(*args, **kw):
        t = empty(*args, **kw).as_subclass(_Made)
        t.owner, t.marked = on[-1], []
        made.append(t)
        return t

    @contextlib.contextmanager
    def stream(s):
        on.append(on[-1] if s is None else s)
        yield
        on.pop()

    monkeypatch.setattr(torch, "empty", make)
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: {here.cuda_stream: here, side.cuda_stream: side}[handle])
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *device: on[-1])
    monkeypatch.setattr(binding, "load_library", lambda: _Library())
    monkeypatch.setattr(binding, "_device_of", lambda t, what: 0)
    monkeypatch.setattr(binding, "_ptr_on", lambda device, t, what: t.data_ptr())
    monkeypatch.setattr(binding, "_dev_ptr", lambda t, what: t.data_ptr())
    return here, side, made


D = lrbi.Desc(64, 96, 32, 32, 4)
W, X, DY = torch.zeros(64, 96), torch.zeros(96, 40), torch.zeros(64, 40)
IP, IZ = torch.zeros(6 * 32, 1, dtype=torch.int32), torch.zeros(6 * 4, 2, dtype=torch.int32)
CODES4, CODES8, SCALES = torch.zeros(64, 48, dtype=torch.uint8), torch.zeros(96, 64, dtype=torch.uint8), torch.zeros(96, 4, dtype=torch.uint8)
MP, MZ, TP = torch.zeros(6, 32, 4), torch.zeros(6, 4, 32), torch.zeros(6)
CONV, ACT = lrbi.Desc(64, 36, 32, 32, 4), torch.zeros(2, 5, 6, 4)
CELL = lrbi.Desc(64, 48, 32, 32, 4)
TOKENS, ROW = torch.zeros(40, dtype=torch.int64), torch.zeros(40)
RESULT = lrbi.TokenLogprobs(ROW, ROW, torch.zeros(2, 40), None, None)
# (call, tensors it hands out, scratch that it makes for itself)
CALLS = {
    "decode_mask": (lambda s: lrbi.decode_mask(D, IP, IZ, stream=s), 1, 0),
    "masked_gemm": (lambda s: lrbi.masked_gemm(D, W, IP, IZ, X, stream=s), 1, 0),
    "decode_and_gemm": (lambda s: lrbi.decode_and_gemm(D, W, IP, IZ, X, stream=s), 2, 0),
    "masked_conv3x3": (lambda s: lrbi.masked_conv3x3(CONV, torch.zeros(64, 36), IP, IZ, ACT, stream=s), 1, 0),
    "masked_gemm_t": (lambda s: lrbi.masked_gemm_t(D, W, IP, IZ, DY, stream=s), 1, 0),
    "masked_grad": (lambda s: lrbi.masked_grad(D, DY, X, IP, IZ, stream=s), 1, 0),
    "threshold_eval": (lambda s: lrbi.threshold_eval(D, W, 0.0, MP, MZ, TP, TP, want_factors=True, stream=s), 4, 0),
    "search_thresholds": (lambda s: lrbi.search_thresholds(D, W, 0.0, MP, MZ, 0.9, [0.5], 4, 10, want_factors=True, stream=s), 6, 1),
    "lstm_step": (lambda s: lrbi.lstm_step(CELL, torch.zeros(64, 48), IP, IZ, torch.zeros(48, 8), torch.zeros(16, 8), torch.zeros(16, 8), stream=s), 0, 1),
    "nmf": (lambda s: lrbi.nmf(D, W, MP, MZ, 3, stream=s), 0, 1),
    "quant_pack": (lambda s: lrbi.quant_pack(D, W, IP, IZ, stream=s), 2, 0),
    "quant_unpack": (lambda s: lrbi.quant_unpack(CODES4, SCALES[:64], 96, torch.float32, stream=s), 1, 0),
    "quant_matvec": (lambda s: lrbi.quant_matvec(CODES4, SCALES[:64], X, stream=s), 1, 0),
    "checkpoint_pack": (lambda s: lrbi.checkpoint_pack(X, stream=s), 2, 0),
    "checkpoint_unpack": (lambda s: lrbi.checkpoint_unpack(CODES8, SCALES, 40, torch.float32, stream=s), 1, 0),
    "checkpoint_grad": (lambda s: lrbi.checkpoint_grad(D, DY, CODES8, SCALES, IP, IZ, stream=s), 1, 0),
    "token_logprobs": (lambda s: lrbi.token_logprobs(DY, TOKENS, top=3, stream=s), 5, 1),
    "token_logprobs_grad": (lambda s: lrbi.token_logprobs_grad(DY, TOKENS, RESULT, ROW, stream=s), 1, 0),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_of_the_calls_stream(torch_stand_in, name):
    here, side, made = torch_stand_in
    call, outputs, scratch = CALLS[name]
    call(side)
    assert len(made) == outputs + scratch
    assert all(t.owner is side for t in made)
    assert sum(t.marked == [here] for t in made) == outputs and all(t.marked in ([here], []) for t in made)


@pytest.mark.parametrize("name", CALLS)
def test_current_stream(torch_stand_in, name):
    """Without a stream, or with the current one: that one's memory, and nothing to mark."""
    here, _, made = torch_stand_in
    call, outputs, scratch = CALLS[name]
    binding._look_up_torch()
    old, binding._current_stream = binding._current_stream, lambda: here.cuda_stream
    try:
        for s in (None, here):
            made.clear()
            call(s)
            assert len(made) == outputs + scratch and all(t.owner is here and not t.marked for t in made)
    finally:
        binding._current_stream = old


@pytest.mark.parametrize("name", CALLS)
def test_stream_of_another_library(torch_stand_in, name):
    """An object with nothing but a stream's handle."""
    here, side, made = torch_stand_in
    CALLS[name][0](types.SimpleNamespace(cuda_stream=side.cuda_stream))
    assert all(t.owner is side for t in made) and sum(t.marked == [here] for t in made) == CALLS[name][1]
