"""Argument checks of the token log probabilities, the 4-bit weights and the activation checkpoints, without a GPU: every
refusal comes before any GPU work is queued."""
import ctypes

import pytest
import torch

import paper_1905_05686_amd as lrbi

P = 4096  # an aligned address that is never touched


def _call(name, good, **change):
    args = dict(good, **change)
    lib = lrbi.load_library()
    return getattr(lib, name)(*[ctypes.byref(v) if isinstance(v, lrbi.Desc) else v for v in args.values()])


DESC = lrbi.Desc(100, 70, 64, 64, 4)
PACK = dict(desc=DESC, dtype=lrbi.BF16, W=P, ldw=70, ip=P, iz=P, codes=P, ldc=48, scales=P, lds=4, stream=None)
UNPACK = dict(dtype=lrbi.BF16, codes=P, ldc=48, scales=P, lds=4, m=100, n=70, W=P, ldw=70, stream=None)
MATVEC = dict(dtype=lrbi.BF16, codes=P, ldc=48, scales=P, lds=4, m=100, n=70, X=P, ldx=3, N=3, Y=P, ldy=3, stream=None)
CPACK = dict(dtype=lrbi.F16, X=P, ldx=70, n=100, N=70, codes=P, ldc=96, scales=P, lds=4, stream=None)
CUNPACK = dict(dtype=lrbi.F16, codes=P, ldc=96, scales=P, lds=4, n=100, N=70, X=P, ldx=70, stream=None)
CGRAD = dict(desc=DESC, dtype=lrbi.F16, dY=P, lddy=40, codes=P, ldc=64, scales=P, lds=4, N=40, ip=P, iz=P, dW=P, lddw=70, stream=None)
LOGP = dict(dtype=lrbi.F32, L=P, ldl=9, V=50, N=9, tok=P, logp=P, entropy=P, stats=P, top=3, ids=P, top_logp=P, ws=P, bytes=1 << 30,
            stream=None)
GRAD = dict(dtype=lrbi.F32, L=P, ldl=9, V=50, N=9, tok=P, stats=P, entropy=P, gl=P, gh=P, dL=P, lddl=9, stream=None)

NULL, SHAPE, RANK, DTYPE, PITCH, ALIGN, WORKSPACE, FLAGS = -1, -2, -3, -4, -5, -6, -8, -9
MOST = 0x7FFFFF00

CASES = [("lrbi_quant_pack", PACK, c, s) for c, s in [
    (dict(W=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(ip=None), NULL), (dict(iz=None), NULL),
    (dict(dtype=7), DTYPE), (dict(ldw=69), PITCH), (dict(ldc=32), PITCH), (dict(ldc=56), PITCH), (dict(lds=2), PITCH),
    (dict(lds=6), PITCH), (dict(W=P + 1), ALIGN), (dict(codes=P + 8), ALIGN), (dict(scales=P + 2), ALIGN), (dict(ip=P + 2), ALIGN),
    (dict(iz=P + 4), ALIGN), (dict(desc=lrbi.Desc(0, 70, 64, 64, 4)), SHAPE), (dict(desc=lrbi.Desc(100, 70, 64, 64, 0)), RANK),
    (dict(desc=lrbi.Desc(100, 70, 64, 64, 4, 1 << 30)), FLAGS)]]
CASES += [("lrbi_quant_unpack", UNPACK, c, s) for c, s in [
    (dict(W=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(dtype=-1), DTYPE), (dict(m=0), SHAPE),
    (dict(n=0), SHAPE), (dict(m=MOST + 1), SHAPE), (dict(ldw=69), PITCH), (dict(ldc=40), PITCH), (dict(lds=0), PITCH),
    (dict(codes=P + 4), ALIGN), (dict(scales=P + 1), ALIGN), (dict(W=P + 1), ALIGN)]]
CASES += [("lrbi_quant_matvec", MATVEC, c, s) for c, s in [
    (dict(X=None), NULL), (dict(Y=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(dtype=3), DTYPE),
    (dict(m=0), SHAPE), (dict(n=-1), SHAPE), (dict(N=0), SHAPE), (dict(N=MOST + 1, ldx=MOST + 1, ldy=MOST + 1), SHAPE),
    (dict(ldx=2), PITCH), (dict(ldy=2), PITCH), (dict(ldc=32), PITCH), (dict(lds=2), PITCH), (dict(X=P + 1), ALIGN), (dict(Y=P + 1), ALIGN),
    (dict(codes=P + 8), ALIGN), (dict(scales=P + 2), ALIGN)]]
CASES += [("lrbi_checkpoint_pack", CPACK, c, s) for c, s in [
    (dict(X=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(dtype=9), DTYPE), (dict(n=0), SHAPE),
    (dict(N=0), SHAPE), (dict(ldx=69), PITCH), (dict(ldc=64), PITCH), (dict(ldc=104), PITCH), (dict(lds=2), PITCH),
    (dict(X=P + 1), ALIGN), (dict(codes=P + 8), ALIGN), (dict(scales=P + 2), ALIGN)]]
CASES += [("lrbi_checkpoint_unpack", CUNPACK, c, s) for c, s in [
    (dict(X=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(dtype=9), DTYPE), (dict(n=0), SHAPE),
    (dict(N=-3), SHAPE), (dict(ldx=69), PITCH), (dict(ldc=64), PITCH), (dict(lds=2), PITCH), (dict(X=P + 1), ALIGN),
    (dict(codes=P + 8), ALIGN), (dict(scales=P + 2), ALIGN)]]
CASES += [("lrbi_checkpoint_grad", CGRAD, c, s) for c, s in [
    (dict(dY=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(ip=None), NULL), (dict(iz=None), NULL),
    (dict(dW=None), NULL), (dict(dtype=9), DTYPE), (dict(N=0), SHAPE), (dict(lddy=39), PITCH), (dict(lddw=69), PITCH),
    (dict(ldc=32), PITCH), (dict(lds=1), PITCH), (dict(dY=P + 1), ALIGN), (dict(dW=P + 1), ALIGN), (dict(codes=P + 8), ALIGN),
    (dict(scales=P + 2), ALIGN), (dict(ip=P + 2), ALIGN), (dict(iz=P + 4), ALIGN), (dict(desc=lrbi.Desc(100, 70, 64, 64, 300)), RANK)]]
CASES += [("lrbi_token_logprobs", LOGP, c, s) for c, s in [
    (dict(L=None), NULL), (dict(stats=None), NULL), (dict(ws=None), NULL), (dict(tok=None), NULL), (dict(logp=None), NULL),
    (dict(ids=None), NULL), (dict(top_logp=None), NULL), (dict(dtype=5), DTYPE), (dict(V=0), SHAPE), (dict(N=0), SHAPE),
    (dict(top=-1), SHAPE), (dict(top=65), SHAPE), (dict(V=MOST + 1), SHAPE), (dict(ldl=8), PITCH), (dict(L=P + 2), ALIGN),
    (dict(tok=P + 4), ALIGN), (dict(logp=P + 2), ALIGN), (dict(entropy=P + 2), ALIGN), (dict(stats=P + 1), ALIGN),
    (dict(ids=P + 4), ALIGN), (dict(top_logp=P + 2), ALIGN), (dict(ws=P + 8), ALIGN), (dict(bytes=8), WORKSPACE)]]
CASES += [("lrbi_token_logprobs_grad", GRAD, c, s) for c, s in [
    (dict(L=None), NULL), (dict(stats=None), NULL), (dict(dL=None), NULL), (dict(gl=None, gh=None), NULL), (dict(tok=None), NULL),
    (dict(entropy=None), NULL), (dict(dtype=5), DTYPE), (dict(V=0), SHAPE), (dict(N=0), SHAPE), (dict(ldl=8), PITCH),
    (dict(lddl=8), PITCH), (dict(L=P + 2), ALIGN), (dict(dL=P + 2), ALIGN), (dict(tok=P + 4), ALIGN), (dict(gl=P + 2), ALIGN),
    (dict(gh=P + 2), ALIGN), (dict(stats=P + 2), ALIGN), (dict(entropy=P + 2), ALIGN)]]


@pytest.mark.parametrize("name,good,change,status", CASES, ids=["%s-%s" % (n[5:], ",".join(c)) for n, _, c, _ in CASES])
def test_refused(name, good, change, status):
    assert _call(name, good, **change) == status


def test_workspace_size():
    with pytest.raises(lrbi.LrbiError) as e:
        lrbi.token_logprobs_workspace_bytes(lrbi.F32, 50, 9, 65)
    assert e.value.status == SHAPE
    with pytest.raises(lrbi.LrbiError) as e:
        lrbi.token_logprobs_workspace_bytes(4, 50, 9)
    assert e.value.status == DTYPE
    lib = lrbi.load_library()
    assert lib.lrbi_token_logprobs_workspace_bytes(lrbi.F32, 50, 9, 0, None) == NULL
    none, some = (lrbi.token_logprobs_workspace_bytes(lrbi.F16, 10000, 20, t) for t in (0, 8))
    assert 0 < none < some
    # a workspace one byte short is refused
    need = lrbi.token_logprobs_workspace_bytes(lrbi.F32, 50, 9, 3)
    assert _call("lrbi_token_logprobs", LOGP, bytes=need - 1) == WORKSPACE


def test_binding_refuses_wrong_tensors():
    W = torch.zeros(100, 70)
    codes, scales = torch.zeros(100, 48, dtype=torch.uint8), torch.zeros(100, 4, dtype=torch.uint8)
    for call in (lambda: lrbi.quant_pack(DESC, W.t()), lambda: lrbi.quant_pack(DESC, W),  # the last one: no device tensor
                 lambda: lrbi.quant_pack(DESC, W, out=(codes[:99], scales)), lambda: lrbi.quant_pack(DESC, W, out=(codes[:, :47], scales)),
                 lambda: lrbi.quant_unpack(codes, scales, 97, torch.float32), lambda: lrbi.quant_unpack(codes, scales[:50], 70, torch.float32),
                 lambda: lrbi.quant_unpack(codes.int(), scales, 70, torch.float32),
                 lambda: lrbi.quant_unpack(codes, scales, 70, torch.float32, out=torch.zeros(100, 71)),
                 lambda: lrbi.quant_matvec(codes, scales, torch.zeros(97, 2)), lambda: lrbi.quant_matvec(codes, scales, torch.zeros(2, 70).t()),
                 lambda: lrbi.quant_matvec(codes, scales[1:], torch.zeros(70, 2)),
                 lambda: lrbi.quant_matvec(codes, scales, torch.zeros(70, 2), out=torch.zeros(100, 3)),
                 lambda: lrbi.checkpoint_pack(torch.zeros(70)), lambda: lrbi.checkpoint_pack(torch.zeros(70, 10).t()),
                 lambda: lrbi.checkpoint_unpack(codes, scales, 49, torch.float16),
                 lambda: lrbi.checkpoint_grad(DESC, torch.zeros(99, 20), codes, scales, W, W),
                 lambda: lrbi.checkpoint_grad(DESC, torch.zeros(100, 20), codes, scales, W, W),
                 lambda: lrbi.token_logprobs(torch.zeros(5)), lambda: lrbi.token_logprobs(torch.zeros(5, 6).t()),
                 lambda: lrbi.token_logprobs(torch.zeros(5, 6), torch.zeros(5, dtype=torch.int64)),
                 lambda: lrbi.token_logprobs(torch.zeros(5, 6), torch.zeros(6, dtype=torch.int32)),
                 lambda: lrbi.token_logprobs(torch.zeros(5, 6), out=lrbi.TokenLogprobs(torch.zeros(6), *[torch.zeros(6)] * 4)),
                 lambda: lrbi.token_logprobs(torch.zeros(5, 6), top=-1)):
        with pytest.raises(ValueError):
            call()
