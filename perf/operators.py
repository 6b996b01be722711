"""The language-model operators of this library as its users call them: which calls are timed, on which inputs, what their
results are by definition, and the same results from elementary torch operations.

Four groups, which meet in a pruned language model:
  * token log probabilities: the logits Y [V, N] of a masked product (row = word, column = token) are turned into the log
    probability of a given word per column, the column's entropy and its most likely words; and the gradient of the first
    two with respect to the logits, which the masked layer's backward pass takes;
  * 4-bit weights: a pruned weight matrix in 4-bit floating-point codes (sign, 2 exponent bits, 1 mantissa bit) with one
    power-of-two scale per 32 weights of a row, and its product with one or a few columns;
  * 8-bit activation checkpoints: the layer input X [n, N] kept for the backward pass in 8-bit codes (sign, 4, 3) with one
    power-of-two scale per 32 batch columns, and the masked weight gradient from it.
Both formats: scale byte b stands for 2^(b - 127), the smallest power of two at which no value of the block rounds past the
largest code (6 and 448), within the bounds at which every code's value is a number of the source type.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}

# the most a drawn case may take: logits, weights, and multiply-adds of a gradient
MOST_LOGITS = 65536 * 4096
MOST_LOGITS_SERVED = 65536 * 256
MOST_WEIGHTS = 16384 * 16384
MOST_GRAD = 8192 * 8192 * 1024


def listed():
    return [
        # one new word of a language model with 10000 words (Penn Treebank's vocabulary): all latency
        dict(name="logprobs_one", op="logprobs", V=10000, N=1, top=8, banned=False, dtype="f16"),
        # 256 sequences served together, a large vocabulary of which each column may use a part
        dict(name="logprobs_batch", op="logprobs", V=65536, N=256, top=20, banned=True, dtype="bf16"),
        # a training step of the LSTM language model: 20 sequences of 35 words, loss with an entropy term and its gradient
        dict(name="loss_sequences", op="loss", V=10000, N=700, dtype="f32"),
        # the same with a large vocabulary and batch
        dict(name="loss_large", op="loss", V=65536, N=4096, dtype="bf16"),
        # LeNet-5's first fully connected layer on one input
        dict(name="matvec_small", op="matvec", m=500, n=800, N=1, dtype="f32"),
        # one input through a layer of a size met in large models
        dict(name="matvec_large", op="matvec", m=16384, n=16384, N=1, dtype="bf16"),
        # weights put into 4 bits when a model is loaded, and taken out again: an LSTM layer's gates, a large layer with cut-off tiles
        dict(name="weights_lstm", op="weights", m=6000, n=3000, r=300, c=300, k=8, dtype="f16"),
        dict(name="weights_large", op="weights", m=16000, n=9224, r=512, c=512, k=32, dtype="bf16"),
        # a layer input put into 8 bits and taken out: a small batch, a large one
        dict(name="checkpoint_small", op="checkpoint", n=800, N=100, dtype="f32"),
        dict(name="checkpoint_large", op="checkpoint", n=16384, N=4096, dtype="bf16"),
        # the weight gradient from the checkpoint: AlexNet's 9216 -> 4096 layer with cut-off tiles on a ragged batch, and
        # an 8192 -> 8192 layer on a large one
        dict(name="grad_ragged", op="grad", m=4100, n=9224, r=256, c=256, k=16, N=131, dtype="f16"),
        dict(name="grad_large", op="grad", m=8192, n=8192, r=512, c=512, k=32, N=1024, dtype="bf16"),
    ]


def _log_size(rng, lo, hi):
    return max(1, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Spread over the logarithm; half of them odd or ragged, half multiples of 64."""
    v = _log_size(rng, lo, hi)
    return v if v < 64 or rng.random() < 0.5 else v // 64 * 64


def draw(rng):
    op = rng.choice(["logprobs", "loss", "matvec", "weights", "checkpoint", "grad"])
    dtype = rng.choice(["f16", "bf16", "f16", "bf16", "f32"])
    if op == "logprobs":
        V = _size(rng, 1000, 131072)
        return dict(op=op, V=V, N=min(_size(rng, 1, 256), MOST_LOGITS_SERVED // V), top=rng.choice([0, 1, 5, 20, rng.randint(2, 32)]),
                    banned=rng.random() < 0.5, dtype=dtype)
    if op == "loss":
        V = _size(rng, 1000, 131072)
        return dict(op=op, V=V, N=min(_size(rng, 16, 4096), MOST_LOGITS // (2 if dtype == "f32" else 1) // V), dtype=dtype)
    if op == "checkpoint":
        return dict(op=op, n=_size(rng, 200, 16384), N=_size(rng, 8, 4096 if dtype != "f32" else 2048), dtype=dtype)
    if op == "matvec":
        m = _size(rng, 200, 16384)
        return dict(op=op, m=m, n=_size(rng, 200, 16384), N=rng.choice([1, 1, 1, rng.randint(2, 8), rng.randint(2, 32)]), dtype=dtype)
    r = rng.choice([64, 100, 128, 256, 300, 512])
    c = rng.choice([r, r, 64, 128, 256, 320, 512, 576])
    k = rng.choice([4, 8, 16, 32, rng.randint(3, 64)])
    m, n = _size(rng, 200, 8192), _size(rng, 200, 9216)
    r, c = min(r, m), min(c, n)
    if rng.random() < 0.5:  # whole tiles
        m, n = max(1, m // r) * r, max(1, n // c) * c
    case = dict(op=op, m=m, n=n, r=r, c=c, k=k, dtype=dtype)
    if op == "grad":
        case["N"] = max(1, min(_size(rng, 8, 1024), MOST_GRAD // (16 if dtype == "f32" else 2) // (m * n)))
    return case


# --------------------------------------------------------------------------------------------------------- inputs

def _ceil(a, b):
    return -(-a // b)


def _packed_bits(gen, rows, bits, words, p):
    """[rows, words] int32 of Bernoulli(p) bits, the bits past `bits` zero."""
    out = torch.zeros((rows, words), dtype=torch.int32, device="cuda")
    first = 32 * torch.arange(words, device="cuda")
    for b in range(32):
        one = torch.rand((rows, words), device="cuda", generator=gen) < p
        out |= (one & (first + b < bits)).to(torch.int32) << b
    return out


def _factors(case, gen):
    """Packed factors of a mask that keeps about a tenth of the weights."""
    p = math.sqrt(1.0 - 0.9 ** (1.0 / case["k"]))
    tiles = _ceil(case["m"], case["r"]) * _ceil(case["n"], case["c"])
    return (_packed_bits(gen, tiles * case["r"], case["k"], _ceil(case["k"], 32), p),
            _packed_bits(gen, tiles * case["k"], case["c"], 2 * _ceil(case["c"], 64), p))


def _normal(gen, shape, sigma=1.0):
    return torch.randn(shape, device="cuda", generator=gen) * sigma


def _activations(gen, shape, dtype):
    """Layer inputs: rows of different size, as the units of a trained layer have."""
    return (_normal(gen, shape) * torch.exp(_normal(gen, (shape[0], 1)))).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]
    s = dict(case=case)
    if op in ("logprobs", "loss"):
        V, N = case["V"], case["N"]
        tokens = torch.randint(0, V, (N,), device="cuda", generator=gen)
        # a column's sharpness varies; its own word stands out by a few units
        logits = _normal(gen, (V, N)) * (1.0 + 2.0 * torch.rand((1, N), device="cuda", generator=gen))
        logits.scatter_add_(0, tokens[None], 4.0 * torch.rand((1, N), device="cuda", generator=gen) + 2.0)
        if case.get("banned"):  # words that a column may not use
            out = torch.rand((V, N), device="cuda", generator=gen) < 0.2
            out.scatter_(0, tokens[None], False)
            logits.masked_fill_(out, -math.inf)
        s["logits"], s["tokens"] = logits.to(dt), tokens
        if op == "loss":
            s["tokens"][torch.rand(N, device="cuda", generator=gen) < 0.1] = -1  # padding: no word
            s["g_logp"] = -torch.rand(N, device="cuda", generator=gen) / N
            s["g_entropy"] = -0.01 * torch.rand(N, device="cuda", generator=gen) / N
        return s
    if op == "matvec":
        m, n, N = case["m"], case["n"], case["N"]
        W = _normal(gen, (m, n), math.sqrt(2.0 / n))
        W.masked_fill_(torch.rand((m, n), device="cuda", generator=gen) < 0.5, 0.0)
        s["codes"], s["scales"] = _pack4(W, dt)
        s["X"] = _normal(gen, (n, N)).to(dt)
        return s
    if op == "checkpoint":
        s["X"] = _activations(gen, (case["n"], case["N"]), dt)
        return s
    s["ip"], s["iz"] = _factors(case, gen)
    if op == "weights":
        s["W"] = _normal(gen, (case["m"], case["n"]), math.sqrt(2.0 / case["n"])).to(dt)
    else:
        s["dY"] = _normal(gen, (case["m"], case["N"])).to(dt)
        s["codes"], s["scales"] = _pack8(_activations(gen, (case["n"], case["N"]), dt), dt)
    return s


# ---------------------------------------------------------------------------------------------------- formats

# bounds of the scale exponents, by source type: every code's value is then a number of the type
BOUNDS4 = {torch.float16: (-23, 13), torch.bfloat16: (-125, 125), torch.float32: (-125, 125)}
BOUNDS8 = {torch.float16: (-15, 8), torch.bfloat16: (-117, 120), torch.float32: (-117, 120)}
# larger magnitudes are cut: 1.875 times the type's largest power of two, 240 at the largest scale
MOST8 = {torch.float16: 1.875 * 2.0 ** 15, torch.bfloat16: 1.875 * 2.0 ** 127, torch.float32: 1.875 * 2.0 ** 127}


def _power(e):
    """2^e as a 32-bit number, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _blocks(x):
    """[rows, blocks, 32], rows filled up with zeros."""
    wide = _ceil(x.shape[1], 32) * 32
    return torch.nn.functional.pad(x.float(), (0, wide - x.shape[1])).reshape(x.shape[0], wide // 32, 32)


def _scaled(b, shift, past, bounds):
    """The values in units of their block's scale, and its exponent.  The largest code lies in the binade that ends at
    2^shift; past(a): whether a of that binade rounds past it."""
    mant, ex = torch.frexp(b.abs().amax(dim=2))
    e = ex - shift + past(mant * 2.0 ** shift).to(torch.int32)
    e = torch.where(mant == 0, bounds[0], e).clamp(*bounds)
    return b * _power(-e)[:, :, None], e


def _scaled4(W, dt):
    return _scaled(_blocks(W), 3, lambda a: a >= 7.0, BOUNDS4[dt])  # 7 lies between 6 and 8, and 8 is the even one


def _scaled8(X, dt):
    return _scaled(_blocks(X.float().clamp(-MOST8[dt], MOST8[dt])), 9, lambda a: a > 464.0, BOUNDS8[dt])  # here 448 is the even one


def _scale_bytes(e):
    """Rows of whole 4-byte pieces."""
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 4))


def _round4(v):
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return torch.copysign(((a / step).round() * step).clamp(max=6.0), v)


def _pack4(W, dt):
    """4-bit codes, two a byte with the lower column in the lower half, rows of whole 16-byte pieces; scale bytes."""
    v, e = _scaled4(W, dt)
    v = _round4(v)
    a = v.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code |= (v < 0).to(torch.uint8) << 3
    code = code.reshape(W.shape[0], -1, 2)
    return code[:, :, 0] | code[:, :, 1] << 4, _scale_bytes(e)


def _unpack4(codes, scales, n):
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    v = table[torch.stack((codes & 15, codes >> 4), dim=2).int()].reshape(codes.shape[0], -1, 32)
    v = v * _power(scales.int() - 127)[:, :v.shape[1], None]
    return v.reshape(codes.shape[0], -1)[:, :n]


def _pack8(X, dt):
    v, e = _scaled8(X, dt)
    return v.to(torch.float8_e4m3fn).view(torch.uint8).reshape(X.shape[0], -1), _scale_bytes(e)


def _unpack8(codes, scales, N):
    v = codes.view(torch.float8_e4m3fn).float().reshape(codes.shape[0], -1, 32)
    return (v * _power(scales.int() - 127)[:, :v.shape[1], None]).reshape(codes.shape[0], -1)[:, :N]


def _mask(case, ip, iz):
    """The decoded mask [m, n]: per tile the Boolean product of its factors."""
    m, n, r, c, k = (case[x] for x in "mnrck")
    rows, cols = _ceil(m, r), _ceil(n, c)
    shifts = torch.arange(32, device="cuda", dtype=torch.int32)
    a = ((ip.unsqueeze(-1) >> shifts) & 1).reshape(ip.shape[0], -1)[:, :k].reshape(rows * cols, r, k).float()
    b = ((iz.unsqueeze(-1) >> shifts) & 1).reshape(iz.shape[0], -1)[:, :c].reshape(rows * cols, k, c).float()
    t = torch.bmm(a, b) > 0.5
    return t.reshape(rows, cols, r, c).permute(0, 2, 1, 3).reshape(rows * r, cols * c)[:m, :n]


# ------------------------------------------------------------------------------------------------------- one pass

def run(s):
    return _own(s) if own else _plain(s)


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    dt = DTYPES[case["dtype"]]
    if op in ("logprobs", "loss"):
        x = s["logits"].float()
        m = x.amax(dim=0)
        d = x - m
        e = d.exp()
        total = e.sum(dim=0)
        log_total = total.log()
        entropy = log_total - torch.where(e > 0, d * e, 0.0).sum(dim=0) / total
        word = s["tokens"] >= 0
        logp = torch.where(word, d.gather(0, s["tokens"].clamp(min=0)[None])[0] - log_total, 0.0)
        if op == "logprobs":
            ids, top = _most_likely(s["logits"], case["top"])
            return dict(logp=logp, entropy=entropy, top_ids=ids, top_logp=torch.where(ids >= 0, top - m - log_total, -math.inf))
        p = e / total
        logs = d - log_total
        grad = -p * (s["g_logp"] * word + s["g_entropy"] * (torch.where(p > 0, logs, 0.0) + entropy))
        grad.scatter_add_(0, s["tokens"].clamp(min=0)[None], (s["g_logp"] * word)[None])
        return dict(logp=logp, entropy=entropy, grad=grad.to(dt))
    if op == "matvec":
        return (_unpack4(s["codes"], s["scales"], case["n"]) @ s["X"].float()).to(dt)
    if op == "weights":
        kept = torch.where(_mask(case, s["ip"], s["iz"]), s["W"].float(), 0.0)
        v, e = _scaled4(kept, dt)
        return (_round4(v) * _power(e)[:, :, None]).reshape(case["m"], -1)[:, :case["n"]].to(dt)
    if op == "checkpoint":
        return _unpack8(*_pack8(s["X"], dt), case["N"]).to(dt)
    dW = s["dY"].float() @ _unpack8(s["codes"], s["scales"], case["N"]).T
    return torch.where(_mask(case, s["ip"], s["iz"]), dW, 0.0).to(dt)


def _most_likely(logits, top):
    """The `top` largest logits of every column, equal ones by the lower word: as 64-bit keys that no two words share."""
    x = logits.float()
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    word = torch.arange(x.shape[0], device="cuda")[:, None]
    ids = ((order << 32) - word).topk(top, dim=0)[1]
    values = x.gather(0, ids)
    return torch.where(values > -math.inf, ids, -1), values


def _own(s):
    """The calls a program makes.  What it allocates once (outputs, workspaces, descriptors) is kept in the state: the first
    call makes its outputs, the later ones fill them."""
    import paper_1905_05686_amd as lrbi
    case, op = s["case"], s["case"]["op"]
    dt = DTYPES[case["dtype"]]
    kept = s.setdefault("kept", {})
    if op in ("logprobs", "loss"):
        top = case.get("top", 0)
        if not kept:
            code = {"f32": lrbi.F32, "f16": lrbi.F16, "bf16": lrbi.BF16}[case["dtype"]]
            size = lrbi.token_logprobs_workspace_bytes(code, case["V"], case["N"], top)
            kept["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        r = kept["out"] = lrbi.token_logprobs(s["logits"], s["tokens"], top=top, out=kept.get("out"), workspace=kept["ws"])
        if op == "logprobs":
            return dict(logp=r.logp, entropy=r.entropy, top_ids=r.top_ids, top_logp=r.top_logp)
        kept["grad"] = lrbi.token_logprobs_grad(s["logits"], s["tokens"], r, s["g_logp"], s["g_entropy"], out=kept.get("grad"))
        return dict(logp=r.logp, entropy=r.entropy, grad=kept["grad"])
    if op == "matvec":
        kept["Y"] = lrbi.quant_matvec(s["codes"], s["scales"], s["X"], out=kept.get("Y"))
        return kept["Y"]
    if op == "checkpoint":
        kept["packed"] = lrbi.checkpoint_pack(s["X"], out=kept.get("packed"))
        kept["X"] = lrbi.checkpoint_unpack(*kept["packed"], case["N"], dt, out=kept.get("X"))
        return kept["X"]
    if "desc" not in kept:
        kept["desc"] = lrbi.Desc(case["m"], case["n"], case["r"], case["c"], case["k"])
    if op == "weights":
        kept["packed"] = lrbi.quant_pack(kept["desc"], s["W"], s["ip"], s["iz"], out=kept.get("packed"))
        kept["W"] = lrbi.quant_unpack(*kept["packed"], case["n"], dt, out=kept.get("W"))
        return kept["W"]
    kept["dW"] = lrbi.checkpoint_grad(kept["desc"], s["dY"], s["codes"], s["scales"], s["ip"], s["iz"], out=kept.get("dW"))
    return kept["dW"]


def work(case):
    """Each input once, each output once."""
    op, es = case["op"], 4 if case["dtype"] == "f32" else 2
    if op in ("logprobs", "loss"):
        V, N = case["V"], case["N"]
        if op == "logprobs":
            return {"bytes": V * N * es + N * (16 + 12 * case["top"]), "flops": 5.0 * V * N}
        return {"bytes": 2 * V * N * es + 24 * N, "flops": 12.0 * V * N}
    if op == "checkpoint":
        n, N = case["n"], case["N"]
        return {"bytes": 2 * n * N * (es + 1) + 2 * n * _ceil(N, 32), "flops": 0}
    m, n = case["m"], case["n"]
    if op == "matvec":
        N = case["N"]
        return {"bytes": m * n / 2 + m * _ceil(n, 32) + (m + n) * N * es, "flops": 2.0 * m * n * N}
    factors = (case["k"] * (_ceil(n, case["c"]) * m + _ceil(m, case["r"]) * n)) / 8
    if op == "weights":
        return {"bytes": 2 * (m * n * es + m * n / 2 + m * _ceil(n, 32)) + factors, "flops": 0}
    N = case["N"]
    return {"bytes": (m * n + m * N) * es + n * N + n * _ceil(N, 32) + factors, "flops": 2.0 * m * n * N}


# ---------------------------------------------------------------------------------------------- results in 64 bits

def _exact_mask(case, ip, iz):
    m, n, r, c, k = (case[x] for x in "mnrck")
    cols = _ceil(n, c)
    i, j = torch.arange(m, device="cuda"), torch.arange(n, device="cuda")
    out = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    tile = (i // r)[:, None] * cols + (j // c)[None, :]
    for l in range(k):  # the rank's own definition: or over l of (I_p)[i, l] and (I_z)[l, j]
        p = (ip[:, l // 32].long() >> (l % 32)) & 1
        a = p[tile * r + (i % r)[:, None]]
        z = (iz[(tile * k + l), (j % c // 32)[None, :]].long() >> (j % c % 32)[None, :]) & 1
        out |= (a & z).bool()
    return out


def _exact_power(e):
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_store(x, largest, mantissa, least, bounds):
    """Values of blocks of 32 at the smallest power of two, within `bounds`, at which none rounds past `largest`."""
    x = x.double()
    rows, cols = x.shape
    wide = torch.zeros((rows, _ceil(cols, 32) * 32), dtype=torch.float64, device="cuda")
    wide[:, :cols] = x
    b = wide.reshape(rows, -1, 32)
    most = b.abs().amax(dim=2, keepdim=True)

    def rounded(v):
        step = _exact_power(torch.frexp(v.abs().clamp(min=2.0 ** least))[1] - 1 - mantissa)
        return torch.round(v / step) * step

    start = torch.frexp(most.clamp(min=2.0 ** -160) / largest)[1] - 2
    scale = None
    for up in range(3, -1, -1):
        e = start + up
        fits = rounded(most / _exact_power(e)) <= largest
        scale = e if scale is None else torch.where(fits, e, scale)
    scale = _exact_power(scale.clamp(*bounds))
    return (rounded(b / scale).clamp(-largest, largest) * scale).reshape(rows, -1)[:, :cols]


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    dt = DTYPES[case["dtype"]]
    if op in ("logprobs", "loss"):
        x = s["logits"].double()
        lse = torch.logsumexp(x, dim=0)
        logs = x - lse
        p = torch.exp(logs)
        entropy = -torch.special.xlogy(p, p).sum(dim=0)
        known = s["tokens"] >= 0
        at = torch.where(known, s["tokens"], 0)
        logp = torch.where(known, logs[at, torch.arange(case["N"], device="cuda")], 0.0)
        if op == "logprobs":
            # by value, then by word: a stable sort keeps equal logits in the order of the words
            values, ids = torch.sort(x, dim=0, descending=True, stable=True)
            values, ids = values[:case["top"]], ids[:case["top"]]
            return dict(logp=logp, entropy=entropy, top_ids=torch.where(torch.isinf(values), -1, ids), top_logp=values - lse)
        a, b = s["g_logp"].double() * known, s["g_entropy"].double()
        grad = -p * a - b * (torch.special.xlogy(p, p) + p * entropy)
        grad[at, torch.arange(case["N"], device="cuda")] += a
        return dict(logp=logp, entropy=entropy, grad=grad)
    if op == "matvec":
        n = case["n"]
        low, high = (s["codes"] & 15).double(), torch.div(s["codes"], 16, rounding_mode="floor").double()
        code = torch.stack((low, high), dim=2).reshape(case["m"], -1)[:, :n]
        size = code % 8  # 0, 0.5, then 2^(exponent - 1) (1 + mantissa / 2)
        value = torch.where(size < 2, size / 2, _exact_power(torch.floor(size / 2) - 1) * (1 + (size % 2) / 2))
        value = torch.where(code >= 8, -value, value)
        scale = _exact_power(s["scales"].long() - 127).repeat_interleave(32, dim=1)[:, :n]
        return (value * scale) @ s["X"].double()
    if op == "weights":
        W = s["W"].double() * _exact_mask(case, s["ip"], s["iz"])
        return _exact_store(W, 6.0, 1, 0, BOUNDS4[dt])
    if op == "checkpoint":
        return _exact_store(s["X"].double().clamp(-MOST8[dt], MOST8[dt]), 448.0, 3, -6, BOUNDS8[dt])
    code = s["codes"][:, :case["N"]].int()
    exponent, mantissa = (code >> 3) & 15, (code & 7).double()
    X = torch.where(exponent == 0, mantissa * 2.0 ** -9, _exact_power(exponent - 7) * (1 + mantissa / 8))
    X = torch.where(code >= 128, -X, X) * _exact_power(s["scales"].long() - 127).repeat_interleave(32, dim=1)[:, :case["N"]]
    return (s["dY"].double() @ X.T) * _exact_mask(case, s["ip"], s["iz"])
