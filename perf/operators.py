"""The operators around a quantized model's linears whose speed is tracked, each beside a plain form of it.

Kinds of pass (a case's "kind"):
  logprobs  what a model answers with: of every row of logits the log probability of the given token, the entropy, and
            the top alternatives with their log probabilities (evaluation, serving, the teacher's pass of a distillation)
  loss      the distillation loss of every row against a teacher's top log probabilities (validation)
  grad      the same loss and its gradient with respect to the logits (a training step; the gradient goes on as dY)
  mx_quant  a matrix to microscaled 4-bit floating point, blocks of 32 (weights once, activations in front of a product)
  mx_linear activations to microscaled 4-bit floating point, and their product with a matrix that is stored so
"""
import math

import torch

own = False

MX_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # Serving one stream of a GPT-2 model: one row of its vocabulary, with five alternatives. Latency counts.
        dict(name="logprobs_gpt2_n1_top5", kind="logprobs", n=1, vocab=50257, bf16=True, top=5, temperature=1.0, pad=0, masked=0),
        # Perplexity of a prompt of 2048 tokens; the vocabulary is padded to a multiple of 64 with masked columns.
        dict(name="logprobs_eval_n2048_f32", kind="logprobs", n=2048, vocab=50304, bf16=False, top=0, temperature=1.0, pad=0, masked=47),
        # The teacher's pass over a batch of a distillation: 64 alternatives of every token, odd rows in a wider buffer.
        dict(name="logprobs_teacher_n4096_top64", kind="logprobs", n=4096, vocab=50257, bf16=True, top=64, temperature=2.0, pad=47, masked=0),
        # Validation of a short batch.
        dict(name="loss_n192_k32", kind="loss", n=192, vocab=50257, bf16=True, k=32, temperature=1.0, tail=True, pad=0),
        # Validation of a long one, logits in fp32, no tail.
        dict(name="loss_n2048_k64_f32", kind="loss", n=2048, vocab=50272, bf16=False, k=64, temperature=2.0, tail=False, pad=0),
        # The training step of 4 x 512 tokens: the tail of the teacher's distribution counts as one class.
        dict(name="grad_n2048_k64", kind="grad", n=2048, vocab=50257, bf16=True, k=64, temperature=2.0, tail=True, pad=47),
        # A ragged batch with a small odd vocabulary, logits in fp32.
        dict(name="grad_n333_k20_f32", kind="grad", n=333, vocab=32001, bf16=False, k=20, temperature=1.0, tail=False, pad=0),
        # The weights of an OPT-6.7B linear (FFN up), once per model.
        dict(name="mx_quant_opt_6.7b", kind="mx_quant", rows=16384, cols=4096, bf16=False),
        # The activations of a short ragged batch.
        dict(name="mx_quant_ragged", kind="mx_quant", rows=777, cols=1000, bf16=True),
        # One token through an OPT-6.7B linear (qkv): what counts is streaming 27 MB of weights.
        dict(name="mx_linear_opt_6.7b_n1", kind="mx_linear", n=1, d_in=4096, d_out=12288, bf16=True, bias=True),
        # A training-sized batch through a GPT-2-XL linear (FFN up), fp32 result.
        dict(name="mx_linear_gpt2_xl_n4096", kind="mx_linear", n=4096, d_in=1600, d_out=6400, bf16=False, bias=True),
        # A prompt of 2048 tokens through an OPT-13B linear (FFN up): the largest product.
        dict(name="mx_linear_opt_13b_n2048", kind="mx_linear", n=2048, d_in=5120, d_out=20480, bf16=True, bias=False),
    ]


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], spread evenly over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(-(-lo // step) * step, min(hi // step * step, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["logprobs", "loss", "grad", "mx_quant", "mx_linear", "mx_linear"])
    c = dict(kind=kind, bf16=rng.random() < 0.6)
    if kind in ("logprobs", "loss", "grad"):
        vocab = _log(rng, 1000, 131072, rng.choice([1, 1, 8, 64]))
        most = (4096 if kind == "logprobs" else 2048) * 50257 // (1 if c["bf16"] else 2)  # elements, so that bytes are at most the listed ones'
        c.update(vocab=vocab, n=_log(rng, 1, min(4096, most // vocab)), temperature=rng.choice([1.0, 1.0, 2.0, 0.7]),
                 pad=rng.choice([0, 0, -vocab % 64, 3]))
        if kind == "logprobs":
            c.update(top=rng.choice([0, 1, 5, 20, 64, rng.randint(1, 128)]), masked=rng.choice([0, 0, rng.randint(1, 99)]))
        else:
            c.update(k=rng.choice([1, 8, 20, 64, rng.randint(1, 128)]), tail=rng.random() < 0.5)
    elif kind == "mx_quant":
        cols = _log(rng, 512, 16384, rng.choice([1, 8, 32]))
        c.update(cols=cols, rows=_log(rng, 1, 16384 * 4096 // cols))
    else:
        d_in, d_out = _log(rng, 512, 6400 if not c["bf16"] else 16384, 8), _log(rng, 512, 16384)
        n = rng.choice([1, rng.randint(1, 16), _log(rng, 17, 4096), _log(rng, 128, 4096)])
        c.update(d_in=d_in, d_out=d_out, n=min(n, 2048 * 5120 * 20480 // (d_in * d_out)), bias=rng.random() < 0.5)
    return c


def _dtype(c):
    return torch.bfloat16 if c["bf16"] else torch.float32


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731
    if c["kind"] == "mx_quant":
        # rows of different size, and one weight in a thousand twenty times the others
        x = rand(c["rows"], c["cols"]) * 0.02 * torch.exp(rand(c["rows"], 1))
        far = torch.rand((c["rows"], c["cols"]), generator=gen, device="cuda") < 1e-3
        return dict(case=c, X=torch.where(far, 20.0 * x, x).to(_dtype(c)))
    if c["kind"] == "mx_linear":
        W = rand(c["d_out"], c["d_in"]) * 0.02
        codes, scales = _pack(*_mx(W))
        return dict(case=c, X=rand(c["n"], c["d_in"]).bfloat16(), codes=codes, scales=scales,
                    bias=rand(c["d_out"]) * 0.02 if c["bias"] else None)
    n, v = c["n"], c["vocab"]
    # what a trained model gives: most tokens far below the few that are likely
    logits = rand(n, v) * 2.0
    likely = torch.randint(v, (n, 8), generator=gen, device="cuda")
    logits.scatter_add_(1, likely, 8.0 + 3.0 * rand(n, 8))
    if c.get("masked"):
        logits[:, v - c["masked"]:] = -math.inf
        likely = likely.clamp_(max=v - c["masked"] - 1)
    buf = torch.zeros((n, v + c["pad"]), dtype=_dtype(c), device="cuda")
    x = buf[:, :v]
    x.copy_(logits)
    if c["kind"] == "logprobs":
        return dict(case=c, logits=x, targets=likely[:, 0].contiguous())
    k = min(c["k"], v)
    teacher = torch.log_softmax((logits + 0.5 * rand(n, v)) / c["temperature"], dim=1)
    logp, index = teacher.topk(k, dim=1)
    st = dict(case=c, logits=x, index=index.to(torch.int32), logp=logp.contiguous())
    if c["kind"] == "grad":
        # the mean over the tokens of a batch, one in eight of them padding
        kept = (torch.rand(n, generator=gen, device="cuda") >= 0.125).float()
        st["dloss"] = kept / kept.sum().clamp(min=1.0)
    return st


# ---------------------------------------------------------------- microscaled 4-bit values and their container

def _mx(x):
    """(signed multiples of the block's scale [rows][d], exponents of the scales [rows][blocks]) in 32 bits: the scale is the power
    of two two below the block's largest magnitude, values go to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6, ties to the even code."""
    rows, d = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -d % 32)).view(rows, -1, 32)
    top = v.abs().amax(dim=2)
    e = (torch.frexp(top)[1] - 3).clamp(min=-127)
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    a = torch.ldexp(v, -e.unsqueeze(2))
    size = a.abs()
    # steps of 1/2 below 2, of 1 below 4, of 2 from there on; a tie goes to the even multiple, which is the even code
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
    near = (torch.round(size / step) * step).clamp(max=6.0)
    return torch.copysign(near, a).reshape(rows, -1)[:, :d], e


def _pack(values, e):
    """The container: codes uint8 [rows][64 * ceil(d / 128)], two a byte, even column low; scales (exponent + 127) uint8
    [ceil(rows / 128)][ceil(d / 128)][32][4][4], that of row r and block b at [r / 128][b / 4][r % 32][r / 32 % 4][b % 4]."""
    rows, d = values.shape
    size = values.abs()
    code = torch.where(size < 2.0, size * 2.0, torch.where(size < 4.0, size + 2.0, size / 2.0 + 4.0)).to(torch.uint8)
    code = torch.nn.functional.pad(code | (torch.signbit(values).to(torch.uint8) << 3), (0, -d % 128))
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -e.shape[1] % 4, 0, -rows % 128))
    return codes.contiguous(), s.view(-1, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _unpack(codes, scales, rows, d):
    """The values of a container in 32 bits."""
    code = torch.stack((codes & 15, codes >> 4), dim=2).view(rows, -1)
    v = torch.tensor(MX_VALUES + tuple(-x for x in MX_VALUES), device=codes.device)[code.int()]
    s = scales.permute(0, 3, 2, 1, 4).reshape(-1, scales.shape[1] * 4)[:rows].int() - 127
    return torch.ldexp(v.view(rows, -1, 32), s.unsqueeze(2)).view(rows, -1)[:, :d]


# ---------------------------------------------------------------- the plain forms

def _logprobs(x, targets, top, temperature):
    n, v = x.shape
    z = x.float() / temperature
    z = z - z.amax(dim=1, keepdim=True)
    e = torch.exp(z)
    s = e.sum(dim=1)
    log_s = torch.log(s)
    logprob = z.gather(1, targets[:, None])[:, 0] - log_s
    entropy = log_s - torch.where(e > 0, e * z, 0.0).sum(dim=1) / s
    if not top:
        return logprob, entropy, z.new_empty((n, 0)), torch.empty((n, 0), dtype=torch.int32, device=x.device)
    # the order of the values, then the lower index: one key for both
    bits = (x.float() + 0.0).view(torch.int32)
    order = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    place = torch.arange(v, device=x.device)
    key = order.long() * (1 << 20) + ((1 << 20) - 1 - place)
    index = key.topk(min(top, v), dim=1)[1]
    best = z.gather(1, index) - log_s[:, None]
    index = torch.where(best == -math.inf, -1, index)
    more = top - index.shape[1]
    return (logprob, entropy, torch.nn.functional.pad(best, (0, more), value=-math.inf),
            torch.nn.functional.pad(index, (0, more), value=-1).to(torch.int32))


def _distill(x, index, logp, temperature, tail, dloss=None):
    """Loss of each row, and with dloss the gradient: sum p (log p - log q) over the teacher's tokens, whose p add up to one without
    a tail; with it also r (log r - log rho), where r and rho are what teacher and student give to all other tokens. Where the two
    are near one another these terms cancel, so each class gives p (log p - log q) - p + q, which is never negative, in 64 bits."""
    z = x.float() / temperature
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    s = e.sum(dim=1, keepdim=True)
    index = index.long()
    logp = logp.double()
    p = torch.exp(logp)
    if not tail:
        total = p.sum(dim=1, keepdim=True)
        p, logp = p / total, logp - torch.log(total)
    log_q = x.gather(1, index).double() / temperature - top - torch.log(s.double())
    mass = p.sum(dim=1, keepdim=True)
    rest = e.scatter(1, index, 0.0).sum(dim=1, keepdim=True)
    rho = (rest / s).double()
    r = torch.where(rest > 0, (1.0 - mass).clamp(min=0.0), 0.0) if tail else torch.zeros_like(mass)
    off = logp - log_q
    loss = torch.where(p > 0, p * (off + torch.expm1(-off)), torch.exp(log_q)).sum(dim=1)
    off = torch.log(r) - torch.log(rho)
    loss = loss + (torch.where(r > 0, r * (off + torch.expm1(-off)), rho) + (mass + r - 1.0))[:, 0]
    if dloss is None:
        return loss.float()
    mass, others = (mass + r).float(), torch.where(rest > 0, r / rho, 0.0).float()
    q = e / s
    grad = (q * (mass - others)).scatter(1, index, q.gather(1, index) * mass - p.float())
    return loss.float(), (grad * (dloss[:, None] / temperature)).to(x.dtype)


def run(state):
    c = state["case"]
    if own:
        import paper_2210_03858_b200 as bcq
        if c["kind"] == "logprobs":
            return bcq.token_logprobs(state["logits"], state["targets"], top_k=c["top"], temperature=c["temperature"])
        if c["kind"] == "loss":
            return bcq.distill_loss(state["logits"], state["index"], state["logp"], temperature=c["temperature"], tail=c["tail"])
        if c["kind"] == "grad":
            return bcq.distill_grad(state["logits"], state["index"], state["logp"], state["dloss"], temperature=c["temperature"],
                                    tail=c["tail"])
        if c["kind"] == "mx_quant":
            return bcq.mx_dequantize(bcq.mx_quantize(state["X"]), out_dtype=torch.bfloat16)
        W = bcq.MxMatrix(state["codes"], state["scales"], c["d_out"], c["d_in"])
        return bcq.mx_linear(bcq.mx_quantize(state["X"]), W, bias=state["bias"], out_dtype=_dtype(c))
    if c["kind"] == "logprobs":
        return _logprobs(state["logits"], state["targets"], c["top"], c["temperature"])
    if c["kind"] in ("loss", "grad"):
        return _distill(state["logits"], state["index"], state["logp"], c["temperature"], c["tail"], state.get("dloss"))
    if c["kind"] == "mx_quant":
        values, e = _mx(state["X"])
        d = c["cols"]
        return (values * torch.exp2(e.float()).repeat_interleave(32, dim=1)[:, :d]).bfloat16()
    values, e = _mx(state["X"])
    X = values * torch.exp2(e.float()).repeat_interleave(32, dim=1)[:, :c["d_in"]]
    Y = X @ _unpack(state["codes"], state["scales"], c["d_out"], c["d_in"]).t()
    if c["bias"]:
        Y = Y + state["bias"]
    return Y.to(_dtype(c))


def work(case):
    c = case
    e = 2 if c["bf16"] else 4
    if c["kind"] == "mx_quant":
        m = c["rows"] * c["cols"]
        return {"bytes": m * (e + 2), "flops": 3.0 * m}  # values come out in bf16
    if c["kind"] == "mx_linear":
        w = c["d_in"] * c["d_out"]
        return {"bytes": w * 17 / 32 + 2 * c["n"] * c["d_in"] + e * c["n"] * c["d_out"] + (4 * c["d_out"] if c["bias"] else 0),
                "flops": 2.0 * c["n"] * w}
    m = c["n"] * c["vocab"]
    if c["kind"] == "logprobs":
        # a difference, an exponential, two sums and a product an element
        return {"bytes": m * e + c["n"] * (8 + 8 + 8 * c["top"]), "flops": 5.0 * m}
    if c["kind"] == "loss":
        return {"bytes": m * e + c["n"] * (8 * c["k"] + 4), "flops": 3.0 * m}
    return {"bytes": 2 * m * e + c["n"] * (8 * c["k"] + 8), "flops": 5.0 * m}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_mx(x):
    """Values in 64 bits: each magnitude is compared with the points halfway between neighbours, which go to the even code."""
    rows, d = x.shape
    v = torch.zeros((rows, -(-d // 32) * 32), dtype=torch.float64, device=x.device)
    v[:, :d] = x.double()
    v = v.view(rows, -1, 32)
    top = v.abs().max(dim=2, keepdim=True)[0]
    e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
    e = torch.where(torch.exp2(e) > top, e - 1.0, torch.where(torch.exp2(e + 1.0) <= top, e + 1.0, e))
    scale = torch.exp2(torch.where(top > 0, (e - 2.0).clamp(min=-127.0), -127.0))
    a = v.abs() / scale
    code = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int()
            + (a > 5.0).int())
    near = torch.tensor(MX_VALUES, dtype=torch.float64, device=x.device)[code.long()] * scale
    return torch.where(v < 0, -near, near).reshape(rows, -1)[:, :d]


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["kind"] == "mx_quant":
        return _exact_mx(st["X"])
    if c["kind"] == "mx_linear":
        b = torch.arange(-(-c["d_in"] // 32), device="cuda")
        r = torch.arange(c["d_out"], device="cuda")[:, None]
        scale = torch.exp2(st["scales"][r // 128, b // 4, r % 32, r // 32 % 4, b % 4].double() - 127.0)
        k = torch.arange(c["d_in"], device="cuda")
        W = torch.empty((c["d_out"], c["d_in"]), dtype=torch.float64, device="cuda")
        table = torch.tensor(MX_VALUES, dtype=torch.float64, device="cuda")
        for lo in range(0, c["d_out"], 2048):
            code = (st["codes"][lo:lo + 2048, k // 2].long() >> (4 * (k % 2))) & 15
            W[lo:lo + 2048] = table[code & 7] * (1 - 2 * (code >> 3)) * scale[lo:lo + 2048, k // 32]
        Y = torch.mm(_exact_mx(st["X"]), W.t())
        return Y if st["bias"] is None else Y + st["bias"].double()
    x = st["logits"].double()
    T = c["temperature"]
    n = c["n"]
    rows = torch.arange(n, device="cuda")[:, None]
    lse = torch.logsumexp(x / T, dim=1)
    if c["kind"] == "logprobs":
        lp = x / T - lse[:, None]
        entropy = -(torch.exp(lp) * lp.clamp(min=-1e6)).sum(dim=1)
        best, index = torch.sort(x, dim=1, descending=True, stable=True)
        best, index = best[:, :c["top"]] / T - lse[:, None], index[:, :c["top"]]
        index = index.masked_fill(torch.isinf(best), -1).to(torch.int32)
        short = c["top"] - best.shape[1]
        if short > 0:
            best = torch.cat((best, best.new_full((n, short), -math.inf)), dim=1)
            index = torch.cat((index, index.new_full((n, short), -1)), dim=1)
        return lp[rows[:, 0], st["targets"]], entropy, best, index
    index, lp = st["index"].long(), st["logp"].double()
    q = torch.exp(x / T - lse[:, None])
    p = torch.exp(lp)
    if not c["tail"]:
        p = p / p.sum(dim=1, keepdim=True)
    log_q = x[rows, index] / T - lse[:, None]
    kl = (p * (torch.log(p.clamp(min=1e-300)) - log_q)).sum(dim=1)
    t = torch.zeros_like(q)
    t[rows, index] = p
    mass = p.sum(dim=1, keepdim=True)
    grad = q * mass - t
    if c["tail"]:
        outside = torch.ones_like(q, dtype=torch.bool)
        outside[rows, index] = False
        rho = (q * outside).sum(dim=1, keepdim=True)
        r = (1.0 - mass).clamp(min=0.0) * (rho > 0)
        safe = torch.where(rho > 0, rho, 1.0)
        kl = kl + (r * (torch.log(r.clamp(min=1e-300)) - torch.log(safe)))[:, 0]
        grad = q * (mass + r) - t - outside * q * (r / safe)
    if c["kind"] == "loss":
        return kl
    return kl, grad * (st["dloss"].double()[:, None] / T)
