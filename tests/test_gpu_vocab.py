"""Operators over rows of logits -- log probabilities with entropy and top alternatives, the distillation loss and its gradient --
against their formulas in 64 bits.

Tolerances.  A thread (of 128 at least) adds up at most vocab / 256 + 8 pairs of exponentials, each addition of positive terms within 2^-24 of the
result; the sums of threads, warps and CTAs are joined in at most 24 steps of three operations; an exponential is within 2^-22, its
argument (three roundings of a number up to |z|) within 3 |z| 2^-24.  So a row's sum S is within
    eps_s = (vocab / 256 + 8 + 72) 2^-24 + 2^-22 + 3 z 2^-24,  z <= 40: what lies lower adds less than 2^-40
of itself, a log probability within eps_s + 4 |lp| 2^-24, the entropy log S - sum(e z) / S within 4 eps_s (1 + H).  A gradient element
w / T (q P - p) is within (2 eps_s + 2^-20) |w| / T max(q P, p), plus half a step of its type.  The loss is computed in 64 bits from S
and the logits, where an error of S moves it by eps_s sum|p - q| <= 2 eps_s: near the minimum by less."""
import itertools
import math

import pytest

import paper_2210_03858_b200 as bcq
from paper_2210_03858_b200 import build as bcq_build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _built():
    bcq_build.build_library()
    yield
    bcq.check_device()


def eps_s(vocab):
    return (vocab / 256 + 80) * 2.0 ** -24 + 2.0 ** -22 + 120 * 2.0 ** -24


def make_logits(n, vocab, dtype, pad=0, offset=0, seed=0, scale=3.0):
    """[n][vocab] of which rows start `offset` elements into rows of vocab + pad; what lies between is NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((n, vocab + pad), float("nan"), dtype=dtype, device="cuda").view(-1)
    buf = torch.cat((torch.full((offset,), float("nan"), dtype=dtype, device="cuda"), buf))
    x = buf[offset:].view(n, vocab + pad)[:, :vocab]
    x.copy_(torch.randn((n, vocab), generator=g, device="cuda") * scale)
    return x


def ref_logprobs(x, targets, k, T):
    x = x.double()
    z = (x - x.amax(dim=1, keepdim=True)) / T  # (first: next to 3e38 the logarithm of a sum of nine equals is nothing)
    lp = z - torch.logsumexp(z, dim=1, keepdim=True)
    p = torch.exp(lp)
    entropy = -torch.where(p > 0, p * lp, 0.0).sum(dim=1)
    order = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
    top = lp.gather(1, order)
    index = torch.where(top == -INF, -1, order)
    more = k - top.shape[1]
    top = torch.nn.functional.pad(top, (0, more), value=-INF)
    index = torch.nn.functional.pad(index, (0, more), value=-1)
    given = None if targets is None else lp.gather(1, targets[:, None])[:, 0]
    return given, entropy, top, index.to(torch.int32)


def close(out, ref, tol):
    """|out - ref| <= tol where finite, infinities and NaN in the same places."""
    out, ref = out.double(), ref.double()
    ref = torch.where(ref.abs() > torch.finfo(torch.float32).max, ref * INF, ref)  # what overflows fp32
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(out), fine) and torch.equal(torch.isnan(out), torch.isnan(ref))
    assert torch.equal(out[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)])
    far = ((out - ref).abs() - tol)[fine] if torch.is_tensor(tol) and tol.dim() else ((out - ref).abs()[fine] - tol)
    assert not far.numel() or float(far.max()) <= 0, float(far.max())


def check_logprobs(x, targets, k, T=1.0):
    vocab = x.shape[1]
    got = bcq.token_logprobs(x, targets, top_k=k, temperature=T)
    ref = ref_logprobs(x, targets, k, T)
    e = eps_s(vocab)
    if targets is None:
        assert got[0] is None
    else:
        close(got[0], ref[0], e + 4 * ref[0].abs() * 2.0 ** -24)
    close(got[1], ref[1], 4 * e * (1 + ref[1]))
    assert torch.equal(got[3], ref[3])
    close(got[2], ref[2], e + 4 * ref[2].abs() * 2.0 ** -24)
    for a, b in zip(got, bcq.token_logprobs(x, targets, top_k=k, temperature=T)):
        assert a is None or torch.equal(a, b)


BF16, F32 = torch.bfloat16, torch.float32


# vocab, pad, offset (elements before the first row)
LAYOUTS = [(1, 0, 0), (2, 3, 1), (7, 0, 5), (8, 0, 0), (33, 0, 3), (1000, 0, 0), (2047, 2, 7), (8191, 0, 0), (32001, 0, 1),
           (50257, 47, 0), (50257, 0, 0), (131072, 0, 0)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab,pad,offset", LAYOUTS)
def test_logprobs_layouts(dtype, vocab, pad, offset):
    for n, k in ((1, 5), (3, 64), (40, 1), (700 if vocab < 60000 else 300, 20)):
        x = make_logits(n, vocab, dtype, pad, offset, seed=vocab + n)
        targets = torch.randint(vocab, (n,), generator=torch.Generator().manual_seed(n)).cuda()
        check_logprobs(x, targets, k)


@pytest.mark.parametrize("k", [0, 1, 2, 31, 127, 128])
@pytest.mark.parametrize("n,vocab", [(2, 100), (5, 3000), (200, 3000), (6, 50257), (500, 20001)])
def test_logprobs_list_lengths_and_temperatures(k, n, vocab):
    for dtype, T in ((BF16, 0.5), (F32, 3.0)):
        x = make_logits(n, vocab, dtype, seed=k)
        check_logprobs(x, None if k % 2 else torch.zeros(n, dtype=torch.int64, device="cuda"), k, T)


@pytest.mark.parametrize("n", [2, 400])
@pytest.mark.parametrize("vocab", [37, 5000, 50257])
def test_logprobs_ties_go_to_the_lowest_index(n, vocab):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    for dtype, k in itertools.product((BF16, F32), (1, 20, 128)):
        few = torch.randint(-2, 3, (n, vocab), generator=g, device="cuda").to(dtype)  # long runs of equals, zeros of both signs
        few[0] = 0.25                                                                 # nothing else
        few[1] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, -0.0, 0.0)
        few[-1, vocab // 2:] = -INF
        check_logprobs(few, None, k)
        check_logprobs(few * 1e-4, None, k)
        rising = torch.arange(vocab, device="cuda", dtype=torch.float32).repeat(n, 1)  # all but a few of the last batches are small
        check_logprobs((rising / vocab).to(dtype), None, k)
        check_logprobs((-rising / vocab).to(dtype), None, k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,vocab", [(6, 9), (12, 50257), (900, 2001)])
def test_logprobs_masked_rows(dtype, n, vocab):
    x = make_logits(n, vocab, dtype, seed=1)
    x[0] = -INF
    x[0, vocab // 2] = 3.0                   # one token: certain
    x[1, 3:] = -INF                          # fewer than the list asks for
    x[2] = torch.finfo(dtype).min            # equals, at the lowest value
    x[3, : vocab // 2] = torch.finfo(dtype).min
    x[4, 1:] = torch.finfo(dtype).min
    x[4, 0] = torch.finfo(dtype).max
    targets = torch.arange(n, device="cuda") % vocab
    targets[0], targets[1] = vocab // 2, 2
    check_logprobs(x, targets, 7)
    # rows that are no distribution; the others are as they were
    good = bcq.token_logprobs(x, targets, top_k=7)
    x[5] = -INF
    bad = [5]
    for i, v in ((n - 1, float("nan")), (2, INF)):
        x[i, (vocab * 3) // 4] = v
        bad.append(i)
    got = bcq.token_logprobs(x, targets, top_k=7)
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    fine[bad] = False
    for a, b in zip(got, good):
        assert torch.equal(a[fine], b[fine])
        if a.dtype == torch.int32:
            assert bool((a[~fine] == -1).all())
        else:
            assert bool(torch.isnan(a[~fine]).all())


def test_logprobs_targets_without_a_token_and_empty_batches():
    x = make_logits(4, 100, F32)
    t = torch.tensor([-100, -1, 99, 100], device="cuda")
    lp = bcq.token_logprobs(x, t)[0]
    assert lp[:2].tolist() == [0.0, 0.0] and torch.isfinite(lp[2]) and torch.isnan(lp[3])
    lp, h, top, index = bcq.token_logprobs(x[:0], t[:0], top_k=3)
    assert lp.shape == (0,) and h.shape == (0,) and top.shape == (0, 3) and index.shape == (0, 3)


# ---------------------------------------------------------------- distillation

def ref_distill(x, index, logp, T, tail):
    """(loss, d loss / d logits, size of the terms of the latter) in 64 bits, entry by entry as the definition has it."""
    x, index = x.double(), index.long()
    n, vocab = x.shape
    z = (x - x.amax(dim=1, keepdim=True)) / T
    lq = z - torch.logsumexp(z, dim=1, keepdim=True)
    q = torch.exp(lq)
    there = index >= 0
    p = torch.where(there, torch.exp(logp.double()), 0.0)
    if not tail:
        total = p.sum(dim=1, keepdim=True)
        p = torch.where(total > 0, p / total, 0.0)
    safe = index.clamp(min=0)
    loss = torch.where(p > 0, p * (torch.log(p) - lq.gather(1, safe)), 0.0).sum(dim=1)
    mass = p.sum(dim=1, keepdim=True)
    t = torch.zeros_like(q).scatter_add_(1, safe, p)
    named = torch.zeros_like(q).scatter_add_(1, safe, there.double()) > 0
    r = torch.zeros_like(mass)
    share = torch.zeros_like(q)
    if tail:
        lrho = torch.logsumexp(torch.where(named, -INF, lq), dim=1, keepdim=True)
        r = torch.where(lrho > -INF, (1.0 - mass).clamp(min=0.0), 0.0)
        loss = loss + torch.where(r > 0, r * (torch.log(r) - lrho), 0.0)[:, 0]
        share = torch.where(named | (lrho == -INF), 0.0, torch.exp(lq - lrho))
    P = mass + r
    return loss, (q * P - t - share * r) / T, (q * P + t + share * r) / T


def teacher_of(x, k, T, seed=0, noise=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    lp = torch.log_softmax((x.float() + noise * torch.randn(x.shape, generator=g, device="cuda")) / T, dim=1)
    top, index = lp.topk(min(k, x.shape[1]), dim=1)
    return index.to(torch.int32).contiguous(), top.contiguous()


def check_distill(x, index, logp, T, tail, w=None, out=None):
    n, vocab = x.shape
    w = torch.linspace(-1.0, 2.0, n, device="cuda") if w is None else w
    loss, grad, size = ref_distill(x, index, logp, T, tail)
    before = x.clone()
    e = eps_s(vocab)
    got = bcq.distill_loss(x, index, logp, T, tail)
    tol = 2 * e + 2.0 ** -22 * loss.abs().clamp(max=1e30)
    close(got, loss, tol)
    got2, d = bcq.distill_grad(x, index, logp, w, T, tail, out=out)
    close(got2, loss, tol)
    half = torch.finfo(x.dtype).eps / 2
    wd = w.double()[:, None]
    # elements below the smallest normal number of the type have its absolute step
    close(d, grad * wd, (2 * e + 2.0 ** -20) * size * wd.abs() + half * (grad * wd).abs() * 1.01 + 2.0 ** -125)
    assert d.shape == x.shape and d.dtype == x.dtype
    if out is None:
        assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(before))
        again = bcq.distill_grad(x, index, logp, w, T, tail)
        assert torch.equal(got2, again[0]) and torch.equal(d, again[1])
    return got, d


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab,pad,offset", LAYOUTS)
def test_distill_layouts(dtype, vocab, pad, offset):
    for n, k, T, tail in ((1, 5, 1.0, True), (3, 64, 2.0, False), (40, 1, 0.7, True), (320, 20, 1.0, False), (300, 33, 2.0, True)):
        x = make_logits(n, vocab, dtype, pad, offset, seed=vocab + n)
        check_distill(x, *teacher_of(x, k, T, n), T, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [262144, 393216])
def test_distill_largest_vocabularies(dtype, vocab):
    for n in (2, 150, 460):  # (the last: a CTA has a whole row, and an SM room for one CTA)
        x = make_logits(n, vocab, dtype, seed=n)
        check_distill(x, *teacher_of(x, 128, 1.0), 1.0, True)
    check_logprobs(x, None, 128)


@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_distill_lists_that_are_not_a_top(dtype, tail):
    vocab = 5003
    x = make_logits(9, vocab, dtype, pad=1, seed=3)
    index, logp = teacher_of(x, 40, 1.0)
    logp = logp.clone()
    index[0] = -1                                  # no entry
    index[1, 5:] = -1
    index[2] = index[2, 0]                         # one token, forty times
    index[3, 10:20] = index[3, 0:10]
    logp[4, 7] = -INF                              # an entry without mass
    index[5] = torch.arange(40, device="cuda", dtype=torch.int32)           # the first elements of the row
    index[6] = torch.arange(vocab - 40, vocab, device="cuda", dtype=torch.int32)
    logp[2] = math.log(1.0 / 64)
    x[7, ::2] = -INF
    x[7, index[7].long()] = 1.0
    x[8] = torch.finfo(dtype).min                  # equals
    x[4, index[4, 3].long()] = -INF                # a token of the teacher that the student excludes: an infinite loss
    check_distill(x, index, logp, 1.0, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_distill_tail_at_its_ends(dtype):
    # every token named: no tail
    x = make_logits(5, 30, dtype, seed=2)
    index, logp = teacher_of(x, 30, 1.0)
    check_distill(x, index, logp, 1.0, True)
    # all tokens that are not named are masked
    x = make_logits(5, 4000, dtype, seed=2)
    index, logp = teacher_of(x, 16, 1.0)
    y = torch.full_like(x, -INF).scatter(1, index.long(), x.gather(1, index.long()))
    check_distill(y, index, logp, 1.0, True)
    # what the student gives to the others is below the smallest float, and its logarithm is not
    y = x - 200.0
    y.scatter_(1, index.long(), 50.0)
    check_distill(y, index, logp, 1.0, True)
    # and the other way round
    y = x + 200.0
    y.scatter_(1, index.long(), -50.0)
    check_distill(y, index, logp, 1.0, True)
    # the teacher's mass is more than one by its rounding
    check_distill(x, index, torch.log_softmax(logp, dim=1) + 1e-6, 1.0, True)


@pytest.mark.parametrize("tail", [True, False])
def test_distill_near_the_teacher(tail):
    # p and q a rounding apart: the loss is a sum of squares of small differences, and stays one
    x = make_logits(64, 32000, F32, seed=8)
    index, logp = teacher_of(x, 64, 2.0, noise=1e-3)
    loss, _, _ = ref_distill(x, index, logp, 2.0, tail)
    got = bcq.distill_loss(x, index, logp, 2.0, tail)
    # off by S's error times |p - q| (below 2e-3 here), and by the rounding 2^-24 of the teacher's own 64 log probabilities
    ref_noise = 2.0 ** -23 * 20
    close(got, loss, eps_s(32000) * 4e-3 + ref_noise * 4e-3 + 1e-3 * loss.abs() if tail else 2 * eps_s(32000) + 1e-6)
    if tail:
        assert bool((got >= 0).all())


def test_distill_rows_without_a_result():
    x = make_logits(6, 3001, BF16, seed=4)
    index, logp = teacher_of(x, 8, 1.0)
    w = torch.ones(6, device="cuda")
    good = bcq.distill_loss(x, index, logp)
    good2, good_grad = bcq.distill_grad(x, index, logp, w)  # (its threads add up other elements: another order)
    x[1, 7] = float("nan")
    x[2, index[2, 3].long()] = INF
    x[3] = -INF
    index[4, 0] = 3001                      # no such token
    w[5] = 0.0
    for loss, before in ((bcq.distill_loss(x, index, logp), good), (bcq.distill_grad(x, index, logp, w)[0], good2)):
        assert torch.isnan(loss[1:5]).all() and torch.equal(loss[[0, 5]], before[[0, 5]])
    d = bcq.distill_grad(x, index, logp, w)[1]
    assert torch.isnan(d[1:5]).all() and torch.equal(d[0], good_grad[0]) and not d[5].any()
    # rows that count nothing have no gradient, whatever they hold
    assert not bcq.distill_grad(x, index, logp, torch.zeros(6, device="cuda"))[1].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_distill_in_place_and_into_a_wider_buffer(dtype):
    for n, vocab in ((3, 50257), (200, 4001)):
        x = make_logits(n, vocab, dtype, pad=5, seed=6)
        index, logp = teacher_of(x, 12, 1.0)
        w = torch.rand(n, device="cuda")
        loss, d = bcq.distill_grad(x, index, logp, w)
        assert d.stride(0) % 8 == 0 and d.data_ptr() % 16 == 0
        for shift in (0, 1, 3):
            buf = torch.full((n, vocab + 11), 7.0, dtype=dtype, device="cuda")
            out = buf[:, shift:shift + vocab]
            bcq.distill_grad(x, index, logp, w, out=out)
            assert torch.equal(out, d)
            assert bool((buf[:, :shift] == 7).all()) and bool((buf[:, shift + vocab:] == 7).all())
        loss2, same = bcq.distill_grad(x, index, logp, w, out=x)
        assert same is x and torch.equal(x, d) and torch.equal(loss, loss2)


def test_distill_gradient_is_that_of_the_loss():
    # central differences of the loss along the gradient and along single tokens
    n, vocab, k = 4, 300, 6
    x = make_logits(n, vocab, F32, seed=9, scale=1.0)
    for tail, T in ((True, 1.0), (False, 2.0)):
        index, logp = teacher_of(x, k, T, noise=1.0)
        _, d = bcq.distill_grad(x, index, logp, torch.ones(n, device="cuda"), T, tail)
        h = 2.0 ** -6
        for j in [0, 1, vocab - 1] + index[0, :3].tolist():
            step = torch.zeros_like(x)
            step[:, j] = h
            diff = (bcq.distill_loss(x + step, index, logp, T, tail).double() - bcq.distill_loss(x - step, index, logp, T, tail).double()) / (2 * h)
            # third derivatives of the loss are below 2 / T^3: h^2 / 6 of them; both losses within 2 eps_s
            assert float((diff - d[:, j].double()).abs().max()) <= h * h / 3 + 2 * eps_s(vocab) / h


def test_cross_entropy_is_a_list_of_one():
    x = make_logits(37, 50257, BF16, seed=12)
    label = torch.randint(50257, (37, 1), generator=torch.Generator().manual_seed(1)).cuda()
    loss, d = bcq.distill_grad(x, label.to(torch.int32), torch.zeros((37, 1), device="cuda"), torch.full((37,), 1 / 37, device="cuda"), tail=False)
    lp = bcq.token_logprobs(x, label[:, 0])[0]
    assert float((loss + lp).abs().max()) <= 4 * eps_s(50257) + 8 * 2.0 ** -24 * float(lp.abs().max())
    ref = torch.softmax(x.double(), dim=1)
    ref[torch.arange(37), label[:, 0]] -= 1
    assert float((d.double() - ref / 37).abs().max()) <= (2.0 ** -8 * 1.01 + 4 * eps_s(50257)) / 37


@pytest.mark.parametrize("call", ["logprobs", "loss", "grad"])
def test_operands_that_cannot_be_passed_on(call):
    x = make_logits(3, 50, F32)
    index, logp = teacher_of(x, 4, 1.0)
    w, t = torch.ones(3, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    f = {"logprobs": lambda x=x, t=t, k=2, **kw: bcq.token_logprobs(x, t, top_k=k, **kw),
         "loss": lambda x=x, index=index, logp=logp, **kw: bcq.distill_loss(x, index, logp, **kw),
         "grad": lambda x=x, index=index, logp=logp, w=w, **kw: bcq.distill_grad(x, index, logp, w, **kw)}[call]
    f()
    for bad in (x.half(), x.double(), "logits"):
        with pytest.raises(TypeError):
            f(x=bad)
    for bad in (x[0], x.t(), x[:, ::2], x.cpu()):
        with pytest.raises(ValueError):
            f(x=bad)
    for T in (0.0, float("nan"), 1e9):
        with pytest.raises(bcq.BcqError):
            f(temperature=T)
    with pytest.raises(bcq.BcqError):
        f(x=x[:1].expand(3, 50))            # rows on top of each other
    if call == "logprobs":
        for bad, error in ((t.int(), TypeError), (t[:2], ValueError), (t.cpu(), ValueError), (t.repeat(2)[::2], ValueError)):
            with pytest.raises(error):
                f(t=bad)
        for k in (-1, 129):
            with pytest.raises(bcq.BcqError):
                f(k=k)
    else:
        for bad, error in ((index.long(), TypeError), (index[:2], ValueError), (index[0], ValueError), (index.cpu(), ValueError), (index[:, :2], ValueError)):
            with pytest.raises(error):
                f(index=bad)
        for bad, error in ((logp.double(), TypeError), (logp[:, :3].contiguous(), ValueError)):
            with pytest.raises(error):
                f(logp=bad)
        with pytest.raises(bcq.BcqError):
            f(index=index[:, :0].contiguous(), logp=logp[:, :0].contiguous())
    if call == "grad":
        for bad, error in ((w[:2], ValueError), (w.double(), TypeError)):
            with pytest.raises(error):
                f(w=bad)
        for bad, error in ((torch.empty((3, 51), device="cuda"), ValueError), (torch.empty((3, 50), device="cuda", dtype=BF16), TypeError),
                           (torch.empty((50, 3), device="cuda").t(), ValueError)):
            with pytest.raises(error):
                f(out=bad)


# ---------------------------------------------------------------- streams and graphs

def test_vocab_operators_on_a_side_stream_and_in_a_graph():
    x = make_logits(24, 50257, BF16, seed=5)
    x2 = make_logits(24, 50257, BF16, seed=55)
    targets = torch.randint(50257, (24,), generator=torch.Generator().manual_seed(2)).cuda()
    w = torch.rand(24, device="cuda")

    def chain():
        lp, h, top, index = bcq.token_logprobs(x, targets, top_k=16)
        loss, d = bcq.distill_grad(x, index, top, w)
        return lp, h, top, index, loss, d, bcq.distill_loss(x, index, top)

    expect = [t.clone() for t in chain()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = chain()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(expect, got):
        assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = chain()
    keep = x.clone()
    for values in (x2, keep):
        x.copy_(values)
        expect = [t.clone() for t in chain()]
        for t in got:
            t.zero_()
        g.replay()
        g.replay()
        for a, b in zip(expect, got):
            assert torch.equal(a, b)
