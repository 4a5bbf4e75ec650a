"""The operators over rows of logits where exponents and probabilities are at the ends of their range: finite masks of any size, large
logits, temperatures from 1/512 to 512, lists of a teacher down to probabilities that fp64 does not hold.

Tolerances are those derived in test_gpu_vocab.py, which hold for any size of the logits: a sum's base is the same number for all of its
terms.  One term more: a gradient element is w / T times a power of two that is 0 below 2^-126, twice at most, so it is off by up to
2^-125 |w| / T.  Temperatures are exact in fp32 (the reference takes them in fp64)."""
import math

import pytest

import paper_2210_03858_b200 as bcq
from paper_2210_03858_b200 import build as bcq_build
from test_gpu_vocab import check_logprobs, close, eps_s, make_logits, ref_distill, teacher_of

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
INF = math.inf
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    bcq_build.build_library()
    yield
    bcq.check_device()


def check_distill(x, index, logp, T, tail, w=None):
    n, vocab = x.shape
    w = torch.linspace(-1.0, 2.0, n, device="cuda") if w is None else w
    ref, grad, size = ref_distill(x, index, logp, T, tail)
    if tail:
        # the shares of the tokens outside the list in their sum, relative to its own largest (next to 1e20 the logarithm of a sum of many is nothing, in
        # 64 bits too)
        named = torch.zeros(x.shape, device="cuda").scatter_add_(1, index.long().clamp(min=0), (index >= 0).float()) > 0
        rest = torch.where(named, -INF, x.double())
        share = torch.nan_to_num(torch.softmax((rest - rest.amax(dim=1, keepdim=True)) / T, dim=1))
        lq = torch.log_softmax((x.double() - x.double().amax(dim=1, keepdim=True)) / T, dim=1)
        t = torch.zeros_like(lq).scatter_add_(1, index.long().clamp(min=0), torch.where(index >= 0, torch.exp(logp.double()), 0.0))
        mass = t.sum(dim=1, keepdim=True)
        r = torch.where(share.sum(dim=1, keepdim=True) > 0, (1.0 - mass).clamp(min=0.0), 0.0)
        grad, size = (torch.exp(lq) * (mass + r) - t - share * r) / T, (torch.exp(lq) * (mass + r) + t + share * r) / T
    e = eps_s(vocab)
    tol = 2 * e + 2.0 ** -22 * ref.abs().clamp(max=1e30)
    loss = bcq.distill_loss(x, index, logp, T, tail)
    close(loss, ref, tol)
    loss2, d = bcq.distill_grad(x, index, logp, w, T, tail)
    close(loss2, ref, tol)
    wd = w.double()[:, None]
    half = torch.finfo(x.dtype).eps / 2
    close(d, grad * wd, (2 * e + 2.0 ** -20) * size * wd.abs() + half * (grad * wd).abs() * 1.01 + 2.0 ** -125 * (wd.abs() / T).clamp(min=1.0))
    return loss, d


FINITE_MASKS = [-7.2e5, -1e9, -1e10, -1e12, -1e20]


def place(x, index, value, keep=()):
    """x with `value` in all columns but those of index and of keep."""
    cols = torch.cat([index.long()] + [torch.full_like(index[:, :1], j).long() for j in keep], dim=1)
    return torch.full_like(x, value).scatter(1, cols, x.gather(1, cols))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [0.296875, 0.5, 1.0, 2.0])
@pytest.mark.parametrize("mask", FINITE_MASKS)
def test_logprobs_finite_masks_of_any_size(dtype, T, mask):
    for n, vocab in ((3, 50257), (600, 5003)):
        x = make_logits(n, vocab, dtype, seed=3)
        _, index = x.float().topk(12, dim=1)
        targets = index[:, 5].contiguous()
        check_logprobs(place(x, index, mask), targets, 20, T)          # most columns: most threads see nothing else
        check_logprobs(place(x, index[:, 5:6], mask), targets, 0, T)
        check_logprobs(torch.full_like(x, mask), targets, 5, T)        # the whole row
        check_logprobs(torch.full_like(x, -mask), targets, 5, T)
        check_logprobs(place(x, index, -mask), targets, 5, T)
        check_logprobs((x.float() + mask).to(dtype), targets, 5, T)
        check_logprobs((x.float() - mask).to(dtype), targets, 5, T)


@pytest.mark.parametrize("T", [1.0, 1 / 512, 512.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_large_logits_on_both_sides_of_a_line(T, sign):
    # rows whose elements lie on both sides of |x| log2(e) / T = 2^k: threads whose maxima are on different sides meet
    for lg in (10, 16, 20, 24):
        at = sign * 2.0 ** lg * math.log(2.0) * T
        for n, vocab in ((2, 20001), (350, 3001)):
            x = (make_logits(n, vocab, F32, seed=lg) * T + at).contiguous()
            check_logprobs(x, torch.arange(n, device="cuda"), 10, T)
            index, logp = teacher_of(make_logits(n, vocab, F32, seed=lg), 10, 1.0)
            for tail in (True, False):
                check_distill(x, index, logp, T, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("lg", [9, 10, 11, 29, 30, 31, 32, 40])
def test_large_logits_some_steps_apart(dtype, sign, lg):
    # |x| log2(e) / T around 2^lg, elements a few steps of their type from one another, and a few much further down
    for n, vocab, T in ((2, 20001, 1.0), (350, 3001, 0.75), (5, 3001, 1 / 256)):
        at = sign * 2.0 ** lg * math.log(2.0) * T
        step = max(T, abs(at) * torch.finfo(dtype).eps)
        x = (make_logits(n, vocab, F32, seed=lg) * step + at).to(dtype)
        x[:, ::3] -= 30.0 * step
        check_logprobs(x, torch.arange(n, device="cuda"), 10, T)
        index, logp = teacher_of(make_logits(n, vocab, F32, seed=lg + 1), 10, 1.0)
        _, likely = x.float().topk(10, dim=1)
        for at_index in (index, likely.to(torch.int32)):
            for tail in (True, False):
                check_distill(x, at_index, logp, T, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
@pytest.mark.parametrize("mask", FINITE_MASKS)
def test_distill_finite_masks_of_any_size(dtype, tail, mask):
    for n, vocab, T in ((3, 50257, 1.0), (500, 5003, 0.296875), (40, 5003, 2.0)):
        x = make_logits(n, vocab, dtype, seed=4)
        index, logp = teacher_of(x, 16, T)
        for y in (place(x, index, mask), place(x, index, mask, keep=(0, vocab - 1)), place(x, index[:, :1], mask), torch.full_like(x, mask),
                  torch.full_like(x, -mask), (x.float() + mask).to(dtype), (x.float() - mask).to(dtype)):
            check_distill(y, index, logp, T, tail)
        # what the teacher leaves to all others is next to nothing
        sharp = torch.log_softmax(logp, dim=1) - 1e-7
        check_distill(place(x, index, mask), index, sharp, T, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
def test_distill_gradient_of_large_logits(dtype, tail):
    # |c m| from 2^5 to 2^24, of the whole row and of the tokens outside the list
    for n, vocab in ((2, 50257), (300, 3001)):
        x = make_logits(n, vocab, dtype, seed=11)
        index, logp = teacher_of(x, 16, 1.0)
        for size in (20.0, 300.0, 700.0, 1000.0, 3e4, 1e5, 1e6, 1e7):
            for y in ((x.float() + size).to(dtype), (x.float() - size).to(dtype), (x.float() - size).to(dtype).scatter(1, index.long(), x.gather(1, index.long()))):
                check_distill(y, index, logp, 1.0, tail)
                check_distill(y, index, torch.log_softmax(logp, dim=1) - 1e-6, 1.0, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1 / 512, 1 / 64, 512.0])
def test_temperatures_near_both_ends(dtype, T):
    for n, vocab in ((3, 50257), (400, 4001)):
        x = make_logits(n, vocab, dtype, pad=3, seed=13, scale=5.0)
        targets = torch.arange(n, device="cuda")
        check_logprobs(x, targets, 64, T)
        index, logp = teacher_of(x, 100, T)     # (log probabilities down to some -10000)
        for tail in (True, False):
            check_distill(x, index, logp, T, tail)
        # rows whose results are in another place than the logits': single elements and vectors
        buf = torch.empty((n, vocab + 9), dtype=dtype, device="cuda")
        w = torch.rand(n, device="cuda")
        _, d = bcq.distill_grad(x, index, logp, w, T)
        for shift in (0, 1, 2):
            assert torch.equal(bcq.distill_grad(x, index, logp, w, T, out=buf[:, shift:shift + vocab])[1], d)
        assert torch.equal(bcq.distill_grad(x, index, logp, w, T, out=x)[1], d)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tail", [True, False])
def test_loss_of_tokens_that_the_teacher_all_but_excludes(dtype, tail):
    # p = exp(lp) is a subnormal fp64 number from -708.4 on and 0 from -745.2 on; the student finds these tokens likely
    x = torch.zeros((2, 2), dtype=dtype, device="cuda")
    index = torch.tensor([[0, 1], [1, 0]], dtype=torch.int32, device="cuda")
    for lp in (-30.0, -700.0, -712.0, -720.0, -744.0, -745.0, -750.0, -1e5):
        logp = torch.tensor([[0.0, lp]] * 2, device="cuda")
        got, _ = check_distill(x, index, logp, 1.0, tail)
        assert float((got - math.log(2.0)).abs().max()) <= 2 * eps_s(2)
    x = make_logits(200, 1003, dtype, seed=21)
    index, logp = teacher_of(x, 8, 1.0)
    for values in ((-700.0, -715.0, -740.0, -750.0), (-20.0, -29.0, -31.0, -50.0), (-708.0, -709.0, -710.0, -744.5)):
        low = logp.clone()
        low[:, :4] = torch.tensor(values, device="cuda")    # the student's likeliest
        check_distill(x, index, low, 1.0, tail)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_probabilities_are_normalised_however_small_they_are(dtype):
    # without a tail a constant added to a list's log probabilities changes nothing; multiples of 2^-10, so that it is added exactly
    x = make_logits(60, 2003, dtype, seed=22)
    index, logp = teacher_of(x, 9, 1.0)
    logp = torch.round(logp * 1024.0) / 1024.0
    index[5, 1:] = -1
    logp[6, 3:] = -INF
    w = torch.linspace(-1.0, 2.0, 60, device="cuda")
    loss, d = check_distill(x, index, logp, 1.0, False, w)
    for shift in (-690.0, -705.0, -735.0, -800.0, -2000.0, 500.0, 1000.0):
        got, grad = bcq.distill_grad(x, index, logp + shift, w, 1.0, False)
        assert torch.equal(got, bcq.distill_grad(x, index, logp, w, 1.0, False)[0]) and torch.equal(grad, d), shift
        assert torch.equal(bcq.distill_loss(x, index, logp + shift, 1.0, False), loss), shift
    # a list that gives nothing to any of its tokens is none
    logp[:] = -INF
    loss, d = bcq.distill_grad(x, index, logp, w, 1.0, False)
    assert not loss.any() and not d.any()


def test_lists_that_are_refused_are_not_allocated():
    x = make_logits(64, 100, F32)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.max_memory_allocated()
    for k in (129, 10 ** 6, 2 ** 31 - 1):
        with pytest.raises(bcq.BcqError):
            bcq.token_logprobs(x, top_k=k)
    assert torch.cuda.max_memory_allocated() - before <= 4096
