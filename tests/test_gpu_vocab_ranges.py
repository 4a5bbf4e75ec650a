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
