"""What the operators over logits refuse, before anything is launched (no GPU is needed: the pointers are never followed)."""
import ctypes as C

import pytest

import paper_2210_03858_b200 as bcq
from paper_2210_03858_b200 import build as bcq_build

P, NULL = C.c_void_p(256), C.c_void_p(0)
ODD = C.c_void_p(257)


@pytest.fixture(scope="module", autouse=True)
def _built():
    bcq_build.build_library()


def logprobs(n=4, vocab=100, x=P, ld=100, dtype=1, targets=P, k=0, T=1.0, lp=P, h=P, top=NULL, index=NULL):
    return bcq.lib().bcq_token_logprobs(n, vocab, x, ld, dtype, targets, k, T, lp, h, top, index, None)


def loss(n=4, vocab=100, k=5, x=P, ld=100, dtype=1, index=P, lp=P, T=1.0, tail=1, out=P):
    return bcq.lib().bcq_distill_loss(n, vocab, k, x, ld, dtype, index, lp, T, tail, out, None)


def grad(n=4, vocab=100, k=5, x=P, ld=100, dtype=1, index=P, lp=P, T=1.0, tail=1, w=P, out=P, d=C.c_void_p(512), ldd=100):
    return bcq.lib().bcq_distill_grad(n, vocab, k, x, ld, dtype, index, lp, T, tail, w, out, d, ldd, None)


@pytest.mark.parametrize("call", [logprobs, loss, grad])
def test_rows(call):
    assert call(n=-1) == -2
    assert call(vocab=0) == -2
    assert call(ld=99) == -2
    assert call(vocab=393217, ld=400000) in (-4, -2)  # (the gradient's own pitch is checked too)
    assert call(dtype=2) == -4
    assert call(x=NULL) == -1
    assert call(x=ODD) == -3
    assert call(x=C.c_void_p(258), dtype=0) == -3
    for T in (0.0, -1.0, 1e-4, 1e4, float("nan"), float("inf")):
        assert call(T=T) == -2
    assert call(n=0, x=NULL) == 0


def test_logprobs():
    assert logprobs(k=-1) == -2
    assert logprobs(k=129, top=P, index=P) == -4
    assert logprobs(k=3, top=NULL, index=P) == -1
    assert logprobs(k=3, top=P, index=NULL) == -1
    assert logprobs(targets=NULL) == -1
    assert logprobs(lp=NULL) == -1


@pytest.mark.parametrize("call", [loss, grad])
def test_teacher(call):
    assert call(k=0) == -2
    assert call(k=129) == -4
    assert call(index=NULL) == -1
    assert call(lp=NULL) == -1


def test_results():
    assert loss(out=NULL) == -1
    assert grad(w=NULL) == -1
    assert grad(d=NULL) == -1
    assert grad(ldd=99) == -2
    assert grad(d=ODD) == -3
    assert grad(d=P, ldd=104) == -2  # in place, with another pitch


def test_tensors_on_the_host_are_refused():
    torch = pytest.importorskip("torch")
    x, i, f = torch.zeros(2, 10), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, 3)
    for call in (lambda: bcq.token_logprobs(x), lambda: bcq.distill_loss(x, i, f), lambda: bcq.distill_grad(x, i, f, torch.zeros(2))):
        with pytest.raises(ValueError):
            call()
