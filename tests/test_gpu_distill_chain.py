"""The operators as they are used together: a teacher whose linear is held in microscaled 4-bit floating point, its top log
probabilities, a student in binary codes, the distillation loss, the scales' and the activations' gradients, and the update.

Each stage is compared with its formula in 64 bits on what the stage before gave.  dlogits is rounded to bf16 once (within 2^-8 of
itself, counted at both of its users): a scale's gradient is a sum of dY x b over tokens and a group's columns, off by at most
(2^-8 + n 2^-23) of the sum of the magnitudes; dX multiplies dY with levels rounded to fp16 (2^-11), (2^-8 + 2^-11 + d_out 2^-23)."""
import pytest

import paper_2210_03858_b200 as bcq
from paper_2210_03858_b200 import build as bcq_build
from paper_2210_03858_b200.dist import AlphaBucket

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _built():
    bcq_build.build_library()
    yield
    bcq.check_device()


@pytest.mark.parametrize("n,d_in,vocab,q,g,T,tail", [(40, 256, 1003, 3, 64, 2.0, True), (130, 192, 4000, 2, 192, 1.0, False), (7, 512, 521, 4, 128, 1.0, True)])
def test_distillation_step(n, d_in, vocab, q, g, T, tail):
    gen = torch.Generator(device="cuda").manual_seed(n)
    W = torch.randn((vocab, d_in), generator=gen, device="cuda") * 0.1
    X = torch.randn((n, d_in), generator=gen, device="cuda").bfloat16()
    # the teacher, in the 4-bit format of the tensor core
    Wt = bcq.mx_quantize(W)
    teacher_logits = bcq.mx_linear(X, Wt)
    Xq = bcq.mx_dequantize(bcq.mx_quantize(X)).double()
    ref = Xq @ bcq.mx_dequantize(Wt).double().t()
    size = Xq.abs() @ bcq.mx_dequantize(Wt).double().abs().t()
    assert bool(((teacher_logits.double() - ref).abs() <= (d_in / 32 + 12) * 2.0 ** -23 * size).all())
    _, _, top, index = bcq.token_logprobs(teacher_logits, top_k=16, temperature=T)
    lp = torch.log_softmax(teacher_logits.double() / T, dim=1)
    assert float((lp.gather(1, index.long()) - top.double()).abs().max()) <= 2e-5  # (eps_s of the log probabilities' own test, and 4 |lp| 2^-24)
    assert bool((lp.gather(1, index.long())[:, -1:] >= lp.scatter(1, index.long(), -1e9).amax(dim=1, keepdim=True)).all())

    # the student
    bits, alpha, _ = bcq.quantize(W, q, g)
    G = bcq.num_groups(d_in, g)
    scales, grads = AlphaBucket([(q, vocab, G)], "cuda"), AlphaBucket([(q, vocab, G)], "cuda")
    scales[0].copy_(alpha)
    logits = bcq.linear_fwd(X, bits, scales[0], d_in, g, out_dtype=torch.bfloat16)
    w = torch.full((n,), 1.0 / n, device="cuda")
    w[-1] = 0.0  # padding
    loss, dY = bcq.distill_grad(logits, index, top, w, temperature=T, tail=tail)
    assert torch.isfinite(loss).all() and not dY[-1].any()

    # its gradients
    x = (logits.double() / T).requires_grad_()
    lq = torch.log_softmax(x, dim=1)
    p = torch.exp(top.double())
    if not tail:
        p = p / p.sum(dim=1, keepdim=True)
    L = (p * (torch.log(p) - lq.gather(1, index.long()))).sum(dim=1)
    if tail:
        r = (1 - p.sum(dim=1)).clamp(min=0)
        rho = torch.exp(lq).scatter(1, index.long(), 0.0).sum(dim=1)
        L = L + r * (torch.log(r) - torch.log(rho))
    (L * w.double()).sum().backward()
    assert float((loss.double() - L.detach()).abs().max()) <= 4e-5
    ref_dY = x.grad / T
    q_size = torch.softmax(x.detach(), dim=1).scatter_add(1, index.long(), p) * w.double()[:, None] / T
    assert bool(((dY.double() - ref_dY).abs() <= 2.0 ** -8 * ref_dY.abs() * 1.01 + 2e-5 * q_size + 2.0 ** -120).all())

    dalpha = bcq.linear_bwd_alpha(dY, X, bits, d_in, g, out=grads[0])
    dX = bcq.linear_bwd_x(dY, bits, scales[0], d_in, g)
    word = torch.arange(d_in, device="cuda")
    b = ((bits[:, :, word // 32].long() >> (word % 32)) & 1).double() * 2 - 1                    # [q][vocab][d_in]
    full, mass = dY.double().t() @ X.double(), dY.double().abs().t() @ X.double().abs()
    pad = G * g - d_in
    group = lambda t: torch.nn.functional.pad(t, (0, pad)).view(*t.shape[:-1], G, g).sum(dim=-1)  # noqa: E731
    tol = group(mass)[None] * ((n + g) * 2.0 ** -23)
    assert bool(((dalpha.double() - group(b * full)).abs() <= tol + 1e-30).all())
    W_hat = (b * alpha.double().repeat_interleave(g, dim=2)[:, :, :d_in]).sum(dim=0)
    size = (b.abs() * alpha.double().abs().repeat_interleave(g, dim=2)[:, :, :d_in]).sum(dim=0)
    off = (dX.double() - dY.double() @ W_hat).abs()
    assert bool((off <= (dY.double().abs() @ size) * (2.0 ** -10 + vocab * 2.0 ** -23) + 1e-30).all())

    # the update of the trained scales, and another pass with them
    m, v = torch.zeros_like(scales.flat), torch.zeros_like(scales.flat)
    seg = bcq.Segments(scales.plane_segments(1), "cuda", scales=[1.0 / g])
    bcq.alpha_adamw(scales.flat, grads.flat, m, v, 1, 1e-4, segments=seg)
    assert torch.equal(scales[0][1:], alpha[1:]) and not torch.equal(scales[0][0], alpha[0])
    again = bcq.distill_loss(bcq.linear_fwd(X, bits, scales[0], d_in, g, out_dtype=torch.bfloat16), index, top, temperature=T, tail=tail)
    assert torch.isfinite(again).all()


def test_a_captured_distillation_step_is_the_eager_one():
    gen = torch.Generator(device="cuda").manual_seed(5)
    n, d_in, vocab, q, g = 64, 256, 2003, 3, 64
    W = torch.randn((vocab, d_in), generator=gen, device="cuda") * 0.1
    X = torch.randn((n, d_in), generator=gen, device="cuda").bfloat16()
    Wt = bcq.mx_quantize(W)
    bits, alpha, _ = bcq.quantize(W, q, g)
    w = torch.full((n,), 1.0 / n, device="cuda")

    def step():
        _, _, top, index = bcq.token_logprobs(bcq.mx_linear(X, Wt, out_dtype=torch.bfloat16), top_k=8)
        loss, dY = bcq.distill_grad(bcq.linear_fwd(X, bits, alpha, d_in, g, out_dtype=torch.bfloat16), index, top, w)
        return loss, dY, bcq.linear_bwd_alpha(dY, X, bits, d_in, g), bcq.linear_bwd_x(dY, bits, alpha, d_in, g)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    X.copy_(torch.randn((n, d_in), generator=gen, device="cuda").bfloat16())
    expect = step()
    graph.replay()
    for a, b in zip(got, expect):
        assert torch.equal(a, b)
