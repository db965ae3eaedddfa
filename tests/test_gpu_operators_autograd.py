"""Matrix operators under autograd: what they are asked for they give, and what they cannot give they refuse (needs an MI355X).

Operands are small whole numbers, so that products, their sums and differences of either are exact in every type.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1802_02422_amd as ivf

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SIZES, R, C = [5, 0, 40, 3], 24, 17


def whole(seed, *shape, dtype=F32):
    return torch.randint(-2, 3, shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def offsets():
    return torch.tensor([0] + SIZES).cumsum(0).int().cuda()


def product(x, w, transposed):
    out, at = [], 0
    for i, n in enumerate(SIZES):
        out.append(x[at:at + n].double() @ (w[i] if transposed else w[i].t()).double())
        at += n
    return torch.cat(out + [torch.zeros(x.shape[0] - at, out[0].shape[1], dtype=torch.float64, device=x.device)])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("transposed", [False, True])
def test_grouped_product_has_gradients(dtype, transposed):
    print("case: product", dtype, transposed, flush=True)
    n = sum(SIZES) + 2                                         # two rows of no group
    x, w = whole(1, n, R if transposed else C, dtype=dtype).requires_grad_(), whole(2, 4, R, C, dtype=dtype).requires_grad_()
    c = whole(3, n, C if transposed else R)
    y = ivf.ivf_grouped_product(x, w, offsets(), transposed=transposed, out_dtype=F32)
    (y * c).sum().backward()
    u, v = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    (product(u, v, transposed) * c).sum().backward()
    assert x.grad.dtype == dtype and torch.equal(x.grad.double(), u.grad) and torch.equal(w.grad.double(), v.grad)
    # a sum: its gradient is expanded; only one operand asks
    x.grad = None
    ivf.ivf_grouped_product(x, w.detach(), offsets(), transposed=transposed).sum().backward()
    u.grad = None
    product(u, v.detach(), transposed).sum().backward()
    assert torch.equal(x.grad.double(), u.grad)


def test_grouped_product_twice():
    """Gradients of gradients go through the same operators."""
    print("case: twice", flush=True)
    n = sum(SIZES)
    x, w = whole(4, n, C).requires_grad_(), whole(5, 4, R, C).requires_grad_()
    u, v = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    results = []
    for f, a, b in ((lambda a, b: ivf.ivf_grouped_product(a, b, offsets()), x, w), (lambda a, b: product(a, b, False), u, v)):
        ga, gb = torch.autograd.grad(f(a, b).square().sum(), (a, b), create_graph=True)
        (ga.square().sum() + gb.sum()).backward()
        results.append((a.grad.double(), b.grad.double()))
    # sums of up to some 10^5 whole numbers, each step rounded to 2^-24 at most where it passes 2^24
    for got, want in zip(*results):
        assert (got - want).abs().max() <= 1e-5 * want.abs().max()


def test_grouped_gradient_has_gradients():
    print("case: gradient", flush=True)
    n = sum(SIZES)
    dy, x, c = whole(6, n, R).requires_grad_(), whole(7, n, C).requires_grad_(), whole(8, 4, R, C)
    (ivf.ivf_grouped_gradient(dy, x, offsets()) * c).sum().backward()
    a, b = dy.detach().double().requires_grad_(), x.detach().double().requires_grad_()
    at, total = 0, 0.0
    for i, s in enumerate(SIZES):
        total = total + ((a[at:at + s].t() @ b[at:at + s]) * c[i]).sum()
        at += s
    total.backward()
    assert torch.equal(dy.grad.double(), a.grad) and torch.equal(x.grad.double(), b.grad)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("transposed", [False, True])
def test_product_with_4_bit_rows_has_gradients(dtype, transposed):
    print("case: 4 bits", dtype, transposed, flush=True)
    b = ivf.ivf_mx4_quantise(whole(9, 30, 45))
    values = ivf.ivf_mx4_expand(b).double()
    a = whole(10, 6, 30 if transposed else 45, dtype=dtype).requires_grad_()
    c = whole(11, 6, 45 if transposed else 30)
    (ivf.ivf_mx4_rows_product(a, b, transposed=transposed, out_dtype=F32) * c).sum().backward()
    assert torch.equal(a.grad.double(), c.double() @ (values.t() if transposed else values))


def test_no_gradient_is_refused():
    print("case: refused", flush=True)
    x = torch.randn(6, 6, device="cuda", requires_grad=True)
    w = torch.randn(1, 6, 6, device="cuda")
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    b = ivf.ivf_mx4_quantise(x.detach())
    for f in (lambda: ivf.ivf_orthogonalise(x, [(1.5, -0.5, 0.0)]), lambda: ivf.ivf_mx4_quantise(x),
              lambda: ivf.ivf_grouped_product(x, w, off, out=torch.empty(6, 6, device="cuda")),
              lambda: ivf.ivf_grouped_gradient(x, x, off, out=torch.empty(1, 6, 6, device="cuda")),
              lambda: ivf.ivf_mx4_rows_product(x, b, out=torch.empty(6, 6, device="cuda"))):
        with pytest.raises(ivf.IvfError):
            f()
        with torch.no_grad():
            f()
    assert not ivf.ivf_orthogonalise(x.detach(), [(1.5, -0.5, 0.0)]).requires_grad


def test_rotations_are_learned_from_rows_that_ask_for_gradients():
    """By turns, not by descent: nothing of it is followed."""
    print("case: rotations", flush=True)
    from paper_1802_02422_amd import rotations
    x = torch.randn(60, 32, device="cuda", requires_grad=True)
    off = torch.tensor([0, 25, 60], dtype=torch.int32, device="cuda")
    R, errors = rotations.learn(x, off, rounds=2)
    same, _ = rotations.learn(x.detach(), off, rounds=2)
    assert torch.equal(R, same) and not R.requires_grad and not errors.requires_grad
    assert torch.equal(rotations.keep(x, R, off).codes, rotations.keep(x.detach(), R, off).codes)
