"""Orthogonalising steps where scales and sums decide: runs of steps that shrink a matrix, matrices far below eps, shapes of every tile
(needs an MI355X).

Tolerances.  A matrix in two fp16 terms is within 2^-22 of itself, and a product leaves as much out; its fp32 sums round by 2^-23 of the sum so far,
three times for 16 products, with random signs: for up to 512 products like sqrt(3 x 33) < 10 of them at once.  A product is thus within 8 x 2^-22 of the size of
what it is made of (for signs at random ||A|| ||Y||_F, A's largest singular value), and a step with its three products within 24 x 2^-22 of (|a| + |b| s^2 + |c| s^4) f, s
the largest singular value and f = ||X||_F.  Sums of more products count as their root.  An error that is there already is multiplied by the largest
derivative |a + 3 b t^2 + 5 c t^4| or quotient |a + b t^2 + c t^4| over singular values t up to s.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1802_02422_amd as ivf

F32 = torch.float32
POLAR, UPDATE = [(1.875, -1.25, 0.375)] * 12, [(3.4445, -4.775, 2.0315)] * 5
STEP = 24 * 2.0 ** -22


def gen(seed):
    return torch.Generator().manual_seed(seed)


def reference(x, coefs, eps):
    """(the result in 64 bits, the bound of the head for its error's norm) of every matrix."""
    y = x.double()
    y = y / (y.flatten(-2).norm(dim=-1)[..., None, None] + eps)
    tol = torch.zeros(y.shape[:-2], dtype=torch.float64, device=y.device)
    unit = STEP * max(1.0, math.sqrt(max(y.shape[-2:]) / 512))
    grid = torch.linspace(0, 1, 2001, dtype=torch.float64, device=y.device)
    for a, b, c in coefs:
        turned = y.shape[-2] > y.shape[-1]
        A = y.mT.contiguous() @ y if turned else y @ y.mT.contiguous()
        f, s = y.flatten(-2).norm(dim=-1), torch.linalg.eigvalsh(A)[..., -1].clamp(min=0).sqrt()
        t = (grid * s[..., None]) ** 2
        grow = torch.maximum((a + 3 * b * t + 5 * c * t * t).abs(), (a + b * t + c * t * t).abs()).amax(-1)
        tol = tol * grow + unit * (abs(a) + abs(b) * s ** 2 + abs(c) * s ** 4) * f
        F = b * A + c * (A @ A)
        y = a * y + (y @ F if turned else F @ y)
    return y, tol


def check(x, coefs, eps=1e-7, dtype=F32):
    x = x.to(dtype)
    ref, tol = reference(x, coefs, eps)
    got = ivf.ivf_orthogonalise(x.cuda(), coefs, eps=eps).to(x.device)
    size = ref.flatten(-2).norm(dim=-1)
    last = {F32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}[dtype]
    err = (got.double() - ref).flatten(-2).norm(dim=-1)
    print("relative error", (err / size).max().item(), "bound", (tol / size + last).max().item(), flush=True)
    assert got.dtype == dtype and got.isfinite().all()
    assert (err <= tol + last * size).all()


LONG = {"no_linear_growth": [(0.5, 0.0, 1e-3)] * 24, "tiny_last": [(0.5, 0.0, 1e-11)] * 18, "shrink_30": [(0.5, 0.5, 0.0)] * 30,
        "shrink_40": [(0.6, 0.4, 0.0)] * 40, "halves": [(0.5, 0.0, 0.0)] * 60, "down_then_up": [(0.5, 0.5, 0.0)] * 20 + [(2.0, 0.0, 0.0)] * 20,
        "only_last": [(0.0, 0.0, 1.0)] * 2, "sign": [(-0.7, 0.2, 0.1)] * 50, "more_than_an_argument": [(0.9, 0.05, 0.01)] * 300,
        "grow": [(1.5, 0.3, 0.2)] * 3}
SMALL = [(2, 40, 24), (3, 96, 96), (1, 1, 1), (2, 128, 70)]
LARGE = [(1, 60, 200), (2, 200, 140), (1, 257, 300)]


@pytest.mark.parametrize("coefs", LONG, ids=list(LONG))
@pytest.mark.parametrize("shape", SMALL)
def test_runs_of_steps_on_small_matrices(coefs, shape):
    """The values leave their bounds behind: what is computed keeps its accuracy relative to what is left."""
    print("case:", coefs, shape, flush=True)
    check(torch.randn(*shape, generator=gen(len(coefs))), LONG[coefs], eps=0.0)


@pytest.mark.parametrize("size,eps", [(1e-30, 1e-7), (1e-4, 1.0), (1e-12, 1e-7), (1e20, 1e3)])
def test_small_matrices_far_below_eps(size, eps):
    print("case: below eps", size, eps, flush=True)
    check(torch.randn(4, 50, 33, generator=gen(3)) * size, POLAR[:5], eps=eps)
    check(torch.randn(2, 20, 96, generator=gen(4)) * size, UPDATE, eps=eps)


def test_small_matrices_infinite_or_not_a_number():
    """Whatever the coefficients: all of the matrix, and no other."""
    print("case: infinite", flush=True)
    for coefs in (POLAR[:3], [(1.5, -0.5, 0.0)] * 2, [(2.0, 0.0, 0.0)], [(0.0, 0.0, 1.0)]):
        x = torch.randn(4, 30, 40, generator=gen(5))
        x[1, 3, 4], x[2, 29, 39] = float("inf"), float("nan")
        got = ivf.ivf_orthogonalise(x.cuda(), coefs).cpu()
        assert got[[1, 2]].isnan().all() and got[[0, 3]].isfinite().all()


def plain(x, coefs):
    y = x / (x.square().sum((1, 2), keepdim=True).sqrt() + 1e-7)
    for a, b, c in coefs:
        A = torch.bmm(y, y.transpose(1, 2).contiguous())
        y = a * y + torch.bmm(b * A + c * torch.bmm(A, A), y)
    return y


@pytest.mark.parametrize("shape", [(64, 96, 96), (64, 64, 128)])
@pytest.mark.parametrize("kind", ["diagonal", "noise", "rank3", "strong"])
def test_small_matrices_as_accurate_as_32_bits(kind, shape):
    """Against the same steps in fp32, whose sums of about a hundred products are off by some 2^-22 of their size; two terms (2^-22 at most, 2^-24.8 on average, of either
    operand and as much left out) add a few per cent to that, so a fifth more is never reached unless sums are rounded more often."""
    print("case: as 32 bits", kind, shape, flush=True)
    b, r, k = shape
    g = gen(17)
    noise, low = torch.randn(b, r, k, generator=g), torch.randn(b, r, 3, generator=g) @ torch.randn(b, 3, k, generator=g)
    d = torch.arange(min(r, k))
    coefs = UPDATE
    if kind == "diagonal":
        x, coefs = 0.2 * noise / k ** 0.5, POLAR[:10]
        x[:, d, d] += 0.3 + torch.rand(b, min(r, k), generator=g)
    elif kind == "noise":
        x = noise / k ** 0.5
    elif kind == "rank3":
        x = 1e-4 * noise + low / (r * k) ** 0.5
    else:
        x = noise / max(r, k) ** 0.5 + 4 * low / (r * k) ** 0.5
    ref = reference(x, coefs, 1e-7)[0]
    got, same = ivf.ivf_orthogonalise(x.cuda(), coefs).double().cpu() - ref, plain(x.cuda(), coefs).double().cpu() - ref
    print("error", got.norm().item(), "in fp32", same.norm().item(), flush=True)
    assert got.norm() <= 1.2 * same.norm()


@pytest.mark.parametrize("coefs", LONG, ids=list(LONG))
@pytest.mark.parametrize("shape", LARGE)
def test_runs_of_steps_on_large_matrices(coefs, shape):
    print("case:", coefs, shape, flush=True)
    check(torch.randn(*shape, generator=gen(len(coefs))), LONG[coefs], eps=0.0)


@pytest.mark.parametrize("size,eps", [(1e-30, 1e-7), (1e-4, 1.0), (1e-12, 1e-7), (1e20, 1e3)])
def test_large_matrices_far_below_eps(size, eps):
    print("case: below eps", size, eps, flush=True)
    check(torch.randn(2, 150, 233, generator=gen(3)) * size, POLAR[:5], eps=eps)
    check(torch.randn(1, 300, 136, generator=gen(4)) * size, UPDATE, eps=eps)


def test_large_matrices_infinite_or_not_a_number():
    print("case: infinite", flush=True)
    for coefs in (POLAR[:3], [(1.5, -0.5, 0.0)] * 2, [(2.0, 0.0, 0.0)], [(0.0, 0.0, 1.0)]):
        x = torch.randn(4, 130, 40, generator=gen(5))
        x[1, 3, 4], x[2, 129, 39] = float("inf"), float("nan")
        got = ivf.ivf_orthogonalise(x.cuda(), coefs).cpu()
        assert got[[1, 2]].isnan().all() and got[[0, 3]].isfinite().all()


# tiles of 64 and of 128 for both kinds of product, more than eight tiles on the shorter side for each, ends inside a tile and inside 32
TILES = [(1, 129, 129), (2, 150, 1000), (1, 700, 650), (70, 200, 300), (180, 200, 200), (2, 600, 3300), (12, 1100, 1060), (60, 140, 1030)]


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16])
@pytest.mark.parametrize("shape", TILES)
def test_large_matrices_of_every_tile(shape, dtype):
    print("case: tiles", shape, dtype, flush=True)
    b, r, k = shape
    x = torch.randn(b, r, k, generator=torch.Generator(device="cuda").manual_seed(sum(shape)), device="cuda") / math.sqrt(r * k)
    check(x, UPDATE[:3], dtype=dtype)
    out = ivf.ivf_orthogonalise(x, UPDATE[:3])
    assert torch.equal(out, ivf.ivf_orthogonalise(x, UPDATE[:3]))
    # rows and columns exchanged: the same steps on the other side
    turned = ivf.ivf_orthogonalise(x.transpose(1, 2).contiguous(), UPDATE[:3])
    assert (turned.transpose(1, 2) - out).flatten(1).norm(dim=1).max() <= 1e-4 * out.flatten(1).norm(dim=1).min()


def test_coefficients_from_a_generator():
    """Looked at once: a step that is no triple is refused wherever it stands, others give what a list gives."""
    print("case: generator", flush=True)
    x = torch.randn(2, 20, 30, generator=gen(6)).cuda()
    assert torch.equal(ivf.ivf_orthogonalise(x, (c for c in POLAR[:3])), ivf.ivf_orthogonalise(x, POLAR[:3]))
    with pytest.raises(ivf.IvfError):
        ivf.ivf_orthogonalise(x, (c for c in [(1.5, -0.5, 0.0), (1.5, -0.5)]))
    with pytest.raises(ivf.IvfError):
        ivf.ivf_orthogonalise(x, (c for c in [(1.5, -0.5, 0.0), (1.5, -0.5, 0.1, 0.2)]))
    with pytest.raises(ivf.IvfError):
        ivf.ivf_orthogonalise(x, POLAR, out="x")


@pytest.mark.parametrize("shape", [(2, 60, 40), (1, 150, 140), (2, 90, 300)])
def test_no_square_without_its_coefficient(shape):
    """A^2 would leave the range of 32 bits where the result, which has none of it, does not."""
    print("case: no square", shape, flush=True)
    check(torch.randn(*shape, generator=gen(8)), [(1e11, 0.0, 0.0), (1.0, 1e-10, 0.0)], eps=0.0)
