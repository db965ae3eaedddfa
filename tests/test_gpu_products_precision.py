"""Products in fp32 are as accurate as plain fp32 (needs an MI355X).

Six products of bfloat16 terms leave out 2^-21 of a product at most and 2^-24 on average, which is what rounding a product to fp32 takes; what else there is are the roundings of
the sums.  Plain fp32 rounds its sum for every product or two, these kernels once for 16 products (and a sum of a 128th the size five times): the errors' norm has to be below plain's.
Sums of up to 128 products, which are rounded six times for 16, may reach it.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1802_02422_amd as ivf


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("K", [128, 160, 1024, 4100])
@pytest.mark.parametrize("rows", [7, 100, 300])
def test_grouped_product_as_accurate_as_32_bits(rows, K, transposed):
    print("case:", rows, K, transposed, flush=True)
    g, G, cols = gen(K + rows), 12, 96
    x = torch.randn(G * rows, K, generator=g, device="cuda")
    w = torch.randn(*((G, K, cols) if transposed else (G, cols, K)), generator=g, device="cuda")
    off = torch.arange(G + 1, device="cuda", dtype=torch.int32) * rows
    got = ivf.ivf_grouped_product(x, w, off, transposed=transposed).view(G, rows, cols)
    a, b = x.view(G, rows, K), w if transposed else w.transpose(1, 2).contiguous()
    ref = torch.bmm(a.double(), b.double())
    err, plain = (got - ref).norm().item(), (torch.bmm(a, b) - ref).norm().item()
    print("error", err, "in fp32", plain, flush=True)
    assert err <= (1.0 if K > 128 else 1.1) * plain


@pytest.mark.parametrize("rows", [100, 1000, 5000])
def test_grouped_gradient_as_accurate_as_32_bits(rows):
    print("case:", rows, flush=True)
    g, G, R, C = gen(rows), 5, 96, 130
    x, dy = torch.randn(G * rows, C, generator=g, device="cuda"), torch.randn(G * rows, R, generator=g, device="cuda")
    off = torch.arange(G + 1, device="cuda", dtype=torch.int32) * rows
    got = ivf.ivf_grouped_gradient(dy, x, off)
    a, b = dy.view(G, rows, R).transpose(1, 2).contiguous(), x.view(G, rows, C)
    ref = torch.bmm(a.double(), b.double())
    err, plain = (got - ref).norm().item(), (torch.bmm(a, b) - ref).norm().item()
    print("error", err, "in fp32", plain, flush=True)
    assert err <= plain


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(400, 700), (513, 385), (129, 1030)])
def test_grouped_gradient_of_many_tiles(R, C, dtype):
    """Eight tiles of 128 x 128 and more, dealt to the XCDs by slices: ragged ends, long, short and empty groups, lines that are no whole words."""
    print("case: tiles", R, C, dtype, flush=True)
    sizes = [300, 0, 1, 1100, 77]
    n, g = sum(sizes), gen(R)
    dy, x = torch.randn(n, R + 1, generator=g, device="cuda").to(dtype)[:, 1:], torch.randn(n, C + 3, generator=g, device="cuda").to(dtype)[:, 2:-1]
    off = torch.tensor([0] + sizes).cumsum(0).int().cuda()
    got = ivf.ivf_grouped_gradient(dy, x, off, out_dtype=torch.float32)
    assert torch.equal(got, ivf.ivf_grouped_gradient(dy, x, off, out_dtype=torch.float32))
    at = 0
    for i, s in enumerate(sizes):
        a, b = dy[at:at + s].double(), x[at:at + s].double()
        ref, size = a.t().contiguous() @ b, a.abs().t().contiguous() @ b.abs()
        # a rounding of 2^-23 of the sum so far for 16 products, and of the pieces' sums; fp32 leaves 2^-21 of each product out as well
        tol = size * ((2.0 ** -20 if dtype == torch.float32 else 0.0) + 2 * (s / 16 + 8) * 2.0 ** -23) + 1e-37
        assert ((got[i].double() - ref).abs() <= tol).all()
        at += s
