"""Infinities and NaN in the operands of products: as in fp32 arithmetic, however many rows there are and whichever kernel takes them (needs an MI355X).

Where the products' sum in 64 bits is infinite or NaN the result has to be the same; others are those of the finite operands, whose accuracy is not asked here (2^-6 of the
sum of magnitudes, above every rounding of a result).
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1802_02422_amd as ivf

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
TYPES = [F32, F16, BF16]
INF, NAN = float("inf"), float("nan")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def simple(g, *shape):
    """Values of one significant bit and zeros, so that later terms are zero, next to values of many bits."""
    v = torch.randn(*shape, generator=g)
    few = torch.sign(v) * torch.exp2(torch.randint(-2, 3, shape, generator=g).float()) * (torch.rand(*shape, generator=g) > 0.05)
    return torch.where(torch.rand(*shape, generator=g) < 0.5, few, v)


def planted(g, v):
    """Infinities of both signs and a NaN, in rows and columns of their own and together."""
    n, k = v.shape
    for value in (INF, -INF, NAN, INF):
        v[int(torch.randint(n, (1,), generator=g)), int(torch.randint(k, (1,), generator=g))] = value
    return v


def same(got, a, b):
    """got against a b in 64 bits (elements one by one, so that no library's shortcut decides)."""
    ref = torch.stack([(row[:, None] * b).sum(0) for row in a.double()]) if len(a) else got.double().cpu()
    size = a.double().nan_to_num(0, 0, 0).abs() @ b.nan_to_num(0, 0, 0).abs()
    got = got.double().cpu()
    assert torch.equal(got.isnan(), ref.isnan())
    whole = ref.isinf()
    assert torch.equal(got[whole], ref[whole]) and not got[~whole].isinf().any()
    fine = ref.isfinite()
    assert ((got - ref).abs()[fine] <= 2.0 ** -6 * size[fine] + 1e-6).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("rows", [4, 5, 40, 100, 300])
def test_grouped_product(rows, transposed, dtype):
    print("case: grouped", rows, transposed, dtype, flush=True)
    for K, cols in ((96, 96), (40, 150), (260, 33)):
        g = gen(rows + K)
        x, w = simple(g, 3 * rows, K), simple(g, 3, K if transposed else cols, cols if transposed else K)
        planted(g, x[:rows])
        planted(g, w[1])
        x, w = x.to(dtype), w.to(dtype)
        off = torch.arange(4, dtype=torch.int32).cuda() * rows
        got = ivf.ivf_grouped_product(x.cuda(), w.cuda(), off, transposed=transposed, out_dtype=F32)
        for i in range(3):
            m = w[i].double()
            same(got[i * rows:(i + 1) * rows], x[i * rows:(i + 1) * rows], m if transposed else m.t())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [3, 40, 700])
def test_grouped_gradient(rows, dtype):
    """700 rows: groups in several pieces, whose sums are joined."""
    print("case: gradient", rows, dtype, flush=True)
    for R, C in ((96, 96), (20, 150)):
        g = gen(rows + R)
        dy, x = simple(g, 3 * rows, R), simple(g, 3 * rows, C)
        planted(g, dy[:rows])
        planted(g, x[rows:2 * rows])
        dy, x = dy.to(dtype), x.to(dtype)
        got = ivf.ivf_grouped_gradient(dy.cuda(), x.cuda(), torch.arange(4, dtype=torch.int32).cuda() * rows, out_dtype=F32)
        for i in range(3):
            same(got[i], dy[i * rows:(i + 1) * rows].t(), x[i * rows:(i + 1) * rows].double())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("size", [(4, 300, 96), (5, 300, 96), (4, 200, 520), (40, 200, 520), (300, 260, 520), (130, 131100, 64)])
def test_mx4_rows_product(size, transposed, dtype):
    m, n, D = size
    if n > 1000 and transposed:
        m = 5
    print("case: by 4 bits", size, transposed, dtype, flush=True)
    g = gen(m + n + D)
    b = ivf.ivf_mx4_quantise(simple(g, n, D).cuda())
    a = planted(g, simple(g, m, n if transposed else D)).to(dtype)
    values = ivf.ivf_mx4_expand(b).cpu().double()
    got = ivf.ivf_mx4_rows_product(a.cuda(), b, transposed=transposed, out_dtype=F32)
    some = ~a.isfinite().all(1)
    some[:3] = True
    if transposed:
        same(got.cpu()[some], a[some], values)
    else:
        same(got.cpu()[some][:, :400], a[some], values[:400].t())
