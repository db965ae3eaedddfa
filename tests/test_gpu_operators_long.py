"""Matrix operators past the 2^32 threads of a launch and past 2^31 elements: several launches, each with its own run of the work (needs an MI355X; up to 80 GB of its memory).

Values are small whole numbers or powers of two, whose sums every type holds, so results are compared exactly.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_1802_02422_amd as ivf

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("100 GB of free memory are needed")
    yield
    torch.cuda.empty_cache()


def whole(*shape, dtype=BF16, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-4, 5, shape, generator=g, device="cuda", dtype=torch.int8).to(dtype)


def test_grouped_operators_with_many_groups():
    G, R, C, n = (1 << 24) + 11, 2, 3, 4000
    print("case: groups", G, flush=True)
    g = torch.Generator().manual_seed(2)
    who = torch.cat([torch.randint(0, G, (n - 4,), generator=g), torch.tensor([0, G - 1, G - 1, (1 << 24) - 1])]).sort().values
    off = torch.zeros(G + 1, dtype=torch.int32)
    off[1:] = torch.bincount(who, minlength=G).cumsum(0)
    w, x, dy = whole(G, R, C), whole(n, C, seed=3), whole(n, R, seed=4)
    of = who.cuda()
    got = ivf.ivf_grouped_product(x, w, off.cuda())
    assert torch.equal(got.float(), (w[of].float() * x[:, None].float()).sum(2))
    got = ivf.ivf_grouped_product(dy, w, off.cuda(), transposed=True)
    assert torch.equal(got.float(), (w[of].float() * dy[:, :, None].float()).sum(1))
    dw = ivf.ivf_grouped_gradient(dy.float(), x.float(), off.cuda())
    ref = torch.zeros(G, R, C, device="cuda").index_add_(0, of, dy.float()[:, :, None] * x.float()[:, None])
    assert torch.equal(dw, ref)


def test_orthogonalise_many_matrices():
    batch = (1 << 26) + 9
    print("case: matrices", batch, flush=True)
    x = whole(batch, 2, 2, dtype=F32)
    x[:, 0, 0] += 9
    got = ivf.ivf_orthogonalise(x, [(1.5, -0.5, 0.0)] * 2)
    some = torch.cat([torch.arange(0, batch, 65537), torch.arange((1 << 26) - 5, batch)]).cuda()
    y = x[some].double()
    y = y / (y.flatten(1).norm(dim=1)[:, None, None] + 1e-7)
    for _ in range(2):
        y = 1.5 * y - 0.5 * y @ y.mT.contiguous() @ y
    assert (got[some] - y).abs().max() < 1e-5


def test_quantise_many_rows():
    n = (1 << 30) + 7                                          # four lanes a row
    print("case: quantise", n, flush=True)
    x = whole(n, 1)
    rows = ivf.ivf_mx4_quantise(x)
    some = torch.cat([torch.arange(0, n, 1 << 20), torch.arange((1 << 30) - 100, n)]).cuda()
    part = ivf.ivf_mx4_quantise(x[some])
    assert torch.equal(rows.codes[some], part.codes) and torch.equal(rows.scales[some], part.scales)
    assert torch.equal(ivf.ivf_mx4_expand(part), x[some].float())


def test_expand_many_rows():
    n = (1 << 29) + 5                                          # eight lanes a row
    print("case: expand", n, flush=True)
    codes = torch.empty(n, 16, dtype=torch.uint8, device="cuda").random_(0, 256, generator=torch.Generator(device="cuda").manual_seed(5))
    scales = torch.full((n, 1), 127, dtype=torch.uint8, device="cuda")
    out = ivf.ivf_mx4_expand(ivf.Mx4Rows(codes, scales, 32))
    some = torch.cat([torch.arange(0, n, 1 << 19), torch.arange((1 << 29) - 100, n)]).cuda()
    assert torch.equal(out[some], ivf.ivf_mx4_expand(ivf.Mx4Rows(codes[some], scales[some], 32)))


def test_products_with_many_rows_in_4_bits():
    n = (1 << 31) + 300                                        # 2^24 tiles of 128 rows and more
    print("case: products", n, flush=True)
    codes = torch.empty(n, 16, dtype=torch.uint8, device="cuda")
    codes.view(torch.int64).random_(generator=torch.Generator(device="cuda").manual_seed(6))
    scales = torch.full((n, 1), 126, dtype=torch.uint8, device="cuda")
    b = ivf.Mx4Rows(codes, scales, 32)
    some = torch.cat([torch.arange(0, n, 1 << 20), torch.arange((1 << 31) - 150, n)]).cuda()
    few = ivf.Mx4Rows(codes[some], scales[some], 32)
    a = whole(5, 32)
    got = ivf.ivf_mx4_rows_product(a, b)
    assert torch.equal(got[:, some], ivf.ivf_mx4_rows_product(a, few))
    del got
    a4 = ivf.ivf_mx4_quantise(a[:1])
    got = ivf.ivf_mx4_product(a4, b, out_dtype=BF16)
    assert torch.equal(got[:, some], ivf.ivf_mx4_product(a4, few, out_dtype=BF16))


def test_rows_of_no_whole_words_take_no_scratch():
    """bfloat16 rows at odd places against long 4-bit rows: no room for values that are not expanded for them."""
    print("case: scratch", flush=True)
    n, D = 65536, 1024
    b = ivf.ivf_mx4_quantise(whole(n, D))
    a = whole(256, D + 8, seed=3)
    out = torch.empty(256, n, dtype=F32, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    ivf.ivf_mx4_rows_product(a[:, 3:3 + D], b, out=out)
    assert torch.cuda.max_memory_allocated() == before
    assert torch.equal(out[:, :50], a[:, 3:3 + D].float() @ ivf.ivf_mx4_expand(b)[:50].t().contiguous())
