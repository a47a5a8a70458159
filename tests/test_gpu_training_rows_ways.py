"""Products of rows of codes give a row the same bits whichever way the call is dealt out: dot products for one or two rows, whole tiles of one SM or
of a pair, clusters whose sums meet, shares that are joined.  The sums are exact, and the epilogue's roundings are the same everywhere."""
import pytest
import torch

pytestmark = pytest.mark.gpu
tr = pytest.importorskip("paper_2506_17974_b200.training")
ACTS = ["none", "relu", "gelu", "silu"]
ROWS = [1, 2, 3, 40, 130, 600, 1300]


def operands(rows, cin, cout, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    draw = lambda r: torch.randint(-127, 128, (r, cin), generator=g, device="cuda", dtype=torch.int8)                     # noqa: E731
    x, w = draw(rows), draw(cout)
    sx = torch.rand(rows, generator=g, device="cuda") * 2 + 0.1
    sw = (torch.rand(cout, generator=g, device="cuda") + 0.5) / (73 * 73 * cin ** 0.5)
    return x, sx, tr.Rows8(w, sw), torch.randn(cout, generator=g, device="cuda"), torch.randn(rows, cout, generator=g, device="cuda")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cin,cout", [(512, 4096), (4096, 640), (16384, 128), (131056, 130), (48, 1001)])
def test_a_row_does_not_depend_on_the_others(act, dtype, cin, cout):
    x, sx, w8, bias, res = operands(ROWS[-1], cin, cout, cin + cout)
    res = res.to(dtype)
    for b, r in ((None, None), (bias, None), (bias, res)):
        first, kept = None, None
        for n in reversed(ROWS):
            x8 = tr.Rows8(x[:n], sx[:n])
            y = tr.linear_rows8(x8, w8, b, act, None if r is None else r[:n], dtype).y
            both = tr.linear_rows8(x8, w8, b, act, None if r is None else r[:n], dtype, save_z8=True, save_y8=True)       # never by dot products
            if first is None:
                first, kept = y, both
            assert y.equal(first[:n]) and both.y.equal(first[:n]), (n, b is None, r is None)
            for a, k in ((both.z8, kept.z8), (both.y8, kept.y8)):
                assert a.codes.equal(k.codes[:n]) and a.exps.equal(k.exps[:n]), (n, b is None, r is None)
