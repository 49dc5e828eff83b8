"""Products by element over long reduced indices, and the second order of bfloat16 rows.

Tolerance.  An instruction adds 16 products of parts to a sum and is off by at most a last bit, 2^-23, of a number no larger than the sum of the |products|.  Rows of bfloat16: three instructions for every 16
indices in one sum, and the weights' parts stand for 2^-24 of them: (3 n / 16 + 4) 2^-23 times that sum, and 2^-8 of the result for its rounding.  Rows of fp32: twelve for every 32 indices in a sum of their
own, of which n / 32 are added, and six products of parts off by 2^-24 each: (n / 32 + 16) 2^-23.  fp64: four for every 16 in one sum, (n / 4 + 4) 2^-52, and as much for the sums it is compared with, which
are made as n of them."""
import pytest

from test_gpu_products_by_element import Batch, by_elements, gp  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("signs", ["one", "both"])
@pytest.mark.parametrize("n,k", [(100, 4096), (700, 16_384), (130, 65_536), (40, 65_536), (300, 20_001), (2, 65_535)])
def test_long_sums(gp, n, k, signs, dtype):  # noqa: F811
    """k_in long for Y, k_out long for dX; of one sign, what is cut off adds up."""
    import torch
    print(f"products long {n} {k} {signs} {dtype}", flush=True)
    for k_in, k_out in ((k, 24), (24, k)):
        b = Batch(gp, n, 2, k_in, k_out, 1, dtype)
        if signs == "one":
            for t in (b.X, b.W, b.dY):
                t.copy_(0.5 + torch.rand(t.shape, device="cuda", dtype=torch.float64))
        Y, dX, dW = b.all(residual=False)
        z, X, W, dY = b.z, b.X.double(), b.W.double(), b.dY.double()
        want, most = by_elements(z, X, W, dY), by_elements(z, X.abs(), W.abs(), dY.abs())
        for got, w, m, terms in ((Y, want[0], most[0], k_in), (dX, want[1], most[1], k_out)):
            u = {"f32": (terms / 32 + 16) * 2.0 ** -23, "bf16": (3 * terms / 16 + 4) * 2.0 ** -23, "f64": (1.25 * terms + 4) * 2.0 ** -52}[dtype]
            last = 2.0 ** -8 if dtype == "bf16" else 0.0
            off = (got.double() - w).abs()
            assert torch.isfinite(got).all() and (off <= u * m * (1 + last) + last * w.abs()).all(), float((off / (u * m + last * w.abs()).clamp_min(1e-300)).max())
        assert torch.isfinite(dW).all()


def test_second_order_of_bfloat16_rows(gp):  # noqa: F811
    import torch
    for n, components, widths in ((11, 3, (48, 36)), (64, 64, (128, 96)), (400, 3, (48, 36)), (3000, 1, (128, 128))):
        b = Batch(gp, n, 5, *widths, components, "bf16")
        HX = b.block(widths[0], values=torch.randn(n, components, widths[0], dtype=torch.float64, device="cuda"))
        ddY, W2 = b.block(widths[1], out=True), b.skewed(b.W.shape, b.weights)
        b.group()
        b.forward(ddY, X=HX)
        b.backward(None, W2, X=HX)
        torch.cuda.synchronize()
        b.X.copy_(HX)       # (for batches of this size the helper compares with the batch's own rows)
        b.check(ddY, None, W2, residual=False)
