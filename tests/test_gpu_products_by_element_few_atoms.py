"""Products by element of batches without a grouping whose rows are many, or wide: those that the call groups itself.  Tolerances as in tests/test_gpu_products_by_element.py, whose helpers
are used."""
import numpy as np
import pytest

from test_gpu_products_by_element import NAN, Batch, gp  # noqa: F401

pytestmark = pytest.mark.gpu

# atoms, elements, k_in, k_out, components: on both sides of what the call decides by, for Y, dX and dW apart
SIZES = [(64, 1, 128, 128, 64), (64, 1, 33, 65, 64), (64, 1, 1, 70, 64), (64, 1, 2, 3, 64), (64, 8, 1024, 1024, 1), (33, 2, 1024, 640, 3), (64, 5, 257, 129, 7), (64, 1024, 96, 96, 64), (4, 1, 256, 256, 64),
         (15, 4, 1024, 520, 7), (1, 3, 512, 512, 64), (64, 89, 512, 512, 3), (64, 1, 700, 1, 7), (17, 2, 2048, 64, 1), (64, 1, 16, 2048, 7)]


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_oracle(gp, size, dtype):  # noqa: F811
    n, elements, k_in, k_out, components = size
    print(f"products few atoms {size} {dtype}", flush=True)
    b = Batch(gp, n, elements, k_in, k_out, components, dtype)
    b.check(*b.all())
    b.check(*b.all(residual=False), residual=False)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
def test_strides_and_addresses(gp, dtype):  # noqa: F811
    for k_in, k_out, components, gap, skew in ((128, 128, 64, (5, 9), 1), (96, 64, 64, (64, 0), 0), (33, 65, 64, (1, 3), 3), (1024, 512, 3, (0, 7), 1)):
        print(f"products few atoms strides {k_in} {k_out} {components} {gap} {skew} {dtype}", flush=True)
        b = Batch(gp, 64, 3, k_in, k_out, components, dtype, gap=gap, skew=skew)
        b.check(*b.all())


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
def test_they_take_the_tiles(gp, dtype):  # noqa: F811
    """64 atoms of 64 rows have the bits that they have in a batch of 65 whose last atom has no element, which comes with a grouping; alone or with the other result."""
    import torch
    for components, widths in ((64, (128, 128)), (64, (96, 200))):
        b = Batch(gp, 64, 3, *widths, components, dtype, padded=False)
        got = b.all()
        big = Batch(gp, 65, 3, *widths, components, dtype, padded=False, z=torch.cat([b.z, b.z.new_tensor([-1])]))
        big.W.copy_(b.W)
        for name in ("X", "dY", "residual"):
            getattr(big, name)[:64].copy_(getattr(b, name))
        want = big.all()
        for x, y in zip(got[:2], want[:2]):
            assert torch.equal(x, y[:64])
        x, w = b.block(widths[0]), b.skewed(b.W.shape, b.weights)
        gp.gp_backward(b.cfg, b.n, b.z, None, None, b.W, b.dY, x, None, b.ws, b.ws_bytes)
        gp.gp_backward(b.cfg, b.n, b.z, None, b.X, None, b.dY, None, w, b.ws, b.ws_bytes)
        assert torch.equal(x, got[1]) and torch.equal(w, got[2])
        assert torch.equal(b.all()[2], got[2])


@pytest.mark.parametrize("which", ["one", "none", "bounds"])
def test_distributions(gp, which):  # noqa: F811
    import torch
    n, elements = 64, 20
    z = {"one": torch.full((n,), 7), "none": torch.full((n,), -1), "bounds": torch.tensor([0, elements - 1, elements, -1, 2 ** 31 - 1, -2 ** 31]).repeat(n)[:n]}[which]
    for dtype in ("f32", "bf16", "f64"):
        b = Batch(gp, n, elements, 128, 100, 64, dtype, z=z)
        Y, dX, dW = b.all()
        b.check(Y, dX, dW)
        if which == "none":
            assert torch.equal(Y, b.residual) and not dX.any() and not dW.any()


def test_nothing_beyond_the_workspace(gp):  # noqa: F811
    import torch
    for size in ((64, 1, 128, 128, 64), (64, 1024, 40, 30, 64), (64, 2, 1024, 1024, 3)):
        n, elements, k_in, k_out, components = size
        for dtype in ("f32", "f64", "bf16"):
            b = Batch(gp, n, elements, k_in, k_out, components, dtype)
            edge = 4096
            whole = torch.full((b.ws_bytes + 2 * edge,), 77, dtype=torch.uint8, device="cuda")
            b.ws = whole[edge:edge + b.ws_bytes]
            b.check(*b.all())
            assert (whole[:edge] == 77).all() and (whole[edge + b.ws_bytes:] == 77).all()


def test_graphs(gp):  # noqa: F811
    """Captured and replayed on other atoms and rows, with the program's own work between."""
    import torch
    for n, elements, k_in, k_out, components, dtype in ((64, 6, 128, 96, 64, "f32"), (48, 3, 1024, 512, 3, "bf16")):
        b = Batch(gp, n, elements, k_in, k_out, components, dtype)
        out = (b.block(k_out, out=True), b.block(k_in), b.skewed(b.W.shape, b.weights))
        b.all()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.forward(out[0], b.residual)
            b.backward(out[1], out[2])
        for turn in range(3):
            for t in out:
                t.fill_(NAN)
            b.z.copy_(torch.randint(-1, elements + 1, (n,), device="cuda"))
            b.X.copy_(torch.randn(b.X.shape, device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            b.check(*out)
            for x, y in zip(out, b.all()):
                assert torch.equal(x, y)


def test_extreme_values(gp):  # noqa: F811
    """Values that the parts do not stand for, in rows that the tiles take."""
    import torch
    b = Batch(gp, 64, 3, 128, 64, 64, "f32", padded=False, z=torch.arange(64) % 3)
    scale = 10.0 ** torch.linspace(-36, 30, 64, dtype=torch.float64, device="cuda")[:, None, None]
    b.X.copy_(b.X.double() * scale)
    b.dY.copy_(b.dY.double() / scale.clamp(1e-34, 1e34))
    b.W.mul_(1e-6)
    b.residual.zero_()
    b.check(*b.all())
    b = Batch(gp, 64, 3, 128, 64, 64, "bf16", padded=False, z=torch.arange(64) % 3)
    y0, dx0, dw0 = b.all(residual=False)
    b.X[4, 3, 5] = float("inf")
    y, dx, dw = b.all(residual=False)
    assert not torch.isfinite(y[4, 3]).any() and torch.equal(dx, dx0) and not torch.isfinite(dw[1, 5]).any()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[4, 3] = False
    assert torch.isfinite(y[keep]).all() and torch.isfinite(dw[1, 6:]).all() and torch.isfinite(dw[0]).all()


def test_the_residual_may_be_the_output(gp):  # noqa: F811
    import torch
    for dtype in ("f32", "f64", "bf16"):
        b = Batch(gp, 64, 4, 128, 96, 64, dtype)
        first = b.all()
        Y = b.residual.clone()
        b.forward(Y, Y)
        assert torch.equal(Y, first[0])
