"""Products by element (include/gp.h) through the C ABI against the fp64 oracle.

Tolerances.  A result is a sum of n products (n = k_in for Y, k_out for dX, the element's rows for dW).  In fp32 each product and each addition
is off by at most one last bit, 2^-23, of a number that is no larger than the sum of the |products| (a rounding is half of that; a
matrix instruction may cut instead): (n + 4) 2^-23 times that sum, the 4 for parts, residual and joining chunks.  fp64: 2^-52 in the place
of 2^-23.  A result of bfloat16 is rounded once more: 2^-8 of it.  Below the normal numbers a last bit has a fixed size, 2^-149 in fp32 and 2^-133 in
bfloat16 (2^-1074 in fp64), so a rounding there is off by that however small the number is: (n + 4) 2^-149 and, for a result of bfloat16, 2^-134 more.
"""
import numpy as np
import pytest

from oracle import products_by_element as op

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gp():
    import torch
    assert torch.cuda.is_available()
    from paper_2504_10700_amd import gp_binding
    return gp_binding


ROWS = {"f32": "float32", "f64": "float64", "bf16": "bfloat16"}
UNIT = {"f32": 2.0 ** -23, "f64": 2.0 ** -52, "bf16": 2.0 ** -23}
NAN = float("nan")


def dtypes(dtype):
    import torch
    rows = getattr(torch, ROWS[dtype])
    return rows, torch.float32 if dtype == "bf16" else rows


class Batch:
    """Tensors of one call.  gap: elements between an atom's block and the next; skew: elements the buffers begin after an aligned address."""

    def __init__(self, gp, n, elements, k_in, k_out, components=1, dtype="f32", gap=(0, 0), skew=0, padded=True, seed=5, z=None, ungrouped=False):
        import torch
        self.gp, self.n, self.elements, self.k_in, self.k_out, self.components, self.dtype = gp, n, elements, k_in, k_out, components, dtype
        self.rows, self.weights = dtypes(dtype)
        self.skew, self.gap = skew, gap
        self.ld_in, self.ld_out = components * k_in + gap[0], components * k_out + gap[1]
        kind = {"f32": gp.SC_F32, "f64": gp.SC_F64, "bf16": gp.SC_BF16}[dtype]
        self.cfg = gp.make_config(elements, k_in, k_out, components, kind, ld_in=self.ld_in if gap[0] else 0, ld_out=self.ld_out if gap[1] else 0)
        g = torch.Generator(device="cuda").manual_seed(seed)
        if z is None:
            z = torch.randint(0, max(1, elements - elements // 3), (n,), generator=g, device="cuda")   # a third of the elements is absent
            if padded:
                u = torch.rand(n, generator=g, device="cuda")
                z = torch.where(u < 0.05, -1 - z, torch.where(u > 0.95, elements + z, z))
        self.z = torch.as_tensor(z, device="cuda").int()
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
        self.X, self.residual, self.dY = (self.block(k, normal(n, components, k), out) for k, out in ((k_in, False), (k_out, True), (k_out, True)))
        self.W = self.skewed((elements, k_in, k_out), self.weights)
        self.W.copy_(normal(elements, k_in, k_out) * k_in ** -0.5)
        self.ws_bytes = gp.gp_workspace_bytes(self.cfg, n)
        self.ws = torch.full((self.ws_bytes,), 255, dtype=torch.uint8, device="cuda")
        nbytes = gp.gp_grouping_bytes(self.cfg, n)
        self.grouping = torch.full((max(nbytes, 1),), 255, dtype=torch.uint8, device="cuda") if n > gp.GP_UNGROUPED else None
        self.grouping_bytes = nbytes

    def skewed(self, shape, dtype, fill=NAN):
        import torch
        n = int(np.prod(shape))
        return torch.full((n + self.skew,), fill, dtype=dtype, device="cuda")[self.skew:].view(shape)

    def block(self, k, values=None, out=False):
        """[n][components][k] with the batch's gaps, NaN around (and in it without values)."""
        ld = self.ld_out if out or k != self.k_in else self.ld_in
        whole = self.skewed((self.n, ld), self.rows)
        view = whole[:, :self.components * k].unflatten(1, (self.components, k))
        if values is not None:
            view.copy_(values)
        view.whole = whole
        return view

    def group(self, stream=None):
        self.gp.gp_group(self.cfg, self.n, self.z, self.grouping, self.grouping_bytes, stream)

    def forward(self, Y, residual=None, X=None, stream=None):
        self.gp.gp_forward(self.cfg, self.n, self.z, self.grouping, self.X if X is None else X, self.W, residual, Y, self.ws, self.ws_bytes, stream)

    def backward(self, dX, dW, X=None, stream=None):
        self.gp.gp_backward(self.cfg, self.n, self.z, self.grouping, self.X if X is None else X, self.W, self.dY, dX, dW, self.ws, self.ws_bytes, stream)

    def all(self, residual=True):
        import torch
        self.group()
        Y, dX = self.block(self.k_out, out=True), self.block(self.k_in)
        dW = self.skewed(self.W.shape, self.weights)
        self.forward(Y, self.residual if residual else None)
        self.backward(dX, dW)
        torch.cuda.synchronize()
        return Y, dX, dW

    def check(self, Y, dX, dW, residual=True, X=None):
        f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
        z, X, W, dY, R = self.z.cpu().numpy(), f64(self.X if X is None else X), f64(self.W), f64(self.dY), f64(self.residual) if residual else None
        if self.n > 2000 or self.k_in * self.k_out * self.n > 5e7:
            z, X, W, dY = self.z, self.X.double(), self.W.double(), self.dY.double()
            wY, wdX, wdW = by_elements(z, X, W, dY)
            mY, mdX, mdW = by_elements(z, X.abs(), W.abs(), dY.abs())
            if residual:
                wY, mY = wY + self.residual.double(), mY + self.residual.double().abs()
            wY, wdX, wdW, mY, mdX, mdW = (f64(t) for t in (wY, wdX, wdW, mY, mdX, mdW))
            z = self.z.cpu().numpy()
        else:
            wY, (wdX, wdW) = op.forward(z, X, W, R), op.backward(z, X, W, dY)
            mY, (mdX, mdW) = op.forward(z, abs(X), abs(W), None if R is None else abs(R)), op.backward(z, abs(X), abs(W), abs(dY))
        u, last = UNIT[self.dtype], 2.0 ** -8 if self.dtype == "bf16" else 0.0
        counts = np.bincount(np.where((z >= 0) & (z < self.elements), z, self.elements), minlength=self.elements + 1)[:self.elements]
        terms = (counts * self.components)[:, None, None]
        for name, got, want, most, n, rounded in (("Y", Y, wY, mY, self.k_in, last), ("dX", dX, wdX, mdX, self.k_out, last), ("dW", dW, wdW, mdW, terms, 0.0)):
            if got is None:
                continue
            got = f64(got)
            off = np.abs(got - want)
            allowed = (n + 4) * (u * most + (0.0 if self.dtype == "f64" else 2.0 ** -149)) * (1 + rounded) + np.maximum(rounded * np.abs(want), 2.0 ** -134 if rounded else 0.0)
            assert np.isfinite(got).all(), name
            assert (off <= allowed).all(), (name, float((off / np.maximum(allowed, 1e-300)).max()))
        for t in (Y, dX):
            if t is not None and hasattr(t, "whole"):
                k = t.shape[1] * t.shape[2]
                assert t.whole[:, k:].isnan().all()      # between the blocks nothing is written


def by_elements(z, X, W, dY):
    """The oracle's results by plain fp64 products on the device, an element at a time (large batches)."""
    import torch
    Y = torch.zeros(X.shape[:2] + (W.shape[2],), dtype=torch.float64, device="cuda")
    dX, dW = torch.zeros(X.shape, dtype=torch.float64, device="cuda"), torch.zeros_like(W)
    for e in range(W.shape[0]):
        i = torch.nonzero(z == e)[:, 0]
        if i.numel():
            x, g = X[i], dY[i]
            Y[i], dX[i] = x @ W[e], g @ W[e].t().contiguous()
            dW[e] = x.flatten(0, 1).t().contiguous() @ g.flatten(0, 1)
    return Y, dX, dW


SIZES = [(1, 5, 8, 8, 1), (1, 3, 1, 1, 1), (7, 89, 128, 128, 1), (33, 4, 33, 65, 3), (64, 4, 33, 65, 3), (65, 4, 33, 65, 3), (61, 89, 128, 128, 1), (200, 1, 64, 64, 1),
         (200, 89, 40, 24, 5), (500, 1024, 16, 16, 1), (777, 10, 96, 41, 1), (1000, 6, 128, 64, 3), (2049, 12, 7, 130, 1), (300, 5, 257, 129, 7),
         (90, 3, 31, 1, 64), (150, 7, 512, 384, 1)]


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_oracle(gp, size, dtype):
    n, elements, k_in, k_out, components = size
    print(f"products {size} {dtype}", flush=True)
    b = Batch(gp, n, elements, k_in, k_out, components, dtype)
    b.check(*b.all())


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("n", [20, 300])
def test_strides_and_addresses(gp, n, dtype):
    """Blocks of wider rows, tensors that begin at any element."""
    for k_in, k_out, components, gap, skew in ((64, 128, 3, (13 * 64, 13 * 128), 0), (64, 128, 3, (5, 9), 1), (33, 17, 1, (1, 0), 3), (128, 64, 1, (0, 3), 1)):
        print(f"products strides {k_in} {k_out} {components} {gap} {skew} {dtype}", flush=True)
        b = Batch(gp, n, 5, k_in, k_out, components, dtype, gap=gap, skew=skew)
        b.check(*b.all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(20_000, 89, 128, 128, 1), (6_001, 3, 128, 128, 3), (4_000, 16, 1024, 512, 1), (70_001, 1, 64, 128, 1)],
                         ids=lambda s: "x".join(map(str, s)))
def test_large_batches(gp, size, dtype):
    n, elements, k_in, k_out, components = size
    print(f"products {size} {dtype}", flush=True)
    b = Batch(gp, n, elements, k_in, k_out, components, dtype)
    b.check(*b.all(residual=False), residual=False)


@pytest.mark.parametrize("n", [5, 100, 3000])
@pytest.mark.parametrize("which", ["one", "last", "none", "sorted", "bounds"])
def test_distributions(gp, n, which):
    import torch
    elements = 20
    z = {"one": torch.full((n,), 7), "last": torch.full((n,), elements - 1), "none": torch.full((n,), -1), "sorted": torch.arange(n) * elements // n,
         "bounds": torch.tensor([0, elements - 1, elements, -1, 2 ** 31 - 1, -2 ** 31]).repeat(n)[:n]}[which]
    b = Batch(gp, n, elements, 64, 48, 1, "f32", z=z)
    Y, dX, dW = b.all()
    b.check(Y, dX, dW)
    if which == "none":
        assert torch.equal(Y, b.residual) and not dX.any() and not dW.any()
    b.check(*b.all(residual=False), residual=False)


def test_the_grouping(gp):
    """Offsets and order are those of a stable sort, for every size of the sort."""
    import torch
    for n, elements in ((65, 1), (128, 1024), (1000, 89), (2048, 1023), (2049, 1024), (5000, 3), (40_000, 1024), (300_000, 89)):
        b = Batch(gp, n, elements, 1, 1)
        b.group()
        key = torch.where((b.z >= 0) & (b.z < elements), b.z, elements).long()
        words = b.grouping.view(torch.int32)
        room = -(-(elements + 2) // 64) * 64
        assert torch.equal(words[room:room + n].long(), torch.argsort(key, stable=True)), (n, elements)
        ends = torch.bincount(key, minlength=elements + 1).cumsum(0)
        assert words[0] == 0 and torch.equal(words[1:elements + 2].long(), ends), (n, elements)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
def test_one_result_alone_is_the_same(gp, dtype):
    import torch
    for n in (9, 400):
        b = Batch(gp, n, 6, 72, 40, 3, dtype)
        _, dX, dW = b.all()
        x, w = b.block(72), b.skewed(b.W.shape, b.weights)
        gp.gp_backward(b.cfg, n, b.z, b.grouping, None, b.W, b.dY, x, None, b.ws, b.ws_bytes)
        gp.gp_backward(b.cfg, n, b.z, b.grouping, b.X, None, b.dY, None, w, b.ws, b.ws_bytes)
        assert torch.equal(x, dX) and torch.equal(w, dW)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_results_repeat_and_the_residual_may_be_the_output(gp, dtype):
    import torch
    for n in (17, 3000):
        b = Batch(gp, n, 12, 128, 96, 1, dtype)
        first = b.all()
        for x, y in zip(first, b.all()):
            assert torch.equal(x, y)
        Y = b.residual.clone()
        b.forward(Y, Y)
        assert torch.equal(Y, first[0])


def test_one_grouping_serves_all_calls_on_a_batch(gp):
    """Another width, type and number of components on the same grouping."""
    n = 500
    a = Batch(gp, n, 30, 64, 64, 1, "f32")
    a.group()
    for components, dtype in ((3, "f32"), (1, "f64"), (5, "bf16")):
        b = Batch(gp, n, 30, 32, 80, components, dtype, z=a.z)
        b.grouping = a.grouping
        b.group = lambda stream=None: None
        b.check(*b.all())


def test_no_rows(gp):
    import torch
    for dtype in ("f32", "f64", "bf16"):
        b = Batch(gp, 0, 6, 72, 40, 3, dtype)
        dW = b.skewed(b.W.shape, b.weights)
        b.backward(None, dW)
        assert not dW.any()
        b.forward(None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [20, 600])
def test_extreme_values(gp, n, dtype):
    """Rows and weights over the whole range of the numbers, and ones that are not finite: only what they reach is not."""
    import torch
    b = Batch(gp, n, 4, 96, 64, 1, dtype, padded=False, z=torch.arange(n) % 3)
    scale = 10.0 ** torch.linspace(-37, 36, n, dtype=torch.float64, device="cuda")[:, None, None]
    b.X.copy_(b.X.double() * scale)
    b.dY.copy_(b.dY.double() * 1e-3)
    b.residual.zero_()
    Y, dX, dW = b.all()
    b.check(Y, dX, dW)
    b.W.mul_(1e-30)
    Y, dX, dW = b.all()
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    want, most = op.forward(b.z.cpu().numpy(), f64(b.X), f64(b.W)), op.forward(b.z.cpu().numpy(), abs(f64(b.X)), abs(f64(b.W)))
    tiny = 2.0 ** -149 * 100 if dtype == "f32" else 2.0 ** -133      # below the normal numbers: a last bit a term
    assert (np.abs(f64(Y) - want) <= 100 * 2.0 ** -23 * most + (2.0 ** -8 if dtype == "bf16" else 0) * abs(want) + tiny).all()
    b = Batch(gp, n, 4, 96, 64, 1, dtype, padded=False, z=torch.arange(n) % 3)
    Y, dX, dW = b.all(residual=False)
    b.X[4, 0, 5], b.X[10, 0, 90], b.X[11, 0, 0] = float("inf"), NAN, -3e38
    b.W[2, 7, 3] = float("inf")
    y, dx, dw = b.all(residual=False)
    bad = torch.zeros_like(Y, dtype=torch.bool)
    bad[4], bad[10] = True, True
    bad[b.z == 2, :, 3] = True
    assert not torch.isfinite(y[4]).any() and y[10].isnan().all() and not torch.isfinite(y[b.z == 2][:, :, 3]).any()
    rest = ~bad
    rest[11] = False
    off = (y.double() - Y.double()).abs()[rest]
    assert torch.isfinite(y[rest]).all() and (off <= 100 * 2.0 ** -23 * 100 + 2.0 ** -7 * Y.double().abs()[rest]).all()
    assert not torch.isfinite(dx[b.z == 2][:, :, 7]).any() and torch.isfinite(dx[b.z != 2]).all()
    assert not torch.isfinite(dw[1, 5]).any() and dw[1, 90].isnan().all() and torch.isfinite(dw[1, 6:90]).all() and torch.isfinite(dw[0]).all()


def test_second_order_by_the_same_calls(gp):
    import torch
    for n, dtype in ((11, "f64"), (400, "f64"), (400, "f32")):
        b = Batch(gp, n, 5, 48, 36, 3, dtype)
        HX = b.block(48, values=torch.randn(n, 3, 48, dtype=torch.float64, device="cuda"))
        ddY, W2 = b.block(36), b.skewed(b.W.shape, b.weights)
        b.group()
        b.forward(ddY, X=HX)
        b.backward(None, W2, X=HX)
        b.check(ddY, None, W2, residual=False, X=HX)


def test_gradients_against_differences(gp):
    """fp64: the loss is linear in each argument, so a difference over any distance is the gradient up to rounding."""
    import torch
    b = Batch(gp, 300, 6, 24, 20, 3, "f64")
    _, dX, dW = b.all()
    loss = lambda: (lambda Y: (b.forward(Y), (Y * b.dY).sum().item())[1])(b.block(20))  # noqa: E731
    g = torch.Generator().manual_seed(1)
    for value, grad in ((b.X, dX), (b.W, dW)):
        for _ in range(10):
            at = tuple(int(torch.randint(0, s, (), generator=g)) for s in value.shape)
            kept = value[at].item()
            value[at] = kept + 1
            up = loss()
            value[at] = kept - 1
            down = loss()
            value[at] = kept
            assert abs((up - down) / 2 - grad[at].item()) < 1e-9


def test_graphs_and_streams(gp):
    """Grouping, forward and backward captured together and replayed on other data; two graphs, each with its own workspace and grouping."""
    import torch
    made = []
    for n, components, dtype in ((800, 1, "f32"), (25, 3, "bf16")):
        b = Batch(gp, n, 9, 64, 96, components, dtype)
        out = (b.block(96), b.block(64), b.skewed(b.W.shape, b.weights))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        b.group(side)       # the first use of a kernel loads it
        b.forward(out[0], b.residual, stream=side)
        b.backward(out[1], out[2], stream=side)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            b.group()
            b.forward(out[0], b.residual)
            b.backward(out[1], out[2])
        made.append((b, out, graph))
    for turn in range(3):
        for b, out, graph in made:
            for t in out:
                t.fill_(NAN)
            b.z.copy_(torch.randint(-1, 10, (b.n,), device="cuda"))
            b.X.copy_(torch.randn(b.X.shape, device="cuda"))
        for b, out, graph in made:
            graph.replay()
        torch.cuda.synchronize()
        for b, out, graph in made:
            b.check(*out)
            for x, y in zip(out, b.all()):
                assert torch.equal(x, y)


def test_another_stream(gp):
    import torch
    b = Batch(gp, 700, 9, 64, 96, 1, "f32")
    want = b.all()
    side = torch.cuda.Stream()
    out = (b.block(96), b.block(64), b.skewed(b.W.shape, b.weights))
    torch.cuda.synchronize()
    b.group(side)
    b.forward(out[0], b.residual, stream=side)
    b.backward(out[1], out[2], stream=side)
    side.synchronize()
    for x, y in zip(out, want):
        assert torch.equal(x, y)


WIDTHS = [(2, 2), (3, 5), (8, 2), (2, 200), (31, 33), (65, 8), (129, 127), (192, 66), (1, 70), (70, 1)]


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("widths", WIDTHS, ids=lambda s: "x".join(map(str, s)))
def test_odd_widths(gp, widths, dtype):
    """Widths that end inside every kind of tile, dense and in wider rows that begin at any element, below and above the size that needs a grouping."""
    for n, components, gap, skew in ((9, 3, (0, 0), 0), (64, 1, (1, 3), 1), (130, 3, (0, 0), 0), (400, 1, (7, 1), 1)):
        print(f"products widths {widths} {dtype} {n} {components} {gap} {skew}", flush=True)
        b = Batch(gp, n, 3, *widths, components, dtype, gap=gap, skew=skew)
        b.check(*b.all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_calls_at_the_same_time(gp, dtype):
    """Two calls on two streams read the same grouping and weights; each has its own workspace."""
    import torch
    b = Batch(gp, 5000, 7, 96, 160, 1, dtype)
    want = b.all(residual=False)
    streams = [torch.cuda.Stream() for _ in range(2)]
    made = []
    torch.cuda.synchronize()
    for s in streams:
        ws = torch.full((b.ws_bytes,), 255, dtype=torch.uint8, device="cuda")
        made.append((ws, torch.full_like(want[0], NAN), torch.full_like(want[1], NAN), torch.full_like(want[2], NAN)))
    torch.cuda.synchronize()
    for turn in range(3):
        for s, (ws, Y, dX, dW) in zip(streams, made):
            gp.gp_forward(b.cfg, b.n, b.z, b.grouping, b.X, b.W, None, Y, ws, b.ws_bytes, s)
            gp.gp_backward(b.cfg, b.n, b.z, b.grouping, b.X, b.W, b.dY, dX, dW, ws, b.ws_bytes, s)
    torch.cuda.synchronize()
    for _, *got in made:
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_values_beyond_the_parts_in_the_gradients(gp):
    """Rows whose values differ by the whole range of the numbers meet in one dW; the gradients' rows too."""
    import torch
    for dtype in ("f32", "bf16"):
        for n in (40, 900):
            b = Batch(gp, n, 3, 72, 40, 2, dtype, padded=False, z=torch.arange(n) % 3)
            up = 10.0 ** torch.linspace(-36, 30, n, dtype=torch.float64, device="cuda")[:, None, None]
            b.X.copy_(b.X.double() * up)
            b.dY.copy_(b.dY.double() / up.clamp(1e-34, 1e34))
            b.W.mul_(1e-6)
            b.residual.zero_()
            print(f"products range {dtype} {n}", flush=True)
            b.check(*b.all())


@pytest.mark.parametrize("n", [64, 70])
def test_offsets_past_32_bits(gp, n):
    """Blocks as far apart as they may be: the last atom's begin beyond 2^31 elements (n = 64: 2^32 bytes)."""
    import torch
    k, elements, ld = 64, 3, gp.GP_MAX_STRIDE
    cfg = gp.make_config(elements, k, k, 1, gp.SC_BF16, ld_in=ld, ld_out=ld)
    g = torch.Generator(device="cuda").manual_seed(2)
    z = (torch.arange(n, device="cuda") % (elements + 1)).int()                  # the last of them is no element
    far = lambda: torch.empty((n - 1) * ld + k, dtype=torch.bfloat16, device="cuda").as_strided((n, k), (ld, 1))  # noqa: E731
    X, dY, Y, dX = far(), far(), far(), far()
    for t in (X, dY):
        t.copy_(torch.randn(n, k, generator=g, device="cuda"))
    W = torch.randn(elements, k, k, generator=g, device="cuda") / 8
    dW = torch.full_like(W, NAN)
    nbytes, ws_bytes = gp.gp_grouping_bytes(cfg, n), gp.gp_workspace_bytes(cfg, n)
    grouping = torch.empty(nbytes, dtype=torch.uint8, device="cuda") if nbytes else None
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
    gp.gp_group(cfg, n, z, grouping, nbytes)
    gp.gp_forward(cfg, n, z, grouping, X, W, None, Y, ws, ws_bytes)
    gp.gp_backward(cfg, n, z, grouping, X, W, dY, dX, dW, ws, ws_bytes)
    torch.cuda.synchronize()
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    zs, x, w, dy = z.cpu().numpy(), f64(X)[:, None], f64(W), f64(dY)[:, None]
    wY, (wdX, wdW) = op.forward(zs, x, w, None), op.backward(zs, x, w, dy)
    mY, (mdX, mdW) = op.forward(zs, abs(x), abs(w), None), op.backward(zs, abs(x), abs(w), abs(dy))
    for got, want, most, terms, last in ((Y, wY[:, 0], mY[:, 0], k, 2.0 ** -8), (dX, wdX[:, 0], mdX[:, 0], k, 2.0 ** -8), (dW, wdW, mdW, n, 0.0)):
        assert (abs(f64(got) - want) <= (terms + 4) * 2.0 ** -23 * most * (1 + last) + last * abs(want)).all()


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
def test_the_grouping_of_another_batch_stays_inside(gp, dtype):
    """A larger and a smaller batch's: rows may be missing or taken twice, but what lies around the call's tensors and its workspace stays as it was."""
    import torch
    b = Batch(gp, 500, 6, 64, 72, 2, dtype, gap=(3, 5))
    want = b.all()
    for n in (70, 400, 5000):
        other = Batch(gp, n, 6, 64, 72, 2, dtype, seed=n)
        other.group()
        edge = 4096
        ws = torch.full((b.ws_bytes + 2 * edge,), 77, dtype=torch.uint8, device="cuda")
        Y, dX, dW = b.block(72, out=True), b.block(64), b.skewed(b.W.shape, b.weights)
        print(f"grouping of {n} atoms {dtype}", flush=True)
        gp.gp_forward(b.cfg, b.n, b.z, other.grouping, b.X, b.W, None, Y, ws[edge:], b.ws_bytes)
        gp.gp_backward(b.cfg, b.n, b.z, other.grouping, b.X, b.W, b.dY, dX, dW, ws[edge:], b.ws_bytes)
        torch.cuda.synchronize()
        assert (ws[:edge] == 77).all() and (ws[edge + b.ws_bytes:] == 77).all()
        for t in (Y, dX):
            assert t.whole[:, t.shape[1] * t.shape[2]:].isnan().all()
    for x, y in zip(b.all(), want):
        assert torch.equal(x, y)
