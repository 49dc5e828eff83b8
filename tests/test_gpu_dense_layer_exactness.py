"""The dense layer (include/dl.h) where a wrong last bit shows: results far smaller than their terms, derivatives far below 1, overflow.

Tolerances stand with each test; u = 2^-24.
"""
import numpy as np
import pytest

import test_gpu_dense_layer as base
from oracle import dense_layer as od
from test_gpu_dense_layer import MANY, Layer, host, lib  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def signs(n):
    """1, -1, 1, -1, ... and the index of the pair."""
    i = np.arange(n)
    return 1.0 - 2.0 * (i % 2), i // 2


def sparse(rng, rows, k):
    """Rows of zeros but for up to four pairs of equal neighbours, +1 or -1 each."""
    x = np.zeros((rows, k))
    pairs = rng.random((rows, k // 2)).argsort(axis=1)[:, :4] if rows <= 4000 else rng.integers(0, k // 2, (rows, 4))
    sign = rng.choice([-1.0, 1.0], pairs.shape)
    for c in range(pairs.shape[1]):
        for odd in (0, 1):
            x[np.arange(rows), 2 * pairs[:, c] + odd] = sign[:, c]
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
@pytest.mark.parametrize("rows,k_in,k_out", [(40, 10, 14), (300, 64, 64), (MANY, 64, 64), (MANY, 32, 200), (20_011, 64, 1280), (8003, 128, 128), (600, 1000, 1024),
                                             (2100, 1024, 260), (6000, 264, 128)])
def test_every_bit_of_a_weight_counts(lib, rows, k_in, k_out, act, dtype):
    """W[k][n] = +-(2 + c 2^-12) + j 2^-19, neighbours of opposite sign: their equal partners in a row cancel all but the j.  At most eight terms below 4 in
    size, all multiples of 2^-19: exact in fp32 in any order, so a result in fp32 is exact and one in bfloat16 rounded once."""
    torch = lib.torch
    print(f"dense layer, bits of W, {rows} {k_in} {k_out} {act} {dtype}", flush=True)
    rng = np.random.default_rng(rows + k_in)
    (s_k, p_k), (s_n, p_n) = signs(k_in), signs(k_out)
    common = 2 + (2 * rng.integers(0, 1024, (k_in // 2 + 1, k_out // 2 + 1)) + 1) * 2.0 ** -12
    W = s_k[:, None] * s_n[None] * common[np.ix_(p_k, p_n)] + rng.integers(-31, 32, (k_in, k_out)) * 2.0 ** -19
    layer = Layer(lib, rows, k_in, k_out, act, dtype, bias=False, residual=False)
    layer.W.copy_(torch.tensor(W))
    for t, k in ((layer.X, k_in), (layer.HX, k_in), (layer.dY, k_out)):
        t.copy_(torch.tensor(sparse(rng, rows, k)))
    X, Wd, dY, HX = (t.double() for t in (layer.X, layer.W, layer.dY, layer.HX))
    assert torch.equal(layer.W.double().cpu(), torch.tensor(W))

    def same(name, got, ref):
        wrong = int((got != ref.to(got.dtype)).sum())
        assert wrong == 0, f"{name}: {wrong} of {got.numel()} elements differ"

    Y, Z = layer.forward()
    z = torch.matmul(X, Wd)
    assert 0 < z.abs().max() < 2.0 ** -10
    same("Z", Z, z)
    same("Y", Y, z.clamp(min=0) if act == "relu" else z)
    gate = layer.wide(1, torch.where(torch.rand(rows, 1, device="cuda") < 0.9, 1.0, -1.0).expand(rows, k_out))
    on = (gate.double() > 0).double() if act == "relu" else torch.ones_like(z)
    given = gate if act == "relu" else None
    same("dX", layer.backward(given, "X")[0], torch.matmul(dY * on, Wd.t().contiguous()))
    same("dX beside dW", layer.backward(given)[0], torch.matmul(dY * on, Wd.t().contiguous()))
    same("ddY", layer.double_backward(given)[0], torch.matmul(HX, Wd) * on)


def near_pairs(order, act, count):
    """Pairs of pre-activations (bfloat16 numbers) whose derivatives of that order agree to 2^-14 while the first 16 bits of the derivatives differ most from them."""
    import torch
    bf16 = lambda x: torch.tensor(x, dtype=torch.float32).bfloat16().double().numpy()  # noqa: E731
    z = np.unique(bf16(np.linspace(-4, 4, 200_001)))
    z = z[np.abs(z) >= 2.0 ** -6]
    d = od.activation(act, z)[order]
    whole = d.astype(np.float32).astype(np.float64)
    rest = whole - bf16(whole)
    rest -= bf16(rest)
    i = np.argsort(d)
    gap = np.abs(rest[i[1:]] - rest[i[:-1]]) * (np.abs(d[i[1:]] - d[i[:-1]]) <= 2.0 ** -14)
    best = np.argsort(gap)[::-1][:count]
    assert gap[best].min() > 40 * 2.0 ** -24
    return z[i[best]], z[i[best + 1]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,k_in", [(48, 8), (MANY, 64), (MANY, 132), (20_003, 260)])
def test_every_bit_of_a_derivative_counts(lib, rows, k_in, act, dtype):
    """dX = w (act'(z) - act'(z~)) and X2 = w (act''(z) - act''(z~)) for pairs that nearly cancel.  Each derivative in fp32 is within 4 u (act') and 8 u (act'') of its
    value for |z| <= 4 (u of the exponential, the reciprocal and six to ten operations on values below 1): 8 u and 16 u of the pair, and the result's last rounding."""
    torch, u = lib.torch, 2.0 ** -24
    print(f"dense layer, bits of derivatives, {rows} {k_in} {act} {dtype}", flush=True)
    pairs = 16
    layer = Layer(lib, rows, k_in, 2 * pairs, act, dtype, bias=False, residual=False)
    w = torch.tensor([1.0, -2.0, 0.5, 4.0], device="cuda").repeat(k_in // 4)
    layer.W.copy_(w[:, None] * torch.tensor(signs(2 * pairs)[0], device="cuda")[None])
    mine = torch.arange(rows, device="cuda") % pairs
    own_pair = (torch.arange(2 * pairs, device="cuda") // 2)[None] == mine[:, None]
    layer.HX.zero_()
    layer.HX[:, 0] = 1.0                                    # V = W[0] = +-1
    for order, bound in ((1, 8 * u), (2, 16 * u)):
        a, b = near_pairs(order, act, pairs)
        Z = layer.wide(1, torch.tensor(np.stack([a, b], 1).reshape(-1), device="cuda")[None].expand(rows, 2 * pairs))
        if order == 1:
            layer.dY.copy_(own_pair.double())
            got = (layer.backward(Z, "X")[0], layer.backward(Z)[0])
        else:
            layer.dY.copy_(own_pair.double() * torch.tensor(signs(2 * pairs)[0], device="cuda")[None])
            got = (layer.double_backward(Z, "X")[1], layer.double_backward(Z)[1])
        d = od.activation(act, host(Z)[0])[order]
        want = torch.tensor(d[0::2] - d[1::2], device="cuda")[mine][:, None] * w.double()
        slack = bound * w.abs().double() + 2.0 ** -8 * want.abs()
        for g in got:
            assert ((g.double() - want).abs() <= slack).all(), f"order {order}: {(((g.double() - want).abs() - slack) / w.abs()).max().item() / u:.1f} u beyond"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("column", [4, 5, 6, 7])
@pytest.mark.parametrize("rows,k_in,k_out", [(MANY, 64, 64), (MANY, 32, 128), (MANY, 64, 260), (MANY, 100, 100), (50, 64, 64)])
def test_a_product_beyond_the_largest_number_is_infinite(lib, rows, k_in, k_out, column, dtype):
    """1.5 2^127 times 2^17 (1 - 2^-10), which is 2^17 in eight bits and -2^7 beside it: infinity, not the difference of two infinities; everything else of the row
    is an exact product."""
    torch = lib.torch
    print(f"dense layer, overflow in column {column}, {rows} {k_in} {k_out} {dtype}", flush=True)
    layer = Layer(lib, rows, k_in, k_out, "none", dtype, bias=False, residual=False)
    large, factor, row = 1.5 * 2.0 ** 127, 2.0 ** 17 * (1 - 2.0 ** -10), rows // 2
    layer.W.fill_(0.5)
    layer.W[column, column] = factor
    layer.X[row] = 0
    layer.X[row, column] = large
    layer.dY[row] = 0
    layer.dY[row, column] = -large
    Y, _ = layer.forward()
    for got, k, value in ((Y, k_out, large), (layer.backward(None, "X")[0], k_in, -large)):
        want = torch.full((k,), 0.5 * value, dtype=torch.float64, device="cuda")
        want[column] = float("inf") if value > 0 else -float("inf")
        assert torch.equal(got[row].double(), want)
        assert torch.isfinite(got[:row]).all() and torch.isfinite(got[row + 1:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1.0, 1e15])
@pytest.mark.parametrize("z", [-40.0, -48.0, -60.0, -74.0, -80.0])
@pytest.mark.parametrize("rows,k_in,k_out", [(20, 64, 64), (MANY, 64, 64), (MANY, 132, 72), (3000, 512, 256)])
def test_small_derivatives_are_not_zero(lib, rows, k_in, k_out, z, size, dtype):
    """SiLU far left: act' and act'' are some z exp(z), 1e-16 to 1e-33, and all that the gradients are made of.  One sign, so each result is relative to
    itself: 2^-15 for the exponential (|z| u = 5e-6 and a few u), the sums of the parts and 3 sqrt(n) u for a sum over the rows; bfloat16 rows 2^-8."""
    torch = lib.torch
    print(f"dense layer, pre-activations of {z}, dY {size}, {rows} {k_in} {k_out} {dtype}", flush=True)
    layer = Layer(lib, rows, k_in, k_out, "silu", dtype, bias=False, residual=False)
    for t in (layer.X, layer.W, layer.HX, layer.dY):
        t.abs_().add_(0.5)
    layer.dY.mul_(size)
    Z = layer.wide(1, torch.full((rows, k_out), z, device="cuda"))
    first, second = np.exp(z) * (1 + z), np.exp(z) * (2 + z)       # (the rest is some exp(2 z))
    X, W, dY, HX = (t.double() for t in (layer.X, layer.W, layer.dY, layer.HX))
    G, S = dY * first, torch.matmul(HX, W) * dY * second
    Wt, Xt, Ht = W.t().contiguous(), X.t().contiguous(), HX.t().contiguous()
    slack = 2.0 ** -15 + 3 * rows ** 0.5 * 2.0 ** -24
    for name, got, want in zip(("dX", "dW", "db"), layer.backward(Z), (G @ Wt, Xt @ G, G.sum(0))):
        assert ((got.double() / want - 1).abs() <= slack + (2.0 ** -8 if name == "dX" and dtype == "bf16" else 0)).all(), name
    for name, got, want in zip(("ddY", "X2", "W2", "b2"), layer.double_backward(Z), (torch.matmul(HX, W) * first, S @ Wt, Xt @ S + Ht @ G, S.sum(0))):
        assert ((got.double() / want - 1).abs() <= slack + (2.0 ** -8 if name in ("ddY", "X2") and dtype == "bf16" else 0)).all(), name


@pytest.mark.parametrize("rows,k", [(7000, 1), (7000, 4), (70_000, 20)])
def test_exponentials_far_out(lib, rows, k):
    """SiLU in fp32 relative to itself, far left too.  The logistic p = 1 / (1 + e): 3 u of the exponential (the hardware's unit of 2 u, the correction), u of the
    sum, 2 u of the reciprocal; z p one more: 8 u with the stored z exact.  act' = p + z p q for z <= -3: 8 u of p, 16 u of z p q, which is up to 1.6
    times the sum there: 40 u, and the sum of k equal terms."""
    torch, u = lib.torch, 2.0 ** -24
    print(f"dense layer, exponentials {rows} {k}", flush=True)
    layer = Layer(lib, rows, k, k, "silu", "f32", bias=False, residual=False)
    layer.W.zero_()
    layer.W.fill_diagonal_(1.0)
    layer.X.copy_(torch.linspace(-86.0, 20.0, rows, device="cuda")[:, None].expand(rows, k))
    Y, Z = layer.forward()
    z = host(Z)
    e = np.exp(-z)
    want = z / (1 + e)
    off = np.abs(host(Y) / want - 1)
    assert off.max() <= 8 * u, f"{off.max() / u:.1f} u at {z.flat[off.argmax()]}"
    layer.dY.fill_(1.0)
    left = z[:, 0] <= -3
    p = 1 / (1 + e[left])
    want = p + z[left] * p * (1 - p)
    off = np.abs(host(layer.backward(Z, "X")[0])[left] / want - 1)
    assert off.max() <= 40 * u, f"{off.max() / u:.1f} u at {z[left].flat[off.argmax()]}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(2500, 4096, 2304), (2048, 2560, 4096), (20_000, 1280, 1280), (6000, 1280, 1280), (700, 24_576, 128), (1500, 2048, 2560)],
                         ids=lambda s: "x".join(map(str, s)))
def test_wide_layers_in_few_chunks(lib, shape, dtype):
    """Small integers: every sum exact, whatever the number of chunks."""
    base.test_small_integers_are_exact(lib, shape, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("rows,k_in,k_out", [(1, 8, 8), (777, 256, 48), (3000, 65, 67), (20_000, 128, 16), (MANY, 64, 64), (20_000, 1280, 1280), (2500, 2560, 4096),
                                             (8003, 1024, 72)])
def test_column_sums_by_themselves(lib, rows, k_in, k_out, dtype):
    """db and b2 without dW and W2: small integers, exact; with and without dX; the workspace holds NaN."""
    torch = lib.torch
    print(f"dense layer, db alone {rows} {k_in} {k_out} {dtype}", flush=True)
    for act in ("none", "relu"):
        layer = Layer(lib, rows, k_in, k_out, act, dtype)
        layer.dY.copy_(layer.dY.clamp(-3, 3).round())
        Z = layer.wide(1, layer.R)
        want = (layer.dY.double() * (Z.double() > 0 if act == "relu" else 1)).sum(0)
        for wanted in ("b", "Xb"):
            layer.ws.fill_(255)
            assert torch.equal(layer.backward(Z, wanted)[2].double(), want)
    layer = Layer(lib, rows, k_in, k_out, "silu", dtype)
    Z = layer.wide(1, layer.R)
    whole = layer.double_backward(Z)[3].double()
    for wanted in ("b", "Xb"):
        layer.ws.fill_(255)
        got = layer.double_backward(Z, wanted)[3].double()
        # |S| is below 8 for some 64 terms of unit size in V; sums of n in two orders differ by sqrt(n) units of it
        assert (got - whole).abs().max() <= 64 * rows ** 0.5 * (2.0 ** -52 if dtype == "f64" else 2.0 ** -23) + 1e-30


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k_in,k_out", [(66_001, 1024, 64), (20_000, 1280, 1280)])
def test_column_sums_do_not_cost_a_whole_dw(lib, rows, k_in, k_out, dtype):
    """Their operands are a sixteenth of those of dW (or the products a twentieth): below half of its time with room for noise."""
    torch = lib.torch
    print(f"dense layer, time of db alone {rows} {k_in} {k_out} {dtype}", flush=True)
    layer = Layer(lib, rows, k_in, k_out, "none", dtype)

    def microseconds(want):
        times = []
        for _ in range(25):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(4):
                lib.dl.dl_backward(layer.cfg, rows, layer.X, layer.W, None, layer.dY, None, dW if "W" in want else None, db, layer.ws, layer.nbytes)
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end) * 250)
        return sorted(times)[12]
    dW, db = layer.weights(layer.W), layer.weights(layer.b)
    both, alone = microseconds("Wb"), microseconds("b")
    print(f"dW and db {both:.1f} us, db {alone:.1f} us", flush=True)
    assert alone < 0.5 * both


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_the_largest_preactivations_in_fp64(lib, act):
    """act' is 1 or 0 and act'' 0 to the last bit from some 800 on, up to the largest numbers."""
    torch = lib.torch
    z = torch.tensor([s * x for x in (800.0, 1e5, 1e100, 1e289, 1e300, 1e308) for s in (1, -1)], device="cuda", dtype=torch.float64)[:, None]
    layer = Layer(lib, len(z), 1, 1, act, "f64", bias=False, residual=False)
    for t in (layer.W, layer.dY, layer.HX):
        t.fill_(1.0)
    layer.X.copy_(z)
    Y, Z = layer.forward()
    on = (z > 0).double()
    assert torch.equal(Z, z) and torch.equal(Y, z.clamp(min=0)) and torch.equal(layer.backward(Z)[0], on)
    ddY, X2, W2, _ = layer.double_backward(Z)
    assert torch.equal(ddY, on) and not X2.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e30, 1e34])
@pytest.mark.parametrize("rows,k_in,k_out", [(20, 64, 64), (MANY, 64, 64), (MANY, 132, 72), (MANY, 64, 260), (3000, 512, 256)])
def test_large_gradients(lib, rows, k_in, k_out, size, dtype):
    """SiLU with an upstream gradient near the largest numbers in a few rows; the others are as they would be without.  All of one sign: relative, 2^-16 for the sums
    of 66 001 rows and less elsewhere, bfloat16 rows 2^-8."""
    torch = lib.torch
    print(f"dense layer, some dY of {size}, {rows} {k_in} {k_out} {dtype}", flush=True)
    layer = Layer(lib, rows, k_in, k_out, "silu", dtype, bias=False, residual=False)
    for t in (layer.X, layer.W, layer.HX, layer.dY):
        t.abs_().add_(0.5)
    layer.W.mul_(0.125)
    layer.dY[3::1000] *= size
    Z = layer.wide(1, torch.rand(rows, k_out, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda") - 0.5)
    X, W, dY, HX, z = (t.double() for t in (layer.X, layer.W, layer.dY, layer.HX, Z))
    p = torch.sigmoid(z)
    first, second = p + z * p * (1 - p), p * (1 - p) * (2 + z * (1 - 2 * p))
    V = torch.matmul(HX, W)
    G, S = dY * first, V * dY * second
    Wt, Xt, Ht = W.t().contiguous(), X.t().contiguous(), HX.t().contiguous()
    want = dict(dX=torch.matmul(G, Wt), dW=torch.matmul(Xt, G), db=G.sum(0), ddY=V * first, X2=torch.matmul(S, Wt), W2=torch.matmul(Xt, S) + torch.matmul(Ht, G), b2=S.sum(0))
    assert all(w.max() < 3e38 for w in want.values())
    got = dict(zip(("dX", "dW", "db", "ddY", "X2", "W2", "b2"), layer.backward(Z) + layer.double_backward(Z)))
    for name, w in want.items():
        off = (got[name].double() / w - 1).abs().max().item()
        assert off <= 2.0 ** -16 + (2.0 ** -8 if dtype == "bf16" and name in ("dX", "ddY", "X2") else 0), f"{name}: {off}"
