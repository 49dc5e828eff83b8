"""The dense layer (include/dl.h) through the C ABI against its fp64 oracle, evaluated on the rounded inputs.

Tolerances, element by element, u = 2^-24 (2^-53 for fp64):
  a sum of k products in any order: (k + 2) u sum |a||b|, twice that where an operand itself was rounded on the way;
  act, act' and act'' as evaluated: 16 u (1 + |z|), 32 u, 128 u (act'' is below 1.2 in size, act' below 1.13, and the
  exponential's relative error |z| u meets a factor that falls with it);
  bfloat16 results: one rounding, 2^-8 of the value (half a unit of the eighth bit), on top of 2^-16 sum |a||b| (weights may enter with 16 bits there).
"""
import numpy as np
import pytest

from oracle import dense_layer as od

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -24}


@pytest.fixture(scope="module")
def lib():
    import torch
    assert torch.cuda.is_available()
    from paper_2504_10700_amd import dl_binding as dl

    class Lib:
        pass
    Lib.torch, Lib.dl, Lib.dev = torch, dl, torch.device("cuda:0")
    Lib.row = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}
    Lib.weight = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.float32}
    Lib.kind = {"f32": dl.SC_F32, "f64": dl.SC_F64, "bf16": dl.SC_BF16}
    return Lib


def host(x):
    return x.double().cpu().numpy()


class Layer:
    """One layer's tensors on the device, rows `spread` times as wide as the layer with NaN in between."""

    def __init__(self, lib, rows, k_in, k_out, act, dtype, bias=True, residual=True, spread=(1, 1), seed=1, scale=1.0):
        self.lib, self.rows, self.k_in, self.k_out, self.act, self.dtype, self.spread = lib, rows, k_in, k_out, act, dtype, spread
        torch = lib.torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
        self.W = (normal(k_in, k_out) / k_in ** 0.5).to(lib.weight[dtype])
        self.b = normal(k_out).to(lib.weight[dtype]) if bias else None
        self.X = self.wide(0, normal(rows, k_in) * scale)
        self.R = self.wide(1, normal(rows, k_out)) if residual else None
        self.dY = self.wide(1, normal(rows, k_out))
        self.HX = self.wide(0, normal(rows, k_in))
        act_id = {"none": lib.dl.DL_NONE, "relu": lib.dl.DL_RELU, "silu": lib.dl.DL_SILU, "gelu": lib.dl.DL_GELU}[act]
        self.cfg = lib.dl.make_config(k_in, k_out, act_id, lib.kind[dtype], ld_in=spread[0] * k_in if spread[0] > 1 else 0,
                                      ld_out=spread[1] * k_out if spread[1] > 1 else 0)
        self.nbytes = lib.dl.dl_workspace_bytes(self.cfg, rows)
        self.ws = torch.full((self.nbytes,), 255, dtype=torch.uint8, device="cuda")

    def wide(self, side, values=None):
        k = (self.k_in, self.k_out)[side]
        full = self.lib.torch.full((self.rows, self.spread[side] * k), float("nan"), dtype=self.lib.row[self.dtype], device="cuda")
        if values is not None:
            full[:, :k] = values.to(full.dtype)
        return full[:, :k]

    def gaps_untouched(self, *tensors):
        for t in tensors:
            if t is not None and t._base is not None and t._base.shape[1] > t.shape[1]:
                assert self.lib.torch.isnan(t._base[:, t.shape[1]:]).all(), "an element between the rows was written"

    def weights(self, like):
        return self.lib.torch.full_like(like, float("nan"))

    def forward(self, want_z=True, stream=None):
        Y, Z = self.wide(1), self.wide(1) if want_z else None
        self.lib.dl.dl_forward(self.cfg, self.rows, self.X, self.W, self.b, self.R, Y, Z, stream)
        return Y, Z

    def backward(self, Z, want="XWb"):
        dX = self.wide(0) if "X" in want else None
        dW = self.weights(self.W) if "W" in want else None
        db = self.weights(self.W[0]) if "b" in want else None
        self.lib.dl.dl_backward(self.cfg, self.rows, self.X, self.W, Z, self.dY, dX, dW, db, self.ws, self.nbytes)
        return dX, dW, db

    def double_backward(self, Z, want="XWb"):
        ddY = self.wide(1)
        X2 = self.wide(0) if "X" in want else None
        W2 = self.weights(self.W) if "W" in want else None
        b2 = self.weights(self.W[0]) if "b" in want else None
        self.lib.dl.dl_double_backward(self.cfg, self.rows, self.X, self.W, Z, self.dY, self.HX, ddY, X2, W2, b2, self.ws, self.nbytes)
        return ddY, X2, W2, b2


def near(name, got, ref, slack, dtype, rows):
    """|got - ref| <= slack, plus the final rounding of a result with bfloat16 rows."""
    got = host(got)
    if dtype == "bf16" and rows:
        slack = 1.01 * slack + 1.01 * 2.0 ** -8 * np.abs(ref)
    worst = float(np.max((np.abs(got - ref) - slack) / (np.abs(ref).mean() + 1e-300))) if got.size else -1.0
    assert np.isfinite(got).all(), f"{name}: not finite"
    assert worst <= 0, f"{name}: beyond its bound by {worst:.2e} of the mean"


def check_layer(layer, calls=("forward", "backward", "second")):
    act, dtype, u = layer.act, layer.dtype, U[layer.dtype]
    X, W, dY, HX = host(layer.X), host(layer.W), host(layer.dY), host(layer.HX)
    b = None if layer.b is None else host(layer.b)
    R = None if layer.R is None else host(layer.R)
    n, ki, ko = layer.rows, layer.k_in, layer.k_out
    parts = 2.0 ** -16 if dtype == "bf16" else 0.0     # of sum |a||b|, results in bfloat16 rows
    Y, Z = layer.forward()
    layer.gaps_untouched(Y, Z)
    if "forward" in calls:
        Yr, Zr = od.forward(act, X, W, b, R)
        e = ((ki + 2) * u + parts) * (np.abs(X) @ np.abs(W) + (0 if b is None else np.abs(b)))
        near("Z", Z, Zr, e, dtype, True)
        near("Y", Y, Yr, 1.2 * e + 16 * u * (1 + np.abs(Zr) + (0 if R is None else np.abs(R))), dtype, True)
    Zh = host(Z)                                        # the backward calls are functions of the stored Z
    first, second = od.activation(act, Zh)[1:]
    Zd = None if act == "none" else Z
    if "backward" in calls:
        dX, dW, db = layer.backward(Zd)
        layer.gaps_untouched(dX)
        rX, rW, rb = od.backward(act, X, W, Zh, dY)
        g = np.abs(dY) * (np.abs(first) + 1)            # |G|, and the error of act' beside it
        near("dX", dX, rX, ((2 * ko + 40) * u + parts) * (g @ np.abs(W).T), dtype, True)
        near("dW", dW, rW, (2 * n + 40) * u * (np.abs(X).T @ g), dtype, False)
        near("db", db, rb, (2 * n + 40) * u * g.sum(0), dtype, False)
    if "second" in calls:
        ddY, X2, W2, b2 = layer.double_backward(Zd)
        layer.gaps_untouched(ddY, X2)
        rY, rX, rW, rb = od.double_backward(act, X, W, Zh, dY, HX)
        v = np.abs(HX) @ np.abs(W)                      # |V|
        near("ddY", ddY, rY, ((2 * ki + 40) * u + parts) * v * (np.abs(first) + 1), dtype, True)
        s = v * np.abs(dY) * (np.abs(second) + (1 if act in ("silu", "gelu") else 0))
        g = np.abs(dY) * (np.abs(first) + 1)
        near("X2", X2, rX, ((2 * ki + 2 * ko + 160) * u + 2 * parts) * (s @ np.abs(W).T), dtype, True)
        near("W2", W2, rW, (2 * n + 2 * ki + 160) * u * (np.abs(X).T @ s + np.abs(HX).T @ g), dtype, False)
        near("b2", b2, rb, (2 * n + 2 * ki + 160) * u * s.sum(0), dtype, False)


# one row to many; one column to wide; sizes around the tiles of 16, 32, 64 and 128
SHAPES = [(1, 1, 1), (1, 8, 64), (2, 64, 1), (3, 5, 7), (16, 16, 16), (17, 33, 15), (63, 64, 65), (64, 64, 64), (65, 61, 129),
          (127, 128, 128), (129, 100, 36), (380, 8, 64), (1000, 64, 64), (1029, 64, 80), (2500, 3, 130), (777, 256, 48), (500, 64, 1280),
          (5, 1024, 300), (300, 1025, 9), (4100, 128, 16), (1, 2000, 3)]


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_oracle(lib, shape, dtype):
    act = od.ACTIVATIONS[(shape[0] + shape[1] + shape[2]) % 4]
    print(f"dense layer {shape} {dtype} {act}", flush=True)
    check_layer(Layer(lib, *shape, act, dtype))


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("act", od.ACTIVATIONS)
@pytest.mark.parametrize("bias,residual", [(True, True), (False, False), (True, False), (False, True)])
def test_activations_bias_and_residual(lib, act, dtype, bias, residual):
    print(f"dense layer {act} {dtype} bias {bias} residual {residual}", flush=True)
    check_layer(Layer(lib, 333, 64, 72, act, dtype, bias, residual, scale=3.0))


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("shape,spread", [((200, 64, 64), (4, 1)), ((200, 64, 64), (1, 3)), ((131, 17, 33), (3, 2)), ((1030, 128, 16), (4, 1))],
                         ids=str)
def test_strided_rows(lib, shape, spread, dtype):
    print(f"dense layer strides {shape} {spread} {dtype}", flush=True)
    check_layer(Layer(lib, *shape, "silu", dtype, spread=spread))


@pytest.mark.parametrize("dtype,rows,k_in,k_out,act", [("f32", 70_001, 64, 64, "silu"), ("bf16", 70_001, 64, 64, "gelu"),
                                                       ("f32", 20_011, 64, 1280, "none"), ("bf16", 20_011, 64, 1280, "none"),
                                                       ("f64", 20_011, 128, 16, "silu"), ("f32", 3000, 1024, 512, "gelu"),
                                                       ("bf16", 3000, 1024, 512, "gelu"), ("bf16", 40_003, 128, 128, "silu")])
def test_many_rows(lib, dtype, rows, k_in, k_out, act):
    print(f"dense layer {rows} x {k_in} -> {k_out} {dtype} {act}", flush=True)
    check_layer(Layer(lib, rows, k_in, k_out, act, dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,k_in,k_out", [(777, 64, 64), (5000, 64, 128), (300, 200, 96)])
def test_optional_outputs_and_repetition(lib, dtype, rows, k_in, k_out):
    """Outputs left out do not change the others, and a call repeats to the bit."""
    torch = lib.torch
    print(f"dense layer optional outputs {rows} {k_in} {k_out} {dtype}", flush=True)
    for act in ("silu", "relu", "none"):
        layer = Layer(lib, rows, k_in, k_out, act, dtype)
        Y, Z = layer.forward()
        assert torch.equal(layer.forward(want_z=False)[0], Y) and torch.equal(layer.forward()[1], Z)
        Zd = None if act == "none" else Z
        for call in (layer.backward, layer.double_backward):
            whole = call(Zd)
            assert all(torch.equal(a, b) for a, b in zip(whole, call(Zd)))
            for want in ("X", "W", "b", "Xb", "Wb", "XW"):
                for full, part in zip(whole, call(Zd, want)):
                    # (a product may be cut differently where fewer results are wanted: equal up to the bound of its sums)
                    if part is not None:
                        d = (full.double() - part.double()).abs().max().item()
                        assert d <= 1e-4 * (full.double().abs().max().item() + 1e-30) or dtype == "bf16" and d <= 2 ** -7 * full.double().abs().max().item()


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
def test_no_rows(lib, dtype):
    torch = lib.torch
    layer = Layer(lib, 0, 64, 96, "silu", dtype)
    layer.forward()
    dX, dW, db = layer.backward(layer.wide(1))
    assert not dW.any() and not db.any()
    ddY, X2, W2, b2 = layer.double_backward(layer.wide(1))
    assert not W2.any() and not b2.any()
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("k_in,k_out", [(64, 64), (20, 132), (64, 1280)])
def test_values_that_are_not_finite_stay_in_their_row(lib, dtype, value, k_in, k_out):
    """A row of X or dY that holds one changes its own row of the results only; its own row is what the arithmetic says."""
    torch = lib.torch
    print(f"dense layer with {value} {dtype} {k_in} {k_out}", flush=True)
    layer = Layer(lib, 300, k_in, k_out, "none", dtype)
    Y0, _ = layer.forward()
    dX0 = layer.backward(None)[0]
    layer.X[77, 3] = value
    layer.dY[205, 5] = value
    Y, _ = layer.forward()
    dX, dW, db = layer.backward(None)
    bound = {"f32": 1e-5, "f64": 1e-13, "bf16": 2.0 ** -7}[dtype]
    for got, before, row, w in ((Y, Y0, 77, layer.W[3]), (dX, dX0, 205, layer.W[:, 5])):
        keep = torch.arange(300, device="cuda") != row
        assert (got[keep].double() - before[keep].double()).abs().max() <= bound * before.double().abs().max()
        want = value * w.double()                      # NaN, or an infinity with the sign of the weight
        assert torch.equal(torch.isnan(got[row]), torch.isnan(want))
        assert torch.equal(got[row].double()[~torch.isnan(want)], want[~torch.isnan(want)])
    assert not torch.isfinite(dW[3]).any() and not torch.isfinite(dW[:, 5]).any() and not torch.isfinite(db[5])
    keep_k, keep_n = torch.arange(k_in, device="cuda") != 3, torch.arange(k_out, device="cuda") != 5
    assert torch.isfinite(dW[keep_k][:, keep_n]).all() and torch.isfinite(db[keep_n]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-36, 1e-25, 1e18, 3e37])
def test_values_of_every_size(lib, dtype, size):
    """Sums over rows or weights far from 1 in size keep the relative error of their type."""
    torch = lib.torch
    print(f"dense layer, values of size {size} {dtype}", flush=True)
    layer = Layer(lib, 200, 64, 64, "none", dtype, bias=False, residual=False)
    layer.X.copy_((layer.X.double().clamp(-3, 3) * size).to(layer.X.dtype))
    layer.W.copy_(layer.W.clamp(-0.1, 0.1))
    X, W = host(layer.X), host(layer.W)
    Y, _ = layer.forward()
    ref, magnitude = X @ W, np.abs(X) @ np.abs(W)
    slack = (66 * 2.0 ** -24 + (2.0 ** -8 + 2.0 ** -16 if dtype == "bf16" else 0)) * magnitude + 2.0 ** -125 * 2.0 ** -8
    assert (np.abs(host(Y) - ref) <= slack).all()
    layer.dY.copy_(layer.dY.clamp(-3, 3) * 1e-3)
    dW = layer.backward(None)[1]
    dY = host(layer.dY)
    assert (np.abs(host(dW) - X.T @ dY) <= 240 * 2.0 ** -24 * (np.abs(X).T @ np.abs(dY)) + 2.0 ** -125).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "f64"])
def test_activations_far_out(lib, act, dtype):
    """Pre-activations from -1e30 to 1e30: values and gradients are those of the limits, never NaN."""
    torch = lib.torch
    z = np.array([-1e30, -1e12, -3e4, -200, -90, -30, -5, 0, 5, 30, 90, 200, 3e4, 1e12, 1e30])
    layer = Layer(lib, len(z), 1, 1, act, dtype, bias=False, residual=False)
    layer.W.fill_(1.0)
    layer.X.copy_(torch.tensor(z)[:, None])
    layer.dY.fill_(1.0)
    layer.HX.fill_(1.0)
    Y, Z = layer.forward()
    value, first, second = od.activation(act, host(layer.X))
    value, first, second = (np.where(np.abs(z)[:, None] > 100, lim, x) for x, lim in
                            ((value, np.maximum(z, 0)[:, None]), (first, (z > 0)[:, None] * 1.0), (second, 0.0)))
    tol = 1e-5 if dtype == "f32" else 1e-13
    assert (np.abs(host(Y) - value) <= tol * (1 + np.abs(value))).all()
    assert (np.abs(host(layer.backward(Z)[0]) - first) <= tol).all()
    ddY, X2, _, _ = layer.double_backward(Z)
    assert (np.abs(host(ddY) - first) <= tol).all() and (np.abs(host(X2) - second) <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_beyond_32_bits(lib, dtype):
    """Rows so far apart that element offsets pass 2^31 (and byte offsets 2^32)."""
    torch = lib.torch
    rows, ld, k = 1100, 2_100_000, 24
    print(f"dense layer, {rows} rows {ld} elements apart, {dtype}", flush=True)
    full = torch.empty(rows * ld, dtype=lib.row[dtype], device="cuda").view(rows, ld)
    layer = Layer(lib, rows, k, k, "silu", dtype)
    dense_x, dense_dy = layer.X, layer.dY
    Y0, Z0 = layer.forward()
    dX0, dW0, db0 = layer.backward(Z0)
    cfg = lib.dl.make_config(k, k, lib.dl.DL_SILU, lib.kind[dtype], ld_in=ld, ld_out=ld)
    x, dy, r, y, z, dx = (full[:, 1000 * i:1000 * i + k] for i in range(6))
    for wide, dense in ((x, dense_x), (dy, dense_dy), (r, layer.R)):
        wide.copy_(dense)
    dW, db = torch.empty_like(dW0), torch.empty_like(db0)
    lib.dl.dl_forward(cfg, rows, x, layer.W, layer.b, r, y, z)
    lib.dl.dl_backward(cfg, rows, x, layer.W, z, dy, dx, dW, db, layer.ws, layer.nbytes)
    for a, b in ((y, Y0), (z, Z0), (dx, dX0), (dW, dW0), (db, db0)):
        assert torch.equal(a, b)


def test_a_stack_of_layers_against_automatic_differentiation(lib):
    """Three layers with a residual, first and second order, chained as a radial network is: the gradient of a loss on the
    gradient with respect to the input (a force) for every weight."""
    torch, dl = lib.torch, lib.dl
    rows, widths, acts = 301, (8, 64, 64, 80), ("silu", "silu", "none")
    ids = {"silu": dl.DL_SILU, "none": dl.DL_NONE}
    g = torch.Generator(device="cuda").manual_seed(9)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64)  # noqa: E731
    Ws = [new(a, b) / a ** 0.5 for a, b in zip(widths, widths[1:])]
    bs = [new(b) for b in widths[1:]]
    X0, dY, H0 = new(rows, 8), new(rows, 80), new(rows, 8)
    cfgs = [dl.make_config(a, b, ids[t], dl.SC_F64) for a, b, t in zip(widths, widths[1:], acts)]
    nbytes = max(dl.dl_workspace_bytes(c, rows) for c in cfgs)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    Xs, Zs = [X0], []
    for i, c in enumerate(cfgs):                      # the second layer adds its input
        Y, Z = torch.empty(rows, widths[i + 1], dtype=torch.float64, device="cuda"), torch.empty(rows, widths[i + 1], dtype=torch.float64, device="cuda")
        dl.dl_forward(c, rows, Xs[i], Ws[i], bs[i], Xs[i] if i == 1 else None, Y, Z)
        Xs.append(Y)
        Zs.append(Z)
    grads, up = [None] * 3, [None, None, dY]          # up[i]: gradient of layer i's output
    for i in (2, 1, 0):
        dX, dW, db = torch.empty_like(Xs[i]), torch.empty_like(Ws[i]), torch.empty_like(bs[i])
        dl.dl_backward(cfgs[i], rows, Xs[i], Ws[i], Zs[i], up[i], dX, dW, db, ws, nbytes)
        grads[i] = (dX, dW, db)
        if i:
            up[i - 1] = dX + up[i] if i == 1 else dX
    # loss = sum(H0 * dX of the first layer): its cotangents run forward through the second-order passes ...
    H, seconds = H0, []
    for i in range(3):
        ddY, X2 = torch.empty_like(Zs[i]), torch.empty_like(Xs[i])
        W2, b2 = torch.empty_like(Ws[i]), torch.empty_like(bs[i])
        dl.dl_double_backward(cfgs[i], rows, Xs[i], Ws[i], Zs[i], up[i], H, ddY, X2, W2, b2, ws, nbytes)
        seconds.append((X2, W2, b2))
        H = ddY + H if i == 1 else ddY
    # ... and what they leave on the activations runs backward as an ordinary gradient
    total_W, total_b, back = [s[1].clone() for s in seconds], [s[2].clone() for s in seconds], None
    for i in (2, 1, 0):
        if back is not None:
            dX, dW, db = torch.empty_like(Xs[i]), torch.empty_like(Ws[i]), torch.empty_like(bs[i])
            dl.dl_backward(cfgs[i], rows, Xs[i], Ws[i], Zs[i], back, dX, dW, db, ws, nbytes)
            total_W[i] += dW
            total_b[i] += db
            back = seconds[i][0] + dX + (back if i == 1 else 0)
        else:
            back = seconds[i][0]
    # the same in torch, on the CPU
    cpu = lambda x: x.cpu().clone().requires_grad_(True)  # noqa: E731
    tW, tb, tx, tdy = [cpu(w) for w in Ws], [cpu(b) for b in bs], cpu(X0), dY.cpu()
    h = tx
    for i in range(3):
        z = h @ tW[i] + tb[i]
        y = torch.nn.functional.silu(z) if acts[i] == "silu" else z
        h = y + h if i == 1 else y
    first = torch.autograd.grad((tdy * h).sum(), [tx] + tW + tb, create_graph=True)
    second = torch.autograd.grad((H0.cpu() * first[0]).sum(), [tx] + tW + tb, allow_unused=True)
    for got, want in zip([grads[0][0]] + [q[1] for q in grads] + [q[2] for q in grads], first):
        assert (got.cpu() - want).abs().max() <= 1e-12 * want.abs().max()
    for got, want in zip([back] + total_W + total_b, second):
        want = torch.zeros_like(got.cpu()) if want is None else want
        assert (got.cpu() - want).abs().max() <= 1e-12 * (want.abs().max() + 1)


def test_other_stream_and_graph_replay(lib):
    torch = lib.torch
    layer = Layer(lib, 2000, 64, 96, "silu", "f32")
    Y, Z = layer.forward()
    dX, dW, db = layer.backward(Z)
    ref = [t.clone() for t in (Y, Z, dX, dW, db)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = [layer.wide(1), layer.wide(1), layer.wide(0), layer.weights(layer.W), layer.weights(layer.b)]

    def step():
        lib.dl.dl_forward(layer.cfg, 2000, layer.X, layer.W, layer.b, layer.R, out[0], out[1])
        lib.dl.dl_backward(layer.cfg, 2000, layer.X, layer.W, out[1], layer.dY, out[2], out[3], out[4], layer.ws, layer.nbytes)
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(3):
        if replay:
            layer.X.mul_(0.5)
            Y, Z = layer.forward()
            ref = [t.clone() for t in (Y, Z, *layer.backward(Z))]
        for t in out:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, ref)), f"replay {replay}"


# ---- many rows: the results of whole rows on the bfloat16 matrix cores, where an fp32 number is the sum of three bfloat16 ones

MANY = 66_001


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k_in,k_out,act", [(72, 36, "gelu"), (20, 192, "silu"), (24, 72, "relu"), (100, 324, "silu"), (64, 132, "none"), (132, 64, "relu"),
                                            (40, 4, "silu"), (8, 64, "gelu"), (192, 200, "silu"), (63, 64, "silu"), (64, 65, "none")])
def test_many_rows_of_odd_widths(lib, k_in, k_out, act, dtype):
    print(f"dense layer {MANY} x {k_in} -> {k_out} {dtype} {act}", flush=True)
    check_layer(Layer(lib, MANY, k_in, k_out, act, dtype))


EXACT = SHAPES + [(300, 20, 132), (700, 64, 260), (3000, 64, 260), (5000, 128, 192), (5000, 192, 320), (9000, 33, 195), (2100, 1280, 4), (2100, 4, 1280),
                  (250, 1024, 1024), (600, 1000, 1024), (2100, 1024, 1028), (6000, 128, 1240), (3000, 256, 512), (8003, 128, 128), (5000, 200, 200),
                  (MANY, 64, 64), (MANY, 24, 192), (MANY, 64, 260), (MANY, 100, 324), (MANY, 192, 136), (MANY, 65, 67), (20_011, 64, 1280)]


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("shape", EXACT, ids=lambda s: "x".join(map(str, s)))
def test_small_integers_are_exact(lib, shape, dtype):
    """Sums of products of small integers are exact in any order: no term may be missing, wrong or counted twice.  (Results in bfloat16 rows: rounded once.)"""
    torch = lib.torch
    act = ("none", "relu")[sum(shape) % 2]
    print(f"dense layer {shape} {dtype} {act}, integers", flush=True)
    layer = Layer(lib, *shape, act, dtype)
    for t in (layer.X, layer.W, layer.b, layer.R, layer.dY, layer.HX):
        t.copy_(t.clamp(-3, 3).round() if t is not layer.W else (t * shape[1] ** 0.5).clamp(-3, 3).round())
    X, W, b, R, dY, HX = (t.double() for t in (layer.X, layer.W, layer.b, layer.R, layer.dY, layer.HX))

    def same(name, got, ref):
        assert torch.equal(got, ref.to(got.dtype)), f"{name}: {int((got != ref.to(got.dtype)).sum())} elements differ"

    Y, Z = layer.forward()
    z = X @ W + b
    same("Z", Z, z)
    same("Y", Y, (z.clamp(min=0) if act == "relu" else z) + R)
    gate = (Z.double() > 0).double() if act == "relu" else torch.ones_like(z)
    G = dY * gate
    dX, dW, db = layer.backward(Z if act == "relu" else None)
    same("dX", dX, G @ W.T.contiguous())
    same("dW", dW, X.T.contiguous() @ G)
    same("db", db, G.sum(0))
    ddY, X2, W2, b2 = layer.double_backward(Z if act == "relu" else None)
    same("ddY", ddY, (HX @ W) * gate)
    assert not X2.any() and not b2.any()
    same("W2", W2, HX.T.contiguous() @ G)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("spread", [(4, 1), (1, 3), (3, 2)], ids=str)
@pytest.mark.parametrize("k_in,k_out", [(64, 64), (68, 140)])
def test_many_strided_rows(lib, k_in, k_out, spread, dtype):
    print(f"dense layer {MANY} x {k_in} -> {k_out} strides {spread} {dtype}", flush=True)
    check_layer(Layer(lib, MANY, k_in, k_out, "silu", dtype, spread=spread))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("k_in,k_out", [(64, 64), (128, 192)])
def test_many_rows_far_out(lib, k_in, k_out, act, dtype):
    """Pre-activations of several tens: most derivatives are 0 or 1, many too small for their own parts."""
    print(f"dense layer {MANY} x {k_in} -> {k_out} {dtype} {act}, wide rows", flush=True)
    check_layer(Layer(lib, MANY, k_in, k_out, act, dtype, scale=30.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("k_in,k_out", [(64, 64), (24, 192), (64, 260)])
def test_many_rows_with_values_that_are_not_finite(lib, dtype, value, k_in, k_out):
    torch = lib.torch
    print(f"dense layer {MANY} rows with {value} {dtype} {k_in} {k_out}", flush=True)
    layer = Layer(lib, MANY, k_in, k_out, "none", dtype)
    u = 2.0 ** -24
    absolute = lambda t: t.double().abs()  # noqa: E731
    part = 2.0 ** -16 if dtype == "bf16" else 0.0
    slack_y = 2 * ((k_in + 4) * u + part) * (absolute(layer.X) @ absolute(layer.W) + absolute(layer.b) + absolute(layer.R))
    slack_x = 2 * ((k_out + 4) * u + part) * (absolute(layer.dY) @ absolute(layer.W).T.contiguous())
    Y0, _ = layer.forward()
    dX0 = layer.backward(None)[0]
    for row, column in ((77, 3), (40_000, 17), (MANY - 1, 0)):
        layer.X[row, column] = value
        layer.dY[row - 30, column + 2] = value
    Y, _ = layer.forward()
    dX, dW, db = layer.backward(None)
    last = 2.0 ** -7 if dtype == "bf16" else 2 * u
    keep = torch.ones(MANY, dtype=torch.bool, device="cuda")
    keep_x = keep.clone()
    keep_k, keep_n = torch.ones(k_in, dtype=torch.bool, device="cuda"), torch.ones(k_out, dtype=torch.bool, device="cuda")
    for row, column in ((77, 3), (40_000, 17), (MANY - 1, 0)):
        keep[row] = keep_x[row - 30] = False
        keep_k[column] = keep_n[column + 2] = False
        for got, r, w in ((Y, row, layer.W[column]), (dX, row - 30, layer.W[:, column + 2])):
            want = value * w.double()
            assert torch.equal(torch.isnan(got[r]), torch.isnan(want))
            assert torch.equal(got[r].double()[~torch.isnan(want)], want[~torch.isnan(want)])
    assert ((Y.double() - Y0.double()).abs() <= slack_y + last * absolute(Y0))[keep].all()
    assert ((dX.double() - dX0.double()).abs() <= slack_x + last * absolute(dX0))[keep_x].all()
    assert not torch.isfinite(dW[~keep_k]).any() and not torch.isfinite(dW[:, ~keep_n]).any() and not torch.isfinite(db[~keep_n]).any()
    X, dY = layer.X.double(), layer.dY.double()
    X[~keep], dY[~keep_x] = 0, 0                       # (those rows touch other columns too)
    finite = (layer.X.double()[~keep][:, keep_k].T @ layer.dY.double()[~keep][:, keep_n] +
              layer.X.double()[~keep_x][:, keep_k].T @ layer.dY.double()[~keep_x][:, keep_n])
    ref = X[:, keep_k].T @ dY[:, keep_n] + finite
    magnitude = absolute(layer.X)[:, keep_k].T @ absolute(layer.dY)[:, keep_n]
    assert ((dW[keep_k][:, keep_n].double() - ref).abs() <= 2 * (MANY + 4) * u * magnitude).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), 3e38, 1e-42])
@pytest.mark.parametrize("k_in,k_out", [(64, 64), (24, 260)])
def test_many_rows_with_an_unusual_weight(lib, dtype, value, k_in, k_out):
    """One weight that is not finite, close to the largest number, or below the smallest normal one: its column of Y and of dX show it, no other."""
    torch = lib.torch
    print(f"dense layer {MANY} rows, a weight of {value} {dtype} {k_in} {k_out}", flush=True)
    layer = Layer(lib, MANY, k_in, k_out, "none", dtype, bias=False, residual=False)
    layer.X.clamp_(-1, 1)
    layer.dY.clamp_(-1, 1)
    layer.W[5, 9] = value
    Y, _ = layer.forward()
    dX = layer.backward(None, "X")[0]
    u, part, last = 2.0 ** -24, 2.0 ** -16 if dtype == "bf16" else 0.0, 2.0 ** -8 if dtype == "bf16" else 0.0
    X, W, dY = layer.X.double(), layer.W.double(), layer.dY.double()
    for got, a, b, column, k in ((Y, X, W, 9, k_in), (dX, dY, W.T.contiguous(), 5, k_out)):
        keep = torch.arange(got.shape[1], device="cuda") != column
        ref, magnitude = a @ b[:, keep], a.abs() @ b[:, keep].abs()
        assert ((got[:, keep].double() - ref).abs() <= 1.01 * ((k + 2) * u + part) * magnitude + last * ref.abs()).all()
        factor = a[:, 5 if column == 9 else 9] * W[5, 9]
        if np.isfinite(value):
            ref, magnitude = (a @ b[:, ~keep])[:, 0], (a.abs() @ b[:, ~keep].abs())[:, 0]
            assert ((got[:, column].double() - ref).abs() <= 1.01 * ((k + 2) * u + part) * magnitude + last * ref.abs()).all()
        else:
            assert torch.equal(torch.isnan(got[:, column]), torch.isnan(factor))
            assert torch.equal(got[:, column].double()[~torch.isnan(factor)], factor[~torch.isnan(factor)])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [1e-36, 1e-30, 1e-25, 1e18, 3e37])
def test_many_rows_of_every_size(lib, dtype, size):
    """A third of the rows and of the entries of other rows far from 1 in size."""
    torch = lib.torch
    print(f"dense layer {MANY} rows, values of size {size} {dtype}", flush=True)
    layer = Layer(lib, MANY, 64, 64, "none", dtype, bias=False, residual=False)
    x = layer.X.double().clamp(-3, 3)
    x[MANY // 3:2 * MANY // 3] *= size
    x[2 * MANY // 3::50, ::7] *= size
    layer.X.copy_(x.to(layer.X.dtype))
    layer.W.copy_(layer.W.clamp(-0.1, 0.1))
    X, W = host(layer.X), host(layer.W)
    Y, _ = layer.forward()
    ref, magnitude = X @ W, np.abs(X) @ np.abs(W)
    slack = (66 * 2.0 ** -24 + (2.0 ** -8 + 2.0 ** -16 if dtype == "bf16" else 0)) * magnitude + 2.0 ** -125 * 2.0 ** -8
    assert (np.abs(host(Y) - ref) <= slack).all()
    layer.dY.copy_(layer.dY.clamp(-3, 3) * 1e-3)
    dW = layer.backward(None)[1]
    dY = host(layer.dY)
    assert (np.abs(host(dW) - X.T @ dY) <= (MANY + 40) * 2.0 ** -24 * (np.abs(X).T @ np.abs(dY)) + 2.0 ** -125).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k_in,k_out", [(64, 64), (128, 192)])
def test_many_rows_optional_outputs_and_repetition(lib, dtype, k_in, k_out):
    torch = lib.torch
    print(f"dense layer optional outputs {MANY} {k_in} {k_out} {dtype}", flush=True)
    for act in ("silu", "relu", "none"):
        layer = Layer(lib, MANY, k_in, k_out, act, dtype)
        Y, Z = layer.forward()
        assert torch.equal(layer.forward(want_z=False)[0], Y) and torch.equal(layer.forward()[1], Z)
        Zd = None if act == "none" else Z
        for call in (layer.backward, layer.double_backward):
            whole = call(Zd)
            layer.ws.fill_(255)
            assert all(torch.equal(a, b) for a, b in zip(whole, call(Zd)))
            for want in ("X", "W", "b", "Xb", "Wb", "XW"):
                for full, part in zip(whole, call(Zd, want)):
                    # (a product may be cut differently where fewer results are wanted: equal up to the bound of its sums)
                    if part is not None:
                        d = (full.double() - part.double()).abs().max().item()
                        assert d <= (2.0 ** -7 if dtype == "bf16" else 1e-4) * full.double().abs().max().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows_offsets_beyond_32_bits(lib, dtype):
    torch = lib.torch
    ld, k = 40_000, 64
    print(f"dense layer, {MANY} rows {ld} elements apart, {dtype}", flush=True)
    full = torch.empty(MANY * ld, dtype=lib.row[dtype], device="cuda").view(MANY, ld)
    layer = Layer(lib, MANY, k, k, "silu", dtype)
    Y0, Z0 = layer.forward()
    dX0, dW0, db0 = layer.backward(Z0)
    cfg = lib.dl.make_config(k, k, lib.dl.DL_SILU, lib.kind[dtype], ld_in=ld, ld_out=ld)
    x, dy, r, y, z, dx = (full[:, 1000 * i:1000 * i + k] for i in range(6))
    for wide, dense in ((x, layer.X), (dy, layer.dY), (r, layer.R)):
        wide.copy_(dense)
    dW, db = torch.empty_like(dW0), torch.empty_like(db0)
    nbytes = lib.dl.dl_workspace_bytes(cfg, MANY)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    lib.dl.dl_forward(cfg, MANY, x, layer.W, layer.b, r, y, z)
    lib.dl.dl_backward(cfg, MANY, x, layer.W, z, dy, dx, dW, db, ws, nbytes)
    for a, b in ((y, Y0), (z, Z0), (dx, dX0), (dW, dW0), (db, db0)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("rows", [5, 2000, MANY])
def test_relu_of_infinities(lib, dtype, rows):
    """max(z, 0) and its derivative are 0 at minus infinity; infinity stays."""
    layer = Layer(lib, rows, 32, 32, "relu", dtype, bias=False, residual=False)
    layer.W.zero_()
    layer.W.fill_diagonal_(1.0)
    layer.X.zero_()
    layer.X[rows // 2] = 1.0
    layer.X[3, :] = 0.0
    layer.X[3, 4], layer.X[4, 5] = -float("inf"), float("inf")
    Y, Z = layer.forward()
    Z[3, :], Z[4, :] = -float("inf"), float("inf")     # (0 times infinity beside the diagonal: put the pre-activations in by hand)
    dX, dW, db = layer.backward(Z, "X")
    assert not dX[3].any()
    assert lib.torch.equal(dX[4], layer.dY[4])
    layer.X.zero_()
    layer.b = layer.W[0].clone().zero_()
    layer.b[7], layer.b[8] = -float("inf"), float("inf")
    Y, Z = layer.forward()
    assert not Y[:, :8].any() and lib.torch.isinf(Y[:, 8]).all() and (Z[:, 7] == -float("inf")).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,act", [((600, 1000, 1024), "gelu"), ((8003, 128, 128), "silu"), ((3001, 256, 512), "relu"), ((6000, 128, 1240), "silu"),
                                       ((5000, 200, 200), "gelu")], ids=str)
def test_long_sums_of_fewer_rows(lib, shape, act, dtype):
    print(f"dense layer {shape} {dtype} {act}", flush=True)
    check_layer(Layer(lib, *shape, act, dtype))
    check_layer(Layer(lib, *shape, act, dtype, spread=(2, 3), scale=20.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(600, 1000, 1024), (8003, 128, 128)], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_long_sums_with_values_that_are_not_finite(lib, shape, value, dtype):
    torch = lib.torch
    rows, k_in, k_out = shape
    print(f"dense layer {shape} with {value} {dtype}", flush=True)
    layer = Layer(lib, *shape, "none", dtype)
    layer.X[rows - 1, 3], layer.dY[70, k_out - 1] = value, value
    Y, _ = layer.forward()
    dX, dW, db = layer.backward(None)
    for got, row in ((Y, rows - 1), (dX, 70)):
        keep = torch.arange(rows, device="cuda") != row
        assert torch.isfinite(got[keep]).all() and not torch.isfinite(got[row]).any()
    assert not torch.isfinite(dW[3]).any() and not torch.isfinite(dW[:, -1]).any()
    keep = torch.arange(k_in, device="cuda") != 3
    assert torch.isfinite(dW[keep][:, :-1]).all() and torch.isfinite(db[:-1]).all() and not torch.isfinite(db[-1])


@pytest.mark.parametrize("k_in,k_out", [(64, 1024), (64, 64), (128, 192), (1000, 72)])
@pytest.mark.parametrize("rows", [800, 22_985, MANY])
def test_weight_gradients_of_bfloat16_rows_are_those_of_fp32(lib, rows, k_in, k_out):
    """dW, db, W2 and b2 are fp32 whatever the rows are.  Values of one sign, so that no sum is small beside its terms: each relative to its own
    size, (64 + sqrt(n)) u for sums whose roundings are independent, 32 u (1 + |z|) + 256 u for what enters them; on average 64 u = 2^-18, which weights
    cut to two bfloat16 numbers would pass by half."""
    torch = lib.torch
    print(f"dense layer weight gradients {rows} {k_in} {k_out}", flush=True)
    layer = Layer(lib, rows, k_in, k_out, "silu", "bf16", bias=False, residual=False)
    for t in (layer.X, layer.dY, layer.HX, layer.W):
        t.abs_()
    # weights that lose 1.5 2^-18 of themselves with their third bfloat16 number
    layer.W.copy_((layer.W.bfloat16().float().clamp(min=2.0 ** -8)) * (1 + 2.0 ** -9 + 2.0 ** -18 + 2.0 ** -19))
    Z = (torch.rand(rows, k_out, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") - 0.5).to(torch.bfloat16)   # act'' > 0
    z, X, W, dY, HX = (t.double() for t in (Z, layer.X, layer.W, layer.dY, layer.HX))
    p = torch.sigmoid(z)
    first, second = p + z * p * (1 - p), p * (1 - p) * (2 + z * (1 - 2 * p))
    G, S = dY * first, (HX @ W) * dY * second
    _, dW, db = layer.backward(Z)
    _, _, W2, b2 = layer.double_backward(Z)
    bound = (64 + rows ** 0.5 + 32 * 1.5 + 256 + k_in ** 0.5) * 2.0 ** -24
    mean = lambda got, want: ((got.double() - want) / want).mean().abs().item()  # noqa: E731
    for name, got, want in (("dW", dW, X.T.contiguous() @ G), ("db", db, G.sum(0)), ("W2", W2, X.T.contiguous() @ S + HX.T.contiguous() @ G), ("b2", b2, S.sum(0))):
        assert ((got.double() - want) / want).abs().max() <= bound, name
        assert mean(got, want) <= 2.0 ** -18, name
