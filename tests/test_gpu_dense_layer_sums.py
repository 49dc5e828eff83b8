"""Every result of the dense layer's backward passes (include/dl.h) relative to itself, whatever is left out of a call.

All terms of a sum have one sign here (X, W, dY, HX positive, pre-activations where act' and act'' are), so a result is as large as its terms and a lost term, a
wrong derivative or a result of another product shows however many rows there are.

Tolerance, u = 2^-24 (2^-53): n rows summed in any fixed order 64 u + sqrt(n) u (roundings of a chain of sums are independent, a part of 64 is counted in full), V
sqrt(k_in) u, act' and act'' 8 u of 0.1 to 1, so 80 u, the products of these a few u; the reference in fp64 as much again for SC_F64.  bfloat16 rows: results in them 2^-8
of the last rounding.  The mean of the errors: 64 u.
"""
import pytest

from test_gpu_dense_layer import MANY, Layer, lib  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu

A = 0.7978845608028654   # sqrt(2 / pi)


def derivatives(torch, act, z):
    """act' and act'' in fp64."""
    if act == "none":
        return torch.ones_like(z), torch.zeros_like(z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * (1 - p), p * (1 - p) * (2 + z * (1 - 2 * p))
    t = torch.tanh(A * (z + 0.044715 * z ** 3))
    u1, u2 = A * (1 + 3 * 0.044715 * z ** 2), 6 * A * 0.044715 * z
    d = 1 - t * t
    return 0.5 * (1 + t) + 0.5 * z * d * u1, d * u1 + 0.5 * z * (d * u2 - 2 * t * d * u1 * u1)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu", "none"])
@pytest.mark.parametrize("rows,k_in,k_out", [(70, 64, 64), (800, 64, 1024), (800, 300, 96), (22_985, 64, 64), (22_985, 64, 1024), (22_985, 1000, 72), (22_985, 65, 67),
                                             (MANY, 64, 64), (MANY, 20, 132), (MANY, 128, 192), (MANY, 132, 64), (MANY, 64, 1), (6000, 1280, 1280)])
def test_each_result_relative_to_itself(lib, rows, k_in, k_out, act, dtype):
    torch = lib.torch
    print(f"dense layer sums {rows} {k_in} {k_out} {act} {dtype}", flush=True)
    layer = Layer(lib, rows, k_in, k_out, act, dtype, bias=False, residual=False)
    for t in (layer.X, layer.dY, layer.HX, layer.W):
        t.abs_().clamp_(min=2.0 ** -6)
    Z = (torch.rand(rows, k_out, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") - 0.5).to(layer.X.dtype)
    X, W, dY, HX = (t.double() for t in (layer.X, layer.W, layer.dY, layer.HX))
    Wt, Xt, Ht = W.t().contiguous(), X.t().contiguous(), HX.t().contiguous()
    first, second = derivatives(torch, act, Z.double())
    V = torch.matmul(HX, W)
    G, S = dY * first, V * dY * second
    u = 2.0 ** -53 if dtype == "f64" else 2.0 ** -24
    rX, rW, rb = torch.matmul(G, Wt), torch.matmul(Xt, G), G.sum(0)
    rY, r2, rV, rc = V * first, torch.matmul(S, Wt), torch.matmul(Xt, S) + torch.matmul(Ht, G), S.sum(0)

    def compare(name, got, ref, long, in_rows):
        bound = (64 + long ** 0.5 + k_in ** 0.5 + 160 + 16) * u * (2 if dtype == "f64" else 1)
        assert bound < 1e-4
        if not ref.any():
            assert not got.any(), name
            return
        off = (got.double() - ref) / ref
        rounding = 2.0 ** -8 if dtype == "bf16" and in_rows else 0.0
        assert off.abs().max() <= bound + rounding, f"{name}: {off.abs().max().item() / u:.0f} u"
        if not rounding:
            assert off.mean().abs() <= 64 * u, f"{name}: on average {off.mean().item() / u:.0f} u"

    given = None if act == "none" else Z
    for wanted in ("XWb", "X", "W", "b", "XW", "Wb", "Xb"):
        dX, dW, db = layer.backward(given, wanted)
        ddY, X2, W2, b2 = layer.double_backward(given, wanted)
        for name, got, ref, long, in_rows in (("dX", dX, rX, k_out, True), ("dW", dW, rW, rows, False), ("db", db, rb, rows, False), ("ddY", ddY, rY, k_in, True),
                                              ("X2", X2, r2, k_out, True), ("W2", W2, rV, rows, False), ("b2", b2, rc, rows, False)):
            if got is not None:
                compare(f"{name} of a call for {wanted}", got, ref, long, in_rows)
