"""How exact the orthogonalised update's products are: its results and those of the same formulas in plain fp32, both against fp64.

Tolerance.  An fp32 value enters a product as two fp16 parts, off by at most half a last bit of 22, 2^-23, where fp32 arithmetic takes it as it is; the product of the two second
parts, at most 2^-22 of the whole, is left out; so a product is off by up to 2^-21, which the rounding of an fp32 product (2^-24) is not by a factor of eight.  The sums are
fp32 on both sides, and the steps after it carry both errors alike.  So the kernels may be off by eight times what the formulas in fp32 are, both as whole matrices
(Frobenius norm); an fp32 result that happens to come out better than half a last bit of a step counts as that, 2^-24 of the result a step.  A product with a single part, off by 2^-12, is beyond it by a
factor of hundreds.
"""
import numpy as np
import pytest

from oracle import orthogonalised_update as oo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ou():
    import torch
    assert torch.cuda.is_available()
    from paper_2504_10700_amd import ou_binding
    return ou_binding


def in_fp32(U, steps, coefficients, eps):
    """The formulas in plain fp32 (the norm in fp64, as the library has it)."""
    a, b, c = (np.float32(v) for v in coefficients)
    X = (U / (np.sqrt((U ** 2).sum()) + eps)).astype(np.float32)
    turned = X.shape[0] > X.shape[1]
    X = X.T if turned else X
    for _ in range(steps):
        S = X @ X.T
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.T if turned else X


def compare(ou, shapes, steps, coefficients, eps=1e-7, make=None, dtype="float32"):
    """One call on a list of batches [count][rows][cols] of normal numbers, or of make(generator, shape); returns the worst ratio of the errors."""
    import torch
    g = np.random.default_rng(11)
    values = [(make or (lambda rng, s: rng.normal(size=s)))(g, s) for s in shapes]
    grad = [torch.tensor(v).to(getattr(torch, dtype)).cuda() for v in values]
    weight = [torch.zeros(s, device="cuda") for s in shapes]                     # rate -1, scale 1: the update itself, in fp32
    cfg = ou.make_config(rate=-1.0, steps=steps, coefficients=coefficients, eps=eps)
    tensors = ou.make_tensors(grad, None, weight, None)
    nbytes = ou.ou_workspace_bytes(cfg, tensors)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    ou.ou_step(cfg, tensors, ws, nbytes)
    torch.cuda.synchronize()
    worst = 0.0
    for gr, w in zip(grad, weight):
        for U, X in zip(gr.double().cpu().numpy(), w.double().cpu().numpy()):
            want = oo.iterate(U, steps, eps, coefficients)
            norm = lambda x: np.sqrt((x ** 2).sum())  # noqa: E731
            plain = max(norm(in_fp32(U, steps, coefficients, eps) - want), steps * 2.0 ** -24 * norm(want))
            off = norm(X - want)
            worst = max(worst, off / plain)
            assert off <= 8 * plain, (U.shape, off / plain, off / norm(want))
    return worst


WAYS = [(2, 64, 64), (1, 33, 50), (2, 128, 128), (1, 100, 70), (1, 64, 1280), (1, 700, 40), (3, 128, 300), (1, 300, 90), (1, 200, 300), (1, 257, 131)]
GROWING = [((8.28, -23.6, 17.3), 2), ((8.0, -10.0, 4.0), 2), ((30.0, -40.0, 20.0), 1), ((1000.0, -1000.0, 0.0), 1), ((0.0, 4000.0, -4000.0), 1), ((0.0, 200.0, -200.0), 1),
           ((0.0, 1000.0, 0.0), 1), ((3.0, 0.0, 0.0), 6)]


@pytest.mark.parametrize("coefficients,steps", GROWING, ids=str)
def test_growing_coefficients(ou, coefficients, steps):
    """Bounds that grow by up to 1024 over the steps: every kernel, each alone and all in one list."""
    for shapes in [[s] for s in WAYS] + [WAYS]:
        print(f"update growing {coefficients} {steps} {shapes}", flush=True)
        print("times the error of fp32:", compare(ou, shapes, steps, coefficients), flush=True)


@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("size", [1e-320, 1e-300, 1e-200, 1e-150, 1e-140, 1e100, 1e140, 1e150, 1e200, 1e305])
def test_fp64_gradients_of_every_size(ou, size, steps):
    """The squares of such elements are not all numbers, but U / (|U| + eps) is one.  The gradient is a power of two times normal numbers (below the normal numbers: whatever is left of
    them), so a gradient of ordinary size and an eps that goes with it have the same result but for roundings.  X has norm 1 and is off by four last bits u (2^-52: a root, a sum, a quotient and
    two products, half a bit each, here and in the oracle); the products of a step by 8 u sqrt(n m) as the other tests of the update have it; a step makes what is before it at most 4 times as
    large; here and in the oracle, so once more as much: less than 4 u (1 + 8 sqrt(n m) steps) 4^steps."""
    import torch
    g = torch.Generator().manual_seed(5)
    up = 2.0 ** np.floor(np.log2(size))
    for shape in ((2, 40, 70), (1, 130, 100)):
        small = torch.randn(shape, generator=g, dtype=torch.float64)
        grad = (small * up).cuda()
        reference = grad.cpu().numpy() / up
        for eps in (up * 2.0 ** -20, up):
            if eps == 0 or not np.isfinite(eps):
                continue
            update = torch.full(shape, float("nan"), dtype=torch.float64, device="cuda")
            cfg = ou.make_config(rate=0.0, steps=steps, eps=eps)
            tensors = ou.make_tensors([grad], None, None, [update])
            nbytes = ou.ou_workspace_bytes(cfg, tensors)
            ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
            ou.ou_step(cfg, tensors, ws, nbytes)
            for U, X in zip(reference, update.cpu().numpy()):
                want = oo.iterate(U, steps, eps / up)
                m = min(U.shape)
                allowed = 2.0 ** -50 * (1 + 8 * np.sqrt(max(U.shape) * m) * steps) * 4.0 ** steps
                assert np.sqrt(((X - want) ** 2).sum()) <= allowed, (size, eps, steps, shape)


@pytest.mark.parametrize("dtype", ["float32", "float64", "bfloat16"])
def test_zeros_stay_zero_for_every_eps(ou, dtype):
    """Also where 1 / eps is beyond the largest number; and a mixed list keeps them apart."""
    import torch
    t = getattr(torch, dtype)
    for shape in ((2, 40, 60), (2, 100, 128), (2, 64, 300), (2, 130, 140)):
        for steps in (0, 1, 5):
            grad = torch.zeros(shape, dtype=t, device="cuda")
            grad[1] = torch.eye(shape[1], shape[2], dtype=t, device="cuda")
            update = torch.full(shape, float("nan"), dtype=t, device="cuda")
            cfg = ou.make_config(rate=0.0, steps=steps, eps=5e-324)
            tensors = ou.make_tensors([grad], None, None, [update])
            nbytes = ou.ou_workspace_bytes(cfg, tensors)
            ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
            ou.ou_step(cfg, tensors, ws, nbytes)
            assert not update[0].any(), (shape, steps)
            assert torch.isfinite(update[1]).all() and (update[1].diagonal() > 0).all(), (shape, steps)


SMALL_LINEAR = [((0.0, 1.0, 0.0), 3), ((0.0, 0.1, 0.0), 3), ((0.001, 1.0, 0.0), 5), ((0.0, 2.0, -1.0), 2), ((0.0, 0.0, 1.0), 2)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("coefficients,steps", SMALL_LINEAR, ids=str)
def test_coefficients_without_a_linear_term(ou, coefficients, steps, dtype):
    """Singular values become cubes of small numbers, far below the bound of the largest there can be."""
    for shapes in [[s] for s in WAYS] + [WAYS]:
        print(f"update without a linear term {coefficients} {steps} {dtype} {shapes}", flush=True)
        print("times the error of fp32:", compare(ou, shapes, steps, coefficients, dtype=dtype), flush=True)


@pytest.mark.parametrize("coefficients,steps", [((0.05, 1.5, 1.0), 2), ((0.05, 1.5, 1.0), 3), ((0.03, 1.5, 1.0), 2), ((1.0, 30.0, -30.0), 1), ((1.0, 34.0, -34.0), 1), ((0.1, -0.1, 0.1), 9), ((0.01, 0.01, 0.0), 4)], ids=str)
def test_coefficients_about_the_limit_of_the_parts(ou, coefficients, steps):
    """On both sides of the ratio to which parts serve, and bounds that shrink.  (With the second, 2.55 becomes 133 and then more than OU_MAX_GROWTH: refused.)"""
    if (coefficients, steps) == ((0.05, 1.5, 1.0), 3):
        with pytest.raises(ou.ScError):
            compare(ou, WAYS, steps, coefficients)
        return
    for scale in (1.0, 1e-9):     # the second far below eps
        make = lambda rng, s: rng.normal(size=s) * scale  # noqa: E731
        for shapes in [[s] for s in WAYS] + [WAYS]:
            print(f"update about the limit {coefficients} {steps} {scale} {shapes}", flush=True)
            print("times the error of fp32:", compare(ou, shapes, steps, coefficients, make=make), flush=True)


def test_options_on_fp32_instructions(ou):
    """Momentum, weights, what is left out and addresses at any element there too."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(9)
    coefficients = (0.0, 2.0, -1.0)
    for skew in (0, 1):
        for nesterov in (True, False):
            new = lambda s, t=torch.float32: torch.randn(int(np.prod(s)) + skew, generator=g, device="cuda").to(t)[skew:].view(s)  # noqa: E731
            shapes = [(2, 64, 64), (1, 130, 260), (3, 90, 20), (0, 7, 7)]
            types = [torch.float32, torch.bfloat16, torch.float32, torch.bfloat16]
            grad, momentum, weight, update = [new(s, t) for s, t in zip(shapes, types)], [new(s) for s in shapes], [new(s) for s in shapes], [new(s, t) for s, t in zip(shapes, types)]
            f64 = lambda x: x.double().cpu().numpy()  # noqa: E731
            before = [tuple(f64(x[i]) for x in (grad, momentum, weight)) for i in range(3)]
            cfg = ou.make_config(rate=0.5, decay=0.1, steps=2, coefficients=coefficients, nesterov=nesterov)
            tensors = ou.make_tensors(grad, momentum, weight, update, scale=[1.0, 2.0, 3.0, 4.0])
            nbytes = ou.ou_workspace_bytes(cfg, tensors)
            ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
            ou.ou_step(cfg, tensors, ws, nbytes)
            for i, (G, M, W) in enumerate(before):
                wM, wX, wW = oo.step(G, M, W, nesterov=nesterov, steps=2, rate=0.5, decay=0.1, scale=1.0 + i, coefficients=coefficients, form=oo.iterate)
                assert (np.abs(f64(momentum[i]) - wM) <= 2 * 2.0 ** -23 * (np.abs(0.95 * M) + np.abs(G))).all(), i
                U = G + 0.95 * wM if nesterov else wM
                for k in range(G.shape[0]):
                    norm = lambda x: np.sqrt((x ** 2).sum())  # noqa: E731
                    # U is rounded three times (2^-23 each, of terms no larger than |G| + |M|), which two steps make 25 times as much (cubes: three times a step, and a third for X itself)
                    plain = norm(in_fp32(U[k], 2, coefficients, 1e-7) - wX[k]) + 2.0 ** -23 * norm(wX[k])
                    allowed = 8 * plain + 25 * 3 * 2.0 ** -23 * norm(wX[k]) * norm(np.abs(G[k]) + np.abs(M[k])) / norm(U[k])
                    assert norm(f64(update[i])[k] - wX[k]) <= allowed + (2.0 ** -8 * norm(wX[k]) if types[i] == torch.bfloat16 else 0), (i, k)
                    assert norm(f64(weight[i])[k] - wW[k]) <= 0.5 * (1 + i) * allowed + 4 * 2.0 ** -23 * norm(W[k]), (i, k)


LARGER = [(1, 513, 1030), (1, 700, 700), (1, 1030, 257), (1, 64, 8192), (1, 128, 20_000), (1, 260, 9000)]
HELD = [((3.4445, -4.7750, 2.0315), 1), ((3.4445, -4.7750, 2.0315), 5), ((0.1, 4.0, -3.0), 1), ((0.1, 2.0, 1.0), 2), ((1.5, -0.5, 0.0), 8), ((2.0, -1.5, 0.5), 4)]


def decaying(rng, s):
    """Singular values from 1 down to 1e-6."""
    count, rows, cols = s
    m = min(rows, cols)
    q = lambda n: np.linalg.qr(rng.normal(size=(n, m)))[0]  # noqa: E731
    return np.stack([(q(rows) * np.logspace(0, -6, m)) @ q(cols).T for _ in range(count)])


def one_direction(rng, s):
    """Nearly of rank one: a large S off the diagonal, sums of one sign."""
    count, rows, cols = s
    return rng.uniform(0.5, 1.5, (count, rows, 1)) * rng.uniform(0.5, 1.5, (count, 1, cols)) + 1e-3 * rng.normal(size=s)


@pytest.mark.parametrize("make", [None, decaying, one_direction], ids=["normal", "decaying", "one_direction"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("coefficients,steps", HELD, ids=str)
def test_products_as_exact_as_in_fp32(ou, coefficients, steps, dtype, make):
    """The usual coefficients, and ones that leave most of a result to the products: a part that is lost on the way shows here."""
    for shapes in [[s] for s in WAYS + (LARGER if make is None else [])] + [WAYS]:
        print(f"update exactness {coefficients} {steps} {dtype} {shapes}", flush=True)
        print("times the error of fp32:", compare(ou, shapes, steps, coefficients, make=make, dtype=dtype), flush=True)


@pytest.mark.parametrize("shape", [(1, 64, 64), (1, 128, 100), (1, 100, 600), (1, 256, 384)], ids=lambda s: "x".join(map(str, s)))
def test_rows_far_smaller_than_the_others(ou, shape):
    """A row i of a step's result is a X_i + P_i X.  Elements of P are off by up to 2^-38 (|b| + |c| 1.2^2) 1.2^2, 1.2 the largest a singular value can be, and twice that as S is too; so a small row
    by as much times sqrt(m) |X| beside eight times what fp32 does to it; what is off before a step is at most 4 times as much after it."""
    import torch
    a, b, c = oo.COEFFICIENTS
    steps, m = 5, min(shape[1:])
    for size in (1e-4, 1e-6, 1e-8):
        U = np.random.default_rng(2).normal(size=shape)
        U[0, 1::7] *= size
        grad = torch.tensor(U).float().cuda()
        update = torch.zeros(shape, device="cuda")
        cfg = ou.make_config(rate=0.0, steps=steps)
        tensors = ou.make_tensors([grad], None, None, [update])
        nbytes = ou.ou_workspace_bytes(cfg, tensors)
        ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
        ou.ou_step(cfg, tensors, ws, nbytes)
        U = grad[0].double().cpu().numpy()
        want, plain = oo.iterate(U, steps), in_fp32(U, steps, oo.COEFFICIENTS, 1e-7)
        norm = lambda x: np.sqrt((x[1::7] ** 2).sum(1))  # noqa: E731
        off, there = norm(update[0].double().cpu().numpy() - want), norm(want)
        worst = np.maximum(norm(plain - want).max(), steps * 2.0 ** -24 * there.max())
        beside = 2.0 ** -38 * 3 * (abs(b) + abs(c) * 1.44) * 1.44 * np.sqrt(m) * 1.2 * sum(4.0 ** k for k in range(steps))
        print(f"rows of {size}: relative {(off / there).max():.2e}, in fp32 {(norm(plain - want) / there).max():.2e}", flush=True)
        assert (off <= 8 * worst + beside).all(), (size, off.max(), worst, beside)
