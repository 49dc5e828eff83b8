"""The orthogonalised update (include/ou.h) through the C ABI against the fp64 oracle.

Tolerances.  Momentum and weight are a few operations an element: 4 roundings of half a last bit, of numbers no larger than the sum of the
terms' sizes.  The iteration is held as a whole matrix: a product's sums of n terms are off by about sqrt(n) last bits u (2^-23: a
matrix instruction may cut, fp64 2^-52), a step by 8 of them (four products' worth, each rounded twice) times the size of
what it makes, |X| <= 1.3 sqrt(m) in the Frobenius norm once the first step is done, and every step makes the errors before it at most 4 times as large (the
slope of a x + b x^3 + c x^5 and its difference quotients on 0..1.3 are below 4): 8 u sqrt(n) sqrt(m) (1 + 4 + .. + 4^(steps - 1)) + u 4^steps.
An update of bfloat16 is rounded once more, 2^-8 of each element.  fp64 results meet an oracle of the same precision, which computes them as
they are defined (not by singular values, whose decomposition has errors of its own) and is off by as much: twice the bound.
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


NAN = float("nan")


def unit(t):
    import torch
    return 2.0 ** -52 if t == torch.float64 else 2.0 ** -23


class List:
    def __init__(self, ou, shapes, types, seed=3, momentum=True, weight=True, update=True, scale=None, skew=0, **config):
        import torch
        self.ou, self.shapes = ou, shapes
        self.types = [getattr(torch, t) for t in (types if isinstance(types, (list, tuple)) else [types] * len(shapes))]
        wide = [torch.float64 if t == torch.float64 else torch.float32 for t in self.types]
        g = torch.Generator(device="cuda").manual_seed(seed)

        def new(shape, t, scale):
            n = int(np.prod(shape))
            x = torch.randn(n + skew, generator=g, device="cuda", dtype=torch.float64).mul_(scale).to(t)
            return x[skew:].view(shape)
        self.grad = [new(s, t, 1e-2) for s, t in zip(shapes, self.types)]
        self.momentum = [new(s, t, 3e-2) for s, t in zip(shapes, wide)] if momentum else None
        self.weight = [new(s, t, 0.2) for s, t in zip(shapes, wide)] if weight else None
        self.update = [new(s, t, NAN) for s, t in zip(shapes, self.types)] if update else None
        self.scale = scale or [1.0 + i for i in range(len(shapes))]
        self.config = dict(rate=0.02, decay=0.1, steps=5)
        self.config.update(config)
        self.cfg = ou.make_config(**self.config)
        self.remake()

    def remake(self):
        import torch
        self.tensors = self.ou.make_tensors(self.grad, self.momentum, self.weight, self.update, self.scale)
        self.nbytes = self.ou.ou_workspace_bytes(self.cfg, self.tensors)
        self.ws = torch.full((self.nbytes,), 255, dtype=torch.uint8, device="cuda")

    def step(self, stream=None):
        self.ou.ou_step(self.cfg, self.tensors, self.ws, self.nbytes, stream)

    def host(self):
        f64 = lambda x: x.double().cpu().numpy().reshape((-1,) + tuple(x.shape[-2:]))  # noqa: E731
        return [[None if x is None else f64(x[i]) for x in (self.grad, self.momentum, self.weight, self.update)] for i in range(len(self.shapes))]

    def check(self, before, form=None):
        import torch
        c = self.config
        mu, steps, nesterov = c.get("momentum", 0.95), c["steps"], c.get("nesterov", True)
        worst = 0.0
        for i, ((G, M, W, _), (_, M1, W1, X1)) in enumerate(zip(before, self.host())):
            if G.shape[0] == 0:
                continue
            u = unit(self.types[i])
            bf16 = self.types[i] == torch.bfloat16
            wM, wX, wW = oo.step(G, M, W, mu=mu, nesterov=nesterov, steps=steps, rate=c["rate"], decay=c["decay"], scale=self.scale[i],
                                 form=form or (oo.iterate if u < 2.0 ** -50 else oo.orthogonalise),
                                 coefficients=c.get("coefficients", oo.COEFFICIENTS))
            if M is not None:
                assert (np.abs(M1 - wM) <= 2 * u * (np.abs(mu * M) + np.abs(G))).all(), i
            m, n = min(G.shape[1:]), max(G.shape[1:])
            allowed = 8 * u * np.sqrt(n) * np.sqrt(m) * sum(4.0 ** k for k in range(steps)) + 4 * u * 4.0 ** steps
            allowed *= 2 if u < 2.0 ** -50 else 1
            for k in range(G.shape[0]):
                if X1 is not None:
                    off = np.sqrt(((X1[k] - wX[k]) ** 2).sum())
                    here = allowed + (2.0 ** -8 * np.sqrt((wX[k] ** 2).sum()) if bf16 else 0)
                    assert off <= here, (i, k, off / here)
                    worst = max(worst, off / here)
                if W1 is not None:
                    off = np.sqrt(((W1[k] - wW[k]) ** 2).sum())
                    here = abs(c["rate"] * self.scale[i]) * allowed + 4 * u * np.sqrt((W[k] ** 2).sum())
                    assert off <= here, (i, k, off / here)
        return worst


SHAPES = [(1, 1, 1), (3, 1, 7), (2, 7, 1), (1, 8, 64), (2, 64, 64), (1, 64, 8), (1, 64, 300), (1, 300, 64), (2, 65, 65), (1, 63, 129), (1, 128, 128),
          (1, 129, 128), (1, 128, 127), (2, 40, 200), (1, 200, 200), (1, 260, 131)]


@pytest.mark.parametrize("dtype", ["float32", "float64", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_against_the_oracle(ou, shape, dtype, steps):
    import torch
    print(f"update {shape} {dtype} {steps}", flush=True)
    x = List(ou, [shape], dtype, steps=steps)
    before = x.host()
    x.step()
    torch.cuda.synchronize()
    print("of the allowed error:", x.check(before), flush=True)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_large_matrices(ou, dtype):
    import torch
    x = List(ou, [(1, 513, 1030), (1, 700, 700), (1, 1030, 257)], dtype)
    before = x.host()
    x.step()
    torch.cuda.synchronize()
    print("of the allowed error:", x.check(before, oo.iterate), flush=True)


@pytest.mark.parametrize("number", [1, 5, 40, 120])
def test_lists(ou, number):
    """Lists of every length and of all types at once, empty batches among them, addresses at any element."""
    import torch
    shapes = [((i * 7) % 4, 1 + (i * 29) % 90, 1 + (i * 53) % 140) for i in range(number)]
    types = [("float32", "bfloat16", "float64")[i % 3] for i in range(number)]
    for skew in (0, 1):
        print(f"update list {number} skew {skew}", flush=True)
        x = List(ou, shapes, types, skew=skew)
        before = x.host()
        x.step()
        torch.cuda.synchronize()
        x.check(before)


@pytest.mark.parametrize("options", [dict(momentum=False), dict(weight=False), dict(update=False), dict(momentum=False, update=False)], ids=str)
def test_what_is_left_out(ou, options):
    import torch
    x = List(ou, [(3, 20, 30), (1, 70, 20), (2, 128, 128)], ["float32", "bfloat16", "float64"], **options)
    before = x.host()
    x.step()
    torch.cuda.synchronize()
    x.check(before)


def test_options(ou):
    """Another momentum, without Nesterov's step, no decay, other coefficients and numbers of steps."""
    import torch
    for kw in (dict(nesterov=False), dict(decay=0.0), dict(rate=-0.5), dict(coefficients=(1.5, -0.5, 0.0), steps=7), dict(coefficients=(2.0, -1.5, 0.5), steps=3),
               dict(steps=2, rate=0.0)):
        x = List(ou, [(2, 50, 70), (1, 150, 140)], ["float32", "float64"], **kw)
        before = x.host()
        x.step()
        torch.cuda.synchronize()
        x.check(before)


def test_it_orthogonalises(ou):
    """Singular values that are not much smaller than the largest come near 1, whatever the size of the gradient."""
    import torch
    for scale in (1e-30, 1.0, 1e30):
        x = List(ou, [(2, 96, 160), (1, 200, 128)], "float32", momentum=False, weight=False)
        for g in x.grad:
            g.mul_(scale * 1e2)
        if scale < 1e-20:     # far below eps nothing is left to normalise: with a small one there is
            x.cfg = ou.make_config(rate=0.0, eps=1e-40)
        x.step()
        for t in x.update:
            s = torch.linalg.svdvals(t.double())
            assert 0.5 < s.min().item() and s.max().item() < 1.35, scale


def test_gradients_far_below_eps(ou):
    """U / (|U| + eps) is then about U / eps, and the iteration a^5 of it: nothing is lost to small numbers on the way."""
    import torch
    for size in (1e-12, 1e-20, 1e-30):
        x = List(ou, [(1, 48, 64), (1, 160, 140)], "float32", momentum=False, weight=False, scale=[1.0, 1.0])
        for g in x.grad:
            g.mul_(size * 1e2)
        x.step()
        for g, t in zip(x.grad, x.update):
            norm = g.double().square().sum().sqrt().item()
            want = g.double() / (norm + 1e-7) * 3.4445 ** 5
            top = 3.4445 ** 5 * norm / 1e-7
            # (each step multiplies by a + b s^2 + ..: relative to a that is |b| / a s^2 < 1.4 s^2, s the largest value before the last step)
            assert ((t.double() - want).abs() <= want.abs() * (30 * 2.0 ** -23 + 5 * 1.4 * top ** 2) + 2.0 ** -149).all(), size


def test_zero_and_not_finite_matrices(ou):
    import torch
    for steps in (0, 5):
        x = List(ou, [(5, 40, 72), (2, 150, 130)], "float32", momentum=False, steps=steps)
        x.grad[0][1] = 0.0
        x.grad[0][3, 4, 5] = float("inf")
        x.grad[1][0, 149, 129] = NAN
        before = x.host()
        weights = [w.clone() for w in x.weight]
        x.step()
        assert not x.update[0][1].any() and torch.equal(x.weight[0][1], weights[0][1] * torch.tensor(1 - 0.02 * 0.1, dtype=torch.float32, device="cuda"))
        if steps:
            assert x.update[0][3].isnan().all() and x.weight[0][3].isnan().all()
        else:
            assert x.update[0][3].isnan().sum() == 1 and x.update[0][3, 4, 5].isnan() and (x.update[0][3] == 0).sum() == 40 * 72 - 1
        assert x.update[1][0].isnan().all()
        x.shapes = [(3, 40, 72), (1, 150, 130)]
        keep = [torch.tensor([0, 2, 4], device="cuda"), torch.tensor([1], device="cuda")]
        for name in ("grad", "weight", "update"):
            setattr(x, name, [t[k] for t, k in zip(getattr(x, name), keep)])
        x.check([[None if v is None else v[k.cpu().numpy()] for v in b] for b, k in zip(before, keep)])


def test_results_repeat(ou):
    import torch
    shapes = [(1, 8, 64), (4, 128, 128), (1, 300, 500), (1, 64, 1280)]
    a, b = List(ou, shapes, "float32"), List(ou, shapes, "float32")
    a.step()
    b.ws.zero_()
    b.step()
    for x, y in zip(a.momentum + a.weight + a.update, b.momentum + b.weight + b.update):
        assert torch.equal(x, y)
    # alone these sizes take the same kernels as in this list
    for i, s in enumerate(shapes):
        c = List(ou, shapes, "float32")
        c.shapes, c.scale = [s], [c.scale[i]]
        for name in ("grad", "momentum", "weight", "update"):
            setattr(c, name, [getattr(c, name)[i]])
        c.remake()
        c.step()
        assert torch.equal(c.update[0], a.update[i]) and torch.equal(c.weight[0], a.weight[i])


def test_graphs_and_streams(ou):
    """Two captured steps, each with its own workspace, replayed on changing gradients, with the program's own work between."""
    import torch
    made = []
    for shapes, dtype in (([(3, 128, 128), (1, 64, 300)], "float32"), ([(1, 200, 150), (2, 8, 64)], "bfloat16")):
        x, eager = List(ou, shapes, dtype), List(ou, shapes, dtype)
        x.step()
        eager.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.step()
        made.append((x, eager, graph))
    side = torch.cuda.Stream()
    for turn in range(3):
        for x, eager, graph in made:
            for g, h in zip(x.grad, eager.grad):
                g.copy_(torch.randn(g.shape, device="cuda"))
                h.copy_(g)
        torch.cuda.synchronize()
        for x, eager, graph in made:
            graph.replay()
        for x, eager, graph in made:
            eager.step(side)
        torch.cuda.synchronize()
        for x, eager, graph in made:
            for p, q in zip(x.momentum + x.weight + x.update, eager.momentum + eager.weight + eager.update):
                assert torch.equal(p, q)


def test_an_empty_list(ou):
    x = List(ou, [(0, 8, 8)], "float32")
    x.step()
    ou.ou_step(x.cfg, ou.make_tensors([], [], [], []), x.ws, x.nbytes)


LONG = [(1, 3, 4500), (1, 64, 2049), (1, 5000, 100), (3, 128, 4097), (2, 2500, 33), (1, 1, 65536), (1, 1, 1), (1, 65536, 2)]


@pytest.mark.parametrize("dtype", ["float32", "float64", "bfloat16"])
@pytest.mark.parametrize("shape", LONG, ids=lambda s: "x".join(map(str, s)))
def test_long_matrices(ou, shape, dtype):
    """One side far longer than the other: more than one piece of columns to a slice."""
    import torch
    print(f"update long {shape} {dtype}", flush=True)
    for skew in (0, 1):
        x = List(ou, [shape], dtype, skew=skew)
        before = x.host()
        x.step()
        torch.cuda.synchronize()
        x.check(before, oo.iterate)


def test_every_way_in_one_list(ou):
    """Sizes about the limits between the kernels, of all types, in one call."""
    import torch
    shapes = [(n, r, c) for n, r, c in ((2, 64, 64), (1, 64, 65), (3, 65, 64), (1, 128, 128), (2, 128, 129), (1, 129, 64), (1, 129, 129), (2, 257, 130), (0, 200, 200),
                                        (1, 2, 300), (5, 33, 31), (1, 192, 448))]
    for types in (["float32", "bfloat16"] * 6, ["float32", "float64", "bfloat16"] * 4):
        for skew in (0, 1):
            x = List(ou, shapes, types, skew=skew)
            before = x.host()
            x.step()
            torch.cuda.synchronize()
            x.check(before, oo.iterate)


def test_calls_at_the_same_time(ou):
    """Two lists on two streams, each with its own workspace."""
    import torch
    shapes = [(3, 200, 300), (2, 100, 90), (1, 40, 700)]
    want, a, b = List(ou, shapes, "float32"), List(ou, shapes, "float32"), List(ou, shapes, "float32")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for turn in range(3):
        want.step()
        for s, x in zip(streams, (a, b)):
            x.step(s)
    torch.cuda.synchronize()
    for x in (a, b):
        for p, q in zip(x.momentum + x.weight + x.update, want.momentum + want.weight + want.update):
            assert torch.equal(p, q)


@pytest.mark.parametrize("shape", [(131_073, 128, 128), (140_001, 64, 256), (33_001, 256, 260)], ids=lambda s: "x".join(map(str, s)))
def test_batches_past_32_bits(ou, shape):
    """More than 2^31 elements in a tensor: the first and the last matrices."""
    import torch
    count, rows, cols = shape
    g = torch.Generator(device="cuda").manual_seed(4)
    grad = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    ends = [0, 1, count - 2, count - 1]
    for i in ends:
        grad[i] = torch.randn(rows, cols, generator=g, device="cuda") * 1e-2
    update = torch.empty_like(grad)
    cfg = ou.make_config(0.02, steps=2)
    tensors = ou.make_tensors([grad], None, None, [update])
    nbytes = ou.ou_workspace_bytes(cfg, tensors)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    ou.ou_step(cfg, tensors, ws, nbytes)
    torch.cuda.synchronize()
    u = 2.0 ** -23
    for i in ends:
        want = oo.iterate(grad[i].double().cpu().numpy(), 2)
        allowed = 8 * u * np.sqrt(rows * cols) * 5 + 4 * u * 16 + 2.0 ** -8 * np.sqrt((want ** 2).sum())
        assert np.sqrt(((update[i].double().cpu().numpy() - want) ** 2).sum()) <= allowed, i
    assert not update[2:count - 2].any()
