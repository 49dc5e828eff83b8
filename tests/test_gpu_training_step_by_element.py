"""The training example with the self connection (gp.h) and the orthogonalised update (ou.h) in it: gradients of the whole chain against differences of
its loss, the matrices' step against the oracle, and the products and the update together in a captured graph.

Tolerances.  Differences: as in test_gpu_training_step.py, central ones of step h = 1e-5 in fp64, relative error of h^2 and of u / h.  The update: the bound of
test_gpu_orthogonalised_update.py, 8 u sqrt(n) sqrt(m) (1 + 4 + .. + 4^(steps - 1)) + 4 u 4^steps in the Frobenius norm, times the rate and the scale, and
4 u of the weight; u = 2^-23 (a matrix instruction may cut).
"""
import numpy as np
import pytest

from oracle import orthogonalised_update as oo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ts():
    import torch
    assert torch.cuda.is_available()
    from paper_2504_10700_amd import training_step
    return training_step


@pytest.mark.parametrize("atoms", [40, 80])      # without and with a grouping
def test_gradients_against_differences(ts, atoms):
    import torch
    model = ts.Model(atoms, 5, 8, elements=5, l_Y=1, dtype=ts.sc.SC_F64, self_connection=True)
    loss = model.loss().item()
    model.backward()
    gradients = [g.clone() for g in model.gradients]
    assert any(p is model.W_own for p in model.parameters) and model.dW_own.any()
    generator = torch.Generator(device="cuda").manual_seed(3)
    h = 1e-5
    for p, g in zip(model.parameters, gradients):
        direction = torch.randn(p.shape, generator=generator, device="cuda", dtype=p.dtype)
        values = []
        saved = p.clone()
        for s in (h, -h):
            p.copy_(saved + s * direction)
            values.append(model.loss().item())
        p.copy_(saved)
        slope, want = (values[0] - values[1]) / (2 * h), (g * direction).sum().item()
        scale = (g.abs() * direction.abs()).sum().item()
        print(tuple(p.shape), slope, want, flush=True)
        assert abs(slope - want) <= 1e-6 * scale + 1e-9 * (1 + abs(loss))


@pytest.mark.parametrize("connected", [False, True])
def test_steps_are_those_of_the_oracle(ts, connected):
    """Each parameter takes its own step, once, from the clipped gradients."""
    import torch
    model = ts.Model(500, 8, 64, max_norm=1.0, self_connection=connected, orthogonalised=True)
    matrices = [x.W for x in model.radial] + [model.readout[0].W] + ([model.W_own] if connected else [])
    momentum = {id(w): np.zeros(tuple(w.shape)) for w in matrices}
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    u = 2.0 ** -23
    for turn in range(3):
        before = [f64(p) for p in model.parameters]
        loss = model.step()
        assert torch.isfinite(loss)
        for p, g, old in zip(model.parameters, model.gradients, before):
            new, g = f64(p), f64(g)
            if id(p) not in momentum:
                assert (abs(new - (old - model.learning_rate * g)) <= 2 * u * (abs(old) + abs(model.learning_rate * g))).all()
                continue
            shape = (-1,) + p.shape[-2:]
            scale = max(1.0, p.shape[-1] / p.shape[-2]) ** 0.5
            M, _, W = oo.step(g.reshape(shape), momentum[id(p)].reshape(shape), old.reshape(shape), mu=0.95, nesterov=True, steps=5, rate=1e-3, decay=0.0,
                              scale=scale, form=oo.iterate, coefficients=oo.COEFFICIENTS)
            m, n = min(p.shape[-2:]), max(p.shape[-2:])
            allowed = 1e-3 * scale * (8 * u * np.sqrt(n * m) * sum(4.0 ** k for k in range(5)) + 4 * u * 4.0 ** 5)
            off = np.sqrt(((new.reshape(shape) - W) ** 2).sum(axis=(1, 2)))
            assert (off <= allowed + 4 * u * np.sqrt((W ** 2).sum(axis=(1, 2)))).all()
            absent = ~g.reshape(shape).any(axis=(1, 2)) & ~momentum[id(p)].reshape(shape).any(axis=(1, 2))
            assert (new.reshape(shape)[absent] == old.reshape(shape)[absent]).all()      # elements that no atom has
            # the device's own momentum, within a rounding of the oracle's, is what the next turn starts from
            own = f64(model.momentum[[w is p for w in matrices].index(True)])
            assert (abs(own.reshape(shape) - M) <= 4 * u * (abs(momentum[id(p)].reshape(shape)) + abs(g.reshape(shape)))).all()
            momentum[id(p)] = own


def test_products_and_update_in_one_graph(ts):
    """Grouping, both passes of the products and the update of their weights, captured once and replayed on other batches: as the same calls give them eagerly."""
    import torch
    gp, ou = ts.gp, ts.ou
    n, elements, k_in, k_out = 700, 6, 64, 96
    cfg, update = gp.make_config(elements, k_in, k_out), ou.make_config(0.01)

    class Side:
        def __init__(self):
            g = torch.Generator(device="cuda").manual_seed(11)
            new = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
            self.z = torch.zeros(n, dtype=torch.int32, device="cuda")
            self.X, self.dY, self.W = new(n, k_in), new(n, k_out), new(elements, k_in, k_out) / 8
            self.Y, self.dX, self.dW, self.M = (torch.zeros_like(t) for t in (self.dY, self.X, self.W, self.W))
            self.T = ou.make_tensors([self.dW], [self.M], [self.W])
            byte = lambda b: torch.empty(b, dtype=torch.uint8, device="cuda")  # noqa: E731
            self.grouping = byte(gp.gp_grouping_bytes(cfg, n))
            self.ws = byte(max(gp.gp_workspace_bytes(cfg, n), ou.ou_workspace_bytes(update, self.T)))

        def run(self):
            gp.gp_group(cfg, n, self.z, self.grouping, self.grouping.numel())
            gp.gp_forward(cfg, n, self.z, self.grouping, self.X, self.W, None, self.Y, self.ws, self.ws.numel())
            gp.gp_backward(cfg, n, self.z, self.grouping, self.X, self.W, self.dY, self.dX, self.dW, self.ws, self.ws.numel())
            ou.ou_step(update, self.T, self.ws, self.ws.numel())

    captured, eager = Side(), Side()
    captured.run()
    eager.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    generator = torch.Generator(device="cuda").manual_seed(5)
    for turn in range(4):
        z = torch.randint(-1, elements + 1 - turn, (n,), generator=generator, device="cuda").int()
        X = torch.randn(n, k_in, generator=generator, device="cuda")
        for side in (captured, eager):
            side.z.copy_(z)
            side.X.copy_(X)
        eager.run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in ("Y", "dX", "dW", "M", "W"):
            assert torch.equal(getattr(captured, name), getattr(eager, name)), (turn, name)


def test_the_command(ts, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["training_step", "--atoms", "200", "--degree", "5", "--channels", "64", "--steps", "2", "--self-connection", "--orthogonalised"])
    ts.main()
    lines = capsys.readouterr().out.splitlines()
    assert lines[0].startswith("200 atoms") and len(lines) == 3 and "nan" not in lines[2]
