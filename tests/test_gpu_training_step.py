"""The training example (training_step.py): gradients of the whole chain against differences of its loss, and steps of descent."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ts():
    import torch
    assert torch.cuda.is_available()
    from paper_2504_10700_amd import training_step
    return training_step


def test_gradients_against_differences(ts):
    """fp64: central differences along random directions of each parameter, relative error of h^2 and of u / h."""
    import torch
    model = ts.Model(40, 5, 8, elements=5, l_Y=1, dtype=ts.sc.SC_F64)
    loss = model.loss().item()
    model.backward()
    gradients = [g.clone() for g in model.gradients]
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


def test_steps_descend_and_repeat(ts):
    import torch
    runs = []
    for _ in range(2):
        model = ts.Model(500, 8, 64, max_norm=1.0)
        losses = torch.stack([model.step() for _ in range(30)])
        assert torch.isfinite(losses).all() and losses[-1] < 0.9 * losses[0]
        # clipped in place: the gradients' norm is at most 1
        norm = torch.sqrt(sum((g.double() ** 2).sum() for g in model.gradients)).item()
        assert norm <= 1 + 1e-5 and abs(norm - min(1.0, model.norm[0].item())) <= 1e-4
        runs.append([p.clone() for p in model.parameters[2:]])
    # every call of the library has a fixed order of sums (the example's index_add_ of energies may not): equal up to a few roundings
    for a, b in zip(*runs):
        assert (a - b).abs().max() <= 1e-4 * a.abs().max()
