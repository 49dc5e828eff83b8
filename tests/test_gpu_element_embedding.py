"""The element embedding (include/ee.h) through the C ABI against its fp64 oracle.

Tolerances: the forward is one product (two roundings of u = 2^-24 or 2^-53, bfloat16 rows one more of 2^-8); the gradient is a
sum of n_z rows in some fixed order, (n_z + 2) u sum |dY|, n_z the rows of that element.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -24}


@pytest.fixture(scope="module")
def ee():
    import torch
    assert torch.cuda.is_available()
    from paper_2504_10700_amd import ee_binding
    return ee_binding


def make_z(rng, n, elements, mode):
    if mode == "uniform":
        return rng.integers(0, elements, n)
    if mode == "one":                                   # all atoms of one element
        return np.full(n, elements // 2)
    if mode == "grouped":
        return np.sort(rng.integers(0, elements, n))
    if mode == "outside":                               # a third is padding, of every kind
        z = rng.integers(0, elements, n)
        bad = rng.choice([-1, elements, -2 ** 31, 2 ** 31 - 1, elements + 1023, 1 << 20], n)
        return np.where(rng.random(n) < 0.34, bad, z)
    return np.minimum((elements ** rng.random(n) - 1).astype(np.int64), elements - 1)    # "ranked"


def check(ee, n, elements, channels, dtype, mode, scale=0.3, seed=1):
    import torch
    row = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}[dtype]
    table = torch.float64 if dtype == "f64" else torch.float32
    kind = {"f32": ee.SC_F32, "f64": ee.SC_F64, "bf16": ee.SC_BF16}[dtype]
    rng = np.random.default_rng(seed)
    z = make_z(rng, n, elements, mode).astype(np.int32)
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = torch.randn(elements, channels, generator=g, device="cuda", dtype=torch.float64).to(table)
    dY = torch.randn(n, channels, generator=g, device="cuda", dtype=torch.float64).to(row)
    zd = torch.tensor(z, device="cuda")
    cfg = ee.make_config(elements, channels, scale, kind)
    Y = torch.full((n, channels), float("nan"), dtype=row, device="cuda")
    ee.ee_forward(cfg, n, zd, T, Y)
    nbytes = ee.ee_workspace_bytes(cfg, n)
    ws = torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda")
    runs = []
    for _ in range(2):
        dT = torch.full_like(T, float("nan"))
        ee.ee_backward(cfg, n, zd, dY, dT, ws, nbytes)
        runs.append(dT)
    assert torch.equal(*runs), "the gradient does not repeat to the bit"
    # the oracle's sums, here as products with index lists (the oracle itself walks row by row: small cases below)
    inside = (z >= 0) & (z < elements)
    T64, d64 = T.double().cpu().numpy(), dY.double().cpu().numpy()
    want = np.zeros((n, channels))
    want[inside] = scale * T64[z[inside]]
    u = U[dtype]
    got = Y.double().cpu().numpy()
    assert (np.abs(got - want) <= (3 * u + (2.0 ** -8 if dtype == "bf16" else 0)) * np.abs(want)).all()
    assert not got[~inside].any()
    sums, sizes = np.zeros((elements, channels)), np.zeros((elements, channels))
    np.add.at(sums, z[inside], d64[inside])
    np.add.at(sizes, z[inside], np.abs(d64[inside]))
    count = np.bincount(z[inside], minlength=elements)[:, None]
    got = runs[0].double().cpu().numpy()
    assert (np.abs(got - scale * sums) <= (count + 3) * u * abs(scale) * sizes).all()
    assert not got[count[:, 0] == 0].any(), "rows of absent elements must be zero"
    return z, T64, d64, Y, runs[0]


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("n,elements,channels", [(1, 1, 1), (1, 89, 128), (61, 89, 128), (64, 5, 3), (65, 2, 130), (1000, 10, 64), (1024, 1024, 20),
                                                 (1025, 7, 66), (3001, 89, 100), (2049, 1, 128), (5000, 1023, 36), (5000, 1024, 36),
                                                 (5000, 1025, 256), (9000, 50_000, 40), (20_000, 89, 257), (4097, 999_999, 4)])
@pytest.mark.parametrize("mode", ["uniform", "ranked", "outside"])
def test_against_sums_in_64_bits(ee, n, elements, channels, dtype, mode):
    print(f"embedding {n} {elements} {channels} {dtype} {mode}", flush=True)
    check(ee, n, elements, channels, dtype, mode)


@pytest.mark.parametrize("n", [63, 64, 65, 128, 1500, 4096, 70_001])
@pytest.mark.parametrize("mode", ["one", "grouped"])
def test_runs_over_many_pieces(ee, n, mode):
    print(f"embedding runs {n} {mode}", flush=True)
    check(ee, n, 4, 128, "f32", mode)
    check(ee, n, 2000, 64, "f32", mode)


def test_large_batch(ee):
    print("embedding 200000 x 128", flush=True)
    check(ee, 200_000, 89, 128, "f32", "uniform")
    check(ee, 300_000, 30_000, 16, "f64", "ranked")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_against_the_oracle(ee, dtype):
    from oracle import element_embedding as oe
    z, T, dY, Y, dT = check(ee, 150, 9, 33, dtype, "outside", scale=-1.25)
    got, want = Y.double().cpu().numpy(), oe.forward(z, T, -1.25)
    assert np.abs(got - want).max() <= 2.0 ** -8 * np.abs(want).max()
    want = oe.backward(z, dY, 9, -1.25)
    assert np.abs(dT.double().cpu().numpy() - want).max() <= 1e-5 * np.abs(want).max()


def test_no_rows_and_values_that_are_not_finite(ee):
    import torch
    cfg = ee.make_config(6, 40, 1.0)
    dT = torch.full((6, 40), float("nan"), device="cuda")
    ee.ee_backward(cfg, 0, None, None, dT, None, 0)
    assert not dT.any()
    for n in (200, 3000):
        z = torch.arange(n, device="cuda", dtype=torch.int32) % 7       # 6 is outside
        dY = torch.ones(n, 40, device="cuda")
        dY[6::7] = float("nan")                                          # rows without a part in the gradient
        dY[2, 5] = float("inf")
        nbytes = ee.ee_workspace_bytes(cfg, n)
        ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        ee.ee_backward(cfg, n, z, dY, dT, ws, nbytes)
        assert torch.isinf(dT[2, 5])
        dT[2, 5] = 0
        assert torch.isfinite(dT).all()


def test_offsets_beyond_32_bits(ee):
    """More than 2^31 elements of Y and dY, more than 2^32 bytes."""
    import torch
    n, k = 70_000, 32_768
    print(f"embedding {n} x {k} bf16", flush=True)
    cfg = ee.make_config(3, k, 1.0, ee.SC_BF16)
    z = (torch.arange(n, device="cuda") % 3).int()
    T = torch.randn(3, k, device="cuda")
    Y = torch.empty(n, k, dtype=torch.bfloat16, device="cuda")
    ee.ee_forward(cfg, n, z, T, Y)
    assert torch.equal(Y[-3:], T.bfloat16()[z[-3:].long()]) and torch.equal(Y[:3], T.bfloat16()[z[:3].long()])
    assert torch.equal(Y[65_535:65_538], T.bfloat16()[z[65_535:65_538].long()])
    Y.fill_(0)
    Y[-1], Y[0] = 2.0, 1.0
    dT, nbytes = torch.empty_like(T), ee.ee_workspace_bytes(cfg, n)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    ee.ee_backward(cfg, n, z, Y, dT, ws, nbytes)
    want = torch.zeros_like(T)
    want[0] += 1.0
    want[(n - 1) % 3] += 2.0
    assert torch.equal(dT, want)


def test_other_stream_and_graph_replay(ee):
    import torch
    n, cfg = 5000, ee.make_config(89, 128, 0.5)
    z = torch.randint(0, 89, (n,), device="cuda", dtype=torch.int32)
    dY, T = torch.randn(n, 128, device="cuda"), torch.randn(89, 128, device="cuda")
    nbytes = ee.ee_workspace_bytes(cfg, n)
    ws = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    Y, dT = torch.empty_like(dY), torch.empty_like(T)

    def step():
        ee.ee_forward(cfg, n, z, T, Y)
        ee.ee_backward(cfg, n, z, dY, dT, ws, nbytes)
    step()
    ref = Y.clone(), dT.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        Y.zero_()
        dT.zero_()
        step()
    side.synchronize()
    assert torch.equal(Y, ref[0]) and torch.equal(dT, ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for replay in range(3):
        if replay:
            z.copy_(z.roll(replay * 7))
            step()
            ref = Y.clone(), dT.clone()
        Y.fill_(float("nan"))
        dT.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, ref[0]) and torch.equal(dT, ref[1]), f"replay {replay}"


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("n,elements,channels", [(61, 89, 128), (1500, 89, 128), (4097, 1024, 20), (33_001, 1025, 64), (200_003, 89, 128), (32_768, 50_000, 72),
                                                 (70_001, 1, 64), (90_001, 700, 33)])
def test_sums_of_small_integers_are_exact(ee, n, elements, channels, dtype):
    """No row may be missing or counted twice, however many it is summed with."""
    import torch
    print(f"embedding of integers {n} {elements} {channels} {dtype}", flush=True)
    row = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}[dtype]
    table = torch.float64 if dtype == "f64" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(n)
    z = (elements * torch.rand(n, generator=g, device="cuda") ** 2 * 1.01).to(torch.int32)       # some beyond the table
    dY = torch.randint(-5, 6, (n, channels), generator=g, device="cuda").to(row)
    dT = torch.full((elements, channels), float("nan"), dtype=table, device="cuda")
    cfg = ee.make_config(elements, channels, 0.5, {"f32": ee.SC_F32, "f64": ee.SC_F64, "bf16": ee.SC_BF16}[dtype])
    nbytes = ee.ee_workspace_bytes(cfg, n)
    ee.ee_backward(cfg, n, z, dY, dT, torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda"), nbytes)
    inside = z < elements
    want = torch.zeros(elements, channels, dtype=torch.float64, device="cuda").index_add_(0, z[inside].long(), dY[inside].double()) * 0.5
    assert torch.equal(dT, want.to(table))


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("n,elements,channels", [(838, 10_000, 64), (839, 10_000, 64), (128, 65_536, 33), (8, 999_999, 4), (67, 999_999, 4), (70, 999_999, 4), (1024, 65_536, 33), (1024, 65_537, 33), (1024, 8192, 130), (1024, 8193, 130)])
def test_few_rows_of_long_tables(ee, n, elements, channels, dtype):
    print(f"embedding {n} {elements} {channels} {dtype}", flush=True)
    check(ee, n, elements, channels, dtype, "outside")


@pytest.mark.parametrize("elements,channels", [(1_000_000, 4301), (999_999, 1025)])
def test_tables_of_more_waves_than_a_launch_has(ee, elements, channels):
    """Three rows of a table of 4.3 (1.0) thousand million numbers: 68 (17) million waves' worth of dT, every element of it written."""
    import torch
    print(f"embedding 3 {elements} {channels}", flush=True)
    cfg = ee.make_config(elements, channels, 2.0)
    z = torch.tensor([elements - 1, 7, elements - 1], device="cuda", dtype=torch.int32)
    dY = torch.arange(3 * channels, device="cuda", dtype=torch.float32).view(3, channels)
    dT = torch.full((elements, channels), float("nan"), device="cuda")
    nbytes = ee.ee_workspace_bytes(cfg, 3)
    ee.ee_backward(cfg, 3, z, dY, dT, torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes)
    assert torch.equal(dT[-1], 2 * (dY[0] + dY[2])) and torch.equal(dT[7], 2 * dY[1])
    dT[-1], dT[7] = 0, 0
    assert all(not part.any() for part in dT.split(50_000))
    Y = torch.empty_like(dY)
    dT[7] = dY[1]
    ee.ee_forward(cfg, 3, z, dT, Y)
    assert not Y[0].any() and torch.equal(Y[1], 2 * dY[1])


@pytest.mark.parametrize("n", [31, 32, 33, 64, 65, 127, 130, 257, 512, 1023, 1024])
@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("elements,used,channels", [(1, 1, 64), (2, 2, 130), (89, 1, 128), (89, 2, 257), (6, 6, 1024), (1001, 3, 33), (65_536, 1, 66)])
def test_few_rows_of_few_elements(ee, n, dtype, elements, used, channels):
    """Small integers, exact: rows that several waves share, the last one of a workgroup's elements beyond the table, indices outside it between them."""
    import torch
    print(f"embedding {n} rows of {used} of {elements} elements {channels} {dtype}", flush=True)
    row = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}[dtype]
    table = torch.float64 if dtype == "f64" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(n)
    which = torch.randperm(elements, generator=g, device="cuda")[:used]
    z = which[torch.randint(0, used, (n,), generator=g, device="cuda")].int()
    z[5::11] = elements
    z[7::13] = -1
    dY = torch.randint(-9, 10, (n, channels), generator=g, device="cuda").to(row)
    dT = torch.full((elements, channels), float("nan"), dtype=table, device="cuda")
    cfg = ee.make_config(elements, channels, 0.25, {"f32": ee.SC_F32, "f64": ee.SC_F64, "bf16": ee.SC_BF16}[dtype])
    nbytes = ee.ee_workspace_bytes(cfg, n)
    ee.ee_backward(cfg, n, z, dY, dT, torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda"), nbytes)
    inside = (z >= 0) & (z < elements)
    want = torch.zeros(elements, channels, dtype=torch.float64, device="cuda").index_add_(0, z[inside].long(), dY[inside].double()) * 0.25
    assert torch.equal(dT, want.to(table))


@pytest.mark.parametrize("elements", [2, 89, 10_000])
def test_a_small_batch_of_one_element_is_no_slower_than_a_larger_one(ee, elements):
    """1024 rows are searched, 1025 sorted: the same work but for one row, however unevenly the elements are used (half as much again for noise)."""
    import torch
    print(f"embedding, time of 1024 rows of one of {elements} elements", flush=True)

    def microseconds(n):
        cfg = ee.make_config(elements, 128, 1.0)
        z, dY = torch.full((n,), elements // 2, device="cuda", dtype=torch.int32), torch.randn(n, 128, device="cuda")
        dT, nbytes = torch.empty(elements, 128, device="cuda"), ee.ee_workspace_bytes(cfg, n)
        ws, times = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), []
        for _ in range(25):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(4):
                ee.ee_backward(cfg, n, z, dY, dT, ws, nbytes)
            end.record()
            torch.cuda.synchronize()
            times.append(start.elapsed_time(end) * 250)
        return sorted(times)[12]
    few, more = microseconds(1024), microseconds(1025)
    print(f"1024 rows {few:.1f} us, 1025 rows {more:.1f} us", flush=True)
    assert few < 1.5 * more
