"""Host-side checks of the dense layer, the element embedding and the gradient clipping (no GPU): exports against the
headers, constants, argument errors."""
import ctypes
import os
import re

import pytest

dl = pytest.importorskip("paper_2504_10700_amd.dl_binding")
from paper_2504_10700_amd import ee_binding as ee  # noqa: E402
from paper_2504_10700_amd import gc_binding as gc  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def header(name):
    return open(os.path.join(ROOT, "include", name)).read()


@pytest.mark.parametrize("name,module", [("dl", dl), ("ee", ee), ("gc", gc)])
def test_library_exports_every_declared_symbol(name, module):
    declared = set(re.findall(r"^sc_status\s+(%s_\w+)\s*\(" % name, header(name + ".h"), flags=re.M))
    assert declared == set(module.EXPORTS)
    for fn in declared:
        assert getattr(module.lib, fn) is not None
    for const, value in re.findall(r"\b((?:DL|EE|GC)_[A-Z]\w*)\s*=?\s+([0-9]+)\b", header(name + ".h")):
        assert getattr(module, const) == int(value), const


def refused(status, f, *args, **kw):
    with pytest.raises(dl.ScError) as e:
        f(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_dense_layer_refusals():
    good = dl.make_config(8, 64, dl.DL_SILU)
    assert dl.dl_workspace_bytes(good, 0) >= 256
    assert 256 <= dl.dl_workspace_bytes(good, 100) <= dl.dl_workspace_bytes(good, 1_000_000)
    for bad in (dl.make_config(0, 64), dl.make_config(8, 0), dl.make_config(8, 64, 4), dl.make_config(8, 64, -1), dl.make_config(8, 64, dtype=3),
                dl.make_config(8, 64, ld_in=7), dl.make_config(8, 64, ld_out=63), dl.make_config(8, 64, ld_in=-8)):
        refused(INVALID, dl.dl_workspace_bytes, bad, 10)
        refused(INVALID, dl.dl_forward, bad, 10, 16, 16, None, None, 16, None, stream=0)
    refused(UNSUPPORTED, dl.dl_workspace_bytes, dl.make_config(dl.DL_MAX_WIDTH + 1, 8), 10)
    refused(UNSUPPORTED, dl.dl_workspace_bytes, dl.make_config(8, 8, ld_in=dl.DL_MAX_STRIDE + 1), 10)
    refused(UNSUPPORTED, dl.dl_workspace_bytes, dl.make_config(8, 8, ld_out=dl.DL_MAX_STRIDE + 1), 10)
    refused(INVALID, dl.dl_workspace_bytes, good, -1)
    refused(INVALID, dl.dl_workspace_bytes, good, (1 << 30) + 1)
    short = dl.make_config(8, 64)
    short.struct_size -= 4
    refused(INVALID, dl.dl_workspace_bytes, short, 10)
    assert dl.lib.dl_workspace_bytes(None, 10, ctypes.byref(ctypes.c_size_t())) == INVALID
    assert dl.lib.dl_workspace_bytes(ctypes.byref(good), 10, None) == INVALID
    refused(INVALID, dl.dl_forward, good, 10, None, 16, None, None, 16, None, stream=0)
    refused(INVALID, dl.dl_forward, good, 10, 16, 16, 8, None, 16, None, stream=0)                  # misaligned bias
    dl.dl_forward(good, 0, None, None, None, None, None, None, stream=0)                            # nothing to do
    n = dl.dl_workspace_bytes(good, 10)
    refused(INVALID, dl.dl_backward, good, 10, 16, 16, 16, 16, None, None, None, 256, n, stream=0)  # no output
    refused(INVALID, dl.dl_backward, good, 10, 16, 16, None, 16, 16, None, None, 256, n, stream=0)  # Z is needed
    refused(INVALID, dl.dl_backward, good, 10, 16, 16, 16, 24, 16, None, None, 256, n, stream=0)    # misaligned
    refused(WORKSPACE, dl.dl_backward, good, 10, 16, 16, 16, 16, 16, None, None, 256, n - 1, stream=0)
    refused(WORKSPACE, dl.dl_backward, good, 10, 16, 16, 16, 16, 16, None, None, None, n, stream=0)
    refused(WORKSPACE, dl.dl_backward, good, 10, 16, 16, 16, 16, 16, None, None, 128, n, stream=0)
    refused(INVALID, dl.dl_double_backward, good, 10, 16, 16, 16, 16, 16, None, 16, 16, 16, 256, n, stream=0)   # ddY
    refused(WORKSPACE, dl.dl_double_backward, good, 10, 16, 16, 16, 16, 16, 16, 16, 16, 16, 256, n - 1, stream=0)


def test_embedding_refusals():
    good = ee.make_config(89, 128, 0.1)
    assert 256 <= ee.ee_workspace_bytes(good, 0) <= ee.ee_workspace_bytes(good, 100) <= ee.ee_workspace_bytes(good, 1_000_000)
    for bad in (ee.make_config(0, 128), ee.make_config(89, 0), ee.make_config(89, 128, dtype=5), ee.make_config(89, 128, float("nan")),
                ee.make_config(89, 128, float("inf"))):
        refused(INVALID, ee.ee_workspace_bytes, bad, 10)
    refused(UNSUPPORTED, ee.ee_workspace_bytes, ee.make_config(ee.EE_MAX_ELEMENTS + 1, 8), 10)
    refused(UNSUPPORTED, ee.ee_workspace_bytes, ee.make_config(8, ee.EE_MAX_CHANNELS + 1), 10)
    refused(INVALID, ee.ee_workspace_bytes, good, -1)
    refused(INVALID, ee.ee_forward, good, 10, None, 16, 16, stream=0)
    refused(INVALID, ee.ee_forward, good, 10, 16, 16, 20, stream=0)
    ee.ee_forward(good, 0, None, None, None, stream=0)
    n = ee.ee_workspace_bytes(good, 10_000)
    refused(INVALID, ee.ee_backward, good, 10_000, 16, 16, None, 256, n, stream=0)
    refused(INVALID, ee.ee_backward, good, 10_000, None, 16, 16, 256, n, stream=0)
    refused(WORKSPACE, ee.ee_backward, good, 10_000, 16, 16, 16, 256, n - 1, stream=0)
    refused(WORKSPACE, ee.ee_backward, good, 10_000, 16, 16, 16, 64, n, stream=0)


def test_clipping_refusals():
    good = gc.make_config(10.0)
    one = (gc.gc_tensor * 2)(gc.gc_tensor(256, 256, 5, gc.SC_F32, 0), gc.gc_tensor(512, 512, 5, gc.SC_BF16, 0))
    n = gc.gc_workspace_bytes(good, one)
    assert n >= 256 and gc.gc_workspace_bytes(good, (gc.gc_tensor * 500)(*[one[0]] * 500)) > n
    for bad in (gc.make_config(0.0), gc.make_config(-1.0), gc.make_config(float("nan")), gc.make_config(1.0, -1e-6),
                gc.make_config(1.0, float("nan")), gc.make_config(1.0, float("inf")), gc.make_config(1.0, dtype=gc.SC_BF16)):
        refused(INVALID, gc.gc_workspace_bytes, bad, one)
    refused(INVALID, gc.gc_clip, good, one, None, 256, n, stream=0)
    refused(WORKSPACE, gc.gc_clip, good, one, 16, 256, n - 1, stream=0)
    refused(WORKSPACE, gc.gc_clip, good, one, 16, 100, n, stream=0)
    for field, value in (("src", None), ("src", 257), ("dst", 258), ("numel", -1), ("dtype", 3), ("dst", None)):
        bad = (gc.gc_tensor * 2)(*one)
        setattr(bad[1] if field == "dst" and value is None else bad[0], field, value)
        refused(INVALID, gc.gc_clip, good, bad, 16, 256, n, stream=0)
    import torch
    x = torch.zeros(4, 4)
    for src, dst in (([x.half()], None), ([x.t()[1:]], None), ([x], [x.double()]), ([x], [x[:2]]), ([x], [])):
        with pytest.raises(ValueError):
            gc.make_tensors(src, dst)


@pytest.mark.parametrize("dtype", [dl.SC_F32, dl.SC_F64, dl.SC_BF16])
def test_dense_layer_workspace_of_wide_layers(dtype):
    """Without an activation: W transposed and partial results, which stay a small part of dY, or below three times W where that is large, or below 270 MB."""
    row, weight = {dl.SC_F32: 4, dl.SC_F64: 8, dl.SC_BF16: 2}[dtype], 8 if dtype == dl.SC_F64 else 4
    for rows in (1, 100, 2500, 8192, 24_414, 65_536, 1_000_000):
        for k_in, k_out in ((64, 64), (64, 1280), (1280, 64), (1280, 1280), (2048, 2048), (2560, 2560), (4096, 2304), (4096, 4096), (16_384, 16_384),
                            (dl.DL_MAX_WIDTH, 128), (dl.DL_MAX_WIDTH, dl.DL_MAX_WIDTH), (1279, 4097)):
            n, w = dl.dl_workspace_bytes(dl.make_config(k_in, k_out, dl.DL_NONE, dtype), rows), k_in * k_out * weight
            assert n - w <= max(rows * k_out * weight / 4, 3 * w if k_in * k_out > 8 << 20 else 0, 270e6) * 1.01 + 1024, (rows, k_in, k_out)
    # one chunk needs no partial results
    assert dl.dl_workspace_bytes(dl.make_config(4096, 4096, dl.DL_NONE, dl.SC_F64), 20_000) <= 4096 * 4096 * 8 + 1024
    assert dl.dl_workspace_bytes(dl.make_config(dl.DL_MAX_WIDTH, dl.DL_MAX_WIDTH, dl.DL_NONE, dl.SC_F32), 8192) <= dl.DL_MAX_WIDTH ** 2 * 4 + 1024


def test_embedding_refuses_a_scale_that_its_type_does_not_hold():
    for dtype in (dl.SC_F32, dl.SC_BF16):
        refused(INVALID, ee.ee_workspace_bytes, ee.make_config(89, 128, 1e39, dtype), 10)
        refused(INVALID, ee.ee_workspace_bytes, ee.make_config(89, 128, -1e39, dtype), 10)
        refused(INVALID, ee.ee_forward, ee.make_config(89, 128, 1e39, dtype), 10, 16, 16, 16, stream=0)
        ee.ee_workspace_bytes(ee.make_config(89, 128, 3e38, dtype), 10)
    ee.ee_workspace_bytes(ee.make_config(89, 128, 1e300, dl.SC_F64), 10)
