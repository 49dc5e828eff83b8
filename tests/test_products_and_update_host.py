"""Host-side checks of the products by element and the orthogonalised update (no GPU): exports against the headers,
constants, argument errors."""
import ctypes
import math
import os
import re

import pytest

gp = pytest.importorskip("paper_2504_10700_amd.gp_binding")
from paper_2504_10700_amd import ou_binding as ou  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def header(name):
    return open(os.path.join(ROOT, "include", name)).read()


@pytest.mark.parametrize("name,module", [("gp", gp), ("ou", ou)])
def test_library_exports_every_declared_symbol(name, module):
    declared = set(re.findall(r"^sc_status\s+(%s_\w+)\s*\(" % name, header(name + ".h"), flags=re.M))
    assert declared == set(module.EXPORTS)
    for fn in declared:
        assert getattr(module.lib, fn) is not None
    found = re.findall(r"\b((?:GP|OU)_[A-Z]\w*)\s*=?\s+([0-9]+)\b", header(name + ".h"))
    assert len(found) >= 5
    for const, value in found:
        assert getattr(module, const) == int(value), const


def refused(status, f, *args, **kw):
    with pytest.raises(gp.ScError) as e:
        f(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_product_refusals():
    good = gp.make_config(89, 128, 64, components=3)
    assert gp.gp_grouping_bytes(good, gp.GP_UNGROUPED) == 0 < gp.gp_grouping_bytes(good, gp.GP_UNGROUPED + 1)
    assert 256 <= gp.gp_workspace_bytes(good, 0) <= gp.gp_workspace_bytes(good, 1_000_000)
    for bad in (gp.make_config(0, 8, 8), gp.make_config(8, 0, 8), gp.make_config(8, 8, 0), gp.make_config(8, 8, 8, components=0),
                gp.make_config(8, 8, 8, dtype=3), gp.make_config(8, 8, 8, dtype=-1), gp.make_config(8, 8, 8, components=3, ld_in=23),
                gp.make_config(8, 8, 8, components=3, ld_out=23), gp.make_config(8, 8, 8, ld_in=-8)):
        refused(INVALID, gp.gp_workspace_bytes, bad, 10)
        refused(INVALID, gp.gp_grouping_bytes, bad, 10)
        refused(INVALID, gp.gp_group, bad, 100, 16, 256, 1 << 20, stream=0)
        refused(INVALID, gp.gp_forward, bad, 10, 16, None, 16, 16, None, 16, 256, 1 << 20, stream=0)
    for big in (gp.make_config(gp.GP_MAX_ELEMENTS + 1, 8, 8), gp.make_config(8, gp.GP_MAX_WIDTH + 1, 8), gp.make_config(8, 8, gp.GP_MAX_WIDTH + 1),
                gp.make_config(8, 8, 8, components=gp.GP_MAX_COMPONENTS + 1), gp.make_config(8, 8, 8, ld_in=gp.GP_MAX_STRIDE + 1),
                gp.make_config(8, 8, 8, ld_out=gp.GP_MAX_STRIDE + 1)):
        refused(UNSUPPORTED, gp.gp_workspace_bytes, big, 10)
    gp.gp_workspace_bytes(gp.make_config(8, 8, 8, components=2), gp.GP_MAX_ROWS // 2)
    refused(UNSUPPORTED, gp.gp_workspace_bytes, gp.make_config(8, 8, 8, components=2), gp.GP_MAX_ROWS // 2 + 1)
    refused(INVALID, gp.gp_workspace_bytes, good, -1)
    odd = gp.make_config(8, 8, 8)
    odd.reserved = 1
    refused(INVALID, gp.gp_workspace_bytes, odd, 10)
    short = gp.make_config(8, 64, 64)
    short.struct_size -= 4
    refused(INVALID, gp.gp_workspace_bytes, short, 10)
    n = ctypes.c_size_t()
    assert gp.lib.gp_workspace_bytes(None, 10, ctypes.byref(n)) == INVALID
    assert gp.lib.gp_workspace_bytes(ctypes.byref(good), 10, None) == INVALID
    assert gp.lib.gp_grouping_bytes(ctypes.byref(good), 10, None) == INVALID


def test_product_refusals_of_the_calls():
    cfg, bf = gp.make_config(8, 64, 64), gp.make_config(8, 64, 64, dtype=gp.SC_BF16)
    group, ws = gp.gp_grouping_bytes(cfg, 100), gp.gp_workspace_bytes(cfg, 100)
    gp.gp_group(cfg, 0, None, None, 0, stream=0)                             # nothing to do
    gp.gp_group(cfg, gp.GP_UNGROUPED, None, None, 0, stream=0)
    refused(INVALID, gp.gp_group, cfg, 100, None, 256, group, stream=0)
    refused(INVALID, gp.gp_group, cfg, 100, 18, 256, group, stream=0)        # misaligned z
    refused(INVALID, gp.gp_group, cfg, 100, 16, None, group, stream=0)
    refused(INVALID, gp.gp_group, cfg, 100, 16, 128, group, stream=0)
    refused(WORKSPACE, gp.gp_group, cfg, 100, 16, 256, group - 1, stream=0)
    gp.gp_forward(cfg, 0, None, None, None, None, None, None, None, 0, stream=0)
    good = [cfg, 100, 16, 256, 16, 16, 16, 16, 256, ws]                     # z, grouping, X, W, residual, Y, workspace
    for at, value, status in ((2, None, INVALID), (2, 18, INVALID), (3, None, INVALID), (3, 128, INVALID), (4, None, INVALID), (4, 18, INVALID),
                              (5, None, INVALID), (5, 18, INVALID), (6, 18, INVALID), (7, None, INVALID), (7, 18, INVALID), (8, None, WORKSPACE),
                              (8, 128, WORKSPACE), (9, ws - 1, WORKSPACE)):
        args = list(good)
        args[at] = value
        refused(status, gp.gp_forward, *args, stream=0)
    refused(INVALID, gp.gp_forward, bf, 100, 16, 256, 17, 16, None, 16, 256, ws, stream=0)     # rows of bfloat16: two bytes
    refused(INVALID, gp.gp_forward, bf, 100, 16, 256, 18, 18, None, 18, 256, ws, stream=0)     # but weights of four
    good = [cfg, 100, 16, 256, 16, 16, 16, 16, 16, 256, ws]                 # z, grouping, X, W, dY, dX, dW, workspace
    for at, value, status in ((2, None, INVALID), (3, None, INVALID), (3, 64, INVALID), (4, None, INVALID), (4, 18, INVALID), (5, None, INVALID),
                              (6, None, INVALID), (7, 18, INVALID), (8, 18, INVALID), (9, None, WORKSPACE), (9, 64, WORKSPACE), (10, ws - 1, WORKSPACE)):
        args = list(good)
        args[at] = value
        refused(status, gp.gp_backward, *args, stream=0)
    refused(INVALID, gp.gp_backward, cfg, 100, 16, 256, 16, 16, 16, None, None, 256, ws, stream=0)   # no output
    refused(INVALID, gp.gp_backward, cfg, 0, None, None, None, None, None, None, None, None, 0, stream=0)
    gp.gp_backward(cfg, 0, None, None, None, None, None, 16, None, None, 0, stream=0)                 # dX of no rows: nothing to do


def tensors(*items):
    """grad, momentum, weight, update, scale, count, rows, cols, dtype"""
    return (ou.ou_tensor * len(items))(*[ou.ou_tensor(*x, 0) for x in items])


OK = (256, 512, 1024, 2048, 1.0, 2, 8, 64, 0)


def test_update_refusals():
    cfg, one = ou.make_config(rate=0.02), tensors(OK)
    n = ou.ou_workspace_bytes(cfg, one)
    assert n >= 256 and ou.ou_workspace_bytes(cfg, tensors()) >= 256
    for field, value in (("struct_size", 8), ("steps", -1), ("flags", 2), ("a", math.inf), ("b", math.nan), ("c", math.inf), ("momentum", math.nan),
                         ("rate", math.inf), ("decay", math.nan), ("eps", 0.0), ("eps", -1.0), ("eps", math.nan), ("eps", math.inf)):
        bad = ou.make_config(rate=0.02)
        setattr(bad, field, value)
        refused(INVALID, ou.ou_workspace_bytes, bad, one)
        refused(INVALID, ou.ou_step, bad, one, 256, n, stream=0)
    refused(UNSUPPORTED, ou.ou_workspace_bytes, ou.make_config(rate=0.02, steps=ou.OU_MAX_STEPS + 1), one)
    refused(UNSUPPORTED, ou.ou_workspace_bytes, ou.make_config(rate=0.02, coefficients=(40.0, 0.0, 0.0), steps=2), one)   # 1600
    refused(UNSUPPORTED, ou.ou_workspace_bytes, ou.make_config(rate=0.02, coefficients=(0.0, 8000.0, -8000.0), steps=1), one)   # 1487 inside
    ou.ou_workspace_bytes(ou.make_config(rate=0.02, coefficients=(0.0, 4000.0, -4000.0), steps=1), one)
    ou.ou_workspace_bytes(ou.make_config(rate=0.02, coefficients=(1.5, -0.5, 0.0), steps=ou.OU_MAX_STEPS), one)
    ou.ou_workspace_bytes(ou.make_config(rate=0.02, coefficients=(1024.0, 0.0, 0.0), steps=1), one)
    for at, value in ((0, None), (0, 258), (1, 514), (2, 1026), (3, 2050), (4, math.nan), (5, -1), (6, 0), (7, 0), (8, 3)):
        bad = list(OK)
        bad[at] = value
        refused(INVALID, ou.ou_workspace_bytes, cfg, tensors(OK, tuple(bad)))
    refused(INVALID, ou.ou_workspace_bytes, cfg, tensors((256, 512, None, None, 1.0, 2, 8, 64, 0)))    # no result
    double = (256, 512, 1024, 2048, 1.0, 2, 8, 64, 1)
    for kw, scale in ((dict(rate=0.02, momentum=1e39), 1.0), (dict(rate=1e30), 1e10), (dict(rate=1e30, decay=1e10), 1.0), (dict(rate=1e-9), 1e39)):
        refused(INVALID, ou.ou_workspace_bytes, ou.make_config(**kw), tensors(OK[:4] + (scale,) + OK[5:]))   # beyond fp32
        ou.ou_workspace_bytes(ou.make_config(**kw), tensors(double[:4] + (scale,) + double[5:]))
    refused(INVALID, ou.ou_workspace_bytes, ou.make_config(rate=1e200), tensors(double[:4] + (1e200,) + double[5:]))
    odd = tensors(OK)
    odd[0].reserved = 1
    refused(INVALID, ou.ou_workspace_bytes, cfg, odd)
    ou.ou_workspace_bytes(cfg, tensors((258, 512, 1024, 2050, 1.0, 2, 8, 64, 2)))                      # bfloat16 gradient and update
    refused(INVALID, ou.ou_workspace_bytes, cfg, tensors((258, 514, 1024, 2050, 1.0, 2, 8, 64, 2)))
    ou.ou_workspace_bytes(cfg, tensors((None, None, None, None, 1.0, 0, 8, 64, 0)))                    # an empty batch needs nothing
    refused(UNSUPPORTED, ou.ou_workspace_bytes, cfg, tensors((256, None, 256, None, 1.0, 1, ou.OU_MAX_SIDE + 1, 1, 0)))
    refused(UNSUPPORTED, ou.ou_workspace_bytes, cfg, tensors((256, None, 256, None, 1.0, ou.OU_MAX_TILES + 1, 1, 1, 0)))
    refused(UNSUPPORTED, ou.ou_workspace_bytes, cfg, tensors(OK, (256, None, 256, None, 1.0, ou.OU_MAX_TILES - 1, 1, 1, 0)))
    refused(UNSUPPORTED, ou.ou_workspace_bytes, cfg, tensors((256, None, 256, None, 1.0, 2 ** 62, 60_000, 60_000, 0)))
    b = ctypes.c_size_t()
    assert ou.lib.ou_workspace_bytes(None, 1, one, ctypes.byref(b)) == INVALID
    assert ou.lib.ou_workspace_bytes(ctypes.byref(cfg), -1, one, ctypes.byref(b)) == INVALID
    assert ou.lib.ou_workspace_bytes(ctypes.byref(cfg), 1, None, ctypes.byref(b)) == INVALID
    assert ou.lib.ou_workspace_bytes(ctypes.byref(cfg), ou.OU_MAX_TENSORS + 1, one, ctypes.byref(b)) == UNSUPPORTED
    assert ou.lib.ou_workspace_bytes(ctypes.byref(cfg), 1, one, None) == INVALID
    refused(WORKSPACE, ou.ou_step, cfg, one, None, n, stream=0)
    refused(WORKSPACE, ou.ou_step, cfg, one, 256, n - 1, stream=0)
    refused(WORKSPACE, ou.ou_step, cfg, one, 128, n, stream=0)
    ou.ou_step(cfg, tensors(), None, 0, stream=0)                                                       # nothing to do
    ou.ou_step(cfg, tensors((None, None, None, None, 1.0, 0, 8, 64, 0)), None, 0, stream=0)


def test_update_tensors():
    import torch
    f, b = torch.zeros(3, 8, 64), torch.zeros(8, 64, dtype=torch.bfloat16)
    t = ou.make_tensors([f, b], weight=[f, b.float()], scale=[2.0, 1.0])
    assert (t[0].count, t[0].rows, t[0].cols, t[0].scale, t[1].count, t[1].dtype) == (3, 8, 64, 2.0, 1, ou.SC_BF16)
    assert t[0].momentum is None and t[0].update is None
    for bad in (dict(weight=[f]), dict(weight=[f, b]), dict(weight=[f, b.float().t()]), dict(update=[f, b.float()]), dict(momentum=[f, b]),
                dict(weight=[f.double(), b.float()]), dict(weight=[f[:2], b.float()]), dict(scale=[1.0])):
        with pytest.raises(ValueError):
            ou.make_tensors([f, b], **bad)
    for bad in (torch.zeros(8), torch.zeros(8, 64).t(), torch.zeros(8, 8, dtype=torch.int32)):
        with pytest.raises(ValueError):
            ou.make_tensors([bad], update=[bad])
