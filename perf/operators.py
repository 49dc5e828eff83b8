"""The trainable parts beside the equivariant kernels, as a list of timed cases.

A model around the tensor product and the contraction has three more kinds of work in each step: the embedding of
the elements that the first layer's features come from, the dense layers that make the radial weights R of every edge and the
readout, and the global norm of all gradients that clips them before the weights change.

  dense   Z = X W + b,  Y = act(Z) + residual                                       (dl_forward)
          G = dY act'(Z),  dX = G W^T,  dW = X^T G,  db = sum of G over the rows    (dl_backward)
          and the gradients of sum(HX * dX) with respect to dY, X, W, b             (dl_double_backward)
  embed   Y[i] = scale * table[z_i], and the gradient of the table                  (ee_forward, ee_backward)
  clip    norm = sqrt(sum over all tensors of x^2), coefficient = min(1, max_norm / (norm + eps)), coefficient * x   (gc_clip)

Ranges: 1 to a million rows, 1 to 1280 columns, tables of 2 to 65 536 rows, lists of a dozen to several hundred tensors; fp32,
fp64 and bfloat16 rows (weights and their gradients stay fp32 beside bfloat16 rows, as everywhere in this library).
"""
from __future__ import annotations

import math

import torch

own = False

ROW_TYPE = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16}
WEIGHT_TYPE = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.float32}
BYTES = {"f32": 4, "f64": 8, "bf16": 2}
WEIGHT_BYTES = {"f32": 4, "f64": 8, "bf16": 4}
ELEMENTS = 89
MAX_NORM, EPS = 10.0, 1e-6
GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


# ---- the cases ---------------------------------------------------------------------------------


def _dense(name, call, rows, k_in, k_out, act="silu", bias=True, residual=False, dtype="f32", spread=1):
    """spread: X is one column block of rows that are `spread` times as wide."""
    return {"name": name, "op": "dense", "call": call, "rows": rows, "k_in": k_in, "k_out": k_out, "act": act, "bias": bias,
            "residual": residual, "dtype": dtype, "spread": spread}


def _embed(name, rows, channels, elements=ELEMENTS, dtype="f32"):
    return {"name": name, "op": "embed", "rows": rows, "channels": channels, "elements": elements, "dtype": dtype}


def _clip(name, layers, channels, active=True, dtype="f32"):
    return {"name": name, "op": "clip", "layers": layers, "channels": channels, "active": active, "dtype": dtype}


def listed():
    return [
        # first radial layer of one small molecule (19 atoms with 20 neighbours): latency of a single call
        _dense("dense_one_molecule", "forward", 380, 8, 64),
        # hidden radial layer of the training step of 10 000 atoms with about 20 neighbours each, forward and backward
        _dense("dense_hidden_step", "step", 199_003, 64, 64, residual=True),
        # ... and its second-order pass, which a loss on forces needs
        _dense("dense_hidden_second", "second", 199_003, 64, 64),
        # last radial layer of the same step: 10 paths x 128 channels of R per edge
        _dense("dense_radial_step", "step", 199_003, 64, 1280, act="none", bias=False),
        # the same for the batch of 50 000 atoms, rows stored as bfloat16
        _dense("dense_radial_bf16", "step", 990_001, 64, 1280, act="none", bias=False, dtype="bf16"),
        # readout from the scalar channels of [atom][component][channel] features, double precision
        _dense("dense_readout_f64", "step", 10_000, 128, 16, dtype="f64", spread=4),
        # a wide layer on bfloat16 rows, where the matrix cores count
        _dense("dense_wide_backward", "backward", 8191, 1024, 1024, act="gelu", dtype="bf16"),
        # features of one small structure: latency
        _embed("embed_one_molecule", 61, 128),
        # features of the large batch, six elements with a tenth of the atoms each
        _embed("embed_200k_atoms", 200_000, 128),
        # a large table of types, most of them rare, rows stored as bfloat16
        _embed("embed_large_table", 32_768, 512, elements=50_000, dtype="bf16"),
        # gradients of a model of two layers
        _clip("clip_two_layers", 2, 128),
        # gradients of a deep and wide model
        _clip("clip_24_layers", 24, 512),
    ]


def _log_size(rng, lo, hi):
    """A size spread evenly over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(["dense", "embed", "clip"], [6, 2, 2])[0]
    if op == "dense":
        dtype = rng.choices(["f32", "bf16", "f64"], [5, 3, 2])[0]
        call = rng.choice(["forward", "backward", "second", "step"])
        k_in = rng.choice([8, 16, 64, 64, 128, 256, _log_size(rng, 1, 1280)])
        k_out = rng.choice([16, 64, 64, 128, 1280, 1024, _log_size(rng, 1, 1280)])
        most = min(1_000_000, int((1.5e8 if dtype == "f64" else 3e8) / (k_in + k_out)), int((1e10 if dtype == "f64" else 4e10) / (k_in * k_out)))
        act = rng.choice(["silu", "silu", "gelu", "relu", "none"])
        if dtype == "bf16" and call == "step":
            act = "none"      # a rounded Z between the two calls would make the gradients depend on its last bit
        case = _dense("", call, _log_size(rng, 1, most), k_in, k_out, act=act, bias=rng.random() < 0.7, residual=rng.random() < 0.5,
                      dtype=dtype, spread=rng.choice([1, 1, 1, 4]))
    elif op == "embed":
        case = _embed("", _log_size(rng, 1, 400_000), rng.choice([64, 128, 256, _log_size(rng, 1, 512)]),
                      elements=rng.choice([ELEMENTS, _log_size(rng, 2, 65_536)]), dtype=rng.choice(["f32", "f32", "f64", "bf16"]))
    else:
        case = _clip("", _log_size(rng, 1, 32), _log_size(rng, 8, 400), active=rng.random() < 0.8,
                     dtype=rng.choice(["f32", "f32", "f64", "bf16", "mixed"]))
    del case["name"]
    return case


def _lengths(case):
    """Elements of each parameter tensor: the embedding, then per layer four radial layers (three biases), the channel mixing of four
    orders, the weights of 86 paths for each element, and a readout with its bias."""
    k = case["channels"]
    layer = [8 * 64, 64, 64 * 64, 64, 64 * 64, 64, 64 * 10 * k, 4 * k * k, ELEMENTS * 86 * k, k * 16 + 16]
    return [ELEMENTS * k] + layer * case["layers"]


def _types(case):
    """Type of each parameter tensor: one for all, or fp32 and bfloat16 in turn."""
    n = len(_lengths(case))
    if case["dtype"] == "mixed":
        return [torch.float32 if i % 2 else torch.bfloat16 for i in range(n)]
    return [ROW_TYPE[case["dtype"]]] * n


def _packed(case):
    """Lengths of the tensors of each type."""
    lengths, types = _lengths(case), _types(case)
    return {t: [n for n, u in zip(lengths, types) if u == t] for t in dict.fromkeys(types)}


def _views(case, buckets):
    return [x for t, lengths in _packed(case).items() for x in buckets[t].split(lengths)]


def _gated(case):
    """Do the backward passes depend on Z?"""
    return case["act"] != "none"


def work(case):
    if case["op"] == "clip":
        n = sum(_lengths(case))
        nbytes = sum(a * torch.empty(0, dtype=t).element_size() for a, t in zip(_lengths(case), _types(case)))
        return {"bytes": 2 * nbytes, "flops": 3 * n}
    b, w = BYTES[case["dtype"]], WEIGHT_BYTES[case["dtype"]]
    r = case["rows"]
    if case["op"] == "embed":
        k, z = case["channels"], case["elements"]
        return {"bytes": 8 * r + 2 * r * k * b + (min(r, z) + z) * k * w, "flops": 3 * r * k}
    ki, ko, gated = case["k_in"], case["k_out"], int(_gated(case))
    product, weights, x, y = 2 * r * ki * ko, (ki * ko + ko * int(case["bias"])) * w, r * ki * b, r * ko * b
    forward = {"bytes": x + weights + y * (1 + gated + int(case["residual"])), "flops": product}
    backward = {"bytes": 2 * x + 2 * weights + y * (1 + gated), "flops": 2 * product}
    second = {"bytes": 3 * x + 2 * weights + y * (2 + gated), "flops": (2 + 2 * gated) * product}
    if case["call"] == "step":
        return {m: forward[m] + backward[m] for m in forward}
    return {"forward": forward, "backward": backward, "second": second}[case["call"]]


# ---- inputs ------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, scale=1.0: torch.randn(*shape, generator=g, device="cuda") * scale  # noqa: E731
    make = {"dense": _prepare_dense, "embed": _prepare_embed, "clip": _prepare_clip}[case["op"]]
    state = make(case, g, normal)
    state["case"] = case
    if own:
        _plan(state)
    return state


def _prepare_dense(case, g, normal):
    t, w = ROW_TYPE[case["dtype"]], WEIGHT_TYPE[case["dtype"]]
    r, ki, ko = case["rows"], case["k_in"], case["k_out"]
    s = {"X": normal(r, case["spread"] * ki).to(t)[:, :ki], "W": normal(ki, ko, scale=ki ** -0.5).to(w),
         "b": normal(ko, scale=0.1).to(w) if case["bias"] else None}
    if case["residual"] and case["call"] in ("forward", "step"):
        s["R"] = normal(r, ko).to(t)
    if case["call"] != "forward":
        s["dY"] = normal(r, ko).to(t)
    if case["call"] in ("backward", "second") and _gated(case):
        z = s["X"].to(w) @ s["W"]
        s["Z"] = (z if s["b"] is None else z.add_(s["b"])).to(t)
    if case["call"] == "second":
        s["HX"] = normal(r, case["spread"] * ki).to(t)[:, :ki]
    return s


def _prepare_embed(case, g, normal):
    n, k, z = case["rows"], case["channels"], case["elements"]
    u = torch.rand(n, generator=g, device="cuda")
    rest = torch.randint(0, z, (n,), generator=g, device="cuda")
    if z <= 1024:     # elements: six dominant ones with a tenth of the atoms each
        dominant = torch.tensor([0, 5, 6, 7, 13, 25], device="cuda") % z
        index = torch.where(u < 0.6, dominant[(u * 10).long().clamp_(max=5)], rest)
    else:             # a table of types: frequencies fall with the rank
        index = (z ** u.double() - 1).long().clamp_(0, z - 1)
    return {"z": index.int(), "T": normal(z, k).to(WEIGHT_TYPE[case["dtype"]]), "dY": normal(n, k).to(ROW_TYPE[case["dtype"]])}


def _prepare_clip(case, g, normal):
    # the gradients of one type are views of one bucket, packed as the all-reduce of data-parallel training takes them
    size = MAX_NORM * (2.5 if case["active"] else 0.4) / math.sqrt(sum(_lengths(case)))
    buckets = {t: normal(sum(lengths), scale=size).to(t) for t, lengths in _packed(case).items()}
    return {"buckets": buckets, "grads": _views(case, buckets)}


# ---- one pass ----------------------------------------------------------------------------------


def run(state):
    forms = {"dense": (_dense_plain, _dense_own), "embed": (_embed_plain, _embed_own), "clip": (_clip_plain, _clip_own)}
    return forms[state["case"]["op"]][own](state)


def _gate(act, z):
    """act(z), act'(z), act''(z)."""
    if act == "none":
        return z, torch.ones_like(z), torch.zeros_like(z)
    if act == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on, torch.zeros_like(z)
    if act == "silu":
        u, u1, u2 = z, 1.0, 0.0
    else:
        u, u1, u2 = 2 * GELU_A * (z + GELU_B * z * z * z), 2 * GELU_A * (1 + 3 * GELU_B * z * z), 12 * GELU_A * GELU_B * z
    s = 1 / (1 + torch.exp(-u))
    d1 = s * (1 - s)
    d2 = d1 * (1 - 2 * s)
    return z * s, s + z * d1 * u1, 2 * d1 * u1 + z * (d2 * u1 * u1 + d1 * u2)


def _dense_plain(state):
    case = state["case"]
    t, w = ROW_TYPE[case["dtype"]], WEIGHT_TYPE[case["dtype"]]
    act, call, out = case["act"], case["call"], {}
    X, W, Z = state["X"].to(w), state["W"], state.get("Z")
    if call in ("forward", "step"):
        Z = X @ W
        if state["b"] is not None:
            Z = Z + state["b"]
        Y = _gate(act, Z)[0]
        if "R" in state:
            Y = Y + state["R"].to(w)
        out["Y"] = Y.to(t)
        if _gated(case):
            out["Z"] = Z.to(t)
    if call in ("backward", "step"):
        G = state["dY"].to(w)
        if _gated(case):
            G = G * _gate(act, Z.to(w))[1]
        out["dX"], out["dW"] = (G @ W.t()).to(t), X.t() @ G
        if case["bias"]:
            out["db"] = G.sum(0)
    if call == "second":
        dY, HX = state["dY"].to(w), state["HX"].to(w)
        V = HX @ W
        if _gated(case):
            _, d1, d2 = _gate(act, Z.to(w))
            S = V * dY * d2
            out["ddY"], out["X2"], out["W2"] = (V * d1).to(t), (S @ W.t()).to(t), X.t() @ S + HX.t() @ (dY * d1)
            if case["bias"]:
                out["b2"] = S.sum(0)
        else:
            out["ddY"], out["X2"], out["W2"] = V.to(t), torch.zeros_like(HX, dtype=t), HX.t() @ dY
            if case["bias"]:
                out["b2"] = torch.zeros_like(state["b"])
    return out


def _embed_plain(state):
    t, w = ROW_TYPE[state["case"]["dtype"]], WEIGHT_TYPE[state["case"]["dtype"]]
    T, index, scale = state["T"], state["z"].long(), state["case"]["elements"] ** -0.5
    dT = torch.zeros_like(T).index_add_(0, index, state["dY"].to(w) * scale)
    return {"Y": (T[index] * scale).to(t), "dT": dT}


def _clip_plain(state):
    w = torch.float64 if state["case"]["dtype"] == "f64" else torch.float32
    norm = torch.stack([(x.to(w) * x.to(w)).sum() for x in state["grads"]]).sum().sqrt()
    coefficient = (MAX_NORM / (norm + EPS)).clamp(max=1.0)
    return {"norm": norm, "coefficient": coefficient, "clipped": [(x.to(w) * coefficient).to(t) for t, x in state["buckets"].items()]}


# ---- the same passes through the library ---------------------------------------------------------


def _plan(state):
    """What a program keeps beside its tensors: configuration, outputs, workspace."""
    from paper_2504_10700_amd import dl_binding as dl
    from paper_2504_10700_amd import ee_binding as ee
    from paper_2504_10700_amd import gc_binding as gc
    case = state["case"]
    kind = {"f32": dl.SC_F32, "f64": dl.SC_F64, "bf16": dl.SC_BF16, "mixed": dl.SC_F32}[case["dtype"]]
    if case["op"] == "dense":
        act = {"none": dl.DL_NONE, "relu": dl.DL_RELU, "silu": dl.DL_SILU, "gelu": dl.DL_GELU}[case["act"]]
        r, ki, ko = case["rows"], case["k_in"], case["k_out"]
        cfg = dl.make_config(ki, ko, act, kind, ld_in=case["spread"] * ki)
        rows_out = lambda: torch.empty((r, ko), dtype=ROW_TYPE[case["dtype"]], device="cuda")  # noqa: E731
        rows_in = lambda: torch.empty((r, case["spread"] * ki), dtype=ROW_TYPE[case["dtype"]], device="cuda")[:, :ki]  # noqa: E731
        new_b = lambda: None if state["b"] is None else torch.empty_like(state["b"])  # noqa: E731
        out = {}
        if case["call"] in ("forward", "step"):
            out["Y"] = rows_out()
            if _gated(case):
                out["Z"] = rows_out()
        if case["call"] in ("backward", "step"):
            out.update(dX=rows_in(), dW=torch.empty_like(state["W"]), db=new_b())
        if case["call"] == "second":
            out.update(ddY=rows_out(), X2=rows_in(), W2=torch.empty_like(state["W"]), b2=new_b())
        nbytes = 0 if case["call"] == "forward" else dl.dl_workspace_bytes(cfg, r)
        state.update(lib=dl, cfg=cfg, out=out)
    elif case["op"] == "embed":
        cfg = ee.make_config(case["elements"], case["channels"], case["elements"] ** -0.5, kind)
        nbytes = ee.ee_workspace_bytes(cfg, case["rows"])
        state.update(lib=ee, cfg=cfg, out={"Y": torch.empty_like(state["dY"]), "dT": torch.empty_like(state["T"])})
    else:
        cfg = gc.make_config(MAX_NORM, EPS, kind if case["dtype"] == "f64" else dl.SC_F32)
        clipped = {t: torch.empty_like(x) for t, x in state["buckets"].items()}
        both = torch.empty(2, dtype=torch.float64 if case["dtype"] == "f64" else torch.float32, device="cuda")
        tensors = gc.make_tensors(state["grads"], _views(case, clipped))
        nbytes = gc.gc_workspace_bytes(cfg, tensors)
        state.update(lib=gc, cfg=cfg, both=both, tensors=tensors, clipped=list(clipped.values()))
    state["ws"], state["ws_bytes"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda"), nbytes


def _dense_own(state):
    case, dl, cfg, out = state["case"], state["lib"], state["cfg"], state["out"]
    r, X, W, Z = case["rows"], state["X"], state["W"], state.get("Z")
    if case["call"] in ("forward", "step"):
        Z = out.get("Z")
        dl.dl_forward(cfg, r, X, W, state["b"], state.get("R"), out["Y"], Z)
    if case["call"] in ("backward", "step"):
        dl.dl_backward(cfg, r, X, W, Z, state["dY"], out["dX"], out["dW"], out["db"], state["ws"], state["ws_bytes"])
    if case["call"] == "second":
        dl.dl_double_backward(cfg, r, X, W, Z, state["dY"], state["HX"], out["ddY"], out["X2"], out["W2"], out["b2"], state["ws"],
                              state["ws_bytes"])
    return {name: x for name, x in out.items() if x is not None}


def _embed_own(state):
    ee, cfg, out, n = state["lib"], state["cfg"], state["out"], state["case"]["rows"]
    ee.ee_forward(cfg, n, state["z"], state["T"], out["Y"])
    ee.ee_backward(cfg, n, state["z"], state["dY"], out["dT"], state["ws"], state["ws_bytes"])
    return out


def _clip_own(state):
    state["lib"].gc_clip(state["cfg"], state["tensors"], state["both"], state["ws"], state["ws_bytes"])
    return {"norm": state["both"][0], "coefficient": state["both"][1], "clipped": state["clipped"]}


# ---- the definition in 64 bits -------------------------------------------------------------------


def exact(case, seed):
    global own
    before, own = own, False      # inputs alone
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"dense": _dense_exact, "embed": _embed_exact, "clip": _clip_exact}[case["op"]](case, s)


def _act_exact(act, z):
    """act(z) from its definition; derivatives by differentiating this function."""
    if act == "none":
        return z
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    return 0.5 * z * (1 + torch.tanh(GELU_A * (z + GELU_B * z ** 3)))


def _slopes_exact(act, z):
    """act' and act'' at z by automatic differentiation, a slice of rows at a time."""
    if act in ("none", "relu"):
        first = torch.ones_like(z) if act == "none" else (z > 0).double()
        return first, torch.zeros_like(z)
    firsts, seconds = [], []
    for part in z.split(max(1, (1 << 25) // z.shape[1])):
        v = part.detach().clone().requires_grad_(True)
        one = torch.autograd.grad(_act_exact(act, v).sum(), v, create_graph=True)[0]
        seconds.append(torch.autograd.grad(one.sum(), v)[0].detach())
        firsts.append(one.detach())
    return torch.cat(firsts), torch.cat(seconds)


def _dense_exact(case, s):
    X, W = s["X"].double().contiguous(), s["W"].double()
    out, Z = {}, None
    if case["call"] in ("forward", "step"):
        Z = torch.matmul(X, W) if s["b"] is None else torch.addmm(s["b"].double(), X, W)
        out["Y"] = _act_exact(case["act"], Z)
        if "R" in s:
            out["Y"] = out["Y"] + s["R"].double()
        if _gated(case):
            out["Z"] = Z
    elif "Z" in s:
        Z = s["Z"].double()
    if case["call"] == "forward":
        return out
    dY = s["dY"].double()
    first, second = _slopes_exact(case["act"], Z) if _gated(case) else (None, None)
    G = dY if first is None else dY * first
    if case["call"] in ("backward", "step"):
        out["dX"] = torch.matmul(G, W.t().contiguous())
        out["dW"] = torch.matmul(X.t().contiguous(), G)
        if case["bias"]:
            out["db"] = G.sum(dim=0)
        return out
    HX = s["HX"].double().contiguous()
    V = torch.matmul(HX, W)
    out["ddY"] = V if first is None else V * first
    S = torch.zeros_like(V) if second is None else V * dY * second
    out["X2"] = torch.matmul(S, W.t().contiguous())
    out["W2"] = torch.matmul(torch.cat([X, HX]).t().contiguous(), torch.cat([S, G]))
    if case["bias"]:
        out["b2"] = S.sum(dim=0)
    return out


def _embed_exact(case, s):
    scale, T, z = 1 / math.sqrt(case["elements"]), s["T"].double(), s["z"].long()
    order = torch.argsort(z, stable=True)                 # rows of one index together, then sums of runs as segments
    counts = torch.bincount(z, minlength=case["elements"])
    dT = torch.segment_reduce(s["dY"].double()[order], "sum", lengths=counts, axis=0)
    return {"Y": scale * torch.index_select(T, 0, z), "dT": scale * dT}


def _clip_exact(case, s):
    flat = torch.cat([x.double() for x in s["buckets"].values()])
    norm = torch.linalg.vector_norm(flat)
    coefficient = torch.clamp(MAX_NORM / (norm + EPS), max=1.0)
    return {"norm": norm, "coefficient": coefficient, "clipped": list((flat * coefficient).split([x.numel() for x in s["buckets"].values()]))}
