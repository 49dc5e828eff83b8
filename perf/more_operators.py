"""Weights that belong to an element, and the update of weight matrices, as a list of timed cases.

A model around the symmetric contraction keeps a weight matrix per chemical element: the self connection of an interaction layer mixes the
channels of an atom by the matrix of the atom's element, order by order.  (The same product, with a type of site or an expert in the
element's place, is the layer of a mixture of experts.)  Its gradient is a batch of matrices, most of them small, and those are what an
optimizer with orthogonalised updates works on, together with the matrices of the dense layers.

  product  Y[i] = X[i] W[z_i] + residual[i],   dX[i] = dY[i] W[z_i]^T,   dW[z] = sum over the atoms with z_i = z of X[i]^T dY[i]
           an atom has `components` rows (2 l + 1 of order l); an index outside the elements (padding) has no product
           (gp_group: atoms in the order of their elements, once for a batch; gp_forward, gp_backward)
  update   M = mu M + G,  U = G + mu M,  X = U / (|U| + eps),  `steps` times X = a X + (b A + c A A) X with A = X X^T, on the shorter side;
           then W = (1 - rate decay) W - rate scale X, or X itself, for every matrix of a list                              (ou_step)

Ranges: 1 to 200 000 atoms of 1 to 1024 elements, 1 to 4096 columns, 1 to 7 components; lists of one to some hundred tensors, matrices
from 8 x 64 to some thousand on a side, batches of them.  fp32, fp64, bfloat16 rows or gradients (weights, their gradients in the product and
the momentum stay fp32 beside them, as everywhere in this library).
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
A, B, C = 3.4445, -4.7750, 2.0315
MU, RATE, DECAY, EPS = 0.95, 0.02, 0.01, 1e-7


# ---- the cases ---------------------------------------------------------------------------------


def _product(name, call, atoms, k_in, k_out, elements=ELEMENTS, components=1, spread=1, residual=False, padded=False, dtype="f32"):
    """spread: X and Y are the blocks of one order in rows of that many components.  padded: some indices are outside the elements."""
    return {"name": name, "op": "product", "call": call, "atoms": atoms, "k_in": k_in, "k_out": k_out, "elements": elements,
            "components": components, "spread": spread, "residual": residual, "padded": padded, "dtype": dtype}


def _model(name, layers, channels, elements=0, apply=True, steps=5, dtype="f32"):
    """All matrices of a model of `layers` layers; elements: with a self connection of that many elements in each."""
    return {"name": name, "op": "update", "layers": layers, "channels": channels, "elements": elements, "count": 0, "rows": 0, "cols": 0,
            "apply": apply, "steps": steps, "dtype": dtype}


def _matrices(name, count, rows, cols, apply=True, steps=5, dtype="f32"):
    return {"name": name, "op": "update", "layers": 0, "channels": 0, "elements": 0, "count": count, "rows": rows, "cols": cols,
            "apply": apply, "steps": steps, "dtype": dtype}


def listed():
    return [
        # one row by one of eight wide matrices, as an answer is made row by row: latency, and the bytes of one matrix
        _product("product_one_row", "forward", 1, 1024, 1024, elements=8, dtype="bf16"),
        # self connection of one small molecule: latency
        _product("product_one_molecule", "step", 61, 128, 128, residual=True),
        # self connection of a training step of 10 000 atoms, invariant channels, forward and backward
        _product("product_step", "step", 10_000, 128, 128, residual=True),
        # ... of the order l = 1 in [atom][component][channel] features of l <= 3, with padding at the end of some structures
        _product("product_vectors", "step", 49_999, 128, 128, components=3, spread=16, padded=True),
        # ... of the batch of 200 000 atoms, rows stored as bfloat16
        _product("product_200k_bf16", "step", 200_000, 128, 128, dtype="bf16"),
        # double precision, odd widths
        _product("product_odd_f64", "step", 3001, 96, 41, elements=10, dtype="f64"),
        # wide layer of 64 types of sites on bfloat16 rows, where the matrix cores count
        _product("product_wide_bf16", "step", 16_384, 1024, 2048, elements=64, dtype="bf16"),
        # the matrices of a model of two layers: latency
        _model("update_two_layers", 2, 128),
        # ... with the self connections of 89 elements in each layer: a batch of small matrices
        _model("update_elements", 2, 128, elements=ELEMENTS),
        # a deep and wide model, bfloat16 gradients
        _model("update_24_layers_bf16", 24, 512, dtype="bf16"),
        # one wide layer of odd sizes, the update itself
        _matrices("update_odd", 1, 1001, 2003, apply=False),
        # large square matrices, where the matrix cores count
        _matrices("update_large", 2, 4096, 4096),
    ]


def _log_size(rng, lo, hi):
    """A size spread evenly over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.6:
        dtype = rng.choices(["f32", "bf16", "f64"], [5, 4, 2])[0]
        k_in = rng.choice([64, 128, 128, 256, 1024, _log_size(rng, 1, 4096)])
        k_out = rng.choice([64, 128, 128, 512, 2048, _log_size(rng, 1, 4096)])
        elements = min(rng.choice([8, 64, ELEMENTS, ELEMENTS, _log_size(rng, 1, 1024)]), max(1, 134_000_000 // (k_in * k_out)))
        components = rng.choice([1, 1, 1, 3, 5, 7])
        spread = 16 if components > 1 or rng.random() < 0.2 else 1
        most = min(200_000, int(1e8 / (spread * (k_in + k_out))), int((1e9 if dtype == "f64" else 1e10) / (components * k_in * k_out)))
        case = _product("", rng.choice(["forward", "backward", "step", "step"]), _log_size(rng, 1, max(1, most)), k_in, k_out, elements=elements,
                        components=components, spread=spread, residual=rng.random() < 0.5, padded=rng.random() < 0.3, dtype=dtype)
    else:
        dtype = rng.choices(["f32", "bf16", "f64"], [5, 3, 1])[0]
        apply, steps = rng.random() < 0.6, rng.choice([1, 3, 5, 5, 5, 6])
        if rng.random() < 0.4:
            layers, channels = _log_size(rng, 1, 6 if dtype == "f64" else 24), rng.choice([64, 128, _log_size(rng, 16, 256 if dtype == "f64" else 512)])
            case = _model("", layers, channels, elements=rng.choice([0, ELEMENTS]) if layers * channels <= 512 else 0, apply=apply, steps=steps, dtype=dtype)
        else:
            rows, cols = (rng.choice([64, 128, 256, _log_size(rng, 1, 1500 if dtype == "f64" else 4000)]) for _ in range(2))
            cost = min(rows, cols) ** 2 * (4 * max(rows, cols) + 2 * min(rows, cols))
            most = max(1, min(200, int((3e10 if dtype == "f64" else 4e11) / cost), 16_000_000 // (rows * cols)))
            case = _matrices("", _log_size(rng, 1, most), rows, cols, apply=apply, steps=steps, dtype=dtype)
    del case["name"]
    return case


def _shapes(case):
    """(count, rows, columns) of the tensors of a list: four radial layers, the channel mixing of four orders, the readout, the self connection."""
    if case["count"]:
        return [(case["count"], case["rows"], case["cols"])]
    k = case["channels"]
    layer = [(1, 8, 64), (1, 64, 64), (1, 64, 64), (1, 64, 10 * k), (4, k, k), (1, k, 16)]
    return (layer + ([(case["elements"], k, k)] if case["elements"] else [])) * case["layers"]


def _views(case, flat):
    """The tensors of a list as views of one buffer."""
    shapes = _shapes(case)
    return [x.view(s) for x, s in zip(flat.split([math.prod(s) for s in shapes]), shapes)]


def _scale(shape):
    """The size of an update by the shape of its matrix [k_in][k_out]."""
    return math.sqrt(max(1.0, shape[2] / shape[1]))


def work(case):
    b, w = BYTES[case["dtype"]], WEIGHT_BYTES[case["dtype"]]
    if case["op"] == "update":
        n = sum(math.prod(s) for s in _shapes(case))
        step = sum(c * min(r, k) ** 2 * (3 * max(r, k) + min(r, k)) for c, r, k in _shapes(case))   # products of X X^T and A A: half of them are distinct
        return {"bytes": n * (b + 2 * w + (2 * w if case["apply"] else b)), "flops": case["steps"] * step + 10 * n}
    rows, ki, ko = case["atoms"] * case["components"], case["k_in"], case["k_out"]
    used = min(case["elements"], case["atoms"])
    product, x, y = 2 * rows * ki * ko, rows * ki * b, rows * ko * b
    forward = {"bytes": 4 * case["atoms"] + x + y * (1 + int(case["residual"])) + used * ki * ko * w, "flops": product}
    backward = {"bytes": 4 * case["atoms"] + 2 * x + y + (used + case["elements"]) * ki * ko * w, "flops": 2 * product}
    if case["call"] == "step":
        return {m: forward[m] + backward[m] for m in forward}
    return {"forward": forward, "backward": backward}[case["call"]]


# ---- inputs ------------------------------------------------------------------------------------


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape, scale=1.0: torch.randn(*shape, generator=g, device="cuda") * scale  # noqa: E731
    state = (_prepare_product if case["op"] == "product" else _prepare_update)(case, g, normal)
    state["case"] = case
    if own:
        _plan(state)
    return state


def _block(case, rows, k):
    """The block of one order, [atom][component][k], of rows [atom][spread][k]: order l = 1 begins at component 1."""
    first = 1 if case["spread"] > case["components"] else 0
    return rows[:, first:first + case["components"]]


def _prepare_product(case, g, normal):
    t, w = ROW_TYPE[case["dtype"]], WEIGHT_TYPE[case["dtype"]]
    n, ki, ko, z = case["atoms"], case["k_in"], case["k_out"], case["elements"]
    u = torch.rand(n, generator=g, device="cuda")
    index = torch.randint(0, z, (n,), generator=g, device="cuda")
    if z > 64:     # chemical elements: six dominant ones with a tenth of the atoms each
        dominant = torch.tensor([0, 5, 6, 7, 13, 25], device="cuda")
        index = torch.where(u < 0.6, dominant[(u * 10).long().clamp_(max=5)], index)
    if case["padded"]:
        index = torch.where(u > 0.97, -1, index)
    s = {"z": index.int(), "W": normal(z, ki, ko, scale=ki ** -0.5).to(w), "X": _block(case, normal(n, case["spread"], ki).to(t), ki)}
    if case["residual"] and case["call"] != "backward":
        s["R"] = _block(case, normal(n, case["spread"], ko).to(t), ko)
    if case["call"] != "forward":
        s["dY"] = _block(case, normal(n, case["spread"], ko).to(t), ko)
    return s


def _prepare_update(case, g, normal):
    # gradients, momenta and weights of a model are views of one buffer each, as the all-reduce of data-parallel training takes them
    t, w = ROW_TYPE[case["dtype"]], WEIGHT_TYPE[case["dtype"]]
    n = sum(math.prod(s) for s in _shapes(case))
    grad, momentum = normal(n, scale=1e-3), normal(n, scale=3e-3)
    for i, (x, m) in enumerate(zip(_views(case, grad), _views(case, momentum))):
        # rows and columns of different size, as the inputs and the upstream gradients of a layer make them; absent elements have no gradient yet
        x.mul_(torch.exp(normal(x.shape[0], x.shape[1], 1))).mul_(torch.exp(normal(x.shape[0], 1, x.shape[2])))
        if x.shape[0] == ELEMENTS:
            absent = torch.rand(ELEMENTS, 1, 1, generator=g, device="cuda") < 0.2
            x.masked_fill_(absent, 0.0)
            m.masked_fill_(absent, 0.0)
    s = {"grad": grad.to(t), "momentum": momentum.to(w)}
    if case["apply"]:
        s["weight"] = normal(n, scale=0.1).to(w)
    return s


# ---- one pass ----------------------------------------------------------------------------------


def run(state):
    forms = {"product": (_product_plain, _product_own), "update": (_update_plain, _update_own)}
    return forms[state["case"]["op"]][own](state)


def _product_plain(state):
    """Rows sorted by element, and a product for each element that is present (their numbers are read back, as its program has to)."""
    case, W = state["case"], state["W"]
    t, w, z = ROW_TYPE[case["dtype"]], WEIGHT_TYPE[case["dtype"]], state["z"].long()
    group = torch.where((z >= 0) & (z < case["elements"]), z, case["elements"])
    order = torch.argsort(group, stable=True)
    counts = torch.bincount(group, minlength=case["elements"] + 1).tolist()
    present = [e for e in range(case["elements"]) if counts[e]]
    split = lambda rows: rows[order].to(w).split(counts)  # noqa: E731

    def joined(parts, like):
        """The rows of the elements, in the order of the batch."""
        out = torch.zeros((case["atoms"], case["components"], parts[0].shape[2] if parts else like), dtype=w, device="cuda")
        if parts:
            out[order[:sum(p.shape[0] for p in parts)]] = torch.cat(parts)
        return out

    out, X = {}, split(state["X"])
    if case["call"] != "backward":
        Y = joined([X[e] @ W[e] for e in present], case["k_out"])
        out["Y"] = (Y + state["R"].to(w) if "R" in state else Y).to(t)
    if case["call"] != "forward":
        dY = split(state["dY"])
        out["dX"] = joined([dY[e] @ W[e].t() for e in present], case["k_in"]).to(t)
        dW = torch.zeros_like(W)
        if present:
            dW[torch.tensor(present, device="cuda")] = torch.stack([X[e].flatten(0, 1).t() @ dY[e].flatten(0, 1) for e in present])
        out["dW"] = dW
    return out


def _update_plain(state):
    case = state["case"]
    t, w = ROW_TYPE[case["dtype"]], WEIGHT_TYPE[case["dtype"]]
    G, M = state["grad"].to(w), state["momentum"]
    M.mul_(MU).add_(G)
    U = G + MU * M
    update = torch.empty_like(U)
    for shape, u, x in zip(_shapes(case), _views(case, U), _views(case, update)):
        X = (u / (u.double().square().sum((1, 2), keepdim=True).sqrt() + EPS)).to(w)
        X = X.transpose(1, 2) if shape[1] > shape[2] else X
        for _ in range(case["steps"]):
            S = X @ X.transpose(1, 2)
            X = A * X + (B * S + C * (S @ S)) @ X
        x.copy_((X.transpose(1, 2) if shape[1] > shape[2] else X) * (_scale(shape) if case["apply"] else 1.0))
    if not case["apply"]:
        return {"momentum": M, "update": update.to(t)}
    state["weight"].mul_(1 - RATE * DECAY).sub_(RATE * update)
    return {"momentum": M, "weight": state["weight"]}


# ---- the same from the definition, in 64 bits ----------------------------------------------------


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = kept
    return (_product_exact if case["op"] == "product" else _update_exact)(state)


def _product_exact(state):
    case, out = state["case"], {}
    z = state["z"].tolist()
    atoms = {}
    for i, e in enumerate(z):
        if 0 <= e < case["elements"]:
            atoms.setdefault(e, []).append(i)
    shape = (case["atoms"], case["components"])
    Y = state["R"].double() if "R" in state else torch.zeros(*shape, case["k_out"], dtype=torch.float64, device="cuda")
    dX = torch.zeros(*shape, case["k_in"], dtype=torch.float64, device="cuda")
    dW = torch.zeros(state["W"].shape, dtype=torch.float64, device="cuda")
    for e, mine in atoms.items():
        i = torch.tensor(mine, device="cuda")
        weight, x = state["W"][e].double(), state["X"][i].double().reshape(-1, case["k_in"])
        if case["call"] != "backward":
            Y[i] += torch.mm(x, weight).view(len(mine), case["components"], case["k_out"])
        if case["call"] != "forward":
            g = state["dY"][i].double().reshape(-1, case["k_out"])
            dX[i] = torch.mm(g, weight.t()).view(len(mine), case["components"], case["k_in"])
            dW[e] = torch.mm(x.t(), g)
    if case["call"] != "backward":
        out["Y"] = Y
    if case["call"] != "forward":
        out.update(dX=dX, dW=dW)
    return out


def _update_exact(state):
    """The polynomial of the singular values as a p(A) X with p(A) = a + b A + c A^2, matrix after matrix."""
    case = state["case"]
    G = state["grad"].double()
    M = MU * state["momentum"].double() + G
    U, out = G + MU * M, []
    for shape, batch in zip(_shapes(case), _views(case, U)):
        x = batch / (torch.linalg.vector_norm(batch, dim=(1, 2), keepdim=True) + EPS)
        turned = shape[1] > shape[2]
        x = x.transpose(1, 2).contiguous() if turned else x
        one = torch.eye(x.shape[1], dtype=torch.float64, device="cuda")
        for _ in range(case["steps"]):
            gram = torch.bmm(x, x.transpose(1, 2).contiguous())
            x = torch.bmm(A * one + torch.bmm(gram, B * one + C * gram), x)
        x = x.transpose(1, 2) if turned else x
        out.append((x * _scale(shape) if case["apply"] else x).reshape(-1))
    update = torch.cat(out)
    if not case["apply"]:
        return {"momentum": M, "update": update}
    return {"momentum": M, "weight": (1 - RATE * DECAY) * state["weight"].double() - RATE * update}


# ---- the same passes through the library ---------------------------------------------------------


def _plan(state):
    """What a program keeps beside its tensors: configuration, outputs, the buffer of the grouping, workspace."""
    case = state["case"]
    if case["op"] == "product":
        from paper_2504_10700_amd import gp_binding as gp
        kind = {"f32": gp.SC_F32, "f64": gp.SC_F64, "bf16": gp.SC_BF16}[case["dtype"]]
        n, ki, ko = case["atoms"], case["k_in"], case["k_out"]
        cfg = gp.make_config(case["elements"], ki, ko, components=case["components"], dtype=kind, ld_in=case["spread"] * ki, ld_out=case["spread"] * ko)
        rows = lambda k: _block(case, torch.empty((n, case["spread"], k), dtype=ROW_TYPE[case["dtype"]], device="cuda"), k)  # noqa: E731
        out = {}
        if case["call"] != "backward":
            out["Y"] = rows(ko)
        if case["call"] != "forward":
            out.update(dX=rows(ki), dW=torch.empty_like(state["W"]))
        grouping = torch.empty(max(gp.gp_grouping_bytes(cfg, n), 256), dtype=torch.uint8, device="cuda")
        nbytes = gp.gp_workspace_bytes(cfg, n)
        state.update(lib=gp, cfg=cfg, out=out, grouping=grouping)
    else:
        from paper_2504_10700_amd import ou_binding as ou
        kind = {"f32": ou.SC_F32, "f64": ou.SC_F64, "bf16": ou.SC_BF16}[case["dtype"]]
        cfg = ou.make_config(rate=RATE, momentum=MU, decay=DECAY, steps=case["steps"], eps=EPS, nesterov=True)
        result = state["weight"] if case["apply"] else torch.empty_like(state["grad"])
        views = {"weight" if case["apply"] else "update": _views(case, result)}
        tensors = ou.make_tensors(_views(case, state["grad"]), momentum=_views(case, state["momentum"]), scale=[_scale(s) for s in _shapes(case)], **views)
        nbytes = ou.ou_workspace_bytes(cfg, tensors)
        state.update(lib=ou, cfg=cfg, tensors=tensors, result=result)
    state["ws"], state["ws_bytes"] = torch.empty(max(nbytes, 256), dtype=torch.uint8, device="cuda"), nbytes


def _product_own(state):
    case, gp, cfg, out, n = state["case"], state["lib"], state["cfg"], state["out"], state["case"]["atoms"]
    z, grouping, ws, nbytes = state["z"], state["grouping"], state["ws"], state["ws_bytes"]
    gp.gp_group(cfg, n, z, grouping, grouping.numel())
    if case["call"] != "backward":
        gp.gp_forward(cfg, n, z, grouping, state["X"], state["W"], state.get("R"), out["Y"], ws, nbytes)
    if case["call"] != "forward":
        gp.gp_backward(cfg, n, z, grouping, state["X"], state["W"], state["dY"], out["dX"], out["dW"], ws, nbytes)
    return out


def _update_own(state):
    state["lib"].ou_step(state["cfg"], state["tensors"], state["ws"], state["ws_bytes"])
    return {"momentum": state["momentum"], "weight" if state["case"]["apply"] else "update": state["result"]}
