"""The operators that training a synthesis net adds to the decoder, and the
calls of them whose speed and outputs are looked at:

  linear    pic.linear: y = act(x w^T + b) + residual, for one row to millions
  backward  pic.linear_backward: the gradients of x, w and b
  clip      pic.GradClip: the norm of many gradient tensors, and their clipping

Every case is a dict of plain values.  ``prepare`` makes the inputs of a case
on the GPU from a seed, ``run`` is one pass (the framework's call where ``own``
is true, elementary torch operations in fp32 where it is not), ``exact`` is the
definition in fp64 and ``work`` the bytes and operations a pass needs.
"""
import math
import random

import torch

own = False

_DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"fp32": 4, "fp16": 2, "bf16": 2}


def _linear(name, dtype, rows, inp, outp, act, bias=True, residual=False, train=False, pad=0, shift=0):
    # pad, shift: x is the columns [shift, shift + inp) of a tensor that is inp + pad wide
    return {"name": name, "op": "linear", "dtype": dtype, "rows": rows, "inp": inp, "outp": outp, "act": act,
            "bias": bias, "residual": residual, "train": train, "pad": pad, "shift": shift}


def _backward(name, dtype, rows, inp, outp, act, pad=0, shift=0):
    return {"name": name, "op": "backward", "dtype": dtype, "rows": rows, "inp": inp, "outp": outp, "act": act,
            "pad": pad, "shift": shift}


def _clip(name, kind, dtype, max_norm, **sizes):
    return {"name": name, "op": "clip", "kind": kind, "dtype": dtype, "max_norm": max_norm, **sizes}


def listed():
    return [
        # one row through an output projection: a net conditioned by one vector, latency and weight traffic
        _linear("linear_one_row", "bf16", 1, 4096, 4096, "none", residual=True),
        # a small batch through a widening layer
        _linear("linear_few_rows", "fp16", 24, 4096, 16384, "gelu"),
        # a training or prompt-sized batch through the same layer
        _linear("linear_many_rows", "bf16", 4096, 4096, 16384, "gelu"),
        # the hidden layer of the 7-64-64-3 net over one 768x512 image, keeping z for the backward pass
        _linear("linear_pixels", "fp16", 768 * 512, 64, 64, "relu", train=True),
        # sizes that fit no tile, x a slice of a wider tensor
        _linear("linear_odd", "bf16", 1021, 1111, 777, "gelu", residual=True, train=True, pad=5, shift=3),
        # a caller that wants fp32 weights and arithmetic
        _linear("linear_fp32", "fp32", 2048, 1024, 4096, "gelu"),
        # the gradient of a large layer
        _backward("backward_many_rows", "bf16", 4096, 4096, 8192, "gelu"),
        # the gradient of the hidden layer of 7-64-64-3 over one 768x512 image
        _backward("backward_pixels", "fp16", 768 * 512, 64, 64, "relu"),
        # the gradient of the hidden layer of 7-40-40-3 over a 256x256 crop in fp32
        _backward("backward_fp32", "fp32", 256 * 256, 40, 40, "gelu"),
        # the per-image nets of a 64-image batch: very many very small tensors
        _clip("clip_nets", "nets", "fp32", 1.0, images=64, levels=7, width=64),
        # two blocks of large matrices
        _clip("clip_layers", "layers", "bf16", 1.0, layers=2, width=4096, hidden=16384),
        # tensors of all sizes, of all three types, at odd offsets in their buffers
        _clip("clip_ragged", "ragged", "mixed", 0.5, count=1000, lo=1, hi=100000, sizes_seed=7),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# a drawn case needs no more operations or bytes than the largest listed one of its type
_MOST_FLOPS = {"fp32": 1.7e10, "fp16": 5.4e11, "bf16": 5.4e11}
_MOST_BYTES = {"fp32": 1.6e8, "fp16": 3.0e8, "bf16": 3.0e8}


def draw(rng):
    op = rng.choice(["linear", "linear", "backward", "clip"])
    if op == "clip":
        kind = rng.choice(["nets", "layers", "ragged"])
        max_norm = rng.choice([0.1, 1.0, 1e4])  # 1e4: nothing is clipped
        if kind == "nets":
            case = _clip("", kind, rng.choice(["fp32", "fp16"]), max_norm, images=_log(rng, 1, 128),
                         levels=rng.randint(2, 12), width=rng.choice([8, 16, 24, 32, 40, 64, 100, 128]))
        elif kind == "layers":
            width = _log(rng, 64, 4096)
            case = _clip("", kind, rng.choice(["fp32", "bf16"]), max_norm, layers=rng.randint(1, 2), width=width,
                         hidden=_log(rng, width, 4 * width if width < 2000 else 2 * width))
        else:
            case = _clip("", kind, "mixed", max_norm, count=_log(rng, 2, 1500), lo=1,
                         hi=_log(rng, 100, 100000), sizes_seed=rng.randint(0, 10**6))
        del case["name"]
        return case
    while True:
        dtype = rng.choice(["bf16", "fp16", "fp32"])
        act = rng.choice(["none", "relu", "gelu"])
        if rng.random() < 0.4:  # a layer of a synthesis net over an image
            rows = _log(rng, 4096, 2000000)
            inp, outp = rng.choice([rng.randint(3, 128), 16, 32, 40, 64]), rng.choice([rng.randint(3, 128), 16, 64])
        else:
            rows = _log(rng, 1, 16384)
            inp, outp = _log(rng, 200, 16384), _log(rng, 200, 16384)
            if rng.random() < 0.6:
                inp, outp = -(-inp // 64) * 64, -(-outp // 64) * 64
        if 3072 in (rows, inp, outp):
            continue
        pad = rng.choice([0, 0, 0, 8, rng.randint(1, 40)])
        shift = rng.randint(0, pad)
        if op == "linear":
            case = _linear("", dtype, rows, inp, outp, act, bias=rng.random() < 0.8, residual=rng.random() < 0.4,
                           train=rng.random() < 0.4, pad=pad, shift=shift)
        else:
            case = _backward("", dtype, rows, inp, outp, act, pad=pad, shift=shift)
        w = work(case)
        if w["flops"] <= _MOST_FLOPS[dtype] and w["bytes"] <= _MOST_BYTES[dtype]:
            del case["name"]
            return case


def _clip_layout(case):
    """(dtype, first element in that type's buffer, elements) of each tensor, and the buffers' sizes: a
    program's gradients are slices of one buffer for each type."""
    if case["kind"] == "nets":
        w = case["width"]
        per = [w * case["levels"], w, w * w, w, 3 * w, 3]
        shapes = [(n, case["dtype"], 0) for n in per * case["images"]]
    elif case["kind"] == "layers":
        w, h = case["width"], case["hidden"]
        per = [w * w] * 4 + [w * h, h, h * w, w, w, w]
        shapes = [(n, case["dtype"], 0) for n in per * case["layers"]]
    else:
        r = random.Random(case["sizes_seed"])
        shapes = [(_log(r, case["lo"], case["hi"]), r.choice(["fp32", "fp16", "bf16"]), r.randint(0, 9))
                  for _ in range(case["count"])]
    ends, places = {}, []
    for n, dtype, gap in shapes:
        first = ends.get(dtype, 0) + gap
        places.append((dtype, first, n))
        ends[dtype] = first + n
    return places, ends


def _slices(buffers, places):
    return [buffers[dtype][first:first + n] for dtype, first, n in places]


def _inputs(case, seed):
    """The tensors of a case, on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)

    if case["op"] == "clip":
        places, ends = _clip_layout(case)
        return {"places": places, "grads": {t: normal(n, 0.02, _DTYPES[t]) for t, n in ends.items()}}
    t = _DTYPES[case["dtype"]]
    M, K, N = case["rows"], case["inp"], case["outp"]
    wide = normal((M, K + case["pad"]), 1.0, t)
    s = {"x": wide[:, case["shift"]:case["shift"] + K], "w": normal((N, K), 1.4 / math.sqrt(K), t)}
    if case["op"] == "linear":
        s["b"] = normal((N,), 0.1, t) if case["bias"] else None
        s["r"] = normal((M, N), 1.0, t) if case["residual"] else None
    else:
        s["dy"] = normal((M, N), 0.02, t)
        s["z"] = normal((M, N), 1.4, t)  # x w^T + b of the forward pass
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "clip":
        # clipped gradients go to buffers of their own, so that every pass has the same gradients to clip
        s["out"] = {t: torch.zeros_like(g) for t, g in s["grads"].items()}
        s["from"], s["to"] = _slices(s["grads"], s["places"]), _slices(s["out"], s["places"])
        if own:
            from paper_2609_09020_gb300 import pic
            s["clip"] = pic.GradClip(s["from"], out=s["to"])
    return s


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return (0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
    return torch.ones_like(z)


def _plain(s):
    case = s["case"]
    if case["op"] == "clip":
        total = torch.zeros((), device="cuda")
        for g in s["from"]:
            f = g.float()
            total = total + (f * f).sum()
        norm = torch.sqrt(total)
        coef = torch.clamp(case["max_norm"] / (norm + 1e-6), max=1.0)
        for g, out in zip(s["from"], s["to"]):
            out.copy_(g.float() * coef)
        return {"norm": norm, "grads": s["out"]}
    x, w, t = s["x"].float(), s["w"].float(), s["w"].dtype
    if case["op"] == "linear":
        z = x @ w.t()
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z, case["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return {"y": y.to(t), "z": z.to(t)} if case["train"] else {"y": y.to(t)}
    dz = s["dy"].float() * _act_grad(s["z"].float(), case["act"])
    return {"dx": (dz @ w).to(t), "dw": (dz.t() @ x).to(t), "db": dz.sum(0).to(t)}


def run(state):
    if not own:
        return _plain(state)
    from paper_2609_09020_gb300 import pic
    case = state["case"]
    if case["op"] == "clip":
        norm = state["clip"].clip(case["max_norm"])
        return {"norm": norm, "grads": state["out"]}
    if case["op"] == "linear":
        if case["train"]:
            y, z = pic.linear(state["x"], state["w"], state["b"], act=case["act"], residual=state["r"],
                              save_pre=True)
            return {"y": y, "z": z}
        return {"y": pic.linear(state["x"], state["w"], state["b"], act=case["act"], residual=state["r"])}
    dx, dw, db = pic.linear_backward(state["dy"], state["x"], state["w"], act=case["act"], pre=state["z"])
    return {"dx": dx, "dw": dw, "db": db}


def exact(case, seed):
    """The definitions in fp64, a block of rows at a time."""
    s = _inputs(case, seed)
    if case["op"] == "clip":
        mine = {t: torch.zeros_like(g, dtype=torch.bool) for t, g in s["grads"].items()}
        for m in _slices(mine, s["places"]):
            m.fill_(True)
        kept = {t: torch.where(mine[t], g.double(), 0.0) for t, g in s["grads"].items()}
        norm = math.sqrt(sum(float(torch.linalg.vecdot(g, g)) for g in kept.values()))
        coef = min(1.0, case["max_norm"] / (norm + 1e-6))
        return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": {t: g * coef for t, g in kept.items()}}
    phi = torch.distributions.Normal(0.0, 1.0, validate_args=False)
    x, w, act = s["x"].double(), s["w"].double(), case["act"]
    step = 65536
    if case["op"] == "linear":
        y = torch.empty((case["rows"], case["outp"]), dtype=torch.float64, device="cuda")
        z = torch.empty_like(y) if case["train"] else None
        for i in range(0, case["rows"], step):
            v = torch.einsum("mk,nk->mn", x[i:i + step], w)
            if s["b"] is not None:
                v += s["b"].double()[None, :]
            if z is not None:
                z[i:i + step] = v
            if act == "relu":
                v = torch.where(v > 0, v, torch.zeros_like(v))
            elif act == "gelu":
                v = v * torch.special.ndtr(v)
            if s["r"] is not None:
                v = v + s["r"][i:i + step].double()
            y[i:i + step] = v
        return {"y": y, "z": z} if case["train"] else {"y": y}
    dx = torch.empty((case["rows"], case["inp"]), dtype=torch.float64, device="cuda")
    dw = torch.zeros((case["outp"], case["inp"]), dtype=torch.float64, device="cuda")
    db = torch.zeros((case["outp"],), dtype=torch.float64, device="cuda")
    for i in range(0, case["rows"], step):
        z = s["z"][i:i + step].double()
        d = s["dy"][i:i + step].double()
        if act == "relu":
            d = torch.where(z > 0, d, torch.zeros_like(d))
        elif act == "gelu":
            d = d * (torch.special.ndtr(z) + z * torch.exp(phi.log_prob(z)))
        dx[i:i + step] = torch.einsum("mn,nk->mk", d, w)
        dw += torch.einsum("mn,mk->nk", d, x[i:i + step])
        db += torch.einsum("mn->n", d)
    return {"dx": dx, "dw": dw, "db": db}


def work(case):
    if case["op"] == "clip":
        places, _ = _clip_layout(case)
        return {"bytes": sum(2 * n * _BYTES[t] for t, _, n in places) + 4, "flops": sum(3 * n for _, _, n in places)}
    e, M, K, N = _BYTES[case["dtype"]], case["rows"], case["inp"], case["outp"]
    if case["op"] == "linear":
        extra = N * case["bias"] + M * N * (case["residual"] + case["train"])
        return {"bytes": e * (M * K + N * K + M * N + extra), "flops": 2 * M * N * K}
    z = M * N if case["act"] != "none" else 0
    return {"bytes": e * (M * N + z + 2 * M * K + 2 * N * K + N), "flops": 4 * M * N * K}
