"""The operators that training many nets at once adds beside one linear layer, and
the calls of them whose speed and outputs are looked at:

  linear    pic.grouped_linear: y = act(x w_g^T + b_g) for rows sorted by group,
            group g's rows being [offsets[g], offsets[g + 1])
  backward  pic.grouped_linear_backward: the gradients of x, w and b
  orth      pic.Orthogonalizer: an update of every matrix of a list with its singular
            values drawn to about one, by Newton-Schulz products

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
_STEPS, _COEFFICIENTS, _EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def _grouped(name, op, dtype, groups, rows, inp, outp, act, spread="ragged", train=False, bias=True, pad=0, shift=0,
             sizes_seed=1):
    # spread: how the rows go to the groups ("even", "ragged", "few": some groups have none)
    # pad, shift: x is the columns [shift, shift + inp) of a tensor that is inp + pad wide
    return {"name": name, "op": op, "dtype": dtype, "groups": groups, "rows": rows, "inp": inp, "outp": outp,
            "act": act, "spread": spread, "train": train, "bias": bias, "pad": pad, "shift": shift,
            "sizes_seed": sizes_seed}


def _orth(name, kind, dtype, **sizes):
    return {"name": name, "op": "orth", "kind": kind, "dtype": dtype, **sizes}


def listed():
    return [
        # the hidden layer of 24 images' own 7-64-64-3 nets, images of different sizes, keeping z for the gradient
        _grouped("grouped_nets_pixels", "linear", "fp16", 24, 1000000, 64, 64, "relu", train=True),
        # the hidden layer of 64 images' 7-40-40-3 nets over a 32x32 crop each, in fp32
        _grouped("grouped_nets_fp32", "linear", "fp32", 64, 64 * 1024, 40, 40, "gelu", spread="even", train=True),
        # eight wide layers that share a training batch's rows unevenly
        _grouped("grouped_many_rows", "linear", "bf16", 8, 8192, 4096, 4096, "gelu"),
        # single rows for many wide layers, some without any: weight traffic
        _grouped("grouped_few_rows", "linear", "bf16", 64, 96, 2048, 4096, "none", spread="few"),
        # sizes that fit no tile, x a slice of a wider tensor
        _grouped("grouped_odd", "linear", "fp16", 37, 3001, 333, 517, "gelu", train=True, pad=5, shift=3),
        # the gradient of the first case's layers
        _grouped("grouped_backward_pixels", "backward", "fp16", 24, 1000000, 64, 64, "relu"),
        # the gradient of the wide layers
        _grouped("grouped_backward_many_rows", "backward", "bf16", 8, 8192, 4096, 4096, "gelu"),
        # the gradient of middling layers in fp32
        _grouped("grouped_backward_fp32", "backward", "fp32", 16, 4096, 256, 512, "gelu"),
        # the weight gradients of 64 images' 7-64-64-3 nets
        _orth("orth_nets", "nets", "fp32", images=64, levels=7, width=64),
        # one square fp32 matrix: a chain of dependent products
        _orth("orth_one", "layers", "fp32", count=1, width=1024, hidden=0),
        # the matrices of a wide block
        _orth("orth_layers", "layers", "bf16", count=4, width=2048, hidden=8192),
        # matrices of all shapes and of all three types
        _orth("orth_odd", "ragged", "mixed", count=24, lo=8, hi=1500, sizes_seed=7),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# a drawn case needs no more operations or bytes than the largest listed one of its kind and type
_MOST_FLOPS = {"fp32": 1.0e11, "fp16": 5.4e11, "bf16": 5.4e11}
_MOST_BYTES = {"fp32": 8.0e8, "fp16": 1.0e9, "bf16": 1.0e9}
_MOST_ORTH = 2.0e12


def draw(rng):
    while True:
        op = rng.choice(["linear", "linear", "backward", "backward", "orth"])
        if op == "orth":
            kind = rng.choice(["nets", "layers", "ragged"])
            if kind == "nets":
                case = _orth("", kind, rng.choice(["fp32", "fp16"]), images=_log(rng, 1, 128), levels=rng.randint(2, 12),
                             width=rng.choice([8, 16, 24, 32, 40, 64, 100, 128]))
            elif kind == "layers":
                width = _log(rng, 96, 2048)
                case = _orth("", kind, rng.choice(["fp32", "bf16", "bf16"]), count=rng.randint(1, 4), width=width,
                             hidden=rng.choice([0, _log(rng, width, 4 * width)]))
            else:
                case = _orth("", kind, "mixed", count=_log(rng, 2, 40), lo=1, hi=_log(rng, 40, 1500),
                             sizes_seed=rng.randint(0, 10**6))
            if work(case)["flops"] > _MOST_ORTH:
                continue
        else:
            dtype = rng.choice(["bf16", "fp16", "fp32"])
            act = rng.choice(["none", "relu", "gelu"])
            groups = _log(rng, 1, 128)
            if rng.random() < 0.4:  # layers of images' nets
                rows = _log(rng, 4096, 1500000)
                inp, outp = rng.choice([rng.randint(3, 128), 16, 32, 40, 64]), rng.choice([rng.randint(3, 128), 16, 64])
                spread = rng.choice(["ragged", "even"])
            else:
                rows = _log(rng, 1, 16384)
                inp, outp = _log(rng, 130, 8192), _log(rng, 130, 8192)
                if rng.random() < 0.6:
                    inp, outp = -(-inp // 64) * 64, -(-outp // 64) * 64
                spread = rng.choice(["ragged", "ragged", "even", "few"])
            pad = rng.choice([0, 0, 0, 8, rng.randint(1, 40)])
            case = _grouped("", op, dtype, groups, rows, inp, outp, act, spread=spread,
                            train=op == "linear" and rng.random() < 0.4, bias=op == "backward" or rng.random() < 0.8,
                            pad=pad, shift=rng.randint(0, pad), sizes_seed=rng.randint(0, 10**6))
            w = work(case)
            if w["flops"] > _MOST_FLOPS[dtype] or w["bytes"] > _MOST_BYTES[dtype]:
                continue
        del case["name"]
        return case


def _offsets(case):
    """The groups' first rows, and the end: all rows belong to a group."""
    r = random.Random(case["sizes_seed"])
    G, M = case["groups"], case["rows"]
    if case["spread"] == "even":
        share = [1.0] * G
    elif case["spread"] == "ragged":
        share = [r.uniform(0.1, 2.0) for _ in range(G)]
    else:  # every row by itself to one of a random half of the groups
        used = r.sample(range(G), -(-G // 2))
        share = [0] * G
        for _ in range(M):
            share[r.choice(used)] += 1
    ends, total = [0], 0.0
    for s in share:
        total += s
        ends.append(int(round(M * total / sum(share))))
    return ends


def _shapes(case):
    """(dtype, rows, columns) of each matrix."""
    if case["kind"] == "nets":
        w = case["width"]
        return [(case["dtype"], r, c) for _ in range(case["images"]) for r, c in ((w, case["levels"]), (w, w), (3, w))]
    if case["kind"] == "layers":
        w, h = case["width"], case["hidden"]
        return [(case["dtype"], r, c) for r, c in [(w, w)] * case["count"] + ([(h, w), (w, h)] if h else [])]
    r = random.Random(case["sizes_seed"])
    return [(r.choice(["fp32", "fp16", "bf16"]), _log(r, case["lo"], case["hi"]), _log(r, case["lo"], case["hi"]))
            for _ in range(case["count"])]


def _matrices(buffers, shapes):
    """The matrices that lie one behind another in their types' buffers."""
    at, out = dict.fromkeys(buffers, 0), []
    for t, r, c in shapes:
        out.append(buffers[t][at[t]:at[t] + r * c].view(r, c))
        at[t] += r * c
    return out


def _inputs(case, seed):
    """The tensors of a case, on the GPU, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(shape, std, dtype):
        return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)

    if case["op"] == "orth":
        # a program's gradients are slices of one buffer for each type
        shapes = _shapes(case)
        buffers = {t: torch.empty(sum(r * c for u, r, c in shapes if u == t), dtype=_DTYPES[t], device="cuda")
                   for t in sorted({t for t, _, _ in shapes})}
        grads = _matrices(buffers, shapes)
        for g in grads:
            r, c = g.shape
            # a weight gradient: few directions that most samples share, and what is left of each
            k = min(r, c, 16)
            few = normal((r, k), 1.0, torch.float32) @ normal((k, c), 1.0, torch.float32)
            g.copy_((few / math.sqrt(k) + normal((r, c), 0.5, torch.float32)) * 0.01)
        return {"grads": grads}
    t = _DTYPES[case["dtype"]]
    G, M, K, N = case["groups"], case["rows"], case["inp"], case["outp"]
    wide = normal((M, K + case["pad"]), 1.0, t)
    s = {"x": wide[:, case["shift"]:case["shift"] + K], "w": normal((G, N, K), 1.4 / math.sqrt(K), t),
         "ends": _offsets(case)}
    s["offsets"] = torch.tensor(s["ends"], dtype=torch.int64, device="cuda")
    if case["op"] == "linear":
        s["b"] = normal((G, N), 0.1, t) if case["bias"] else None
    else:
        s["dy"] = normal((M, N), 0.02, t)
        s["z"] = normal((M, N), 1.4, t) if case["act"] != "none" else None  # x w^T + b of the forward pass
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "orth":
        # updates go to tensors of their own, so that every pass has the same gradients
        shapes = _shapes(case)
        s["out"] = {t: torch.zeros(sum(r * c for u, r, c in shapes if u == t), dtype=_DTYPES[t], device="cuda")
                    for t in sorted({t for t, _, _ in shapes})}
        s["to"] = _matrices(s["out"], shapes)
        if own:
            from paper_2609_09020_gb300 import pic
            s["orth"] = pic.Orthogonalizer(s["grads"], out=s["to"])
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
    return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain(s):
    case = s["case"]
    if case["op"] == "orth":
        a, b, c = _COEFFICIENTS
        for g, out in zip(s["grads"], s["to"]):
            x = g.float()
            x = x / (torch.sqrt((x * x).sum()) + _EPS)
            if g.shape[0] > g.shape[1]:
                x = x.t()
            for _ in range(_STEPS):
                p = x @ x.t()
                x = a * x + (b * p + c * (p @ p)) @ x
            out.copy_(x.t() if g.shape[0] > g.shape[1] else x)
        return {"out": s["out"]}
    M, K, N, t = case["rows"], case["inp"], case["outp"], s["w"].dtype
    blocks = [(g, i, j) for g, (i, j) in enumerate(zip(s["ends"], s["ends"][1:]))]
    if case["op"] == "linear":
        y = torch.empty((M, N), dtype=t, device="cuda")
        pre = torch.empty((M, N), dtype=t, device="cuda") if case["train"] else None
        for g, i, j in blocks:
            if j > i:
                z = s["x"][i:j].float() @ s["w"][g].float().t()
                if s["b"] is not None:
                    z = z + s["b"][g].float()
                if pre is not None:
                    pre[i:j] = z
                y[i:j] = _act(z, case["act"])
        return {"y": y, "z": pre} if case["train"] else {"y": y}
    dx = torch.empty((M, K), dtype=t, device="cuda")
    dw = torch.zeros((case["groups"], N, K), dtype=t, device="cuda")
    db = torch.zeros((case["groups"], N), dtype=t, device="cuda")
    for g, i, j in blocks:
        if j > i:
            dz = s["dy"][i:j].float()
            if case["act"] != "none":
                dz = dz * _act_grad(s["z"][i:j].float(), case["act"])
            dx[i:j] = dz @ s["w"][g].float()
            dw[g] = dz.t() @ s["x"][i:j].float()
            db[g] = dz.sum(0)
    return {"dx": dx, "dw": dw, "db": db}


def run(state):
    if not own:
        return _plain(state)
    from paper_2609_09020_gb300 import pic
    case = state["case"]
    if case["op"] == "orth":
        state["orth"].orthogonalize(steps=_STEPS, coefficients=_COEFFICIENTS, eps=_EPS)
        return {"out": state["out"]}
    x, w, offsets = state["x"], state["w"], state["offsets"]
    if case["op"] == "linear":
        if case["train"]:
            y, z = pic.grouped_linear(x, w, offsets, state["b"], act=case["act"], save_pre=True)
            return {"y": y, "z": z}
        return {"y": pic.grouped_linear(x, w, offsets, state["b"], act=case["act"])}
    dx, dw, db = pic.grouped_linear_backward(state["dy"], x, w, offsets, act=case["act"], pre=state["z"])
    return {"dx": dx, "dw": dw, "db": db}


def exact(case, seed):
    """The definitions in fp64, a block of a group's rows at a time."""
    s = _inputs(case, seed)
    if case["op"] == "orth":
        a, b, c = _COEFFICIENTS
        done = {}
        for (t, _, _), g in zip(_shapes(case), s["grads"]):
            x = g.double()
            x /= torch.linalg.vector_norm(x) + _EPS
            for _ in range(_STEPS):
                # on the side with fewer products: (a + b X X^T + c (X X^T)^2) X = X (a + b X^T X + c (X^T X)^2)
                left = x.shape[0] <= x.shape[1]
                p = torch.einsum("ij,kj->ik", x, x) if left else torch.einsum("ji,jk->ik", x, x)
                q = b * p + c * torch.mm(p, p)
                q.diagonal().add_(a)
                x = torch.mm(q, x) if left else torch.mm(x, q)
            done.setdefault(t, []).append(x.reshape(-1))
        return {"out": {t: torch.cat(done[t]) for t in sorted(done)}}
    phi = torch.distributions.Normal(0.0, 1.0, validate_args=False)
    M, K, N, act = case["rows"], case["inp"], case["outp"], case["act"]
    lens = torch.diff(s["offsets"])
    step, new = 65536, {"dtype": torch.float64, "device": "cuda"}
    pieces, first = [], 0
    for g, n in enumerate(lens.tolist()):
        pieces += [(g, slice(i, min(i + step, first + n))) for i in range(first, first + n, step)]
        first += n
    if case["op"] == "linear":
        y = torch.empty((M, N), **new)
        pre = torch.empty((M, N), **new) if case["train"] else None
        for g, at in pieces:
            v = torch.einsum("mk,nk->mn", s["x"][at].double(), s["w"][g].double())
            if s["b"] is not None:
                v += s["b"][g].double()[None, :]
            if pre is not None:
                pre[at] = v
            if act == "relu":
                v = torch.where(v > 0, v, torch.zeros_like(v))
            elif act == "gelu":
                v = v * torch.special.ndtr(v)
            y[at] = v
        return {"y": y, "z": pre} if case["train"] else {"y": y}
    dx = torch.empty((M, K), **new)
    dw, db = torch.zeros((case["groups"], N, K), **new), torch.zeros((case["groups"], N), **new)
    for g, at in pieces:
        d = s["dy"][at].double()
        if act == "relu":
            d = torch.where(s["z"][at] > 0, d, torch.zeros_like(d))
        elif act == "gelu":
            z = s["z"][at].double()
            d = d * (torch.special.ndtr(z) + z * torch.exp(phi.log_prob(z)))
        dx[at] = torch.einsum("mn,nk->mk", d, s["w"][g].double())
        dw[g] += torch.einsum("mn,mk->nk", d, s["x"][at].double())
        db[g] += torch.einsum("mn->n", d)
    return {"dx": dx, "dw": dw, "db": db}


def work(case):
    if case["op"] == "orth":
        # with m <= n the sides: a step is X X^T and its square, both symmetric, and a product with X
        sides = [(t, min(r, c), max(r, c)) for t, r, c in _shapes(case)]
        return {"bytes": sum(2 * m * n * _BYTES[t] for t, m, n in sides),
                "flops": _STEPS * sum(3 * m * m * n + m * m * m for _, m, n in sides)}
    e, M, K, N = _BYTES[case["dtype"]], case["rows"], case["inp"], case["outp"]
    ends = _offsets(case)
    used = sum(j > i for i, j in zip(ends, ends[1:]))  # groups whose weights are read
    if case["op"] == "linear":
        return {"bytes": e * (M * K + used * N * (K + case["bias"]) + M * N * (1 + case["train"])) + 8 * len(ends),
                "flops": 2 * M * N * K}
    z = M * N if case["act"] != "none" else 0
    return {"bytes": e * (M * N + z + 2 * M * K + used * N * K + case["groups"] * N * (K + 1)) + 8 * len(ends),
            "flops": 4 * M * N * K}
