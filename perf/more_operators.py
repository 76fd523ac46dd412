"""Timing cases of the operators at the two ends of the sampling loop around the verifier.

A model's logits become candidates (over a token vocabulary, or over the physical registers themselves, under masks of occupied
registers), and the gradients that come out of the loss over their verdicts are bounded before they are applied:

* ``sample``  ``vl_token_sample``: one token a row from a given random number, with temperature, top-k, top-p and min-p, its log
              probability under the model and under what was kept, and how many entries were kept
* ``norm``    ``vl_grad_norm``: the global norm of many gradient tensors
* ``clip``    ``vl_clip_grads``: the norm, and the gradients with the loss scale taken out and the norm bounded

``run`` computes them in plain torch operations, or, where ``own`` is true, through the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_SLAB = 1 << 25                 # logits that the plain form takes at a time
MAX_LOGITS = 1 << 27            # of a drawn case: as many as the largest listed one has
MAX_GRADIENT = 3 << 26          # elements of a drawn case's gradients: fewer than the largest listed one has


def listed():
    return [
        # one decoding step of one sample
        dict(name="sample_1x131072_top_p", op="sample", rows=1, vocab=131072, dtype="bf16", scale=1.25, top_k=0, top_p=0.95, min_p=0.0),
        # one decoding step of the 100 samples of pass@100
        dict(name="sample_100x32768_top_k_top_p", op="sample", rows=100, vocab=32768, dtype="f16", scale=1.0, top_k=50, top_p=0.9,
             min_p=0.0),
        # temperature alone, a vocabulary of odd size: rows that start at any 4-byte boundary
        dict(name="sample_1009x50021", op="sample", rows=1009, vocab=50021, dtype="f32", scale=0.8, top_k=0, top_p=1.0, min_p=0.0),
        # one decoding step of many samples of many programs
        dict(name="sample_1024x131072_top_p", op="sample", rows=1024, vocab=131072, dtype="bf16", scale=1.0, top_k=0, top_p=0.95,
             min_p=0.0),
        # a head over registers, the smallest program: 64 definitions, 16 registers
        dict(name="sample_registers_64x16", op="sample", rows=64, vocab=16, dtype="f32", scale=1.0, top_k=4, top_p=1.0, min_p=0.05,
             masks=64, occupied=0.5, widths=False),
        # a head over registers: 2,000 definitions of a GEMM-shaped kernel, 100 samples, masks of the definitions, tuple widths
        dict(name="sample_registers_200000x256", op="sample", rows=200000, vocab=256, dtype="bf16", scale=1.0, top_k=0, top_p=1.0,
             min_p=0.02, masks=2000, occupied=0.6, widths=True),
        # the same for a kernel with 512 registers, its best sixteen registers and of these the likely ones
        dict(name="sample_registers_25000x512_top_k_top_p", op="sample", rows=25000, vocab=512, dtype="f32", scale=0.7, top_k=16,
             top_p=0.9, min_p=0.0, masks=2500, occupied=0.6, widths=True),
        # the gradient norm of a small head, watched during training
        dict(name="norm_head", op="norm", layers=1, width=96, head=256, dtype="f32", loss_scale=1.0, size=1.0),
        # of a model of 200 million parameters
        dict(name="norm_16x1024", op="norm", layers=16, width=1024, head=512, dtype="bf16", loss_scale=1.0, size=1.0),
        # clipping the small head's gradients
        dict(name="clip_head", op="clip", layers=1, width=96, head=256, dtype="f32", loss_scale=1.0, size=30.0),
        # of a model of 13 million parameters in fp16 halves under a loss scale, biases and norms in fp32
        dict(name="clip_4x512_f16", op="clip", layers=4, width=512, head=256, dtype="f16", loss_scale=4096.0, size=5.0),
        # of a model of 300 million parameters
        dict(name="clip_24x1024", op="clip", layers=24, width=1024, head=512, dtype="f32", loss_scale=1.0, size=3.0),
    ]


def draw(rng):
    op = rng.choice(["sample", "sample", "sample", "norm", "clip", "clip"])
    if op != "sample":
        n = _log_int(rng, 1, 400)
        total = _log_int(rng, 4 * n, MAX_GRADIENT)
        return dict(op=op, tensors=n, elements=total, shape_seed=rng.randrange(1 << 30), dtype=rng.choice(["f32", "f16", "bf16", "mixed"]),
                    loss_scale=rng.choice([1.0, 1.0, 256.0, 4096.0]), size=round(math.exp(rng.uniform(-1.0, 4.0)), 3))
    case = dict(op=op, dtype=rng.choice(["f32", "f16", "bf16"]), scale=round(rng.uniform(0.7, 1.6), 2))
    rules = rng.choice(["", "k", "p", "m", "kp", "pm", "kpm"])
    case["top_k"] = _log_int(rng, 1, 200) if "k" in rules else 0
    case["top_p"] = round(rng.uniform(0.5, 0.99), 3) if "p" in rules else 1.0
    case["min_p"] = round(math.exp(rng.uniform(math.log(0.005), math.log(0.3))), 4) if "m" in rules else 0.0
    if rng.random() < 0.45:     # registers
        case.update(vocab=_log_int(rng, 8, 1100), masks=_log_int(rng, 8, 4000), occupied=round(rng.uniform(0.1, 0.7), 2),
                    widths=rng.random() < 0.5)
        case["rows"] = _log_int(rng, 24, min(200000, MAX_LOGITS // 2 // case["vocab"]))
    else:
        case.update(vocab=_log_int(rng, 500, 200000), pad=rng.choice([0, 0, 8, 3, 64]))
        case["rows"] = _log_int(rng, 1, min(5000, MAX_LOGITS // (case["vocab"] + case["pad"])))
    return case


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    return _logit_inputs(case, seed) if case["op"] == "sample" else _gradient_inputs(case, seed)


def _logit_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 41)
    R, V, pad = case["rows"], case["vocab"], case.get("pad", 0)
    gpu = dict(generator=gen, device="cuda")
    store = torch.empty((R, V + pad), dtype=_TYPES[case["dtype"]], device="cuda")
    store.normal_(0.0, 2.0, generator=gen)
    x = store[:, :V]
    if not case.get("masks"):
        # a model's row: a few likely tokens, some dozens of possible ones, the rest far below; one row in fifty without favourites
        n = min(64, max(1, V // 8))
        at = torch.arange(n, device="cuda") * (V // n) + torch.randint(0, V // n, (R, n), **gpu)     # each another entry
        height = math.log(V) + 4.0 + 5.0 * torch.rand((R, 1), **gpu)
        height = torch.where(torch.rand((R, 1), **gpu) < 0.02, torch.zeros_like(height), height)
        fall = torch.empty((R, n), device="cuda").exponential_(0.4, generator=gen)
        lift = height * (1.0 - fall.clamp(max=20.0) / 20.0)
        x.scatter_(1, at, (x.gather(1, at).float() * 0.25 + lift).to(x.dtype))
    st = dict(case=case, x=x, uniform=torch.rand(R, **gpu), occupied=None, mask_rows=None, widths=None)
    if case.get("masks"):
        n, W = case["masks"], (V + 31) // 32
        share = torch.rand(n, 1, **gpu) * 0.4 + case["occupied"] - 0.2
        share[torch.rand(n, 1, **gpu) < 0.01] = 1.5       # definitions that no register is left for
        # occupied registers come in runs: tuples of live values
        runs = torch.rand(n, (V + 3) // 4, **gpu).repeat_interleave(4, dim=1)[:, :V]
        bits = torch.zeros((n, W * 32), dtype=torch.int64, device="cuda")
        bits[:, :V] = (runs < share).to(torch.int64)
        words = (bits.view(n, W, 32) << torch.arange(32, device="cuda")).sum(dim=2)
        st["occupied"] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
        row = torch.arange(R, device="cuda")
        st["mask_rows"] = (row % n).to(torch.int32)
        if case["widths"]:
            kinds = torch.tensor([1, 1, 1, 1, 1, 1, 1, 2, 2, 4], dtype=torch.uint8, device="cuda")
            st["widths"] = kinds[torch.randint(0, 10, (n,), **gpu)][row % n].contiguous()
    return st


def _shapes(case):
    """(elements, type) of every tensor."""
    if "layers" in case:        # projections, a feed-forward pair, biases and norms of every layer, a head over registers
        d, t, out = case["width"], case["dtype"], []
        for _ in range(case["layers"]):
            out += [(d * d, t)] * 4 + [(4 * d * d, t)] * 2 + [(4 * d, "f32"), (d, "f32"), (d, "f32"), (d, "f32")]
        return out + [(d * case["head"], t), (case["head"], "f32")]
    gen = torch.Generator().manual_seed(case["shape_seed"])     # the sizes belong to the case, the values to the seed
    share = torch.randn(case["tensors"], generator=gen, dtype=torch.float64).mul_(1.5).exp_()
    sizes = (share / share.sum() * case["elements"]).long().clamp_(min=1).tolist()
    kinds = torch.randint(0, 3, (case["tensors"],), generator=gen).tolist()
    return [(n, ["f32", "f16", "bf16"][k] if case["dtype"] == "mixed" else case["dtype"]) for n, k in zip(sizes, kinds)]


def _gradient_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 43)
    shapes = _shapes(case)
    total = sum(n for n, _ in shapes)
    # a global norm of about `size`, under the loss scale; tensors differ in how large their gradients are
    each = case["size"] * case["loss_scale"] / math.sqrt(total)
    weight = (0.5 * torch.randn(len(shapes), generator=gen, device="cuda")).exp().tolist()
    grads = []
    for (n, t), w in zip(shapes, weight):
        g = torch.empty(n, dtype=_TYPES[t], device="cuda")
        grads.append(g.normal_(0.0, min(each * w, 8000.0), generator=gen))
    st = dict(case=case, grads=grads, scale=1.0 / case["loss_scale"])
    if case["op"] == "clip":
        # the results are pieces of one buffer for each type, from 16 bytes to 16 bytes, as an optimiser keeps them
        st["flat"] = [torch.zeros(size, dtype=_TYPES[t], device="cuda") for t, (size, _) in _places(shapes).items()]
        st["outs"] = [None] * len(grads)
        for buffer, (_, pieces) in zip(st["flat"], _places(shapes).values()):
            for j, start in pieces:
                st["outs"][j] = buffer[start:start + shapes[j][0]]
    return st


def _places(shapes):
    """For each type the size of its buffer, and the tensors' numbers and where in it they begin."""
    out = {}
    for j, (n, t) in enumerate(shapes):
        size, pieces = out.get(t, (0, []))
        per = 16 // _BYTES[t]
        out[t] = (size + (n + per - 1) // per * per, pieces + [(j, size)])
    return out


_MAX_NORM = 1.0


# ---------------------------------------------------------------- the plain forms

def _closed(st, a, b):
    """Truth values [b - a, V]: entries of the rows a..b that are masked out; None where none is."""
    if st["occupied"] is None:
        return None
    V = st["case"]["vocab"]
    at = torch.arange(V, device="cuda", dtype=torch.int32)
    taken = ((st["occupied"][:, (at >> 5).long()] >> (at & 31)) & 1).bool()
    # a tuple of width w at i needs the next taken entry, or the end, to be w away
    nxt = torch.where(taken, at, torch.full_like(at, V)).flip(1).cummin(1).values.flip(1)
    room = nxt - at
    w = st["widths"][a:b].to(torch.int32)[:, None] if st["widths"] is not None else 1
    return room[st["mask_rows"][a:b].long()] < w


def _plain_sample(st):
    """The weights and their sums in 64 bits: tokens are decided at the borders between them."""
    case = st["case"]
    R, V, scale = case["rows"], case["vocab"], float(case["scale"])
    scale = float(torch.tensor(scale, dtype=torch.float32))     # what a 32-bit argument holds
    parts = []
    step = max(1, _SLAB // V)
    for a in range(0, R, step):
        b = min(R, a + step)
        x = st["x"][a:b].float()
        closed = _closed(st, a, b)
        if closed is not None:
            x = x.masked_fill(closed, -math.inf)
        top = x.amax(dim=1, keepdim=True)
        alive = top > -math.inf
        base = torch.where(alive, top, torch.zeros_like(top)).double()
        w = torch.exp((x.double() - base) * scale)
        total = w.sum(dim=1)
        # largest first, the lowest number first among equals
        best, order = torch.sort(x, dim=1, descending=True, stable=True)
        ws = w.gather(1, order)
        place = torch.arange(V, device="cuda")
        kept = best > -math.inf
        if case["top_k"]:
            kept &= place < case["top_k"]
        if case["top_p"] < 1.0:
            sums = torch.cumsum(torch.where(kept, ws, torch.zeros_like(ws)), dim=1)
            reached = sums >= case["top_p"] * sums[:, -1:]
            kept &= torch.cat([torch.zeros_like(reached[:, :1]), reached[:, :-1]], dim=1).logical_not()
        if case["min_p"] > 0.0:
            kept &= ws >= case["min_p"]
        count = kept.sum(dim=1)
        here = torch.zeros_like(kept).scatter_(1, order, kept)
        sums = torch.cumsum(torch.where(here, w, torch.zeros_like(w)), dim=1)
        T = sums[:, -1:]
        tok = torch.searchsorted(sums, st["uniform"][a:b, None].double() * T, right=True).clamp(max=V - 1)
        z = (x.gather(1, tok).double() - base) * scale
        ok = alive[:, 0]
        none = torch.full_like(total, -math.inf)
        parts.append([torch.where(ok, tok[:, 0], torch.full_like(count, -1)),
                      torch.where(ok, z[:, 0] - torch.log(total), none).float(),
                      torch.where(ok, z[:, 0] - torch.log(T[:, 0]), none).float(), count.to(torch.int32)])
    return tuple(torch.cat(c) for c in zip(*parts))


def _plain_norm(st):
    squares = [g.float().square().sum(dtype=torch.float64) for g in st["grads"]]
    return torch.sqrt(torch.stack(squares).sum()) * st["scale"]


def _plain_clip(st):
    norm = _plain_norm(st)
    factor = torch.where(norm > _MAX_NORM, _MAX_NORM / norm, torch.ones_like(norm))
    factor = torch.where(torch.isfinite(norm), factor, torch.zeros_like(factor))
    by = (factor * st["scale"]).float()
    for g, o in zip(st["grads"], st["outs"]):
        o.copy_((g.float() * by).to(o.dtype))
    return tuple(st["flat"]) + (norm.float(), factor.float())


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        if op == "norm":
            return _plain_norm(st).float()
        return _plain_sample(st) if op == "sample" else _plain_clip(st)
    from paper_2506_17506_b200 import binding as vl
    if op == "sample":
        out = vl.vl_token_sample(st["x"], st["uniform"], occupied=st["occupied"], mask_rows=st["mask_rows"], widths=st["widths"],
                                 scale=case["scale"], top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])
        return out.tokens, out.logprob, out.drawn_logprob, out.kept
    if op == "norm":
        return vl.vl_grad_norm(st["grads"], scale=st["scale"]).norm
    out = vl.vl_clip_grads(st["grads"], _MAX_NORM, scale=st["scale"], outs=st["outs"])
    return tuple(st["flat"]) + (out.norm, out.factor)


def work(case):
    if case["op"] == "sample":
        R, V = case["rows"], case["vocab"]
        words = case.get("masks", 0) * ((V + 31) // 32) * 4
        row = 4 + (4 if case.get("masks") else 0) + (1 if case.get("widths") else 0) + 8 + 4 + 4 + 4
        return {"bytes": R * V * _BYTES[case["dtype"]] + words + R * row, "flops": R * V * 6}
    shapes = _shapes(case)
    size = sum(n * _BYTES[t] for n, t in shapes)
    total = sum(n for n, _ in shapes)
    if case["op"] == "norm":
        return {"bytes": size + 4, "flops": 2 * total}
    return {"bytes": 2 * size + 8, "flops": 3 * total}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    return _exact_sample(st) if case["op"] == "sample" else _exact_gradients(st)


def _open_64(st, a, b):
    """Open entries of the rows a..b, tuple by tuple from the definition: register i + s is free for every s below the width."""
    V = st["case"]["vocab"]
    n = b - a
    free = torch.ones((n, V), dtype=torch.bool, device="cuda")
    if st["occupied"] is None:
        return free
    words = st["occupied"][st["mask_rows"][a:b].long()].long() & 0xFFFFFFFF
    free = (((words[:, :, None] >> torch.arange(32, device="cuda")) & 1) == 0).reshape(n, -1)[:, :V]
    if st["widths"] is None:
        return free
    w = st["widths"][a:b].long()[:, None]
    opened = free.clone()
    for s in range(1, int(w.max())):
        later = torch.zeros_like(free)
        if s < V:
            later[:, :V - s] = free[:, s:]
        opened &= later | (w <= s)
    return opened


def _exact_sample(st):
    """Without an order of the entries: the lowest logit that is kept is searched for by halves, among the numbers of a 32-bit type."""
    case = st["case"]
    R, V = case["rows"], case["vocab"]
    scale = float(torch.tensor(case["scale"], dtype=torch.float32))
    parts = []
    step = max(1, (1 << 25) // V)
    for a in range(0, R, step):
        b = min(R, a + step)
        x = st["x"][a:b].double()
        opened = _open_64(st, a, b)
        x[~opened] = -math.inf
        M = x.amax(dim=1, keepdim=True)
        dead = M == -math.inf
        M = torch.where(dead, torch.zeros_like(M), M)
        prob = torch.exp(scale * (x - M))
        bits = st["x"][a:b].float().add(0.0).view(torch.int32).long()
        rank = torch.where(bits < 0, -(bits & 0x7FFFFFFF) - 1, bits)          # ascends with the logit
        rank[x == -math.inf] = -(1 << 40)
        everything = prob.sum(dim=1, keepdim=True)

        def lowest(enough):
            """The highest rank for which enough(entries of at least that rank) holds."""
            lo, hi = torch.full((b - a, 1), -(1 << 32), device="cuda"), torch.full((b - a, 1), 1 << 32, device="cuda")
            for _ in range(34):
                mid = (lo + hi) >> 1
                ok = enough(rank >= mid)
                lo, hi = torch.where(ok, mid, lo), torch.where(ok, hi, mid)
            return lo

        def first_of(equal, m):
            """Of the entries that are marked, the first m of each row."""
            return equal & (torch.cumsum(equal.to(torch.int32), dim=1) <= m)

        chosen = rank > -(1 << 40)
        if case["top_k"]:
            cut = lowest(lambda s: s.sum(dim=1, keepdim=True) >= case["top_k"])
            above = rank > cut
            chosen = chosen & (above | first_of(rank == cut, case["top_k"] - above.sum(dim=1, keepdim=True)))
        if case["top_p"] < 1.0:
            among = torch.where(chosen, prob, torch.zeros_like(prob))
            need = case["top_p"] * among.sum(dim=1, keepdim=True)
            cut = lowest(lambda s: torch.where(s, among, torch.zeros_like(among)).sum(dim=1, keepdim=True) >= need)
            above = chosen & (rank > cut)
            lacks = need - torch.where(above, prob, torch.zeros_like(prob)).sum(dim=1, keepdim=True)
            level = torch.where(chosen & (rank == cut), prob, torch.zeros_like(prob)).amax(dim=1, keepdim=True)
            m = torch.ceil(lacks / torch.where(level > 0, level, torch.ones_like(level))).clamp(min=1)
            chosen = above | first_of(chosen & (rank == cut), m)
        if case["min_p"] > 0.0:
            chosen = chosen & (prob >= case["min_p"])
        count = chosen.sum(dim=1)
        part = torch.where(chosen, prob, torch.zeros_like(prob))
        T = part.sum(dim=1, keepdim=True)
        passed = torch.cumsum(part, dim=1) > st["uniform"][a:b, None].double() * T
        tok = passed.to(torch.uint8).argmax(dim=1, keepdim=True)
        z = scale * (x.gather(1, tok) - M)
        vals = [tok, z - torch.log(everything), z - torch.log(T)]
        vals = [torch.where(dead, torch.full_like(v, -1 if v is tok else -math.inf), v)[:, 0] for v in vals]
        parts.append(vals + [count.to(torch.int32)])
    return tuple(torch.cat(c) for c in zip(*parts))


def _exact_gradients(st):
    scale = st["scale"]
    norm = math.sqrt(math.fsum(float((g.double() * scale).square().sum()) for g in st["grads"]))
    gpu = dict(dtype=torch.float64, device="cuda")
    if st["case"]["op"] == "norm":
        return torch.tensor(norm, **gpu)
    factor = 0.0 if not math.isfinite(norm) else _MAX_NORM / norm if norm > _MAX_NORM else 1.0
    flat = [torch.zeros(b.shape, **gpu) for b in st["flat"]]
    for buffer, (_, pieces) in zip(flat, _places(_shapes(st["case"])).values()):
        for j, start in pieces:
            buffer[start:start + st["grads"][j].numel()] = st["grads"][j].double() * (scale * factor)
    return tuple(flat) + (torch.tensor(norm, **gpu), torch.tensor(factor, **gpu))
