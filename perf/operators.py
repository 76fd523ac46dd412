"""Timing cases of the operators that score and train the model behind the candidates.

A user of the verifier has logits of a model (over a token vocabulary, or over the physical registers themselves), the
tokens that were sampled from them, and the verdicts.  Three operators work on these:

* ``score``   ``vl_token_logprobs``: log probability of the given token of every row, entropy, and the best alternatives,
              with occupied registers masked out
* ``grad``    ``vl_token_logprobs_backward``: its gradient to the logits
* ``policy``  ``vl_policy_loss``: verdicts to rewards, advantages within each program's samples, the clipped objective over
              ragged samples and its derivative to every token's log probability

``run`` computes them in plain torch operations, or, where ``own`` is true, through the framework's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "f16": 2, "bf16": 2}
_SLAB = 1 << 27                 # elements of logits that the plain form and the 64-bit one take at a time
MAX_ELEMENTS = 1 << 28          # logits of a drawn case: fewer than the largest listed one has
MAX_TOKENS = 16_000_000


def listed():
    return [
        # one decoding step of one sample: alternatives of one token; a launch and a row that one block would be slow on
        dict(name="score_1x131072", op="score", rows=1, vocab=131072, dtype="bf16", scale=1.25, top=20, tokens="i64"),
        # one decoding step of the 100 samples of pass@100
        dict(name="score_100x32768_top5", op="score", rows=100, vocab=32768, dtype="f16", scale=1.0, top=5, tokens="i64"),
        # the tokens of a sampled dictionary under a vocabulary of odd size: rows that start at any 4-byte boundary
        dict(name="score_1009x50021", op="score", rows=1009, vocab=50021, dtype="f32", scale=1.0, top=0, tokens="i32"),
        # the training step's forward half
        dict(name="score_4096x131072", op="score", rows=4096, vocab=131072, dtype="bf16", scale=1.0, top=0, tokens="i64"),
        # a head over registers, the smallest program: 64 definitions, 16 registers
        dict(name="score_registers_64x16", op="score", rows=64, vocab=16, dtype="f32", scale=1.0, top=4, tokens="u16",
             masks=64, occupied=0.5, widths=False),
        # a head over registers: 2,000 definitions of a GEMM-shaped kernel, 100 samples, masks of the definitions, tuple widths
        dict(name="score_registers_200000x256", op="score", rows=200000, vocab=256, dtype="bf16", scale=1.0, top=0, tokens="u16",
             masks=2000, occupied=0.6, widths=True),
        # the same with its best four registers, for a kernel with 512 registers
        dict(name="score_registers_25000x512_top4", op="score", rows=25000, vocab=512, dtype="f32", scale=0.5, top=4, tokens="u16",
             masks=2500, occupied=0.6, widths=True),
        # the backward halves of the same steps
        dict(name="grad_333x50021", op="grad", rows=333, vocab=50021, dtype="f16", scale=1.0, tokens="i64", entropy=False),
        dict(name="grad_4096x131072", op="grad", rows=4096, vocab=131072, dtype="bf16", scale=1.0, tokens="i64", entropy=True),
        dict(name="grad_registers_200000x256", op="grad", rows=200000, vocab=256, dtype="bf16", scale=1.0, tokens="u16",
             masks=2000, occupied=0.6, widths=True, entropy=True),
        # the loss over the 100 samples of one kernel, samples as long as a GEMM's allocation is on average
        dict(name="policy_1x100", op="policy", programs=1, samples=100, tokens=113, spread=0.3, fails=0.15, normalise=True,
             per_token=False, ref=False),
        # over 10,000 samples of one kernel as long as an attention kernel's allocation, kept near a reference model
        dict(name="policy_1x10000_ref", op="policy", programs=1, samples=10000, tokens=1944, spread=0.5, fails=0.05, normalise=True,
             per_token=True, ref=True),
    ]


def draw(rng):
    op = rng.choice(["score", "score", "grad", "grad", "policy"])
    if op == "policy":
        programs = _log_int(rng, 1, 300)
        samples = _log_int(rng, 4, min(10000, 200000 // programs))
        tokens = _log_int(rng, 4, max(1, min(9000, MAX_TOKENS // (2 * programs * samples))))
        return dict(op=op, programs=programs, samples=samples, tokens=tokens, spread=round(rng.uniform(0.0, 0.8), 2),
                    fails=round(rng.uniform(0.0, 0.6), 2), normalise=rng.random() < 0.7, per_token=rng.random() < 0.5,
                    ref=rng.random() < 0.4)
    case = dict(op=op, dtype=rng.choice(["f32", "f16", "bf16"]), scale=round(rng.uniform(0.4, 2.0), 2))
    if rng.random() < 0.45:     # registers
        case.update(vocab=_log_int(rng, 8, 1100), tokens="u16", masks=_log_int(rng, 8, 4000), occupied=round(rng.uniform(0.1, 0.7), 2),
                    widths=rng.random() < 0.5)
        top_rows = min(200000, MAX_ELEMENTS // 4 // case["vocab"])
    else:
        case.update(vocab=_log_int(rng, 500, 200000), tokens=rng.choice(["i32", "i64"]), pad=rng.choice([0, 0, 8, 3, 64]))
        top_rows = min(20000, MAX_ELEMENTS // (case["vocab"] + case["pad"]))
    case["rows"] = _log_int(rng, 24 if case["tokens"] == "u16" else 1, top_rows)
    if op == "score":
        case["top"] = rng.choice([0, 0, 1, 3, 8, 20, 32])
    else:
        case["entropy"] = rng.random() < 0.5
    return case


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    return _policy_inputs(case, seed) if case["op"] == "policy" else _logit_inputs(case, seed)


def _logit_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 17)
    R, V, pad = case["rows"], case["vocab"], case.get("pad", 0)
    store = torch.empty((R, V + pad), dtype=_TYPES[case["dtype"]], device="cuda")
    store.normal_(0.0, 2.0, generator=gen)
    x = store[:, :V]
    tok = torch.randint(0, V, (R,), generator=gen, device="cuda")
    # a sampled token is a likely one more often than not
    lift = torch.rand(R, generator=gen, device="cuda") * 12.0
    row = torch.arange(R, device="cuda")
    x[row, tok] = (x[row, tok].float() + lift).to(x.dtype)
    tok[torch.rand(R, generator=gen, device="cuda") < 0.01] = 65535 if case["tokens"] == "u16" else -1    # rows that do not count
    st = dict(case=case, x=x, tokens=tok, occupied=None, mask_rows=None, widths=None)
    if case["tokens"] == "u16":
        st["tokens"] = tok.to(torch.int32).to(torch.uint16)
    elif case["tokens"] == "i32":
        st["tokens"] = tok.to(torch.int32)
    if case.get("masks"):
        n, W = case["masks"], (V + 31) // 32
        share = torch.rand(n, 1, generator=gen, device="cuda") * 0.4 + case["occupied"] - 0.2
        share[torch.rand(n, 1, generator=gen, device="cuda") < 0.01] = 1.5       # definitions that no register is left for
        # occupied registers come in runs: tuples of live values
        runs = torch.rand(n, (V + 3) // 4, generator=gen, device="cuda").repeat_interleave(4, dim=1)[:, :V]
        bits = torch.zeros((n, W * 32), dtype=torch.int64, device="cuda")
        bits[:, :V] = (runs < share).to(torch.int64)
        words = (bits.view(n, W, 32) << torch.arange(32, device="cuda")).sum(dim=2)
        st["occupied"] = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
        st["mask_rows"] = (row % n).to(torch.int32)
        if case["widths"]:
            kinds = torch.tensor([1, 1, 1, 1, 1, 1, 1, 2, 2, 4], dtype=torch.uint8, device="cuda")
            st["widths"] = kinds[torch.randint(0, 10, (n,), generator=gen, device="cuda")][row % n].contiguous()
    if case["op"] == "grad":
        by = (4096.0 if case["dtype"] == "f16" else 1.0) / R        # 16-bit halves train under a scaled loss
        st["g"] = torch.randn(R, generator=gen, device="cuda") * by
        st["h"] = torch.randn(R, generator=gen, device="cuda") * (0.01 * by) if case["entropy"] else None
        st["stats"], st["entropy"] = _row_statistics(st)
    return st


def _policy_inputs(case, seed):
    rng = np.random.default_rng(1_000_003 * seed + 29)
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * seed + 31)
    G, K = case["programs"], case["samples"]
    shape = np.random.default_rng(G + 1000 * K + 7 * case["tokens"])     # the sizes belong to the case, the values to the seed
    sizes = [K] * G if G == 1 else [int(k) for k in shape.integers(max(1, K // 2), K + K // 2 + 1, G)]
    N = sum(sizes)
    lens = np.maximum(0, np.rint(case["tokens"] * np.exp(case["spread"] * shape.standard_normal(N) - 0.5 * case["spread"] ** 2)))
    lens = np.minimum(lens, 60000).astype(np.int64)
    off = np.concatenate([[0], np.cumsum(lens)])
    T = int(off[-1])
    v = np.zeros((N, 4), dtype=np.int32)
    bad = rng.random(N) < case["fails"]
    v[:, 0] = np.where(bad, rng.choice([2, 4, 8, 10], N), 1)
    v[:, 1] = np.where(bad, rng.integers(0, 2000, N), -1)
    v[:, 2] = np.where(v[:, 0] & 8, rng.integers(1, 200, N), 0)
    v[:, 3] = rng.integers(0, 400, N)
    verdicts = torch.from_numpy(v).cuda()
    lp = -torch.empty(T, device="cuda").exponential_(1.5, generator=gen)
    old = lp + 0.12 * torch.randn(T, generator=gen, device="cuda")
    ref = lp + 0.2 * torch.randn(T, generator=gen, device="cuda") if case["ref"] else None
    return dict(case=case, outs=list(verdicts.split(sizes)), sizes=sizes, token_off=torch.from_numpy(off).cuda(), lp=lp, old=old, ref=ref)


_COSTS = dict(pair_cost=0.001, bank_cost=0.0005)
_CLIP = dict(clip_lo=0.2, clip_hi=0.28)
_EPS, _KL = 1e-6, 0.04


# ---------------------------------------------------------------- the plain forms

def _closed(occupied, mask_rows, widths, R, V, a, b):
    """Truth values [b - a, V]: entries of the rows a..b that are masked out; None where none is."""
    if occupied is None and widths is None:
        return None
    dev = (occupied if occupied is not None else widths).device
    at = torch.arange(V, device=dev, dtype=torch.int32)
    if occupied is not None:
        taken = ((occupied[:, (at >> 5).long()] >> (at & 31)) & 1).bool()
    else:
        taken = torch.zeros((1, V), dtype=torch.bool, device=dev)
    # a tuple of width w at i needs the next taken entry, or the end, to be w away
    nxt = torch.where(taken, at, torch.full_like(at, V)).flip(1).cummin(1).values.flip(1)
    room = nxt - at
    rows = mask_rows[a:b].long() if mask_rows is not None else (torch.arange(a, b, device=dev) if occupied is not None
                                                              else torch.zeros(b - a, dtype=torch.long, device=dev))
    w = widths[a:b].to(torch.int32)[:, None] if widths is not None else 1
    return room[rows] < w


def _token_of(tokens, V):
    t = tokens.to(torch.int32 if tokens.dtype == torch.uint16 else tokens.dtype).long()
    return t, (t >= 0) & (t < V)


def _slabs(R, V):
    step = max(1, _SLAB // V)
    return [(a, min(R, a + step)) for a in range(0, R, step)]


def _row_terms(st, a, b):
    case, V = st["case"], st["case"]["vocab"]
    x = st["x"][a:b].float()
    closed = _closed(st["occupied"], st["mask_rows"], st["widths"], case["rows"], V, a, b)
    if closed is not None:
        x = x.masked_fill(closed, -math.inf)
    top = x.amax(dim=1)
    base = torch.where(top == -math.inf, torch.zeros_like(top), top)
    d = (x - base[:, None]) * case["scale"]
    e = torch.exp(d)
    s = e.sum(dim=1)
    return x, top, d, e, s


def _row_statistics(st):
    """What a user has from the forward call: ([rows, 2] largest logit and log of the sum, entropy)."""
    R, V = st["case"]["rows"], st["case"]["vocab"]
    stats, ent = [], []
    for a, b in _slabs(R, V):
        _, top, d, e, s = _row_terms(st, a, b)
        _, counts = _token_of(st["tokens"][a:b], V)
        h = torch.log(s) - (e * torch.where(e > 0, d, torch.zeros_like(d))).sum(dim=1) / s
        zero = torch.zeros_like(h)
        h = torch.where((s > 0) & counts, h, zero)
        stats.append(torch.where(counts[:, None], torch.stack([top, torch.log(s)], dim=1), zero[:, None]))
        ent.append(h)
    return torch.cat(stats), torch.cat(ent)


def _plain_score(st):
    case = st["case"]
    R, V, k = case["rows"], case["vocab"], case["top"]
    parts = []
    for a, b in _slabs(R, V):
        x, top, d, e, s = _row_terms(st, a, b)
        t, counts = _token_of(st["tokens"][a:b], V)
        zero = torch.zeros_like(s)
        log_sum = torch.log(s)
        lt = d.gather(1, torch.where(counts, t, torch.zeros_like(t))[:, None])[:, 0] - log_sum
        lt = torch.where(s > 0, lt, torch.full_like(lt, -math.inf))
        h = log_sum - (e * torch.where(e > 0, d, torch.zeros_like(d))).sum(dim=1) / s
        h = torch.where(s > 0, h, zero)
        out = [torch.where(counts, lt, zero), torch.where(counts, h, zero),
               torch.where(counts[:, None], torch.stack([top, log_sum], dim=1), zero[:, None])]
        if k:
            # largest first, the lowest index first among equals: both in one 64-bit key
            bits = (x + 0.0).view(torch.int32).long()
            order = torch.where(bits < 0, -(bits & 0x7FFFFFFF) - 1, bits)
            key = (order << 32) | (0xFFFFFFFF - torch.arange(V, device=x.device))
            best = torch.topk(key, min(k, V), dim=1).values
            at = 0xFFFFFFFF - (best & 0xFFFFFFFF)
            there = (x.gather(1, at) > -math.inf) & counts[:, None]
            lp = torch.where(there, d.gather(1, at) - log_sum[:, None], torch.full_like(at, -1).float() * math.inf)
            at = torch.where(there, at, torch.full_like(at, -1)).to(torch.int32)
            if k > V:
                lp = torch.nn.functional.pad(lp, (0, k - V), value=-math.inf)
                at = torch.nn.functional.pad(at, (0, k - V), value=-1)
            out += [at, lp]
        parts.append(out)
    return tuple(torch.cat(c) for c in zip(*parts))


def _plain_grad(st):
    case = st["case"]
    R, V, scale = case["rows"], case["vocab"], case["scale"]
    dx = torch.empty((R, V), dtype=st["x"].dtype, device="cuda")
    for a, b in _slabs(R, V):
        x = st["x"][a:b].float()
        closed = _closed(st["occupied"], st["mask_rows"], st["widths"], R, V, a, b)
        if closed is not None:
            x = x.masked_fill(closed, -math.inf)
        t, counts = _token_of(st["tokens"][a:b], V)
        t = torch.where(counts, t, torch.zeros_like(t))
        top, log_sum = st["stats"][a:b, 0], st["stats"][a:b, 1]
        alive = counts & (log_sum > -math.inf)
        g = st["g"][a:b]
        if closed is not None:
            g = torch.where(closed.gather(1, t[:, None])[:, 0], torch.zeros_like(g), g)
        g = torch.where(alive, g, torch.zeros_like(g))
        l = (x - torch.where(alive, top, torch.zeros_like(top))[:, None]) * scale - torch.where(alive, log_sum, torch.zeros_like(top))[:, None]
        p = torch.exp(l)
        f = g[:, None]
        if st["h"] is not None:
            h = torch.where(alive, st["h"][a:b], torch.zeros_like(g))
            f = f + h[:, None] * torch.where(p > 0, l + st["entropy"][a:b, None], torch.zeros_like(l))
        out = -p * f
        out.scatter_add_(1, t[:, None], g[:, None])
        out = torch.where(alive[:, None], out * scale, torch.zeros_like(out))
        dx[a:b] = out.to(dx.dtype)
    return dx


def _plain_policy(st):
    case, N, T = st["case"], sum(st["sizes"]), st["lp"].numel()
    v = torch.cat(st["outs"])
    reward = (v[:, 0] & 1).double() - _COSTS["pair_cost"] * v[:, 2].double() - _COSTS["bank_cost"] * v[:, 3].double()
    G = len(st["sizes"])
    size = torch.tensor(st["sizes"], dtype=torch.float64, device="cuda")
    group = torch.repeat_interleave(torch.arange(G, device="cuda"), size.long(), output_size=N)
    first = torch.cumsum(size.long(), 0) - size.long()
    place = group * max(st["sizes"]) + torch.arange(N, device="cuda") - first[group]

    def mean_of(x):
        table = torch.zeros((G, max(st["sizes"])), dtype=torch.float64, device="cuda")
        table.view(-1)[place] = x
        return table.sum(dim=1) / size

    adv = reward - mean_of(reward)[group]
    if case["normalise"]:
        var = mean_of(adv * adv)
        adv = adv / (torch.sqrt(var)[group] + _EPS)
    off = st["token_off"]
    lens = off[1:] - off[:-1]
    owner = torch.repeat_interleave(torch.arange(N, device="cuda"), lens, output_size=T)
    A = adv[owner]
    w = torch.full_like(A, 1.0 / max(T, 1)) if case["per_token"] else (1.0 / (N * lens.double()))[owner]
    rho = torch.exp(st["lp"].double() - st["old"].double())     # in 64 bits: next to the clip's borders a step decides
    lo, hi = 1.0 - _CLIP["clip_lo"], 1.0 + _CLIP["clip_hi"]
    surr = torch.minimum(rho * A, rho.clamp(lo, hi) * A)
    inside = torch.where(A > 0, rho <= hi, rho >= lo)
    dlp = -torch.where(inside, rho * A, torch.zeros_like(A))
    loss = -surr
    if case["ref"]:
        q = st["ref"].double() - st["lp"].double()
        loss = loss + _KL * (torch.expm1(q) - q)
        dlp = dlp - _KL * torch.expm1(q)
    return (w * loss).sum().float(), adv.float(), (w * dlp).float()


# ---------------------------------------------------------------- one pass

def run(st):
    op = st["case"]["op"]
    if not own:
        return {"score": _plain_score, "grad": _plain_grad, "policy": _plain_policy}[op](st)
    from paper_2506_17506_b200 import binding as vl
    case = st["case"]
    if op == "score":
        out = vl.vl_token_logprobs(st["x"], st["tokens"], occupied=st["occupied"], mask_rows=st["mask_rows"], widths=st["widths"],
                                   scale=case["scale"], top=case["top"])
        return (out.logprob, out.entropy, out.row_stats) + ((out.top_ids, out.top_logprobs) if case["top"] else ())
    if op == "grad":
        return vl.vl_token_logprobs_backward(st["x"], st["tokens"], st["stats"], st["g"], entropy=st["entropy"], g_entropy=st["h"],
                                             occupied=st["occupied"], mask_rows=st["mask_rows"], widths=st["widths"],
                                             scale=case["scale"])
    return tuple(vl.vl_policy_loss(st["outs"], st["token_off"], st["lp"], st["old"], ref_logprob=st["ref"],
                                   normalise=case["normalise"], eps=_EPS, kl=_KL if case["ref"] else 0.0,
                                   per_token=case["per_token"], **_COSTS, **_CLIP))


def work(case):
    if case["op"] == "policy":
        n = case["programs"] * case["samples"]
        T = n * case["tokens"]
        return {"bytes": n * (16 + 8 + 4) + T * (12 + (4 if case["ref"] else 0)), "flops": T * 12}
    R, V = case["rows"], case["vocab"]
    words = case.get("masks", 0) * ((V + 31) // 32) * 4
    row = {"u16": 2, "i32": 4, "i64": 8}[case["tokens"]] + (4 if case.get("masks") else 0) + (1 if case.get("widths") else 0)
    elements = R * V * _BYTES[case["dtype"]]
    if case["op"] == "score":
        return {"bytes": elements + words + R * (row + 16 + 8 * case["top"]), "flops": R * V * 7}
    return {"bytes": 2 * elements + words + R * (row + 12 + (8 if case["entropy"] else 0)), "flops": R * V * 8}


# ---------------------------------------------------------------- the definitions in 64 bits

def _open_64(st, a, b):
    """Open entries of the rows a..b, tuple by tuple from the definition: register i + s is free for every s below the width."""
    case, V = st["case"], st["case"]["vocab"]
    n = b - a
    free = torch.ones((n, V), dtype=torch.bool, device="cuda")
    if st["occupied"] is not None:
        words = st["occupied"][st["mask_rows"][a:b].long()].long() & 0xFFFFFFFF
        shift = torch.arange(32, device="cuda")
        free = (((words[:, :, None] >> shift) & 1) == 0).reshape(n, -1)[:, :V]
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


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "policy":
        return _exact_policy(st)
    R, V, scale = case["rows"], case["vocab"], float(case["scale"])
    parts = []
    for a in range(0, R, max(1, (1 << 26) // V)):
        b = min(R, a + max(1, (1 << 26) // V))
        z = st["x"][a:b].double() * scale
        shut = ~_open_64(st, a, b)
        z[shut] = -math.inf
        tok = st["tokens"][a:b].to(torch.int32 if case["tokens"] == "u16" else torch.int64).long()
        kept = (tok >= 0) & (tok < V)
        tok = tok.clamp(0, V - 1)
        lse = torch.logsumexp(z, dim=1)
        dead = lse == -math.inf
        logp = z - torch.where(dead, torch.zeros_like(lse), lse)[:, None]
        prob = logp.exp()
        ent = torch.special.entr(prob).sum(dim=1)
        if case["op"] == "score":
            biggest = z.amax(dim=1)
            rest = torch.where(dead, lse, lse - torch.where(dead, torch.zeros_like(lse), biggest))
            vals = [logp.gather(1, tok[:, None])[:, 0], ent, torch.stack([biggest / scale, rest], dim=1)]
            for v in vals:
                v[~kept] = 0.0
            if case["top"]:
                k = case["top"]
                ids = torch.full((b - a, k), -1, dtype=torch.int64, device="cuda")
                lps = torch.full((b - a, k), -math.inf, dtype=torch.float64, device="cuda")
                left = torch.where(shut, torch.full_like(z, -math.inf), st["x"][a:b].double())
                rows = torch.arange(b - a, device="cuda")
                for j in range(min(k, V)):
                    best = left.amax(dim=1)
                    first = (left == best[:, None]).to(torch.uint8).argmax(dim=1)      # the lowest index among equals
                    ok = (best > -math.inf) & kept
                    ids[ok, j] = first[ok]
                    lps[ok, j] = logp[rows, first][ok]
                    left[rows, first] = -math.inf
                vals += [ids.to(torch.int32), lps]
            parts.append(vals)
        else:
            # d logp[t] = [i = t] - p;  d entropy = -p (ln p + entropy)
            g = st["g"][a:b].double()
            g = torch.where(shut.gather(1, tok[:, None])[:, 0], torch.zeros_like(g), g)
            dx = -prob * g[:, None]
            dx[torch.arange(b - a, device="cuda"), tok] += g
            if st["h"] is not None:
                dx += st["h"][a:b].double()[:, None] * (torch.special.entr(prob) - prob * ent[:, None])
            dx *= scale
            dx[~kept | dead] = 0.0
            parts.append([dx])
    done = tuple(torch.cat(c) for c in zip(*parts))
    return done if case["op"] == "score" else done[0]


def _exact_policy(st):
    """Program by program and sample by sample on the host, in 64 bits."""
    case = st["case"]
    lp, old = st["lp"].double().cpu().numpy(), st["old"].double().cpu().numpy()
    ref = st["ref"].double().cpu().numpy() if case["ref"] else None
    off = st["token_off"].cpu().numpy()
    N, T = sum(st["sizes"]), len(lp)
    adv = []
    for out in st["outs"]:
        v = out.cpu().numpy().astype(np.float64)
        r = (v[:, 0] == 1) * 1.0 - _COSTS["pair_cost"] * v[:, 2] - _COSTS["bank_cost"] * v[:, 3]
        c = r - math.fsum(r) / len(r)
        adv.append(c / (math.sqrt(math.fsum(c * c) / len(r)) + _EPS) if case["normalise"] else c)
    adv = np.concatenate(adv)
    dlp, terms = np.zeros(T), np.zeros(N)
    lo, hi = math.log1p(-_CLIP["clip_lo"]), math.log1p(_CLIP["clip_hi"])
    for k in range(N):
        s = slice(off[k], off[k + 1])
        n = off[k + 1] - off[k]
        if n == 0:
            continue
        w = 1.0 / T if case["per_token"] else 1.0 / (N * n)
        d, A = lp[s] - old[s], adv[k]
        if A > 0:
            loss, grad = -np.exp(np.minimum(d, hi)) * A, np.where(d <= hi, -np.exp(d) * A, 0.0)
        else:
            loss, grad = -np.exp(np.maximum(d, lo)) * A, np.where(d >= lo, -np.exp(d) * A, 0.0)
        if ref is not None:
            q = ref[s] - lp[s]
            loss, grad = loss + _KL * (np.expm1(q) - q), grad - _KL * np.expm1(q)
        dlp[s] = w * grad
        terms[k] = w * loss.sum()
    gpu = dict(dtype=torch.float64, device="cuda")
    return torch.tensor(math.fsum(terms), **gpu), torch.tensor(adv, **gpu), torch.tensor(dlp, **gpu)
