"""What a program that answers with an evicted cache asks of this library around the attention, as measurable cases.

Such a program rotates the queries and keys of its tokens by their positions (``rotate``) before they are scored, cached or attended
to.  Where it drafts several continuations at once, or decodes blocks in order, its response rows do not all see each other: the
drafted tree becomes a mask (``mask``), once a step, and every layer attends with it over the evicted cache and the response's own
rows (``attend``).  At the end of the step every row's logits become a token and the confidence in it (``sample``).

Cases of ``attend``: ``dtype``, ``B`` sequences of ``H`` key/value heads with ``g`` query heads each, head_dim ``d``, ``n`` response
rows, per-head caches of ``keep_lo`` .. ``keep_hi`` rows, spread evenly over the logarithm, and ``shape``, who sees whom among the
response rows: "tree" (a node sees itself and its ancestors), "blocks" (a row sees its block of eight and the blocks before it).
``mask``: ``B`` trees of ``n`` nodes.  ``rotate``: ``T`` tokens from position ``far`` on, of which the first ``width`` elements of a
head are rotated, as ``layout`` "halves" or "pairs", with frequencies scaled by ``scaling``.  ``sample``: ``rows`` rows of ``V``
logits; ``filters`` says which of the limits are set, ``sharp`` whether a few tokens stand out, as they mostly do.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

_BASE, _TRAINED, _SLOW, _FAST = 500000.0, 8192.0, 1.0, 32.0
_BLOCK = 8


def _attend(name, B, H, d, n, keep_lo, keep_hi, g=1, dtype="bf16", shape="tree"):
    return {"name": name, "op": "attend", "dtype": dtype, "B": B, "H": H, "g": g, "d": d, "n": n, "keep_lo": keep_lo,
            "keep_hi": keep_hi, "shape": shape}


def _mask(name, B, n):
    return {"name": name, "op": "mask", "B": B, "n": n}


def _rotate(name, B, H, d, T, width, layout="halves", scaling="plain", factor=1.0, far=0, g=1, dtype="bf16", order="bhtd"):
    return {"name": name, "op": "rotate", "dtype": dtype, "B": B, "H": H, "g": g, "d": d, "T": T, "width": width, "layout": layout,
            "scaling": scaling, "factor": factor, "far": far, "order": order}


def _sample(name, rows, V, filters, temperature=1.0, dtype="bf16", sharp=True):
    return {"name": name, "op": "sample", "dtype": dtype, "rows": rows, "V": V, "filters": filters, "temperature": temperature,
            "sharp": sharp}


def listed():
    return [
        # the smallest attention: a draft of 8 fp32 tokens over 32 rows of each of four heads; nothing but latency
        _attend("attend, 8 tokens, fp32", 1, 4, 64, 8, 32, 32, dtype="f32"),
        # a tree of 64 nodes, 32 heads with 4k rows each: the reading of the cache
        _attend("attend, 64 nodes, 4k rows", 1, 32, 128, 64, 4096, 4096),
        # a grouped-query model over a long odd prompt that is kept whole: 336 query rows a head, matrix work
        _attend("attend, 48 nodes, 30k rows", 1, 4, 128, 48, 30011, 30011, g=7),
        # blocks of eight in order, in the ragged batch: many short heads
        _attend("attend, ragged batch", 8, 32, 128, 32, 64, 1024, shape="blocks"),
        # the mask of one drafted tree, and of a large batch of large ones
        _mask("mask, 64 nodes", 1, 64),
        _mask("mask, 64 trees of 512", 64, 512),
        # the next token of a grouped-query model: latency
        _rotate("rotate, one token", 1, 4, 128, 1, 128, far=30011, g=7),
        # a partly rotated fp32 batch with pairs side by side, a token's heads together
        _rotate("rotate, part, fp32", 8, 12, 64, 500, 32, layout="pairs", scaling="linear", factor=4.0, g=1, dtype="f32", order="bthd"),
        # all of a 32k prompt's rows, four times the length that the frequencies were trained for
        _rotate("rotate, 32k prompt", 1, 32, 128, 32768, 128, scaling="bands", factor=4.0),
        # the next token, from an odd number of fp32 logits, 50 best ones, of these 0.9 of the mass
        _sample("sample, one row, fp32", 1, 32001, "kp", 0.8, dtype="f32"),
        # a denoising step: every masked position of a response of 256, with a temperature and nothing else
        _sample("sample, 256 rows", 256, 126464, "", 0.7),
        # requests of many users in a batch: every row has its own temperature and limits, some have none
        _sample("sample, mixed batch", 64, 152064, "mixed", 1.0),
    ]


# The most that a drawn case may ask for: logits of the attention, elements of a cache padded to its longest head, rotated elements,
# logits that are sampled from.
_MOST_LOGITS = 45 << 20
_MOST_CACHED = 256 * 1024 * 128
_MOST_ROTATED = 64 * 32768 * 128
_MOST_SAMPLED = 256 * 126464


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend"] * 4 + ["rotate"] * 3 + ["sample"] * 3 + ["mask"])
    while True:
        dtype = rng.choice(["f32", "bf16", "bf16"])
        if op == "mask":
            c = _mask("", _spread(rng, 1, 64), _spread(rng, 1, 512))
            break
        if op == "sample":
            c = _sample("", _spread(rng, 1, 512), _spread(rng, 1000, 160000), rng.choice(["", "k", "p", "m", "kp", "kpm", "mixed", "mixed"]),
                        round(rng.uniform(0.3, 1.5), 3), dtype, rng.random() < 0.8)
            if c["rows"] * c["V"] * (2 if dtype == "f32" else 1) <= _MOST_SAMPLED:
                break
            continue
        B = 1 if rng.random() < 0.5 else rng.randint(2, 8)
        H = rng.choice([2, 4, 8, 12, 28, 32])
        g = 1 if H > 8 else rng.choice([1, 4, 7])
        d = rng.choice([64, 128, 128])
        if op == "rotate":
            scaling = rng.choice(["plain", "linear", "base", "bands"])
            width = d if rng.random() < 0.6 else 16 * rng.randint(1, d // 16)
            c = _rotate("", B, H, d, _spread(rng, 1, 32768), width, rng.choice(["halves", "halves", "pairs"]), scaling,
                        1.0 if scaling == "plain" else round(rng.uniform(1.5, 16.0), 2), _spread(rng, 1, 1000000), g, dtype,
                        rng.choice(["bhtd", "bthd"]))
            if B * H * (g + 1) * c["T"] * d * (2 if dtype == "f32" else 1) <= _MOST_ROTATED:
                break
            continue
        small = dtype == "f32"           # fp32 is for short caches
        keep_hi = _spread(rng, 8, 1024) if small else _spread(rng, 32, 32768)
        keep_lo = max(1, int(keep_hi * rng.uniform(0.05, 1.0)))
        c = _attend("", B, H, d, _spread(rng, 1, 64 if small else 256), keep_lo, keep_hi, g, dtype, rng.choice(["tree", "tree", "blocks"]))
        logits = B * H * g * c["n"] * (keep_hi + c["n"]) * (16 if small else 1)
        if logits <= _MOST_LOGITS and B * H * (keep_hi + c["n"]) * d <= _MOST_CACHED:
            break
    return {k: v for k, v in c.items() if k != "name"}


def _kept(c):
    """Rows of each head, in an order without a trend."""
    lo, hi, count, stride = c["keep_lo"], c["keep_hi"], c["B"] * c["H"], 37
    v = [int(round(math.exp(math.log(lo) + math.log(hi / lo) * (i / (count - 1) if count > 1 else 1.0)))) for i in range(count)]
    while math.gcd(stride, count) != 1:
        stride += 1
    return [v[i * stride % count] for i in range(count)]


# ---- inputs
def _parents(B, n, seed):
    """Drafted trees, a level after the other: a node hangs from one of the last few nodes before it, the first one from nothing."""
    rng = random.Random(seed)
    return [[-1] + [rng.randrange(max(0, i - 1 - n // 8), i) for i in range(1, n)] for _ in range(B)]


def _words(seen):
    """[..., n, n] truth values -> the words of a mask, [..., n, (n + 31) // 32] int32: bit j % 32 of word j // 32 for column j."""
    n = seen.shape[-1]
    bits = torch.zeros(seen.shape[:-1] + ((n + 31) // 32 * 32,), dtype=torch.int64, device=seen.device)
    bits[..., :n] = seen
    weight = torch.ones(32, dtype=torch.int64, device=seen.device) << torch.arange(32, device=seen.device)
    words = (bits.unflatten(-1, (-1, 32)) * weight).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def _ancestors(parents):
    """[B, n] -> [B, n, n]: whether node j is node i or above it."""
    n = parents.shape[1]
    node = torch.arange(n, device=parents.device)
    reach = ((parents.unsqueeze(2) == node) | (node[:, None] == node)).float()      # one step up, or none
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (torch.matmul(reach, reach) > 0).float()                            # twice as many
    return reach > 0


def _frequencies(c):
    """Radians a position of each rotated pair, float64, and what the rotated elements are multiplied by."""
    width, factor = c["width"], c["factor"]
    base = _BASE * factor ** (width / (width - 2.0)) if c["scaling"] == "base" and width > 2 else _BASE
    freq = base ** (-2.0 * torch.arange(width // 2, dtype=torch.float64, device="cuda") / width)
    if c["scaling"] == "linear":
        return freq / factor, 1.0
    if c["scaling"] == "bands":
        keep = ((_TRAINED * freq / (2.0 * math.pi) - _SLOW) / (_FAST - _SLOW)).clamp(0.0, 1.0)
        return freq * (keep + (1.0 - keep) / factor), 1.0 + 0.1 * math.log(factor)
    return freq, 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    s = SimpleNamespace(op=op, case=case, call=None)
    if op == "mask":
        s.parents = torch.tensor(_parents(case["B"], case["n"], seed), dtype=torch.int32, device="cuda")
        s.mask = torch.zeros((case["B"], case["n"], (case["n"] + 31) // 32), dtype=torch.int32, device="cuda")
        return s
    s.dt = dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32

    def gauss(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def even(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    if op == "sample":
        rows, V, filters = case["rows"], case["V"], case["filters"]
        logits = gauss(rows, V).mul_(2.0)
        if case["sharp"]:                  # a few dozen tokens that the context makes likely, their logits spread widely
            logits.scatter_add_(1, (even(rows, 32) * V).long().clamp_(max=V - 1), 10.0 + 3.0 * gauss(rows, 32))
        s.logits = logits.to(dt)
        s.u = even(rows)
        s.temperature = torch.full((rows,), case["temperature"], device="cuda")
        s.k = s.p = s.m = None
        if "k" in filters:
            s.k = torch.full((rows,), 50, dtype=torch.int32, device="cuda")
        if "p" in filters:
            s.p = torch.full((rows,), 0.9, device="cuda")
        if filters == "m" or "pm" in filters:
            s.m = torch.full((rows,), 0.05, device="cuda")
        if filters == "mixed":
            s.temperature = 0.3 + 1.2 * even(rows)
            s.temperature = torch.where(even(rows) < 0.125, torch.zeros_like(s.temperature), s.temperature)   # (greedy)
            s.k = torch.where(even(rows) < 0.5, torch.exp(1.0 + 5.0 * even(rows)).int(), torch.zeros(rows, dtype=torch.int32, device="cuda"))
            s.p = torch.where(even(rows) < 0.5, 0.5 + 0.49 * even(rows), torch.ones(rows, device="cuda"))
            s.m = torch.where(even(rows) < 0.25, 0.2 * even(rows), torch.zeros(rows, device="cuda"))
        s.token = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s.prob, s.logprob = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        return s

    B, H, g, d = (case[k] for k in ("B", "H", "g", "d"))
    if op == "rotate":
        T = case["T"]

        def room(heads):
            if case["order"] == "bhtd":
                return torch.empty((B, heads, T, d), dtype=dt, device="cuda")
            return torch.empty((B, T, heads, d), dtype=dt, device="cuda").transpose(1, 2)

        s.Q, s.K = room(H * g).normal_(generator=gen), room(H).normal_(generator=gen)
        s.Qr, s.Kr = room(H * g).zero_(), room(H).zero_()
        first = case["far"] + (even(B, 1) * 64).long()                  # each sequence goes on from where it is
        s.positions = (first + torch.arange(T, device="cuda")).to(torch.int32)
        s.freq, s.amplitude = _frequencies(case)
        return s

    n = case["n"]
    kept = _kept(case)
    s.cap, s.most = sum(kept), max(kept)
    s.lens = torch.tensor(kept, device="cuda")
    ends = s.lens.cumsum(0)
    s.start = ends - s.lens
    s.cu = torch.cat((ends.new_zeros(1), ends)).to(torch.int32)
    # keys have channels of their own size, a few of them large, as keys behind a rotation have; logits have a spread of about one
    channel = torch.exp(0.5 * gauss(B * H, 1, d))
    channel = channel / channel.square().mean(2, keepdim=True).sqrt()
    head = torch.repeat_interleave(torch.arange(B * H, device="cuda"), s.lens, output_size=s.cap)
    s.K, s.V = (gauss(s.cap, d) * channel[head, 0]).to(dt), gauss(s.cap, d).to(dt)
    s.Q = gauss(B, H * g, n, d).to(dt)
    s.Kr = (gauss(B, H, n, d) * channel.view(B, H, 1, d)).to(dt)
    s.Vr = gauss(B, H, n, d).to(dt)
    if case["shape"] == "tree":
        s.seen = _ancestors(torch.tensor(_parents(B, n, seed), dtype=torch.int32, device="cuda"))
    else:
        block = torch.arange(n, device="cuda") // _BLOCK
        s.seen = (block[:, None] >= block[None, :]).expand(B, n, n).contiguous()
    s.mask = _words(s.seen)
    s.O, s.lse = torch.zeros_like(s.Q), torch.zeros(B * H * g * n, device="cuda")
    return s


# ---- the operators, plainly
def _plain_attend(s):
    B, H, g, d, n = (s.case[k] for k in ("B", "H", "g", "d", "n"))
    place = torch.arange(s.most, device="cuda")
    live = place < s.lens[:, None]
    at = torch.where(live, s.start[:, None] + place, 0)                 # where each head's rows lie
    bits = (s.mask.unsqueeze(-1) >> torch.arange(32, dtype=torch.int32, device="cuda")).bitwise_and(1).flatten(-2)[..., :n]
    Q = s.Q.float().view(B * H, g * n, d)
    K = torch.cat((s.K.float()[at], s.Kr.float().flatten(0, 1)), 1)
    V = torch.cat((s.V.float()[at], s.Vr.float().flatten(0, 1)), 1)
    logits = torch.matmul(Q, K.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
    logits[:, :, :s.most].masked_fill_(~live[:, None], -math.inf)
    logits.view(B, H, g, n, -1)[..., s.most:].masked_fill_(bits.view(B, 1, 1, n, n) == 0, -math.inf)
    top = logits.amax(2, keepdim=True)
    p = torch.exp(logits.sub_(top))
    total = p.sum(2, keepdim=True)
    O = (torch.matmul(p, V) / total).view(B, H * g, n, d)
    return {"O": O.to(s.dt), "lse": (top + torch.log(total)).flatten()}


def _plain_rotate(s):
    half = s.case["width"] // 2
    angle = s.positions.double().unsqueeze(-1) * s.freq                 # [B, T, half]
    cos, sin = ((f(angle) * s.amplitude).float().unsqueeze(1) for f in (torch.cos, torch.sin))
    out = {}
    for name, x in (("Q", s.Q), ("K", s.K)):
        y = x.float()
        if s.case["layout"] == "halves":
            a, b = y[..., :half], y[..., half:2 * half]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin, y[..., 2 * half:]), -1)
        else:
            a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
            turned = torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2), y[..., 2 * half:]), -1)
        out[name] = turned.to(s.dt)
    return out


def _plain_sample(s):
    V = s.case["V"]
    x = s.logits.float()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices           # ties: the lower index first
    down = x.gather(1, order).double()
    top = down[:, :1]
    T = s.temperature.double().unsqueeze(1)
    w = torch.exp((down - top) / torch.where(T > 0, T, 1.0))
    rank = torch.arange(V, device="cuda")
    keep = torch.ones_like(w, dtype=torch.bool)
    if s.k is not None:
        keep &= (rank < s.k.unsqueeze(1)) | (s.k.unsqueeze(1) <= 0)
    if s.p is not None:
        mass = torch.where(keep, w, 0.0)
        upto = mass.cumsum(1)
        before = torch.cat((torch.zeros_like(upto[:, :1]), upto[:, :-1]), 1)
        p = s.p.double().unsqueeze(1)
        keep &= (rank == 0) | (p >= 1) | (before < p * upto[:, -1:])
    if s.m is not None:
        keep &= w >= s.m.double().unsqueeze(1)
    keep &= (T > 0) | (rank == 0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, w, 0.0))     # in the order of the tokens
    upto = kept.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= s.u.double().unsqueeze(1) * total).sum(1, keepdim=True)
    last = torch.where(kept > 0, rank, 0).amax(1, keepdim=True)
    token = torch.minimum(token, last)
    prob = kept.gather(1, token) / total
    logprob = x.gather(1, token).double() - top - torch.log(torch.exp(x.double() - top).sum(1, keepdim=True))
    return {"token": token.squeeze(1).to(torch.int32), "prob": prob.squeeze(1).float(), "logprob": logprob.squeeze(1).float()}


# ---- the operators, as a program calls them
def _handle(s):
    """What such a program keeps from call to call: the description, the frequencies and the workspace."""
    from paper_2510_09309_amd import binding as mk
    c, h = s.case, SimpleNamespace(mk=mk)
    if s.op == "mask":
        return h
    dtype = mk.MASKKV_BF16 if s.dt == torch.bfloat16 else mk.MASKKV_F32
    if s.op == "sample":
        size = mk.maskkv_sample_workspace_bytes(c["rows"], c["V"], dtype)
    else:
        n = c["n"] if s.op == "attend" else 1
        h.desc = mk.Desc(B=c["B"], H=c["H"], d=c["d"], dtype=dtype, n_resp=n, P_max=c.get("keep_hi", 0), q_per_kv=0 if c["g"] == 1 else c["g"])
        size = mk.maskkv_attend_tree_workspace_bytes(h.desc, s.cap) if s.op == "attend" else 0
    if s.op == "rotate":
        layout = mk.ROTARY_HALVES if c["layout"] == "halves" else mk.ROTARY_PAIRS
        scaling = {"plain": mk.ROTARY_PLAIN, "linear": mk.ROTARY_LINEAR, "base": mk.ROTARY_BASE, "bands": mk.ROTARY_BANDS}[c["scaling"]]
        h.rotary = mk.maskkv_rotary_frequencies(c["width"], layout, _BASE, scaling, c["factor"], _TRAINED, _SLOW, _FAST)
    h.ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    return h


def _call(s):
    if s.call is None:
        s.call = _handle(s)
    h = s.call
    mk = h.mk
    if s.op == "mask":
        mk.maskkv_tree_mask(s.parents, s.mask)
        return {"mask": s.mask}
    if s.op == "attend":
        mk.maskkv_attend_tree(h.desc, s.Q, s.K, s.V, s.cu, s.cap, s.Kr, s.Vr, s.mask, 0.0, s.O, s.lse, h.ws)
        return {"O": s.O, "lse": s.lse}
    if s.op == "rotate":
        mk.maskkv_rotate(h.desc, h.rotary, s.positions, s.case["T"], s.Q, s.Qr, s.K, s.Kr)
        return {"Q": s.Qr, "K": s.Kr}
    mk.maskkv_sample(s.logits, s.temperature, s.k, s.p, s.m, s.u, s.token, s.prob, s.logprob, h.ws)
    return {"token": s.token, "prob": s.prob, "logprob": s.logprob}


def run(s):
    if own:
        return _call(s)
    if s.op == "mask":
        return {"mask": _words(_ancestors(s.parents))}
    return {"attend": _plain_attend, "rotate": _plain_rotate, "sample": _plain_sample}[s.op](s)


def work(case):
    op = case["op"]
    if op == "mask":             # parents in, bits out
        return {"bytes": case["B"] * case["n"] * 4 * (1 + (case["n"] + 31) // 32), "flops": 0}
    eb = 2 if case["dtype"] == "bf16" else 4
    if op == "sample":           # logits, four parameters and a random number a row in, three numbers out
        return {"bytes": case["rows"] * (case["V"] * eb + 20 + 12), "flops": 0}
    B, H, g, d = (case[k] for k in ("B", "H", "g", "d"))
    if op == "rotate":           # rows in and out, positions
        elements = B * H * (g + 1) * case["T"]
        return {"bytes": elements * d * 2 * eb + B * case["T"] * 4, "flops": 3 * elements * case["width"]}
    n, rows = case["n"], sum(_kept(case))
    queries = B * H * g * n
    return {"bytes": (rows + B * H * n) * 2 * d * eb + queries * (2 * d * eb + 4) + B * n * ((n + 31) // 32) * 4,
            "flops": 4 * g * n * d * (rows + B * H * n)}


# ---- the definitions in 64 bits, a head or a row at a time
def exact(case, seed):
    if case["op"] == "mask":             # (truth values: there is nothing that could be nearer)
        return None
    s = prepare(case, seed)
    if s.op == "rotate":
        if case["B"] * case["H"] * (case["g"] + 1) * case["T"] * case["d"] > _MOST_ROTATED:
            return None
        half, out = case["width"] // 2, {}
        i = torch.arange(half, device="cuda")
        first, second = (i, i + half) if case["layout"] == "halves" else (2 * i, 2 * i + 1)
        for name, x in (("Q", s.Q), ("K", s.K)):
            y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
            for b in range(case["B"]):
                turn = s.amplitude * torch.exp(1j * torch.outer(s.positions[b].double(), s.freq))
                for h in range(x.shape[1]):
                    row = x[b, h].double()
                    z = torch.complex(row[:, first], row[:, second]) * turn
                    row[:, first], row[:, second] = z.real, z.imag
                    y[b, h] = row
            out[name] = y
        return out
    if s.op == "sample":
        probs, logprobs = [], []
        for r in range(case["rows"]):
            x, T = s.logits[r].double(), float(s.temperature[r])
            logs = x - torch.logsumexp(x, 0)
            if T <= 0:
                best = torch.nonzero(x == x.max())[0, 0]
                probs.append(torch.ones((), dtype=torch.float64, device="cuda"))
                logprobs.append(logs[best])
                continue
            share = torch.exp(x / T - torch.logsumexp(x / T, 0))
            keep = torch.ones_like(share, dtype=torch.bool)
            limit_k = int(s.k[r]) if s.k is not None else 0
            limit_p = float(s.p[r]) if s.p is not None else 1.0
            if 0 < limit_k < x.numel() or limit_p < 1.0:
                values, counts = torch.unique(x, return_counts=True)      # ascending
                values, counts = values.flip(0), counts.flip(0)
                number = counts.clone()
                if 0 < limit_k < x.numel():                               # of each value, from the largest one down, how many stay
                    number = torch.minimum(counts, (limit_k - (counts.cumsum(0) - counts)).clamp(min=0))
                if limit_p < 1.0:
                    each = torch.exp(values / T - torch.logsumexp(x / T, 0))
                    mass = (each * number).cumsum(0)
                    room = limit_p * mass[-1] - (mass - each * number)    # one stays where the mass before it leaves some of this
                    number = torch.minimum(number, torch.ceil(room / each.clamp(min=1e-300)).clamp(min=0, max=x.numel()).long())
                    number[0] = max(int(number[0]), 1)
                cut = int((number < counts).long().argmax()) if bool((number < counts).any()) else -1
                if cut >= 0:
                    keep = x > values[cut]
                    ties = torch.nonzero(x == values[cut])[:int(number[cut]), 0]
                    keep[ties] = True
            if s.m is not None:
                keep &= share >= float(s.m[r]) * share.max()
            kept = torch.nonzero(keep)[:, 0]
            upto = torch.cumsum(share[kept], 0)
            at = int(torch.searchsorted(upto, float(s.u[r]) * upto[-1], right=True).clamp(max=kept.numel() - 1))
            probs.append(share[kept[at]] / upto[-1])
            logprobs.append(logs[kept[at]])
        return {"token": None, "prob": torch.stack(probs), "logprob": torch.stack(logprobs)}
    scale = float(case["d"]) ** -0.5
    H, g, n, d = (case[k] for k in ("H", "g", "n", "d"))
    ends = s.cu.tolist()
    out, norms = [], []
    for i in range(case["B"] * H):
        b, h, a, e = i // H, i % H, ends[i], ends[i + 1]
        q = s.Q[b, h * g:(h + 1) * g].double().reshape(-1, d)
        k = torch.cat((s.K[a:e], s.Kr[b, h])).double()
        v = torch.cat((s.V[a:e], s.Vr[b, h])).double()
        logits = q @ k.T * scale
        logits[:, e - a:] += torch.where(s.seen[b], 0.0, -math.inf).double().repeat(g, 1)
        norm = torch.logsumexp(logits, 1)
        out.append(torch.exp(logits - norm[:, None]) @ v)
        norms.append(norm)
    return {"O": torch.stack(out).view(case["B"], H * g, n, d), "lse": torch.stack(norms).flatten()}
