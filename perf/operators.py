"""What a program that keeps its evicted cache in 4 bits, and goes on evicting from it, asks of this library, as measurable cases.

A program compresses a layer's prompt cache once (score, select, and then ``compact``: the kept rows of K and V go into a cache of
4-bit values with one power-of-two scale for 32 of them), reads that cache at every denoising step (``attend``: the response
span's queries over the cached rows and the response's own K and V), adds up over the steps what attention each cached row gets
(``accumulate``, from the softmax normalisers that the attention returns), and after some steps keeps only the rows that got
most (``evict``: a smaller cache, with the rows' accumulated weights and prompt positions).

A case: ``op``, ``dtype`` of Q, K and V, ``cache`` ("mx": 4 bits, "plain": rows of ``dtype``), ``B`` sequences of ``H`` key/value
heads with ``g`` query heads each, head_dim ``d``, ``n`` response tokens, prompts of ``P`` tokens, and per-head caches of
``keep_lo`` .. ``keep_hi`` rows, spread evenly over the logarithm.  ``evict`` keeps about the share ``part`` of every head's rows.

A cached row's 32 neighbours along the head dimension share the smallest power of two 2^e for which none of them is larger than
6 * 2^e (-124 <= e <= 125), and each is the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times 2^e, ties to the even one of their order.
"""
import math
from types import SimpleNamespace

import torch

own = False

_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_DECAY = 0.9


def _case(name, op, B, H, d, n, P, keep_lo, keep_hi, g=1, dtype="bf16", cache="mx", part=0.5):
    return {"name": name, "op": op, "dtype": dtype, "cache": cache, "B": B, "H": H, "g": g, "d": d, "n": n, "P": P,
            "keep_lo": keep_lo, "keep_hi": keep_hi, "part": part}


def listed():
    return [
        # the smallest eviction into 4 bits: a short fp32 prompt, four heads, 32 rows of each; nothing but latency
        _case("compact, 512 tokens, fp32", "compact", 1, 4, 64, 64, 512, 32, 32, dtype="f32"),
        # one 32-head layer of a 32k prompt, budgets two to one, 256 rows a head on average
        _case("compact, 32k prompt", "compact", 1, 32, 128, 256, 32768, 171, 341),
        # the batched ragged workload: 256 heads, 64 ... 1024 rows of each
        _case("compact, ragged batch", "compact", 8, 32, 128, 512, 16384, 64, 1024),
        # the smallest attention: 64 fp32 queries over 32 cached and 64 response rows
        _case("attend, 512 tokens, fp32", "attend", 1, 4, 64, 64, 512, 32, 32, dtype="f32"),
        # a single response token of a grouped-query model over a long odd prompt that is kept whole: the reading of the cache
        _case("attend, one token, 30k rows", "attend", 1, 4, 128, 1, 30011, 30011, 30011, g=7),
        # a block of 32 response tokens, 32 heads with 4k rows each: the cache is large and the queries are few
        _case("attend, 32 tokens, 4k rows", "attend", 1, 32, 128, 32, 8192, 4096, 4096),
        # a denoising step of the 32k-prompt configuration: as many response rows as cached ones
        _case("attend, 256 tokens", "attend", 1, 32, 128, 256, 32768, 171, 341),
        # a denoising step of the batched ragged workload: matrix work
        _case("attend, ragged batch", "attend", 8, 32, 128, 512, 16384, 64, 1024),
        # the attention that the cached rows of one layer get in such a step, from a cache in 4 bits ...
        _case("accumulate, 256 tokens", "accumulate", 1, 32, 128, 256, 32768, 171, 341),
        # ... and of the ragged batch, from a cache of bf16 rows
        _case("accumulate, ragged batch", "accumulate", 8, 32, 128, 512, 16384, 64, 1024, cache="plain"),
        # half of one layer's cached bf16 rows is given up
        _case("evict, 256 rows a head", "evict", 1, 32, 128, 256, 32768, 171, 341, cache="plain"),
        # and of the ragged batch's rows in 4 bits
        _case("evict, ragged batch", "evict", 8, 32, 128, 512, 16384, 64, 1024),
    ]


# The most that a drawn case may ask for: logits of the ragged batch, padded to its longest head; cached elements of K; prompt elements.
_MOST_LOGITS = 256 * 512 * 1536
_MOST_CACHED = 32 * 4096 * 128
_MOST_PROMPT = 8 * 32 * 16384 * 128


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["compact", "compact", "attend", "attend", "attend", "attend", "accumulate", "accumulate", "evict", "evict"])
    while True:
        small = rng.random() < 0.2           # fp32 is for short prompts and few heads
        dtype = "f32" if small and rng.random() < 0.6 else "bf16"
        B = 1 if small or rng.random() < 0.5 else rng.randint(2, 8)
        H = rng.choice([2, 4, 8, 12] if small else [4, 8, 16, 28, 32])
        g = 1 if H > 8 else rng.choice([1, 4, 7])
        d = rng.choice([64, 128, 128])
        n = _spread(rng, 1, 128) if small else _spread(rng, 1, 512)
        keep_hi = _spread(rng, 8, 1024) if small else _spread(rng, 32, 32768)
        keep_lo = max(1, int(keep_hi * rng.uniform(0.05, 1.0)))
        P = max(keep_hi, _spread(rng, 300, 32768))
        cache = "mx" if op in ("compact", "attend") else rng.choice(["mx", "mx", "plain"])
        c = _case("", op, B, H, d, n, P, keep_lo, keep_hi, g, dtype, cache, round(rng.uniform(0.2, 0.9), 3))
        logits = B * H * g * n * (keep_hi + n) * (16 if dtype == "f32" else 1)
        if logits <= _MOST_LOGITS and B * H * keep_hi * d <= _MOST_CACHED and B * H * P * d <= _MOST_PROMPT:
            return {k: v for k, v in c.items() if k != "name"}


def _kept(c):
    """Rows of each head, in an order without a trend."""
    lo, hi, count, stride = c["keep_lo"], c["keep_hi"], c["B"] * c["H"], 37
    v = [int(round(math.exp(math.log(lo) + math.log(hi / lo) * (i / (count - 1) if count > 1 else 1.0)))) for i in range(count)]
    while math.gcd(stride, count) != 1:
        stride += 1
    return [v[i * stride % count] for i in range(count)]


def _budgets(c):
    """Rows of each head after a further eviction: about ``part`` of them, every head another share."""
    return [max(0, int(k * c["part"] * (0.6 + 0.8 * ((i * 29) % 17) / 16.0))) for i, k in enumerate(_kept(c))]


# ---- the 4-bit values, plainly
def _round(x):
    """[..., d] float32 -> the exponents e [..., d/32] and the values in units of 2^e [..., d/32, 32]."""
    y = x.unflatten(-1, (-1, 32))
    most = y.abs().amax(-1)
    fraction, exponent = torch.frexp(most)                 # most = fraction * 2^exponent, 0.5 <= fraction < 1
    e = exponent - 3 + (fraction > 0.75)
    e = torch.where(most > 0, e, -124).clamp(-124, 125)
    y = torch.ldexp(y, -e.unsqueeze(-1))
    size = y.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    return e, torch.copysign((torch.round(size / step) * step).clamp(max=6.0), y)


def _pack(x):
    """[R, d] -> codes [R, d/2] (the even element in the low four bits; 8 is the sign) and scales [R, d/32] (e + 127), uint8."""
    e, v = _round(x.float())
    code = torch.searchsorted(torch.tensor(_VALUES, device=x.device), v.abs().contiguous()).to(torch.uint8)
    code = (code | (torch.signbit(v).to(torch.uint8) << 3)).flatten(-2)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), (e + 127).to(torch.uint8)


def _unpack(codes, scales):
    """The float32 values [R, d] of packed rows."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return torch.ldexp(v.unflatten(-1, (-1, 32)), scales.int().unsqueeze(-1) - 127).flatten(-2)


# ---- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    B, H, g, d, n, P = (case[k] for k in ("B", "H", "g", "d", "n", "P"))
    BH = B * H
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    s = SimpleNamespace(op=case["op"], mx=case["cache"] == "mx", B=B, H=H, g=g, d=d, n=n, P=P, dt=dt, call=None)

    def gauss(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def room(*shape, dtype=dt):
        return torch.zeros(shape, dtype=dtype, device="cuda")

    def packed(rows):
        return [room(rows, d // 2, dtype=torch.uint8), room(rows, d // 32, dtype=torch.uint8)]

    # keys have channels of their own size, a few of them large, as keys behind a rotation have; logits have a spread of about one
    channel = torch.exp(0.5 * gauss(BH, 1, d))
    channel = channel / channel.square().mean(2, keepdim=True).sqrt()
    kept = _kept(case)
    s.cap, s.most = sum(kept), max(kept)
    s.lens = torch.tensor(kept, device="cuda")
    ends = s.lens.cumsum(0)
    s.start = ends - s.lens
    s.cu = torch.cat((ends.new_zeros(1), ends)).to(torch.int32)
    s.head = torch.repeat_interleave(torch.arange(BH, device="cuda"), s.lens, output_size=s.cap)
    at = torch.arange(s.cap, device="cuda") - s.start[s.head]           # a row's place in its head
    # positions in the prompt: one of each head's equal parts of it for each row, ascending
    size, more = P // s.lens[s.head], P % s.lens[s.head]
    first = at * size + torch.minimum(at, more)
    s.idx = (first + (torch.rand(s.cap, generator=gen, device="cuda") * size).long()).clamp(max=P - 1).to(torch.int32)

    if s.op == "compact":
        s.K = torch.empty((B, H, P, d), dtype=dt, device="cuda").normal_(generator=gen).mul_(channel.view(B, H, 1, d).to(dt))
        s.V = torch.empty((B, H, P, d), dtype=dt, device="cuda").normal_(generator=gen)
        s.cache, s.Kc, s.Vc = packed(s.cap) + packed(s.cap), room(s.cap, d), room(s.cap, d)
        return s

    K, V = gauss(s.cap, d) * channel[s.head, 0], gauss(s.cap, d)
    s.K, s.V = K.to(dt), V.to(dt)
    if s.mx:
        s.cache = [*_pack(s.K), *_pack(s.V)]
    if s.op == "evict":
        # accumulated attention: heavy-tailed, and one row in eight never got any that fp32 can tell from none
        s.weights = torch.exp(1.5 * gauss(s.cap)) * (torch.rand(s.cap, generator=gen, device="cuda") > 0.125)
        after = [min(a, b) for a, b in zip(_budgets(case), kept)]
        s.budgets = torch.tensor(_budgets(case), dtype=torch.int32, device="cuda")
        s.cap_out = sum(after)
        s.Kc, s.Vc = room(s.cap_out, d), room(s.cap_out, d)
        s.cache_out = packed(s.cap_out) + packed(s.cap_out)
        s.rows, s.idx_out, s.weights_out = (room(s.cap_out, dtype=t) for t in (torch.int32, torch.int32, torch.float32))
        s.cu_out = room(BH + 1, dtype=torch.int32)
        return s
    s.Q = gauss(B, H * g, n, d).to(dt)
    s.Kr = (gauss(B, H, n, d) * channel.view(B, H, 1, d)).to(dt)
    s.Vr = gauss(B, H, n, d).to(dt)
    if s.op == "attend":
        s.O, s.lse = room(B, H * g, n, d), room(BH * g * n, dtype=torch.float32)
    else:
        s.lse = _attend(s)[1].flatten()
        s.weights = torch.exp(gauss(s.cap))
        s.weights_out = room(s.cap, dtype=torch.float32)
    return s


# ---- the operators, plainly
def _cached(s, k):
    """The cached rows of K (k = 0) or V (k = 1) as float32."""
    return _unpack(*s.cache[2 * k:2 * k + 2]) if s.mx else (s.V if k else s.K).float()


def _padded(s):
    """Where each head's rows lie, [BH, most rows], and which of those places have one."""
    place = torch.arange(s.most, device="cuda")
    live = place < s.lens[:, None]
    return torch.where(live, s.start[:, None] + place, 0), live


def _compact(s):
    K, V = (x.flatten(0, 1)[s.head, s.idx.long()].float() for x in (s.K, s.V))
    values = []
    values += [torch.ldexp(v, e.unsqueeze(-1)).flatten(-2).to(s.dt) for e, v in (_round(K), _round(V))]
    return {"K": values[0], "V": values[1]}


def _attend(s):
    at, live = _padded(s)
    Q = s.Q.float().view(s.B * s.H, s.g * s.n, s.d)
    K = torch.cat((_cached(s, 0)[at], s.Kr.float().flatten(0, 1)), 1)
    V = torch.cat((_cached(s, 1)[at], s.Vr.float().flatten(0, 1)), 1)
    logits = torch.matmul(Q, K.transpose(1, 2)) * (1.0 / math.sqrt(s.d))
    logits[:, :, :s.most].masked_fill_(~live[:, None], -math.inf)
    top = logits.amax(2, keepdim=True)
    p = torch.exp(logits.sub_(top))
    total = p.sum(2, keepdim=True)
    O = (torch.matmul(p, V) / total).view(s.B, s.H * s.g, s.n, s.d)
    return O.to(s.dt), (top + torch.log(total)).squeeze(2)


def _accumulate(s):
    at, live = _padded(s)
    Q = s.Q.float().view(s.B * s.H, s.g * s.n, s.d)
    logits = torch.matmul(Q, _cached(s, 0)[at].transpose(1, 2)) * (1.0 / math.sqrt(s.d))
    got = torch.exp(logits.sub_(s.lse.view(s.B * s.H, -1, 1))).sum(1)
    return {"weights": _DECAY * s.weights + got[live]}


def _evict(s):
    at, live = _padded(s)
    w = torch.where(live, s.weights[at], -math.inf)
    order = torch.sort(w, dim=1, descending=True, stable=True).indices           # ties: the lower row first
    rank = torch.empty_like(order).scatter_(1, order, torch.arange(s.most, device="cuda").expand_as(order))
    keep = torch.minimum(s.budgets.clamp(min=0), s.lens)
    rows = at[(rank < keep[:, None]) & live]
    cu = torch.cat((keep.new_zeros(1), keep.cumsum(0))).to(torch.int32)
    values = {"K": _cached(s, 0)[rows].to(s.dt), "V": _cached(s, 1)[rows].to(s.dt)}
    return values | {"rows": rows.to(torch.int32), "idx": s.idx[rows], "weights": s.weights[rows], "cu": cu}


# ---- the operators, as a program calls them
def _handle(s):
    """What such a program keeps from call to call: the description, the caches and the workspace."""
    from paper_2510_09309_amd import binding as mk
    dtype = mk.MASKKV_BF16 if s.dt == torch.bfloat16 else mk.MASKKV_F32
    h = SimpleNamespace(mk=mk, desc=mk.Desc(B=s.B, H=s.H, d=s.d, dtype=dtype, n_resp=s.n, P_max=s.P, q_per_kv=0 if s.g == 1 else s.g))
    if s.mx:
        h.cache = mk.MxCache(*s.cache)
    if s.op == "evict" and s.mx:
        h.cache_out = mk.MxCache(*s.cache_out)
    if s.op == "attend":
        size = mk.maskkv_attend_mx_workspace_bytes(h.desc, s.cap)
        h.ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    return h


def _call(s):
    if s.call is None:
        s.call = _handle(s)
    h = s.call
    mk = h.mk
    if s.op == "compact":
        mk.maskkv_compact_mx(h.desc, s.K, s.V, s.idx, s.cu, s.cap, h.cache)
        mk.maskkv_expand_mx(h.desc, h.cache, s.cu, s.cap, s.Kc, s.Vc)
        return {"K": s.Kc, "V": s.Vc}
    if s.op == "attend":
        mk.maskkv_attend_mx(h.desc, s.Q, h.cache, s.cu, s.cap, s.Kr, s.Vr, 0.0, s.O, s.lse, h.ws)
        return {"O": s.O, "lse": s.lse.view(s.B * s.H, -1)}
    if s.op == "accumulate":
        if s.mx:
            mk.maskkv_accumulate_mx(h.desc, s.Q, h.cache, s.cu, s.cap, 0.0, s.lse, _DECAY, s.weights, s.weights_out)
        else:
            mk.maskkv_accumulate(h.desc, s.Q, s.K, s.cu, s.cap, 0.0, s.lse, _DECAY, s.weights, s.weights_out)
        return {"weights": s.weights_out}
    if s.mx:
        mk.maskkv_evict_mx(h.desc, s.weights, s.cu, s.cap, s.budgets, h.cache, s.idx, h.cache_out, s.idx_out, s.rows,
                           s.weights_out, s.cu_out, s.cap_out)
        mk.maskkv_expand_mx(h.desc, h.cache_out, s.cu_out, s.cap_out, s.Kc, s.Vc)
    else:
        mk.maskkv_evict(h.desc, s.weights, s.cu, s.cap, s.budgets, s.K, s.V, s.idx, s.Kc, s.Vc, s.idx_out, s.rows,
                        s.weights_out, s.cu_out, s.cap_out)
    return {"K": s.Kc, "V": s.Vc, "rows": s.rows, "idx": s.idx_out, "weights": s.weights_out, "cu": s.cu_out}


def run(s):
    if own:
        return _call(s)
    if s.op == "compact":
        return _compact(s)
    if s.op == "attend":
        return dict(zip(("O", "lse"), _attend(s)))
    return _accumulate(s) if s.op == "accumulate" else _evict(s)


def work(case):
    B, H, g, d, n = (case[k] for k in ("B", "H", "g", "d", "n"))
    eb = 2 if case["dtype"] == "bf16" else 4
    kept = _kept(case)
    rows = sum(kept)
    wide, narrow = d * eb, d // 2 + d // 32              # bytes of a row of K or V
    cached = narrow if case["cache"] == "mx" else wide
    queries = B * H * g * n
    if case["op"] == "compact":              # rows and positions in, packed rows out, and back as the values they stand for
        return {"bytes": rows * (2 * wide + 4 + 2 * narrow) + rows * 2 * wide, "flops": 0}
    if case["op"] == "attend":
        return {"bytes": rows * 2 * cached + 2 * B * H * n * wide + queries * (2 * wide + 4), "flops": 4 * g * n * d * (rows + B * H * n)}
    if case["op"] == "accumulate":
        return {"bytes": rows * (cached + 8) + queries * (wide + 4), "flops": 2 * g * n * d * rows}
    out = sum(min(a, b) for a, b in zip(_budgets(case), kept))       # weights in; rows, weights and positions in and out
    return {"bytes": rows * 4 + out * (4 * cached + 4 + 8 + 4) + (out * 2 * wide if case["cache"] == "mx" else 0), "flops": 0}


# ---- the definitions in 64 bits, one head at a time
def _nearest(x):
    """The 4-bit values of float64 rows, from a list of all sixteen: the nearest, and of two as near the even one."""
    y = x.view(x.shape[0], -1, 1, 32).transpose(2, 3)
    most = y.abs().amax((2, 3), keepdim=True)
    e = torch.ceil(torch.log2(torch.where(most > 0, most, 2.0 ** -130) / 6.0))
    e = torch.where(most > 6.0 * 2.0 ** e, e + 1, torch.where(most <= 6.0 * 2.0 ** (e - 1), e - 1, e)).clamp(-124, 125)
    unit = 2.0 ** e
    even = torch.tensor([0.0, 1.0, 2.0, 4.0], dtype=torch.float64, device=x.device)
    odd = torch.tensor([0.5, 1.5, 3.0, 6.0], dtype=torch.float64, device=x.device)
    size = y.abs() / unit
    a, b = (size - even).abs().min(-1, keepdim=True), (size - odd).abs().min(-1, keepdim=True)
    v = torch.where(a.values <= b.values, even[a.indices], odd[b.indices])
    return (torch.sign(y) * v * unit).reshape(x.shape)


def _stored(s, k):
    """The cached rows that a case's bytes stand for, as float64."""
    if not s.mx:
        return (s.V if k else s.K).double()
    codes, scales = s.cache[2 * k], s.cache[2 * k + 1]
    nibbles = torch.empty((codes.shape[0], s.d), dtype=torch.int64, device=codes.device)
    nibbles[:, 0::2], nibbles[:, 1::2] = codes & 15, codes >> 4
    exponent, half = (nibbles & 7) >> 1, (nibbles & 1).double()          # two bits of exponent, one of mantissa
    size = torch.where(exponent == 0, 0.5 * half, (1.0 + 0.5 * half) * 2.0 ** (exponent.double() - 1))
    size = torch.where(nibbles >= 8, -size, size)
    return size * (2.0 ** (scales.double() - 127)).repeat_interleave(32, 1)


def exact(case, seed):
    s = prepare(case, seed)
    ends = s.cu.tolist()
    heads = [(i, ends[i], ends[i + 1]) for i in range(s.B * s.H)]
    if s.op == "compact":
        K = torch.cat([_nearest(s.K[i // s.H, i % s.H, s.idx[a:b].long()].double()) for i, a, b in heads])
        V = torch.cat([_nearest(s.V[i // s.H, i % s.H, s.idx[a:b].long()].double()) for i, a, b in heads])
        return {"K": K, "V": V}
    K, V = _stored(s, 0), _stored(s, 1)
    if s.op == "evict":
        budgets, chosen = _budgets(case), []
        weights = s.weights.tolist()
        for i, a, b in heads:
            best = sorted(range(a, b), key=lambda r: (-weights[r], r))[:budgets[i]]
            chosen += sorted(best)
        chosen = torch.tensor(chosen, dtype=torch.int64, device="cuda")
        return {"K": K[chosen], "V": V[chosen], "rows": None, "idx": None, "weights": s.weights[chosen].double(), "cu": None}
    scale = float(s.d) ** -0.5
    out, norms, got = [], [], []
    for i, a, b in heads:
        q = s.Q[i // s.H, i % s.H * s.g:(i % s.H + 1) * s.g].double().reshape(-1, s.d)
        if s.op == "accumulate":
            p = torch.exp(q @ K[a:b].T * scale - s.lse.view(s.B * s.H, -1)[i].double()[:, None])
            got.append(_DECAY * s.weights[a:b].double() + p.sum(0))
            continue
        k = torch.cat((K[a:b], s.Kr[i // s.H, i % s.H].double()))
        v = torch.cat((V[a:b], s.Vr[i // s.H, i % s.H].double()))
        logits = q @ k.T * scale
        norm = torch.logsumexp(logits, 1)
        out.append(torch.exp(logits - norm[:, None]) @ v)
        norms.append(norm)
    if s.op == "accumulate":
        return {"weights": torch.cat(got)}
    return {"O": torch.stack(out).view(s.B, s.H * s.g, s.n, s.d), "lse": torch.stack(norms)}
