"""The operators around attention, as a program of the library's users calls them:

  rotary   positions with several axes on Q and K, and the gradients' way back
  cache    keys and values quantised into a paged 4-bit cache, and read back
  attend   attention of new tokens over such a cache

`listed()` and `draw()` give the cases, `prepare()` a case's inputs, `run()` one
pass: in elementary torch operations, or where `own` is true by the library's
calls.  `exact()` computes the same in 64 bits.

The cache's format (both sides take its bytes as they are): elements are e2m1
(0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives), 32 of them along the head
dimension share a power of two, stored as its exponent plus 127.  The power of
a block whose largest magnitude is a is 2^(e - 2), e the exponent of a, or one
more where a >= 1.75 * 2^e (which would round past 6).  A page of `page`
tokens holds, for each head and each 32 tokens, 34 d bytes: K's codes
[d/32][32 tokens][16], V's codes [d/32][16 pairs][4][2][4] (token 16 b + 4 a + c
at [a][b][c]), K's exponents [16][d/32][2] (token 16 b + a at [a][.][b]) and
V's exponents [4][d/32][2][4] (tokens as V's codes).  A byte holds elements
2 i (low half) and 2 i + 1 of its token.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "f16": 2, "bf16": 2}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # the next token of 64 sequences: text, image and video positions mixed, far into their contexts
        {"name": "rotary_step", "op": "rotary", "B": 64, "L": 1, "Hq": 16, "Hk": 8, "d": 128, "dtype": "bf16",
         "axes": 3, "rot": 128, "pairs": "half", "spectrum": "shared", "far": 1000000, "inverse": False},
        # a video's latent grid before a long bidirectional call
        {"name": "rotary_video", "op": "rotary", "B": 1, "L": 32768, "Hq": 16, "Hk": 16, "d": 128, "dtype": "bf16",
         "axes": 3, "rot": 128, "pairs": "adjacent", "spectrum": "per_axis", "far": 128, "inverse": False},
        # the fp32 gradients that the backward leaves, back through the rotation of an image's tokens
        {"name": "rotary_grad", "op": "rotary", "B": 2, "L": 65536, "Hq": 8, "Hk": 8, "d": 64, "dtype": "f32",
         "axes": 2, "rot": 64, "pairs": "half", "spectrum": "per_axis", "far": 256, "inverse": True},
        # one new token of each of 64 sequences joins the cache
        {"name": "cache_step", "op": "cache", "B": 64, "L": 1, "H": 8, "d": 128, "dtype": "bf16", "page": 64,
         "max_len": 8192, "packed": False},
        # ragged prompts, packed, that begin and end inside pages
        {"name": "cache_ragged", "op": "cache", "B": 7, "L": 1501, "H": 5, "d": 96, "dtype": "f16", "page": 32,
         "max_len": 2111, "packed": True},
        # a whole long prompt
        {"name": "cache_prompt", "op": "cache", "B": 1, "L": 262144, "H": 8, "d": 64, "dtype": "bf16", "page": 256,
         "max_len": 262144, "packed": False},
        # one sequence's next token over a short cache: latency
        {"name": "step_one", "op": "attend", "B": 1, "L": 1, "Hq": 16, "Hk": 8, "d": 128, "dtype": "bf16",
         "page": 64, "max_len": 1000, "packed": False, "causal": True},
        # a serving batch's next tokens, grouped heads, contexts of all lengths
        {"name": "step_batch", "op": "attend", "B": 64, "L": 1, "Hq": 32, "Hk": 8, "d": 128, "dtype": "bf16",
         "page": 64, "max_len": 16384, "packed": False, "causal": True},
        # the next token of one sequence of a million
        {"name": "step_long", "op": "attend", "B": 1, "L": 1, "Hq": 16, "Hk": 8, "d": 128, "dtype": "bf16",
         "page": 256, "max_len": 1048576, "packed": False, "causal": True},
        # five drafted tokens at once, a head of keys for each head of queries
        {"name": "draft", "op": "attend", "B": 16, "L": 5, "Hq": 8, "Hk": 8, "d": 64, "dtype": "f16",
         "page": 128, "max_len": 8192, "packed": False, "causal": True},
        # ragged chunks, packed, in full precision
        {"name": "chunk_ragged", "op": "attend", "B": 3, "L": 203, "Hq": 12, "Hk": 4, "d": 96, "dtype": "f32",
         "page": 32, "max_len": 3001, "packed": True, "causal": True},
        # a chunk of a long prompt over what came before
        {"name": "chunk_long", "op": "attend", "B": 1, "L": 4096, "Hq": 16, "Hk": 4, "d": 128, "dtype": "bf16",
         "page": 64, "max_len": 32768, "packed": False, "causal": True},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary", "cache", "attend", "attend"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "rotary":
        d = 32 * rng.randint(1, 8)
        Hq = _spread(rng, 1, 32)
        Hk = rng.choice([0, Hq, max(1, Hq // rng.randint(2, 8))])
        rows = _spread(rng, 1, 2 * 65536 * 16 * 64 // ((Hq + Hk) * d))
        B = min(rows, rng.choice([1, 1, 2, 3, 17, 64]))
        return {"op": op, "B": B, "L": rows // B, "Hq": Hq, "Hk": Hk, "d": d, "dtype": dtype,
                "axes": rng.randint(1, 4), "rot": 16 * rng.randint(1, d // 16),
                "pairs": rng.choice(["half", "adjacent"]), "spectrum": rng.choice(["shared", "per_axis"]),
                "far": _spread(rng, 16, 4000000), "inverse": rng.random() < 0.4}
    d = 32 * rng.randint(1, 8)
    page = rng.choice([32, 64, 128, 256])
    packed = rng.random() < 0.5
    if op == "cache":
        H = _spread(rng, 1, 16)
        rows = _spread(rng, 1, 262144 * 8 * 64 // (H * d))
        B = min(rows, rng.choice([1, 2, 5, 31, 64]))
        L = max(1, rows // B)
        return {"op": op, "B": B, "L": L, "H": H, "d": d, "dtype": dtype, "page": page,
                "max_len": L + rng.randint(0, 4000), "packed": packed}
    Hk = _spread(rng, 1, 16)
    Hq = Hk * rng.choice([1, 1, 2, 4, 5, 8, 16])
    L = rng.choice([1, 1, rng.randint(2, 9), _spread(rng, 10, 4096)])
    B = rng.choice([1, 1, 2, 3, 16, 64])
    most = min(2 ** 20, 64 * 16384 * 8 * 128 // (B * Hk * d), 4096 * 32768 * 16 * 128 // (B * Hq * d * L))
    return {"op": op, "B": B, "L": L, "Hq": Hq, "Hk": Hk, "d": d, "dtype": dtype, "page": page,
            "max_len": _spread(rng, 1, max(1, most)), "packed": packed, "causal": rng.random() < 0.8}


def _shape(c):
    """Per sequence: the tokens in the cache after the call, and how many of them (or of the queries) are new.

    The first sequence is the longest; the others end anywhere, some of many with nothing."""
    frac = [1.0] + [(b * 0.6180339887) % 1.0 for b in range(1, c["B"])]
    lens = [max(int(c["max_len"] * f), 0) for f in frac]
    new = [max(0, int(c["L"] * (f if b else 1.0) + 0.5)) for b, f in enumerate(reversed(frac))] if c["packed"] else [c["L"]] * c["B"]
    if c["packed"]:
        new[0] = c["L"]
    if c["op"] == "cache":
        lens = [max(n, m) for n, m in zip(lens, new)]
    return lens, new


def work(c):
    if c["op"] == "rotary":
        n = c["B"] * c["L"] * (c["Hq"] + c["Hk"]) * c["d"]
        # each value is read and written once; two products and a sum for each rotated one
        return {"bytes": 2 * n * SIZES[c["dtype"]] + 4 * c["axes"] * c["B"] * c["L"],
                "flops": 3 * n * c["rot"] // c["d"]}
    lens, new = _shape(c)
    if c["op"] == "cache":
        n = sum(new) * c["H"] * c["d"]
        # K and V in, their codes and exponents out; and the way back
        return {"bytes": 2 * 2 * n * SIZES[c["dtype"]] + 2 * n * 34 // 32, "flops": 8 * n}
    seen = 0
    for n, m in zip(lens, new):
        for_each = n * m
        if c["causal"]:  # query i of m sees n - m + 1 + i tokens, none where that is not positive
            first = max(0, m - n)
            for_each = (m - first) * (n - m + 1 + first + n) // 2 if m > first else 0
        seen += for_each
    read = sum(n if m and not (c["causal"] and n == 0) else 0 for n, m in zip(lens, new))
    rows = sum(new) * c["Hq"]
    return {"bytes": read * c["Hk"] * c["d"] * 34 // 32 + 2 * rows * c["d"] * SIZES[c["dtype"]] + 4 * rows,
            "flops": 4 * seen * c["Hq"] * c["d"]}


# ---------------------------------------------------------------- the inputs
def _sections(c):
    """Pairs of each axis: as even as they go, the first axes smaller."""
    n, a = c["rot"] // 2, c["axes"]
    return [(i + 1) * n // a - i * n // a for i in range(a)]


def _quantise(x):
    """Codes (an int64 each) and exponents of blocks of 32 along the last dimension; x fp32."""
    blocks = x.unflatten(-1, (x.shape[-1] // 32, 32))
    top = blocks.abs().amax(-1)
    e = torch.frexp(top)
    power = torch.where(top > 0, e.exponent - 3 + (e.mantissa >= 0.875), -127).clamp(-127, 127)
    u = torch.ldexp(blocks, -power.unsqueeze(-1)).abs()
    # borders between neighbouring levels; a tie goes to the level of even code
    at = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device)
    code = torch.bucketize(u, at, right=False) + ((u == 0.75) | (u == 1.75) | (u == 3.5)).long()
    return (code + 8 * (blocks < 0)).flatten(-2), (power + 127).to(torch.uint8)


def _bytes_of(codes):
    return (codes[..., 0::2] + 16 * codes[..., 1::2]).to(torch.uint8)


def _tiles(k, v):
    """34 d bytes for each 32 tokens of k and v [..., 32, d] (fp32), in the cache's order."""
    d = k.shape[-1]
    lead = k.shape[:-2]
    kc, ke = _quantise(k)
    vc, ve = _quantise(v)
    kc = _bytes_of(kc).reshape(*lead, 32, d // 32, 16).transpose(-3, -2)
    vc = _bytes_of(vc).reshape(*lead, 2, 4, 4, d // 32, 16).movedim((-2, -1, -4, -5, -3), (-5, -4, -3, -2, -1))
    ke = ke.reshape(*lead, 2, 16, d // 32).movedim((-2, -1, -3), (-3, -2, -1))
    ve = ve.reshape(*lead, 2, 4, 4, d // 32).movedim((-3, -1, -4, -2), (-4, -3, -2, -1))
    return torch.cat([x.flatten(len(lead)) for x in (kc, vc, ke, ve)], -1)


def _keys(g, shape, device):
    """Keys have channels that are larger than the others throughout."""
    k = torch.randn(shape, generator=g, device=device)
    d = shape[-1]
    gain = torch.ones(d, device=device)
    gain[torch.arange(3, d, 17, device=device)] = 4.0
    return k * gain


def prepare(c, seed):
    dev = "cuda"
    g = torch.Generator(dev)
    g.manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]
    s = {"c": c}
    if own:
        import paper_2604_20819_amd as cq
        s["cq"] = cq
    if c["op"] == "rotary":
        heads = [h for h in (c["Hq"], c["Hk"]) if h]
        s["x"] = [torch.randn(c["B"], c["L"], h, c["d"], generator=g, device=dev).to(dt) for h in heads]
        s["y"] = [torch.empty_like(x) for x in s["x"]]
        s["pos"] = torch.randint(0, c["far"], (c["axes"], c["B"], c["L"]), generator=g, device=dev, dtype=torch.int32)
        if own:
            s["plan"] = cq.cqsa_rotary_plan(c["d"], _sections(c), theta=10000.0, pairs=c["pairs"],
                                            spectrum=c["spectrum"])
        return s
    lens, new = _shape(c)
    H = c["H"] if c["op"] == "cache" else c["Hk"]
    P, d, B = c["page"], c["d"], c["B"]
    need = [-(-n // P) for n in lens]
    most = max(max(need), 1)
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device=dev)
    # the pages of a sequence lie anywhere in the pool; the table's unused entries hold -1
    left = torch.tensor(need).cumsum(0) - torch.tensor(need)
    col = torch.arange(most).expand(B, most)
    idx = (col + left[:, None]).clamp(max=n_pages - 1).to(dev)
    s["pages"] = torch.where(col.to(dev) < torch.tensor(need, device=dev)[:, None], order[idx], -1).to(torch.int32)
    s["lengths"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    start = torch.tensor([0] + new).cumsum(0)
    s["start"] = start.to(dev, torch.int32) if c["packed"] else None
    rows = (1, max(1, int(start[-1]))) if c["packed"] else (B, c["L"])
    if c["op"] == "cache":
        s["k"] = _keys(g, (*rows, H, d), dev).to(dt)
        s["v"] = torch.randn(*rows, H, d, generator=g, device=dev).to(dt)
        s["data"] = torch.zeros(n_pages, H * (P // 32) * 34 * d, dtype=torch.uint8, device=dev)
        s["codes"] = torch.zeros(n_pages * P, 2, H, d // 2, dtype=torch.uint8, device=dev)
        s["powers"] = torch.zeros(n_pages * P, 2, H, d // 32, dtype=torch.uint8, device=dev)
        s["ko"], s["vo"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    else:
        s["data"] = torch.empty(n_pages, H * (P // 32) * 34 * d, dtype=torch.uint8, device=dev)
        step = max(1, 2 ** 26 // (H * P * d))
        for i in range(0, n_pages, step):  # a part of the pool at a time: it may be large
            m = min(step, n_pages - i)
            k = _keys(g, (m, H, P // 32, 32, d), dev)
            v = torch.randn(m, H, P // 32, 32, d, generator=g, device=dev)
            s["data"][i:i + m] = _tiles(k, v).reshape(m, -1)
        s["q"] = torch.randn(*rows, c["Hq"], d, generator=g, device=dev).to(dt)
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(rows[0], c["Hq"], rows[1], device=dev)
    if own:
        s["cache"] = cq.Cache4(n_pages, H, d, page_size=P, data=s["data"])
        s["batch"] = cq.CacheBatch(s["pages"], s["lengths"], q_start=s["start"], max_len=max(c["max_len"], 1),
                                   max_q=c["L"] if c["packed"] else 0)
        if c["op"] == "attend":
            s["space"] = cq.cqsa_cache_attend_workspace(s["cache"], s["batch"], s["q"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    c = s["c"]
    if own:
        cq = s["cq"]
        if c["op"] == "rotary":
            cq.cqsa_rotary(s["plan"], s["pos"], s["x"], s["y"], inverse=c["inverse"])
            return s["y"]
        if c["op"] == "cache":
            cq.cqsa_cache_write(s["cache"], s["batch"], s["k"], s["v"])
            cq.cqsa_cache_read(s["cache"], s["batch"], s["ko"], s["vo"])
            return s["ko"], s["vo"]
        cq.cqsa_cache_attend(s["cache"], s["batch"], s["q"], s["o"], s["lse"], causal=c["causal"],
                             workspace=s["space"])
        return s["o"], s["lse"]
    if c["op"] == "rotary":
        return _rotary(s)
    return _cache(s) if c["op"] == "cache" else _attend(s)


def _rotary(s):
    c = s["c"]
    pos, half = s["pos"], c["rot"] // 2
    dev = pos.device
    secs = torch.tensor(_sections(c), device=dev)
    axis = torch.repeat_interleave(torch.arange(c["axes"], device=dev), secs, output_size=half)
    pair = torch.arange(half, device=dev, dtype=torch.float64)
    if c["spectrum"] == "shared":
        turn = pair / half
    else:
        turn = (pair - (secs.cumsum(0) - secs)[axis]) / secs[axis]
    # positions may be far: the angles in 64 bits
    angle = pos.double()[axis].movedim(0, -1) * 10000.0 ** -turn
    if c["inverse"]:
        angle = -angle
    cos, sin = angle.cos().float().unsqueeze(2), angle.sin().float().unsqueeze(2)

    def turned(x):
        y = x.float()
        if c["pairs"] == "half":
            a, b = y[..., :half], y[..., half:2 * half]
            return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., 2 * half:]], -1).to(x.dtype)
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        both = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        return torch.cat([both, y[..., 2 * half:]], -1).to(x.dtype)

    return [turned(x) for x in s["x"]]


def _rows_of(s, total):
    """For each of `total` rows (all sequences'): its sequence and its place among the sequence's new tokens."""
    c = s["c"]
    row = torch.arange(total, device=s["lengths"].device)
    if not c["packed"]:
        return row // c["L"], row % c["L"], torch.full_like(s["lengths"], c["L"]).long()
    start = s["start"].long()
    b = torch.searchsorted(start, row, right=True).sub(1).clamp(max=c["B"] - 1)
    return b, row - start[b], start[1:] - start[:-1]


def _values(codes, powers):
    """fp32 values of packed codes [..., d/2] and exponents [..., d/32]."""
    table = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=codes.device)
    both = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    scale = torch.ldexp(torch.ones((), device=codes.device), powers.int() - 127)
    return (table[both.int()].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _cache(s):
    c = s["c"]
    k, v = (x.flatten(0, 1).float() for x in (s["k"], s["v"]))
    b, i, new = _rows_of(s, k.shape[0])
    at = s["lengths"].long()[b] - new[b] + i
    slot = s["pages"].long()[b, at // c["page"]] * c["page"] + at % c["page"]
    codes, powers = _quantise(torch.stack([k, v], 1))
    s["codes"][slot] = _bytes_of(codes)
    s["powers"][slot] = powers
    both = _values(s["codes"][slot], s["powers"][slot]).to(s["k"].dtype)
    return both[:, 0].reshape(s["k"].shape), both[:, 1].reshape(s["v"].shape)


def _attend(s):
    c = s["c"]
    H, d, B, P = c["Hk"], c["d"], c["B"], c["page"]
    G = c["Hq"] // H
    tiles = s["data"][s["pages"].clamp(min=0).long()].reshape(B, -1, H, P // 32, 34 * d)
    tiles = tiles.transpose(1, 2).reshape(B, H, -1, 34 * d)
    kc, vc, ke, ve = tiles.split([16 * d, 16 * d, d, d], -1)
    n = tiles.shape[2] * 32
    kc = kc.unflatten(-1, (d // 32, 32, 16)).transpose(-3, -2).reshape(B, H, n, d // 2)
    ke = ke.unflatten(-1, (16, d // 32, 2)).movedim(-1, -3).reshape(B, H, n, d // 32)
    vc = vc.unflatten(-1, (d // 32, 16, 4, 2, 4)).permute(0, 1, 2, 6, 5, 7, 3, 4).reshape(B, H, n, d // 2)
    ve = ve.unflatten(-1, (4, d // 32, 2, 4)).permute(0, 1, 2, 5, 3, 6, 4).reshape(B, H, n, d // 32)
    k, v = _values(kc, ke), _values(vc, ve)
    q = s["q"].flatten(0, 1).float()
    row_b, row_i, new = _rows_of(s, q.shape[0])
    padded = q.new_zeros(B, c["L"], c["Hq"], d)
    padded[row_b, row_i] = q
    x = padded.reshape(B, c["L"], H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * c["L"], d)
    scores = torch.matmul(x, k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    key = torch.arange(n, device=q.device)
    seen = s["lengths"].long()[:, None].expand(B, c["L"])
    if c["causal"]:
        seen = seen - new[:, None] + 1 + torch.arange(c["L"], device=q.device)
    hidden = (key >= seen[..., None])[:, None, None].expand(B, 1, G, c["L"], n).reshape(B, 1, G * c["L"], n)
    scores.masked_fill_(hidden, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=-3e38)
    weights = scores.sub_(top).exp_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights, v) / total.clamp(min=1e-38)
    lse = (top + total.log()).squeeze(-1)
    out = out.reshape(B, H, G, c["L"], d).permute(0, 3, 1, 2, 4).reshape(B, c["L"], c["Hq"], d)
    lse = lse.reshape(B, H, G, c["L"]).permute(0, 3, 1, 2).reshape(B, c["L"], c["Hq"])
    o = out[row_b, row_i].to(s["q"].dtype).reshape(s["q"].shape)
    lse = lse[row_b, row_i].reshape(*s["q"].shape[:3]).transpose(1, 2).contiguous()
    return o, lse


# ---------------------------------------------------------------- in 64 bits
def exact(c, seed):
    global own
    was, own = own, False
    try:
        s = prepare(c, seed)
    finally:
        own = was
    if c["op"] == "rotary":
        return _exact_rotary(c, s)
    if c["op"] == "cache":
        return [_exact_rounded(x) for x in (s["k"], s["v"])]
    return _exact_attend(c, s)


def _exact_rotary(c, s):
    half = c["rot"] // 2
    freq, axis = [], []
    for a, n in enumerate(_sections(c)):
        for j in range(n):
            freq.append(10000.0 ** (-(len(freq) / half if c["spectrum"] == "shared" else j / n)))
            axis.append(a)
    dev = s["pos"].device
    w = torch.tensor(freq, dtype=torch.float64, device=dev)
    angle = s["pos"].double()[torch.tensor(axis, device=dev)].permute(1, 2, 0) * w
    turn = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)[:, :, None]
    i = torch.arange(half, device=dev)
    first, second = (i, i + half) if c["pairs"] == "half" else (2 * i, 2 * i + 1)
    out = []
    for x in s["x"]:
        y = x.double()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return out


def _exact_rounded(x):
    """Every block's values at the nearest multiple that its power allows, by division and steps."""
    y = x.double().unflatten(-1, (x.shape[-1] // 32, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140)))
    e = e + (2 * 2.0 ** e <= top).double() - (2.0 ** e > top).double()
    power = (e - 2 + (top >= 1.75 * 2.0 ** e).double()).clamp(min=-127.0)
    u = (y.abs() / 2.0 ** power).clamp(max=6.0)
    step = torch.where(u < 2, 0.5, torch.where(u < 4, 1.0, 2.0))
    return (torch.round(u / step) * step * 2.0 ** power * torch.sign(y)).flatten(-2)


def _exact_attend(c, s):
    H, d, P = c["Hk"], c["d"], c["page"]
    G = c["Hq"] // H
    dev = s["q"].device
    lens, new = _shape(c)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=dev)
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), dtype=torch.float64, device=dev)
    e = torch.arange(d, device=dev)
    begin = 0
    for b, (n, m) in enumerate(zip(lens, new)):
        for h in range(H if n else 0):
            # a token's bytes by their offsets in its 32 tokens' 34 d
            at = torch.arange(n, device=dev)
            t = at % 32
            base = (s["pages"][b].long()[at // P] * H + h) * (P * 34 * d // 32) + at % P // 32 * (34 * d)
            blk, sub = e // 32, e % 32 // 2
            row = t // 4 % 4 * 8 + t // 16 * 4 + t % 4
            k_at = (blk * 512 + sub)[None] + (t * 16)[:, None]
            v_at = (16 * d + blk * 512 + sub * 32)[None] + row[:, None]
            ke_at = (32 * d + 2 * blk)[None] + (t % 16 * (d // 16) + t // 16)[:, None]
            ve_at = (33 * d + 8 * blk)[None] + (t // 4 % 4 * (d // 4) + t // 16 * 4 + t % 4)[:, None]
            flat = s["data"].view(-1)
            kv = []
            for code, power in ((k_at, ke_at), (v_at, ve_at)):
                nib = flat[base[:, None] + code].int() >> (4 * (e % 2)).int() & 15
                kv.append(level[nib] * 2.0 ** (flat[base[:, None] + power].double() - 127))
            r = slice(begin, begin + m) if c["packed"] else slice(None)
            q = s["q"][0 if c["packed"] else b, r, h * G:(h + 1) * G].double()
            x = torch.matmul(q.transpose(0, 1).reshape(-1, d), kv[0].t()) / math.sqrt(d)
            if c["causal"]:
                last = n - m + torch.arange(m, device=dev).repeat(G)
                x = x.masked_fill(at[None] > last[:, None], -math.inf)
            z = torch.logsumexp(x, -1)
            w = torch.exp(x - z.clamp(min=-1e300)[:, None])
            o = torch.matmul(w, kv[1]).reshape(G, m, d).transpose(0, 1)
            out[0 if c["packed"] else b, r, h * G:(h + 1) * G] = o
            lse[0 if c["packed"] else b, h * G:(h + 1) * G, r] = z.reshape(G, m)
        begin += m
    return out, lse
