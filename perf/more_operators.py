"""What the speed of the KV cache held in 8 or 4 bits is measured on: one pass of
each use through the Python binding, beside the same operators in plain torch
operations.

The format, for keys and values apart: the head_dim elements of a row are cut into
blocks of 32.  A block has one scale 2^e, kept as the byte e + 127, and a code for
each element: 8 bits (sign, 4 bits of exponent, 3 of mantissa, at most 448) or 4
bits (sign, 2, 1, at most 6; two to a byte, the even element in the low half).
e is the smallest whole number, -100 at least, with max|x| <= most * 2^e, and an
element's code is the one nearest to x * 2^-e, ties to the even code.

A case is a dict of plain values; its ``kind`` says what one pass does:

  chunk  new tokens' keys and values go into the cache, and the sequences so far
         are read back as packed rows (what a prompt's next part attends to)
  round  the values that a cache would hold for packed rows (the update, which
         recomputes keys and values, has to attend to what the rollout did)
  step   a decode step: every sequence's new token goes into the cache, then its
         queries attend to the sequence

``lens`` seeds a case's own sequence lengths, so that a case always has the same
work; everything else is drawn from the seed given to ``prepare``.
"""
import math
import random

import torch

own = False

BLOCK = 32
LEAST = -100
#: bits: (mantissa bits, exponent of the smallest normal, largest magnitude)
FORMATS = {8: (3, -6, 448.0), 4: (1, 0, 6.0)}


def listed():
    return [
        # a few short prompts of a small model into an 8-bit cache: latency
        {"name": "chunk_short", "kind": "chunk", "seqs": 3, "before_lo": 0, "before_hi": 0, "lo": 5, "hi": 70, "lens": 1,
         "hkv": 2, "dim": 64, "page": 16, "kbits": 8, "vbits": 8, "pad": 3},
        # the prompts of a rollout in one part, 4 bits
        {"name": "chunk_prompts", "kind": "chunk", "seqs": 8, "before_lo": 0, "before_hi": 0, "lo": 1024, "hi": 4096, "lens": 2,
         "hkv": 8, "dim": 128, "page": 64, "kbits": 4, "vbits": 4, "pad": 0},
        # one more part of long prompts: most of what is read is there already; keys in 8 bits, values in 4
        {"name": "chunk_long", "kind": "chunk", "seqs": 3, "before_lo": 8000, "before_hi": 31000, "lo": 500, "hi": 1000, "lens": 3,
         "hkv": 8, "dim": 128, "page": 64, "kbits": 8, "vbits": 4, "pad": 64},
        # the update's rows for a few short samples of a small model
        {"name": "round_small", "kind": "round", "rows": 97, "hkv": 4, "dim": 64, "kbits": 8, "vbits": 8, "heads": 16},
        # the update over a packed batch, keys and values inside the projection's rows
        {"name": "round_pack", "kind": "round", "rows": 39855, "hkv": 8, "dim": 128, "kbits": 4, "vbits": 4, "heads": 32},
        # decode at batch 1: latency
        {"name": "step_one", "kind": "step", "seqs": 1, "lo": 700, "hi": 700, "lens": 4, "hkv": 8, "group": 4, "dim": 128,
         "page": 64, "kbits": 8, "vbits": 8},
        # a small model's decode step, ragged, pages of 16
        {"name": "step_small", "kind": "step", "seqs": 16, "lo": 100, "hi": 3000, "lens": 5, "hkv": 4, "group": 4, "dim": 64,
         "page": 16, "kbits": 4, "vbits": 4},
        # a rollout's step in the middle: ragged sequences, keys in 8 bits, values in 4
        {"name": "step_rollout", "kind": "step", "seqs": 64, "lo": 1280, "hi": 16384, "lens": 6, "hkv": 8, "group": 4, "dim": 128,
         "page": 64, "kbits": 8, "vbits": 4},
        # more query heads to a key head than one matrix instruction's columns
        {"name": "step_wide", "kind": "step", "seqs": 10, "lo": 1500, "hi": 12000, "lens": 7, "hkv": 8, "group": 17, "dim": 128,
         "page": 64, "kbits": 4, "vbits": 4},
        # long contexts in 4 bits, all of the same length
        {"name": "step_long", "kind": "step", "seqs": 8, "lo": 32768, "hi": 32768, "lens": 8, "hkv": 8, "group": 8, "dim": 128,
         "page": 64, "kbits": 4, "vbits": 4},
        # the same in 8 bits
        {"name": "step_long_8", "kind": "step", "seqs": 8, "lo": 32768, "hi": 32768, "lens": 9, "hkv": 8, "group": 8, "dim": 128,
         "page": 64, "kbits": 8, "vbits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["chunk", "round", "step", "step"])
    dim = rng.choice([64, 128])
    kbits, vbits = rng.choice([(8, 8), (4, 4), (8, 4), (4, 8)])
    c = {"kind": kind, "dim": dim, "kbits": kbits, "vbits": vbits}
    if kind == "round":
        hkv = rng.choice([1, 2, 4, 8])
        c.update(rows=_log(rng, 1, 39855), hkv=hkv, heads=hkv * rng.choice([1, 4, 8]))
        return c
    c.update(lens=rng.randrange(1 << 20), hkv=rng.choice([1, 2, 3, 4, 8]), page=rng.choice([16, 32, 64, 256]))
    most = 16 * 4096  # keys of all sequences together, at eight heads
    if kind == "chunk":
        seqs = _log(rng, 1, 64)
        hi = _log(rng, 1, max(1, min(4096, most // seqs // 2)))
        before = rng.choice([0, _log(rng, 1, max(1, most // seqs // 2))])
        c.update(seqs=seqs, before_lo=before // 2, before_hi=before, lo=max(1, hi // 8), hi=hi, pad=rng.choice([0, 1, 40]))
    else:
        seqs = _log(rng, 1, 256)
        group = rng.choice([1, 2, 4, 5, 8, 16, 17, 32])
        hi = _log(rng, 1, min(40000, 32 * most // max(8, group) // seqs))
        c.update(seqs=seqs, lo=max(1, hi // rng.choice([1, 2, 16])), hi=hi, group=group)
    return c


# ---------------------------------------------------------------------------
# the format in plain operations, 32 bits
# ---------------------------------------------------------------------------
def _pow2(e):
    """2^e in fp32 for whole e, as bits: a power function need not be exact."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x, bits):
    """bf16 rows [..., d] -> (codes [..., d * bits / 8], scale bytes [..., d / 32])."""
    mant, least, most = FORMATS[bits]
    a = x.float().unflatten(-1, (-1, BLOCK))
    big = a.abs().amax(-1, keepdim=True).clamp(min=2.0 ** LEAST)
    frac, e = torch.frexp(big)                    # big = frac * 2^e, frac in [0.5, 1)
    mfrac, me = math.frexp(most)
    e = torch.where(frac <= mfrac, e - me, e - me + 1).clamp(min=LEAST)
    a = a * _pow2(-e)
    mag = a.abs()
    top = torch.frexp(mag.clamp(min=2.0 ** least))[1] - 1      # the power of two that an element's steps belong to
    n = torch.round(mag * _pow2(mant - top)).int()             # in steps; half goes to the even one
    code = ((top - least) << mant) + n                         # a rounding up to the next power carries into the exponent
    code = torch.where(torch.signbit(a), code + (1 << bits - 1), code).flatten(-2)
    if bits == 4:
        code = code[..., 0::2] + (code[..., 1::2] << 4)
    return code.to(torch.uint8), (e.squeeze(-1) + 127).to(torch.uint8)


def _values_of_codes(bits):
    mant, least, _ = FORMATS[bits]
    values = []
    for c in range(1 << bits):
        field, m = (c >> mant) & ((1 << bits - 1 - mant) - 1), c & ((1 << mant) - 1)
        v = math.ldexp(m if field == 0 else m + (1 << mant), max(field, 1) - 1 + least - mant)
        values.append(-v if c >> bits - 1 else v)
    return values


def _dequantise(codes, scales, values):
    """The values that codes and scales stand for, in fp32 [..., d]; values: those of all codes of this many bits."""
    if values.numel() == 16:
        codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    v = values[codes.int()].unflatten(-1, (-1, BLOCK))
    return (v * _pow2(scales.int().sub_(127)).unsqueeze(-1)).flatten(-2)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _keys(g, shape):
    """Keys have a few channels that are much larger than the others."""
    x = torch.randn(shape, generator=g, device="cuda")
    x[..., 5::29] *= 6.0
    return x.to(torch.bfloat16)


def _vals(g, shape):
    return (0.5 * torch.randn(shape, generator=g, device="cuda")).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _lens(case):
    """(tokens in the cache before, new tokens) of every sequence."""
    r = random.Random(case["lens"])
    if case["kind"] == "step":
        return [(r.randint(case["lo"], case["hi"]) - 1, 1) for _ in range(case["seqs"])]
    return [(r.randint(case["before_lo"], case["before_hi"]), r.randint(case["lo"], case["hi"])) for _ in range(case["seqs"])]


def prepare(case, seed):
    g = _generator(seed)
    s = {"case": dict(case)}
    s["kvalues"], s["vvalues"] = (torch.tensor(_values_of_codes(case[n]), dtype=torch.float32, device="cuda") for n in ("kbits", "vbits"))
    hkv, dim = case["hkv"], case["dim"]
    if case["kind"] == "round":
        # keys and values are parts of the projection's rows
        heads = case["heads"]
        rows = torch.empty((case["rows"], heads + 2 * hkv, dim), dtype=torch.bfloat16, device="cuda")
        rows[:, :heads] = 1.0
        rows[:, heads:heads + hkv] = _keys(g, (case["rows"], hkv, dim))
        rows[:, heads + hkv:] = _vals(g, (case["rows"], hkv, dim))
        s["k"], s["v"] = rows[:, heads:heads + hkv], rows[:, heads + hkv:]
        return s
    lens, page = _lens(case), case["page"]
    used = [-(-(a + b) // page) for a, b in lens]
    pages = sum(used) + 3
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    table = torch.full((len(lens), max(used)), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(used):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s["table"] = table.cuda()
    # the cache as earlier calls left it, whole pages of it; the new tokens' places hold other values
    s["cache"] = (*_quantise(_keys(g, (pages, hkv, page, dim)), case["kbits"]),
                  *_quantise(_vals(g, (pages, hkv, page, dim)), case["vbits"]))
    pad = case.get("pad", 0)
    new = sum(b for _, b in lens) + pad
    s["k"], s["v"] = _keys(g, (new, hkv, dim)), _vals(g, (new, hkv, dim))
    s["seq"] = _i32([i for i, (_, b) in enumerate(lens) for _ in range(b)] + [0] * pad)
    s["pos"] = _i32([a + j for a, b in lens for j in range(b)] + [-1] * pad)
    if case["kind"] == "chunk":
        s["all_seq"] = _i32([i for i, (a, b) in enumerate(lens) for _ in range(a + b)] + [0] * pad)
        s["all_pos"] = _i32([j for a, b in lens for j in range(a + b)] + [-1] * pad)
    else:
        s["q"] = torch.randn((len(lens), hkv * case["group"], dim), generator=g, device="cuda").to(torch.bfloat16)
        s["len"] = _i32([a + b for a, b in lens])
        s["most"] = max(a + b for a, b in lens)
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2609_35140_amd import uattn
    c = s["case"]
    if c["kind"] == "round":
        return uattn.kv_round_mx(s["k"], s["v"], c["kbits"], c["vbits"])
    uattn.kv_write_mx(s["k"], s["v"], s["table"], s["seq"], s["pos"], *s["cache"])
    if c["kind"] == "chunk":
        return uattn.kv_read_mx(*s["cache"], s["table"], s["all_seq"], s["all_pos"])
    return uattn.decode_mx(s["q"], *s["cache"], s["table"], s["len"], s["most"])


# ---------------------------------------------------------------------------
# the operators in plain operations, 32 bits
# ---------------------------------------------------------------------------
def _places(s, seq, pos):
    """Of the tokens that are not padding: which they are, and their pages and slots."""
    page = s["case"]["page"]
    real = (pos >= 0).nonzero().squeeze(1)
    seq, pos = seq[real].long(), pos[real].long()
    return real, s["table"][seq, pos // page].long(), pos % page


def _plain_write(s):
    c, cache = s["case"], s["cache"]
    real, pages, slots = _places(s, s["seq"], s["pos"])
    parts = (*_quantise(s["k"][real], c["kbits"]), *_quantise(s["v"][real], c["vbits"]))
    cache[0][pages, :, slots], cache[1][pages, :, slots] = parts[0], parts[1]
    cache[2][pages, :, slots], cache[3][pages, :, slots] = parts[2], parts[3]


def _plain_read(s, codes, scales, values):
    real, pages, slots = _places(s, s["all_seq"], s["all_pos"])
    out = torch.zeros((s["all_pos"].shape[0], codes.shape[1], s["case"]["dim"]), dtype=torch.bfloat16, device="cuda")
    out[real] = _dequantise(codes[pages, :, slots], scales[pages, :, slots], values).to(torch.bfloat16)
    return out


def _context(s, codes, scales, values):
    """Every sequence's rows in the order of their positions, fp32 [B, Hkv, pages * page, d]; behind a sequence zeros."""
    table = s["table"].long().clamp(min=0)
    v = _dequantise(codes[table], scales[table], values).transpose(1, 2).flatten(2, 3)
    there = torch.arange(v.shape[2], device="cuda") < s["len"][:, None]
    return v.mul_(there[:, None, :, None])


def _plain_step(s):
    c, cache = s["case"], s["cache"]
    k = _context(s, cache[0], cache[1], s["kvalues"])
    q = s["q"].float().view(k.shape[0], c["hkv"], c["group"], c["dim"])
    x = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(c["dim"])
    del k
    behind = torch.arange(x.shape[3], device="cuda") >= s["len"][:, None]
    x = x.masked_fill_(behind[:, None, None, :], -math.inf)
    p = torch.exp(x - x.amax(3, keepdim=True))
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, _context(s, cache[2], cache[3], s["vvalues"])) / total
    return out.view(s["q"].shape).to(torch.bfloat16)


def run(state):
    if own:
        return _own(state)
    c = state["case"]
    if c["kind"] == "round":
        return tuple(_dequantise(*_quantise(state[n], c[n + "bits"]), state[n + "values"]).to(torch.bfloat16) for n in "kv")
    _plain_write(state)
    if c["kind"] == "step":
        return _plain_step(state)
    cache = state["cache"]
    return _plain_read(state, cache[0], cache[1], state["kvalues"]), _plain_read(state, cache[2], cache[3], state["vvalues"])


# ---------------------------------------------------------------------------
# minimal work, and the outputs in 64 bits
# ---------------------------------------------------------------------------
def work(case):
    hkv, dim = case["hkv"], case["dim"]
    held = (case["kbits"] + case["vbits"]) / 8 + 2 / BLOCK  # bytes of an element of K and its fellow of V, with their scales
    if case["kind"] == "round":
        n = case["rows"] * hkv * dim
        return {"bytes": 8 * n, "flops": 8 * n}
    lens = _lens(case)
    new, all_ = sum(b for _, b in lens), sum(a + b for a, b in lens)
    wrote = new * hkv * dim * (4 + held) + 8 * new
    if case["kind"] == "chunk":
        return {"bytes": wrote + all_ * hkv * dim * (held + 4) + 8 * all_ + 4 * case["pad"] * hkv * dim,
                "flops": hkv * dim * (6 * new + 2 * all_)}
    heads = hkv * case["group"]
    return {"bytes": wrote + all_ * hkv * dim * held + 4 * len(lens) * heads * dim, "flops": 4 * all_ * heads * dim}


def _power(e):
    """2^e in fp64 for whole e of any type."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _nearest(x, bits):
    """The values that a cache holds for rows x, in fp64: a search among all magnitudes that a code can have."""
    mags = sorted({abs(v) for v in _lattice(bits)})
    grid = torch.tensor(mags, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    most = FORMATS[bits][2]
    v = x.double().unflatten(-1, (-1, BLOCK))
    big = v.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(big / most)).clamp(min=LEAST)
    e = torch.where(big > most * _power(e), e + 1, e)
    e = torch.where(big <= most * _power(e - 1), e - 1, e).clamp(min=LEAST)
    y = v / _power(e)
    n = torch.bucketize(y.abs(), middle)                               # magnitudes below, halves counted down
    half = y.abs() == middle[n.clamp(max=middle.numel() - 1)]
    n = n + (half & (n % 2 == 1)).long()
    return (torch.sign(y) * grid[n] * _power(e)).flatten(-2)


def _lattice(bits):
    """Magnitudes of all codes by the definition: 2^(field - bias) * (1 + m / 2^mant), or m / 2^mant * 2^least."""
    mant, least, most = FORMATS[bits]
    powers = range(least, int(math.log2(most)) + 1)
    small = [m / 2 ** mant * 2.0 ** least for m in range(2 ** mant)]
    return small + [(1 + m / 2 ** mant) * 2.0 ** p for p in powers for m in range(2 ** mant) if (1 + m / 2 ** mant) * 2.0 ** p <= most]


def _held(codes, scales, bits):
    """The values of a cache's rows in fp64, from the bits of each code."""
    mant, least, _ = FORMATS[bits]
    if bits == 4:
        codes = torch.stack([codes % 16, codes // 16], -1).flatten(-2)
    c = codes.long()
    m, field, neg = c % 2 ** mant, c // 2 ** mant % 2 ** (bits - 1 - mant), c // 2 ** (bits - 1)
    v = torch.where(field == 0, m.double() / 2 ** mant * 2.0 ** least, (1 + m.double() / 2 ** mant) * _power(field + least - 1))
    v = torch.where(neg == 1, -v, v).unflatten(-1, (-1, BLOCK))
    return (v * _power(scales.long() - 127)[..., None]).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    bits = {"k": case["kbits"], "v": case["vbits"]}
    if case["kind"] == "round":
        return tuple(_nearest(s[n], bits[n]) for n in "kv")
    lens, page = _lens(case), case["page"]
    parts = {"k": s["cache"][:2], "v": s["cache"][2:]}
    new = {n: _nearest(s[n], bits[n]) for n in "kv"}
    out, at = [], 0
    for i, (before, count) in enumerate(lens):
        rows = {}
        for n in "kv":
            held = _held(*(t[s["table"][i, :-(-(before + count) // page)].long()] for t in parts[n]), bits[n])
            held = held.transpose(0, 1).flatten(1, 2)[:, :before]      # [Hkv, tokens before, d]
            rows[n] = torch.cat([held, new[n][at:at + count].transpose(0, 1)], 1)
        at += count
        if case["kind"] == "chunk":
            out.append({n: rows[n].transpose(0, 1) for n in "kv"})
            continue
        q = s["q"][i].double().view(case["hkv"], case["group"], -1)
        w = torch.softmax(torch.matmul(q, rows["k"].transpose(1, 2).contiguous()) / math.sqrt(case["dim"]), 2)
        out.append(torch.matmul(w, rows["v"]).flatten(0, 1))
    if case["kind"] == "step":
        return torch.stack(out)
    pad = torch.zeros((case["pad"], case["hkv"], case["dim"]), dtype=torch.float64, device="cuda")
    return tuple(torch.cat([r[n] for r in out] + [pad]) for n in "kv")
