"""What the speed of the row-wise operators around the attention is measured on:
one pass of each through the Python binding, beside the same operator in plain
torch operations.

A case is a dict of plain values; its ``kind`` says which operator one pass runs:

  norm         the seam between two blocks: the block output's norm, its gate
               and scale, the residual sum, the next block's norm
  norm_grad    the gradients of the same
  embed        rows of the embedding table for a pack of tokens
  embed_grad   the table's gradient, every row of it
  logits       penalties for repeated tokens, biases and grammar masks
  logits_grad  the gradient of the same
  logp_grad    the logits' gradient of the token log-probability

``lens`` seeds a case's own sequence lengths, so that a case always has the same
work; everything else is drawn from the seed given to ``prepare``.
"""
import math
import random

import torch

own = False

EPS = 1.0e-6
VOCAB = 151936


def listed():
    return [
        # the norm before a block for one new token: the latency of a decode step at batch 1
        {"name": "norm_token", "kind": "norm", "rows": 1, "hidden": 4096, "block": False, "post": False, "gate": "none",
         "scale": 1.0},
        # prompts of a rollout through a block with norms on both sides and a learned gate
        {"name": "norm_prompts", "kind": "norm", "rows": 9815, "hidden": 4096, "block": True, "post": True, "gate": "shared",
         "scale": 0.5},
        # a small model's update, residual sum and norm
        {"name": "norm_grad_small", "kind": "norm_grad", "rows": 1500, "hidden": 1024, "block": True, "post": False,
         "gate": "none", "scale": 1.0},
        # the policy update over a pack: both norms, a gate of every token's own
        {"name": "norm_grad_pack", "kind": "norm_grad", "rows": 8191, "hidden": 4096, "block": True, "post": True,
         "gate": "token", "scale": 0.25},
        # the tokens of a packed update batch, some rows padded
        {"name": "embed_pack", "kind": "embed", "rows": 39855, "hidden": 4096, "vocab": VOCAB, "scale": 1.0},
        # a small model's table gradient in its weights' type
        {"name": "embed_grad_small", "kind": "embed_grad", "rows": 1900, "hidden": 1024, "vocab": 32000, "scale": 32.0,
         "fp32": False},
        # the update's table gradient in fp32: most rows have no token
        {"name": "embed_grad_pack", "kind": "embed_grad", "rows": 16384, "hidden": 4096, "vocab": VOCAB, "scale": 1.0,
         "fp32": True},
        # a decode step of a small rollout batch: a grammar on half of the sequences, biases on all
        {"name": "logits_step", "kind": "logits", "mode": "step", "batch": 8, "prompt": 1024, "lo": 100, "hi": 3000, "lens": 1,
         "vocab": VOCAB, "bias": 100, "masks": 4},
        # the update's logits over a micro-batch of response tokens: every row's history is its prefix
        {"name": "logits_update", "kind": "logits", "mode": "update", "batch": 4, "prompt": 1024, "lo": 700, "hi": 1300,
         "lens": 2, "vocab": VOCAB, "bias": 0, "masks": 0},
        # their gradient, with a grammar to some requests
        {"name": "logits_grad_update", "kind": "logits_grad", "mode": "update", "batch": 3, "prompt": 500, "lo": 200, "hi": 600,
         "lens": 3, "vocab": 128256, "bias": 0, "masks": 2},
        # the log-probability's gradient over a micro-batch of response tokens
        {"name": "logp_grad_update", "kind": "logp_grad", "rows": 4100, "vocab": VOCAB, "inv_temperature": 1.0},
        # the same for a few short samples of a model with an odd vocabulary
        {"name": "logp_grad_small", "kind": "logp_grad", "rows": 77, "vocab": 50257, "inv_temperature": 1.25},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "embed", "embed_grad", "logits", "logits_grad", "logp_grad"])
    c = {"kind": kind}
    if kind in ("norm", "norm_grad"):
        hidden = 8 * _log(rng, 32, 1024)
        most = (9815 if kind == "norm" else 8191) * 4096 // hidden
        c.update(rows=_log(rng, 1, most), hidden=hidden, block=kind == "norm_grad" or rng.random() < 0.8,
                 post=rng.random() < 0.5, gate=rng.choice(["none", "shared", "token"]), scale=rng.choice([1.0, 0.5, 0.22]))
        if not c["block"]:
            c.update(post=False, gate="none", scale=1.0)
    elif kind in ("embed", "embed_grad"):
        hidden = 8 * _log(rng, 32, 640)
        c.update(rows=_log(rng, 1, (39855 if kind == "embed" else 16384) * 4096 // max(4096, hidden)), hidden=hidden,
                 vocab=rng.choice([32000, 50257, 128256, VOCAB]), scale=rng.choice([1.0, round(math.sqrt(hidden), 3)]))
        if kind == "embed_grad":
            c.update(fp32=rng.random() < 0.5)
            if hidden > 4096:
                c.update(vocab=32000)
    elif kind in ("logits", "logits_grad"):
        mode = rng.choice(["step", "update"])
        hi = _log(rng, 16, 4000 if mode == "step" else 900)
        c.update(mode=mode, batch=_log(rng, 1, 256) if mode == "step" else rng.randint(1, 4), prompt=_log(rng, 1, 4000), lo=max(1, hi // 8),
                 hi=hi, lens=rng.randrange(1 << 20), vocab=rng.choice([32000, 50257, 128256, VOCAB]),
                 bias=rng.choice([0, 30, 300]) if kind == "logits" else 0, masks=rng.choice([0, 1, 3]))
    else:
        c.update(rows=_log(rng, 1, 4000), vocab=rng.choice([32000, 50257, 128256, VOCAB]),
                 inv_temperature=rng.choice([1.0, 0.7, 1.25]))
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, shape, sigma=1.0, mean=0.0):
    return (torch.randn(shape, generator=g, device="cuda") * sigma + mean).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _tokens(g, n, vocab):
    """Token ids as text has them: the k-th most frequent about 1/k as often as the first, spread over the vocabulary."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    k = torch.exp(u * math.log(vocab)).long().clamp(1, vocab) - 1
    return (k * 7919 % vocab).to(torch.int32)


def _rows(g, rows, vocab, sigma):
    """[rows, vocab] bf16 whose rows start at multiples of 16 bytes, as the LM head lays its logits out."""
    stride = (vocab + 7) // 8 * 8
    return _normal(g, (rows, stride), sigma)[:, :vocab]


def _lens(case):
    r = random.Random(case["lens"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


def _num_rows(case):
    return case["batch"] if case["mode"] == "step" else sum(_lens(case))


def _prepare_logits(case, g, s):
    """Sequences of a prompt and a response each, packed one after another; a row has the part of the packed tokens that came
    before its own: the whole sequence so far in a decode step, the prefix of a response position in the update."""
    lens, prompt, vocab = _lens(case), case["prompt"], case["vocab"]
    history, request = [], []
    start = 0
    for b, n in enumerate(lens):
        ends = [n] if case["mode"] == "step" else range(n)
        history += [(start, start + prompt, start + prompt + e) for e in ends]
        request += [b] * len(ends)
        start += prompt + n
    rows = len(history)
    s["tokens"] = _tokens(g, start, vocab)
    s["history"] = _i32(history)
    rep = 1.0 + 0.3 * torch.rand(len(lens), generator=g, device="cuda")
    fre = 0.5 * torch.rand(len(lens), 2, generator=g, device="cuda")
    of = torch.tensor(request, device="cuda")
    s["penalties"] = torch.cat([rep[:, None], fre], 1)[of].contiguous()
    s["logits"] = _rows(g, rows, vocab, 2.5)
    s["bias_ids"] = s["bias_values"] = s["bias_rows"] = s["mask"] = s["mask_rows"] = None
    n = case["bias"]
    if n:
        s["bias_ids"] = torch.cat([torch.randperm(vocab, generator=g, device="cuda")[:n] for _ in lens]).to(torch.int32)
        s["bias_values"] = 4.0 * torch.randn(n * len(lens), generator=g, device="cuda")
        s["bias_rows"] = _i32([(n * b, n * (b + 1)) for b in request])
    m = case["masks"]
    if m:
        # grammars: one leaves a few tokens, the next most of them; the requests behind the last one have none
        words = (vocab + 31) // 32
        keep = torch.tensor([0.002 if i % 2 == 0 else 0.9 for i in range(m)], device="cuda")[:, None]
        bits = torch.rand((m, words * 32), generator=g, device="cuda") < keep
        value = (bits.view(m, words, 32).long() << torch.arange(32, device="cuda")).sum(2)
        s["mask"] = torch.where(value >= 1 << 31, value - (1 << 32), value).to(torch.int32)
        s["mask_rows"] = _i32([b if b < m else -1 for b in request])
    if case["kind"] == "logits_grad":
        s["dout"] = _rows(g, rows, vocab, 0.01)


def prepare(case, seed):
    kind = case["kind"]
    g = _generator(seed)
    s = {"case": dict(case)}
    if kind in ("norm", "norm_grad"):
        rows, hidden = case["rows"], case["hidden"]
        s["residual"] = _normal(g, (rows, hidden), 2.0)
        s["pre"] = _normal(g, (hidden,), 0.1, 1.0)
        s["x"] = _normal(g, (rows, hidden)) if case["block"] else None
        s["post"] = _normal(g, (hidden,), 0.1, 1.0) if case["post"] else None
        s["gate"] = None
        if case["gate"] != "none":
            s["gate"] = _normal(g, (hidden,) if case["gate"] == "shared" else (rows, hidden), 0.3, 0.5)
        if kind == "norm_grad":
            s["dy"] = _normal(g, (rows, hidden))
            s["dresidual"] = _normal(g, (rows, hidden))
    elif kind in ("embed", "embed_grad"):
        ids = _tokens(g, case["rows"], case["vocab"])
        pad = torch.rand(case["rows"], generator=g, device="cuda") < 0.02
        s["ids"] = torch.where(pad, torch.full_like(ids, -1), ids)
        if kind == "embed":
            s["table"] = _normal(g, (case["vocab"], case["hidden"]), 0.02)
        else:
            s["dout"] = _normal(g, (case["rows"], case["hidden"]), 0.01)
    elif kind in ("logits", "logits_grad"):
        _prepare_logits(case, g, s)
    else:
        s["logits"] = _rows(g, case["rows"], case["vocab"], 2.5)
        s["targets"] = _tokens(g, case["rows"], case["vocab"])
        s["dlogp"] = 0.01 * torch.randn(case["rows"], generator=g, device="cuda")
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _own(s):
    from paper_2609_35140_amd import uattn
    c, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        h, y = uattn.residual_norm(s["residual"], s["pre"], x=s["x"], post_weight=s["post"], gate=s["gate"], scale=c["scale"],
                                   eps=EPS)
        return {"residual": h, "y": y} if c["block"] else y
    if kind == "norm_grad":
        d = uattn.residual_norm_backward(s["dy"], s["dresidual"], s["residual"], s["pre"], x=s["x"], post_weight=s["post"],
                                         gate=s["gate"], scale=c["scale"], eps=EPS)
        return dict(zip(("dresidual", "dx", "dpre", "dpost", "dgate"), d))
    if kind == "embed":
        return uattn.embedding(s["ids"], s["table"], scale=c["scale"])
    if kind == "embed_grad":
        return uattn.embedding_backward(s["dout"], s["ids"], c["vocab"], scale=c["scale"],
                                        dtype=torch.float32 if c["fp32"] else torch.bfloat16)
    if kind == "logits":
        return uattn.logits_process(s["logits"], tokens=s["tokens"], history=s["history"], penalties=s["penalties"],
                                    bias_ids=s["bias_ids"], bias_values=s["bias_values"], bias_rows=s["bias_rows"],
                                    mask=s["mask"], mask_rows=s["mask_rows"])
    if kind == "logits_grad":
        return uattn.logits_process_backward(s["dout"], s["logits"], tokens=s["tokens"], history=s["history"],
                                             penalties=s["penalties"], mask=s["mask"], mask_rows=s["mask_rows"])
    return uattn.logprob_backward(s["logits"], s["targets"], s["dlogp"], inv_temperature=c["inv_temperature"])


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _rms(x):
    return 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)


def _plain_norm(s):
    h = s["residual"].float()
    if s["x"] is not None:
        u = s["x"].float()
        if s["post"] is not None:
            u = u * _rms(u) * s["post"].float()
        if s["gate"] is not None:
            u = u * s["gate"].float()
        h = h + s["case"]["scale"] * u
    y = (h * _rms(h) * s["pre"].float()).to(torch.bfloat16)
    return {"residual": h.to(torch.bfloat16), "y": y} if s["x"] is not None else y


def _plain_norm_grad(s):
    h, x, dy = s["residual"].float(), s["x"].float(), s["dy"].float()
    r = _rms(h)
    n = h * r
    a = dy * s["pre"].float()
    ds = s["dresidual"].float() + r * (a - n * (a * n).mean(-1, keepdim=True))
    gate = s["gate"].float() if s["gate"] is not None else None
    u, m, rx, post = x, None, None, None
    if s["post"] is not None:
        rx, post = _rms(x), s["post"].float()
        m = x * rx
        u = m * post
    b = s["case"]["scale"] * ds
    dgate = dpost = None
    if gate is not None:
        dgate = b * u
        dgate = dgate.to(torch.bfloat16) if s["gate"].dim() == 2 else dgate.sum(0)
        b = b * gate
    dx = b
    if m is not None:
        dpost = (b * m).sum(0)
        c = b * post
        dx = rx * (c - m * (c * m).mean(-1, keepdim=True))
    return {"dresidual": ds.to(torch.bfloat16), "dx": dx.to(torch.bfloat16), "dpre": (dy * n).sum(0), "dpost": dpost,
            "dgate": dgate}


def _plain_embed(s):
    ids = s["ids"].long()
    x = s["table"][ids.clamp(min=0)].float() * s["case"]["scale"]
    return (x * (ids >= 0)[:, None]).to(torch.bfloat16)


def _plain_embed_grad(s):
    c, ids = s["case"], s["ids"].long()
    x = s["dout"].float() * (ids >= 0)[:, None]
    d = torch.zeros((c["vocab"], c["hidden"]), device="cuda").index_add_(0, ids.clamp(min=0), x) * c["scale"]
    return d if c["fp32"] else d.to(torch.bfloat16)


def _count(s, first, last):
    """How often each row's tokens history[first] .. history[last] hold each vocabulary entry."""
    rows, vocab = s["logits"].shape
    begin, end = s["history"][:, first].long(), s["history"][:, last].long()
    n = end - begin
    row = torch.repeat_interleave(torch.arange(rows, device="cuda"), n)
    at = torch.arange(row.numel(), device="cuda") - (torch.cumsum(n, 0) - n)[row] + begin[row]
    count = torch.zeros(rows * vocab, device="cuda")
    return count.index_add_(0, row * vocab + s["tokens"][at].long(), torch.ones_like(row, dtype=torch.float32)).view(rows, vocab)


def _allowed(s):
    rows, vocab = s["logits"].shape
    m = s["mask"].long()
    bits = ((m[:, :, None] >> torch.arange(32, device="cuda")) & 1).view(m.shape[0], -1)[:, :vocab].bool()
    return bits[s["mask_rows"].long().clamp(min=0)] | (s["mask_rows"] < 0)[:, None]


def _plain_logits(s):
    x = s["logits"].float()
    rep, freq, pres = (s["penalties"][:, k:k + 1] for k in range(3))
    count = _count(s, 1, 2)
    seen = (_count(s, 0, 1) + count) > 0
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - freq * count
    x = torch.where(count > 0, x - pres, x)
    if s["bias_ids"] is not None:
        at = (s["bias_rows"][:, :1] + torch.arange(s["case"]["bias"], device="cuda")).long()
        x = x.scatter_add(1, s["bias_ids"][at].long(), s["bias_values"][at])
    if s["mask"] is not None:
        x = torch.where(_allowed(s), x, torch.full_like(x, -math.inf))
    return x.to(torch.bfloat16)


def _plain_logits_grad(s):
    d, rep = s["dout"].float(), s["penalties"][:, :1]
    seen = _count(s, 0, 2) > 0
    d = torch.where(seen, torch.where(s["logits"] > 0, d / rep, d * rep), d)
    if s["mask"] is not None:
        d = torch.where(_allowed(s), d, torch.zeros_like(d))
    return d.to(torch.bfloat16)


def _plain_logp_grad(s):
    it = s["case"]["inv_temperature"]
    x = s["logits"].float() * it
    y = s["targets"].long()[:, None]
    e = torch.exp(x - x.max(1, keepdim=True).values)
    at = e.gather(1, y)
    # 1 - p of the target from the others' sum: where p is near 1, their difference would leave no digits
    others = e.scatter(1, y, 0.0).sum(1, keepdim=True)
    g = s["dlogp"][:, None] * it
    return (-g * (e / (others + at))).scatter(1, y, g * (others / (others + at))).to(torch.bfloat16)


_PLAIN = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "embed": _plain_embed, "embed_grad": _plain_embed_grad,
          "logits": _plain_logits, "logits_grad": _plain_logits_grad, "logp_grad": _plain_logp_grad}


def run(state):
    if own:
        return _own(state)
    return _PLAIN[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# minimal work, and the outputs in 64 bits
# ---------------------------------------------------------------------------
def _distinct(rows, vocab):
    """How many vocabulary entries `rows` tokens of _tokens() have, on average."""
    p = torch.log1p(1.0 / torch.arange(1, vocab, dtype=torch.float64)) / math.log(vocab)
    return int(-torch.expm1(rows * torch.log1p(-p)).sum())


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n, h = case["rows"] * case["hidden"], case["hidden"]
        w = 2 * h * (1 + case["post"] + (case["gate"] == "shared"))
        if kind == "norm":
            return {"bytes": 2 * n * ((4 if case["block"] else 2) + (case["gate"] == "token")) + w,
                    "flops": n * (5 + (3 if case["block"] else 0) + 5 * case["post"])}
        # the block's output counts where its norm or gate is to be differentiated
        rows = 5 + (case["post"] or case["gate"] != "none") + 2 * (case["gate"] == "token")
        return {"bytes": 2 * n * rows + 3 * w, "flops": n * (16 + 14 * case["post"])}
    if kind == "embed":
        n = case["rows"] * case["hidden"]
        return {"bytes": 2 * n + 2 * _distinct(case["rows"], case["vocab"]) * case["hidden"] + 4 * case["rows"], "flops": n}
    if kind == "embed_grad":
        n, size = case["rows"] * case["hidden"], 4 if case["fp32"] else 2
        return {"bytes": 2 * n + size * case["vocab"] * case["hidden"] + 4 * case["rows"], "flops": 2 * n}
    if kind in ("logits", "logits_grad"):
        rows, vocab, lens = _num_rows(case), case["vocab"], _lens(case)
        small = 4 * (sum(lens) + case["prompt"] * len(lens)) + 24 * rows + 8 * case["bias"] * len(lens)
        return {"bytes": 4 * rows * vocab + small + 4 * case["masks"] * ((vocab + 31) // 32), "flops": rows * vocab}
    n = case["rows"] * case["vocab"]
    return {"bytes": 4 * n + 8 * case["rows"], "flops": 6 * n}


def _exact_norm(s, case):
    """The residual sum and its norm; with gradients by automatic differentiation of the sum and norm at the given residual."""
    with_grad = case["kind"] == "norm_grad"
    leaf = {k: s[k].double().requires_grad_(with_grad) for k in ("residual", "pre", "x", "post", "gate") if s[k] is not None}
    rms = lambda v: v / torch.sqrt((v ** 2).sum(-1, keepdim=True) / v.shape[-1] + EPS)  # noqa: E731
    branch = None
    if "x" in leaf:
        branch = rms(leaf["x"]) * leaf["post"] if "post" in leaf else leaf["x"]
        branch = case["scale"] * (branch * leaf["gate"] if "gate" in leaf else branch)
    if not with_grad:
        h = leaf["residual"] + branch if branch is not None else leaf["residual"]
        return {"residual": h, "y": rms(h) * leaf["pre"]} if branch is not None else rms(h) * leaf["pre"]
    y = rms(leaf["residual"]) * leaf["pre"]
    back = lambda out, grad, to: torch.autograd.grad(out, to, grad)  # noqa: E731
    dh, dpre = back(y, s["dy"].double(), [leaf["residual"], leaf["pre"]])
    dh = dh + s["dresidual"].double()
    names = [k for k in ("x", "post", "gate") if k in leaf]
    d = dict(zip(names, back(branch, dh, [leaf[k] for k in names])))
    return {"dresidual": dh, "dx": d["x"], "dpre": dpre, "dpost": d.get("post"), "dgate": d.get("gate")}


def _exact_logits(s, case):
    z, tokens, rows = s["logits"], s["tokens"].long(), s["history"].tolist()
    vocab = z.shape[1]
    grad = case["kind"] == "logits_grad"
    out = torch.empty(z.shape, dtype=torch.float64, device="cuda")
    words = s["mask"].cpu().numpy().view("uint8") if s["mask"] is not None else None
    masks = []
    if words is not None:
        import numpy as np
        bits = np.unpackbits(words.reshape(s["mask"].shape[0], -1), axis=1, bitorder="little")[:, :vocab]
        masks = [torch.from_numpy(b.astype(bool)).cuda() for b in bits]
    which = s["mask_rows"].tolist() if masks else [-1] * len(rows)
    bias = s["bias_rows"].tolist() if s["bias_rows"] is not None else None
    pen = s["penalties"].double().tolist()
    for t, (begin, split, end) in enumerate(rows):
        r, f, p = pen[t]
        v = (s["dout"] if grad else z)[t].double()
        said = torch.unique(tokens[begin:end])
        up = z[t].double()[said] > 0
        v[said] = torch.where(up, v[said] / r, v[said] * r)
        if not grad:
            v.index_add_(0, tokens[split:end], torch.full((end - split,), -f, dtype=torch.float64, device="cuda"))
            v[torch.unique(tokens[split:end])] -= p
            if bias:
                lo, hi = bias[t]
                v[s["bias_ids"][lo:hi].long()] += s["bias_values"][lo:hi].double()
        if which[t] >= 0:
            v[~masks[which[t]]] = 0.0 if grad else -math.inf
        out[t] = v
    return out


def _exact_logp_grad(s, case):
    x = s["logits"].double() * case["inv_temperature"]
    g = s["dlogp"].double() * case["inv_temperature"]
    p = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
    p[torch.arange(x.shape[0], device="cuda"), s["targets"].long()] -= 1.0
    return p.mul_(-g[:, None])


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        return _exact_norm(s, case)
    if kind in ("logits", "logits_grad"):
        return _exact_logits(s, case)
    if kind == "logp_grad":
        return _exact_logp_grad(s, case)
    ids = s["ids"].long()
    keep = ids >= 0
    if kind == "embed":
        out = torch.zeros((case["rows"], case["hidden"]), dtype=torch.float64, device="cuda")
        out[keep] = s["table"].double()[ids[keep]] * case["scale"]
        return out
    out = torch.zeros((case["vocab"], case["hidden"]), dtype=torch.float64, device="cuda")
    return out.index_add_(0, ids[keep], s["dout"][keep].double()).mul_(case["scale"])
