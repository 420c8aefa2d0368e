"""Attention over whole prompts, its gradient, and the rotation by positions of
several axes, as cases to time.

Keys of a case: ``op`` (attn, grad, rotary), ``dtype`` (f32, bf16, f16), ``h_q`` /
``h_kv`` query / KV heads, ``d`` head size.

attn and grad: ``B`` sequences of ``t_lo`` to ``t_hi`` rows each, packed one after
the other; their keys are the rows' own (``n_hi`` 0) or ``n_lo`` to ``n_hi`` others;
``causal``: row r of a sequence of t rows and n keys sees keys 0 .. r + n - t, else
all.  ``lse``: the logarithm of the sum of each row's exponentials is a result too
(what a training program keeps for the gradient).  q, k and v of the rows' own
keys are views into one projection's output, and so are their gradients.

rotary: ``rows`` tokens, ``axes`` positions each (all the same in text; time, height
and width in images and video), ``rot`` rotated dimensions, ``interleaved`` pairs
(2i, 2i+1) or else (i, i + rot/2), ``limit`` positions of the table of angles;
``inverse``: turned back, which is the gradient.
"""
import math
import random

import torch

own = False                     # whether run() calls the framework's kernels

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _attn(name, op, dtype, B, h_q, h_kv, d, t_lo, t_hi, n_lo=0, n_hi=0, causal=True, lse=False):
    c = dict(op=op, dtype=dtype, B=B, h_q=h_q, h_kv=h_kv, d=d, t_lo=t_lo, t_hi=t_hi, n_lo=n_lo,
             n_hi=n_hi, causal=causal, lse=lse)
    return dict(c, name=name) if name else c


def _rotary(name, dtype, rows, h_q, h_kv, d, rot, axes, limit, interleaved=False, inverse=False):
    c = dict(op="rotary", dtype=dtype, rows=rows, h_q=h_q, h_kv=h_kv, d=d, rot=rot, axes=axes,
             limit=limit, interleaved=interleaved, inverse=inverse)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token over the states of a prompt: launches and latency.
        _attn("attn_bf16_b1_t1", "attn", "bf16", 1, 32, 8, 128, 1, 1, 700, 700),
        # A serving batch of prompts of odd lengths, from one token on.
        _attn("attn_f16_b16_prompts", "attn", "f16", 16, 32, 8, 128, 1, 900),
        # One long prompt.
        _attn("attn_bf16_b1_t16384", "attn", "bf16", 1, 32, 8, 128, 16384, 16384),
        # A text decoder's rows over an encoder's states of other lengths.
        _attn("cross_bf16_b8_t333", "attn", "bf16", 8, 16, 16, 64, 333, 333, 400, 1500, False),
        # The framework's own type, an odd length, with what training keeps.
        _attn("attn_f32_b2_t1500", "attn", "f32", 2, 16, 16, 64, 1500, 1500, lse=True),
        # The gradient of a training batch of whole sequences.
        _attn("grad_bf16_b4_t2048", "grad", "bf16", 4, 32, 8, 128, 2048, 2048),
        # Documents of odd lengths, packed: wide groups.
        _attn("grad_f16_b24_packed", "grad", "f16", 24, 64, 8, 128, 5, 1100),
        # A fine-tuning step on one short text: few rows, launches.
        _attn("grad_bf16_b1_t120", "grad", "bf16", 1, 16, 16, 64, 120, 120),
        # Long training sequences.
        _attn("grad_bf16_b1_t8192", "grad", "bf16", 1, 32, 8, 128, 8192, 8192),
        # A decode step's rows of 16 users.
        _rotary("rotary_bf16_step", "bf16", 16, 32, 8, 128, 128, 3, 32768),
        # A prompt of text, images and video.
        _rotary("rotary_bf16_video", "bf16", 16001, 32, 8, 128, 128, 3, 32768),
        # The gradient of half-rotated heads in pairs, two axes.
        _rotary("rotary_f16_back", "f16", 5003, 16, 16, 64, 32, 2, 8192, True, True),
    ]


# What a drawn case may cost: below the largest listed ones.
_MAX_FLOPS = 2100e9
_MAX_PAIRS = 1 << 31            # scores of all heads of one sequence, seen or not
_MAX_ROWS = 320 << 20           # bytes of q and k rows of a rotation


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["attn", "attn", "grad", "grad", "rotary"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        h_kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
        h_q = h_kv * rng.choice([1, 1, 2, 4, 4, 5, 8, 16])
        if h_q > 128:
            continue
        d = rng.choice([64, 128, 128, 128, 256])
        size = 4 if dtype == "f32" else 2
        if op == "rotary":
            rot = rng.choice([d, d, d // 2])
            c = _rotary("", dtype, _log(rng, 1, 40000), h_q, h_kv, d, rot, rng.choice([1, 2, 3, 3]),
                        rng.choice([4096, 32768, 131072]), rng.random() < 0.3, rng.random() < 0.4)
            if c["rows"] * (h_q + h_kv) * d * size <= _MAX_ROWS:
                return c
            continue
        B = _log(rng, 1, 64)
        t_hi = _log(rng, 1, 12000)
        t_lo = t_hi if rng.random() < 0.4 else rng.randint(1, t_hi)
        kind = rng.random()         # own keys; a prompt's end over all of it; other states
        causal = True
        n_lo = n_hi = 0
        if kind > 0.7:
            causal = kind < 0.85
            n_lo = t_hi if causal else 1
            n_hi = n_lo + _log(rng, 1, 8000)
        c = _attn("", op, dtype, B, h_q, h_kv, d, t_lo, t_hi, n_lo, n_hi, causal,
                  op == "attn" and rng.random() < 0.5)
        counts = _counts(c)
        if max(h_q * t * n for t, n in counts) > _MAX_PAIRS:
            continue
        # (every sequence is some calls of the plain form)
        if work(c)["flops"] > _MAX_FLOPS * (0.1 if dtype == "f32" else 1):
            continue
        return c


def _counts(c):
    """(rows, keys) of each sequence: part of the case, the same for every seed."""
    r = random.Random(c["B"] * 1000003 + c["t_lo"] * 101 + c["t_hi"] * 7 + c["n_hi"])
    out = []
    for _ in range(c["B"]):
        t = r.randint(c["t_lo"], c["t_hi"])
        out.append((t, r.randint(c["n_lo"], c["n_hi"]) if c["n_hi"] else t))
    return out


def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rotary":
        moved = 2 * c["rows"] * (c["h_q"] + c["h_kv"]) * c["d"] * size + 4 * c["rows"] * c["axes"]
        return {"bytes": moved, "flops": 3 * c["rows"] * (c["h_q"] + c["h_kv"]) * c["rot"]}
    counts = _counts(c)
    rows, keys = sum(t for t, _ in counts), sum(n for _, n in counts)
    if c["causal"]:
        pairs = sum(t * (n - t) + t * (t + 1) // 2 for t, n in counts)
    else:
        pairs = sum(t * n for t, n in counts)
    q, k = rows * c["h_q"] * c["d"] * size, keys * c["h_kv"] * c["d"] * size
    if c["op"] == "attn":
        return {"bytes": 2 * q + 2 * k + (4 * rows * c["h_q"] if c["lse"] else 0),
                "flops": 4 * c["d"] * c["h_q"] * pairs}
    # q, out, dout read and dq written; k, v read, dk, dv written; lse read
    return {"bytes": 4 * q + 4 * k + 4 * rows * c["h_q"], "flops": 10 * c["d"] * c["h_q"] * pairs}


# --- inputs -------------------------------------------------------------------------------

def _positions(c, g):
    """[axes][rows] as a prompt has them: runs of text, whose axes go on together,
    and images and videos, whose axes count frames, lines and columns from where
    the text stopped.  A few rows alone are users' next tokens."""
    r = random.Random(int(torch.randint(1 << 30, (1,), generator=g, device="cuda")))
    n, axes, limit = c["rows"], c["axes"], c["limit"]
    if n <= 64:
        at = torch.tensor([r.randrange(limit) for _ in range(n)], dtype=torch.int32)
        return at.expand(axes, n).contiguous().cuda()
    parts, have, at = [], 0, 0
    while have < n:
        if r.random() < 0.5:
            m = r.randint(1, 400)
            part = torch.arange(m).expand(axes, m)
        else:
            frames, high, wide = r.choice([1, 1, 2, 5]), r.randint(4, 40), r.randint(4, 40)
            grid = torch.meshgrid(torch.arange(frames), torch.arange(high), torch.arange(wide),
                                  indexing="ij")
            part = torch.stack([x.flatten() for x in grid])[-axes:]
        if at + int(part.max()) >= limit:
            at = 0                  # the next sequence
        parts.append(part + at)
        have += part.shape[1]
        at += int(part.max()) + 1
    return torch.cat(parts, 1)[:, :n].to(torch.int32).contiguous().cuda()


def _sections(c):
    """Pairs of each axis: the later ones have the larger shares, as where time has
    16 of 64 pairs, height and width 24 each."""
    half, axes = c["rot"] // 2, c["axes"]
    first = half // 4 if axes == 3 else half // axes
    rest = half - first
    return {1: [half], 2: [first, rest], 3: [first, rest // 2, rest - rest // 2]}[axes]


def _start(counts):
    return torch.tensor([0] + counts, device="cuda").cumsum(0).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _TYPES[c["dtype"]]
    h_q, h_kv, d = c["h_q"], c["h_kv"], c["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = {"case": c}
    if c["op"] == "rotary":
        qk = normal(c["rows"], h_q + h_kv, d).to(dtype)
        s["q"], s["k"] = qk[:, :h_q], qk[:, h_q:]
        s["positions"], s["sections"] = _positions(c, g), _sections(c)
        half = c["rot"] // 2
        i = torch.arange(half, device="cuda", dtype=torch.float64)
        a = torch.arange(c["limit"], device="cuda", dtype=torch.float64)[:, None] \
            * 10000.0 ** (-i / half)
        s["table"] = torch.cat((a.cos(), a.sin()), 1).float()
        s["q_out"] = torch.empty(s["q"].shape, dtype=dtype, device="cuda")
        s["k_out"] = torch.empty(s["k"].shape, dtype=dtype, device="cuda")
        return s

    counts = _counts(c)
    rows, keys = sum(t for t, _ in counts), sum(n for _, n in counts)
    s["scale"] = 1.0 / math.sqrt(d)
    s["T"], s["N"] = c["t_hi"], max(c["n_hi"], c["t_hi"])
    s["row_start"] = _start([t for t, _ in counts])
    s["key_start"] = _start([n for _, n in counts])
    if c["n_hi"]:
        # (scores of some width: q is twice a unit normal's)
        s["q"] = (2 * normal(rows, h_q, d)).to(dtype)
        kv = normal(keys, 2 * h_kv, d).to(dtype)
        s["k"], s["v"] = kv[:, :h_kv], kv[:, h_kv:]
    else:
        qkv = normal(rows, h_q + 2 * h_kv, d)
        qkv[:, :h_q] *= 2
        qkv = qkv.to(dtype)
        s["q"], s["k"], s["v"] = qkv.split((h_q, h_kv, h_kv), 1)
    s["out"] = torch.empty(rows, h_q, d, dtype=dtype, device="cuda")
    s["lse"] = None
    if c["lse"] or c["op"] == "grad":
        s["lse"] = torch.empty(rows, h_q, dtype=torch.float32, device="cuda")
    if c["op"] == "grad":
        _plain_attn(s)              # out and lse, as the forward pass leaves them
        s["d_out"] = normal(rows, h_q, d).to(dtype)
        if c["n_hi"]:
            s["dq"] = torch.empty(rows, h_q, d, dtype=dtype, device="cuda")
            dkv = torch.empty(keys, 2 * h_kv, d, dtype=dtype, device="cuda")
            s["dk"], s["dv"] = dkv[:, :h_kv], dkv[:, h_kv:]
        else:
            dqkv = torch.empty(rows, h_q + 2 * h_kv, d, dtype=dtype, device="cuda")
            s["dq"], s["dk"], s["dv"] = dqkv.split((h_q, h_kv, h_kv), 1)
    if own:
        from paper_2607_19456_amd import binding
        s["workspace"] = binding.prompt_workspace(
            s["q"], s["k"], row_start=s["row_start"], T=s["T"], key_start=s["key_start"],
            N=s["N"], grad=c["op"] == "grad")
    return s


# --- the plain form -----------------------------------------------------------------------

def _sequences(s):
    """Slices of each sequence's rows and keys."""
    t0 = n0 = 0
    for t, n in _counts(s["case"]):
        yield slice(t0, t0 + t), slice(n0, n0 + n)
        t0, n0 = t0 + t, n0 + n


def _scores(c, q, k, scale):
    """[h_kv][t*G][n] in float32, -infinity where the key is not seen."""
    t, n, h = q.shape[0], k.shape[0], c["h_kv"]
    G = c["h_q"] // h
    a = q.float().reshape(t, h, G, -1).transpose(0, 1).reshape(h, t * G, -1)
    x = (a @ k.float().permute(1, 2, 0)).mul_(scale)
    if c["causal"]:
        r = torch.arange(t, device="cuda").repeat_interleave(G)
        hidden = torch.arange(n, device="cuda") > (r + n - t)[:, None]
        x.masked_fill_(hidden, -math.inf)
    return a, x


def _by_head(c, x):
    """[t][h_q][..] as [h_kv][t*G][..] in float32."""
    t, h = x.shape[0], c["h_kv"]
    return x.float().reshape(t, h, c["h_q"] // h, -1).transpose(0, 1).reshape(
        h, t * (c["h_q"] // h), -1)


def _by_row(c, x):
    """and back, [t][h_q][..]."""
    h, G = c["h_kv"], c["h_q"] // c["h_kv"]
    return x.reshape(h, -1, G, x.shape[-1]).transpose(0, 1).flatten(1, 2)


def _plain_attn(s):
    c = s["case"]
    for rows, keys in _sequences(s):
        _, x = _scores(c, s["q"][rows], s["k"][keys], s["scale"])
        top = x.amax(-1, keepdim=True)
        top = torch.where(top > -math.inf, top, 0.0)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        o = (p @ s["v"][keys].float().transpose(0, 1)) / torch.where(total > 0, total, 1.0)
        s["out"][rows] = _by_row(c, o).to(s["out"].dtype)
        if s["lse"] is not None:
            s["lse"][rows] = _by_row(c, top + total.log()).squeeze(-1)
    return (s["out"], s["lse"]) if c["lse"] else (s["out"],)


def _plain_grad(s):
    c = s["case"]
    for rows, keys in _sequences(s):
        a, x = _scores(c, s["q"][rows], s["k"][keys], s["scale"])
        top = x.amax(-1, keepdim=True)
        p = x.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(torch.where(total > 0, total, 1.0))
        g = _by_head(c, s["d_out"][rows])
        k, v = (s[y][keys].float().transpose(0, 1) for y in ("k", "v"))
        s["dv"][keys] = (p.transpose(1, 2) @ g).transpose(0, 1).to(s["dv"].dtype)
        dp = g @ v.transpose(1, 2)
        delta = (p * dp).sum(-1, keepdim=True)
        ds = dp.sub_(delta).mul_(p).mul_(s["scale"])
        s["dq"][rows] = _by_row(c, ds @ k).to(s["dq"].dtype)
        s["dk"][keys] = (ds.transpose(1, 2) @ a).transpose(0, 1).to(s["dk"].dtype)
    return s["dq"], s["dk"], s["dv"]


def _plain_rotary(s):
    c = s["case"]
    half = c["rot"] // 2
    pair = torch.arange(half, device="cuda")
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"),
                                   torch.tensor(s["sections"], device="cuda"), output_size=half)
    at = s["positions"].long()[axis].t()                # [row][pair]
    cos = s["table"][at, pair][:, None]
    sin = s["table"][at, half + pair][:, None]
    if c["inverse"]:
        sin = -sin
    for x, y in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
        x = x.float()
        if c["interleaved"]:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        y.copy_(torch.cat((turned, x[..., 2 * half:]), -1))
    return s["q_out"], s["k_out"]


def run(state):
    s = state
    op = s["case"]["op"]
    if not own:
        return {"attn": _plain_attn, "grad": _plain_grad, "rotary": _plain_rotary}[op](s)
    from paper_2607_19456_amd import binding
    c = s["case"]
    if op == "rotary":
        return binding.rotary_axes(s["q"], s["positions"], s["table"], s["sections"], k=s["k"],
                                   interleaved=c["interleaved"], inverse=c["inverse"],
                                   q_out=s["q_out"], k_out=s["k_out"])
    packed = dict(causal=c["causal"], row_start=s["row_start"], T=s["T"],
                  key_start=s["key_start"], N=s["N"], workspace=s["workspace"])
    if op == "attn":
        binding.prompt_attn(s["q"], s["k"], s["v"], s["scale"], out=s["out"], lse=s["lse"],
                            **packed)
        return (s["out"], s["lse"]) if c["lse"] else (s["out"],)
    return binding.prompt_attn_grad(s["q"], s["k"], s["v"], s["out"], s["lse"], s["d_out"],
                                    s["scale"], dq=s["dq"], dk=s["dk"], dv=s["dv"], **packed)


# --- the definition, in 64 bits -----------------------------------------------------------

def exact(case, seed):
    c = case
    if c["op"] == "rotary":
        return _exact_rotary(c, prepare(dict(c), seed))
    counts = _counts(c)
    if sum(t * n for t, n in counts) * c["h_q"] * c["d"] > 3e12:
        return None
    s = prepare(dict(c), seed)
    G, grad = c["h_q"] // c["h_kv"], c["op"] == "grad"

    def zeros(like):
        return torch.zeros(like.shape, dtype=torch.float64, device="cuda")

    out, lse = zeros(s["q"]), zeros(s["q"][..., 0])
    dq, dk, dv = zeros(s["q"]), zeros(s["k"]), zeros(s["v"])
    first = key0 = 0
    for t, n in counts:
        key = torch.arange(n, device="cuda")
        step = max(1, (1 << 26) // n)
        for head in range(c["h_q"]):
            k = s["k"][key0:key0 + n, head // G].double()
            v = s["v"][key0:key0 + n, head // G].double()
            for r0 in range(0, t, step):
                r = torch.arange(r0, min(t, r0 + step), device="cuda")
                at = slice(first + r0, first + r0 + len(r))
                q = s["q"][at, head].double()
                score = torch.mm(q, k.t()) * s["scale"]
                if c["causal"]:
                    score[key[None, :] - r[:, None] > n - t] = -math.inf
                p = torch.softmax(score, 1)
                if not grad:
                    out[at, head] = torch.mm(p, v)
                    lse[at, head] = torch.logsumexp(score, 1)
                    continue
                g = s["d_out"][at, head].double()
                dp = torch.mm(g, v.t())
                ds = p * (dp - torch.mm(p, v).mul(g).sum(1, keepdim=True)) * s["scale"]
                dq[at, head] = torch.mm(ds, k)
                dk[key0:key0 + n, head // G] += torch.mm(ds.t(), q)
                dv[key0:key0 + n, head // G] += torch.mm(p.t(), g)
        first, key0 = first + t, key0 + n
    if grad:
        return dq, dk, dv
    return (out, lse) if c["lse"] else (out,)


def _exact_rotary(c, s):
    """Each pair as a complex number, times the unit number of its angle."""
    half, out = c["rot"] // 2, []
    table, first = s["table"].double(), [sum(s["sections"][:a]) for a in range(c["axes"])]
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        for i in range(half):
            axis = max(a for a in range(c["axes"]) if first[a] <= i)
            pos = s["positions"][axis].long()
            unit = torch.complex(table[pos, i], table[pos, half + i])
            a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
            z = torch.complex(y[..., a], y[..., b]) * (unit.conj() if c["inverse"] else unit)[:, None]
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    return tuple(out)
