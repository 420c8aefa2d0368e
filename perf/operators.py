"""The paged KV cache's operators, as cases to time: rows appended with the
position rotation on the way, and attention over the pages, with the cache in
32 or 16 bits ("dense") or in 4 bits ("mx4").

Keys of a case: ``op`` (append, attn), ``fmt`` (dense, mx4), ``dtype`` of the
rows (f32, bf16, f16; a dense cache has the same type), ``B`` sequences,
``h_q`` / ``h_kv`` query / KV heads, ``d`` head size, ``page`` rows of a page,
``lo`` / ``hi`` bounds of the rows that a sequence has before the step,
``T`` rows that it submits (``ragged``: at most T, each sequence its own
number), ``causal``, and for append ``rot`` rotated dimensions and
``interleaved``.  An append to a 4-bit cache is followed by the reading back of
its rows, which shows what the cache holds.

The 4-bit form: blocks of 32 values v share 2^X, X = floor(log2 max|v|) - 2,
held as the byte X + 127; a value is held as the nearest of 0, .5, 1, 1.5, 2, 3,
4, 6 times 2^X, ties to the even code, and a sign.  A page of one head is one
run of bytes.  Keys: the rows' codes (two to a byte, the lower one first), then
the rows' scale bytes.  Values: in groups of 8 rows, eight dimensions of each
row in turn (4 bytes a row), then the scale bytes, a block's eight rows in turn.
"""
import math
import random

import torch

own = False                     # whether run() calls the framework's kernels

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _attn(name, fmt, dtype, B, h_q, h_kv, d, page, lo, hi, T=1, ragged=False, causal=True):
    c = dict(op="attn", fmt=fmt, dtype=dtype, B=B, h_q=h_q, h_kv=h_kv, d=d, page=page, lo=lo,
             hi=hi, T=T, ragged=ragged, causal=causal)
    return dict(c, name=name) if name else c


def _append(name, fmt, dtype, B, h_q, h_kv, d, page, lo, hi, T, rot, ragged=False,
            interleaved=False):
    c = dict(op="append", fmt=fmt, dtype=dtype, B=B, h_q=h_q, h_kv=h_kv, d=d, page=page, lo=lo,
             hi=hi, T=T, ragged=ragged, rot=rot, interleaved=interleaved)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user's decode step on a short context: launches and latency.
        _attn("attn_bf16_b1_n700", "dense", "bf16", 1, 32, 8, 128, 16, 700, 700),
        # A serving batch of ordinary, ragged lengths.
        _attn("attn_f16_b16_ragged", "dense", "f16", 16, 32, 8, 128, 16, 200, 4000),
        # The GQA workload in the framework's own type, from pages.
        _attn("attn_f32_b16_n8192", "dense", "f32", 16, 32, 8, 128, 64, 8191, 8191),
        # The long-context workload: ragged contexts of 65536 to 131008 rows.
        _attn("attn_bf16_b4_long", "dense", "bf16", 4, 64, 8, 128, 256, 65536, 131007),
        # Chunks of prompts of odd sizes, batched behind what is cached already.
        _attn("attn_bf16_b4_chunks", "dense", "bf16", 4, 32, 8, 128, 64, 0, 6000, 2048, True),
        # A text decoder's rows over an encoder's states of other lengths.
        _attn("cross_f16_b8_t37", "dense", "f16", 8, 16, 16, 64, 32, 300, 1500, 37, False, False),
        # The long-context workload from a cache a quarter as large.
        _attn("attn_mx4_b4_long", "mx4", "bf16", 4, 64, 8, 128, 256, 65536, 131007),
        # Four draft tokens of each of 16 users, verified in one step.
        _attn("attn_mx4_b16_spec4", "mx4", "f16", 16, 64, 8, 128, 64, 2000, 16000, 4),
        # A decode step's rows of 64 users.
        _append("append_bf16_b64_step", "dense", "bf16", 64, 64, 8, 128, 16, 100, 4000, 1, 128),
        # Prompts of odd lengths; half of each head is rotated, in pairs.
        _append("append_f16_prompts", "dense", "f16", 4, 32, 8, 128, 64, 0, 500, 3000, 64, True,
                True),
        # A decode step's rows of 16 users into 4 bits.
        _append("append_mx4_b16_step", "mx4", "bf16", 16, 32, 8, 128, 16, 100, 4000, 1, 128),
        # A prompt's rows into 4 bits.
        _append("append_mx4_prompts", "mx4", "bf16", 8, 32, 8, 128, 64, 0, 7000, 700, 128),
    ]


# What a drawn case may cost: below the largest listed ones.
_MAX_CACHE = 1200 << 20             # bytes of K and V that a call reads
_MAX_VALUES = 1 << 30               # values of K and V as the sequences' longest one pads them
_MAX_FLOPS = 200e9
_MAX_PAIRS = 1 << 31                # scores, as the longest sequence pads them
_MAX_ROWS = 256 << 20               # bytes of q, K and V rows


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["attn", "attn", "append"])
        fmt = rng.choice(["dense", "mx4"])
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        h_kv = rng.choice([1, 2, 4, 8, 8, 16, 32])
        h_q = h_kv * rng.choice([1, 2, 4, 4, 5, 8, 8, 16, 32])
        if h_q > 128:
            continue
        d = rng.choice([64, 128, 128, 128, 256])
        page = rng.choice([16, 16, 32, 64, 128, 256])
        B = _log(rng, 1, 256)
        hi = _log(rng, 1, 131000)
        lo = hi if rng.random() < 0.25 else rng.randint(0, hi)
        kind = rng.random()         # tokens, drafts of a few, chunks of prompts
        T = 1 if kind < 0.5 else rng.randint(2, 9) if kind < 0.75 else _log(rng, 16, 2048)
        ragged = T > 1 and rng.random() < 0.5
        if op == "attn":
            causal = rng.random() < 0.8
            c = _attn("", fmt, dtype, B, h_q, h_kv, d, page, lo if causal else max(1, lo), hi, T,
                      ragged, causal)
        else:
            rot = rng.choice([d, d, d, d // 2, 0])
            c = _append("", fmt, dtype, B, h_q, h_kv, d, page, lo, hi, T, rot, ragged,
                        rng.random() < 0.3)
        values = 2 * B * h_kv * d * (hi + T + page)
        rows = 4 * B * T * (h_q + 2 * h_kv) * d
        w = work(c)
        if values > _MAX_VALUES or rows > _MAX_ROWS or w["bytes"] > _MAX_CACHE:
            continue
        if w["flops"] > _MAX_FLOPS * (0.1 if dtype == "f32" else 1):
            continue
        if op == "attn" and B * h_q * T * (hi + T + page) > _MAX_PAIRS:
            continue
        return c


def _counts(c):
    """(rows before the step, rows that it submits) of each sequence: part of
    the case, the same for every seed."""
    r = random.Random(c["B"] * 1000003 + c["lo"] * 101 + c["hi"] * 7 + c["T"])
    return [(r.randint(c["lo"], c["hi"]), r.randint(1, c["T"]) if c["ragged"] else c["T"])
            for _ in range(c["B"])]


def _row_bytes(c):
    size = 4 if c["dtype"] == "f32" else 2
    return c["d"] * size if c["fmt"] == "dense" else c["d"] // 2 + c["d"] // 32


def work(case):
    c = case
    counts = _counts(c)
    size = 4 if c["dtype"] == "f32" else 2
    new = sum(n for _, n in counts)
    if c["op"] == "append":
        half = c["rot"] // 2
        # q read and written, K and V read, and written or (mx4) read back
        moved = new * ((2 * c["h_q"] + 4 * c["h_kv"]) * c["d"] * size + 8 * half)
        if c["fmt"] == "mx4":       # in between the rows are written and read in 4 bits
            moved += new * c["h_kv"] * 4 * _row_bytes(c)
        return {"bytes": moved, "flops": 6 * new * (c["h_q"] + c["h_kv"]) * half}
    if c["causal"]:
        keys = sum(p + n for p, n in counts)
        pairs = sum(n * p + n * (n + 1) // 2 for p, n in counts)
    else:
        keys = sum(p for p, _ in counts)
        pairs = sum(n * p for p, n in counts)
    return {"bytes": keys * c["h_kv"] * 2 * _row_bytes(c) + 2 * new * c["h_q"] * c["d"] * size,
            "flops": 4 * c["d"] * c["h_q"] * pairs}


# --- the 4-bit form -----------------------------------------------------------------------

_LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(byte):
    """2^(byte - 127) in float32, for bytes of 1 to 254."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """Codes (uint8, 0..15) and scale bytes of the last axis, in blocks of 32."""
    x = x.unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    X = torch.where(top > 0, torch.frexp(top).exponent - 3, -126).clamp(min=-126)
    y = x.abs() / _power(X + 127)[..., None]
    code = (y > 0.25).to(torch.uint8)
    for at in (1.25, 2.5, 5.0):
        code += y > at
    for at in (0.75, 1.75, 3.5):    # half way to an even code
        code += y >= at
    code += 8 * torch.signbit(x)
    return code.flatten(-2), (X + 127).to(torch.uint8)


def _planes(c, K, V):
    """The codes and scale bytes of K and V, as views: keys [page][head][row][byte]
    twice, values [page][head][group][eight dims][row][byte] and
    [page][head][group][block][row]."""
    d, P = c["d"], c["page"]
    at = P * (d // 2)
    k, v = K.flatten(2), V.flatten(2)
    return (k[:, :, :at].unflatten(2, (P, d // 2)), k[:, :, at:].unflatten(2, (P, d // 32)),
            v[:, :, :at].unflatten(2, (P // 8, d // 8, 8, 4)),
            v[:, :, at:].unflatten(2, (P // 8, d // 32, 8)))


def _put_mx4(c, K, V, page, slot, k, v):
    """Rows k, v [n][head][d] into row `slot` of page `page`."""
    kc, ks, vc, vs = _planes(c, K, V)
    codes, scales = _quantise(k)
    kc[page, :, slot] = codes[..., 0::2] | codes[..., 1::2] << 4
    ks[page, :, slot] = scales
    codes, scales = _quantise(v)
    vc[page, :, slot // 8, :, slot % 8] = (codes[..., 0::2] | codes[..., 1::2] << 4
                                           ).unflatten(-1, (-1, 4))
    vs[page, :, slot // 8, :, slot % 8] = scales


def _values(codes, scales):
    """float32 values of bytes [...][d/2] and scale bytes [...][d/32]."""
    level = torch.tensor(_LEVELS + tuple(-x for x in _LEVELS), device=codes.device)
    byte = torch.arange(256, device=codes.device)
    pair = torch.stack((level[byte & 15], level[byte >> 4]), 1)
    x = pair[codes.to(torch.int32)].flatten(-2)
    return (x.unflatten(-1, (-1, 32)) * _power(scales)[..., None]).flatten(-2)


def _dense_pages(c, K, V, pages):
    """float32 rows [..][head][row][d] of pages."""
    if c["fmt"] == "dense":
        return K[pages].float(), V[pages].float()
    kc, ks, vc, vs = _planes(c, K, V)
    k = _values(kc[pages], ks[pages])
    # [..][head][group][eight dims][row][byte] -> [..][head][group][row][bytes]
    vc = vc[pages].movedim(-2, -3).flatten(-2)
    vs = vs[pages].movedim(-1, -2)
    return k, _values(vc, vs).flatten(-3, -2)


# --- inputs -------------------------------------------------------------------------------

def _table(c, n, device="cuda"):
    """cos and sin of position * 10000^(-2i/rot), [n][rot] in float32."""
    half = c["rot"] // 2
    i = torch.arange(half, device=device, dtype=torch.float64)
    a = torch.arange(n, device=device, dtype=torch.float64)[:, None] \
        * 10000.0 ** (-i / max(half, 1))
    return torch.cat((a.cos(), a.sin()), 1).float()


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = _TYPES[c["dtype"]]
    B, P, h, d = c["B"], c["page"], c["h_kv"], c["d"]
    counts = _counts(c)
    N = sum(n for _, n in counts)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = {"case": c, "scale": 1.0 / math.sqrt(d)}
    # Each sequence's pages lie anywhere in the pool; the table is as wide as the longest needs.
    need = [-(-(p + n) // P) for p, n in counts]
    wide, total = max(need), sum(need) + 3
    where = torch.randperm(total, generator=g, device="cuda", dtype=torch.int32)
    first = torch.tensor([0] + need[:-1], device="cuda").cumsum(0)
    at = torch.arange(wide, device="cuda")[None, :]
    ours = at < torch.tensor(need, device="cuda")[:, None]
    s["pages"] = torch.where(ours, where[(first[:, None] + at).clamp(max=total - 1)], -1) \
        .to(torch.int32).contiguous()
    s["past"] = torch.tensor([p for p, _ in counts], dtype=torch.int32, device="cuda")
    s["T"] = c["T"]
    s["row_start"] = None
    if c["ragged"]:
        s["row_start"] = torch.tensor([0] + [n for _, n in counts], device="cuda").cumsum(0) \
            .to(torch.int32)
    if c["fmt"] == "dense":
        s["K"] = torch.empty(total, h, P, d, dtype=dtype, device="cuda")
        s["V"] = torch.empty_like(s["K"])
        for a in range(0, total, 4096):
            s["K"][a:a + 4096] = normal(*s["K"][a:a + 4096].shape)
            s["V"][a:a + 4096] = normal(*s["V"][a:a + 4096].shape)
    else:
        s["K"] = torch.empty(total, h, P, d // 2 + d // 32, dtype=torch.uint8, device="cuda")
        s["V"] = torch.empty_like(s["K"])
        step = max(1, (1 << 25) // (h * P * d))
        slot = torch.arange(P, device="cuda")
        for a in range(0, total, step):
            n = min(step, total - a)
            page = torch.arange(a, a + n, device="cuda").repeat_interleave(P)
            _put_mx4(c, s["K"], s["V"], page, slot.repeat(n), normal(n * P, h, d),
                     normal(n * P, h, d))
    s["q"] = normal(N, c["h_q"], d).to(dtype)
    if c["op"] == "attn":
        s["out"] = torch.empty_like(s["q"])
        if own:
            from paper_2607_19456_amd import binding
            s["workspace"] = binding.paged_workspace(s["q"], s["K"], s["pages"], T=s["T"])
        return s
    s["k"], s["v"] = normal(N, h, d).to(dtype), normal(N, h, d).to(dtype)
    s["rotary"] = _table(c, wide * P) if c["rot"] else None
    s["q_out"] = torch.empty_like(s["q"])
    if c["fmt"] == "mx4":
        s["k_back"], s["v_back"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    return s


# --- the plain form -----------------------------------------------------------------------

def _places(s):
    """Sequence, number in it, and position of every row."""
    n = torch.arange(s["q"].shape[0], device="cuda")
    if s["row_start"] is None:
        seq, r = n // s["T"], n % s["T"]
    else:
        seq = torch.searchsorted(s["row_start"], n, right=True, out_int32=True) - 1
        r = n - s["row_start"][seq]
    return seq, r, s["past"][seq] + r


def _rotate(c, x, rotary, pos, wide):
    """x [n][heads][d], its first rot dimensions turned by the position's angles."""
    x = x.to(wide)
    half = c["rot"] // 2
    if not half:
        return x
    cos = rotary[pos][:, None, :half].to(wide)
    sin = rotary[pos][:, None, half:].to(wide)
    if c["interleaved"]:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _plain_append(s):
    c = s["case"]
    seq, _, pos = _places(s)
    page = s["pages"][seq, pos // c["page"]]
    slot = pos % c["page"]
    s["q_out"].copy_(_rotate(c, s["q"], s["rotary"], pos, torch.float32))
    if c["fmt"] == "dense":
        s["K"][page, :, slot] = _rotate(c, s["k"], s["rotary"], pos, torch.float32) \
            .to(s["K"].dtype)
        s["V"][page, :, slot] = s["v"]
        return s["q_out"], s["K"], s["V"]
    # in 64 bits: values next to the border between two codes
    _put_mx4(c, s["K"], s["V"], page, slot, _rotate(c, s["k"], s["rotary"], pos, torch.float64),
             s["v"].float())
    kc, ks, vc, vs = _planes(c, s["K"], s["V"])
    s["k_back"].copy_(_values(kc[page, :, slot], ks[page, :, slot]))
    s["v_back"].copy_(_values(vc[page, :, slot // 8, :, slot % 8].flatten(-2),
                              vs[page, :, slot // 8, :, slot % 8]))
    return s["q_out"], s["k_back"], s["v_back"]


def _plain_attn(s):
    c = s["case"]
    B, T, h, G, d = c["B"], c["T"], c["h_kv"], c["h_q"] // c["h_kv"], c["d"]
    seq, r, _ = _places(s)
    q = torch.zeros(B, T, h, G, d, device="cuda")
    q[seq, r] = s["q"].float().unflatten(1, (h, G))
    k, v = _dense_pages(c, s["K"], s["V"], s["pages"].clamp(min=0))
    k, v = (x.movedim(2, 1).flatten(2, 3) for x in (k, v))          # [B][h][key][d]
    score = q.movedim(1, 2).flatten(2, 3) @ k.transpose(2, 3)       # [B][h][T*G][key]
    score.mul_(s["scale"])
    t = torch.arange(T, device="cuda").repeat_interleave(G)
    last = s["past"][:, None] + t if c["causal"] else (s["past"][:, None] - 1).expand(B, T * G)
    hidden = torch.arange(k.shape[2], device="cuda") > last[:, :, None]
    score.masked_fill_(hidden[:, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(total > 0, total, 1.0)
    o = o.unflatten(2, (T, G)).movedim(2, 1).flatten(2, 3)          # [B][T][h_q][d]
    s["out"].copy_(o[seq, r])
    return s["out"]


def run(state):
    s = state
    if not own:
        return _plain_attn(s) if s["case"]["op"] == "attn" else _plain_append(s)
    from paper_2607_19456_amd import binding
    if s["case"]["op"] == "attn":
        return binding.paged_attn(s["q"], s["K"], s["V"], s["pages"], s["past"], s["scale"],
                                  causal=s["case"]["causal"], row_start=s["row_start"], T=s["T"],
                                  out=s["out"], workspace=s["workspace"])
    binding.paged_append(s["K"], s["V"], s["pages"], s["past"], s["k"], s["v"], q=s["q"],
                         q_out=s["q_out"], rotary=s["rotary"],
                         interleaved=s["case"]["interleaved"], row_start=s["row_start"],
                         T=s["T"])
    if s["case"]["fmt"] == "dense":
        return s["q_out"], s["K"], s["V"]
    binding.paged_gather(s["K"], s["V"], s["pages"], s["past"], s["k_back"], s["v_back"],
                         row_start=s["row_start"], T=s["T"])
    return s["q_out"], s["k_back"], s["v_back"]


# --- the definition, in 64 bits -----------------------------------------------------------

def _turned(c, x, pos, table):
    y, half = x.double().clone(), c["rot"] // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        cos, sin = (table[pos, j].double()[:, None] for j in (i, half + i))
        y[..., a] = x[..., a].double() * cos - x[..., b].double() * sin
        y[..., b] = x[..., b].double() * cos + x[..., a].double() * sin
    return y


def _held(x):
    """What the 4-bit form makes of x: steps of half a power of two above 2, of
    a half below."""
    b = x.double().reshape(*x.shape[:-1], -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    one = torch.pow(2.0, torch.floor(torch.log2(top.clamp(min=2.0 ** -124))) - 2)
    y = b / one
    step = torch.pow(2.0, torch.floor(torch.log2(y.abs().clamp(min=1.0))) - 1)
    return (torch.round(y / step) * step).clamp(-6, 6).mul(one).reshape(x.shape)


def _rows64(c, K, V):
    """[head][row][d] of one sequence's pages, what a 4-bit cache stands for by
    its bits: sign, two of exponent, one of mantissa."""
    d, P = c["d"], c["page"]
    if c["fmt"] == "dense":
        return (x.transpose(0, 1).reshape(c["h_kv"], -1, d) for x in (K, V))
    n = K.shape[0]

    def number(code):
        e, m = (code >> 1 & 3).double(), (code & 1).double()
        x = torch.where(e > 0, (1 + m / 2) * 2 ** (e - 1), m / 2)
        return torch.where(code > 7, -x, x)

    out = []
    for x, keys in ((K, True), (V, False)):
        x = x.reshape(n, c["h_kv"], -1)
        code, scale = x[..., :P * d // 2], x[..., P * d // 2:].double()
        if keys:
            code, scale = code.reshape(n, -1, P, d // 2), scale.reshape(n, -1, P, d // 32)
        else:
            code = code.reshape(n, -1, P // 8, d // 8, 8, 4).permute(0, 1, 2, 4, 3, 5) \
                .reshape(n, -1, P, d // 2)
            scale = scale.reshape(n, -1, P // 8, d // 32, 8).transpose(3, 4) \
                .reshape(n, -1, P, d // 32)
        y = torch.stack((number(code & 15), number(code >> 4)), -1).flatten(-2)
        y = y * (2.0 ** (scale - 127)).repeat_interleave(32, -1)
        out.append(y.transpose(0, 1).reshape(c["h_kv"], -1, d))
    return out


def exact(case, seed):
    c = case
    s = prepare(dict(c), seed)
    P, G = c["page"], c["h_q"] // c["h_kv"]
    counts, table = _counts(c), s["pages"].tolist()
    starts = [sum(n for _, n in counts[:b]) for b in range(c["B"])]
    if c["op"] == "append":
        pos = torch.tensor([p + r for p, n in counts for r in range(n)], device="cuda")
        q = _turned(c, s["q"], pos, s["rotary"])
        k = _turned(c, s["k"], pos, s["rotary"])
        if c["fmt"] == "mx4":
            return q, _held(k), _held(s["v"])
        K, V = s["K"].double(), s["V"].double()
        page = torch.tensor([table[b][(p + r) // P] for b, (p, n) in enumerate(counts)
                             for r in range(n)], device="cuda")
        K[page, :, pos % P], V[page, :, pos % P] = k, s["v"].double()
        return q, K, V
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (p, n) in enumerate(counts):
        seen = p + n if c["causal"] else p
        if not seen:
            continue
        mine = torch.tensor(table[b][:-(-seen // P)], device="cuda")
        k, v = (x[:, :seen] for x in _rows64(c, s["K"][mine], s["V"][mine]))
        key = torch.arange(seen, device="cuda")
        for t0 in range(0, n, 256):
            rows = slice(starts[b] + t0, starts[b] + min(n, t0 + 256))
            t = torch.arange(t0, min(n, t0 + 256), device="cuda")
            for h in range(c["h_kv"]):
                kd, vd = k[h].double(), v[h].double()
                x = s["q"][rows, h * G:(h + 1) * G].double() * s["scale"]
                score = x.flatten(0, 1) @ kd.t()
                if c["causal"]:
                    score.masked_fill_(key > (p + t).repeat_interleave(G)[:, None], -math.inf)
                out[rows, h * G:(h + 1) * G] = (torch.softmax(score, 1) @ vd).unflatten(
                    0, (-1, G))
    return out
