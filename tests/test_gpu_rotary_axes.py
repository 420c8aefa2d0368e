"""Rotation by positions of several axes on the GPU against the plain 64-bit form of
prompt_reference.py, its inverse, and what a program does with it."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19456_amd as lib
import prompt_reference as ref

pytestmark = pytest.mark.gpu
TYPES = ["f32", "bf16", "f16"]


def make(device, dtype, rows, h_q, h_kv, d, rot, sections, n=500, seed=0):
    rng = np.random.default_rng(seed)
    q, k = (torch.from_numpy(rng.standard_normal((rows, h, d))).to(ref.DTYPES[dtype])
            for h in (h_q, h_kv))
    pos = torch.from_numpy(rng.integers(0, n, (len(sections), rows)).astype(np.int32))
    return q, k, pos, lib.rotary_table(n, rot, device="cpu")


def check(name, got, x, pos, table, sections, interleaved, inverse):
    want, tol = ref.rotate(x, pos, table, sections, interleaved, inverse)
    err = np.abs(got.double().cpu().numpy() - want)
    worst = np.max(err / tol)
    print(f"  {name}: max error {err.max():.3e}, {worst:.3f} of the bound", flush=True)
    assert worst <= 1.0


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rot,sections", [
    (128, 128, (16, 24, 24)), (64, 64, (32,)), (64, 32, (3, 13)), (256, 128, (1, 0, 60, 3)),
    (256, 256, (128,)), (128, 16, (4, 4)), (64, 48, (0, 24))])
def test_against_the_definition(cuda_device, dtype, d, rot, sections, interleaved, inverse):
    """Axes that begin inside a thread's pairs, empty sections, parts of heads."""
    for rows, h_q, h_kv in ((1, 4, 1), (37, 5, 2), (300, 2, 2)):
        q, k, pos, table = make(cuda_device, dtype, rows, h_q, h_kv, d, rot, sections, seed=rows)
        print(f"{dtype} d={d} rot={rot} {sections} rows={rows}", flush=True)
        a = (pos.to(cuda_device), table.to(cuda_device), sections)
        kw = dict(interleaved=interleaved, inverse=inverse)
        qo, ko = lib.rotary_axes(q.to(cuda_device), *a, k=k.to(cuda_device), **kw)
        check("q", qo, q, pos, table, sections, interleaved, inverse)
        check("k", ko, k, pos, table, sections, interleaved, inverse)
        alone, none = lib.rotary_axes(q.to(cuda_device), *a, **kw)
        assert none is None and torch.equal(alone, qo)


@pytest.mark.parametrize("dtype", TYPES)
def test_positions_outside_the_table_turn_nothing(cuda_device, dtype):
    q, k, pos, table = make(cuda_device, dtype, 40, 4, 2, 64, 64, (10, 12, 10), n=20)
    pos[0, ::3], pos[1, 1::3], pos[2, ::5] = -1, 20, 2 ** 31 - 1
    pos[:, 7] = -2 ** 31
    qo, ko = lib.rotary_axes(q.to(cuda_device), pos.to(cuda_device), table.to(cuda_device),
                             (10, 12, 10), k=k.to(cuda_device))
    check("q", qo, q, pos, table, (10, 12, 10), False, False)
    check("k", ko, k, pos, table, (10, 12, 10), False, False)
    assert torch.equal(qo[7].cpu(), q[7]) and torch.equal(ko[7].cpu(), k[7])


@pytest.mark.parametrize("interleaved,inverse", [(False, False), (True, False), (False, True),
                                                 (True, True)])
@pytest.mark.parametrize("sections", [(16, 16), (32,), (10, 12, 10), (3, 2, 0, 27)])
@pytest.mark.parametrize("dtype", TYPES)
def test_pairs_outside_the_table_are_copied(cuda_device, dtype, sections, interleaved, inverse):
    """To the bit, whatever the pair's other value is: infinities, NaN, zeros of either
    sign, the smallest numbers.  The other axes' pairs are turned as ever."""
    q, k, pos, table = make(cuda_device, dtype, 33, 4, 2, 64, 64, sections, n=20)
    odd = torch.tensor([math.inf, -math.inf, math.nan, -0.0, 0.0, 3.0, -5.0,
                        2.0 ** -24 if dtype == "f16" else 2.0 ** -133]).to(q.dtype)
    bits = torch.int32 if dtype == "f32" else torch.int16
    rng = np.random.default_rng(4)
    for axis in range(len(sections)):
        first = sum(sections[:axis])
        pairs = torch.arange(first, first + sections[axis])
        dims = torch.cat((2 * pairs, 2 * pairs + 1) if interleaved else (pairs, pairs + 32))
        there = pos.clone()
        there[axis] = torch.tensor([-1, 20, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).repeat(9)[:33]
        a = (there.to(cuda_device), table.to(cuda_device), sections)
        kw = dict(interleaved=interleaved, inverse=inverse)
        clean = lib.rotary_axes(q.to(cuda_device), *a, k=k.to(cuda_device), **kw)
        x = [y.clone() for y in (q, k)]
        for y in x:
            y[..., dims] = odd[torch.from_numpy(rng.integers(0, len(odd), (*y.shape[:2],
                                                                           len(dims))))]
        got = lib.rotary_axes(x[0].to(cuda_device), *a, k=x[1].to(cuda_device), **kw)
        for y, z, w in zip(got, x, clean):
            want = w.cpu().clone()
            want[..., dims] = z[..., dims]
            assert torch.equal(y.cpu().view(bits), want.view(bits)), axis


@pytest.mark.parametrize("dtype", TYPES)
def test_views_in_place_and_back(cuda_device, dtype):
    """q and k as views into a projection's output, turned in place, the rest left
    as it was; turned back, what was there, but for two roundings."""
    q, k, pos, table = make(cuda_device, dtype, 61, 4, 2, 128, 96, (16, 16, 16))
    v = torch.randn(61, 2, 128).to(q.dtype)
    qkv = torch.cat((q, k, v), 1).to(cuda_device)
    a = (pos.to(cuda_device), table.to(cuda_device), (16, 16, 16))
    qv, kv = qkv[:, :4], qkv[:, 4:6]
    want = lib.rotary_axes(q.to(cuda_device), *a, k=k.to(cuda_device))
    got = lib.rotary_axes(qv, *a, k=kv, q_out=qv, k_out=kv)
    assert got[0].data_ptr() == qv.data_ptr()
    assert torch.equal(qv, want[0]) and torch.equal(kv, want[1])
    assert torch.equal(qkv[:, 6:].cpu(), v)
    lib.rotary_axes(qv, *a, k=kv, inverse=True, q_out=qv, k_out=kv)
    step = ref.half_step(q.dtype)
    for x, y in ((qv, q), (kv, k)):
        # a pair's length bounds what a rounding of either part moves; cos^2 + sin^2 is
        # 1 but for the table's roundings
        size = torch.cat([torch.hypot(y[..., :48].double(), y[..., 48:96].double())] * 2
                         + [y[..., 96:].double().abs()], -1)
        err = (x.double().cpu() - y.double()).abs()
        assert (err <= size * (3 * step + 2.0 ** -20)).all()


def test_the_gradient_is_the_rotation_back(cuda_device):
    """<turn(x), g> = <x, turn back(g)>, and differences of the first."""
    q, _, pos, table = make(cuda_device, "f32", 30, 4, 1, 64, 64, (8, 12, 12))
    g = torch.randn(q.shape)
    a = (pos.to(cuda_device), table.to(cuda_device), (8, 12, 12))
    back, _ = lib.rotary_axes(g.to(cuda_device), *a, inverse=True)
    y, _ = lib.rotary_axes(q.to(cuda_device), *a)
    size = float((q.double().abs() * 2 * g.double().abs().flip(0)).sum()) + q.numel()
    assert abs(float((y.double().cpu() * g.double()).sum())
               - float((q.double() * back.double().cpu()).sum())) <= 8 * ref.E32 * size * 4
    way = torch.randn(q.shape)
    f = [float((lib.rotary_axes((q + s * way).to(cuda_device), *a)[0].double().cpu()
                * g.double()).sum()) for s in (0.5, -0.5)]     # linear: any step
    assert abs((f[0] - f[1]) - float((way.double() * back.double().cpu()).sum())) \
        <= 64 * ref.E32 * size


def test_one_axis_is_the_append_s_rotation(cuda_device):
    """The same numbers as paged_append's q for the same positions."""
    q, k, _, _ = make(cuda_device, "bf16", 6, 4, 2, 64, 64, (32,))
    table = lib.rotary_table(64, 64)
    K, V = lib.paged_alloc(4, 16, 2, 64)
    pages = torch.arange(4, dtype=torch.int32, device=cuda_device)[None]
    past = torch.tensor([20], dtype=torch.int32, device=cuda_device)
    want = lib.paged_append(K, V, pages, past, k.to(cuda_device), k.to(cuda_device),
                            q=q.to(cuda_device), rotary=table)
    pos = torch.arange(20, 26, dtype=torch.int32, device=cuda_device)[None]
    qo, ko = lib.rotary_axes(q.to(cuda_device), pos, table, (32,), k=k.to(cuda_device))
    assert torch.equal(qo, want)
    assert torch.equal(ko, K[1, :, 4:10].transpose(0, 1))


@pytest.mark.parametrize("dtype", TYPES)
def test_captured(cuda_device, dtype):
    q, k, pos, table = (x.to(cuda_device)
                        for x in make(cuda_device, dtype, 50, 4, 2, 64, 64, (16, 16)))
    out = [torch.empty_like(q), torch.empty_like(k)]
    lib.rotary_axes(q, pos, table, (16, 16), k=k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.rotary_axes(q, pos, table, (16, 16), k=k, q_out=out[0], k_out=out[1])
    for _ in range(3):
        q.copy_(torch.randn(q.shape)), k.copy_(torch.randn(k.shape))
        pos.copy_(torch.randint(0, 500, pos.shape))
        graph.replay()
        torch.cuda.synchronize()
        want = lib.rotary_axes(q, pos, table, (16, 16), k=k)
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_offsets_beyond_32_bits(cuda_device):
    rows, h, d = (1 << 31) // (32 * 128) + 100, 32, 128
    q = torch.zeros(rows, h, d, dtype=torch.bfloat16, device=cuda_device)
    q[-3:] = torch.randn(3, h, d)
    pos = torch.zeros(1, rows, dtype=torch.int32, device=cuda_device)
    pos[0, -3:] = torch.tensor([5, 77, 499])
    table = lib.rotary_table(500, 128)
    want, _ = lib.rotary_axes(q[-3:].clone(), pos[:, -3:].contiguous(), table, (64,))
    got, _ = lib.rotary_axes(q, pos, table, (64,))
    assert torch.equal(got[-3:], want)


# --- the operators as a program uses them ---------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_training_step_of_one_attention(cuda_device, dtype):
    """Turn q and k, attend, and the gradients back through both, against torch's
    gradient in 64 bits of the whole.  The bound: 16-bit q and k are rounded between
    the two, a half step each, which moves a score by 2 u of its terms, and the results
    by what that does to the weights and to dS; twice over for the backward's own
    rounding between its two calls."""
    t, h_q, h_kv, d, sec = [40, 23], 4, 2, 64, (8, 12, 12)
    q, k, pos, table = make(cuda_device, dtype, sum(t), h_q, h_kv, d, 64, sec)
    v, g = torch.randn(sum(t), h_kv, d).to(q.dtype), torch.randn(sum(t), h_q, d).to(q.dtype)
    dev = [x.to(cuda_device) for x in (q, k, v, g, pos, table)]
    rs = torch.tensor([0, 40, 63], dtype=torch.int32, device=cuda_device)
    scale = 1 / math.sqrt(d)
    qt, kt = lib.rotary_axes(dev[0], dev[4], dev[5], sec, k=dev[1])
    lse = torch.empty(sum(t), h_q, device=cuda_device)
    out = lib.prompt_attn(qt, kt, dev[2], scale, row_start=rs, T=40, lse=lse)
    dq, dk, dv = lib.prompt_attn_grad(qt, kt, dev[2], out, lse, dev[3], scale, row_start=rs, T=40)
    dq, dk = lib.rotary_axes(dq, dev[4], dev[5], sec, k=dk, inverse=True)

    x = [y.double().requires_grad_() for y in (q, k, v)]
    cos = torch.cat([table.double()[pos[a].long(), b:b + n] for a, b, n in
                     zip(range(3), (0, 8, 20), sec)], 1)[:, None]
    sin = torch.cat([table.double()[pos[a].long(), 32 + b:32 + b + n] for a, b, n in
                     zip(range(3), (0, 8, 20), sec)], 1)[:, None]

    def turn(y):
        a, b = y[..., :32], y[..., 32:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)

    Q, K = turn(x[0]), turn(x[1])
    total, outs, at = 0.0, [], 0
    size = 0.0
    for n in t:
        s = torch.einsum("thd,nhd->htn", Q[at:at + n], K[at:at + n].repeat_interleave(2, 1)) * scale
        size = max(size, float((Q[at:at + n].abs().amax() * K[at:at + n].abs().amax()) * d * scale))
        s = s.masked_fill(~torch.ones(n, n).tril().bool(), -math.inf)
        o = torch.einsum("htn,nhd->thd", s.softmax(-1), x[2][at:at + n].repeat_interleave(2, 1))
        outs.append(o)
        total = total + (o * g[at:at + n].double()).sum()
        at += n
    want = torch.autograd.grad(total, x)
    u = ref.half_step(q.dtype) + 64 * ref.E32
    # relative to each result's largest value: 2 u a score's terms (its largest possible
    # `size`, which random signs make 1/4 of), and some roundings on the way
    for name, got, w in (("out", out, torch.cat(outs).detach()), ("dq", dq, want[0]),
                         ("dk", dk, want[1]), ("dv", dv, want[2])):
        err = float((got.double().cpu() - w).abs().max() / w.abs().max())
        print(f"  {name}: {err:.2e} of the largest, bound {u * (8 + size):.2e}", flush=True)
        assert err <= u * (8 + size)


def test_a_prompt_of_an_image_then_tokens(cuda_device):
    """Serving: a prompt with an image is turned, attended to whole, and appended to
    the pages as it is; tokens follow, their positions behind the image's.  The whole
    prompt's attention is that of the pages, and a token's that of the packed form."""
    h_q, h_kv, d, P, dt = 4, 2, 64, 16, torch.bfloat16
    text, high, wide = 9, 4, 6
    grid = torch.stack(torch.meshgrid(torch.arange(1), torch.arange(high), torch.arange(wide),
                                      indexing="ij")).reshape(3, -1) + text
    after = text + max(high, wide)
    pos = torch.cat((torch.arange(text).expand(3, -1), grid,
                     torch.arange(after, after + 5).expand(3, -1)), 1).to(torch.int32)
    n = pos.shape[1]
    pos = pos.to(cuda_device)
    table, sec, scale = lib.rotary_table(256, d), (8, 12, 12), 1 / math.sqrt(d)
    gen = torch.Generator(device=cuda_device).manual_seed(1)
    qkv = torch.randn(n + 3, h_q + 2 * h_kv, d, device=cuda_device, generator=gen).to(dt)
    q, k, v = qkv.split((h_q, h_kv, h_kv), 1)
    steps = torch.arange(after + 5, after + 8, dtype=torch.int32, device=cuda_device).expand(3, -1)
    allpos = torch.cat((pos, steps), 1).contiguous()
    qt, kt = lib.rotary_axes(q, allpos, table, sec, k=k)
    whole = lib.prompt_attn(qt, kt, v, scale)

    K, V = lib.paged_alloc(8, P, h_kv, d, dtype=dt)
    pages = torch.tensor([[5, 2, 7, 0]], dtype=torch.int32, device=cuda_device)
    past = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    lib.paged_append(K, V, pages, past, kt[:n], v[:n])
    got = [lib.paged_attn(qt[:n].contiguous(), K, V, pages, past, scale)]
    for i in range(n, n + 3):
        past.fill_(i)
        q1, k1 = lib.rotary_axes(q[i:i + 1], allpos[:, i:i + 1].contiguous(), table, sec,
                                 k=k[i:i + 1])
        assert torch.equal(q1, qt[i:i + 1]) and torch.equal(k1, kt[i:i + 1])
        lib.paged_append(K, V, pages, past, k1, v[i:i + 1])
        got.append(lib.paged_attn(q1, K, V, pages, past, scale))
    # each is within 3 half steps and a rounding of the mean of |v| (bounded by its
    # largest value) of the exact result, in two kernels
    room = 2 * 4 * ref.half_step(dt) * float(v.abs().max())
    assert float((torch.cat(got).float() - whole.float()).abs().max()) <= room
