"""Attention over packed prompts and its gradient on the GPU against the plain
64-bit forms of prompt_reference.py: every type, head size and group, lengths from
none to several tiles, rows that no sequence has poisoned."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19456_amd as lib
import prompt_reference as ref

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def starts(counts):
    return np.concatenate(([0], np.cumsum(counts))).astype(np.int32)


class Case:
    """Arrays of a call on the CPU, everything outside the sequences poisoned."""

    def __init__(self, dtype="bf16", d=64, h_q=4, h_kv=2, t=(37,), n=None, causal=True, seed=0,
                 behind=3, T=None, N=None, scale=None, q_scale=1.5):
        self.t, self.n = list(t), list(t if n is None else n)
        self.type, self.d, self.h_q, self.h_kv = ref.DTYPES[dtype], d, h_q, h_kv
        self.rs, self.ks = starts(self.t), starts(self.n)
        self.rows, self.keys = int(self.rs[-1]) + behind, int(self.ks[-1]) + behind
        self.T, self.N = T or max(max(self.t), 1), N or max(max(self.n), 1)
        self.scale = 1 / math.sqrt(d) if scale is None else scale
        self.causal, self.seed = causal, seed
        rng = np.random.default_rng(seed)

        def normal(rows, heads, by=1.0):
            return torch.from_numpy(rng.standard_normal((rows, heads, d)) * by).to(self.type)

        self.q, self.k = normal(self.rows, h_q, q_scale), normal(self.keys, h_kv)
        self.v, self.g = normal(self.keys, h_kv), normal(self.rows, h_q)
        self.batch = ref.Batch(self.rows, self.keys, self.rs, self.ks, self.T, self.N,
                               len(self.t), causal)
        for x in (self.q, self.g):
            x[torch.from_numpy(~self.batch.mine("q"))] = math.nan
        for x in (self.k, self.v):
            x[torch.from_numpy(~self.batch.mine("k"))] = math.nan
        say(f"{dtype} d={d} h={h_q}/{h_kv} t={self.t[:6]} n={self.n[:6]} causal={causal} "
            f"seed={seed}")

    def packed(self, device):
        return dict(causal=self.causal, row_start=torch.from_numpy(self.rs).to(device), T=self.T,
                    key_start=torch.from_numpy(self.ks).to(device), N=self.N)

    def forward(self, device, lse=True, **kw):
        out = torch.full(self.q.shape, math.nan, dtype=self.type, device=device)
        L = torch.full(self.q.shape[:2], math.nan, device=device) if lse else None
        lib.prompt_attn(self.q.to(device), self.k.to(device), self.v.to(device), self.scale,
                        out=out, lse=L, **{**self.packed(device), **kw})
        torch.cuda.synchronize()
        return out, L

    def backward(self, device, out, lse, **kw):
        nan = [torch.full(x.shape, math.nan, dtype=self.type, device=device)
               for x in (self.q, self.k, self.v)]
        lib.prompt_attn_grad(self.q.to(device), self.k.to(device), self.v.to(device), out, lse,
                             self.g.to(device), self.scale, dq=nan[0], dk=nan[1], dv=nan[2],
                             **{**self.packed(device), **kw})
        torch.cuda.synchronize()
        return nan


def compare(name, got, want, tol, mine):
    got = got.double().cpu().numpy()
    assert np.isnan(got[~mine]).all(), f"{name}: places of no sequence were written"
    got, want, tol = got[mine], want[mine], tol[mine]
    assert np.array_equal(np.isnan(want), np.isnan(got)), f"{name}: NaN elsewhere"
    odd = np.isinf(want)
    assert np.array_equal(got[odd], want[odd]), f"{name}: infinities elsewhere"
    ok = np.isfinite(want)
    if not ok.any():
        return
    err = np.abs(got[ok] - want[ok])
    worst = np.max(err / tol[ok])
    say(f"  {name}: max error {err.max():.3e}, {worst:.3f} of the bound")
    assert worst <= 1.0


def check_forward(c, device, lse=True, **kw):
    out, L = c.forward(device, lse, **kw)
    want, want_L, mass, spread, seen, top_v = ref.attention(c.q, c.k, c.v, c.scale, c.batch)
    mine = c.batch.mine("q")
    compare("out", out, want, ref.tolerance(want, mass, spread, seen, top_v, c.type, c.d), mine)
    if lse:
        with np.errstate(invalid="ignore"):
            compare("lse", L, want_L, ref.lse_tolerance(want_L, spread, seen, c.d), mine)
    return out, L


def check_gradient(c, device, **kw):
    out, L = c.forward(device)
    grads = c.backward(device, out, L, **kw)
    want, tol = ref.gradient(c.q, c.k, c.v, out, L, c.g, c.scale, c.batch)
    for name, x, w, b, which in zip(("dq", "dk", "dv"), grads, want, tol, "qkk"):
        compare(name, x, w, b, c.batch.mine(which))
    return grads


DS = [64, 128, 256]
TYPES = ["f32", "bf16", "f16"]
LENGTHS = [1, 2, 31, 32, 33, 63, 64, 65, 127, 130]


@pytest.mark.parametrize("d", DS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_lengths(cuda_device, dtype, d, causal):
    """From one token on, around every tile's edges, and a sequence of none."""
    check_forward(Case(dtype, d, t=LENGTHS + [0], causal=causal, seed=d), cuda_device)


@pytest.mark.parametrize("d", DS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_gradient_lengths(cuda_device, dtype, d, causal):
    check_gradient(Case(dtype, d, t=LENGTHS + [0], causal=causal, seed=d), cuda_device)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (3, 3), (5, 1), (8, 2), (7, 1), (16, 1), (40, 2),
                                      (10, 5)])
@pytest.mark.parametrize("dtype", TYPES)
def test_head_groups(cuda_device, dtype, h_q, h_kv):
    c = Case(dtype, 64, h_q, h_kv, t=[70, 9, 33], seed=h_q)
    check_forward(c, cuda_device)
    check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 128), ("bf16", 256)])
@pytest.mark.parametrize("causal", [True, False])
def test_long_sequences(cuda_device, dtype, d, causal):
    """Many tiles, of odd numbers; wider tiles of rows."""
    c = Case(dtype, d, 8, 2, t=[517, 1030, 3], causal=causal, seed=1)
    check_forward(c, cuda_device)
    check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_other_keys(cuda_device, dtype, causal):
    """Fewer keys than rows (causal: the first rows see nothing), more, and none."""
    c = Case(dtype, 128, 4, 1, t=[5, 80, 100, 1, 7, 0, 64], n=[80, 5, 0, 300, 6, 9, 64],
             causal=causal, seed=2)
    check_forward(c, cuda_device)
    check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", DS)
@pytest.mark.parametrize("t,n", [(1, 700), (1, 5000), (7, 3001), (40, 1500), (1, 1)])
def test_few_rows_over_many_keys(cuda_device, dtype, d, t, n):
    """The keys read in parts that are put together."""
    check_forward(Case(dtype, d, 8, 2, t=[t], n=[n], seed=n), cuda_device)
    check_forward(Case(dtype, d, 4, 2, t=[t, 3], n=[n, 64], causal=False, seed=n), cuda_device,
                  lse=False)


@pytest.mark.parametrize("dtype", TYPES)
def test_even_sequences_without_starts(cuda_device, dtype):
    """T rows of every sequence, N keys; and one sequence, its own keys."""
    c = Case(dtype, 64, 4, 2, t=[19] * 5, n=[45] * 5, behind=0, seed=3)
    want = check_forward(c, cuda_device)
    a = [x.to(cuda_device) for x in (c.q, c.k, c.v)]
    lse = torch.empty(c.q.shape[:2], device=cuda_device)
    out = lib.prompt_attn(*a, c.scale, T=19, N=45, lse=lse)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    for other in (dict(T=19), dict(T=19, key_start=torch.from_numpy(c.ks).to(cuda_device), N=45),
                  dict(row_start=torch.from_numpy(c.rs).to(cuda_device), T=19, N=45)):
        assert torch.equal(lib.prompt_attn(*a, c.scale, **other), want[0])
    grads = lib.prompt_attn_grad(*a, out, lse, c.g.to(cuda_device), c.scale, T=19, N=45)
    for x, y in zip(grads, c.backward(cuda_device, *want)):
        assert torch.equal(x, y)
    c = Case(dtype, 64, 4, 2, t=[77], behind=0, seed=4)
    want = check_forward(c, cuda_device)[0]
    a = [x.to(cuda_device) for x in (c.q, c.k, c.v)]
    assert torch.equal(lib.prompt_attn(*a, c.scale), want)
    assert torch.equal(lib.prompt_attn(*a, c.scale, row_start=torch.tensor(
        [0, 77], dtype=torch.int32, device=cuda_device), T=77), want)


@pytest.mark.parametrize("dtype", TYPES)
def test_views_into_fused_projections(cuda_device, dtype):
    """Strided q, k, v, d_out, dq, dk and dv: the same bits as contiguous ones, and
    nothing beside them written."""
    c = Case(dtype, 64, 4, 2, t=[50, 81], behind=0, seed=5)
    out, lse = check_forward(c, cuda_device)
    want = c.backward(cuda_device, out, lse)
    qkv = torch.cat((c.q, c.k, c.v), 1).to(cuda_device)
    q, k, v = qkv.split((4, 2, 2), 1)
    wide = torch.full((c.rows, 11, 64), math.nan, dtype=c.type, device=cuda_device)
    g = torch.cat((c.g, c.g), 1).to(cuda_device)[:, 4:]
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)
    lib.prompt_attn(q, k, v, c.scale, out=got, lse=got_lse, **c.packed(cuda_device))
    assert torch.equal(got, out) and torch.equal(got_lse, lse)
    lib.prompt_attn_grad(q, k, v, out, lse, g, c.scale, dq=wide[:, 1:5], dk=wide[:, 6:8],
                         dv=wide[:, 8:10], **c.packed(cuda_device))
    for x, y in zip((wide[:, 1:5], wide[:, 6:8], wide[:, 8:10]), want):
        assert torch.equal(x, y)
    assert torch.isnan(wide[:, [0, 5, 10]]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_out_in_the_place_of_q(cuda_device, dtype):
    """Whole, and with the keys read in parts."""
    for c in (Case(dtype, 64, 4, 2, t=[300, 33], behind=0, seed=25),
              Case(dtype, 128, 8, 2, t=[9], n=[3000], behind=0, seed=26)):
        want, _ = c.forward(cuda_device)
        q = c.q.to(cuda_device)
        lib.prompt_attn(q, c.k.to(cuda_device), c.v.to(cuda_device), c.scale, out=q,
                        **c.packed(cuda_device))
        assert torch.equal(q, want)


def test_the_largest_strides(cuda_device):
    """Tokens 4 MiB apart: offsets within a tile of rows near 2^30."""
    c = Case("bf16", 64, 2, 1, t=[200], behind=0, seed=27)
    out, lse = c.forward(cuda_device)
    want = c.backward(cuda_device, out, lse)
    wide = torch.empty(200, 1 << 21, dtype=torch.bfloat16, device=cuda_device)
    parts, at = {}, 0
    for name, x in (("q", c.q), ("k", c.k), ("v", c.v), ("g", c.g), ("dq", c.q), ("dk", c.k),
                    ("dv", c.v)):
        n = x.shape[1] * 64
        parts[name] = wide[:, at:at + n].unflatten(1, (-1, 64))
        parts[name].copy_(x)
        at += n
    p = c.packed(cuda_device)
    got, L = torch.empty_like(out), torch.empty_like(lse)
    lib.prompt_attn(parts["q"], parts["k"], parts["v"], c.scale, out=got, lse=L, **p)
    assert torch.equal(got, out) and torch.equal(L, lse)
    lib.prompt_attn_grad(parts["q"], parts["k"], parts["v"], out, lse, parts["g"], c.scale,
                         dq=parts["dq"], dk=parts["dk"], dv=parts["dv"], **p)
    for x, y in zip((parts["dq"], parts["dk"], parts["dv"]), want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_starts_that_lie(cuda_device, dtype):
    """Longer sequences than T and N, starts that fall, are negative or beyond the
    arrays: what lies within is taken, the rest is not touched."""
    c = Case(dtype, 64, 4, 2, t=[30, 30, 30], behind=0, seed=6)
    for rs, ks, T, N in (([0, 40, 70, 90], [0, 35, 60, 90], 20, 25),
                         ([-5, 10, 4, 200], [3, 50, 50, 1 << 30], 90, 90),
                         ([50, 20, 90, 90], [90, 0, 60, 61], 64, 64)):
        c.rs, c.ks, c.T, c.N = np.array(rs, np.int32), np.array(ks, np.int32), T, N
        c.batch = ref.Batch(90, 90, c.rs, c.ks, T, N, 3, True)
        if len(set(np.concatenate([np.arange(s, s + n) for s, n in c.batch.q]))) == \
                sum(n for _, n in c.batch.q):
            check_forward(c, cuda_device)
        else:
            c.forward(cuda_device)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.125, 0.7, 1e-6])
def test_scales(cuda_device, dtype, scale):
    c = Case(dtype, 64, 4, 2, t=[40, 70], seed=7, scale=scale)
    check_forward(c, cuda_device)
    check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_calls_give_equal_bits(cuda_device, dtype):
    c = Case(dtype, 128, 8, 2, t=[700, 45], seed=8)
    out, lse = c.forward(cuda_device)
    grads = c.backward(cuda_device, out, lse)
    for _ in range(3):
        again = c.forward(cuda_device)
        assert torch.equal(again[0][:745], out[:745]) and torch.equal(again[1][:745], lse[:745])
        for x, y in zip(c.backward(cuda_device, out, lse), grads):
            assert torch.equal(x[:745], y[:745])


@pytest.mark.parametrize("dtype", TYPES)
def test_without_lse_the_same_out(cuda_device, dtype):
    c = Case(dtype, 64, 4, 2, t=[200, 33], behind=0, seed=9)
    assert torch.equal(c.forward(cuda_device)[0], c.forward(cuda_device, lse=False)[0])


# --- gradients against the function itself -------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_gradient_of_the_function(cuda_device, dtype, causal):
    """Forward and backward together against torch's gradient in 64 bits, and against
    differences of the 64-bit function."""
    c = Case(dtype, 64, 6, 2, t=[45, 70], n=[45, 90], causal=causal, behind=0, seed=10)
    out, lse = c.forward(cuda_device)
    grads = c.backward(cuda_device, out, lse)
    x = [y.double().requires_grad_() for y in (c.q, c.k, c.v)]

    def f(q, k, v):
        total = 0.0
        for rows, keys, seen in c.batch:
            s = torch.einsum("thd,nhd->htn", q[rows], k[keys].repeat_interleave(3, 1)) * c.scale
            s = s.masked_fill(~torch.from_numpy(seen), -math.inf)
            o = torch.einsum("htn,nhd->thd", s.softmax(-1), v[keys].repeat_interleave(3, 1))
            total = total + (o * c.g[rows].double()).sum()
        return total

    want = torch.autograd.grad(f(*x), x)
    own, tol = ref.gradient(c.q, c.k, c.v, out, lse, c.g, c.scale, c.batch, exact=True)
    rng = np.random.default_rng(11)
    for i, name in enumerate(("dq", "dk", "dv")):
        compare(name, grads[i], want[i].numpy(), tol[i], np.ones(len(tol[i]), bool))
        way = torch.from_numpy(rng.standard_normal(x[i].shape))
        step = 1e-5
        with torch.no_grad():
            ends = [f(*(y + sign * step * way if j == i else y for j, y in enumerate(x)))
                    for sign in (1, -1)]
        slope = float(ends[0] - ends[1]) / (2 * step)
        got = float((grads[i].double().cpu() * way).sum())
        # (64-bit differences: 1e-16 of f over the step, and the third derivative's
        # share of its square)
        room = float((tol[i] * way.abs().numpy()).sum()) + 1e-5 * (1 + abs(slope))
        say(f"  {name} along a line: {got:.6f}, differences {slope:.6f}, room {room:.2e}")
        assert abs(got - slope) <= room


# --- values that are not finite -------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 64), ("f16", 128), ("bf16", 256)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_keys_that_are_not_seen_stay_out(cuda_device, dtype, d, bad):
    """v, k, q and d_out with a value that is not finite in places that some rows
    (or keys) see and others of the same tile do not."""
    for which in ("k", "v", "q", "g"):
        c = Case(dtype, d, 4, 2, t=[100, 41], n=[130, 41], seed=12)
        x = getattr(c, which)
        x[60, 1, 3] = bad
        x[90 if which in "qg" else 128, 0, d - 1] = bad
        say(f"  {which}")
        with np.errstate(invalid="ignore", over="ignore"):
            if math.isnan(bad) or which == "v":
                check_forward(c, cuda_device)
            if math.isnan(bad) or which == "g":
                check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_that_are_all_minus_infinity(cuda_device, dtype):
    """Rows of them give 0, an lse of -infinity, and no gradient."""
    c = Case(dtype, 64, 2, 1, t=[70], behind=0, seed=13)
    c.q[20] = 0
    c.q[20, :, 0] = 1.0
    c.k[:, :, 0] = -math.inf
    c.q[:20, :, 0] = c.q[21:, :, 0] = 1.0
    out, lse = c.forward(cuda_device)
    assert torch.equal(out, torch.zeros_like(out)) and (lse == -math.inf).all()
    dq, dk, dv = c.backward(cuda_device, out, lse)
    assert torch.equal(dv, torch.zeros_like(dv))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("h_q,h_kv,B", [(4, 2, 1), (64, 64, 4)])
def test_weights_of_0_meet_infinities(cuda_device, dtype, h_q, h_kv, B):
    """A row sees a thousand keys whose scores are -infinity, one of them with an infinity in
    V, before others: 0 times that is NaN, in its dimension alone, whether the keys are read
    whole (four sequences of 64 heads) or in parts, one of which has no other scores.  Rows of
    such scores alone still give 0."""
    c = Case(dtype, 128, h_q, h_kv, t=[3] * B, n=[3000] * B, causal=False, behind=0, seed=28)
    c.q[:, :, 0] = 1.0
    for b in range(B):
        c.k[3000 * b:3000 * b + 1000, :, 0] = -math.inf
        c.k[3000 * b + 1000:3000 * (b + 1), :, 0] = 0.0
    c.v[100, 0, 3], c.v[777, 1, 5] = math.inf, -math.inf
    out, lse = c.forward(cuda_device)
    G = h_q // h_kv
    want = torch.zeros(c.rows, h_q, 128, dtype=torch.bool)
    want[:3, :G, 3] = want[:3, G:2 * G, 5] = True
    assert torch.equal(torch.isnan(out).cpu(), want)
    for head in (0, G, h_q - 1):
        last = slice(c.keys - 2000, c.keys)
        q, k, v = c.q[-3:, head:head + 1], c.k[last, [head // G]], c.v[last, [head // G]]
        o, L, mass, spread, seen, top = ref.attention(q, k, v, c.scale,
                                                      ref.Batch(3, 2000, T=3, N=2000, causal=False))
        fine = ~want[-3:, head:head + 1].numpy()
        err = np.abs(out[-3:, head:head + 1].double().cpu().numpy() - o)[fine]
        assert (err <= ref.tolerance(o, mass, spread, seen, top, c.type, 128)[fine]).all()
        err = np.abs(lse[-3:, head:head + 1].double().cpu().numpy() - L)
        assert (err <= ref.lse_tolerance(L, spread, seen, 128)).all()
    c.k[:, :, 0] = -math.inf
    out, lse = c.forward(cuda_device)
    assert torch.equal(out, torch.zeros_like(out)) and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_any_size(cuda_device, dtype):
    """Far apart, and so large that a reference's rounding would show."""
    top = {"f32": 3e12, "bf16": 3e12, "f16": 200.0}[dtype]
    for by in (1.0, 40.0, top):
        c = Case(dtype, 64, 4, 2, t=[150], seed=14, q_scale=by, behind=0)
        out, lse = c.forward(cuda_device)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        if by <= 40:
            check_forward(c, cuda_device)
            check_gradient(c, cuda_device)
        else:                       # the largest score's value alone
            s = np.stack([c.q[:, h].double().numpy() @ c.k[:, h // 2].double().numpy().T
                          for h in range(4)])
            s[:, ~np.tri(150, dtype=bool)] = -np.inf
            best = s.argmax(-1)
            two = np.sort(s, -1)[..., -2:]
            clear = (two[..., 1] - two[..., 0]) * c.scale > 1e-4 * np.abs(two[..., 1]) + 40
            for h in range(4):
                rows = np.flatnonzero(clear[h])
                assert len(rows) > 20
                assert torch.equal(out[rows, h].cpu(), c.v[best[h, rows], h // 2])


# --- streams, graphs, long arrays -----------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(cuda_device, dtype):
    """Forward (in parts, and whole) and backward in one graph, replayed over new
    inputs, with eager work between."""
    c = Case(dtype, 64, 4, 2, t=[90, 40], n=[90, 900], behind=0, seed=15)
    dev = [x.to(cuda_device) for x in (c.q, c.k, c.v, c.g)]
    p = c.packed(cuda_device)
    out, lse = torch.empty_like(dev[0]), torch.empty(c.q.shape[:2], device=cuda_device)
    grads = [torch.empty_like(x) for x in dev[:3]]
    ws = [lib.prompt_workspace(*dev[:2], grad=g, **{k: v for k, v in p.items() if k != "causal"})
          for g in (False, True)]

    def step():
        lib.prompt_attn(*dev[:3], c.scale, out=out, lse=lse, workspace=ws[0], **p)
        lib.prompt_attn_grad(*dev[:3], out, lse, dev[3], c.scale, dq=grads[0], dk=grads[1],
                             dv=grads[2], workspace=ws[1], **p)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        for x in dev:
            x.copy_(torch.randn(x.shape, device=cuda_device))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, *grads)]
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, (out, lse, *grads)):
            assert torch.equal(x, y), turn


def test_two_streams(cuda_device):
    """Calls on two streams at once, each with what it allocates for itself."""
    cases = [Case("bf16", 128, 8, 2, t=[900, 300], seed=16), Case("bf16", 128, 8, 2, t=[5], n=[4000],
                                                                  seed=17)]
    want = []
    for c in cases:
        out, lse = c.forward(cuda_device)
        want.append((out, lse, *c.backward(cuda_device, out, lse)))
    inputs = [[x.to(cuda_device) for x in (c.q, c.k, c.v, c.g)] for c in cases]
    packed = [c.packed(cuda_device) for c in cases]
    lse = [torch.full(c.q.shape[:2], math.nan, device=cuda_device) for c in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for c, x, p, L, s in zip(cases, inputs, packed, lse, streams):
            out = lib.prompt_attn(*x[:3], c.scale, lse=L, stream=s, **p)
            got.append((out, L, *lib.prompt_attn_grad(*x[:3], out, L, x[3], c.scale, stream=s,
                                                      **p)))
        torch.cuda.synchronize()
        for c, a, b in zip(cases, got, want):
            rows, keys = c.rs[-1], c.ks[-1]
            for x, y, n in zip(a, b, (rows, rows, rows, keys, keys)):
                assert torch.equal(x[:n], y[:n])


def test_offsets_beyond_32_bits(cuda_device):
    """Sequences that begin more than 2^31 values into their arrays."""
    d, h, far = 128, 8, (1 << 31) // (128 * 8) + 1000
    c = Case("bf16", d, h, h, t=[150], behind=0, seed=18)
    big = {}
    for name in ("q", "k", "v", "g"):
        big[name] = torch.zeros(far + 150, h, d, dtype=torch.bfloat16, device=cuda_device)
        big[name][far:] = getattr(c, name).to(cuda_device)
    start = torch.tensor([far, far + 150], dtype=torch.int32, device=cuda_device)
    out, lse = c.forward(cuda_device)
    want = c.backward(cuda_device, out, lse)
    L = torch.zeros(far + 150, h, device=cuda_device)
    p = dict(row_start=start, T=150, key_start=start, N=150)
    got = lib.prompt_attn(big["q"], big["k"], big["v"], c.scale, lse=L, **p)
    assert torch.equal(got[far:], out) and torch.equal(L[far:], lse)
    grads = lib.prompt_attn_grad(big["q"], big["k"], big["v"], got, L, big["g"], c.scale, **p)
    for x, y in zip(grads, want):
        assert torch.equal(x[far:], y)


def test_many_short_sequences(cuda_device):
    """More sequences than a wave counts at once, some of none."""
    rng = np.random.default_rng(19)
    t = rng.integers(0, 12, 300).tolist()
    c = Case("bf16", 64, 4, 1, t=t, seed=20)
    check_forward(c, cuda_device)
    check_gradient(c, cuda_device)


# --- the forms that large calls take ---------------------------------------------------

@pytest.mark.parametrize("B,t_max,h_q,h_kv", [(65, 300, 4, 1), (128, 90, 8, 2), (200, 40, 12, 1),
                                              (4096, 3, 4, 2), (4100, 2, 8, 1)])
@pytest.mark.parametrize("even", [False, True])
def test_many_sequences(cuda_device, B, t_max, h_q, h_kv, even):
    """More sequences than a wave looks at in a step, and than it looks at in two: all their
    items are found, once each, whether lengths differ (some are 0) or not."""
    rng = np.random.default_rng(B + t_max)
    t = [t_max] * B if even else [int(x) for x in rng.integers(0, t_max + 1, B)]
    n = None if even else [int(x) for x in rng.integers(0, 2 * t_max + 1, B)]
    c = Case("bf16", 64, h_q, h_kv, t=t, n=n, seed=B)
    check_gradient(c, cuda_device)
    check_forward(c, cuda_device)


@pytest.mark.parametrize("dtype,d,h_q,h_kv,B,t,n", [
    ("bf16", 128, 32, 2, 51, (194, 201), None), ("f16", 64, 64, 16, 37, (26, 85), None),
    ("bf16", 128, 8, 8, 35, (515, 719), (1, 4)), ("bf16", 64, 16, 4, 40, (170, 330), (1, 90)),
    ("bf16", 256, 16, 2, 24, (60, 130), None), ("f32", 64, 16, 4, 40, (60, 130), None)])
def test_gradient_of_many_workgroups(cuda_device, dtype, d, h_q, h_kv, B, t, n):
    """Rows and keys are fetched ahead, beyond the last too: while many workgroups share the
    memory, such a fetch may arrive when the results already pass through LDS."""
    rng = np.random.default_rng(B + d)
    counts = rng.integers(t[0], t[1] + 1, B).tolist()
    keys = None if n is None else rng.integers(n[0], n[1] + 1, B).tolist()
    c = Case(dtype, d, h_q, h_kv, t=counts, n=keys, causal=n is None, seed=B)
    out, L = c.forward(cuda_device)
    first = c.backward(cuda_device, out, L)
    for again in range(5):
        for x, y in zip(first, c.backward(cuda_device, out, L)):
            assert torch.equal(x.nan_to_num(nan=7.0), y.nan_to_num(nan=7.0)), f"call {again}"
    check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", DS)
@pytest.mark.parametrize("rows,keys", [(600, 1600), (600, 2500), (100, 1100), (3000, 3000)])
def test_a_workspace_serves_masked_calls_and_others(cuda_device, dtype, d, rows, keys):
    """The workspace's size goes by the arrays, not by what their rows see."""
    q = torch.randn(rows, 4, d, device=cuda_device).to(ref.DTYPES[dtype])
    k = torch.randn(keys, 2, d, device=cuda_device).to(ref.DTYPES[dtype])
    lse = torch.empty(rows, 4, device=cuda_device)
    ws = lib.prompt_workspace(q, k)
    back = lib.prompt_workspace(q, k, grad=True)
    for causal in (True, False):
        out = lib.prompt_attn(q, k, k, 0.1, causal, lse=lse, workspace=ws)
        grads = lib.prompt_attn_grad(q, k, k, out, lse, q, 0.1, causal, workspace=back)
        assert all(torch.isfinite(x).all() for x in (out, *grads))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
def test_long_keys_and_many_rows(cuda_device, dtype, causal):
    """Rows enough to fill the card and keys enough for the form of two blocks of rows a
    wave: a few rows of each head over long keys, and tiles that end anywhere."""
    c = Case(dtype, 128, 64, 64, t=[4, 257, 1], n=[3100, 3000, 3000], causal=causal, seed=21)
    out, L = c.forward(cuda_device)
    rows = [0, 3, 4, 5, 67, 68, 130, 200, 260, 261]
    heads = [0, 31, 63]
    q, k, v = c.q[rows][:, heads], c.k[:, heads], c.v[:, heads]
    for j, r in enumerate(rows):
        b = next(i for i in range(3) if c.rs[i] <= r < c.rs[i + 1])
        t, n = c.t[b], c.n[b]
        seen = (r - c.rs[b]) + n - t + 1 if causal else n
        at = slice(c.ks[b], c.ks[b] + seen)
        sub = ref.Batch(1, seen, T=1, N=seen, B=1, causal=False)
        o, lse, mass, spread, seen_n, top = ref.attention(q[j:j + 1], k[at], v[at], c.scale, sub)
        tol = ref.tolerance(o, mass, spread, seen_n, top, c.type, 128)
        err = np.abs(out[r, heads].double().cpu().numpy() - o[0])
        assert (err <= tol[0]).all(), (r, float((err / tol[0]).max()))
        err = np.abs(L[r, heads].double().cpu().numpy() - lse[0])
        assert (err <= ref.lse_tolerance(lse, spread, seen_n, 128)[0]).all(), r


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_long_keys_that_are_not_seen_stay_out(cuda_device, bad):
    """The same form: a value that is not finite in a tile that only some rows see."""
    c = Case("bf16", 128, 64, 64, t=[300, 260], n=[2300, 2200], seed=22, behind=0)
    clean, L = c.forward(cuda_device)
    again, _ = c.forward(cuda_device, lse=False)
    assert torch.equal(clean, again)
    at = 2300 - 40                              # of the first sequence: rows from 260 on see it
    c.v[at, 5, 7] = bad
    out, L2 = c.forward(cuda_device)
    assert torch.equal(L, L2)
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[260:300, 5, 7] = False
    assert not torch.isfinite(out[260:300, 5, 7]).any()
    # rows of tiles that are left out are summed in another order
    assert torch.isfinite(out[keep]).all()
    room = 4 * ref.half_step(c.type) * float(c.v[torch.isfinite(c.v)].abs().max())
    assert float((out - clean)[keep].abs().max()) <= room
    assert torch.equal(out[300:], clean[300:]) and torch.equal(out[:, 6:], clean[:, 6:])


@pytest.mark.parametrize("scale", [-0.3, 40.0])
def test_long_keys_whose_scores_rise(cuda_device, scale):
    """The same form where the largest score lies far behind: every tile's is higher than
    the last one's by more than what is let pass."""
    c = Case("bf16", 128, 64, 64, t=[256, 1, 1, 1], n=[2300] * 4, causal=False, seed=23, behind=0)
    c.k[:2300, :, 0] = torch.linspace(-20, 20, 2300)[:, None] * (-1 if scale < 0 else 1)
    c.q[:, :, 0] = 3.0
    c.scale = scale / 11.3
    out, L = c.forward(cuda_device)
    heads, rows = [0, 40], [0, 100, 255]
    sub = ref.Batch(3, 2300, T=3, N=2300, B=1, causal=False)
    o, lse, mass, spread, seen_n, top = ref.attention(
        c.q[rows][:, heads], c.k[:2300, heads], c.v[:2300, heads], c.scale, sub)
    tol = ref.tolerance(o, mass, spread, seen_n, top, c.type, 128)
    err = np.abs(out[rows][:, heads].double().cpu().numpy() - o)
    assert (err <= tol).all(), float((err / tol).max())
    err = np.abs(L[rows][:, heads].double().cpu().numpy() - lse)
    assert (err <= ref.lse_tolerance(lse, spread, seen_n, 128)).all()


# --- the binding -------------------------------------------------------------------------

def test_calls_give_the_same_bits_without_the_extension(cuda_device, monkeypatch):
    from paper_2607_19456_amd import binding

    c = Case("bf16", 64, 4, 2, t=[40, 33], behind=0, seed=24)
    x = [y.to(cuda_device) for y in (c.q, c.k, c.v, c.g)]
    start = torch.from_numpy(c.rs).to(cuda_device)
    table = lib.rotary_table(100, 64)
    pos = torch.randint(0, 100, (2, c.rows), dtype=torch.int32, device=cuda_device)

    def steps():
        got = []
        for p in (dict(row_start=start, T=40), dict(row_start=start, T=40, key_start=start, N=40),
                  dict(), dict(causal=False, key_start=start[[0, 2]].contiguous(), N=73)):
            ws = [lib.prompt_workspace(*x[:2], grad=g,
                                       **{k: v for k, v in p.items() if k != "causal"})
                  for g in (False, True)]
            lse = torch.empty(c.rows, 4, device=cuda_device)
            out = lib.prompt_attn(*x[:3], c.scale, lse=lse, workspace=ws[0], **p)
            got += [out, lse, *lib.prompt_attn_grad(*x[:3], out, lse, x[3], c.scale,
                                                    workspace=ws[1], **p)]
        got += lib.rotary_axes(x[0], pos, table, [16, 16], k=x[1])
        got += lib.rotary_axes(x[0], pos, table, (0, 32), k=x[1], interleaved=True, inverse=True)
        return got

    assert binding._call is not None
    first = steps()
    monkeypatch.setattr(binding, "_call", None)
    for a, b in zip(first, steps()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("extension", [True, False])
def test_tensors_that_are_refused(cuda_device, monkeypatch, extension):
    from paper_2607_19456_amd import binding

    if not extension:
        monkeypatch.setattr(binding, "_call", None)
    q = torch.randn(6, 4, 64, device=cuda_device)
    k = torch.randn(6, 2, 64, device=cuda_device)
    lse, ws = torch.empty(6, 4, device=cuda_device), None
    start = torch.tensor([0, 6], dtype=torch.int32, device=cuda_device)
    ws = lib.prompt_workspace(q, k)
    wg = lib.prompt_workspace(q, k, grad=True)
    heads = torch.randn(4, 6, 64, device=cuda_device).transpose(0, 1)

    def attn(q=q, k=k, v=k, **kw):
        return lib.prompt_attn(q, k, v, 0.1, **{"workspace": ws, **kw})

    def grad(q=q, k=k, v=k, out=q, lse=lse, g=q, **kw):
        return lib.prompt_attn_grad(q, k, v, out, lse, g, 0.1, **{"workspace": wg, **kw})

    for call in (lambda: attn(v=k.bfloat16()), lambda: attn(v=k.cpu()), lambda: attn(lse=lse.half()),
                 lambda: attn(row_start=start.long(), T=6), lambda: attn(workspace=ws.float()),
                 lambda: grad(g=q.half()), lambda: grad(dk=k.cpu()), lambda: grad(lse=lse.double())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: attn(q=heads), lambda: attn(v=k[:5]), lambda: attn(v=k[:, :1]),
                 lambda: attn(out=q[:, :2].contiguous()), lambda: attn(out=heads),
                 lambda: attn(lse=lse.t()), lambda: attn(lse=lse[:5]),
                 lambda: attn(row_start=start), lambda: attn(row_start=start[:1], T=6),
                 lambda: attn(T=4), lambda: attn(T=-1), lambda: attn(T=3, N=2),
                 lambda: attn(row_start=start, T=6, key_start=start[[0, 0, 1]].contiguous(), N=6),
                 lambda: grad(g=q[:, :2]), lambda: grad(dq=q[:, :2]), lambda: grad(dv=heads)):
        with pytest.raises(ValueError):
            call()
    many = torch.randn(5000, 2, 64, device=cuda_device)     # read in parts
    for call in (lambda: attn(k=many, v=many, workspace=ws[:3]), lambda: grad(workspace=wg[:40]),
                 lambda: attn(q=torch.randn(6, 3, 64, device=cuda_device)),
                 lambda: attn(q=torch.randn(6, 4, 80, device=cuda_device),
                              k=torch.randn(6, 2, 80, device=cuda_device),
                              v=torch.randn(6, 2, 80, device=cuda_device))):
        with pytest.raises((lib.DecodeAttnError, ValueError)):
            call()
    table, pos = lib.rotary_table(9, 64), torch.zeros(2, 6, dtype=torch.int32, device=cuda_device)
    for call in (lambda: lib.rotary_axes(q, pos.long(), table, (16, 16)),
                 lambda: lib.rotary_axes(q, pos, table.half(), (16, 16)),
                 lambda: lib.rotary_axes(q, pos, table, (16, 16), k=k.half())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: lib.rotary_axes(q, pos, table, (32,)),
                 lambda: lib.rotary_axes(q, pos, table, ()),
                 lambda: lib.rotary_axes(heads, pos, table, (16, 16)),
                 lambda: lib.rotary_axes(q, pos, table, (16, 16), k=k[:5])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lib.DecodeAttnError):
        lib.rotary_axes(q, pos, table, (16, 17))
