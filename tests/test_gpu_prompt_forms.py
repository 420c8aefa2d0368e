"""Attention over packed prompts and its gradient on the GPU: the forms that long
sequences, wide heads and divided tiles take, and what of them an infinity or a NaN
reaches, against the plain 64-bit forms of prompt_reference.py."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19456_amd as lib
import prompt_reference as ref
from test_gpu_prompt import Case, check_forward, check_gradient, compare, say

pytestmark = pytest.mark.gpu


class Hidden(ref.Batch):
    """A batch some of whose pairs are taken out: hide(sequence's number, seen)."""

    def __init__(self, batch, hide):
        self.__dict__.update(batch.__dict__)
        self.hide = hide

    def __iter__(self):
        for b, (rows, keys, seen) in enumerate(ref.Batch.__iter__(self)):
            yield rows, keys, self.hide(b, seen.copy())


def plain(q, k, v, scale, seen):
    """ref.attention's results for finite numbers and one head, q [t][d], k and v [n][d]."""
    s, size = ref.scores(q, k, seen, scale)
    top = np.maximum(s.max(1, keepdims=True), -1e300)
    w = np.exp(s - top)
    z = w.sum(1, keepdims=True)
    some = np.where(z > 0, z, 1.0)
    return ((w @ v) / some, (top + np.log(np.where(z > 0, z, 0.0)))[:, 0], (w @ np.abs(v)) / some,
            size.max(1), seen.sum(1))


def check_heads(c, out, lse, heads):
    """Every row of these query heads."""
    G, mine = c.h_q // c.h_kv, c.batch.mine("q")
    for h in heads:
        q, k, v = (x[:, i].double().numpy() for x, i in ((c.q, h), (c.k, h // G), (c.v, h // G)))
        o, mass = np.zeros((c.rows, 1, c.d)), np.zeros((c.rows, 1, c.d))
        L, spread = np.full((c.rows, 1), -np.inf), np.zeros((c.rows, 1))
        n = np.zeros(c.rows, np.int64)
        for rows, keys, seen in c.batch:
            with np.errstate(divide="ignore"):
                o[rows, 0], L[rows, 0], mass[rows, 0], spread[rows, 0], n[rows] = plain(
                    q[rows], k[keys], v[keys], c.scale, seen)
        top = np.nanmax(np.abs(v))
        compare(f"out of head {h}", out[:, h:h + 1], o,
                ref.tolerance(o, mass, spread, n, top, c.type, c.d), mine)
        compare("lse", lse[:, h:h + 1], L, ref.lse_tolerance(L, spread, n, c.d), mine)


def of_group(c, head):
    """What a KV head and its query heads have of a case: (q, k, v, g), slices."""
    G = c.h_q // c.h_kv
    mine = slice(G * head, G * head + G), slice(head, head + 1)
    return (c.q[:, mine[0]], c.k[:, mine[1]], c.v[:, mine[1]], c.g[:, mine[0]]), mine


def check_group_gradient(c, out, lse, grads, head):
    (q, k, v, g), (wide, one) = of_group(c, head)
    want, tol = ref.gradient(q, k, v, out[:, wide], lse[:, wide], g, c.scale, c.batch)
    for name, x, w, b, which in zip(("dq", "dk", "dv"), (grads[0][:, wide], grads[1][:, one],
                                                         grads[2][:, one]), want, tol, "qkk"):
        compare(f"{name} of KV head {head}", x, w, b, c.batch.mine(which))


# --- long sequences -----------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("h_q,h_kv,t,n,causal", [
    (4, 2, [1553], [1700], True), (6, 2, [1511, 1601], [1511, 1601], True),
    (3, 1, [70, 129], [1600, 1531], False), (4, 1, [1], [1999], True)])
def test_gradient_of_long_sequences_of_64(cuda_device, dtype, h_q, h_kv, t, n, causal):
    """From 1500 keys on, heads of 64 have two blocks of rows a wave in dQ, 64 keys a tile:
    lengths that are no multiples of either, groups of 2, 3 and 4, rows and keys in parts."""
    check_gradient(Case(dtype, 64, h_q, h_kv, t=t, n=n, causal=causal, seed=len(t)), cuda_device)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
def test_gradient_of_long_sequences_of_64_whole(cuda_device, dtype, causal):
    """The same, with as many tiles as compute units, so that none is divided."""
    c = Case(dtype, 64, 40, 20, t=[1653, 70], n=[1600, 1531], causal=causal, seed=30)
    out, lse = c.forward(cuda_device)
    grads = c.backward(cuda_device, out, lse)
    for head in (0, 11, 19):
        check_group_gradient(c, out, lse, grads, head)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
def test_long_keys_of_grouped_heads(cuda_device, dtype, causal):
    """The forward form of two blocks of rows a wave with four heads a group: every row of
    three groups, over sequences whose tiles end anywhere."""
    c = Case(dtype, 128, 32, 8, t=[1500, 611], n=[2200, 2101], causal=causal, seed=31)
    out, lse = c.forward(cuda_device)
    check_heads(c, out, lse, [0, 1, 2, 3, 20, 21, 22, 23, 28, 29, 30, 31])


# --- values that are not finite -------------------------------------------------------

FORMS = [("f32", 64), ("bf16", 64), ("f16", 128), ("bf16", 256), ("f32", 256)]


@pytest.mark.parametrize("dtype,d", FORMS + [("f32", 128), ("bf16", 128)])
@pytest.mark.parametrize("which", ["k", "v", "q", "g"])
def test_nan_stays_out_where_tiles_are_divided(cuda_device, dtype, d, which):
    """Rows and keys in two parts each, whose pairs left out are added to the parts' sums;
    float32 of d = 256, which has no room for zeros beside its tiles."""
    c = Case(dtype, d, 4, 2, t=[300], n=[530], seed=32)
    x = getattr(c, which)
    x[250 if which in "qg" else 525, 1, 3] = math.nan
    x[10 if which in "qg" else 244, 0, d - 1] = math.nan
    with np.errstate(invalid="ignore", over="ignore"):
        check_forward(c, cuda_device)
        check_gradient(c, cuda_device)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("which", ["k", "v", "q", "g"])
def test_nan_stays_out_of_long_sequences_of_64(cuda_device, dtype, which):
    """The form of two blocks of rows a wave, in parts."""
    c = Case(dtype, 64, 2, 1, t=[200], n=[1601], seed=33)
    getattr(c, which)[130 if which in "qg" else 1590, 0, 3] = math.nan
    with np.errstate(invalid="ignore", over="ignore"):
        check_gradient(c, cuda_device)


def test_nan_stays_out_of_long_sequences_of_64_whole(cuda_device):
    """And whole."""
    for which in "kqg":
        c = Case("bf16", 64, 40, 20, t=[1653, 70], n=[1600, 1531], seed=34)
        getattr(c, which)[1000, 1 if which == "k" else 2, 3] = math.nan
        out, lse = c.forward(cuda_device)
        grads = c.backward(cuda_device, out, lse)
        with np.errstate(invalid="ignore", over="ignore"):
            for head in (0, 1):
                check_group_gradient(c, out, lse, grads, head)


@pytest.mark.parametrize("t,n", [([100, 41], [130, 41]), ([300], [530])])
@pytest.mark.parametrize("dtype,d", FORMS)
@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("which", ["k above", "k below", "q", "v"])
def test_infinities_reach_what_sees_them(cuda_device, dtype, d, bad, which, t, n):
    """An infinity in the first KV head, or in its rows, whole and in parts.  Scores of
    +infinity, or of either sign, make NaN of the row, and of dk and dv of the keys that it
    sees; a score of -infinity is a weight of 0: the pair is as if it were not there, but
    that 0 times the infinity is NaN in that dimension of dq.  An infinity in v leaves dv as
    it was; dq of rows that see it and dk of what they see are not finite.  All else is what
    it was without."""
    c = Case(dtype, d, 4, 2, t=t, n=n, seed=35)
    key, row, dim = n[0] - 5, t[0] - 40, 5
    sign = math.copysign(1.0, bad)
    if which[0] == "k":
        # every row of the group has the sign that makes the score's
        c.q[:, :2, dim] = c.q[:, :2, dim].abs() * (sign if which == "k above" else -sign)
    clean = [x.clone() for x in (c.q, c.k, c.v)]
    out0, lse0 = c.forward(cuda_device)
    if which == "q":
        c.q[row, :2, dim] = bad
    elif which == "v":
        c.v[key, 0, dim] = bad
    else:
        c.k[key, 0, dim] = bad
    out, lse = c.forward(cuda_device)
    grads = c.backward(cuda_device, out, lse)

    (_, _, seen), *_ = c.batch
    sees = np.zeros(c.rows, bool)               # rows that see it
    if which == "q":
        sees[row] = True
    else:
        sees[:t[0]] = seen[:, key]
    assert sees.any() and not sees[:t[0]].all()
    seen_by_them = np.zeros(c.keys, bool)       # keys that these see
    seen_by_them[:n[0]] = seen[sees[:t[0]]].any(0)
    mine_q, mine_k = c.batch.mine("q"), c.batch.mine("k")

    def hide(b, seen):
        if b == 0 and which == "k below":
            seen[:, key] = False
        elif b == 0:
            seen[sees[:t[0]]] = False
        return seen

    batch = Hidden(c.batch, hide)
    c.q, c.k, c.v = clean
    for head in (0, 1):
        (q, k, v, g), (wide, one) = of_group(c, head)
        o, L, mass, spread, n_seen, top = ref.attention(q, k, v, c.scale,
                                                        batch if head == 0 else c.batch)
        tol = ref.tolerance(o, mass, spread, n_seen, top, c.type, d)
        tol_L = ref.lse_tolerance(np.where(np.isfinite(L), L, 0.0), spread, n_seen, d)
        got, got_L = out[:, wide].clone(), lse[:, wide].clone()
        # (the gradient's own reference takes out and lse as they are, or as they were
        # where the row is left out of it)
        use, use_L = out[:, wide].clone(), lse[:, wide].clone()
        skip = np.zeros(c.rows, bool)
        if head == 0 and which != "k below":
            skip = sees
            use[sees], use_L[sees] = out0[sees][:, wide], lse0[sees][:, wide]
            if which == "v":
                assert not torch.isfinite(got[sees][..., dim]).any()
                o[sees], tol[sees] = out0[sees][:, wide].double().cpu().numpy(), 0.0
                got[sees, :, dim] = out0[sees][:, wide][..., dim]
                # (the pairs of its tile may be added in another order)
                tol[sees] = 4 * ref.half_step(c.type) * top + 1e-6
                assert torch.equal(got_L[:sum(t)], lse0[:sum(t), wide])
                L[sees], tol_L[sees] = lse0[sees][:, wide].double().cpu().numpy(), 1.0
            else:
                assert torch.isnan(got[sees]).all() and torch.isnan(got_L[sees]).all()
                got[sees], o[sees] = 0.0, 0.0
                got_L[sees], L[sees] = 0.0, 0.0
        compare(f"out of KV head {head}", got, o, tol, mine_q)
        compare("lse", got_L, L, tol_L, mine_q)

        want, tol = ref.gradient(q, k, v, use, use_L, g, c.scale, batch if head == 0 else c.batch)
        dq, dk, dv = (x[:, y].clone() for x, y in zip(grads, (wide, one, one)))
        if head == 0 and which == "k below":
            assert torch.isnan(dq[sees][..., dim]).all()
            dq[sees, :, dim] = torch.from_numpy(want[0][sees, :, dim]).to(dq)
        elif head == 0:
            for x in [dk] + ([dv] if which != "v" else []):
                assert not torch.isfinite(x[seen_by_them]).any()
                x[seen_by_them] = 0.0
            assert not torch.isfinite(dq[sees]).any()
            dq[sees] = 0.0
            want[0][sees] = 0.0
            want[1][seen_by_them] = 0.0
            if which == "v":
                full, full_tol = ref.gradient(q, k, v, use, use_L, g, c.scale, c.batch)
                want, tol = (*want[:2], full[2]), (*tol[:2], full_tol[2])
            else:
                want[2][seen_by_them] = 0.0
        compare(f"dq of KV head {head}", dq, want[0], tol[0], mine_q)
        compare("dk", dk, want[1], tol[1], mine_k)
        compare("dv", dv, want[2], tol[2], mine_k)
        say(f"  {int(skip.sum())} rows, {int(seen_by_them.sum())} keys reached")


# --- the operators as a program uses them ---------------------------------------------

def turned_bound(bound, pos, table, sections):
    """What a bound of the values before a rotation back is after it: each of a pair's
    values is a sum of both, times a cosine and a sine."""
    half = table.shape[1] // 2
    axis = np.repeat(np.arange(len(sections)), sections)
    at = pos.numpy().astype(np.int64)[axis].T               # [row][pair]
    pair = np.arange(half)
    c, s = (np.abs(table.double().numpy()[at, x])[:, None] for x in (pair, half + pair))
    a, b = bound[..., :half], bound[..., half:]
    return np.concatenate((a * c + b * s, b * c + a * s), -1)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("h_q,h_kv,d,t", [(4, 2, 64, [40, 23]), (8, 2, 128, [130])])
def test_a_training_step_value_by_value(cuda_device, dtype, h_q, h_kv, d, t):
    """Turn q and k, attend, the gradient, turned back, each step against its 64-bit form of
    what the step before gave: dq and dk within the gradient's bound as the rotation passes it
    on, and the rotation's own.  A twentieth more of either would be found in most values."""
    c = Case(dtype, d, h_q, h_kv, t=t, behind=0, seed=36)
    sec, rows = (d // 8, d // 8 + 3, d // 4 - 3), sum(t)
    rng = np.random.default_rng(37)
    pos = torch.from_numpy(rng.integers(0, 300, (3, rows)).astype(np.int32))
    table = lib.rotary_table(300, d, device="cpu")
    a = (pos.to(cuda_device), table.to(cuda_device), sec)
    qt, kt = lib.rotary_axes(c.q.to(cuda_device), *a, k=c.k.to(cuda_device))
    for got, x in ((qt, c.q), (kt, c.k)):
        want, tol = ref.rotate(x, pos, table, sec, False, False)
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    c.q, c.k = qt.cpu(), kt.cpu()
    out, lse = check_forward(c, cuda_device)
    dqt, dkt, dv = c.backward(cuda_device, out, lse)
    dq, dk = lib.rotary_axes(dqt, *a, k=dkt, inverse=True)
    want, tol = ref.gradient(c.q, c.k, c.v, out, lse, c.g, c.scale, c.batch)
    compare("dv", dv, want[2], tol[2], np.ones(rows, bool))
    for name, got, before, w, b in (("dq", dq, dqt, want[0], tol[0]),
                                    ("dk", dk, dkt, want[1], tol[1])):
        # the rotation back of the 64-bit gradient, and the bound of rotating what was there
        back, _ = ref.rotate(torch.from_numpy(w), pos, table, sec, False, True)
        _, own = ref.rotate(before.cpu(), pos, table, sec, False, True)
        bound = turned_bound(b, pos, table, sec) + own
        compare(name, got, back, bound, np.ones(rows, bool))
        assert (np.abs(0.05 * back) > bound).mean() > 0.5


class Attention(torch.autograd.Function):
    """How a program that uses autograd has both calls."""

    @staticmethod
    def forward(ctx, q, k, v, scale, start, longest):
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
        out = lib.prompt_attn(q, k, v, scale, row_start=start, T=longest, lse=lse)
        ctx.save_for_backward(q, k, v, out, lse, start)
        ctx.scale, ctx.longest = scale, longest
        return out

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, out, lse, start = ctx.saved_tensors
        return (*lib.prompt_attn_grad(q, k, v, out, lse, d_out.contiguous(), ctx.scale,
                                      row_start=start, T=ctx.longest), None, None, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_in_a_program_that_uses_autograd(cuda_device, dtype):
    """The calls alone are not recorded; inside a function of autograd their gradient is, and
    reaches the projection's weights."""
    c = Case(dtype, 64, 4, 2, t=[50, 33], behind=0, seed=38)
    start = torch.from_numpy(c.rs).to(cuda_device)
    x = torch.randn(83, 64, device=cuda_device).to(c.type)
    w = (torch.randn(64, 8 * 64, device=cuda_device) / 8).to(c.type).requires_grad_()
    qkv = (x @ w).unflatten(1, (8, 64))
    q, k, v = qkv.split((4, 2, 2), 1)
    assert not lib.prompt_attn(q, k, v, c.scale, row_start=start, T=50).requires_grad
    out = Attention.apply(q, k, v, c.scale, start, 50)
    g = c.g.to(cuda_device)
    out.backward(g)
    with torch.no_grad():
        lse = torch.empty(83, 4, device=cuda_device)
        again = lib.prompt_attn(q, k, v, c.scale, row_start=start, T=50, lse=lse)
        d = lib.prompt_attn_grad(q, k, v, again, lse, g, c.scale, row_start=start, T=50)
        want = x.t() @ torch.cat(d, 1).flatten(1)
    assert torch.equal(out, again)
    # (the same product of the same numbers, which the library may add in another order:
    # 83 terms, and a rounding on either side)
    size = x.float().abs().t() @ torch.cat(d, 1).flatten(1).float().abs()
    assert ((w.grad.float() - want.float()).abs()
            <= 83 * 2 * ref.E32 * size + 2 * ref.half_step(c.type) * (want.float().abs() + 1e-6)).all()
