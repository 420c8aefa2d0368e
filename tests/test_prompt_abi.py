"""What prompt attention, its gradient and the rotation by several axes refuse, on
the CPU: every call here fails its checks before anything is enqueued, so no pointer is
read."""
import math

import pytest
import torch

import prompt_reference as ref

binding = pytest.importorskip("paper_2607_19456_amd.binding",
                              reason="HIP library not built")
lib = binding._lib
FAKE = 0x10000          # 16-byte aligned, never read
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, SCALE, WORKSPACE = range(7)
BIG = 1 << 60


def batch(**kw):
    f = dict(row_start=None, key_start=None, B=2, h_q=8, h_kv=2, d=64, rows=6, keys=10, T=3, N=5,
             dtype=1, causal=1)
    f.update(kw)
    for name in ("row_start", "key_start"):
        f[name] = f[name] or 0
    return binding._pack_prompt(*f.values())


def attn(p=None, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128, scale=0.1, out=FAKE, lse=FAKE,
         ws=FAKE, n=BIG):
    return lib.da_prompt_attn(batch() if p is None else p, q, qs, k, ks, v, vs, scale, out, lse, ws,
                              n, None)


def grad(p=None, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128, scale=0.1, out=FAKE, lse=FAKE,
         g=FAKE, gs=512, dq=FAKE, dqs=512, dk=FAKE, dks=128, dv=FAKE, dvs=128, ws=FAKE, n=BIG):
    return lib.da_prompt_attn_grad(batch() if p is None else p, q, qs, k, ks, v, vs, out, lse, g,
                                   gs, scale, dq, dqs, dk, dks, dv, dvs, ws, n, None)


@pytest.mark.parametrize("call", [attn, grad])
def test_batches_that_are_refused(call):
    assert lib.da_prompt_attn(None, *[FAKE, 512] * 3, 0.1, FAKE, None, FAKE, BIG, None) == NULL
    for name in ("B", "h_q", "h_kv", "d", "rows", "keys", "T", "N"):
        for bad in (0, -3):
            assert call(batch(**{name: bad})) == SHAPE, name
    assert call(batch(h_q=9)) == SHAPE                          # h_kv does not divide it
    assert call(batch(rows=7)) == call(batch(keys=9)) == SHAPE  # not B*T, not B*N
    assert call(batch(T=(1 << 28) + 1, rows=6, row_start=FAKE)) == SHAPE
    assert call(batch(N=(1 << 30) + 1, key_start=FAKE)) == SHAPE
    assert call(batch(B=1 << 22, row_start=FAKE, key_start=FAKE)) == SHAPE
    # more workgroups than a grid holds
    many = batch(B=1 << 15, h_q=512, h_kv=512, rows=1 << 30, keys=1 << 30, T=1 << 15, N=1 << 15)
    wide = dict(qs=1 << 15, ks=1 << 15, vs=1 << 15)
    if call is grad:
        wide.update(gs=1 << 15, dqs=1 << 15, dks=1 << 15, dvs=1 << 15)
    assert call(many, **wide) == SHAPE
    wide = {name: 8 * 96 for name in wide}
    assert call(batch(d=96), **wide) == UNSUPPORTED
    for dtype in (-1, 3):
        assert call(batch(dtype=dtype)) == UNSUPPORTED
    for name in ("row_start", "key_start"):
        assert call(batch(**{name: FAKE + 2})) == ALIGN


@pytest.mark.parametrize("call", [attn, grad])
def test_arguments_that_are_refused(call):
    names = ["q", "k", "v", "out"] + (["lse", "g", "dq", "dk", "dv"] if call is grad else [])
    for name in names:
        assert call(**{name: None}) == NULL, name
        assert call(**{name: FAKE + (2 if name == "lse" else 8)}) == ALIGN, name
    strides = ["qs", "ks", "vs"] + (["gs", "dqs", "dks", "dvs"] if call is grad else [])
    for name in strides:
        least = 512 if name in ("qs", "gs", "dqs") else 128
        assert call(**{name: least - 8}) == SHAPE, name
        assert call(**{name: least + 4}) == ALIGN, name
        assert call(**{name: -least}) == SHAPE, name
        assert call(**{name: (1 << 21) + 8}) == SHAPE, name        # more than 4 MiB
    for bad in (math.nan, math.inf, -math.inf):
        assert call(scale=bad) == SCALE
    size = lib.da_prompt_workspace_bytes if call is attn else lib.da_prompt_grad_workspace_bytes
    p = batch(N=5000, keys=10000)
    need = size(p)
    assert need > 16
    assert call(p, ws=None) == call(p, n=0) == call(p, n=need - 1) == WORKSPACE
    assert call(p, ws=FAKE + 8) == ALIGN


def test_sizes():
    for size in (lib.da_prompt_workspace_bytes, lib.da_prompt_grad_workspace_bytes):
        assert size(None) == size(batch(B=0)) == size(batch(d=80)) == size(batch(dtype=5)) == 0
        assert size(batch()) >= 16
    # a row's lse and delta
    assert lib.da_prompt_grad_workspace_bytes(batch()) >= 6 * 8 * 8


def rotary(rows=3, d=64, dtype=1, n=100, rot=64, axes=3, sections=(8, 12, 12, 0), pos=FAKE,
           table=FAKE, q=FAKE, qs=512, h_q=8, qo=FAKE, qos=512, k=FAKE, ks=128, h_kv=2, ko=FAKE,
           kos=128):
    p = binding._pack_rotary(pos or 0, table or 0, rows, d, dtype, n, rot, axes, *sections, 0, 0)
    return lib.da_rotary_axes(p, q, qs, h_q, qo, qos, k, ks, h_kv, ko, kos, None)


def test_rotary_refusals():
    for name in ("pos", "table", "q", "qo", "ko"):
        assert rotary(**{name: None}) == NULL, name
    for name in ("rows", "d", "n", "rot", "axes", "h_q", "h_kv"):
        for bad in (0, -1):
            assert rotary(**{name: bad}) == SHAPE, name
    assert rotary(axes=5) == SHAPE
    assert rotary(rot=80) == SHAPE                              # more than a head has
    for bad in ((8, 12, 11, 0), (8, 12, 13, 0), (-4, 18, 18, 0), (2 ** 31 - 1, 2 ** 31 - 1, 34, 0)):
        assert rotary(sections=bad) == SHAPE, bad
    for name, least in (("qs", 512), ("qos", 512), ("ks", 128), ("kos", 128)):
        assert rotary(**{name: least - 8}) == SHAPE, name
        assert rotary(**{name: least + 4}) == ALIGN, name
    assert rotary(d=96, qs=768, qos=768, ks=192, kos=192) == UNSUPPORTED
    assert rotary(rot=24, sections=(4, 4, 4, 0)) == UNSUPPORTED
    assert rotary(dtype=3) == rotary(dtype=-1) == UNSUPPORTED
    for name in ("q", "qo", "k", "ko", "table"):
        assert rotary(**{name: FAKE + 8}) == ALIGN, name
    assert rotary(pos=FAKE + 2) == ALIGN
    assert rotary(rows=1 << 30, k=None) == SHAPE                # more workgroups than a grid holds


def test_the_binding_refuses():
    q, k = torch.zeros(6, 8, 64), torch.zeros(6, 2, 64)
    for call in (lambda: binding.prompt_attn(q, k, k, 0.1),
                 lambda: binding.prompt_attn_grad(q, k, k, q, q[..., 0], q, 0.1),
                 lambda: binding.prompt_workspace(q, k),
                 lambda: binding.rotary_axes(q, torch.zeros(1, 6, dtype=torch.int32),
                                             torch.zeros(9, 64), (32,)),
                 lambda: binding.prompt_attn(q.double(), k, k, 0.1)):
        with pytest.raises(TypeError):                          # not on the GPU, not a type
            call()
    for call in (lambda: binding.prompt_attn(q[0], k, k, 0.1),
                 lambda: binding.prompt_attn(q, k[0], k, 0.1),
                 lambda: binding.rotary_axes(q[0], None, None, (32,))):
        with pytest.raises(ValueError):
            call()


# --- the reference itself -------------------------------------------------------------

def test_reference_on_a_worked_example():
    """Two keys with scores 0 and ln 3: weights 1/4 and 3/4."""
    k = torch.zeros(2, 1, 64)
    q = torch.zeros(1, 1, 64)
    q[0, 0, 0], k[1, 0, 0] = 1.0, math.log(3)
    v = torch.zeros(2, 1, 64)
    v[0, 0, 0], v[1, 0, 0] = 8.0, 4.0
    b = ref.Batch(1, 2, T=1, N=2, B=1)
    out, lse, *_ = ref.attention(q, k, v, 1.0, b)
    assert abs(out[0, 0, 0] - 5.0) < 1e-6 and abs(lse[0, 0] - math.log(4)) < 1e-7
    g = torch.zeros(1, 1, 64)
    g[0, 0, 0] = 1.0
    (dq, dk, dv), _ = ref.gradient(q, k, v, torch.from_numpy(out), torch.from_numpy(lse), g, 1.0, b)
    # dP = (8, 4), delta = 5: dS = (3/4, -3/4)
    assert abs(dq[0, 0, 0] + 0.75 * math.log(3)) < 1e-6
    assert abs(dk[0, 0, 0] - 0.75) < 1e-6 and abs(dk[1, 0, 0] + 0.75) < 1e-6
    assert abs(dv[0, 0, 0] - 0.25) < 1e-7 and abs(dv[1, 0, 0] - 0.75) < 1e-7


def test_reference_spans_and_what_rows_see():
    assert ref.spans([-5, 10, 4, 200], 3, 90, 90) == [(0, 10), (10, 0), (4, 86)]
    assert ref.spans(None, 2, 3, 6) == [(0, 3), (3, 3)]
    (_, _, seen), = ref.Batch(3, 2, T=3, N=2, B=1)
    assert seen.tolist() == [[False, False], [True, False], [True, True]]
    (_, _, seen), = ref.Batch(1, 3, T=1, N=3, B=1)
    assert seen.tolist() == [[True, True, True]]


def test_reference_rotation_is_a_turn():
    x = torch.randn(4, 2, 64, dtype=torch.float64).float()
    table = binding.rotary_table(50, 64, device="cpu")
    pos = torch.tensor([[0, 3, 7, 49], [1, 1, 0, 20]], dtype=torch.int32)
    for inter in (False, True):
        y, _ = ref.rotate(x, pos, table, (10, 22), inter, False)
        z, _ = ref.rotate(torch.from_numpy(y).float(), pos, table, (10, 22), inter, True)
        assert abs(z - x.double().numpy()).max() < 1e-5
    assert abs(y[0, :, :20] - x[0, :, :20].numpy()).max() < 1e-7    # position 0
