"""What the paged cache's entry points refuse, on the CPU: every call here fails
its checks before anything is enqueued, so no pointer is read."""
import math

import numpy as np
import pytest
import torch

import paged_reference as ref

binding = pytest.importorskip("paper_2607_19456_amd.binding",
                              reason="HIP library not built")
lib = binding._lib
FAKE = 0x10000          # 16-byte aligned, never read
OK, NULL, SHAPE, UNSUPPORTED, ALIGN, SCALE, WORKSPACE = range(7)
BIG = 1 << 40


def batch(**kw):
    f = dict(K=FAKE, V=FAKE, pages=FAKE, past=FAKE, row_start=None, B=2, h_kv=2, d=64, n_pages=5,
             page_rows=16, max_pages=4, rows=6, T=3, dtype=1, format=0)
    f.update(kw)
    for name in ("K", "V", "pages", "past", "row_start"):
        f[name] = f[name] or 0
    return binding._pack_kv(*f.values())


def append(kv=None, k=FAKE, v=FAKE, ks=128, vs=128, q=FAKE, qs=512, h_q=8, q_out=FAKE, rotary=FAKE,
           n=64, rot=64):
    return lib.da_paged_append(batch() if kv is None else kv, k, v, ks, vs, q, qs, h_q, q_out,
                               rotary, n, rot, 0, None)


def gather(kv=None, k=FAKE, v=FAKE):
    return lib.da_paged_gather(batch() if kv is None else kv, k, v, None)


def attn(kv=None, q=FAKE, qs=512, h_q=8, scale=0.1, out=FAKE, ws=FAKE, n=BIG):
    return lib.da_paged_attn(batch() if kv is None else kv, q, qs, h_q, scale, 1, out, ws, n, None)


@pytest.mark.parametrize("call", [append, gather, attn])
def test_batches_that_are_refused(call):
    for name in ("K", "V", "pages", "past"):
        assert call(batch(**{name: None})) == NULL
    for name in ("B", "h_kv", "d", "n_pages", "page_rows", "max_pages", "rows", "T"):
        assert call(batch(**{name: 0})) == SHAPE, name
        assert call(batch(**{name: -3})) == SHAPE, name
    assert call(batch(rows=7)) == SHAPE                         # not B*T
    assert call(batch(max_pages=(1 << 26) + 1)) == SHAPE        # 2^30 positions
    assert call(batch(T=32769, rows=65538)) == SHAPE
    assert call(batch(B=1 << 24, rows=3 << 24)) == SHAPE
    if call is not attn:                          # more workgroups than a grid holds
        assert call(batch(T=32768, rows=1 << 30, B=32768)) == SHAPE
    wide = {append: dict(ks=192, vs=192, qs=768), gather: {}, attn: dict(qs=768)}[call]
    assert call(batch(d=96), **wide) == UNSUPPORTED
    assert call(batch(page_rows=8)) == UNSUPPORTED
    assert call(batch(page_rows=24), **({"n": 96} if call is append else {})) == UNSUPPORTED
    for dtype in (-1, 3):
        assert call(batch(dtype=dtype)) == UNSUPPORTED
    for fmt in (-1, 2):
        assert call(batch(format=fmt)) == UNSUPPORTED
    for name, bad in (("K", FAKE + 8), ("V", FAKE + 4), ("pages", FAKE + 2), ("past", FAKE + 1),
                      ("row_start", FAKE + 2)):
        assert call(batch(**{name: bad})) == ALIGN, name


def test_append_refusals():
    assert append(k=None) == append(v=None) == append(q_out=None) == append(rotary=None) == NULL
    assert append(h_q=0) == append(h_q=-1) == SHAPE
    assert append(n=63) == SHAPE                  # the table ends before the pages
    assert append(rot=80) == append(rot=-16) == SHAPE
    assert append(ks=127) == append(vs=64) == append(qs=511) == SHAPE
    assert append(rot=24) == append(rot=8) == UNSUPPORTED
    assert append(ks=132) == append(vs=129) == append(qs=516) == ALIGN
    for name in ("k", "v", "q", "q_out", "rotary"):
        assert append(**{name: FAKE + 8}) == ALIGN, name


def test_gather_refusals():
    assert gather(k=None) == gather(v=None) == NULL
    assert gather(k=FAKE + 8) == gather(v=FAKE + 4) == ALIGN


def test_attn_refusals():
    assert attn(q=None) == attn(out=None) == NULL
    assert attn(h_q=0) == attn(h_q=7) == attn(h_q=-2) == attn(qs=511) == SHAPE
    assert attn(batch(B=3000, h_kv=1, rows=9000), h_q=8192, qs=8192 * 64) == SHAPE
    assert attn(qs=516) == attn(q=FAKE + 8) == attn(out=FAKE + 4) == ALIGN
    for bad in (math.nan, math.inf, -math.inf):
        assert attn(scale=bad) == SCALE
    need = lib.da_paged_workspace_bytes(2, 8, 2, 64, 3, 1)
    assert need > 0
    assert attn(ws=None) == attn(n=0) == attn(n=need - 1) == WORKSPACE
    assert attn(ws=FAKE + 8) == ALIGN


def test_sizes():
    assert lib.da_paged_page_bytes(16, 128, 1, 0) == 4096
    assert lib.da_paged_page_bytes(16, 128, 0, 0) == 8192
    assert lib.da_paged_page_bytes(64, 64, 2, 1) == 64 * 34
    for bad in ((8, 64, 0, 0), (24, 64, 0, 0), (65536, 64, 0, 0), (16, 96, 0, 0), (16, 64, 3, 0),
                (16, 64, 0, 2)):
        assert lib.da_paged_page_bytes(*bad) == 0, bad
    size = lib.da_paged_workspace_bytes
    for h_q, h_kv, d, T in ((8, 2, 64, 1), (64, 8, 128, 4), (16, 16, 256, 2048)):
        before = 0
        for B in (1, 2, 7, 300, 4000):
            n = size(B, h_q, h_kv, d, T, 1)
            assert 0 < lib.da_paged_workspace_counter_bytes(B, h_q, h_kv, d, T, 1) < n
            assert n >= before > -1 and n > 0
            before = n
    for bad in ((0, 8, 2, 64, 1, 0), (1, 8, 3, 64, 1, 0), (1, 8, 2, 80, 1, 0),
                (1, 8, 2, 64, 0, 0), (1, 8, 2, 64, 32769, 0), (1, 8, 2, 64, 1, 7)):
        assert size(*bad) == lib.da_paged_workspace_counter_bytes(*bad) == 0, bad


def test_binding_refuses_tensors_that_are_not_on_the_gpu_or_do_not_fit():
    K = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    pages, past = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q = torch.zeros(1, 8, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        binding.paged_attn(q, K, K, pages, past, 0.1)
    with pytest.raises(ValueError):
        binding.paged_attn(q[0], K, K, pages, past, 0.1)
    with pytest.raises(ValueError):
        binding.paged_attn(torch.zeros(1, 8, 128, dtype=torch.bfloat16), K, K, pages, past, 0.1)
    with pytest.raises(TypeError):
        binding.paged_attn(q.double(), K, K, pages, past, 0.1)
    with pytest.raises(ValueError):
        binding.paged_append(K, K, pages, past, q[0], q[0])
    with pytest.raises(ValueError):
        binding.paged_alloc(4, 12, 2, 64, device="cpu")
    with pytest.raises(ValueError):
        binding.paged_alloc(4, 16, 2, 64, format="fp8", device="cpu")
    with pytest.raises(TypeError):
        binding.paged_alloc(4, 16, 2, 64, dtype=torch.float64, device="cpu")


def test_workspaces_that_are_refused():
    K, _ = binding.paged_alloc(4, 16, 2, 64, device="cpu")
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    for rows, sequences, t in ((q, 0, None), (q, 5, None), (q, 3, torch.float64)):
        pages = torch.zeros(sequences, 2, dtype=torch.int32)
        with pytest.raises(binding.DecodeAttnError):
            binding.paged_workspace(rows.to(t) if t else rows, K, pages)
    assert binding.paged_workspace_bytes(1, 4, 2, 64, 1, torch.int8) == 0
    assert binding.paged_workspace_counter_bytes(1, 4, 2, 64, 1, torch.int8) == 0


def test_pools_have_the_size_that_the_library_names():
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for fmt in ("dense", "mx4"):
            K, V = binding.paged_alloc(3, 32, 2, 128, dtype=dtype, format=fmt, device="cpu")
            n = 3 * 2 * lib.da_paged_page_bytes(32, 128, binding._DTYPES[dtype],
                                                int(fmt == "mx4"))
            assert K.numel() * K.element_size() == V.numel() * V.element_size() == n


def test_rotary_table():
    """Far positions: float32 angles would be off by whole turns' parts."""
    t = binding.rotary_table(100001, 64, base=10000.0, device="cpu")
    assert t.shape == (100001, 64) and t.dtype == torch.float32
    for pos in (0, 1, 99999, 100000):
        for i in (0, 1, 31):
            a = pos * 10000.0 ** (-2.0 * i / 64)
            assert abs(float(t[pos, i]) - math.cos(a)) <= 1e-7
            assert abs(float(t[pos, 32 + i]) - math.sin(a)) <= 1e-7


# --- the reference itself -----------------------------------------------------------

def test_reference_quantiser_on_worked_values():
    """A block whose largest value is 5: 2^X = 1; ties go to the even code."""
    x = np.zeros(32)
    x[:8] = [5.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -0.26]
    codes, scales = ref.quantise(x)
    assert scales.tolist() == [127]
    assert codes[:8].tolist() == [6, 0, 2, 2, 4, 4, 6, 9]
    assert ref.values(codes, scales)[:8].tolist() == [4, 0, 1, 1, 2, 2, 4, -0.5]
    # the largest value's place in its power of two: 4 <= top / 2^X < 8
    for top in (4.0, 7.999, 8.0, 1e-3, 3e38):
        c, s = ref.quantise(np.full(32, top))
        assert 4 <= top / 2.0 ** (int(s[0]) - 127) < 8
    assert ref.quantise(np.zeros(32))[1].tolist() == [1]
    assert ref.quantise(np.r_[np.inf, np.zeros(31)])[1].tolist() == [255]


def test_reference_pages_are_the_documented_bytes():
    rng = np.random.default_rng(0)
    P, d = 32, 64
    codes = rng.integers(0, 16, (P, d)).astype(np.uint8)
    scales = rng.integers(1, 255, (P, d // 32)).astype(np.uint8)
    k, v = ref.pack_page(codes, scales, False), ref.pack_page(codes, scales, True)
    assert len(k) == len(v) == P * (d // 2 + d // 32)
    for row, dim in ((0, 0), (5, 7), (31, 63), (16, 33)):
        at = row * d // 2 + dim // 2
        assert k[at] >> 4 * (dim % 2) & 15 == codes[row, dim]
        at = (row // 8) * 4 * d + dim // 8 * 32 + row % 8 * 4 + dim % 8 // 2
        assert v[at] >> 4 * (dim % 2) & 15 == codes[row, dim]
        assert k[P * d // 2 + row * (d // 32) + dim // 32] == scales[row, dim // 32]
        assert v[P * d // 2 + (row // 8) * (d // 4) + dim // 32 * 8 + row % 8] \
            == scales[row, dim // 32]
    for value in (False, True):
        c, s = ref.unpack_page(ref.pack_page(codes, scales, value), P, d, value)
        assert np.array_equal(c, codes) and np.array_equal(s, scales)
