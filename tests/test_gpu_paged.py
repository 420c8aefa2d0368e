"""The paged cache on the GPU against the plain 64-bit forms of
paged_reference.py: attention over every type, head size, group and page size,
with places that no row may see poisoned; appends and read-backs bit for bit
where the definition has one answer; a step as a serving loop makes it."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19456_amd as lib
import paged_reference as ref

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def rows_of(counts, extra=0):
    start = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    return torch.from_numpy(start), int(start[-1]) + extra


def check_attn(device, *, dtype="bf16", fmt="dense", d=128, h_q=8, h_kv=2, P=16, past=(37,), T=1,
               counts=None, causal=True, seed=0, behind=0, cache=None, scale=None, wide=None,
               edit=None, q_scale=1.0, q=None):
    """One call against the reference; returns the output."""
    t = ref.DTYPES[dtype]
    n = counts if counts is not None else [T] * len(past)
    held = [p + (c if causal else 0) if p >= 0 else 0 for p, c in zip(past, n)]
    c = cache or ref.Cache(seed, dtype, fmt, d, h_kv, P, held, wide=wide)
    if edit:
        edit(c)
    row_start, N = rows_of(n, behind)
    rng = np.random.default_rng(seed + 1)
    if q is None:
        q = torch.from_numpy(rng.standard_normal((N, h_q, d)) * q_scale).to(t)
    scale = 1 / math.sqrt(d) if scale is None else scale
    past_t = torch.tensor(past, dtype=torch.int32)
    use_start = counts is not None
    K, V, pages = c.to(device)
    out = torch.full((N, h_q, d), math.nan, dtype=t, device=device)
    say(f"attn {dtype} {fmt} d={d} h={h_q}/{h_kv} P={P} past={past[:6]} rows={n[:6]} "
        f"causal={causal} seed={seed}")
    lib.paged_attn(q.to(device), K, V, pages, past_t.to(device), scale, causal=causal,
                   row_start=row_start.to(device) if use_start else None, T=T, out=out)
    torch.cuda.synchronize()
    want, mass, spread, seen, mine, top_v = ref.attention(
        q, c.K, c.V, c.pages.numpy(), past, scale, causal,
        row_start.numpy() if use_start else None, T, h_kv)
    got = out.cpu().double().numpy()
    assert np.isnan(got[~mine]).all(), "rows of no sequence were written"
    tol = ref.tolerance(want, mass, spread, seen, top_v, t, d)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(want)[mine], np.isnan(got)[mine])
    assert np.array_equal(got[mine & True][~fine[mine] & ~np.isnan(want[mine])],
                          want[mine][~fine[mine] & ~np.isnan(want[mine])])
    ok = fine & mine[:, None, None]
    err = np.abs(np.where(ok, got - want, 0.0))
    worst = np.max(err / np.where(ok, tol, 1.0)) if ok.any() else 0.0
    say(f"  max error {err.max():.3e}, {worst:.3f} of the bound")
    assert worst <= 1.0
    return out


TYPES = [(t, f) for t in ("f32", "bf16", "f16") for f in ("dense", "mx4")]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_attention_of_single_tokens(cuda_device, dtype, fmt, d):
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=d, past=[0, 1, 15, 16, 31, 127, 128, 300],
               seed=d)


@pytest.mark.parametrize("h_q,h_kv", [(1, 1), (3, 3), (5, 1), (16, 1), (17, 1), (32, 1), (40, 1),
                                      (64, 2), (15, 3)])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f16", "mx4"), ("f32", "dense")])
def test_attention_of_head_groups(cuda_device, dtype, fmt, h_q, h_kv):
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=64, h_q=h_q, h_kv=h_kv, past=[70, 9],
               seed=h_q)


@pytest.mark.parametrize("P", [16, 32, 64, 128, 1024])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("bf16", "mx4"), ("f32", "dense"),
                                       ("f32", "mx4")])
def test_attention_of_page_sizes(cuda_device, dtype, fmt, P):
    """Pages that end inside a tile, and tiles inside a page."""
    check_attn(cuda_device, dtype=dtype, fmt=fmt, P=P, past=[15, 16, 17, 47, 200, 1030], seed=P)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T", [2, 3, 5, 16, 33, 130])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f16", "dense"), ("f16", "mx4"),
                                       ("f32", "dense"), ("f32", "mx4")])
def test_attention_of_several_rows(cuda_device, dtype, fmt, T, causal):
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=64, h_q=6, h_kv=2, past=[0, 1, 61, 250], T=T,
               causal=causal, seed=T)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_attention_of_ragged_rows(cuda_device, dtype, fmt, d):
    """Sequences of no rows, of one, of many; rows behind the last sequence."""
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=d, h_q=8, h_kv=2, P=32,
               past=[5, 0, 100, 0, 64], T=70, counts=[1, 0, 70, 3, 17], behind=4, seed=d)


def test_rows_beyond_T_are_not_rows(cuda_device):
    """row_start holds 9 rows of a sequence that T allows 4 of."""
    q = torch.randn(9, 4, 64, dtype=torch.bfloat16)
    c = ref.Cache(1, "bf16", "dense", 64, 2, 16, [40])
    K, V, pages = c.to(cuda_device)
    out = torch.full((9, 4, 64), math.nan, dtype=torch.bfloat16, device=cuda_device)
    lib.paged_attn(q.to(cuda_device), K, V, pages,
                   torch.tensor([20], dtype=torch.int32, device=cuda_device), 0.125,
                   row_start=torch.tensor([0, 9], dtype=torch.int32, device=cuda_device), T=4,
                   out=out)
    got = out.cpu()
    assert torch.isfinite(got[:4]).all() and torch.isnan(got[4:]).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f32", "dense"), ("bf16", "mx4")])
def test_rows_that_see_nothing_are_zero(cuda_device, dtype, fmt, causal):
    """Negative and zero pasts beside others, and a batch of nothing else."""
    check_attn(cuda_device, dtype=dtype, fmt=fmt, past=[-1, 0, 40, -2 ** 31, 0], T=3,
               causal=causal, seed=4)
    check_attn(cuda_device, dtype=dtype, fmt=fmt, past=[-1, -7], T=2, causal=causal, seed=5)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("past", [[160], [158], [155, 1000], [2 ** 31 - 1]])
def test_rows_at_the_capacity(cuda_device, past, causal):
    """Positions beyond the table do not exist; its rows see what there is."""
    c = ref.Cache(3, "bf16", "dense", 64, 2, 16, [160] * len(past))
    check_attn(cuda_device, dtype="bf16", d=64, past=past, T=6, causal=causal, cache=c)


@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f32", "dense"), ("f16", "mx4")])
def test_missing_pages_are_not_seen(cuda_device, dtype, fmt, P):
    def edit(c):
        c.pages[0, 0] = -1
        c.pages[0, 3] = c.K.shape[0]
        c.pages[1, :] = -5
        c.pages[2, 1:3] = 2 ** 31 - 1
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=64, P=P, past=[6 * P + 3, 2 * P, 3 * P], T=4,
               edit=edit, seed=P)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_infinities_and_nan_stay_out_of_rows_that_do_not_see_them(cuda_device, dtype):
    """V and K rows of the step's later positions hold infinities and NaN: the
    earlier rows must not, the later ones must."""
    def edit(c):
        for pos, x in ((42, math.inf), (45, math.nan), (46, -math.inf)):
            page, slot = int(c.pages[0, pos // 16]), pos % 16
            c.V[page, 0, slot, 5] = x
            c.V[page, 1, slot, 40:44] = x
        page, slot = int(c.pages[0, 2]), 47 % 16
        c.K[page, 0, slot, 3] = math.nan
    check_attn(cuda_device, dtype=dtype, d=64, h_q=4, h_kv=2, past=[40], T=10, edit=edit, seed=8)
    check_attn(cuda_device, dtype=dtype, d=128, h_q=4, h_kv=2, past=[40], T=10, edit=edit, seed=8)


def test_a_block_of_nan_stays_out_of_rows_that_do_not_see_it(cuda_device):
    def edit(c):
        P, d = 16, 64
        for pos in (42, 45):
            page = int(c.pages[0, pos // P])
            codes, scales = ref.unpack_page(c.V[page, 0].reshape(-1).numpy(), P, d, True)
            scales = scales.copy()
            scales[pos % P, 1] = 255
            c.V[page, 0] = torch.from_numpy(ref.pack_page(codes, scales, True)).reshape(P, -1)
    for dtype in ("bf16", "f32"):
        check_attn(cuda_device, dtype=dtype, fmt="mx4", d=64, h_q=4, h_kv=2, past=[40], T=10,
                   edit=edit, seed=9)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f16", "dense"), ("f32", "dense"),
                                       ("bf16", "mx4")])
def test_scores_that_climb_and_fall(cuda_device, dtype, fmt):
    """Scores of some hundred units, the largest late or early, a negative scale, a
    scale of 0."""
    for scale in (2.0, -1.5, 0.0):
        check_attn(cuda_device, dtype=dtype, fmt=fmt, d=64, past=[900, 3], T=2, scale=scale,
                   seed=11)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f16", "mx4"), ("f32", "dense")])
@pytest.mark.parametrize("B,h_kv,past", [(1, 1, 20011), (2, 2, 9001), (1, 8, 3500)])
def test_long_sequences_are_divided(cuda_device, dtype, fmt, B, h_kv, past):
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=64, h_q=2 * h_kv, h_kv=h_kv, P=64,
               past=[past - 700 * b for b in range(B)], seed=past)


def test_many_sequences(cuda_device):
    """More sequences than a workgroup has threads, empty ones among them."""
    rng = np.random.default_rng(5)
    past = [int(x) for x in rng.integers(-1, 40, 700)]
    check_attn(cuda_device, d=64, h_q=2, h_kv=1, past=past, seed=6)
    counts = [int(x) for x in rng.integers(0, 3, 300)]
    check_attn(cuda_device, d=64, h_q=2, h_kv=1, past=past[:300], T=2, counts=counts, seed=7)


@pytest.mark.parametrize("B,past", [(2, [2999, 499]), (70, None)])
@pytest.mark.parametrize("dtype,T", [("bf16", 1), ("f16", 3), ("bf16", 40), ("f32", 9)])
def test_equal_calls_give_equal_bits(cuda_device, dtype, T, B, past):
    """Whatever the workspace holds behind its counters, which every call leaves
    zeroed; rows of many parts, put together by the merge, and of few, put
    together by the workgroup that finishes last."""
    past = past or [int(x) for x in np.random.default_rng(4).integers(0, 900, B)]
    c = ref.Cache(2, dtype, "dense", 64, 2, 64, [p + T for p in past])
    K, V, pages = c.to(cuda_device)
    q = torch.randn(B * T, 8, 64, device=cuda_device).to(ref.DTYPES[dtype])
    dpast = torch.tensor(past, dtype=torch.int32, device=cuda_device)
    ws = lib.paged_workspace(q, K, pages, T)
    n = lib.paged_workspace_counter_bytes(B, 8, 2, 64, T, q.dtype)
    assert 0 < n < ws.numel() and int(ws[:n].max()) == 0
    outs = []
    for fill in (0, 255, 127):
        ws[n:].fill_(fill)
        outs.append(lib.paged_attn(q, K, V, pages, dpast, 0.09, T=T, workspace=ws).clone())
        assert int(ws[:n].max()) == 0
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    check_attn(cuda_device, dtype=dtype, d=64, h_q=8, h_kv=2, P=64, past=past, T=T, cache=c,
               scale=0.09, q=q.cpu())


def test_the_last_to_finish_has_all_parts(cuda_device):
    """Many calls one after the other, each with new queries, the parts of a row on
    different workgroups: all as from a workspace of their own."""
    past = [int(x) for x in np.random.default_rng(9).integers(100, 1500, 40)]
    c = ref.Cache(3, "bf16", "dense", 64, 4, 64, [p + 1 for p in past])
    K, V, pages = c.to(cuda_device)
    dpast = torch.tensor(past, dtype=torch.int32, device=cuda_device)
    qs = torch.randn(60, 40, 16, 64, device=cuda_device).bfloat16()
    ws = lib.paged_workspace(qs[0], K, pages)
    got = torch.stack([lib.paged_attn(q, K, V, pages, dpast, 0.1, workspace=ws) for q in qs])
    want = torch.stack([lib.paged_attn(q, K, V, pages, dpast, 0.1) for q in qs])
    assert torch.equal(got, want)


def test_calls_on_two_streams(cuda_device):
    """Two calls at once, each with its own workspace."""
    c = ref.Cache(5, "f16", "mx4", 128, 2, 32, [700, 300, 900])
    K, V, pages = c.to(cuda_device)
    past = torch.tensor([699, 299, 899], dtype=torch.int32, device=cuda_device)
    q = torch.randn(2, 3, 16, 128, device=cuda_device).half()
    want = [lib.paged_attn(x, K, V, pages, past, 0.09) for x in q]
    ws = [lib.paged_workspace(q[0], K, pages) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(lib.paged_attn(q[i], K, V, pages, past, 0.09, workspace=ws[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "dense", 128), ("f16", "dense", 64),
                                         ("bf16", "mx4", 128), ("f16", "mx4", 256),
                                         ("f16", "dense", 256), ("bf16", "mx4", 64)])
def test_chunks_over_page_sizes(cuda_device, dtype, fmt, d, P):
    """Many rows a head: row tiles that end inside a token and inside a page."""
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=d, h_q=10, h_kv=2, P=P,
               past=[300, 0, 63], T=90, counts=[90, 77, 1], seed=P + d)


def test_queries_with_a_stride_and_another_stream(cuda_device):
    """q as a view into a fused projection, the call on a stream of its own."""
    c = ref.Cache(12, "f16", "dense", 64, 2, 16, [90, 41])
    K, V, pages = c.to(cuda_device)
    past = torch.tensor([89, 40], dtype=torch.int32, device=cuda_device)
    fused = torch.randn(2, 8 + 4, 64, device=cuda_device).half()
    q = fused[:, :8]
    assert not q.is_contiguous()
    want = lib.paged_attn(q.contiguous(), K, V, pages, past, 0.125)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lib.paged_attn(q, K, V, pages, past, 0.125)
    also = lib.paged_attn(q, K, V, pages, past, 0.125, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(also, want)


@pytest.mark.parametrize("T", [1, 4, 40])
def test_the_largest_scales(cuda_device, T):
    """A finite scale whose product with log2(e) is not: scores of 0 stay 0, so
    queries of zeros give the mean of V."""
    c = ref.Cache(14, "bf16", "dense", 64, 1, 16, [96])
    K, V, pages = c.to(cuda_device)
    past = torch.tensor([96], dtype=torch.int32, device=cuda_device)
    scale = float(np.finfo(np.float32).max)
    q = torch.zeros(T, 8, 64, dtype=torch.bfloat16, device=cuda_device)
    want = lib.paged_attn(q, K, V, pages, past, 0.125, causal=False)
    for s in (scale, -scale):
        got = lib.paged_attn(q, K, V, pages, past, s, causal=False)
        assert torch.isfinite(got).all() and torch.equal(got, want)


def test_what_a_call_allocates_is_of_its_stream(cuda_device):
    """A call on a stream that need not wait for the current one, which is busy: the
    workspace's counters are zero when it runs, and its results are not memory that
    the current stream has still to write."""
    c = ref.Cache(13, "bf16", "dense", 64, 2, 16, [300, 200])
    K, V, pages = c.to(cuda_device)
    past = torch.tensor([299, 199], dtype=torch.int32, device=cuda_device)
    q = torch.randn(2, 8, 64, device=cuda_device).bfloat16()
    table = lib.rotary_table(K.shape[2] * pages.shape[1], 64, device=cuda_device)
    k = torch.randn(2, 2, 64, device=cuda_device).bfloat16()
    want_q = lib.paged_append(K, V, pages, past, k, k, q=q, rotary=table)
    want = lib.paged_attn(q, K, V, pages, past, 0.125)
    n = lib.paged_workspace(q, K, pages).numel()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.randn(4096, 4096, device=cuda_device)
    # blocks of these sizes that the current stream fills late, and gives back
    late = [torch.empty(n, dtype=torch.uint8, device=cuda_device), torch.empty_like(q),
            torch.empty_like(q)]
    torch.cuda.synchronize()
    for _ in range(30):
        busy = busy @ busy * 1e-4
    for x in late:
        x.fill_(1)
    del late, x
    got = lib.paged_attn(q, K, V, pages, past, 0.125, stream=side)
    got_q = lib.paged_append(K, V, pages, past, k, k, q=q, rotary=table, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_q, want_q)


def test_sizes_that_are_not_integers_of_32_bits(cuda_device):
    K, V = lib.paged_alloc(2, 16, 1, 64, device=cuda_device)
    pages = torch.tensor([[0]], dtype=torch.int32, device=cuda_device)
    past = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    start = torch.tensor([0, 1], dtype=torch.int32, device=cuda_device)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device=cuda_device)
    for T in (1 << 40, 1.5):
        with pytest.raises(ValueError, match="32 bits"):
            lib.paged_append(K, V, pages, past, q, q, row_start=start, T=T)
        with pytest.raises(ValueError, match="32 bits"):
            lib.paged_attn(q, K, V, pages, past, 1.0, row_start=start, T=T)


def test_pool_beyond_32_bit_offsets(cuda_device):
    """Pages at both ends of pools of 6 GiB."""
    P, h_kv, d = 256, 8, 128
    n = (6 << 30) // (P * h_kv * d * 2)
    K = torch.empty(n, h_kv, P, d, dtype=torch.bfloat16, device=cuda_device)
    V = torch.empty_like(K)
    small = ref.Cache(13, "bf16", "dense", d, h_kv, P, [P + 40], spare=0)
    q = torch.from_numpy(np.random.default_rng(1).standard_normal((1, 8, d))).bfloat16()
    past = torch.tensor([P + 39], dtype=torch.int32, device=cuda_device)
    Ks, Vs, ps = small.to(cuda_device)
    want = lib.paged_attn(q.to(cuda_device), Ks, Vs, ps, past, 0.1)
    pages = torch.tensor([[n - 1, 0]], dtype=torch.int32, device=cuda_device)
    for at, page in ((n - 1, int(small.pages[0, 0])), (0, int(small.pages[0, 1]))):
        K[at], V[at] = Ks[page], Vs[page]
    assert torch.equal(lib.paged_attn(q.to(cuda_device), K, V, pages, past, 0.1), want)
    k = torch.randn(1, h_kv, d, device=cuda_device).bfloat16()
    at = torch.tensor([P - 1], dtype=torch.int32, device=cuda_device)
    lib.paged_append(K, V, pages, at, k, -k)
    assert torch.equal(K[n - 1, :, P - 1], k[0]) and torch.equal(V[n - 1, :, P - 1], -k[0])


# --- append and gather -------------------------------------------------------------

def check_append(device, *, dtype="bf16", fmt="dense", d=128, h_q=4, h_kv=2, P=16, past=(3,), T=1,
                 counts=None, rot=None, interleaved=False, seed=0, wide=None, behind=0, edit=None,
                 strided=False, in_place=False, spread=1.0):
    t = ref.DTYPES[dtype]
    rot = d if rot is None else rot
    n = counts if counts is not None else [T] * len(past)
    held = [max(p, 0) + c if p >= 0 else 0 for p, c in zip(past, n)]
    c = ref.Cache(seed, dtype, fmt, d, h_kv, P, [min(x, (wide or 10 ** 6) * P) for x in held],
                  wide=wide)
    if edit:
        edit(c)
    row_start, N = rows_of(n, behind)
    rng = np.random.default_rng(seed + 1)
    cap = c.pages.shape[1] * P

    def rows(h):
        x = rng.standard_normal((N, h, d)) * spread ** rng.standard_normal((N, h, d))
        return torch.from_numpy(x).to(t)

    q, k, v = rows(h_q), rows(h_kv), rows(h_kv)
    table = lib.rotary_table(cap, rot, device="cpu") if rot else None
    K, V, pages = c.to(device)
    # a bit pattern of the pools as they were
    if strided:
        fused = torch.cat((q, k, v), 1).to(device)
        dq, dk, dv = fused[:, :h_q], fused[:, h_q:h_q + h_kv], fused[:, h_q + h_kv:]
    else:
        dq, dk, dv = q.to(device), k.to(device), v.to(device)
    q_out = dq if in_place else torch.full_like(q, 9.0).to(device)
    start = row_start.to(device) if counts is not None else None
    past_t = torch.tensor(past, dtype=torch.int32, device=device)
    say(f"append {dtype} {fmt} d={d} P={P} past={past[:6]} rows={n[:6]} rot={rot} "
        f"interleaved={interleaved} seed={seed}")
    lib.paged_append(K, V, pages, past_t, dk, dv, q=dq, q_out=q_out,
                     rotary=None if table is None else table.to(device),
                     interleaved=interleaved, row_start=start, T=T)
    k_back = torch.full_like(k, 9.0).to(device)
    v_back = torch.full_like(v, 9.0).to(device)
    lib.paged_gather(K, V, pages, past_t, k_back, v_back, row_start=start, T=T)
    torch.cuda.synchronize()
    assert past_t.tolist() == list(past)

    tab = table.double().numpy() if rot else np.zeros((cap, 0))
    want_q = (q if in_place else torch.full_like(q, 9.0)).double().numpy().copy()
    want_kb = np.full(k.shape, 9.0)
    want_vb = np.full(v.shape, 9.0)
    KB, VB = c.K.clone(), c.V.clone()          # what the pools become
    near = []                                   # (page, slot) whose K values are rounded ones
    for b, (s, cnt) in enumerate(ref.seq_rows(row_start.numpy(), len(past), T, N)):
        for r in range(cnt):
            pos, page, slot = ref.place(c.pages.numpy(), past, b, r, P, c.K.shape[0])
            want_kb[s + r] = want_vb[s + r] = 0.0
            if pos is None:
                continue
            want_q[s + r] = ref.turn(q[s + r].double().numpy(), pos, tab, interleaved)
            if page is None:
                continue
            kd = ref.turn(k[s + r].double().numpy(), pos, tab, interleaved)
            vd = v[s + r].double().numpy()
            if fmt == "dense":
                KB[page, :, slot] = torch.from_numpy(kd).to(t)
                VB[page, :, slot] = v[s + r]
                near.append((page, slot, s + r, kd))
                want_kb[s + r], want_vb[s + r] = kd, vd
            else:
                for h in range(h_kv):
                    for pool, x, back, value in ((KB, kd, want_kb, False),
                                                 (VB, vd, want_vb, True)):
                        codes, scales = ref.unpack_page(pool[page, h].reshape(-1).numpy(), P, d,
                                                        value)
                        codes, scales = codes.copy(), scales.copy()
                        codes[slot], scales[slot] = ref.quantise(x[h])
                        pool[page, h] = torch.from_numpy(
                            ref.pack_page(codes, scales, value)).reshape(P, -1)
                        back[s + r, h] = ref.values(codes[slot], scales[slot])
    u, e32 = ref.half_step(t), 2.0 ** -24
    # two products and a sum in 32 bits of numbers up to the pair's size, one
    # rounding to the type
    big = float(max(x.abs().max() for x in (q, k)))
    slack = 4 * e32 * big + {torch.float16: 2.0 ** -25}.get(t, 0.0)

    def close(got, want):
        err = np.abs(got - want)
        assert (err <= slack + u * (np.abs(want) + slack)).all(), err.max()

    got_q = q_out.cpu().double().numpy()
    close(got_q, want_q)
    gK, gV = K.cpu(), V.cpu()
    assert torch.equal(gV.view(torch.uint8), VB.view(torch.uint8)), "V pool"
    if fmt == "mx4":
        assert torch.equal(gK, KB), "K pool"
        # read back as the type holds it
        for got, want in ((k_back, want_kb), (v_back, want_vb)):
            w = torch.from_numpy(want).to(t)
            assert torch.equal(torch.nan_to_num(got.cpu(), nan=7e3),
                               torch.nan_to_num(w, nan=7e3))
    else:
        for page, slot, _, kd in near:
            close(gK[page, :, slot].double().numpy(), kd)
            KB[page, :, slot] = gK[page, :, slot]
        assert torch.equal(gK.view(torch.uint8), KB.view(torch.uint8)), "K pool"
        close(k_back.cpu().double().numpy(), want_kb)
        assert np.array_equal(v_back.cpu().double().numpy(), want_vb)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (128, 128), (128, 96), (128, 0), (256, 256),
                                   (256, 32)])
@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_append(cuda_device, dtype, fmt, d, rot, interleaved):
    check_append(cuda_device, dtype=dtype, fmt=fmt, d=d, rot=rot, interleaved=interleaved,
                 past=[0, 14, 31, 100], T=3, seed=d + rot)


@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_append_of_ragged_rows(cuda_device, dtype, fmt):
    """No rows, one, many; rows behind the last sequence; a negative past; rows
    that pass the capacity; a missing page."""
    def edit(c):
        c.pages[2, 2] = -1
    check_append(cuda_device, dtype=dtype, fmt=fmt, d=64, h_q=5, h_kv=1, P=32,
                 past=[0, 7, 40, -1, 150], T=60, counts=[60, 0, 31, 5, 20], wide=5, behind=3,
                 edit=edit, seed=3)


@pytest.mark.parametrize("strided,in_place", [(True, False), (False, True)])
def test_append_of_views_and_in_place(cuda_device, strided, in_place):
    check_append(cuda_device, dtype="bf16", past=[5, 40], T=2, strided=strided, in_place=in_place,
                 seed=21)
    check_append(cuda_device, dtype="f32", fmt="mx4", past=[5, 40], T=2, strided=strided,
                 in_place=in_place, interleaved=True, seed=22)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_codes_of_values_of_every_size(cuda_device, dtype):
    """Values over many powers of two within a block, and ties between codes."""
    check_append(cuda_device, dtype=dtype, fmt="mx4", past=[0, 9], T=40, spread=8.0, seed=31)
    t = ref.DTYPES[dtype]
    ties = np.array([0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.5, -.25, -.75, -5, -3.5, -0.0])
    block = np.concatenate((ties, ties[::-1]))
    x = torch.from_numpy(np.stack([block * 2.0 ** e for e in (0, -3, 7, -10)]).reshape(2, 1, 64)) \
        .to(t)
    x[1, 0, 32:] = 0.0
    K, V = lib.paged_alloc(1, 16, 1, 64, dtype=t, format="mx4", device=cuda_device)
    pages = torch.zeros(1, 1, dtype=torch.int32, device=cuda_device)
    past = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    lib.paged_append(K, V, pages, past, x.to(cuda_device), x.to(cuda_device))
    codes, scales = ref.quantise(x[:, 0].double().numpy())
    for pool, value in ((K, False), (V, True)):
        c, s = ref.unpack_page(pool[0, 0].reshape(-1).cpu().numpy(), 16, 64, value)
        assert np.array_equal(c[:2], codes) and np.array_equal(s[:2], scales)


def test_codes_of_the_smallest_values(cuda_device):
    """Blocks whose largest value is at, above and below the smallest scale's, and
    next to 2^127."""
    rng = np.random.default_rng(8)
    tops = [2.0 ** e for e in (-149, -130, -127, -126, -125, -124, -123, -100, 100, 127)]
    x = np.stack([rng.uniform(-1, 1, 64) * t * (1.99 if t > 1 else 1.0) for t in tops])
    x = torch.from_numpy(x).float()[:, None]
    K, V = lib.paged_alloc(1, 16, 1, 64, dtype=torch.float32, format="mx4", device=cuda_device)
    pages = torch.zeros(1, 1, dtype=torch.int32, device=cuda_device)
    past = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    lib.paged_append(K, V, pages, past, x.to(cuda_device), x.to(cuda_device))
    codes, scales = ref.quantise(x[:, 0].double().numpy())
    for pool, value in ((K, False), (V, True)):
        c, s = ref.unpack_page(pool[0, 0].reshape(-1).cpu().numpy(), 16, 64, value)
        for n, t in enumerate(tops):
            assert np.array_equal(s[n], scales[n]), (t, s[n], scales[n])
            assert np.array_equal(c[n], codes[n]), (t, c[n], codes[n])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_blocks_that_are_not_finite_read_as_nan(cuda_device, dtype):
    t = ref.DTYPES[dtype]
    x = torch.randn(1, 1, 128).to(t)
    x[0, 0, 5], x[0, 0, 70] = math.inf, math.nan
    K, V = lib.paged_alloc(1, 16, 1, 128, dtype=t, format="mx4", device=cuda_device)
    pages = torch.zeros(1, 1, dtype=torch.int32, device=cuda_device)
    past = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    x = x.to(cuda_device)
    lib.paged_append(K, V, pages, past, x, x)
    for y in lib.paged_gather(K, V, pages, past, torch.empty_like(x), torch.empty_like(x)):
        nan = torch.isnan(y.cpu()).reshape(4, 32).all(1).tolist()
        assert nan == [True, False, True, False]
        assert torch.isfinite(y.cpu().reshape(4, 32)[1::2]).all()


# --- together ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,fmt", TYPES)
def test_steps_of_a_serving_loop(cuda_device, dtype, fmt):
    """A prompt, then tokens, of two layers that share a page table: appends,
    attention, past advanced once a step; the steps after the prompt as one
    captured graph, replayed."""
    t = ref.DTYPES[dtype]
    B, h_q, h_kv, d, P, cap = 3, 8, 2, 64, 16, 96
    rng = np.random.default_rng(17)
    layers = [lib.paged_alloc(B * cap // P, P, h_kv, d, dtype=t, format=fmt, device=cuda_device)
              for _ in range(2)]
    pages = torch.from_numpy(rng.permutation(B * cap // P).reshape(B, -1).astype(np.int32))
    table = lib.rotary_table(cap, d, device=cuda_device)
    dpages = pages.to(cuda_device)
    past = torch.zeros(B, dtype=torch.int32, device=cuda_device)
    scale = 1 / math.sqrt(d)

    def draw(n):
        return [[torch.from_numpy(rng.standard_normal((n, h, d))).to(t) for h in (h_q, h_kv, h_kv)]
                for _ in layers]

    def reference(layer, q, host_past, start, T):
        K, V = layers[layer]
        return ref.attention(q, K.cpu(), V.cpu(), pages.numpy(), host_past, scale, True, start, T,
                             h_kv)

    def check(out, r):
        want, mass, spread, seen, mine, top = r
        tol = ref.tolerance(want, mass, spread, seen, top, t, d)
        assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()

    counts = [37, 1, 20]
    start, N = rows_of(counts)
    for i, (q, k, v) in enumerate(draw(N)):
        K, V = layers[i]
        qr = lib.paged_append(K, V, dpages, past, k.to(cuda_device), v.to(cuda_device),
                              q=q.to(cuda_device), rotary=table, row_start=start.to(cuda_device),
                              T=37)
        out = lib.paged_attn(qr, K, V, dpages, past, scale, row_start=start.to(cuda_device), T=37)
        check(out, reference(i, qr.cpu(), [0] * B, start.numpy(), 37))
    past += torch.tensor(counts, dtype=torch.int32, device=cuda_device)

    inputs = [[x.to(cuda_device) for x in y] for y in draw(B)]
    ws = [lib.paged_workspace(inputs[i][0], layers[i][0], dpages) for i in range(2)]
    rotated = [torch.empty_like(y[0]) for y in inputs]
    outs = [torch.empty_like(y[0]) for y in inputs]

    def step():
        for i, (K, V) in enumerate(layers):
            q, k, v = inputs[i]
            lib.paged_append(K, V, dpages, past, k, v, q=q, q_out=rotated[i], rotary=table)
            lib.paged_attn(rotated[i], K, V, dpages, past, scale, out=outs[i], workspace=ws[i])
        past.add_(1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()                                   # warm, and a real step
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for _ in range(5):
        host_past = past.tolist()
        for y in inputs:
            for x in y:
                x.copy_(torch.from_numpy(rng.standard_normal(tuple(x.shape))).to(t))
        graph.replay()
        torch.cuda.synchronize()
        say("replayed step at", host_past)
        assert past.tolist() == [x + 1 for x in host_past]
        for i in range(2):
            check(outs[i], reference(i, rotated[i].cpu(), host_past, None, 1))


def test_float32_pages_agree_with_the_dense_slabs(cuda_device):
    """The same rows appended to slabs and to pages: the same attention within
    the bounds of 32-bit sums."""
    B, h_q, h_kv, d, P, n = 2, 8, 2, 128, 32, 64
    rng = torch.Generator().manual_seed(3)
    K, V = (torch.zeros(B, h_kv, n, d, device=cuda_device) for _ in range(2))
    lens = torch.zeros(B, dtype=torch.int32, device=cuda_device)
    pk, pv = lib.paged_alloc(B * n // P, P, h_kv, d, dtype=torch.float32, device=cuda_device)
    pages = torch.tensor([[3, 0], [1, 2]], dtype=torch.int32, device=cuda_device)
    for step in range(40):
        q, k, v = (torch.randn(B, h, d, generator=rng).to(cuda_device) for h in (h_q, h_kv, h_kv))
        past = lens.clone()
        want = lib.decode_step(q, K, V, k, v, lens, 0.09)
        lib.paged_append(pk, pv, pages, past, k, v)
        got = lib.paged_attn(q, pk, pv, pages, past, 0.09)
        assert (got - want).abs().max().item() <= 1e-5, step
