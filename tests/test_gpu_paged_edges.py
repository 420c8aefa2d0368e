"""The paged cache on the GPU at the edges of its numbers: values that are not
finite or do not fit the type of the rows, weights that all round one way, scores
beyond what 32 bits resolve.  In every kernel that a call may take (16 and 32
query rows a KV head, chunks of more), on items that one workgroup holds and on
items in parts."""
import math

import numpy as np
import pytest
import torch

import paper_2607_19456_amd as lib
import paged_reference as ref
from test_gpu_paged import check_attn

pytestmark = pytest.mark.gpu

P = 16
# Positions of each sequence before the step: one workgroup or a few; in parts that
# the last workgroup puts together (at most 1024 positions, where rows are few); in
# parts that the merge puts together; many sequences.
PASTS = {"short": [40], "parts": [900], "merged": [2900], "many": [40 + 7 * b for b in range(70)]}


def set_v(c, b, head, pos, block, x):
    """Position pos of sequence b gets x in V, in the first dimensions of a block of
    32 (of a 4-bit cache: the block becomes NaN)."""
    page, slot = int(c.pages[b, pos // c.P]), pos % c.P
    if c.fmt == "dense":
        c.V[page, head, slot, 32 * block + 3] = x
        c.V[page, head, slot, 32 * block + 9:32 * block + 13] = x
        return
    edit_scale(c, c.V, True, page, head, slot, block, 255)


def edit_scale(c, pool, value, page, head, slot, block, byte):
    codes, scales = ref.unpack_page(pool[page, head].reshape(-1).numpy(), c.P, c.d, value)
    scales = scales.copy()
    scales[slot, block] = byte
    pool[page, head] = torch.from_numpy(ref.pack_page(codes, scales, value)).reshape(c.P, -1)


def edit_codes(c, page, head, slot, block, codes_in_turn):
    codes, scales = ref.unpack_page(c.V[page, head].reshape(-1).numpy(), c.P, c.d, True)
    codes[slot, 32 * block:32 * block + 32] = np.resize(np.array(codes_in_turn, np.uint8), 32)
    c.V[page, head] = torch.from_numpy(ref.pack_page(codes, scales, True)).reshape(c.P, -1)


def set_k_nan(c, b, head, pos):
    page, slot = int(c.pages[b, pos // c.P]), pos % c.P
    if c.fmt == "dense":
        c.K[page, head, slot, 7] = math.nan
    else:
        edit_scale(c, c.K, False, page, head, slot, 1, 255)


# --- what some rows see and others do not -------------------------------------------

@pytest.mark.parametrize("past", PASTS)
@pytest.mark.parametrize("T", [4, 10, 70])
@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "dense", 64), ("bf16", "dense", 128),
                                         ("f16", "dense", 128), ("f16", "dense", 256),
                                         ("f32", "dense", 64), ("bf16", "mx4", 64),
                                         ("f16", "mx4", 128), ("bf16", "mx4", 256),
                                         ("f32", "mx4", 128)])
def test_what_only_later_rows_see(cuda_device, dtype, fmt, d, T, past):
    """Infinities and NaN in V among the step's own positions, on head 0, and
    before them, on head 1 (which all rows see); NaN in K at the last position but
    one, on head 1.  8, 20 and 140 rows a KV head."""
    pasts = PASTS[past] if past != "many" or T < 70 else PASTS[past][:12]

    def edit(c):
        for b, p in enumerate(pasts):
            if b % 3:
                continue
            set_v(c, b, 0, p + 1, 0, math.inf)
            set_v(c, b, 0, p + T // 2, 1, math.nan)
            set_v(c, b, 0, p + T - 2, 1, -math.inf)
            set_v(c, b, 1, p // 2, 1, math.inf)
            set_v(c, b, 1, p - 1, 0, -math.inf)
            set_k_nan(c, b, 1, p + T - 2)
    check_attn(cuda_device, dtype=dtype, fmt=fmt, d=d, h_q=4, h_kv=2, past=pasts, T=T, edit=edit,
               seed=T + d)


# --- rows whose scores are -infinity ------------------------------------------------

def minus_inf_keys(c, b, lo, hi):
    for pos in range(lo, hi):
        page, slot = int(c.pages[b, pos // c.P]), pos % c.P
        c.K[page, :, slot, 0] = -math.inf


def attend(device, dtype, d, h_q, h_kv, past, T, edit):
    """(result, cache, q) of queries whose first dimension is positive."""
    q = torch.from_numpy(np.random.default_rng(5).standard_normal((len(past) * T, h_q, d)))
    q[..., 0] = q[..., 0].abs() + 0.5
    q = q.to(ref.DTYPES[dtype])
    c = ref.Cache(T, dtype, "dense", d, h_kv, P, [p + T for p in past])
    edit(c)
    K, V, pages = c.to(device)
    print("attn", dtype, "past", past[:6], "rows", T, flush=True)
    out = lib.paged_attn(q.to(device), K, V, pages,
                         torch.tensor(past, dtype=torch.int32, device=device), 1 / math.sqrt(d))
    return out.cpu(), c, q


@pytest.mark.parametrize("past", [[20], [900], [2900], [20 + b % 9 for b in range(300)]],
                         ids=["one", "parts", "merged", "whole"])
@pytest.mark.parametrize("T", [4, 10, 20])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_rows_of_scores_that_are_all_minus_infinity(cuda_device, dtype, T, past):
    """They give 0, whatever V holds: 8, 20 and 40 rows a KV head."""
    past = [20 + b % 9 for b in range(300)] if len(past) > 1 else past

    def edit(c):
        for b, p in enumerate(past):
            minus_inf_keys(c, b, 0, p + T)
            set_v(c, b, 0, 3, 0, math.inf)
            set_v(c, b, 0, 3, 1, math.nan)
            set_v(c, b, 0, p + 1, 1, math.inf)
    out = attend(cuda_device, dtype, 64, 2, 1, past, T, edit)[0]
    assert int(torch.count_nonzero(out)) == 0 and not torch.isnan(out).any()


@pytest.mark.parametrize("past", [[900], [2900], [40] * 130], ids=["parts", "merged", "short"])
@pytest.mark.parametrize("T", [4, 10, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_of_scores_that_are_all_minus_infinity(cuda_device, dtype, T, past):
    """The first half of the keys has weight 0, and 0 times an infinity or a NaN is
    NaN: however the row is divided.  The other results are those without these
    keys' scores."""
    def edit(c):
        for b, p in enumerate(past):
            minus_inf_keys(c, b, 0, p // 2)
            if b % 2 == 0:
                set_v(c, b, 0, 3, 0, math.inf)
                set_v(c, b, 1, 5, 1, math.nan)
    out, c, q = attend(cuda_device, dtype, 64, 4, 2, past, T, edit)
    want, mass, _, seen, _, top = ref.attention(q, c.K, c.V, c.pages.numpy(), past, 1 / 8, True,
                                                None, T, 2)
    finite_k = torch.where(torch.isinf(c.K), torch.zeros_like(c.K), c.K)
    spread = ref.attention(q, finite_k, c.V, c.pages.numpy(), past, 1 / 8, True, None, T, 2)[2]
    got, nan = out.double().numpy(), np.isnan(want)
    assert nan.any() and np.array_equal(np.isnan(got), nan)
    tol = ref.tolerance(np.where(nan, 0, want), np.where(nan, 0, mass), spread, seen, 0.0,
                        ref.DTYPES[dtype], 64)
    assert (np.abs(np.where(nan, 0, got - want)) <= tol).all()


# --- the sum that divides is that of the weights as they are multiplied --------------

@pytest.mark.parametrize("past", [[1400], [500] * 600], ids=["parts", "whole"])
@pytest.mark.parametrize("T", [4, 10, 20, 70])
@pytest.mark.parametrize("dtype,weight", [("bf16", 0.5 * (1 + 0.9 * 2.0 ** -8)),
                                          ("f16", 0.5 * (1 + 0.9 * 2.0 ** -11)),
                                          ("f16", 1.5 * 2.0 ** -16)])
def test_weights_that_all_round_one_way(cuda_device, dtype, weight, T, past):
    """One key at score 0 and all others where their weight is off by 0.9 of half a
    step, or below the normal numbers of float16: V of ones gives ones, since both sums
    are of the same weights and their roundings in 32 bits (at most n * 2^-24, n <
    1500 keys) stay far from half a step of the result."""
    t = ref.DTYPES[dtype]
    B, n = len(past), past[0] + T
    K = torch.zeros(B * -(-n // P), 1, P, 64, dtype=t, device=cuda_device)
    K[..., 0] = -1
    pages = torch.arange(K.shape[0], dtype=torch.int32, device=cuda_device).reshape(B, -1)
    K[pages[:, 0].long(), 0, 0, 0] = 0
    q = torch.zeros(B * T, 2, 64, dtype=t, device=cuda_device)
    q[..., 0] = 1
    out = lib.paged_attn(q, K, torch.ones_like(K), pages,
                         torch.tensor(past, dtype=torch.int32, device=cuda_device),
                         -math.log(weight))
    print(dtype, weight, T, "off by", float((out.double() - 1).abs().max()), flush=True)
    assert torch.equal(out, torch.ones_like(out))


# --- 4-bit blocks at the ends of their range ------------------------------------------

def dense_of(c, t):
    """A dense cache of the same values, rounded to the type."""
    K, V = (torch.zeros(c.K.shape[0], c.h_kv, c.P, c.d, dtype=t) for _ in range(2))
    for page in range(c.K.shape[0]):
        for h in range(c.h_kv):
            for pool, to, value in ((c.K, K, False), (c.V, V, True)):
                with np.errstate(over="ignore"):
                    to[page, h] = torch.from_numpy(ref.page_rows(pool, page, h, c.d, value)).to(t)
    return K, V


def every_code(rng, scales, rows, d):
    """Codes and scale bytes of rows whose blocks have the given bytes in turn."""
    codes = rng.integers(0, 16, (rows, d)).astype(np.uint8)
    codes[:, :16] = np.arange(16)
    return codes, np.resize(np.array(scales, np.uint8), (rows, d // 32))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_blocks_of_every_scale_read_back(cuda_device, dtype):
    """All 256 bytes, all 16 codes: the values rounded to the type."""
    t = ref.DTYPES[dtype]
    rng = np.random.default_rng(3)
    d, n = 64, 128
    c = ref.Cache(1, dtype, "mx4", d, 1, n, [n], spare=0)
    codes, scales = every_code(rng, range(256), n, d)
    for pool, value in ((c.K, False), (c.V, True)):
        pool[0, 0] = torch.from_numpy(ref.pack_page(codes, scales, value)).reshape(n, -1)
    K, V, _ = c.to(cuda_device)
    pages = torch.zeros(1, 1, dtype=torch.int32, device=cuda_device)
    past = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    want = torch.from_numpy(ref.values(codes, scales)).to(t)
    back = [torch.empty(n, 1, d, dtype=t, device=cuda_device) for _ in range(2)]
    for got in lib.paged_gather(K, V, pages, past, *back):
        got = got[:, 0].cpu()
        same = (got == want) | (torch.isnan(got) & torch.isnan(want))
        assert same.all(), [(int(scales[r, x // 32]), int(codes[r, x]), float(got[r, x]),
                             float(want[r, x])) for r, x in (~same).nonzero().tolist()[:8]]


@pytest.mark.parametrize("T", [1, 10, 40])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attention_over_blocks_of_every_scale(cuda_device, dtype, T):
    """One position, so a weight of 1: V comes out as paged_gather reads it, each
    position of a sequence of its own."""
    t = ref.DTYPES[dtype]
    rng = np.random.default_rng(4)
    d, n = 64, 128
    codes, scales = every_code(rng, range(256), n, d)
    c = ref.Cache(1, dtype, "mx4", d, 1, P, [P] * n, spare=0)
    for b in range(n):
        full_c, full_s = np.zeros((P, d), np.uint8), np.full((P, d // 32), 127, np.uint8)
        full_c[0], full_s[0] = codes[b], scales[b]
        c.V[int(c.pages[b, 0]), 0] = torch.from_numpy(
            ref.pack_page(full_c, full_s, True)).reshape(P, -1)
    K, V, pages = c.to(cuda_device)
    want = torch.from_numpy(ref.values(codes, scales)).to(t)
    past = torch.ones(n, dtype=torch.int32, device=cuda_device)
    q = torch.zeros(n * T, 1, d, dtype=t, device=cuda_device)
    out = lib.paged_attn(q, K, V, pages, past, 1.0, causal=False)
    # a result below the normal numbers of 32 bits may be taken for 0
    low = want.double().abs() < 2.0 ** -126
    for got in out.reshape(n, T, d).cpu().unbind(1):
        same = (got == want) | (torch.isnan(got) & torch.isnan(want)) \
            | (low & (got.double().abs() <= 2.0 ** -126))
        assert same.all(), [(int(scales[r, x // 32]), int(codes[r, x]), float(got[r, x]),
                             float(want[r, x])) for r, x in (~same).nonzero().tolist()[:8]]


@pytest.mark.parametrize("past", [[40], [900], [2900]], ids=["short", "parts", "merged"])
@pytest.mark.parametrize("T", [4, 10, 70])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype,scales", [("f16", (141, 142, 143, 144, 180)), ("f32", (253, 254)),
                                          ("bf16", (253, 254))])
def test_4_bit_values_that_do_not_fit_the_type(cuda_device, dtype, scales, d, T, past):
    """V values that are infinities in the rows' type, at positions that only some
    rows see: infinite where they are seen, and nothing where they are not."""
    t = ref.DTYPES[dtype]
    c = ref.Cache(7, dtype, "mx4", d, 2, P, [past[0] + T])
    rng = np.random.default_rng(T)
    for n, byte in enumerate(scales):
        pos = past[0] + 1 + (n * (T - 2)) // len(scales)
        page, slot = int(c.pages[0, pos // P]), pos % P
        block = n % (d // 32)
        edit_scale(c, c.V, True, page, n % 2, slot, block, byte)
        if dtype != "f16":
            # sums in 32 bits of finite values as large as these would be infinite
            edit_codes(c, page, n % 2, slot, block, (0, 7, 15))
    K, V, pages = c.to(cuda_device)
    q = torch.from_numpy(rng.standard_normal((T, 4, d))).to(t)
    dK, dV = dense_of(c, t)
    scale = 1 / math.sqrt(d)
    want, mass, spread, seen, _, _ = ref.attention(q, dK, dV, c.pages.numpy(), past, scale, True,
                                                   None, T, 2)
    out = lib.paged_attn(q.to(cuda_device), K, V, pages,
                         torch.tensor(past, dtype=torch.int32, device=cuda_device), scale)
    got = out.cpu().double().numpy()
    # the largest V that a finite output may hold is that of other dimensions of the
    # same block: the bound goes by each output's own weights, and float16 weights
    # below 2^-14 by the values that they may be of
    with np.errstate(invalid="ignore"):
        finite = np.isfinite(want)
        mass = np.where(finite, mass, 0.0)
        top = float(np.abs(np.nan_to_num(dV.double().numpy(), nan=0, posinf=0, neginf=0)).max())
        tol = ref.tolerance(np.where(finite, want, 0.0), mass, spread, seen, top, t, d)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)])
        assert (np.abs(np.where(finite, got - want, 0.0)) <= tol).all()


# --- scores of any size ---------------------------------------------------------------

@pytest.mark.parametrize("past", [[60, 3], [2900]], ids=["short", "merged"])
@pytest.mark.parametrize("T", [4, 10, 70])
@pytest.mark.parametrize("scale", [2.0 ** 24, -3.0e8, 1e12, 1e30])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("f16", "dense"), ("f32", "dense"),
                                       ("f16", "mx4")])
def test_scores_of_any_size(cuda_device, dtype, fmt, scale, T, past):
    """Finite scores far apart: the one key with the largest has all the weight.
    Rows are looked at whose two largest scores differ by more than the error of
    sums of d products in 32 bits and of the scaling; of a row's next key exp(-100)
    is left, so the result is that key's V, rounded in 32 bits three times."""
    t, d = ref.DTYPES[dtype], 64
    c = ref.Cache(11, dtype, fmt, d, 1, P, [p + T for p in past])
    q = torch.from_numpy(np.random.default_rng(12).standard_normal((T * len(past), 2, d))).to(t)
    K, V, pages = c.to(cuda_device)
    out = lib.paged_attn(q.to(cuda_device), K, V, pages,
                         torch.tensor(past, dtype=torch.int32, device=cuda_device), scale)
    got, looked = out.cpu().double().numpy(), 0
    assert np.isfinite(got).all()
    for b, p in enumerate(past):
        ids = [int(x) for x in c.pages[b, :-(-(p + T) // P)]]
        k = np.concatenate([ref.page_rows(c.K, x, 0, d, False) for x in ids])
        v = np.concatenate([ref.page_rows(c.V, x, 0, d, True) for x in ids])
        for r in range(T):
            n = p + r + 1
            for h in range(2):
                x = q[b * T + r, h].double().numpy()
                s = scale * (k[:n] @ x)
                at = np.argsort(s)
                slack = 4 * (d + 16) * 2.0 ** -24 * abs(scale) * (np.abs(k[:n]) @ np.abs(x)).max()
                if s[at[-1]] - s[at[-2]] <= slack + 100:
                    continue
                looked += 1
                w = v[at[-1]]
                err = np.abs(got[b * T + r, h] - w)
                assert (err <= (ref.half_step(t) + 3 * 2.0 ** -24) * np.abs(w)).all()
    print("rows looked at:", looked, flush=True)
    assert looked > T


@pytest.mark.parametrize("T", [4, 10, 70])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_scores_beyond_32_bits(cuda_device, dtype, T):
    """Infinite in 32 bits, as their difference is then NaN: no row that has one
    passes for one that sees nothing."""
    t, d, past = ref.DTYPES[dtype], 64, 200
    c = ref.Cache(13, dtype, "dense", d, 1, P, [past + T])
    K, V, pages = c.to(cuda_device)
    q = torch.from_numpy(np.random.default_rng(2).standard_normal((T, 2, d))).to(t)
    out = lib.paged_attn(q.to(cuda_device), K, V, pages,
                         torch.tensor([past], dtype=torch.int32, device=cuda_device), 3.0e38)
    assert torch.isnan(out).all()


# --- calls that are allowed and rarely made ----------------------------------------------

@pytest.mark.parametrize("past", [[40, 3], [2900, 700], [50 + 3 * b for b in range(70)]],
                         ids=["short", "merged", "many"])
@pytest.mark.parametrize("T", [1, 10, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_result_in_the_place_of_q(cuda_device, dtype, T, past):
    t = ref.DTYPES[dtype]
    c = ref.Cache(3, dtype, "dense", 64, 2, P, [p + T for p in past])
    K, V, pages = c.to(cuda_device)
    past = torch.tensor(past, dtype=torch.int32, device=cuda_device)
    q = torch.randn(len(past) * T, 8, 64, device=cuda_device).to(t)
    want = lib.paged_attn(q, K, V, pages, past, 0.125)
    assert lib.paged_attn(q, K, V, pages, past, 0.125, out=q) is q
    assert torch.equal(q, want)


@pytest.mark.parametrize("past", [0, 1, 5, 31, 64, 200, 500, 2900])
@pytest.mark.parametrize("T", [1, 4, 10, 70])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "dense"), ("bf16", "mx4"), ("f16", "mx4"),
                                       ("f32", "dense"), ("f32", "mx4")])
def test_a_row_of_nan_leaves_the_others(cuda_device, dtype, fmt, T, past):
    """Queries of NaN and of infinities of either sign: their own rows are NaN, the
    others' as ever but for the rounding of their scores' scaling, which may be another
    one: an error of 2^-23 of scores below 8, of their weights, twice."""
    t = ref.DTYPES[dtype]
    c = ref.Cache(3, dtype, fmt, 64, 2, P, [past + T, 9 + T])
    K, V, pages = c.to(cuda_device)
    past = torch.tensor([past, 9], dtype=torch.int32, device=cuda_device)
    q = torch.randn(2 * T, 4, 64, device=cuda_device).to(t)
    want = lib.paged_attn(q, K, V, pages, past, 0.125)
    bad = torch.zeros(2 * T, 4, dtype=torch.bool, device=cuda_device)
    bad[0, 1] = bad[T - 1, 2] = bad[T, 0] = True
    q[0, 1, 5], q[T - 1, 2, 0::2], q[T - 1, 2, 1::2] = math.nan, math.inf, -math.inf
    q[T, 0] = math.nan
    got = lib.paged_attn(q, K, V, pages, past, 0.125)
    assert torch.isnan(got[bad]).all()
    got, want = got[~bad].double(), want[~bad].double()
    slack = 2 * 8 * 2.0 ** -23 * 4 + 2 * ref.half_step(t)
    assert ((got - want).abs() <= slack * want.abs().max()).all()


@pytest.mark.parametrize("dtype,fmt,d", [("bf16", "dense", 128), ("f32", "mx4", 256),
                                         ("f16", "mx4", 64)])
def test_the_largest_pages(cuda_device, dtype, fmt, d):
    """32768 rows a page: an append at its end, read back, and attention over it."""
    n = 32768
    c = ref.Cache(4, dtype, fmt, d, 1, n, [n - 3, 9], spare=0)
    K, V, pages = c.to(cuda_device)
    past = torch.tensor([n - 3, 9], dtype=torch.int32, device=cuda_device)
    t = ref.DTYPES[dtype]
    k, v, q = (torch.randn(6, h, d, device=cuda_device).to(t) for h in (1, 1, 2))
    lib.paged_append(K, V, pages, past, k, v)
    back = [torch.empty_like(k) for _ in range(2)]
    lib.paged_gather(K, V, pages, past, *back)
    if fmt == "dense":
        assert torch.equal(back[0], k) and torch.equal(back[1], v)
    out = lib.paged_attn(q, K, V, pages, past, 1 / math.sqrt(d))
    want, mass, spread, seen, _, top = ref.attention(
        q.cpu(), K.cpu(), V.cpu(), c.pages.numpy(), [n - 3, 9], 1 / math.sqrt(d), True, None, 3, 1)
    tol = ref.tolerance(want, mass, spread, seen, top, t, d)
    assert (np.abs(out.cpu().double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("T", [1, 4, 12])
@pytest.mark.parametrize("dtype,fmt,pages", [("bf16", "dense", 512), ("f32", "mx4", 512),
                                             ("f16", "mx4", 32768)])
def test_as_many_positions_as_there_are(cuda_device, dtype, fmt, pages, T):
    """Up to 2^30 positions of a sequence, one page of 32768 over and over: the
    attention over that page once.  A wave's sums are chains of at most
    positions / (512 * 4 * 32) additions, each off by 2^-24 of the sum, twice (value and
    divisor); the merges add less; both results are rounded to the type, and the page's
    own result may be off by the bound of its own sums."""
    t, d, n = ref.DTYPES[dtype], 64, 32768
    c = ref.Cache(6, dtype, fmt, d, 1, n, [n], spare=0)
    K, V, _ = c.to(cuda_device)
    q = torch.randn(T, 4, d, device=cuda_device).to(t)
    out = []
    for count in (1, pages):
        table = torch.zeros(1, count, dtype=torch.int32, device=cuda_device)
        past = torch.tensor([count * n], dtype=torch.int32, device=cuda_device)
        print("positions", count * n, flush=True)
        out.append(lib.paged_attn(q, K, V, table, past, 0.125, causal=False).double().cpu())
    largest = float(np.abs(np.nan_to_num(ref.page_rows(c.V, 0, 0, d, True))).max())
    steps = pages * n / (512 * 4 * 32) + n / 16 + 64
    slack = 2 * steps * 2.0 ** -24 * largest + 2 * ref.half_step(t) * largest
    print("off by", float((out[1] - out[0]).abs().max()), "of", slack, flush=True)
    assert (out[1] - out[0]).abs().max() <= slack
