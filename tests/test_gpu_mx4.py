"""Microscaled 4-bit rows against the format's definition in 64 bits:
quantisation bit for bit, lookups bit for bit, products within the rounding of
fp32 sums."""
import threading
import time

import numpy as np
import pytest
import torch

from paper_2206_00470_amd import MX4, Store, _lib, mx4_product, mx4_quantize
from paper_2206_00470_amd.store import interleaved_bf16_tables, interleaved_tables
from tests.helpers import say

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF = {t: torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
TINY = {t: torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2 for t in (F32, BF16, F16)}
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def plain_quantize(x):
    """(codes, scales) of a [rows, dim] float64 array by the definition."""
    rows, dim = x.shape
    nb = -(-dim // 32)
    p = np.zeros((rows, nb * 32))
    p[:, :dim] = x
    p = p.reshape(rows, nb, 32)
    top = np.abs(p).max(axis=2)
    nan = ~np.isfinite(p).all(axis=2)
    t = np.where(nan | (top == 0), 1.0, top)
    s = np.frexp(t)[1] - 1 - 2 + 127
    s = np.where(top == 0, 0, np.clip(s, 0, 254))
    a = np.abs(p) / np.ldexp(1.0, s - 127)[..., None]
    a = np.where(nan[..., None], 0.0, a)
    mid = (GRID[1:] + GRID[:-1]) / 2
    code = np.zeros(a.shape, dtype=np.uint8)
    for k, m in enumerate(mid):   # between codes k and k + 1: the tie goes to the even one
        code += (a > m) | ((a == m) & (k % 2 == 1))
    code |= (np.signbit(p) & ~nan[..., None]).astype(np.uint8) << 3
    code = code.reshape(rows, nb * 32)
    return code[:, 0::2] | code[:, 1::2] << 4, np.where(nan, 255, s).astype(np.uint8)


def plain_values(codes, scales, dim):
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(codes.shape[0], -1)
    v = GRID[c & 7] * np.where(c & 8, -1.0, 1.0)
    f = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return (v.reshape(*scales.shape, 32) * f[..., None]).reshape(codes.shape[0], -1)[:, :dim]


def host(q):
    return q.codes.cpu().numpy(), q.scales.cpu().numpy()


def random_rows(rows, dim, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((rows, dim), generator=g) * torch.exp(torch.randn((rows, 1), generator=g) * spread)


def random_mx4(rows, dim, seed, lo=118, hi=136):
    """Any codes, scales around 1."""
    rng = np.random.default_rng(seed)
    nb = -(-dim // 32)
    codes = rng.integers(0, 256, (rows, 16 * nb), dtype=np.uint8)
    scales = rng.integers(lo, hi, (rows, nb)).astype(np.uint8)
    if dim % 32:   # what lies behind the row is zero
        c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(rows, -1)
        c[:, dim:] = 0
        codes = c[:, 0::2] | c[:, 1::2] << 4
    return MX4(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), dim)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 5), (1, 32), (7, 33), (100, 31), (129, 64), (65, 100), (1000, 300),
                                      (33, 512), (5, 1000), (2, 16384), (2, 16381)])
def test_quantize_bit_for_bit(rows, dim, dtype):
    x = random_rows(rows, dim, dim, spread=3.0).to(dtype)
    codes, scales = plain_quantize(x.double().numpy())
    q = mx4_quantize(x.cuda())
    c, s = host(q)
    assert q.dim == dim and q.rows == rows
    assert np.array_equal(s, scales) and np.array_equal(c, codes)


def test_quantize_borders_and_special_values():
    steps = []
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    for m in mids + list(GRID) + [6.5, 7.0, 7.5, 7.9999995]:
        f = np.float32(m)
        steps += [f, np.nextafter(f, np.float32(9)), np.nextafter(f, np.float32(-1))]
    steps = np.array([v for v in steps if v >= 0], dtype=np.float32)
    rows = []
    for e in (-140, -128, -127, -126, -60, -3, 0, 1, 77, 122, 125):   # scales from the lowest to the highest
        for i in range(0, len(steps), 30):
            r = np.zeros(32, dtype=np.float64)
            part = steps[i:i + 30].astype(np.float64)
            r[:len(part)] = part * np.where(np.arange(len(part)) % 2, -1, 1)
            r[30] = 4.0   # the block's largest: 4 <= max < 8
            rows.append(np.ldexp(r, e))
    x = np.array(rows).astype(np.float32)
    special = np.zeros((8, 32), dtype=np.float32)
    special[1, 3] = np.inf
    special[2, 5] = np.nan
    special[3] = -0.0
    special[4, 0], special[4, 1] = 3.4028235e38, -1.0
    special[5, 7] = 1e-45
    special[6, 7] = 2.0 ** -126
    special[7, 31] = -2.0 ** -125
    x = np.concatenate([x, special])
    codes, scales = plain_quantize(x.astype(np.float64))
    c, s = host(mx4_quantize(torch.from_numpy(x).cuda()))
    assert np.array_equal(s, scales)
    assert np.array_equal(c, codes)
    back = mx4_quantize(torch.from_numpy(x).cuda()).dequantize().cpu().numpy()
    assert np.isnan(back[-7]).all() and np.isnan(back[-6]).all()
    ref = plain_values(codes, scales, 32)
    assert np.array_equal(np.isnan(ref), np.isnan(back)) and np.array_equal(np.nan_to_num(ref), np.nan_to_num(back))


def test_quantize_a_stores_table_as_it_is():
    W0 = random_rows(500, 100, 3).cuda()
    ref = host(mx4_quantize(W0))
    W, G = interleaved_tables(W0)
    assert all(np.array_equal(a, b) for a, b in zip(host(mx4_quantize(Store(W, G).W)), ref))
    Wb, Gb = interleaved_bf16_tables(W0)
    codes, scales = plain_quantize(Wb.double().cpu().numpy())
    c, s = host(mx4_quantize(Store(Wb, Gb).W))
    assert np.array_equal(c, codes) and np.array_equal(s, scales)
    for off, pitch in ((1, 101), (8, 120), (4, 104)):
        wide = torch.zeros((500, pitch + off), device="cuda")
        wide[:, off:off + 100] = W0
        assert all(np.array_equal(a, b) for a, b in zip(host(mx4_quantize(wide[:, off:off + 100])), ref))
    assert mx4_quantize(W0[:0]).dequantize().shape == (0, 100)
    with pytest.raises(TypeError):
        mx4_quantize(W0.t())
    with pytest.raises(TypeError):
        mx4_quantize(W0.double())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("dim", [1, 4, 31, 32, 36, 100, 300, 512, 1001])
def test_mx4_embed_bit_for_bit(dim, dtype):
    q = random_mx4(700, dim, dim, lo=0 if dtype == F32 else 110, hi=255 if dtype == F32 else 140)
    values = torch.from_numpy(plain_values(*host(q), dim))
    exact = values.to(F32)
    # every value is an fp32 number, but 4 and 6 times 2^126 and 2 to 6 times 2^127, which are infinite there
    fits = values.abs() < 2.0 ** 128
    assert torch.equal(exact.double()[fits], values[fits]) and bool(exact[~fits].isinf().all())
    for n in (1, 5, 1029):
        ids = torch.randint(0, 700, (n,), generator=torch.Generator().manual_seed(n))
        ids[2::3] = -5
        got = q.embed(ids.cuda(), scale=1.3, dtype=dtype, pad=-5).cpu()
        ref = (exact[ids.clamp(min=0)] * torch.tensor(1.3)).to(dtype)
        ref[ids == -5] = 0
        assert got.shape == (n, dim) and got.dtype == dtype
        assert torch.equal(got, ref)
    assert torch.equal(q.dequantize(dtype).cpu(), exact.to(dtype))
    assert q.error() == 0


def test_mx4_embed_errors_strides_and_graphs():
    dim = 48
    q = random_mx4(90, dim, 1)
    values = torch.from_numpy(plain_values(*host(q), dim)).float()
    got = q.embed(torch.tensor([3, 90, -1, 89], device="cuda")).cpu()
    assert q.error() == _lib.PS_ERR_KEY_RANGE and q.error() == 0
    assert torch.equal(got[[0, 3]], values[[3, 89]]) and bool((got[[1, 2]] == 0).all())
    ids = torch.randint(0, 90, (77,), device="cuda")
    for pitch, off in ((64, 8), (52, 4), (51, 1)):
        wide = torch.full((77, pitch), 7.0, dtype=BF16, device="cuda")
        q.embed(ids, out=wide[:, off:off + dim])
        assert torch.equal(wide[:, off:off + dim].cpu(), values[ids.cpu()].to(BF16))
        wide[:, off:off + dim] = 7.0
        assert bool((wide == 7.0).all())
    out = torch.empty((77, dim), device="cuda")
    a = random_mx4(5, dim, 2)
    score = torch.empty((5, 90), device="cuda")
    G = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(G):
        q.embed(ids, out=out)
        mx4_product(a, q, out=score)
    for r in range(3):
        ids.random_(0, 90)
        out.fill_(1.0), score.fill_(1.0)
        G.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, q.embed(ids)) and torch.equal(score, mx4_product(a, q))
    fresh = random_mx4(9, dim, 3)
    with pytest.raises(RuntimeError):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            fresh.embed(ids)


def check_product(a, b, dtype, scale, out=None):
    A, B = plain_values(*host(a), a.dim), plain_values(*host(b), b.dim)
    got = mx4_product(a, b, scale=scale, dtype=dtype, out=out)
    f = float(torch.tensor(scale, dtype=F32))
    ref, mag = torch.from_numpy(A @ B.T) * f, torch.from_numpy(np.abs(A) @ np.abs(B).T) * abs(f)
    # exact products added in fp32 in some order: each of the dim additions off by at
    # most 2^-23 (rounded or cut) of the magnitudes so far; the factor's product
    # and the type's rounding once each
    tol = (a.dim + 1) * 2.0 ** -23 * mag + (2.0 ** -24 + HALF[dtype]) * (1 + 2.0 ** -7) * ref.abs() + 2 * TINY[dtype]
    assert got.shape == (a.rows, b.rows) and got.dtype == dtype
    bad = ((got.double().cpu() - ref).abs() > tol).sum()
    assert int(bad) == 0, f"{int(bad)} of {got.numel()} off"
    return got


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("m,n,dim", [(1, 1, 1), (1, 1000, 32), (3, 77, 33), (5, 129, 64), (16, 300, 100), (31, 31, 300),
                                     (32, 4096, 256), (33, 1025, 65), (64, 513, 512), (100, 200, 1000), (257, 383, 96),
                                     (130, 127, 160), (513, 2050, 224), (2, 130, 16384), (129, 140, 2052)])
def test_product(m, n, dim, dtype):
    say(f"product {m} x {n} x {dim} {dtype}")
    check_product(random_mx4(m, dim, 1), random_mx4(n, dim, 2), dtype, 0.7 / dim ** 0.5 * 2.0 ** -8)


def test_product_strides_special_scales_and_order():
    a, b = random_mx4(40, 64, 5), random_mx4(50, 64, 6)
    for pitch, off in ((64, 8), (57, 3)):
        wide = torch.full((40, pitch), 7.0, device="cuda")
        check_product(a, b, F32, 0.5, out=wide[:, off:off + 50])
        wide[:, off:off + 50] = 7.0
        assert bool((wide == 7.0).all())
    # scales at both ends: what is representable is exact, what is not is infinite or zero
    one = lambda s: MX4(torch.full((1, 16), 0x22, dtype=torch.uint8, device="cuda"),
                        torch.full((1, 1), s, dtype=torch.uint8, device="cuda"), 32)
    for s, t in ((0, 127), (127, 127), (254, 0), (254, 127), (0, 254), (1, 127), (60, 200)):
        got = float(mx4_product(one(s), one(t)))
        ref = np.float32(np.ldexp(32.0, s + t - 254)) if s + t - 254 + 5 < 128 else np.inf
        assert got == ref, (s, t, got, ref)
    # a NaN block makes its row NaN and no other
    a.scales[7, 1] = 255
    b.scales[9, 0] = 255
    got = mx4_product(a, b).cpu()
    nan = torch.zeros((40, 50), dtype=torch.bool)
    nan[7], nan[:, 9] = True, True
    assert torch.equal(got.isnan(), nan)
    # the same row has the same scores in any company
    q, t = random_mx4(300, 96, 8), random_mx4(700, 96, 9)
    all_scores = mx4_product(q, t)
    for i in (0, 31, 299):
        alone = mx4_product(MX4(q.codes[i:i + 1].contiguous(), q.scales[i:i + 1].contiguous(), 96), t)
        assert torch.equal(alone[0], all_scores[i])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = mx4_product(q, t, stream=side)
    side.synchronize()
    assert torch.equal(other, all_scores)
    with pytest.raises(ValueError):
        mx4_product(q, b)
    with pytest.raises(ValueError):
        mx4_product(q, t, out=torch.empty((300, 701), device="cuda"))


@pytest.mark.parametrize("m,n,dim,dtype,off", [
    (256, 65_601, 100, F32, 0), (256, 65_601, 100, F32, 3), (259, 131_201, 512, BF16, 0), (300, 120_001, 513, BF16, 0),
    (513, 70_001, 31, F16, 1), (255, 65_901, 64, F32, 0), (2048, 32_768, 64, F32, 0), (2049, 65_600, 33, BF16, 0),
    (2049, 65_601, 300, BF16, 0)])
def test_products_of_every_size_have_the_same_scores(m, n, dim, dtype, off):
    """Large results, their rows whole cache lines or not: the scores are those
    of a few queries at a time (which are checked against 64 bits), and what
    lies around the result stays."""
    say(f"product {m} x {n} x {dim} {dtype}")
    a, b = random_mx4(m, dim, 21), random_mx4(n, dim, 22)
    room = torch.full((m * n + off + 64,), 7.0, dtype=dtype, device="cuda")
    out = room[off:off + m * n].view(m, n)
    mx4_product(a, b, scale=2.0 ** -9, out=out)
    assert bool((room[:off] == 7.0).all()) and bool((room[off + m * n:] == 7.0).all())
    for i in (0, 32, m // 2, m - 20):
        q = MX4(a.codes[i:i + 20].contiguous(), a.scales[i:i + 20].contiguous(), dim)
        assert torch.equal(mx4_product(q, b, scale=2.0 ** -9, dtype=dtype), out[i:i + 20])
    few = MX4(b.codes[n - 40:].contiguous(), b.scales[n - 40:].contiguous(), dim)
    assert torch.equal(check_product(a, few, dtype, 2.0 ** -9), out[:, n - 40:])


def test_a_quantised_table_answers():
    """Scores of a table's own rows: quantise, look queries up, quantise them,
    score them against all rows; each row's best score is its own."""
    rows = random_rows(3000, 128, 11, spread=0.0)
    q = mx4_quantize(rows.cuda())
    ids = torch.arange(0, 3000, 37, device="cuda")
    queries = mx4_quantize(q.embed(ids, dtype=BF16))
    score = check_product(queries, q, F32, 128 ** -0.5)
    assert torch.equal(score.argmax(dim=1), ids)


def test_a_table_used_first_on_two_streams_reports_its_error():
    """The flag that embed makes at its first call is there for every stream."""
    x = mx4_quantize(torch.randn((50, 64), device="cuda"))
    torch.cuda.synchronize()
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    good, bad = torch.arange(50, device="cuda"), torch.full((3,), 50, dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    a = torch.randn((8192, 8192), device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(one):
        b = a @ a                      # the first call's stream is behind
    x.embed(good, stream=one)
    x.embed(bad, stream=two)
    torch.cuda.synchronize()
    assert x.error() == _lib.PS_ERR_KEY_RANGE and x.error() == 0


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("scale", [float("inf"), -float("inf"), float("nan"), -1.0, 1e38, 0.0])
def test_rows_that_are_not_there_are_zeros_whatever_the_factor(scale, dtype):
    """Padding and ids outside the table, as Store.embed gives them: +0 in every bit."""
    dim, word = 45, torch.int32 if dtype == F32 else torch.int16
    W = random_rows(30, dim, 12)
    W[5, 3] = float("inf")                                    # a block of NaN, not looked up by an absent row
    q = mx4_quantize(W.cuda())
    s = Store(W.cuda(), torch.ones((30, dim), device="cuda"))
    ids = torch.tensor([-1, 4, 30, -1, 2 ** 40, 5, -3, -1, 0], device="cuda")
    there = torch.tensor([False, True, False, False, False, True, False, False, True])
    values = q.dequantize().cpu()
    for got in (q.embed(ids, scale=scale, dtype=dtype, pad=-1), s.embed(ids, scale=scale, dtype=dtype, pad=-1)):
        assert not bool(got.view(word)[~there.cuda()].any())
    got = q.embed(ids, scale=scale, dtype=dtype, pad=-1).cpu()[there]
    ref = (values[ids.cpu()[there]] * torch.tensor(scale)).to(dtype)
    assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.nan_to_num(), ref.nan_to_num())
    assert q.error() == _lib.PS_ERR_KEY_RANGE and s.error() == _lib.PS_ERR_KEY_RANGE


def test_a_table_used_first_by_two_threads_reports_its_error():
    """One thread's first lookup waits behind a long stream for its flag, another
    thread's lookup on a stream of its own finds an id outside the table."""
    good, bad = torch.arange(50, device="cuda"), torch.full((3,), 50, dtype=torch.int64, device="cuda")
    a = torch.randn((8192, 8192), device="cuda")
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    for turn in range(3):
        x = mx4_quantize(torch.randn((50, 64), device="cuda"))
        torch.cuda.synchronize()
        with torch.cuda.stream(one):
            for _ in range(4):
                b = a @ a
        first = threading.Thread(target=lambda: x.embed(good, stream=one))
        first.start()
        time.sleep(0.003 * turn)
        got = x.embed(bad, stream=two)
        first.join()
        torch.cuda.synchronize()
        assert not bool(got.any())
        assert x.error() == _lib.PS_ERR_KEY_RANGE and x.error() == 0
