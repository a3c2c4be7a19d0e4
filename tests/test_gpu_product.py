"""Products of rows in 8 bits against their definition: the sums are exact, so a result is off by its roundings alone."""
import pytest
import torch

import layers_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def eight(rows, k, seed, full=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if full:
        return torch.randint(-128, 128, (rows, k), generator=g, device="cuda", dtype=torch.int64).to(torch.int8)
    return (32 * torch.randn(rows, k, generator=g, device="cuda")).round().clamp(-127, 127).to(torch.int8)


def scales(rows, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return 0.01 * torch.exp(torch.randn(rows, generator=g, device="cuda"))


def check(got, x, xs, w, ws, bias, dtype):
    want = ref.product(x, xs, w, ws, None)
    # the sum rounded and two products of it; the bias's sum
    error = 3.01 * ref.U24 * want.abs()
    if bias is not None:
        want = want + bias.double()
        error = error + ref.U24 * (want.abs() + error)
    assert got.dtype is dtype
    far = (got.double() - want).abs()
    tol = ref.rounded(want, dtype, error)
    assert (far <= tol).all(), float((far - tol).max())


def case(m, n, k, dtype=F32, bias=True, full=True, seed=0):
    x, w, xs, ws = eight(m, k, seed, full), eight(n, k, seed + 1, full), scales(m, seed + 2), scales(n, seed + 3)
    b = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(seed + 4), device="cuda") if bias else None
    return x, xs, w, ws, b


# every kernel on both sides of its lines: few rows, tiles of each size, rows at 16 bytes and not, pieces and tiles that end inside a row
SIZES = [(1, 1, 1), (1, 16, 64), (2, 17, 15), (3, 5, 16), (8, 64, 130), (16, 100, 512), (16, 1000, 4096), (16, 33, 577), (17, 40, 1000),
         (32, 255, 2048), (31, 513, 100), (33, 64, 128), (33, 1, 7), (64, 64, 128), (65, 66, 129), (64, 64, 256), (100, 130, 384), (128, 128, 400),
         (200, 300, 250), (257, 255, 640), (1024, 64, 128), (777, 1001, 250), (1500, 1700, 96), (2048, 1792, 272), (1800, 2050, 129), (4096, 4096, 640),
         (4000, 4100, 144), (4100, 3999, 1000), (3840, 4096, 16),
         # stretches of K, of rows that begin anywhere too; wide heads for few rows; tiles of 128 where those of 256 leave a round half empty
         (64, 64, 2048), (70, 3, 4096), (300, 301, 3001), (40, 700, 9000), (512, 512, 2176), (16, 16384, 200), (9, 20001, 1001), (20, 17000, 640),
         (5000, 5000, 640), (4500, 4700, 1153), (8192, 2100, 1024)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_sizes(m, n, k):
    say(f"product {m} {n} {k}")
    dtype = (F32, F16, BF16)[(m + n + k) % 3]
    args = case(m, n, k)
    check(cc.cc_product_i8(*args, dtype=dtype), *args, dtype)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=str)
@pytest.mark.parametrize("m,n,k", [(5, 50, 70), (20, 50, 128), (70, 90, 200), (300, 2300, 256), (4096, 4000, 256)])
def test_types_and_no_bias(m, n, k, dtype):
    say(f"product types {m} {n} {k} {dtype}")
    x, xs, w, ws, _ = case(m, n, k, full=False)
    check(cc.cc_product_i8(x, xs, w, ws, dtype=dtype), x, xs, w, ws, None, dtype)


@pytest.mark.parametrize("m,n,k", [(4, 40, 131071), (70, 65, 131071), (130, 140, 131056)])
def test_largest_sums(m, n, k):
    """All of -128: the largest sum that K admits."""
    say(f"product largest {m} {n} {k}")
    x = torch.full((m, k), -128, device="cuda", dtype=torch.int8)
    w = torch.full((n, k), -128, device="cuda", dtype=torch.int8)
    w[1::2] = 127
    one = torch.ones(max(m, n), device="cuda")
    out = cc.cc_product_i8(x, one[:m], w, one[:n])
    assert (out[:, ::2] == float(torch.tensor(16384 * k, dtype=torch.float64).float())).all()
    assert (out[:, 1::2] == float(torch.tensor(-16256 * k, dtype=torch.float64).float())).all()


@pytest.mark.parametrize("m,n,k", [(7, 70, 130), (40, 100, 200), (250, 300, 384), (2000, 2000, 130), (4100, 4100, 256)])
@pytest.mark.parametrize("by", [0, 1, 16])
def test_strided_rows(m, n, k, by):
    """Rows apart, at any byte, into rows apart that keep what lies between them."""
    say(f"product strided {m} {n} {k} {by}")
    x, xs, w, ws, b = case(m, n, k)
    width = (k + 15) // 16 * 16 + 32
    xa, wa = (torch.full((r, width), 99, device="cuda", dtype=torch.int8) for r in (m, n))
    xa[:, by:by + k], wa[:, by:by + k] = x, w
    out = torch.full((m, n + 7), 5.0, device="cuda", dtype=BF16)
    cc.cc_product_i8(xa[:, by:by + k], xs, wa[:, by:by + k], ws, b, out=out[:, 3:n + 3])
    want = cc.cc_product_i8(x, xs, w, ws, b, dtype=BF16)
    assert torch.equal(out[:, 3:n + 3], want) and (out[:, :3] == 5).all() and (out[:, n + 3:] == 5).all()


@pytest.mark.parametrize("m,n,k", [(8, 30000, 700), (20, 31007, 513), (3, 60000, 130), (2, 131072, 65), (5, 4000, 1500), (7, 8100, 1100)])
def test_few_rows_of_wide_heads(m, n, k):
    """Wavefronts by themselves and in eights, with a channel's K shared and not."""
    say(f"product wide {m} {n} {k}")
    args = case(m, n, k)
    check(cc.cc_product_i8(*args, dtype=F16), *args, F16)


@pytest.mark.parametrize("m,n", [(5, 37), (30, 300), (40, 70)])
def test_ends_of_rows(m, n):
    """Rows that begin at every byte of a word, of every length near the ends of pieces, words, steps and batches of steps."""
    for k in (*range(14, 40), *range(60, 70), *range(127, 134), *range(253, 262), *range(509, 517), *range(1020, 1031)):
        say(f"product ends {m} {n} {k}")
        args = case(m, n, k, seed=k)
        check(cc.cc_product_i8(*args, dtype=F32), *args, F32)


@pytest.mark.parametrize("m,n,k", [(8, 8000, 4001), (32, 600, 3333), (17, 20000, 1003), (1, 40, 9001)])
@pytest.mark.parametrize("by", [0, 1, 2, 3, 4])
def test_few_rows_at_any_byte(m, n, k, by):
    say(f"product few rows at byte {m} {n} {k} {by}")
    x, xs, w, ws, b = case(m, n, k)
    xa, wa = torch.full((m, k + by), 99, device="cuda", dtype=torch.int8), torch.full((n, k + 4), 99, device="cuda", dtype=torch.int8)
    xa[:, by:], wa[:, 4 - by:k + 4 - by] = x, w
    check(cc.cc_product_i8(xa[:, by:], xs, wa[:, 4 - by:k + 4 - by], ws, b), x, xs, w, ws, b, F32)


@pytest.mark.parametrize("m,n,k", [(40, 60, 68), (64, 64, 2052), (300, 300, 412), (2048, 1792, 276), (4096, 4096, 644), (4000, 4100, 1036)])
def test_rows_at_words(m, n, k):
    """Tiles of each size, straight from rows that begin at words of 4 bytes."""
    say(f"product rows at words {m} {n} {k}")
    args = case(m, n, k)
    check(cc.cc_product_i8(*args, dtype=BF16), *args, BF16)
    rows = torch.full((m, k + 8), 99, device="cuda", dtype=torch.int8)
    rows[:, 4:k + 4] = args[0]
    assert torch.equal(cc.cc_product_i8(rows[:, 4:k + 4], *args[1:]), cc.cc_product_i8(*args))


def test_rows_far_apart():
    """Rows of a tile more than 2^32 bytes apart from its first."""
    say("product far rows")
    k, apart = 128, 1 << 25
    x, xs, w, ws, b = case(140, 150, k)
    far = torch.zeros(140 * apart, device="cuda", dtype=torch.int8).view(140, apart)
    far[:, 16:16 + k] = x
    assert torch.equal(cc.cc_product_i8(far[:, 16:16 + k], xs, w, ws, b), cc.cc_product_i8(x, xs, w, ws, b))


@pytest.mark.parametrize("apart", [(1 << 23) - 16, (1 << 23) - 1, 1 << 23])
@pytest.mark.parametrize("which", ["x", "w"])
def test_rows_of_a_large_tile_apart(which, apart):
    """256 rows of a tile whose offsets just fit into 31 bits, straight and through registers, and those that do not."""
    say(f"product large tile apart {which} {apart}")
    m, n, k = (2048, 8192, 640) if which == "x" else (8192, 2048, 640)
    x, xs, w, ws, b = case(m, n, k)
    want = cc.cc_product_i8(x, xs, w, ws, b, dtype=BF16)
    rows = torch.empty(2048 * apart, device="cuda", dtype=torch.int8).view(2048, apart)[:, 16:16 + k]
    rows.copy_(x if which == "x" else w)
    got = cc.cc_product_i8(rows, xs, w, ws, b, dtype=BF16) if which == "x" else cc.cc_product_i8(x, xs, rows, ws, b, dtype=BF16)
    assert torch.equal(got, want)


def test_undefined_rows_stay_theirs():
    for m, n, k in ((5, 40, 64), (90, 40, 64)):
        x, xs, w, ws, b = case(m, n, k)
        want = cc.cc_product_i8(x, xs, w, ws, b)
        xs[2] = float("nan")
        ws[3] = float("inf")
        got = cc.cc_product_i8(x, xs, w, ws, b)
        keep_m, keep_n = [i for i in range(m) if i != 2], [i for i in range(n) if i != 3]
        assert torch.isnan(got[2]).all() and torch.equal(got[keep_m][:, keep_n], want[keep_m][:, keep_n])
        assert not torch.isfinite(got[:, 3]).any()


def test_nothing_and_shapes():
    x, xs, w, ws, b = case(6, 10, 20)
    assert cc.cc_product_i8(x[:0], xs[:0], w, ws, b).shape == (0, 10)
    assert cc.cc_product_i8(x, xs, w[:0], ws[:0]).shape == (6, 0)
    for m in (6, 70):
        none = torch.empty(m, 0, device="cuda", dtype=torch.int8)
        got = cc.cc_product_i8(none, torch.ones(m, device="cuda"), torch.empty(10, 0, device="cuda", dtype=torch.int8), ws, b)
        assert torch.equal(got, b.expand(m, 10))
    got = cc.cc_product_i8(x.view(2, 3, 20), xs.view(2, 3), w, ws, b)
    assert torch.equal(got.view(6, 10), cc.cc_product_i8(x, xs, w, ws, b))
    assert cc.cc_product_i8(x[0], xs[0], w, ws).shape == (10,)


def test_the_same_bits_again():
    for m, n, k in ((8, 300, 1024), (300, 300, 4096), (4096, 4096, 512)):
        args = case(m, n, k)
        first = cc.cc_product_i8(*args, dtype=F32)
        for _ in range(3):
            assert torch.equal(first, cc.cc_product_i8(*args, dtype=F32))


@pytest.mark.parametrize("m,n,k", [(64, 64, 2048), (33, 1000, 4100), (300, 301, 9001)])
def test_a_workspace_is_as_large_as_it_says(m, n, k):
    say(f"product workspace {m} {n} {k}")
    args = case(m, n, k)
    need = cc.cc_product_i8_workspace_bytes(m, n, k)
    assert need > 0
    room = torch.full((need + (16 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    got = cc.cc_product_i8(*args, workspace=room[:need])
    assert (room[need:] == 0x5A).all() and torch.equal(got, cc.cc_product_i8(*args))
    with pytest.raises(cc.CCError):
        cc.cc_product_i8(*args, workspace=room[:need - 256])


@pytest.mark.parametrize("m,n,k", [(5, 40, 64), (20, 17000, 130), (64, 64, 2048), (90, 130, 200), (300, 301, 1001), (2000, 2000, 130), (4096, 4096, 640)])
@pytest.mark.parametrize("large", ["x", "w"])
def test_scales_that_one_product_does_not_hold(m, n, k, large):
    """The sum times one scale may lie beyond 32 bits where the result does not: rows of the largest values times channels of the smallest, and
    the other way round; one row is ordinary."""
    say(f"product scales {m} {n} {k} {large}")
    x, xs, w, ws, b = case(m, n, k)
    up, down = 2.0 ** 124, 2.0 ** -124
    xs, ws = (xs * up, ws * down) if large == "x" else (xs * down, ws * up)
    xs[m // 2] = 2.0 ** -24
    for bias in (None, b):
        check(cc.cc_product_i8(x, xs, w, ws, bias), x, xs, w, ws, bias, F32)


@pytest.mark.parametrize("far", ["x", "w", "both"])
@pytest.mark.parametrize("k,by", [(7, 0), (16, 3), (128, 1), (129, 0), (129, 5), (401, 16), (641, 1), (1153, 4), (1153, 7)])
def test_rows_far_apart_of_any_length(k, by, far):
    """Offsets of 64 bits inside a tile: rows shorter than a piece, K that ends inside a tile, several tiles on their way, rows at any byte."""
    say(f"product far rows {k} {by} {far}")
    m, n, apart = 70, 65, (1 << 23) + 16 * 3 + by % 2
    x, xs, w, ws, b = case(m, n, k, seed=k)

    def spread(t):
        rows = torch.full((t.shape[0] * apart,), 99, device="cuda", dtype=torch.int8).view(t.shape[0], apart)[:, by:by + k]
        return rows.copy_(t)

    got = cc.cc_product_i8(spread(x) if far != "w" else x, xs, spread(w) if far != "x" else w, ws, b)
    check(got, x, xs, w, ws, b, F32)
    assert torch.equal(got, cc.cc_product_i8(x, xs, w, ws, b))
