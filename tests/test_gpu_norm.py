"""The norm with the residual's addition, its gradient and rows in 8 bits against their definitions in 64 bits."""
import math

import pytest
import torch

import layers_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
DTYPES = [F32, F16, BF16]
# below a vector, odd, at and beyond every length that a team holds, rows that no team holds
DIMS = [1, 3, 7, 8, 9, 63, 64, 65, 127, 250, 256, 257, 511, 513, 1000, 1024, 1025, 2049, 4096, 4099, 8192, 8195, 16384, 16387, 40001]


def rows_of(dim):
    return 70 if dim <= 2049 else 5


def made(n, d, dtype, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (spread * torch.randn(n, d, generator=g, device="cuda")).to(dtype)


def near(got, want, tol, what):
    far = (got.double() - want).abs()
    assert not torch.isnan(far).any() and (far <= tol).all(), (what, float((far - tol).max()), float(far.max()))


def forward_error(h, weight, want):
    """r is rounded (to the last place of the smallest values where it is so small), and so is each of two products."""
    w = 1.0 if weight is None else weight.double()
    return 3.01 * ref.U24 * want.abs() + ref.BELOW[F32] * (h.double() * w).abs()


def check_forward(x, residual, weight, eps, quantized=True):
    res = cc.cc_rms_norm(x, weight, residual, eps, quantized=quantized, save_rstd=True)
    h = ref.added(x, residual)
    assert torch.equal(res.sum, h)
    want, r = ref.norm(h, weight, eps)
    near(res.out, want, ref.rounded(want, x.dtype, forward_error(h, weight, want)), "out")
    near(res.rstd, r, 1.001 * ref.U24 * r, "rstd")
    if quantized:
        w = 1.0 if weight is None else weight.double()
        q, scale = ref.eight_bits(h.double() * w, r)
        assert torch.equal(res.q.double(), q)
        near(res.scale, scale, 1.001 * ref.U24 * scale + ref.BELOW[F32], "scale")
    return res


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_forward(dim, dtype):
    say(f"norm forward {dim} {dtype}")
    n = rows_of(dim)
    x, residual = made(n, dim, dtype), made(n, dim, dtype, 1, 4.0)
    for weight in (made(1, dim, F32, 2)[0], made(1, dim, dtype, 3)[0], None):
        check_forward(x, residual, weight, 1e-6)
    check_forward(x, None, None, 1e-2, quantized=False)


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("n", [1, 2, 31, 33, 9000, 70001])
def test_numbers_of_rows(n, dtype):
    say(f"norm rows {n} {dtype}")
    check_forward(made(n, 40, dtype), made(n, 40, dtype, 1), made(1, 40, F32, 2)[0], 1e-6)


def check_backward(go, h, weight, eps, grad_sum, **into):
    rstd = ref.norm(h, weight, eps)[1].float()
    grad_h, grad_w = cc.cc_rms_norm_backward(go.clone() if into.get("in_place") == "out" else go, h, rstd, weight, grad_sum)
    want_h, want_w = ref.norm_backward(go, h, weight, rstd, grad_sum)
    w = torch.ones(h.shape[-1], device="cuda", dtype=torch.float64) if weight is None else weight.double()
    s, normed = rstd.double().unsqueeze(-1), (h.double() * rstd.double().unsqueeze(-1)).abs()
    term = (go.double() * w).abs()
    # the mean: a term is of four roundings, a thread adds at most 64 and what it adds up is added in 64 bits
    mean = (term * normed).mean(-1, keepdim=True)
    # a product rounded, that of h and r twice over, the outer sum, the stream's part
    error = ref.U24 * (s * (normed * 72 * mean + 3 * normed * mean + 3 * term) + 2 * want_h.abs())
    near(grad_h, want_h, ref.rounded(want_h, h.dtype, error), "grad_h")
    if weight is not None:
        # at most 128 additions one after the other up to 4096 rows (rows of a team, teams, workgroups, wavefronts), two roundings a term
        error = 130 * ref.U24 * (go.double() * h.double() * s).abs().flatten(0, -2).sum(0)
        near(grad_w, want_w, ref.rounded(want_w, weight.dtype, error), "grad_weight")
    else:
        assert grad_w is None
    return grad_h, grad_w


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_backward(dim, dtype):
    say(f"norm backward {dim} {dtype}")
    n = rows_of(dim)
    h, go, gs = made(n, dim, dtype, 0, 3.0), made(n, dim, dtype, 1), made(n, dim, dtype, 2)
    check_backward(go, h, made(1, dim, F32, 3)[0], 1e-6, gs)
    check_backward(go, h, made(1, dim, dtype, 4)[0], 1e-6, None)
    check_backward(go, h, None, 1e-6, gs)


@pytest.mark.parametrize("n", [1, 2, 5, 127, 129, 4096])
@pytest.mark.parametrize("dim", [5, 24, 130, 700])
def test_backward_numbers_of_rows(n, dim):
    say(f"norm backward rows {n} {dim}")
    check_backward(made(n, dim, BF16, 1), made(n, dim, BF16, 0), made(1, dim, F32, 3)[0], 1e-6, None)


def test_backward_by_differences():
    """Along a random direction, of a loss in 64 bits of the call's own outputs: fp32 outputs are off by 3 U24 |out|, so a difference over
    2 step is off by at most that times |grad_out| / step, and its curvature by step^2."""
    n, d, eps, step = 4, 96, 1e-2, 2.0 ** -6
    x, w, go = made(n, d, F32), made(1, d, F32, 1)[0], made(n, d, F32, 2)
    direction = made(n, d, F32, 3)
    plus, minus = x + step * direction, x - step * direction
    real = ((plus.double() - minus.double()) / (2 * step))              # what was added, rounded as it is
    outs = [cc.cc_rms_norm(t, w, eps=eps).out.double() for t in (plus, minus)]
    slope = float(((outs[0] - outs[1]) * go.double()).sum() / (2 * step))
    rstd = cc.cc_rms_norm(x, w, eps=eps, save_rstd=True).rstd
    grad = cc.cc_rms_norm_backward(go, x, rstd, w)[0].double()
    rounding = float((3 * ref.U24 * (outs[0].abs() + outs[1].abs()) * go.double().abs()).sum() / (2 * step))
    # the same difference in 64 bits says what the curvature does
    exact = [ref.norm(t, w, eps)[0] for t in (plus, minus)]
    curved = float(((exact[0] - exact[1]) * go.double()).sum() / (2 * step) - (ref.norm_backward(go, x, w, rstd, None)[0] * real).sum())
    assert abs(slope - float((grad * real).sum()) - curved) <= rounding + 100 * ref.U24 * float((grad.abs() * real.abs()).sum())


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("dim", [64, 251, 1021, 5000, 20001])
def test_strided_rows_and_places(dim, dtype):
    """Rows apart, at any element, into rows apart that keep what lies between them; sum over x, over the residual."""
    say(f"norm strided {dim} {dtype}")
    n = 9
    base = made(n, 2 * dim + 5, dtype)
    x, residual = base[:, 1:dim + 1], base[:, dim + 3:2 * dim + 3]
    weight = made(1, dim + 1, F32, 2)[0, 1:]
    want = cc.cc_rms_norm(x.contiguous(), weight.contiguous(), residual.contiguous(), quantized=True, save_rstd=True)
    room = torch.full((n, dim + 3), 7.0, device="cuda", dtype=dtype)
    sums, qs = room.clone(), torch.full((n, dim + 3), 77, device="cuda", dtype=torch.int8)
    res = cc.cc_rms_norm(x, weight, residual, out=room[:, 2:dim + 2], sum=sums[:, 1:dim + 1], q=qs[:, 3:], quantized=True, save_rstd=True)
    for got, expected in ((room[:, 2:dim + 2], want.out), (sums[:, 1:dim + 1], want.sum), (qs[:, 3:], want.q), (res.scale, want.scale), (res.rstd, want.rstd)):
        assert torch.equal(got, expected)
    assert (room[:, :2] == 7).all() and (room[:, dim + 2:] == 7).all() and (sums[:, 0] == 7).all() and (qs[:, :3] == 77).all()
    for place in ("x", "residual"):
        xs, rs = x.clone().contiguous(), residual.clone().contiguous()
        into = xs if place == "x" else rs
        got = cc.cc_rms_norm(xs, weight, rs, sum=into)
        assert got.sum is into and torch.equal(into, want.sum) and torch.equal(got.out, want.out)
    go, gs = made(n, dim, dtype, 5), made(n, dim, dtype, 6)
    grad, gw = cc.cc_rms_norm_backward(go, want.sum, want.rstd, weight, gs)
    a, b = go.clone(), gs.clone()
    got = cc.cc_rms_norm_backward(a, sums[:, 1:dim + 1], want.rstd, weight, gs, grad_h=a)
    assert torch.equal(a, grad) and torch.equal(got[1], gw)
    cc.cc_rms_norm_backward(go, want.sum, want.rstd, weight, b, grad_h=b)
    assert torch.equal(b, grad)
    acc = torch.full((dim,), 2.0, device="cuda")
    cc.cc_rms_norm_backward(go, want.sum, want.rstd, weight, gs, grad_weight=acc, accumulate=True)
    assert torch.equal(acc, gw + 2.0)


def test_undefined_zero_and_extreme_rows():
    d = 300
    for dtype in DTYPES:
        top = torch.finfo(dtype).max
        x = made(8, d, dtype)
        x[0] = 0
        x[1, 17] = math.inf
        x[2, 299] = math.nan
        x[3, 0] = -math.inf
        x[4] = torch.finfo(dtype).tiny
        x[5] = top
        x[6] = torch.finfo(dtype).smallest_normal / 8
        res = cc.cc_rms_norm(x, None, eps=1e-12, quantized=True, save_rstd=True)
        assert (res.q[0] == 0).all() and res.scale[0] == 0 and (res.out[0] == 0).all()
        for bad in (1, 2, 3):
            assert (res.q[bad] == 0).all() and torch.isnan(res.scale[bad]) and torch.isnan(res.out[bad]).any()
        good = [4, 5, 7]
        if dtype is not F32:
            good.append(6)
        want, r = ref.norm(x[good], None, 1e-12)
        near(res.out[good], want, ref.rounded(want, dtype, forward_error(x[good], None, want)), "out")
        assert (res.q[5] == 127).all()                  # squares beyond 32 bits
        q, scale = cc.cc_quantize_rows(x)
        assert (q[0] == 0).all() and scale[0] == 0 and (q[5] == 127).all() and torch.isnan(scale[1:4]).all() and (q[1:4] == 0).all()
        assert (q[4] == 127).all() and (q[6] == 127).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("dim", DIMS)
def test_quantize(dim, dtype):
    say(f"quantize {dim} {dtype}")
    n = rows_of(dim)
    x = made(n, dim, dtype) * torch.exp(3 * made(n, 1, F32, 5)).to(dtype)
    q, scale = cc.cc_quantize_rows(x)
    want, step = ref.eight_bits(x.double(), 1.0)
    assert torch.equal(q.double(), want)
    near(scale, step, 1.001 * ref.U24 * step + ref.BELOW[F32], "scale")
    wide = torch.full((n, dim + 5), 3, device="cuda", dtype=torch.int8)
    apart = torch.zeros(n, dim + 3, device="cuda", dtype=dtype)
    apart[:, 2:dim + 2] = x
    cc.cc_quantize_rows(apart[:, 2:dim + 2], q=wide[:, 1:dim + 1])
    assert torch.equal(wide[:, 1:dim + 1], q) and (wide[:, 0] == 3).all() and (wide[:, dim + 1:] == 3).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_quotients_on_borders(dtype):
    """Every multiple of half a step and its neighbours in the type, with each of some sizes of the largest."""
    halves = torch.arange(-253, 254, device="cuda").float() / 254
    rows = []
    for most in (1.0, 254.0, 127.0, 1.5, 0.1, 3.1415926, 96.0, 2.0 ** -13):
        base = (halves * most).to(dtype)
        up, down = torch.nextafter(base.cpu(), torch.tensor(9e9).to(dtype)).cuda(), torch.nextafter(base.cpu(), torch.tensor(-9e9).to(dtype)).cuda()
        row = torch.cat([base, up, down]).clamp(-most, most)
        row[0] = most
        rows.append(row)
    x = torch.stack(rows)
    assert torch.equal(cc.cc_quantize_rows(x)[0].double(), ref.eight_bits(x.double(), 1.0)[0])
    for weight in (torch.full((x.shape[1],), 3.0, device="cuda"), made(1, x.shape[1], F32, 9)[0]):
        res = cc.cc_rms_norm(x, weight, quantized=True)
        assert torch.equal(res.q.double(), ref.eight_bits(x.double() * weight.double(), 1.0)[0])


def test_products_beyond_32_bits():
    x = torch.tensor([[1e30, -3e30, 2e29, 0.0], [1e-30, 2e-30, 5e-31, 0.0], [1e-44, 3e-44, 0.0, 0.0]], device="cuda")
    weight = torch.tensor([1e25, 2e25, 1e25, 1.0], device="cuda")
    for w in (weight, 1e-35 / weight):
        res = cc.cc_rms_norm(x, w.contiguous(), eps=1e-30, normed=False, quantized=True)
        assert torch.equal(res.q.double(), ref.eight_bits(x.double() * w.double(), 1.0)[0])
        assert res.out is None


def test_nothing_and_shapes():
    w = made(1, 6, F32)[0]
    res = cc.cc_rms_norm(torch.empty(0, 6, device="cuda"), w, quantized=True, save_rstd=True)
    assert res.out.shape == (0, 6) and res.q.shape == (0, 6) and res.scale.shape == (0,)
    grad_h, grad_w = cc.cc_rms_norm_backward(res.out, res.out, res.rstd, w)
    assert grad_h.shape == (0, 6) and (grad_w == 0).all()
    keep = torch.full((6,), 5.0, device="cuda")
    cc.cc_rms_norm_backward(res.out, res.out, res.rstd, w, grad_weight=keep, accumulate=True)
    assert (keep == 5).all()
    x = made(6, 6, BF16).view(2, 3, 6)
    res = cc.cc_rms_norm(x, w, x, quantized=True, save_rstd=True)
    assert res.out.shape == x.shape and res.scale.shape == (2, 3) and res.rstd.shape == (2, 3)
    flat = cc.cc_rms_norm(x.view(6, 6), w, x.view(6, 6), quantized=True)
    assert torch.equal(res.out.view(6, 6), flat.out) and torch.equal(res.q.view(6, 6), flat.q)
    one = cc.cc_rms_norm(x[0, 0], w, quantized=True)
    assert one.scale.shape == () and one.out.shape == (6,)


def test_the_same_bits_again():
    for dim in (250, 3000, 20000):
        x, go, w = made(4000 if dim < 3000 else 100, dim, BF16), made(4000 if dim < 3000 else 100, dim, BF16, 1), made(1, dim, F32, 2)[0]
        rstd = cc.cc_rms_norm(x, w, save_rstd=True).rstd
        first = cc.cc_rms_norm_backward(go, x, rstd, w)
        for _ in range(3):
            assert all(torch.equal(a, b) for a, b in zip(first, cc.cc_rms_norm_backward(go, x, rstd, w)))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("dim", [5, 64, 513, 1025, 1500, 2048, 2049, 4097, 8193, 16384, 16400])
def test_a_workspace_is_as_large_as_it_says(dim, dtype):
    """What lies right behind it stays: with so many rows that every workgroup there can be leaves its sums."""
    say(f"norm workspace {dim} {dtype}")
    n = 9000 if dim <= 2049 else 3000
    h, go, w = made(n, dim, dtype), made(n, dim, dtype, 1), made(1, dim, F32, 2)[0]
    rstd = cc.cc_rms_norm(h, w, save_rstd=True, normed=False).rstd
    need = cc.cc_rms_norm_workspace_bytes(n, dim)
    room = torch.full((need + (32 << 20),), 0x5A, dtype=torch.uint8, device="cuda")
    got = cc.cc_rms_norm_backward(go, h, rstd, w, workspace=room[:need])
    assert (room[need:] == 0x5A).all()
    want = cc.cc_rms_norm_backward(go, h, rstd, w)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("dim", [1, 3, 8, 9, 24, 63, 64, 100, 300, 768, 1021, 1024, 1536, 2050, 5120, 8195, 16384, 16387])
def test_an_infinity_in_any_column(dim, dtype):
    """r is zero wherever in a row an infinity stands: zeros, undefined at the infinity alone, and the gradient of its column's weight alone."""
    say(f"norm infinity {dim} {dtype}")
    columns = sorted({0, dim // 2, *range(max(0, dim - 9), dim)})
    x, residual, weight = made(len(columns) + 1, dim, dtype), made(len(columns) + 1, dim, dtype, 1), made(1, dim, F32, 2)[0]
    for i, column in enumerate(columns):
        if i % 2:
            x[i, column] = -math.inf
        else:
            x[i, column] = residual[i, column] = torch.finfo(dtype).max         # their sum is infinite
    res = cc.cc_rms_norm(x, weight, residual, quantized=True, save_rstd=True)
    h = ref.added(x, residual)
    at = torch.tensor(columns, device="cuda")
    want = torch.zeros(len(columns), dim, device="cuda", dtype=dtype)
    want[torch.arange(len(columns), device="cuda"), at] = math.nan
    assert torch.equal(res.sum, h) and torch.isinf(h[:-1].gather(1, at[:, None])).all()
    assert (res.rstd[:-1] == 0).all() and torch.equal(torch.isnan(res.out[:-1]), torch.isnan(want)) and torch.equal(res.out[:-1].nan_to_num(), want.nan_to_num())
    assert (res.q[:-1] == 0).all() and torch.isnan(res.scale[:-1]).all()
    last, r = ref.norm(h[-1:], weight, 1e-6)
    near(res.out[-1:], last, ref.rounded(last, dtype, forward_error(h[-1:], weight, last)), "out")
    near(res.rstd[-1:], r, 1.001 * ref.U24 * r, "rstd")
    go = made(len(columns) + 1, dim, dtype, 3)
    grad_weight = cc.cc_rms_norm_backward(go, h, res.rstd, weight)[1]
    touched = torch.zeros(dim, device="cuda", dtype=torch.bool)
    touched[at] = True
    assert torch.equal(torch.isnan(grad_weight), touched)
    # of the other columns' terms all but the last row's are zero: two roundings
    want = (go[-1].double() * h[-1].double() * res.rstd[-1].double())[~touched]
    near(grad_weight[~touched], want, ref.rounded(want, F32, 2.01 * ref.U24 * want.abs()), "grad_weight")


# u = c d, the row's largest a b, all four below 2^24; the quotient is so near to a border that 127 u rounded to 64 bits lies on it or beyond
NEAR_BORDERS = [(12050691, 15466566, 12431225, 16776439), (15058646, 12249475, 13652353, 16264741), (10140597, 9095033, 9117779, 16576039),
                (13338359, 16422241, 15533163, 15919379), (15910822, 14294319, 14837975, 16567131), (10766781, 10601041, 8729795, 14253061),
                (13761129, 12186782, 12433791, 14455227), (16383889, 14128151, 14536913, 16643995), (15583471, 14832691, 15567679, 15912765),
                (9712573, 9416399, 6450767, 14347221), (14478006, 10004271, 9616069, 16562213), (14300846, 10685011, 12676981, 14934845)]


def whole_nearest(top, bottom):
    """The whole number nearest to top / bottom, ties to even, in whole numbers."""
    low, rest = divmod(top, bottom)
    return low + (2 * rest > bottom or (2 * rest == bottom and low % 2 == 1))


@pytest.mark.parametrize("size", [0, -80, 40], ids=str)
@pytest.mark.parametrize("numbers", NEAR_BORDERS, ids=lambda n: str(n[0]))
def test_products_of_32_bits_next_to_borders(numbers, size):
    """Both signs, and the same smaller and larger by powers of two, where 32 bits do not hold the product."""
    c, d, a, b = numbers
    want = whole_nearest(127 * c * d, a * b)
    for dim in (5, 700, 17000):
        x, w = torch.zeros(1, dim, device="cuda"), torch.ones(dim, device="cuda")
        scaled = 2.0 ** size
        x[0, 0], x[0, 1], x[0, dim - 2] = a * scaled, c * scaled, -c * scaled
        w[0], w[1], w[dim - 2] = b * scaled, d * scaled, d * scaled
        q = cc.cc_rms_norm(x, w, normed=False, quantized=True).q[0]
        assert [int(q[i]) for i in (0, 1, dim - 2, dim - 1)] == [127, want, -want, 0]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("n,dim", [(70001, 40), (40000, 250), (9001, 700), (3001, 2500), (1500, 5000), (1500, 16384), (130, 16400), (1003, 16400)])
def test_weights_gradient_of_several_rows_a_team(n, dim, dtype):
    """More rows than the teams of all workgroups: 3 to 10 of each, and of rows that no team holds 5 and 32 of each part.  One after the other are
    added these, at most 32 teams, 16 partial sums a lane, 2 lanes and 16 wavefronts: no more than check_backward's 128."""
    say(f"norm backward teams {n} {dim} {dtype}")
    h, go = made(n, dim, dtype, 0, 3.0), made(n, dim, dtype, 1)
    # rows that differ, so that one left out or taken twice shows
    h *= (1 + torch.arange(n, device="cuda") % 7).to(dtype).unsqueeze(1)
    check_backward(go, h, made(1, dim, F32, 3)[0], 1e-6, None)
