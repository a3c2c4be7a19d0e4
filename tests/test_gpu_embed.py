"""Embedding lookup and its gradient against the definition in 64 bits."""
import pytest
import torch

import order_model_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say
from order_model_reference import DTYPES, U, finish, within

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


def make(v, d, n, dtype, seed=0, spread="even"):
    g = torch.Generator().manual_seed(seed)
    table = torch.randn(v, d, generator=g).to(dtype)
    grad = torch.randn(n, d, generator=g).to(dtype)
    if spread == "one":
        ids = torch.full((n,), v // 2, dtype=torch.int32)
    elif spread == "none":
        ids = torch.full((n,), -1, dtype=torch.int32)
    else:
        u = torch.rand(n, generator=g, dtype=torch.float64)
        ids = ((u if spread == "even" else u ** 6) * v).to(torch.int32)
        ids[torch.rand(n, generator=g) < 0.05] = -1
        ids[torch.rand(n, generator=g) < 0.02] = v              # just outside, and far
        ids[torch.rand(n, generator=g) < 0.02] = -(2 ** 31)
    return table, grad, ids


def check(v, d, n, name, spread="even", scale=1.5, seed=0):
    say(f"embed v={v} d={d} n={n} {name} {spread}")
    dtype = DTYPES[name]
    table, grad, ids = make(v, d, n, dtype, seed, spread)
    out = cc.cc_embed(table.cuda(), ids.cuda(), scale)
    want = ref.embed(table, ids, scale)
    within(out, want, finish(want, want.abs() * U, dtype), "rows")
    want, err = ref.embed_backward(grad, ids, v, scale)
    got = cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, scale)
    within(got, want, finish(want, err, dtype), "gradient")
    wide = torch.full((v, d), 7.0, device="cuda")
    cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, scale, grad_table=wide)
    within(wide, want, finish(want, err, torch.float32), "gradient in 32 bits")
    assert torch.equal(cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, scale), got)


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v,d,n", [(1, 1, 1), (2, 3, 1), (8, 8, 64), (65, 33, 1000), (64, 64, 33), (1024, 128, 32), (1025, 250, 4097),
                                   (7, 129, 5000), (3000, 17, 100), (300, 520, 700), (5, 2050, 40)])
def test_sizes(v, d, n, name):
    check(v, d, n, name)


@pytest.mark.parametrize("spread", ["one", "none", "steep"])
@pytest.mark.parametrize("v,d,n", [(9, 40, 20000), (2048, 8, 9000), (70000, 12, 5000), (2100000, 2, 6000)])
def test_frequent_rare_and_absent_ids(v, d, n, spread):
    check(v, d, n, "bf16", spread)


def test_many_tiles_and_segments():
    check(40, 16, 150000, "f32", "steep")
    check(5000, 16, 150000, "f16")


def test_no_tokens():
    ids = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert cc.cc_embed(torch.ones(4, 8, device="cuda"), ids).shape == (0, 8)
    got = cc.cc_embed_backward(torch.zeros(0, 8, device="cuda"), ids, 4)
    assert torch.equal(got, torch.zeros(4, 8, device="cuda"))
    kept = torch.ones(4, 8, device="cuda")
    cc.cc_embed_backward(torch.zeros(0, 8, device="cuda"), ids, 4, grad_table=kept, accumulate=True)
    assert (kept == 1).all()


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_accumulate_adds_and_leaves_absent_rows_alone(name):
    v, d, n, dtype = 200, 24, 3000, DTYPES[name]
    _, grad, ids = make(v, d, n, dtype, 3)
    ids[ids >= 150] = 3
    old = torch.randn(v, d, generator=torch.Generator().manual_seed(9)).to(dtype)
    got = old.cuda()
    cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, 0.5, grad_table=got, accumulate=True)
    want, err = ref.embed_backward(grad, ids, v, 0.5, old)
    within(got, want, finish(want, err, dtype), "sum")
    assert torch.equal(got[150:].cpu(), old[150:])


def test_strides_and_odd_addresses():
    v, d, n = 50, 37, 400
    for dtype in (torch.bfloat16, torch.float32):
        table, grad, ids = make(v, d, n, dtype, 5)
        wide = torch.zeros(v * 41 + 3, dtype=dtype, device="cuda")
        part = wide[3:3 + v * 41].view(v, 41)[:, :d]
        part.copy_(table)
        room = torch.full((n * 40 + 1,), 9.0, dtype=dtype, device="cuda")
        out = room[1:1 + n * 40].view(n, 40)[:, :d]
        cc.cc_embed(part, ids.cuda(), 2.0, out=out)
        want = ref.embed(table, ids, 2.0)
        within(out, want, finish(want, want.abs() * U, dtype), "rows")
        assert (room[1:].view(n, 40)[:, d:] == 9).all() and room[0] == 9
        room[1:].view(n, 40)[:, :d] = grad.cuda()
        into = torch.full((v * 39 + 1,), 5.0, dtype=dtype, device="cuda")
        cc.cc_embed_backward(out, ids.cuda(), v, 2.0, grad_table=into[1:].view(v, 39)[:, :d])
        want, err = ref.embed_backward(grad, ids, v, 2.0)
        within(into[1:].view(v, 39)[:, :d], want, finish(want, err, dtype), "gradient")
        assert (into[1:].view(v, 39)[:, d:] == 5).all() and into[0] == 5


def test_ids_of_any_shape():
    table, grad, ids = make(30, 16, 60, torch.float32)
    out = cc.cc_embed(table.cuda(), ids.view(4, 15).cuda(), 1.0)
    assert out.shape == (4, 15, 16)
    assert torch.equal(out.view(60, 16), cc.cc_embed(table.cuda(), ids.cuda(), 1.0))
    got = cc.cc_embed_backward(grad.view(4, 15, 16).cuda(), ids.view(4, 15).cuda(), 30)
    assert torch.equal(got, cc.cc_embed_backward(grad.cuda(), ids.cuda(), 30))


def test_rows_beyond_32_bits_of_offset():
    v, d = 1 << 20, 2112                                  # 2.2e9 elements
    table = torch.empty(v, d, dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([v - 1, 0, v - 2, v - 1], dtype=torch.int32)
    rows = torch.randn(4, d, generator=torch.Generator().manual_seed(1)).bfloat16()
    for i, k in enumerate(ids.tolist()):
        table[k] = rows[i].cuda()
    say("embed: table of 4.4 GB")
    out = cc.cc_embed(table, ids.cuda())
    assert torch.equal(out.cpu()[1:], rows[1:]) and torch.equal(out.cpu()[0], rows[3])
    cc.cc_embed_backward(rows.cuda(), ids.cuda(), v, 1.0, grad_table=table)
    want = (rows[0].double() + rows[3].double())
    within(table[v - 1], want, finish(want, want.abs() * U, torch.bfloat16), "last row")
    assert torch.equal(table[v - 2].cpu(), rows[2]) and torch.equal(table[0].cpu(), rows[1])
    assert int(torch.count_nonzero(table[1:4096])) == 0 and int(torch.count_nonzero(table[v - 4096:v - 2])) == 0


def test_infinities_stay_in_their_rows():
    table, grad, ids = make(6, 20, 300, torch.float32)
    grad[ids == 2] = float("inf")
    grad[ids == -1] = float("nan")
    got = cc.cc_embed_backward(grad.cuda(), ids.cuda(), 6).cpu()
    want, err = ref.embed_backward(torch.where(torch.isfinite(grad), grad, 0.0), ids, 6, 1.0)
    keep = [0, 1, 3, 4, 5]
    within(got[keep], want[keep], finish(want, err, torch.float32)[keep], "other rows")
    assert torch.isinf(got[2]).all()
