"""The embedding's gradient on both sides of the lines that its kernels are chosen by: few tokens are ranked and many sorted,
runs cross two segments or thousands, and the table is cleared as one piece or row by row."""
import pytest
import torch

import order_model_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say
from order_model_reference import DTYPES, finish, within
from test_gpu_embed import make

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


def gradient(v, d, n, name, spread):
    say(f"embed gradient v={v} d={d} n={n} {name} {spread}")
    dtype = DTYPES[name]
    _, grad, ids = make(v, d, n, dtype, seed=n + d, spread=spread)
    want, err = ref.embed_backward(grad, ids, v, 0.75)
    got = cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, 0.75)
    within(got, want, finish(want, err, dtype), "gradient")
    assert torch.equal(got, cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, 0.75))


@pytest.mark.parametrize("n", [15, 16, 17, 1024, 8191, 12287, 12288, 12289])
@pytest.mark.parametrize("v,spread", [(6, "even"), (9000, "steep"), (1 << 22, "even")])
def test_few_tokens_are_ranked_and_many_are_sorted(n, v, spread):
    gradient(v, 3, n, "f32", spread)


@pytest.mark.parametrize("d", [3, 8, 200, 257, 400, 1000, 1100])
def test_runs_over_many_segments(d):
    gradient(5, d, 9000, "bf16", "one")
    gradient(40, d, 9000, "f32", "even")


@pytest.mark.parametrize("n", [65536, 65537])
@pytest.mark.parametrize("v", [700, 70000])
def test_tiles_that_each_workgroup_adds_up_and_more(n, v):
    gradient(v, 2, n, "f32", "steep")


def test_one_run_over_all_segments():
    gradient(3, 2, 140001, "f32", "one")


@pytest.mark.parametrize("name,wide", [("bf16", False), ("f16", True), ("f32", True)])
@pytest.mark.parametrize("v,d,apart,n", [(300, 7, 9, 40), (300, 7, 9, 20000), (50, 1000, 1003, 60), (3, 40001, 40002, 2), (1, 5, 5, 3), (2, 70000, 70000, 0)])
def test_absent_rows_are_cleared_and_nothing_beside_them(v, d, apart, n, name, wide):
    dtype = DTYPES[name]
    _, grad, ids = make(v, d, n, dtype, spread="steep")
    none = torch.zeros(v, d, dtype=torch.float64)
    want, err = ref.embed_backward(grad, ids, v, 2.0) if n else (none, none)
    whole = torch.full((v + 2, apart), 7.0, device="cuda", dtype=torch.float32 if wide else dtype)
    table = whole[1:-1, :d]
    cc.cc_embed_backward(grad.cuda(), ids.cuda(), v, 2.0, grad_table=table)
    within(table, want, finish(want, err, table.dtype), "gradient")
    table.fill_(7.0)
    assert (whole == 7).all()


@pytest.mark.parametrize("v,n", [(100, 65536), (200, 65536), (200, 65537), (300, 32768), (300, 32769), (1000, 16384), (1000, 16385), (1500, 8193),
                                 (50001, 65536), (50001, 65537), (100000, 32768), (100000, 32769), (600000, 16384), (600000, 16385)])
def test_counts_that_each_workgroup_adds_up_and_more(v, n):
    """Both sides of the line in tiles times digits, for 128 to 2048 digits and one or two passes."""
    gradient(v, 2, n, "f32", "steep")
