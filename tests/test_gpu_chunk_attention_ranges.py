"""ersd_chunk_attention where its kernels have ways of their own: ragged trees, long caches, small pages, gaps, splits,
kernels asked for by name."""
import pytest
import torch

from test_gpu_chunk_attention import DTYPES, TREES, ersd, make, check  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def random_tree(n, seed):
    gen = torch.Generator().manual_seed(seed)
    return [-1] + [int(torch.randint(max(0, i - 20), i, (1,), generator=gen)) for i in range(1, n)]


def poison_behind(k, v, table, lens, rows, R):
    """NaN in every slot behind the counted rows of a sequence."""
    page = k.shape[1]
    for b, (ctx, n) in enumerate(zip(lens.tolist(), rows.tolist())):
        first = max(0, ctx) + max(0, min(n, R))
        slots = torch.arange(first, table.shape[1] * page, device="cuda")
        at = table[b].long()[slots // page]
        k[at, slots % page] = float("nan")
        v[at, slots % page] = float("nan")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", ["4x4", "star", "random"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 5), (90, 4)])
@pytest.mark.parametrize("split", [0, 3])
def test_ragged_trees(ersd, dtype, D, name, window, sinks, split):  # noqa: F811
    """Of a tree's rows the first ones count; what lies behind them is NaN."""
    parent = random_tree(256, 5) if name == "random" else TREES[name]
    R = len(parent)
    q, k, v, table, lens = make(6, R, 6, 2, D, 16, [0, 5, 127, 300, 64, 0], dtype, poison=False)
    lens[5] = -3
    rows = torch.tensor([R, 1, max(1, R // 2), R - 1, 0, R + 9], dtype=torch.int32, device="cuda")
    poison_behind(k, v, table, lens, rows, R)
    check(ersd, q, k, v, table, lens, rows, parent=parent, window=window, sinks=sinks, split=split)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [1, 6, 40, 200])
def test_ragged_chains(ersd, dtype, R):  # noqa: F811
    for D, window in ((64, 0), (128, 7), (128, 0)):
        q, k, v, table, lens = make(5, R, 8, 2, D, 16, [0, 33, 126, 250, 63], dtype, poison=False)
        rows = torch.tensor([R, 1, max(1, R // 3), R - 1, R + 1], dtype=torch.int32, device="cuda")
        poison_behind(k, v, table, lens, rows, R)
        check(ersd, q, k, v, table, lens, rows, window=window, sinks=2)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("R", [1, 5, 17, 100])
def test_32_bit_arithmetic_asked_for(ersd, D, R):  # noqa: F811
    """The way that rounds no weights, in shapes that the tensor cores would take."""
    args = make(2, R, 8, 2, D, 16, [300, 77], torch.bfloat16)
    for kw in (dict(), dict(window=50, sinks=3), dict(split=5)):
        check(ersd, *args, kernel_path=1, **kw)
        assert "tensor" not in ersd.ersd_last_launch()
        check(ersd, *args, kernel_path=2, **kw)
        assert "tensor" in ersd.ersd_last_launch()


def test_tensor_cores_asked_for_where_they_do_not_apply(ersd):  # noqa: F811
    bf = torch.bfloat16
    odd = make(1, 2, 4, 2, 64, 16, [30], bf)
    wide = torch.zeros(*odd[1].shape[:3], 65, dtype=bf, device="cuda")
    for q, k, v, table, lens in (make(1, 2, 4, 2, 64, 16, [30], torch.float32), make(1, 2, 4, 2, 80, 16, [30], bf),
                                 make(1, 2, 4, 2, 256, 16, [30], bf), make(1, 2, 4, 2, 64, 7, [30], bf), make(1, 2, 4, 2, 64, 2, [30], bf),
                                 (odd[0], wide[..., 1:], *odd[2:]), (odd[0], odd[1], wide[..., 1:], *odd[3:])):
        out = torch.full_like(q, 7.0)
        with pytest.raises(ersd.ErsdError) as e:
            ersd.ersd_chunk_attention(q, k, v, table, lens, out, kernel_path=2)
        assert e.value.status == -3
        assert (out == 7).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [1, 17, 130])
def test_bounds_of_the_contexts_change_no_result(ersd, dtype, R):  # noqa: F811
    """A bound, a bound that is too high, and one below the truth."""
    args = make(2, R, 8, 2, 128, 16, [900, 411], dtype)
    for bound in (900, 10 ** 6, 2 ** 31 - 1, 64, 1):
        check(ersd, *args, max_context=bound)
        check(ersd, *args, max_context=bound, window=100, sinks=4)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [4, 12])
@pytest.mark.parametrize("R", [1, 20, 80])
def test_smallest_pages(ersd, D, page, R):  # noqa: F811
    """Pages of four slots, the smallest that tensor cores take: a tile has 32 of them, its copies two boxes to a lane."""
    args = make(2, R, 8, 2, D, page, [1000, 333], torch.bfloat16)
    for kw in (dict(), dict(split=1), dict(window=100, sinks=9), dict(window=3)):
        check(ersd, *args, kernel_path=2, **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("page", [4, 8, 16])
@pytest.mark.parametrize("ctx,window,sinks", [(3000, 300, 4), (3000, 20, 300), (2500, 129, 1100), (1500, 1, 1)])
@pytest.mark.parametrize("split", [0, 1, 2])
def test_gaps_of_many_pages(ersd, dtype, page, ctx, window, sinks, split):  # noqa: F811
    """More pages between first tokens and window than a warp has entries of the block table for, in pages that are not there."""
    q, k, v, table, lens = make(2, 6, 8, 2, 64, page, [ctx, ctx - 77], dtype)
    for b, c in enumerate((ctx, ctx - 77)):
        table[b, -(-sinks // page):(c - window + 1) // page] = (-1, 10 ** 6)[b]
    check(ersd, q, k, v, table, lens, window=window, sinks=sinks, split=split)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("split", range(9, 17))
def test_splits_above_eight(ersd, dtype, split):  # noqa: F811
    for R, ctx in ((1, [5000]), (6, [40]), (40, [2100])):
        check(ersd, *make(1, R, 8, 2, 128, 64, ctx, dtype, seed=split), split=split)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,R,Hq,H,D,page,ctx", [(1, 1, 8, 1, 128, 64, [64000]), (1, 5, 8, 2, 64, 16, [131072]), (2, 17, 8, 2, 128, 16, [40000, 9]),
                                                 (2, 1, 4, 1, 64, 4, [33333, 64001])])
def test_long_caches(ersd, dtype, B, R, Hq, H, D, page, ctx):  # noqa: F811
    args = make(B, R, Hq, H, D, page, ctx, dtype)
    check(ersd, *args)
    check(ersd, *args, split=1, window=30000, sinks=64)
    check(ersd, *args, max_context=100)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [80, 256])
@pytest.mark.parametrize("R,Hq,H", [(9, 8, 2), (37, 2, 2), (12, 8, 2), (7, 7, 1), (16, 8, 2)])
def test_few_and_many_rows_of_other_heads(ersd, dtype, D, R, Hq, H):  # noqa: F811
    """Either side of where the kernels of 32-bit arithmetic change: 48 rows, with bfloat16 36 from 17 heads on."""
    for B in (2, 18):
        check(ersd, *make(B, R, Hq, H, D, 16, [200, 31] * (B // 2), dtype))
        most = 36 if dtype == torch.bfloat16 and B * H > 16 else 48
        assert ("rows_kernel" if R * (Hq // H) <= most else "tile_kernel") in ersd.ersd_last_launch()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("Hq,R", [(71, 1), (71, 5), (300, 1), (300, 9)])
def test_many_heads_share_one(ersd, dtype, Hq, R):  # noqa: F811
    """More query heads to a kv head than a tile has rows."""
    args = make(2, R, Hq, 1, 64, 16, [250, 31], dtype)
    check(ersd, *args)
    if R == 9:
        rows = torch.tensor([4, 9], dtype=torch.int32, device="cuda")
        poison_behind(*args[1:], rows, R)
        check(ersd, *args, rows, parent=TREES["star"], window=20, sinks=1)
