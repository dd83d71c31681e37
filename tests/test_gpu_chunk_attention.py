"""ersd_chunk_attention against its 64-bit form: types, head layouts, lengths, page sizes, trees, windows, strides."""
import pytest
import torch

import operator_reference as ref
from paper_2504_15475_b200 import workloads as wl

pytestmark = pytest.mark.gpu

TREES = {"chain": None, "4x4": list(wl.TREE_4x4), "shared": list(wl.TREE_SPECINFER), "star": list(wl.star_parent(8)),
         "line": list(wl.chain_parent(12))}


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


def make(B, R, Hq, H, D, page, ctx, dtype, seed=0, spare=3, poison=True):
    """A cache whose pages lie in random order; slots behind a sequence's rows hold NaN."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    per = -(-(max(ctx) + R) // page)
    n = B * per + spare
    k = torch.randn(n, page, H, D, generator=gen, device="cuda").to(dtype)
    v = torch.randn(n, page, H, D, generator=gen, device="cuda").to(dtype)
    table = torch.randperm(n, generator=gen, device="cuda")[: B * per].view(B, per).to(torch.int32)
    q = (torch.randn(B, R, Hq, D, generator=gen, device="cuda") * 2).to(dtype)
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    if poison:
        for b in range(B):
            for slot in range(ctx[b] + R, per * page):
                k[table[b, slot // page].item(), slot % page] = float("nan")
                v[table[b, slot // page].item(), slot % page] = float("nan")
    return q, k, v, table, lens


def check(ersd, q, k, v, table, lens, rows=None, **kw):
    out = torch.full_like(q, 7.0)
    opts = {x: kw[x] for x in ("scale", "parent", "window", "sinks") if x in kw}
    ersd.ersd_chunk_attention(q, k, v, table, lens, out, row_counts=rows, **kw)
    launched = ersd.ersd_last_launch()
    want, bound = ref.attention(q, k, v, table, lens, row_counts=rows,
                                weight_bits=2.0 ** -8 if "tensor" in launched else 0.0, **opts)
    behind = torch.isnan(want) & torch.isnan(bound)
    assert (out[behind] == 7.0).all(), "rows that do not count were written"
    want, bound = torch.where(behind, 7.0, want), torch.where(behind, 0.0, bound)
    ref.check(out, want, bound, launched)
    return out


DTYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (128, 8), (64, 20), (80, 16), (128, 256), (256, 16), (33, 7)])
@pytest.mark.parametrize("Hq,H", [(4, 4), (8, 2), (7, 1)])
def test_shapes(ersd, dtype, D, page, Hq, H):
    check(ersd, *make(3, 5, Hq, H, D, page, [0, 131, 300], dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,ctx", [(1, 0), (1, 1), (1, 127), (1, 128), (2, 126), (1, 2000), (16, 63), (17, 64), (33, 500), (64, 0), (130, 70),
                                   (300, 1), (257, 255)])
@pytest.mark.parametrize("split", [0, 1, 3, 8])
def test_lengths(ersd, dtype, R, ctx, split):
    check(ersd, *make(2, R, 8, 2, 64, 16, [ctx, ctx // 2], dtype), split=split)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", sorted(TREES))
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (2, 5), (40, 4), (130, 0), (129, 200), (1000, 3)])
def test_trees_and_windows(ersd, dtype, D, name, window, sinks):
    parent = TREES[name]
    R = 9 if parent is None else len(parent)
    check(ersd, *make(3, R, 8, 2, D, 16, [3, 125, 700], dtype), parent=parent, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_trees(ersd, dtype):
    gen = torch.Generator().manual_seed(5)
    parent = [-1] + [int(torch.randint(max(0, n - 20), n, (1,), generator=gen)) for n in range(1, 256)]
    check(ersd, *make(2, 256, 6, 2, 64, 16, [0, 333], dtype), parent=parent)
    check(ersd, *make(2, 256, 6, 2, 128, 32, [150, 333], dtype), parent=parent, window=8, sinks=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("window", [0, 70])
def test_ragged_rows(ersd, dtype, window):
    """Row counts from none to all, beyond all and below none; lengths below 0 count as 0."""
    q, k, v, table, lens = make(6, 40, 4, 2, 128, 16, [0, 5, 77, 300, 12, 0], dtype)
    lens[5] = -3
    rows = torch.tensor([0, 1, 40, 17, 99, -2], dtype=torch.int32, device="cuda")
    check(ersd, q, k, v, table, lens, rows, window=window, sinks=4)


@pytest.mark.parametrize("dtype", DTYPES)
def test_pages_behind_a_window_are_not_read(ersd, dtype):
    """Pages that no row sees may be given to others: their entries and what they hold do not matter."""
    q, k, v, table, lens = make(2, 3, 8, 2, 64, 16, [1000, 777], dtype)
    for b, ctx in enumerate((1000, 777)):
        table[b, 1:(ctx - 200) // 16] = torch.tensor([-1, 10 ** 6], device="cuda", dtype=torch.int32)[b]
    first_alone = check(ersd, q, k, v, table, lens, window=200, sinks=4)
    # within pages that are read, slots outside the window hold NaN
    for b, ctx in enumerate((1000, 777)):
        for slot in list(range(4, 16)) + list(range((ctx - 200) // 16 * 16, ctx - 199)):
            k[table[b, slot // 16].item(), slot % 16] = float("nan")
            v[table[b, slot // 16].item(), slot % 16] = float("nan")
    again = torch.empty_like(q)
    ersd.ersd_chunk_attention(q, k, v, table, lens, again, window=200, sinks=4)
    assert torch.equal(again, first_alone)


@pytest.mark.parametrize("dtype", DTYPES)
def test_slots_that_do_not_exist(ersd, dtype):
    """Rows behind the last page see what is there, and rows with nothing to see are zeros."""
    q, k, v, table, lens = make(2, 20, 4, 2, 64, 16, [100, 60], dtype, poison=False)
    check(ersd, q, k, v, table[:, :7].contiguous(), lens)                    # 112 slots for 120
    check(ersd, q, k, v, table[:, :7].contiguous(), lens, parent=TREES["4x4"] + [3, 16, 1])
    far = torch.tensor([400, 60], dtype=torch.int32, device="cuda")
    out = check(ersd, q, k, v, table[:, :7].contiguous(), far, window=30)
    assert (out[0] == 0).all()
    for far in (2 ** 31 - 1, 2 ** 30):
        out = torch.full_like(q, 7.0)
        for window, zeros in ((0, False), (5, True)):
            ersd.ersd_chunk_attention(q, k, v, table, torch.full_like(lens, far), out, window=window)
            assert torch.isfinite(out).all() and (out == 0).all() == zeros
    table[0, 2], table[1, 3] = -5, 10 ** 9                                  # pages that do not exist: keys of zeros
    check(ersd, q, k, v, table, lens)


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides(ersd, dtype):
    """Keys and values in one tensor, heads before positions, rows cut out of wider ones, tables of longer rows."""
    D = 64
    q, k, v, table, lens = make(2, 6, 8, 2, D, 16, [90, 33], dtype)
    want = check(ersd, q, k, v, table, lens)
    both = torch.stack([k, v], dim=1)                                       # [pages, 2, page, heads, D]
    heads_first = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v)]
    wide = torch.zeros(2, 6, 8, 3 * D, dtype=dtype, device="cuda")
    wide[..., D:2 * D] = q
    long_table = torch.full((2, table.shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    long_table[:, : table.shape[1]] = table
    for args in ((q, both[:, 0], both[:, 1], table), (q, *heads_first, table), (wide[..., D:2 * D], k, v, table),
                 (q, k, v, long_table[:, : table.shape[1]])):
        assert torch.equal(check(ersd, *args, lens), want)
    # off 16-byte boundaries, and strides that are no multiple of them
    odd = torch.zeros(k.shape[0], 16, 2, D + 1, dtype=dtype, device="cuda")
    odd[..., 1:] = k
    odd_q = torch.zeros(2, 6, 8, D + 3, dtype=dtype, device="cuda")
    odd_q[..., 3:] = q
    check(ersd, odd_q[..., 3:], odd[..., 1:], v, table, lens)
    out = torch.zeros(2, 6, 8, D + 1, dtype=dtype, device="cuda")
    ersd.ersd_chunk_attention(q, k, v, table, lens, out[..., 1:])
    assert torch.equal(out[..., 1:], want) and (out[..., 0] == 0).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_scores(ersd, dtype):
    """Scores of some hundreds, rising and falling along the cache: the maximum moves often; a scale of its own."""
    q, k, v, table, lens = make(2, 4, 4, 2, 128, 16, [900, 400], dtype, poison=False)
    ramp = torch.linspace(-3, 3, k.shape[0], device="cuda")[:, None, None, None]
    check(ersd, q * 8, (k.float() + ramp).to(dtype), v, table, lens)
    check(ersd, q * 8, (k.float() - ramp).to(dtype), v, table, lens, scale=0.5)
    check(ersd, q, k, v, table, lens, scale=-0.1)


@pytest.mark.parametrize("dtype", DTYPES)
def test_far_pages(ersd, dtype):
    """Pages more than 2^31 elements into the cache."""
    D, page, H = 128, 64, 4
    per = page * H * D
    n = (1 << 31) // per + 9
    if torch.cuda.mem_get_info()[0] < 3 * n * per * torch.finfo(dtype).bits // 8:
        pytest.skip("needs the memory of two large caches")
    k = torch.zeros(n, page, H, D, dtype=dtype, device="cuda")
    v = torch.zeros(n, page, H, D, dtype=dtype, device="cuda")
    table = torch.tensor([[n - 1, 3, n - 4, n - 2]], dtype=torch.int32, device="cuda")
    for t in table[0].tolist():
        k[t], v[t] = torch.randn(page, H, D, device="cuda").to(dtype), torch.randn(page, H, D, device="cuda").to(dtype)
    q = torch.randn(1, 5, 8, D, device="cuda").to(dtype)
    check(ersd, q, k, v, table, torch.tensor([240], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_and_on_other_streams(ersd, dtype):
    """Replays follow what the buffers hold at the time; two calls at once do not meet."""
    a = make(2, 5, 8, 2, 128, 16, [500, 300], dtype, seed=1)
    c = make(4, 3, 8, 2, 128, 16, [100, 900, 7, 64], dtype, seed=2)
    outs = [torch.zeros_like(a[0]), torch.zeros_like(c[0])]
    want = [check(ersd, *a), check(ersd, *c)]
    torch.cuda.synchronize()
    st = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        for s, x, o in zip(st, (a, c), outs):
            ersd.ersd_chunk_attention(*x, o, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ersd.ersd_chunk_attention(*a, outs[0])
    outs[0].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0])
    a[4].copy_(torch.tensor([123, 45], dtype=torch.int32))
    a[0].copy_(a[0].flip(1))
    graph.replay()
    torch.cuda.synchronize()
    replayed = outs[0].clone()
    ersd.ersd_chunk_attention(*a, outs[0])
    assert torch.equal(replayed, outs[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R,Hq,parent", [(17, 16, "4x4"), (9, 8, "chain"), (40, 16, "chain")])
def test_full_device(ersd, dtype, R, Hq, parent):
    """As many blocks as fit on the device at once and more, of rows for one to eight warps: warps of a block run
    ahead of one another.  The same call gives the same bits."""
    args = make(37, R, Hq, 4, 128, 64, [(311 * b) % 1500 + 200 for b in range(37)], dtype, poison=False)
    want = check(ersd, *args, parent=TREES[parent])
    out = torch.empty_like(want)
    for _ in range(40):
        ersd.ersd_chunk_attention(*args, out, parent=TREES[parent])
        assert torch.equal(out, want)
