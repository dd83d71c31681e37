"""ersd_cache_append and ersd_cache_commit: copies, bit for bit, and nothing else touched."""
import pytest
import torch

from paper_2504_15475_b200 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


def caches(layers, n, page, H, D, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(layers, n, page, H, D, generator=gen, device="cuda").to(dtype) for _ in range(2)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,R,H,D,page,ctx", [(1, 1, 1, 64, 16, [0]), (3, 5, 2, 128, 16, [0, 14, 33]), (2, 70, 8, 80, 20, [5, 19]),
                                              (4, 3, 3, 33, 7, [6, 7, 0, 20]), (2, 300, 4, 64, 8, [1, 77])])
@pytest.mark.parametrize("ragged", [False, True])
def test_append(ersd, dtype, B, R, H, D, page, ctx, ragged):
    per = -(-(max(ctx) + R) // page)
    (k, v), table = caches(1, B * per + 2, page, H, D, dtype, 1), torch.randperm(B * per + 2)[: B * per].view(B, per)
    k, v = k[0], v[0]
    table[0, -1] = -1                      # a page that does not exist: its rows are not written
    new = torch.randn(2, B, R, H, D, device="cuda").to(dtype)
    rows = [R] * B
    if ragged:
        rows = [(0, R, R + 5, -1)[b % 4] for b in range(B)]
    lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    want = [k.clone(), v.clone()]
    for b in range(B):
        for r in range(max(0, min(R, rows[b]))):
            p = int(table[b, (ctx[b] + r) // page])
            if p >= 0:
                for s in range(2):
                    want[s][p, (ctx[b] + r) % page] = new[s][b, r]
    ersd.ersd_cache_append(new[0], new[1], k, v, table.int().cuda(), lens,
                           torch.tensor(rows, dtype=torch.int32, device="cuda") if ragged else None)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_append_strides_and_missing_slots(ersd):
    """Rows cut out of one projection's result, keys and values in one tensor, heads before positions, and rows
    behind the last page."""
    B, R, H, D, page = 2, 10, 2, 64, 8
    both = torch.zeros(6, 2, H, page, D, dtype=torch.bfloat16, device="cuda")
    k, v = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    fused = torch.randn(B, R, 3 * H, D, device="cuda").bfloat16()
    table = torch.tensor([[5, 2], [0, 3]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([3, 9], dtype=torch.int32, device="cuda")
    ersd.ersd_cache_append(fused[:, :, H:2 * H], fused[:, :, 2 * H:], k, v, table, lens)
    want = torch.zeros_like(both)
    for b in range(B):
        for r in range(R):
            slot = int(lens[b]) + r
            if slot < 16:
                p = int(table[b, slot // page])
                want[p, 0, :, slot % page], want[p, 1, :, slot % page] = fused[b, r, H:2 * H], fused[b, r, 2 * H:]
    assert torch.equal(both, want)
    odd = torch.zeros(6, page, H, D + 1, dtype=torch.bfloat16, device="cuda")       # off 16-byte boundaries
    ersd.ersd_cache_append(fused[:, :, H:2 * H], fused[:, :, 2 * H:], odd[..., 1:], v, table, lens)
    assert torch.equal(odd[..., 1:], k) and (odd[..., 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layers,H,D,page", [(1, 1, 64, 16), (3, 2, 128, 8), (5, 8, 80, 20), (2, 3, 33, 7)])
def test_commit(ersd, dtype, layers, H, D, page):
    """Every node's path of three trees, one after the other in a batch; the longest path is of 20 moves."""
    long = [-1, 0, 0] + list(range(1, 42))   # two interleaved chains: node n hangs on n - 2
    for parent in (list(wl.TREE_4x4), list(wl.TREE_SPECINFER), long):
        nodes = list(range(len(parent)))
        paths = []
        for n in nodes:
            path = [n]
            while path[0]:
                path.insert(0, parent[path[0]])
            paths.append(path)
        D1 = max(len(p) for p in paths)
        B = len(paths)
        ctx = [(5 * b) % 23 for b in range(B)]
        per = -(-(max(ctx) + len(parent)) // page)
        k, v = caches(layers, B * per, page, H, D, dtype, 2)
        table = torch.randperm(B * per).view(B, per)
        want = [k.clone(), v.clone()]
        for b, path in enumerate(paths):
            for j, n in enumerate(path):
                src, dst = ctx[b] + n, ctx[b] + j
                for s, c in enumerate((k, v)):
                    want[s][:, table[b, dst // page], dst % page] = c[:, table[b, src // page], src % page]
        accept = torch.tensor([len(p) - 1 for p in paths], dtype=torch.int32, device="cuda")
        path = torch.tensor([p + [-1] * (D1 - len(p)) for p in paths], dtype=torch.int32, device="cuda")
        lens = torch.tensor(ctx, dtype=torch.int32, device="cuda")
        new = torch.zeros_like(lens)
        ersd.ersd_cache_commit(k, v, table.int().cuda(), lens, path, accept, new)
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
        assert torch.equal(new, lens + accept + 1)


def test_commit_of_one_layer_and_of_nothing(ersd):
    k, v = [c[0] for c in caches(1, 4, 8, 2, 64, torch.bfloat16, 3)]
    before = k.clone(), v.clone()
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    lens = torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    path = torch.tensor([[0, 3, -1], [0, 1, 2]], dtype=torch.int32, device="cuda")
    ersd.ersd_cache_commit(k, v, table, lens, path, torch.tensor([-1, 2], dtype=torch.int32, device="cuda"))
    assert torch.equal(k, before[0]) and torch.equal(v, before[1])     # nothing accepted; nodes in their places
    ersd.ersd_cache_commit(k, v, table, lens, path, torch.tensor([1, 0], dtype=torch.int32, device="cuda"))
    before[0][0, 3], before[1][0, 3] = before[0][0, 5], before[1][0, 5]
    assert torch.equal(k, before[0]) and torch.equal(v, before[1])
