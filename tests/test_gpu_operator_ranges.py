"""The calls around a verification at the ends of their ranges."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_largest_vocabulary(ersd, dtype):
    V = 65535 * 4096 - 7
    x = torch.zeros(1, 1, V, dtype=dtype, device="cuda")
    x[..., ::1000] = 2.0
    tokens = torch.tensor([[0, 4095, 4096, V // 2, V - 1, V]], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    ersd.ersd_process_logits(x, out, bias_tokens=tokens, bias_values=torch.full((1, 6), 0.5, device="cuda"))
    at = tokens[0, :5].long()
    x[0, 0, at] += 0.5
    assert torch.equal(out, x)
    history = torch.tensor([[V - 1, V, 1000, V - 1]], dtype=torch.int32, device="cuda")
    ersd.ersd_process_logits(x, x, history=history, frequency=torch.ones(1, device="cuda"))
    out[0, 0, 1000] -= 1.0
    out[0, 0, V - 1] -= 2.0
    assert torch.equal(out, x)
    with pytest.raises(ersd.ErsdError) as e:
        ersd.ersd_process_logits(*[torch.zeros(1, 1, V + 1, dtype=dtype, device="cuda")] * 2)
    assert e.value.status == -3


def test_expanded_tensors_are_read_but_not_written(ersd):
    """Queries of one row, keys of one head: expanded ones are as good as copies.  Outputs and caches that are written: refused."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for dtype in (torch.float32, torch.bfloat16):
        q = torch.randn(2, 1, 4, 64, generator=gen, device="cuda").to(dtype).expand(2, 3, 4, 64)
        k, v = (torch.randn(4, 16, 1, 64, generator=gen, device="cuda").to(dtype).expand(4, 16, 2, 64) for _ in range(2))
        table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
        lens = torch.tensor([20, 7], dtype=torch.int32, device="cuda")
        out, want = torch.empty(2, 2, 3, 4, 64, dtype=dtype, device="cuda")
        ersd.ersd_chunk_attention(q, k, v, table, lens, out, kernel_path=1)
        ersd.ersd_chunk_attention(q.contiguous(), k.contiguous(), v.contiguous(), table, lens, want, kernel_path=1)
        assert torch.equal(out, want)
        ersd.ersd_chunk_attention(q, k, v, table, lens, out)                # (heads in one place: not for tensor cores)
        assert torch.equal(out, want)
        one = torch.zeros(2, 3, 2, 64, dtype=dtype, device="cuda")
        path, accept = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        whole = k.contiguous()
        for call in (lambda: ersd.ersd_chunk_attention(q, k, v, table, lens, out[:, :1].expand(2, 3, 4, 64)),
                     lambda: ersd.ersd_cache_append(one, one, whole, v, table, lens),
                     lambda: ersd.ersd_cache_append(one, one, k, whole, table, lens),
                     lambda: ersd.ersd_cache_commit(whole, v, table, lens, path, accept),
                     lambda: ersd.ersd_cache_commit(whole.expand(3, *whole.shape), whole.expand(3, *whole.shape), table, lens, path, accept)):
            with pytest.raises(ersd.ErsdError) as e:
                call()
            assert e.value.status == -1


def test_parents_beyond_32_bits(ersd):
    """Numbers that 32 bits do not hold are no nodes, whatever their lower bits say."""
    k = torch.zeros(4, 16, 2, 64, device="cuda")
    table, lens = torch.zeros(1, 4, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.ones(1, 3, 4, 64, device="cuda")
    x = torch.zeros(1, 3, 100, device="cuda")
    drafts = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    for parent in ([-1, 2 ** 32, 0], [2 ** 32 - 1, 0, 0], [-1, 0, -2 ** 32], [-1, 0, 2 ** 40 + 1]):
        with pytest.raises(ValueError):
            ersd.ersd_chunk_attention(q, k, k, table, lens, torch.empty_like(q), parent=parent)
        with pytest.raises(ValueError):
            ersd.ersd_process_logits(x, torch.empty_like(x), draft_tokens=drafts, parent=parent)
