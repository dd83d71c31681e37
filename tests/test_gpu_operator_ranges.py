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
