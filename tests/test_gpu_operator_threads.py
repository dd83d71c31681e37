"""The calls around a verification from several host threads at once: they share nothing that a caller would have to order."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


def at_once(calls):
    """Every call again and again in a thread and on a stream of its own; the errors that were raised."""
    errors, start = [], threading.Barrier(len(calls))

    def work(call):
        try:
            stream = torch.cuda.Stream()
            start.wait()
            for _ in range(1500):
                call(stream)
            stream.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return errors


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logits_of_unlike_shared_memory(ersd, dtype):
    """Calls of one build of the kernel that need more and less shared memory: with masks, with biases of long histories."""
    V = 2048
    x = torch.randn(1, 2, V, device="cuda").to(dtype)
    mask = torch.full((1, 1, V // 32), 0x0F0F0F0F, dtype=torch.int32, device="cuda")
    history = torch.zeros(1, 9000, dtype=torch.int32, device="cuda")
    bias = dict(bias_tokens=torch.tensor([[5]], dtype=torch.int32, device="cuda"), bias_values=torch.ones(1, 1, device="cuda"))
    kinds = [dict(), dict(mask=mask), dict(history=history, frequency=torch.zeros(1, device="cuda"), **bias), dict(mask=mask), dict()]
    outs = [torch.empty_like(x) for _ in kinds]
    want = []
    for kw in kinds:
        y = x.clone()
        if "bias_tokens" in kw:
            y[..., 5] += 1
        if "mask" in kw:
            y.masked_fill_((torch.arange(V, device="cuda") & 4) != 0, -torch.inf)
        want.append(y)
    errors = at_once([lambda s, kw=kw, o=o: ersd.ersd_process_logits(x, o, stream=s, **kw) for kw, o in zip(kinds, outs)])
    assert not errors, errors
    for o, w in zip(outs, want):
        assert torch.equal(o, w)
