"""The calls around a verification as a C caller makes them: structures filled in by hand."""
import ctypes as C

import pytest
import torch

import operator_reference as ref
from test_operator_refusals import LogitOpts, opts, ptr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


def process(ersd, x, out, **o):
    """`x` and `out` [B, R, V]; addresses of tensors among the options."""
    o = {k: t.data_ptr() if torch.is_tensor(t) else t for k, t in o.items()}
    status = ersd.lib().ersd_process_logits(ptr(x.data_ptr()), ptr(out.data_ptr()), 0 if x.dtype == torch.float32 else 1,
                                            *x.shape, ptr(opts(LogitOpts, **o)), ptr(torch.cuda.current_stream().cuda_stream))
    assert status == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,R,V", [(1, 1, 5000), (2, 9, 6001), (1, 17, 20000)])
def test_a_width_without_a_history(ersd, dtype, B, R, V):
    """A mask alone, and nothing at all, from a structure that keeps its history's width; calls with lists of many
    tokens before each, whose lists are still in shared memory."""
    gen = torch.Generator().manual_seed(B * 100 + R)
    x = (torch.randn(B, R, V, generator=gen) * 4).to(dtype)
    mask = torch.randint(-2 ** 31, 2 ** 31, (B, R, -(-V // 32)), generator=gen, dtype=torch.int32)
    history = torch.randint(0, 4096, (B, 3000), generator=gen, dtype=torch.int32).cuda()
    y, m = x.cuda(), mask.cuda()
    out = torch.empty_like(y)
    for width in (300, 8191, 9000, 2 ** 31 - 1):
        for masked in (True, False):
            ersd.ersd_process_logits(y, out, history=history, presence=torch.ones(B, device="cuda"))
            out.fill_(3.0)
            given = dict(mask=m, mask_stride_b=m.stride(0), mask_stride_r=m.stride(1)) if masked else {}
            process(ersd, y, out, history_width=width, **given)
            want, bound = ref.process_logits(x, mask=mask if masked else None)
            ref.check(out.cpu(), want, bound, "width %d" % width)
