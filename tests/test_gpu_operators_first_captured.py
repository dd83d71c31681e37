"""The very first call of a process may be one that is captured: nothing is prepared by then."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
import torch
from paper_2504_15475_b200 import binding as ersd
kind, dtype = sys.argv[1], getattr(torch, sys.argv[2])
rand = lambda *s: torch.randn(*s, device="cuda").to(dtype)
ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
k, v, new = rand(2, 8, 16, 2, 64), rand(2, 8, 16, 2, 64), rand(2, 3, 2, 64)
table, lens, q = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4), ints(2) + 20, rand(2, 3, 8, 64)
long = rand(2, 40, 8, 64)
path, accept = torch.tensor([[0, 2, -1], [0, 1, 2]], dtype=torch.int32, device="cuda"), ints(2) + 1
logits, history, presence = rand(2, 3, 5000), ints(2, 30) + 7, torch.ones(2, device="cuda")
call, result = dict(
    attention=(lambda o: ersd.ersd_chunk_attention(q, k[0], v[0], table, lens, o), torch.zeros_like(q)),
    long_attention=(lambda o: ersd.ersd_chunk_attention(long, k[0], v[0], table, lens - 20, o), torch.zeros_like(long)),
    append=(lambda o: ersd.ersd_cache_append(new, new, o, v[0], table, lens), k[0].clone()),
    commit=(lambda o: ersd.ersd_cache_commit(o, v, table, lens, path, accept), k.clone()),
    logits=(lambda o: ersd.ersd_process_logits(logits, o, history=history, presence=presence), torch.zeros_like(logits)),
)[kind]
untouched = result.clone()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call(result)
assert torch.equal(result, untouched)
graph.replay()
torch.cuda.synchronize()
want = untouched.clone()
call(want)
torch.cuda.synchronize()
assert torch.equal(result, want) and not torch.equal(result, untouched)
print("as it should be")
"""


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("kind", ["attention", "long_attention", "append", "commit", "logits"])
def test_first_call_captured(kind, dtype):
    r = subprocess.run([sys.executable, "-c", PROGRAM, kind, dtype], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "as it should be" in r.stdout, r.stderr[-2000:]
