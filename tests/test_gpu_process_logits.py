"""ersd_process_logits against its 64-bit form: types, vocabularies, rows off 16-byte boundaries, trees, masks."""
import math

import pytest
import torch

import operator_reference as ref
from paper_2504_15475_b200 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


def make(B, R, V, dtype, parent=None, history=40, biases=7, seed=0, ld=None):
    gen = torch.Generator().manual_seed(seed)

    def tokens(*shape):  # a few tokens again and again, some outside the vocabulary
        return (torch.rand(*shape, generator=gen).pow(4.0) * (V + 3)).to(torch.int32) - 1

    a = dict(history=tokens(B, history), history_lens=torch.randint(0, history + 1, (B,), generator=gen, dtype=torch.int32),
             prompt_lens=torch.randint(0, history + 1, (B,), generator=gen, dtype=torch.int32),
             draft_tokens=tokens(B, R - 1 if parent is None else R), parent=parent,
             repetition=torch.rand(B, generator=gen) + 0.6, presence=torch.randn(B, generator=gen),
             frequency=torch.randn(B, generator=gen) * 0.3, bias_tokens=tokens(B, biases),
             bias_values=torch.randn(B, biases, generator=gen) * 5)
    a["bias_values"][:, ::5] = -math.inf
    a["mask"] = torch.randint(-2 ** 31, 2 ** 31, (B, R, -(-V // 32)), generator=gen, dtype=torch.int32)
    a["mask"][:, 0] = 0                       # nothing allowed
    if R > 1:
        a["mask"][:, 1] = -1                  # everything
    x = (torch.randn(B, R, ld or V, generator=gen) * 4).to(dtype)
    x[:, :, ::11] = -math.inf
    x[0, 0, : min(V, 3)] = float("nan")       # masked
    return x, a


def check(ersd, x, a, V=None, in_place=False, cut=None):
    dev = {k: t.cuda() if torch.is_tensor(t) else t for k, t in a.items()}
    want, bound = ref.process_logits(x, **a, V=V)
    y = x.cuda() if cut is None else cut(x)
    out = y if in_place else torch.full_like(y, 3.0) if cut is None else cut(torch.full_like(x, 3.0))
    ersd.ersd_process_logits(y, out, **dev, V=V)
    if V is not None and not in_place:
        assert (out[..., V:] == 3.0).all()
        want, bound = want[..., :V], bound[..., :V]
        out = out[..., :V]
    ref.check(out.cpu(), want, bound, ersd.ersd_last_launch())
    return out


DTYPES = [torch.float32, torch.bfloat16]
PARTS = [("history", "history_lens", "prompt_lens"), ("draft_tokens", "parent"), ("repetition",), ("presence",), ("frequency",),
         ("bias_tokens", "bias_values"), ("mask",)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 31, 32, 33, 100, 2047, 2048, 2049, 5000, 8193, 32000, 50257])
@pytest.mark.parametrize("in_place", [False, True])
def test_vocabularies(ersd, dtype, V, in_place):
    x, a = make(2, 4, V, dtype)
    check(ersd, x, a, in_place=in_place)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [3, 100, 4095, 4097, 9000, 9001])
def test_in_place_without_a_mask(ersd, dtype, V):
    """Tokens that nothing changes are neither read nor written: what they hold stays, NaN among it."""
    for parent, history in ((None, 30), ([-1, 0, 0, 2], 9000)):
        x, a = make(3, 4, V, dtype, parent=parent, history=history, seed=11)
        a["mask"] = None
        check(ersd, torch.nan_to_num(x, nan=1.0), a, in_place=True)
        y = x.cuda()
        before = y.clone()
        ersd.ersd_process_logits(y, y)
        assert torch.equal(y.view(torch.int16 if dtype == torch.bfloat16 else torch.int32),
                           before.view(torch.int16 if dtype == torch.bfloat16 else torch.int32))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("left_out", range(len(PARTS)))
def test_parts_can_be_left_out(ersd, dtype, left_out):
    x, a = make(2, 5, 700, dtype, parent=[-1, 0, 0, 1, 1])
    for name in PARTS[left_out]:
        a[name] = None
    if left_out == 0:
        a["history_lens"] = a["prompt_lens"] = None
    check(ersd, x, a)
    alone = {k: (a[k] if k in PARTS[left_out] else None) for k in a}
    x, full = make(2, 5, 700, dtype, parent=[-1, 0, 0, 1, 1])
    check(ersd, x, {k: (full[k] if k in PARTS[left_out] else None) for k in full} if left_out != 1 else alone)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("parent", [None, list(wl.TREE_4x4), list(wl.TREE_SPECINFER), list(wl.star_parent(8)), [-1]])
def test_trees(ersd, dtype, parent):
    R = 9 if parent is None else len(parent)
    x, a = make(3, R, 1000, dtype, parent=parent, seed=3)
    a["draft_tokens"] = a["draft_tokens"] % 6   # the same token again on a path, and on other paths
    check(ersd, x, a)


@pytest.mark.parametrize("dtype", DTYPES)
def test_one_row_and_long_histories(ersd, dtype):
    x, a = make(1, 1, 4000, dtype, history=20000, seed=4)
    a["mask"] = None
    a["history_lens"] = None
    check(ersd, torch.nan_to_num(x, nan=1.0), a)
    x, a = make(5, 2, 300, dtype, history=1, biases=1, seed=5)
    check(ersd, x, a)
    a["history_lens"] = torch.tensor([-1, 9, 0, 1, 1], dtype=torch.int32)       # outside the width: cut
    a["prompt_lens"] = torch.tensor([-5, 0, 3, 9, 0], dtype=torch.int32)
    check(ersd, x, a)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("biases", [1, 500])
def test_the_later_bias_of_a_token_counts(ersd, dtype, biases):
    x, a = make(2, 2, 50, dtype, biases=biases, seed=6)
    a["mask"] = None
    check(ersd, torch.nan_to_num(x, nan=0.5), a)


@pytest.mark.parametrize("dtype", DTYPES)
def test_shared_masks_and_biases(ersd, dtype):
    x, a = make(3, 4, 777, dtype, seed=7)
    x = torch.nan_to_num(x, nan=2.0)
    for b, r in ((3, 1), (1, 4), (1, 1)):
        check(ersd, x, dict(a, mask=a["mask"][:b, -r:].contiguous(), bias_tokens=a["bias_tokens"][:1], bias_values=a["bias_values"][:1]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_padded_rows_and_boundaries(ersd, dtype):
    """Rows longer than the vocabulary, cut out of longer ones at every distance from a 16-byte boundary."""
    x, a = make(2, 3, 500, dtype, ld=512, seed=8)
    check(ersd, x, a, V=500)
    check(ersd, x.clone(), a, V=500, in_place=False)
    x, a = make(2, 3, 500, dtype, seed=9)
    for lead in range(1, 9):
        for out_lead in (lead, 0, 3):
            wide = torch.full((2, 3, 500 + 16 + lead % 2), 3.0, dtype=dtype, device="cuda")
            wide[..., lead:lead + 500] = x.cuda()
            dst = torch.full((2, 3, 500 + 16), 5.0, dtype=dtype, device="cuda")
            dev = {k: t.cuda() if torch.is_tensor(t) else t for k, t in a.items()}
            ersd.ersd_process_logits(wide[..., lead:lead + 500], dst[..., out_lead:out_lead + 500], **dev)
            want, bound = ref.process_logits(x, **a)
            ref.check(dst[..., out_lead:out_lead + 500].cpu(), want, bound, "lead %d to %d" % (lead, out_lead))
            assert (dst[..., :out_lead] == 5.0).all() and (dst[..., out_lead + 500:] == 5.0).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [6000, 6001])
@pytest.mark.parametrize("mask", [False, True])
def test_frequent_tokens(ersd, dtype, V, mask):
    """Long histories whose tokens lie close together, rows that several blocks share."""
    for parent, B, R, history in ((None, 2, 9, 2000), (list(wl.TREE_4x4), 1, len(wl.TREE_4x4), 9000), (None, 3, 1, 700)):
        x, a = make(B, R, V, dtype, parent=parent, history=history, biases=90, seed=12)
        a["history_lens"] = None
        if not mask:
            a["mask"] = None
            x = torch.nan_to_num(x, nan=1.0)
        check(ersd, x, a)
        if mask:
            check(ersd, x, a, in_place=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 41])
def test_many_sequences(ersd, dtype, V):
    """More blocks than the device runs at a time."""
    x, a = make(1300, 5, V, dtype, parent=[-1, 0, 0, 1, 1], history=70, seed=13)
    check(ersd, x, a)
    check(ersd, x, a, in_place=True)
    a["mask"] = None
    x = torch.nan_to_num(x, nan=1.0)
    check(ersd, x, a)
    check(ersd, x, a, in_place=True)


def test_the_same_call_again_and_captured(ersd):
    x, a = make(4, 9, 32000, torch.bfloat16, history=3000, seed=10)
    dev = {k: t.cuda() if torch.is_tensor(t) else t for k, t in a.items()}
    y, out = x.cuda(), torch.empty_like(x, device="cuda")
    ersd.ersd_process_logits(y, out, **dev)
    first = out.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ersd.ersd_process_logits(y, out, **dev)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), first.view(torch.int16))
    dev["history"].copy_(dev["history"].flip(1))
    graph.replay()
    again = out.clone()
    ersd.ersd_process_logits(y, out, **dev)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
