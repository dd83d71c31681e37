"""What the calls around a verification leave out and refuse at the ends of their ranges, decided on the host (no GPU
needed: every call here is refused before anything is launched)."""
import ctypes as C

import pytest

from test_operator_refusals import EINVAL, EUNSUP, LogitOpts, P, opts, ptr

from paper_2504_15475_b200 import build as ersd_build

BAD_TREE = (C.c_int32 * 3)(0, 0, 0)


@pytest.fixture(scope="module")
def L():
    ersd_build.build()
    from paper_2504_15475_b200 import binding
    return binding.lib()


def logits(L, V=64, **o):
    return L.ersd_process_logits(ptr(P), ptr(0x2000), 1, 1, 3, V, ptr(opts(LogitOpts, **o)), None)


def test_a_width_without_a_history_is_left_out(L):
    """A structure that keeps its width while no history is given: the width plays no part, however large (the last
    check, the tree's, is what refuses the call)."""
    tree = dict(draft_tokens=P, parent=C.cast(BAD_TREE, C.c_void_p))
    for width in (0, 4096, 1 << 30, 0x7FFFFFFF):
        assert logits(L, history_width=width, **tree) == EINVAL, width


def test_histories_beyond_a_count(L):
    """Counts of a token have 29 bits."""
    for width in (1 << 29, (1 << 29) + 1, 1 << 30, 0x7FFFFFFF):
        assert logits(L, history=P, history_width=width, draft_tokens=P, parent=C.cast(BAD_TREE, C.c_void_p)) == EUNSUP, width
    assert logits(L, history=P, history_width=(1 << 29) - 1, draft_tokens=P, parent=C.cast(BAD_TREE, C.c_void_p)) == EINVAL


def test_vocabularies_beyond_the_grid(L):
    """A slice of 4096 tokens to a block, 65535 blocks along the vocabulary."""
    tree = dict(draft_tokens=P, parent=C.cast(BAD_TREE, C.c_void_p))
    most = 65535 * 4096 - 7
    for V in (most + 1, 1 << 28):
        assert logits(L, V=V, **tree) == EUNSUP, V
    assert logits(L, V=most, **tree) == EINVAL
