"""What the calls around a verification leave out and refuse at the ends of their ranges, decided on the host (no GPU
needed: every call here is refused before anything is launched)."""
import ctypes as C

import pytest

from test_operator_refusals import ChunkOpts, EINVAL, EUNSUP, LogitOpts, P, cache, opts, ptr

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


def test_lengths_written_over_what_the_commit_reads(L):
    """Blocks of one sequence read lengths, paths and counts while another writes the new lengths."""
    def commit(out, lens=0x10000, path=0x20000, accept=0x30000, B=4, D=3):
        # (the path's alignment is right, and the cache has a size that is refused last)
        return L.ersd_cache_commit(ptr(cache(layers=(1 << 20) + 1)), ptr(lens), ptr(path), ptr(accept), B, D, ptr(out), None)

    for base, size in ((0x10000, 16), (0x20000, 64), (0x30000, 16)):
        for out in (base, base + 4, base + size - 4, base - 12):
            assert commit(out) == EINVAL, hex(out)
        for out in (base - 16, base + size):
            assert commit(out) == EUNSUP, hex(out)


def test_memory_that_several_rows_would_share(L):
    """Strides of 0 where rows are written: an expanded tensor is no place for outputs or a cache's writes."""
    f32 = dict(dtype=0)
    bad = [dict(k_stride_head=0), dict(v_stride_head=0), dict(k_stride_token=0), dict(v_stride_token=0), dict(k_stride_page=0),
           dict(v_stride_page=0)]
    for kw in bad:
        assert L.ersd_cache_append(ptr(cache(**kw)), ptr(P), ptr(P), ptr(P), 1, 3, None, None) == EINVAL, kw
        assert L.ersd_cache_commit(ptr(cache(**f32, **kw)), ptr(P), ptr(P), ptr(P), 1, 3, None, None) == EINVAL, kw
    assert L.ersd_cache_commit(ptr(cache(layers=2, k_stride_layer=1 << 20)), ptr(P), ptr(P), ptr(P), 1, 3, None, None) == EINVAL
    for b, r, h in ((0, 256, 64), (768, 0, 64), (768, 256, 0)):
        o = opts(ChunkOpts, b_stride_b=b, b_stride_r=r, b_stride_h=h)
        assert L.ersd_chunk_attention(ptr(cache()), ptr(P), ptr(P), ptr(P), 2, 3, 4, ptr(o), None) == EINVAL, (b, r, h)


def test_scales_that_no_power_of_two_can_take(L):
    """The softmax works with scale * log2(e), which has to be a number too."""
    late = dict(parent=C.cast(BAD_TREE, C.c_void_p))  # refused last
    for scale in (2.4e38, -2.4e38, 3e38, 3.4e38):
        assert L.ersd_chunk_attention(ptr(cache()), ptr(P), ptr(P), ptr(P), 1, 300, 4, ptr(opts(ChunkOpts, scale=scale, **late)), None) == EINVAL, scale
    for scale in (2.3e38, -2.3e38, 1e-45, 0.0):
        assert L.ersd_chunk_attention(ptr(cache()), ptr(P), ptr(P), ptr(P), 1, 300, 4, ptr(opts(ChunkOpts, scale=scale, **late)), None) == EUNSUP, scale
