"""The calls around a verification refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest
import torch

from paper_2504_15475_b200 import build as ersd_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EALIGN, EUNSUP = -1, -2, -3
P, ODD = 0x1000, 0x1001       # plausible addresses; never dereferenced
TYPES = {"uint32_t": C.c_uint32, "int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float}


def structure(name):
    """The structure as the header declares it."""
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ersd.h")).read(), flags=re.S)
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, flags=re.S).group(1)
    fields = []
    for d in body.split(";"):
        d = " ".join(d.split()).replace("const ", "")
        if not d:
            continue
        kind, names = d.split(" ", 1)
        for n in names.split(","):
            n = n.strip()
            if kind.endswith("*") or n.startswith("*"):
                fields.append((n.lstrip("* "), C.c_void_p))
            else:
                fields.append((n, TYPES[kind]))
    return type(name, (C.Structure,), {"_fields_": fields})


Cache, ChunkOpts, LogitOpts = structure("ersd_cache"), structure("ersd_chunk_opts"), structure("ersd_logit_opts")


@pytest.fixture(scope="module")
def L():
    ersd_build.build()
    from paper_2504_15475_b200 import binding
    return binding.lib()


def test_layout(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ersd.h"\nint main(void){printf("%zu %zu %zu %zu %zu %zu",'
                   ' sizeof(ersd_cache), offsetof(ersd_cache, v_stride_head), sizeof(ersd_chunk_opts), offsetof(ersd_chunk_opts, b_stride_h),'
                   ' sizeof(ersd_logit_opts), offsetof(ersd_logit_opts, bias_count));return 0;}\n')
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")])
    got = [int(v) for v in subprocess.check_output([str(tmp_path / "t")]).split()]
    assert got == [C.sizeof(Cache), Cache.v_stride_head.offset, C.sizeof(ChunkOpts), ChunkOpts.b_stride_h.offset, C.sizeof(LogitOpts),
                   LogitOpts.bias_count.offset]


def cache(**kw):
    f = dict(struct_size=C.sizeof(Cache), dtype=1, k=P, v=P, num_pages=10, page_size=16, heads=2, head_dim=64, layers=1, max_pages=4,
             block_table=P, table_stride=4, k_stride_page=16 * 128, k_stride_token=128, k_stride_head=64, v_stride_page=16 * 128,
             v_stride_token=128, v_stride_head=64)
    f.update(kw)
    return Cache(**f)


def opts(kind, **kw):
    return kind(struct_size=C.sizeof(kind), **kw)


def ptr(x):
    return C.c_void_p(x) if isinstance(x, int) else x if x is None else C.byref(x)


BAD_CACHES = [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(block_table=None), EINVAL), (dict(dtype=2), EINVAL),
              (dict(num_pages=0), EINVAL), (dict(page_size=0), EINVAL), (dict(heads=0), EINVAL), (dict(head_dim=0), EINVAL),
              (dict(layers=0), EINVAL), (dict(max_pages=0), EINVAL), (dict(k=ODD), EALIGN), (dict(v=ODD), EALIGN),
              (dict(block_table=P + 2), EALIGN), (dict(max_pages=1 << 27), EUNSUP), (dict(heads=65536), EUNSUP)]


def test_attention(L):
    def call(cache_=None, q=P, out=P, lens=P, B=1, R=3, Hq=4, o=None):
        return L.ersd_chunk_attention(ptr(cache_ or cache()), ptr(q), ptr(out), ptr(lens), B, R, Hq, ptr(o), None)

    assert L.ersd_chunk_attention(None, ptr(P), ptr(P), ptr(P), 1, 1, 2, None, None) == EINVAL
    for bad, status in BAD_CACHES:
        if bad.get("heads", 0) > 1:
            assert call(cache(**bad), Hq=65536) == status, bad
        else:
            assert call(cache(**bad)) == status, bad
    for bad, status in [(dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(lens=None), EINVAL), (dict(B=0), EINVAL), (dict(R=0), EINVAL),
                        (dict(Hq=0), EINVAL), (dict(Hq=3), EINVAL), (dict(q=ODD), EALIGN), (dict(out=ODD), EALIGN), (dict(lens=P + 2), EALIGN),
                        (dict(B=65536), EUNSUP), (dict(R=1 << 29), EUNSUP), (dict(cache_=cache(head_dim=257)), EUNSUP)]:
        assert call(**bad) == status, bad
    star = (C.c_int32 * 300)(-1, *([0] * 299))
    keep = [(C.c_int32 * 3)(*p) for p in ((0, 0, 0), (-1, 1, 0), (-1, 0, 5), (-1, -1, 0))]
    for p in keep:
        assert call(o=opts(ChunkOpts, parent=C.cast(p, C.c_void_p))) == EINVAL
    assert call(o=opts(ChunkOpts, parent=C.cast(star, C.c_void_p)), R=300) == EUNSUP
    for bad in (dict(window=-1), dict(sinks=-1), dict(max_context=-1), dict(split=17), dict(split=32), dict(split=-1), dict(kernel_path=3),
                dict(scale=math.nan), dict(scale=math.inf)):
        assert call(o=opts(ChunkOpts, **bad)) == EINVAL, bad
    assert call(o=opts(ChunkOpts, row_counts=P + 2)) == EALIGN


def test_append(L):
    def call(cache_=None, k=P, v=P, lens=P, B=1, R=3, o=None):
        return L.ersd_cache_append(ptr(cache_ or cache()), ptr(k), ptr(v), ptr(lens), B, R, ptr(o), None)

    assert L.ersd_cache_append(None, ptr(P), ptr(P), ptr(P), 1, 1, None, None) == EINVAL
    for bad, status in BAD_CACHES:
        assert call(cache(**bad)) == status, bad
    for bad, status in [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(lens=None), EINVAL), (dict(B=0), EINVAL), (dict(R=0), EINVAL),
                        (dict(k=ODD), EALIGN), (dict(v=ODD), EALIGN), (dict(lens=P + 1), EALIGN), (dict(B=65536), EUNSUP), (dict(R=1 << 30), EUNSUP)]:
        assert call(**bad) == status, bad
    assert call(o=opts(ChunkOpts, row_counts=P + 2)) == EALIGN


def test_commit(L):
    def call(cache_=None, lens=P, path=P, accept=P, B=1, D=3, out=None):
        return L.ersd_cache_commit(ptr(cache_ or cache()), ptr(lens), ptr(path), ptr(accept), B, D, ptr(out), None)

    assert L.ersd_cache_commit(None, ptr(P), ptr(P), ptr(P), 1, 1, None, None) == EINVAL
    for bad, status in BAD_CACHES:
        assert call(cache(**bad)) == status, bad
    for bad, status in [(dict(lens=None), EINVAL), (dict(path=None), EINVAL), (dict(accept=None), EINVAL), (dict(B=0), EINVAL), (dict(D=-1), EINVAL),
                        (dict(out=P), EINVAL), (dict(out=P + 2), EALIGN), (dict(path=P + 2), EALIGN), (dict(accept=P + 2), EALIGN),
                        (dict(lens=P + 2), EALIGN), (dict(B=65536), EUNSUP), (dict(D=256), EUNSUP)]:
        assert call(**bad) == status, bad


def test_logits(L):
    def call(x=P, y=0x2000, dt=1, B=1, R=3, V=64, o=None):
        return L.ersd_process_logits(ptr(x), ptr(y), dt, B, R, V, ptr(o), None)

    for bad, status in [(dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(dt=2), EINVAL), (dict(B=0), EINVAL), (dict(R=0), EINVAL),
                        (dict(V=0), EINVAL), (dict(x=ODD), EALIGN), (dict(y=ODD), EALIGN), (dict(dt=0, x=P + 2), EALIGN), (dict(B=65536), EUNSUP),
                        (dict(V=0x7FFF0001), EUNSUP)]:
        assert call(**bad) == status, bad
    for bad, status in [(dict(ld_in=63), EINVAL), (dict(ld_out=63), EINVAL), (dict(ld_in=-1), EINVAL), (dict(history=P), EINVAL),
                        (dict(history_lens=P), EINVAL), (dict(prompt_lens=P), EINVAL), (dict(history=P, history_width=-1), EINVAL),
                        (dict(bias_tokens=P), EINVAL), (dict(bias_values=P), EINVAL), (dict(bias_count=1, bias_tokens=P), EINVAL),
                        (dict(bias_count=-1), EINVAL), (dict(bias_count=1, bias_tokens=P, bias_values=P, bias_stride=-1), EINVAL),
                        (dict(mask=P, mask_stride_b=-1), EINVAL), (dict(mask=P, mask_stride_r=-1), EINVAL),
                        (dict(history=P + 2, history_width=4), EALIGN), (dict(mask=P + 1), EALIGN), (dict(repetition=P + 2), EALIGN),
                        (dict(bias_count=65536, bias_tokens=P, bias_values=P), EUNSUP)]:
        assert call(o=opts(LogitOpts, **bad)) == status, bad
    assert call(R=257, o=opts(LogitOpts, draft_tokens=P)) == EUNSUP
    assert call(y=P, o=opts(LogitOpts, ld_in=64, ld_out=72)) == EINVAL          # in place with other strides
    for p in ((0, 0, 0), (-1, 2, 0), (-1, 0, -1)):
        keep = (C.c_int32 * 3)(*p)
        assert call(o=opts(LogitOpts, draft_tokens=P, parent=C.cast(keep, C.c_void_p))) == EINVAL


def test_binding_refuses_host_tensors_and_other_objects(L):
    from paper_2504_15475_b200 import binding
    k = torch.zeros(4, 16, 2, 64)
    q, t, n = torch.zeros(1, 2, 4, 64), torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    for call in (lambda x: binding.ersd_chunk_attention(q, x, k, t, n, q), lambda x: binding.ersd_cache_append(q, q, x, k, t, n),
                 lambda x: binding.ersd_cache_commit(x, k, t, n, t, n), lambda x: binding.ersd_process_logits(x, q)):
        with pytest.raises(ValueError, match="must be a CUDA tensor"):
            call(k)
        with pytest.raises(TypeError, match="must be a tensor"):
            call([1, 2])
