"""The binding refuses tensors that do not go together, and nothing is launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ersd():
    from paper_2504_15475_b200 import binding
    binding.lib()
    return binding


def test_attention_and_cache(ersd):
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    k, v, table, lens = z(4, 16, 2, 64), z(4, 16, 2, 64), z(1, 4, dtype=torch.int32), z(1, dtype=torch.int32)
    q, out = z(1, 3, 4, 64), z(1, 3, 4, 64) + 5
    f = ersd.ersd_chunk_attention
    for args, kw in [((q.float(), k, v, table, lens, out), {}), ((q, k, v.float(), table, lens, out), {}), ((q, k.half(), v.half(), table, lens, out), {}),
                     ((q, k, v[:3], table, lens, out), {}), ((q, k, v, table.long(), lens, out), {}), ((q, k, v, table, lens.long(), out), {}),
                     ((q, k, v, table, lens[:0], out), {}), ((q, k, v, table, lens.cpu(), out), {}), ((q[..., :32], k, v, table, lens, out), {}),
                     ((q, k, v, table, lens, out[:, :2]), {}), ((q[0], k, v, table, lens, out), {}), ((q.transpose(2, 3), k, v, table, lens, out), {}),
                     ((z(2, 3, 4, 64), k, v, table, lens, out), {}), ((q, k[None], v[None], table, lens, out), {}),
                     ((q, k, v, table, lens, out), dict(parent=[-1, 0])), ((q, k, v, table, lens, out), dict(row_counts=lens.float())), ((q, k, v, table, lens, out), dict(scale=0.0)),
                     ((z(64).expand(1, 3, 4, 64), k, v, table, lens, out), {})]:
        with pytest.raises((ValueError, TypeError)):
            f(*args, **kw)
    for kw in (dict(window=-1), dict(parent=[-1, 0, 2]), dict(split=17), dict(kernel_path=7)):
        with pytest.raises(ersd.ErsdError) as e:
            f(q, k, v, table, lens, out, **kw)
        assert e.value.status == -1, kw
    with pytest.raises(ersd.ErsdError):
        f(z(1, 3, 3, 64), k, v, table, lens, z(1, 3, 3, 64))
    new = z(1, 3, 2, 64)
    for args in ((new, new[:, :2], k, v, table, lens), (q, q, k, v, table, lens), (new, new, k, v, table, lens, lens.long()),
                 (new.float(), new.float(), k, v, table, lens)):
        with pytest.raises((ValueError, TypeError)):
            ersd.ersd_cache_append(*args)
    path, acc = z(1, 3, dtype=torch.int32), z(1, dtype=torch.int32)
    for args in ((k, v, table, lens, path[0], acc), (k, v, table, lens, path.long(), acc), (k, v, table, lens, path, path), (k, v[None], table, lens, path, acc)):
        with pytest.raises((ValueError, TypeError)):
            ersd.ersd_cache_commit(*args)
    with pytest.raises(ersd.ErsdError):
        ersd.ersd_cache_commit(k, v, table, lens, path, acc, lens)     # the lengths themselves
    torch.cuda.synchronize()
    assert (out == 5).all() and (k == 0).all() and (lens == 0).all()


def test_logits(ersd):
    x = torch.zeros(2, 3, 100, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(x, 5.0)
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    for kw in (dict(history=i(3, 4)), dict(history=i(2, 4).long()), dict(history=i(2, 4), history_lens=i(3)), dict(draft_tokens=i(2, 3)),
               dict(draft_tokens=i(2, 2), parent=[-1, 0, 0]), dict(repetition=f(3)), dict(presence=f(2).double()),
               dict(bias_tokens=i(2, 4)), dict(bias_tokens=i(2, 4), bias_values=f(2, 5)), dict(bias_tokens=i(3, 4), bias_values=f(3, 4)),
               dict(mask=i(2, 3, 3)), dict(mask=i(2, 2, 4)), dict(mask=i(2, 4)), dict(V=101), dict(V=0), dict(mask=i(2, 3, 8)[..., ::2])):
        with pytest.raises((ValueError, TypeError)):
            ersd.ersd_process_logits(x, out, **kw)
    for y in (out.float(), out[:, :2], out[:1], out.cpu(), out.transpose(0, 1)):
        with pytest.raises((ValueError, TypeError)):
            ersd.ersd_process_logits(x, y)
    with pytest.raises(ValueError):
        ersd.ersd_process_logits(x[:, :2], out[:, :2])                # rows at unequal distances
    for kw in (dict(history_lens=i(2)), dict(draft_tokens=i(2, 3), parent=[-1, 0, 2])):
        with pytest.raises(ersd.ErsdError) as e:
            ersd.ersd_process_logits(x, out, **kw)
        assert e.value.status == -1
    torch.cuda.synchronize()
    assert (out == 5).all()
