"""What the reader's calls refuse, on the CPU: the C entry points check every
argument that the host can see before they look for a GPU, and the binding
checks shapes and types before it passes a pointer."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2607_16973_amd as tq  # noqa: E402
from paper_2607_16973_amd._lib import KVCacheView, KVRowsView, RowsView, lib  # noqa: E402

OK, EINVAL, EUNSUPPORTED = 0, -1, -4
P = 4096     # an address that is never used: every call below is refused, or has nothing to do


def cache(**over):
    f = dict(k=P, v=P, k_scale=P, v_scale=P, status=None, pages=8, layers=2, kv_heads=2, head_dim=64, type=0)
    f.update(over)
    return ctypes.byref(KVCacheView(**f))


def rows(data=P, token=128, head=64):
    return ctypes.byref(RowsView(data, token, head))


def append(c=None, layer=0, k=None, v=None, dtype=0, n=3, tables=P, width=2, lens=P, starts=None, nrows=3):
    return lib.tq_kv_append(c or cache(), layer, k or rows(), v or rows(), dtype, n, tables, width, lens, starts, nrows, None)


def attend(c=None, layer=0, q=None, dtype=0, n=3, heads=4, tables=P, width=2, lens=P, starts=None, nrows=3,
           longest=0, scale=0.1, out=P, ws=None, ws_bytes=0):
    return lib.tq_kv_attend(c or cache(), layer, q or rows(), dtype, n, heads, tables, width, lens, starts, nrows,
                            longest, scale, out, None, ws, ws_bytes, None)


@pytest.mark.parametrize("over,status", [
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(k_scale=None), EINVAL), (dict(v_scale=None), EINVAL),
    (dict(k=P + 8), EINVAL), (dict(v=P + 1), EINVAL), (dict(pages=0), EINVAL), (dict(pages=1 << 31), EINVAL),
    (dict(layers=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(kv_heads=5000), EUNSUPPORTED),
    (dict(head_dim=96), EUNSUPPORTED), (dict(head_dim=0), EUNSUPPORTED), (dict(type=2), EINVAL)])
def test_caches(over, status):
    assert append(cache(**over)) == status
    assert attend(cache(**over), heads=40000 if over.get("kv_heads") == 5000 else 4) == status
    assert lib.tq_last_error()


@pytest.mark.parametrize("args,status", [
    (dict(layer=-1), EINVAL), (dict(layer=2), EINVAL), (dict(dtype=2), EINVAL), (dict(n=-1), EINVAL),
    (dict(n=1 << 31, starts=P), EINVAL), (dict(nrows=-1), EINVAL), (dict(width=-1), EINVAL),
    (dict(width=1 << 30), EUNSUPPORTED), (dict(width=1 << 26, nrows=1, n=1), EUNSUPPORTED),
    (dict(lens=None), EINVAL), (dict(tables=None), EINVAL), (dict(n=4), EINVAL), (dict(nrows=0, n=3), EINVAL)])
def test_rows_and_tokens(args, status):
    assert append(**args) == status
    assert attend(**args) == status


def test_vectors():
    for bad in (rows(None), rows(P, -1), rows(P, 1, -1), rows(P + 1)):
        assert append(k=bad) == EINVAL and append(v=bad) == EINVAL and attend(q=bad) == EINVAL
    assert lib.tq_kv_append(cache(), 0, None, rows(), 0, 3, P, 2, P, None, 3, None) == EINVAL
    assert lib.tq_kv_append(None, 0, rows(), rows(), 0, 3, P, 2, P, None, 3, None) == EINVAL


def test_attend_only():
    assert attend(heads=3) == EINVAL and attend(heads=0) == EINVAL and attend(heads=1 << 20) == EUNSUPPORTED
    assert attend(out=None) == EINVAL and attend(out=P + 2) == EINVAL
    assert attend(longest=-1) == EINVAL
    assert attend(scale=math.nan) == EINVAL and attend(scale=math.inf) == EINVAL
    # a long row is split and needs room for its parts
    need = ctypes.c_size_t()
    assert lib.tq_kv_attend_workspace(cache(), 1, 4, 1000, 1, 0, ctypes.byref(need)) == OK and need.value > 0
    for ws, n in ((None, need.value), (P, need.value - 1), (P + 4, need.value)):
        assert attend(n=1, nrows=1, width=1000, ws=ws, ws_bytes=n) == EINVAL
    assert lib.tq_kv_attend_workspace(cache(), 1, 4, 1000, 1, 0, None) == EINVAL
    assert lib.tq_kv_attend_workspace(cache(), 1, 3, 1000, 1, 0, ctypes.byref(need)) == EINVAL
    assert lib.tq_kv_attend_workspace(cache(), 0, 4, 1000, 0, 0, ctypes.byref(need)) == OK and need.value == 0


def test_nothing_to_do_needs_no_gpu():
    assert append(n=0, k=rows(None), v=rows(None), starts=P) == OK
    assert attend(n=0, q=rows(None), out=None, starts=P) == OK
    assert lib.tq_attention(rows(None), rows(None), rows(None), 0, 0, 0, 4, 2, 64, None, None, 0, 0, 1, 0.1, None,
                            None, None) == OK


def prompt(q=None, k=None, v=None, dtype=0, n=5, n_keys=5, heads=4, kv_heads=2, d=64, starts=P, key_starts=None,
           nrows=1, longest=0, scale=0.1, out=P):
    return lib.tq_attention(q or rows(), k or rows(), v or rows(), dtype, n, n_keys, heads, kv_heads, d, starts,
                            key_starts, nrows, longest, 1, scale, out, None, None)


@pytest.mark.parametrize("args,status", [
    (dict(d=80), EUNSUPPORTED), (dict(dtype=5), EINVAL), (dict(heads=3), EINVAL), (dict(kv_heads=0), EINVAL),
    (dict(n=-1), EINVAL), (dict(n_keys=-1), EINVAL), (dict(n=1 << 31, n_keys=1 << 31), EINVAL), (dict(nrows=-1), EINVAL),
    (dict(longest=-1), EINVAL), (dict(scale=math.nan), EINVAL), (dict(n_keys=6), EINVAL), (dict(starts=None), EINVAL),
    (dict(nrows=0), EINVAL), (dict(out=None), EINVAL), (dict(out=P + 4), EINVAL),
    (dict(n=(1 << 31) - 1, n_keys=(1 << 31) - 1), EUNSUPPORTED)])
def test_prompts(args, status):
    assert prompt(**args) == status
    for bad in (rows(None), rows(P, -1), rows(P + 1)):
        assert prompt(q=bad) == EINVAL and prompt(k=bad) == EINVAL and prompt(v=bad) == EINVAL


def pool(**over):
    f = dict(tables=P, lens=P, refs=P, pages=8, rows=3, width=4)
    f.update(over)
    return ctypes.byref(KVRowsView(**f))


def test_pages():
    need = ctypes.c_size_t()
    assert lib.tq_kv_rows_workspace(pool(), 5, ctypes.byref(need)) == OK
    n = need.value
    calls = [lambda p, c, ws, b: lib.tq_kv_resize(p, P, c, ws, b, None),
             lambda p, c, ws, b: lib.tq_kv_fork(p, P, P, 5, c, ws, b, None),
             lambda p, c, ws, b: lib.tq_kv_compact(p, c, P, ws, b, None)]
    for call in calls:
        assert call(None, cache(), P, n) == EINVAL and call(pool(), None, P, n) == EINVAL
        assert call(pool(), cache(pages=9), P, n) == EINVAL
        assert call(pool(), cache(head_dim=32), P, n) == EUNSUPPORTED
        assert call(pool(), cache(), None, n) == EINVAL and call(pool(), cache(), P, 16) == EINVAL
        assert call(pool(), cache(), P + 4, n) == EINVAL
        for over in (dict(tables=None), dict(lens=None), dict(refs=None), dict(pages=0), dict(rows=-1), dict(width=-1)):
            assert call(pool(**over), cache(), P, n) == EINVAL
        assert call(pool(width=1 << 30), cache(), P, n) == EUNSUPPORTED
    assert lib.tq_kv_resize(pool(), None, cache(), P, n, None) == EINVAL
    assert lib.tq_kv_fork(pool(), None, P, 5, cache(), P, n, None) == EINVAL
    assert lib.tq_kv_fork(pool(), P, P, -1, cache(), P, n, None) == EINVAL
    assert lib.tq_kv_compact(pool(), cache(), None, P, n, None) == EINVAL
    assert lib.tq_kv_rows_workspace(pool(), -1, ctypes.byref(need)) == EINVAL


def z(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype)


def test_binding_shapes_and_types():
    st = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        tq.attention(z(5, 4), z(5, 2, 64), z(5, 2, 64), st)
    with pytest.raises(ValueError):
        tq.attention(z(5, 4, 64), z(5, 2, 32), z(5, 2, 64), st)
    with pytest.raises(ValueError):
        tq.attention(z(5, 4, 64), z(5, 2, 64), z(4, 2, 64), st)
    with pytest.raises(TypeError):   # CPU tensors
        tq.attention(z(5, 4, 64), z(5, 2, 64), z(5, 2, 64), st)
    with pytest.raises(TypeError):
        tq.attention(None, z(5, 2, 64), z(5, 2, 64), st)
    with pytest.raises(ValueError):
        tq.KVCache(1, 4, 2, 64, "int4")
    c = [z(1, 4, 2, 64, 64, dtype=torch.int8), z(1, 4, 2, 4, 64, 16, dtype=torch.int8), z(1, 4, 2, 4, dtype=torch.float32),
         z(1, 4, 2, 4, dtype=torch.float32)]
    for i in range(4):
        bad = list(c)
        bad[i] = bad[i][:, :3]
        with pytest.raises(ValueError):
            tq.KVCache.over(*bad)
    with pytest.raises(ValueError):
        tq.KVCache.over(*c, status=z(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        tq.KVCache.over(c[0].half(), *c[1:])
    with pytest.raises(TypeError):
        tq.KVCache.over(*c)
    with pytest.raises(ValueError):
        tq.KVPages.over(z(3, 2, dtype=torch.int32), z(4, dtype=torch.int32), z(5, dtype=torch.int32))
    with pytest.raises(TypeError):
        tq.KVPages.over(z(3, 2, dtype=torch.int32), z(3, dtype=torch.int32), z(5, dtype=torch.int32))
