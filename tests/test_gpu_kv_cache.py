"""The 8-bit cache: appended codes bit for bit against the definition in
float32, attention over it against the float64 form of the stored values.

Tolerance of the attention: weights in float16 (relative 2^-11), the result
rounded once (half a unit e of its type), scores as in the prompt's tests:
|err| <= (2^-11 + 2^-12) sum_j p_j |v_j| + e |out|."""
import math

import numpy as np
import pytest
import torch

import paper_2607_16973_amd as tq
from tests.reader import HostCache, attention64, starts_of

pytestmark = pytest.mark.gpu
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
KINDS = ["int8", "fp8"]


def table_of(lens, width, pages, seed):
    r = np.random.RandomState(seed)
    order = list(r.permutation(pages))
    rows = [[int(order.pop()) for _ in range(-(-n // 64))] for n in lens]
    full = [t + [-1] * (width - len(t)) for t in rows]
    return rows, torch.tensor(full, dtype=torch.int32, device="cuda").reshape(len(lens), width)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def new_values(counts, heads, d, dtype, seed, size=1.0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(2, sum(counts), heads * d + pad, generator=g, device="cuda") * size
    return [t.to(dtype)[:, pad:].unflatten(1, (heads, d)) for t in x]


def same(cache, host, layer, tables, lens):
    """Codes and scales of every block that holds a token."""
    now = HostCache(cache, layer)
    for table, n in zip(tables, lens):
        for b in range(-(-n // 16)):
            p, sub = table[b // 4], b % 4
            for which in range(2):
                assert np.array_equal(now.codes[which][p, :, sub], host.codes[which][p, :, sub]), (p, sub, which)
                assert np.array_equal(now.scales[which][p, :, sub], host.scales[which][p, :, sub]), (p, sub, which)


def dirty(cache):
    """Storage as it may be found: every byte pattern, NaN scales."""
    for t in (cache.k, cache.v):
        t.view(torch.int8).random_(-128, 128)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(math.nan)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,heads", [(64, 1), (128, 3), (256, 2)])
@pytest.mark.parametrize("dtype,pad", [(torch.bfloat16, 0), (torch.float16, 0), (torch.float16, 3)])
def test_append(d, heads, kind, dtype, pad):
    cache = tq.KVCache(2, 40, heads, d, kind)
    dirty(cache)
    host = HostCache(cache, 1)
    before = cache.k[0].view(torch.int8).clone()
    width = 5
    lens = [0] * 6
    rows, tables = table_of([300] * 6, width, 40, 1)
    # whole prompts, single tokens, runs that end inside blocks and pages, a growing scale, an idle row
    for step, counts in enumerate([[1, 16, 17, 130, 64, 0], [1, 1, 1, 1, 1, 0], [15, 30, 2, 5, 64, 1], [3, 0, 47, 1, 100, 33]]):
        new = new_values(counts, heads, d, dtype, 10 + step, 1.0 + step, pad)
        lens = [n + c for n, c in zip(lens, counts)]
        cache.append(1, new[0], new[1], tables, ints(lens), starts_of(counts))
        at = 0
        for r, c in enumerate(counts):
            host.append([t[at:at + c].float().cpu().numpy() for t in new], rows[r], lens[r])
            at += c
        same(cache, host, 1, rows, lens)
    assert torch.equal(cache.k[0].view(torch.int8), before)
    cache.check()


@pytest.mark.parametrize("kind", KINDS)
def test_append_one_token_each_and_values_at_the_edges(kind):
    cache = tq.KVCache(1, 8, 2, 64, kind)
    dirty(cache)
    host = HostCache(cache, 0)
    rows, tables = table_of([64] * 4, 1, 8, 3)
    vals = [0.0, 2.0 ** -120, 1e-30, 1.0, 3.0e38, -0.0, 65504.0, 2.0 ** -100]
    lens = [0] * 4
    for step, x in enumerate(vals):
        new = [torch.full((4, 2, 64), x, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        new[0][:, :, ::3] *= -0.5
        lens = [n + 1 for n in lens]
        cache.append(0, new[0], new[1], tables, ints(lens))
        for r in range(4):
            host.append([t[r:r + 1].float().cpu().numpy() for t in new], rows[r], lens[r])
        same(cache, host, 0, rows, lens)
    cache.check()
    for x in (math.inf, -math.inf, math.nan):
        new = [torch.randn(4, 2, 64, device="cuda").to(torch.bfloat16) for _ in range(2)]
        new[1][2, 1, 7] = x
        lens = [n + 1 for n in lens]
        cache.append(0, new[0], new[1], tables, ints(lens))
        for r in range(4):
            host.append([t[r:r + 1].float().cpu().numpy() for t in new], rows[r], lens[r])
        same(cache, host, 0, rows, lens)
        with pytest.raises(RuntimeError, match="infinite or NaN"):
            cache.check()
        cache.check()


@pytest.mark.parametrize("kind", KINDS)
def test_append_after_a_retreat(kind):
    # drafted tokens are dropped and their places written again
    cache = tq.KVCache(1, 4, 1, 128, kind)
    dirty(cache)
    host = HostCache(cache, 0)
    rows, tables = table_of([128], 2, 4, 5)
    for step, (length, n, size) in enumerate([(40, 40, 1.0), (46, 6, 1.0), (43, 2, 9.0), (45, 1, 0.1), (33, 1, 1.0)]):
        new = new_values([n], 1, 128, torch.float16, 20 + step, size)
        cache.append(0, new[0], new[1], tables, ints([length]), starts_of([n]))
        host.append([t.float().cpu().numpy() for t in new], rows[0], length)
        same(cache, host, 0, rows, [45 if step > 2 else length])


def test_quantisation_error():
    # half a step of the block's scale, e4m3: half a unit of 2^-3 relative
    for kind, step in (("int8", 0.5), ("fp8", 16.0)):
        cache = tq.KVCache(1, 4, 2, 64, kind)
        new = new_values([200], 2, 64, torch.bfloat16, 1, 3.0)
        rows, tables = table_of([200], 4, 4, 0)
        cache.append(0, new[0], new[1], tables, ints([200]), starts_of([200]))
        host = HostCache(cache, 0)
        for got, x, s in zip(host.row(rows[0], 200), new, host.scales):
            scale = np.concatenate([s[p].transpose(1, 0).repeat(16, 0) for p in rows[0]])[:200]
            assert np.all(np.abs(got.numpy() - x.double().cpu().numpy()) <= step * 1.0001 * scale[..., None])


def filled(lens, width, pages, heads, d, kind, seed=0, layers=1):
    """A cache with random content of the rows and dirt everywhere else."""
    cache = tq.KVCache(layers, pages, heads, d, kind)
    dirty(cache)
    rows, tables = table_of(lens, width, pages, seed)
    for layer in range(layers):
        new = new_values(lens, heads, d, torch.float16, 100 + seed + layer)
        cache.append(layer, new[0], new[1], tables, ints(lens), starts_of(lens))
    return cache, rows, tables


def check_attend(cache, host, rows, lens, q, counts, out, lse, scale=None):
    d = q.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    e = HALF[q.dtype]
    t = 0
    for r, (n, c) in enumerate(zip(lens, counts)):
        k, v = host.row(rows[r], n)
        ref, rl, size = attention64(q[t:t + c], k, v, [n - c + i for i in range(c)], scale)
        got, gl = out[t:t + c].double().cpu(), lse[t:t + c].double().cpu()
        assert torch.all((got - ref).abs() <= (2.0 ** -11 + 2.0 ** -12) * size + e * ref.abs() + 2.0 ** -24), (r, n, c)
        assert torch.equal(torch.isinf(gl), torch.isinf(rl))
        fin = ~torch.isinf(rl)
        assert torch.all((gl - rl)[fin].abs() <= 2.0 ** -12 + 2.0 ** -20 * rl[fin].abs())
        t += c


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(3, 3), (8, 2), (20, 1), (40, 1)])
def test_attend_single_tokens(heads, kv_heads, d, kind):
    lens = [1, 0, 15, 16, 17, 63, 64, 65, 300, 129, 777]
    cache, rows, tables = filled(lens, 13, 40, kv_heads, d, kind, layers=2)
    host = HostCache(cache, 1)
    for dtype in (torch.float16, torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(5)
        q = torch.randn(len(lens), heads, d, generator=g, device="cuda").to(dtype)
        out, lse = cache.attend(1, q, tables, ints(lens), return_lse=True)
        check_attend(cache, host, rows, lens, q, [1] * len(lens), out, lse)
        again = cache.attend(1, q, tables, ints(lens), longest=777)
        check_attend(cache, host, rows, lens, q, [1] * len(lens), again, lse)
    cache.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("d,counts", [(64, [4, 1, 0, 9, 2]), (128, [4, 1, 0, 9, 2]), (256, [3, 1, 1, 2, 2]),
                                      (64, [100, 64, 0, 33, 17]), (128, [40, 150, 1, 90, 64]), (256, [30, 64, 0, 33, 90])])
def test_attend_several_tokens(d, counts, kind):
    heads, kv_heads = 6, 2
    lens = [200, 150, 0 if counts[2] == 0 else 5, 90, 64]
    cache, rows, tables = filled(lens, 4, 20, kv_heads, d, kind)
    counts = [min(c, n) for c, n in zip(counts, lens)]
    host = HostCache(cache, 0)
    g = torch.Generator(device="cuda").manual_seed(6)
    wide = torch.randn(sum(counts), heads * d + 5, generator=g, device="cuda").to(torch.bfloat16)
    for q in (wide[:, 5:].unflatten(1, (heads, d)), wide[:, :heads * d].contiguous().view(-1, heads, d).half()):
        out, lse = cache.attend(0, q, tables, ints(lens), starts_of(counts), scale=0.11, return_lse=True)
        check_attend(cache, host, rows, lens, q, counts, out, lse, 0.11)


def test_attend_more_queries_than_tokens():
    # a length shorter than the row's queries: the first of them see nothing
    cache, rows, tables = filled([3, 70], 2, 5, 1, 64, "int8")
    q = torch.randn(8, 2, 64, device="cuda").to(torch.float16)
    out, lse = cache.attend(0, q, tables, ints([3, 70]), starts_of([5, 3]), return_lse=True)
    assert torch.all(out[:2] == 0) and torch.all(lse[:2] == -math.inf)
    check_attend(cache, HostCache(cache, 0), rows, [3, 70], q, [5, 3], out, lse)


@pytest.mark.parametrize("kind", KINDS)
def test_attend_long_row(kind):
    lens = [20011, 3, 9000]
    cache, rows, tables = filled(lens, 313, 460, 1, 64, kind)
    q = torch.randn(3, 4, 64, device="cuda").to(torch.float16)
    out, lse = cache.attend(0, q, tables, ints(lens), return_lse=True)
    check_attend(cache, HostCache(cache, 0), rows, lens, q, [1] * 3, out, lse)
    # the same with a few queries, and cut at `longest`
    q = torch.randn(9, 4, 64, device="cuda").to(torch.bfloat16)
    out, lse = cache.attend(0, q, tables, ints(lens), starts_of([4, 1, 4]), return_lse=True)
    check_attend(cache, HostCache(cache, 0), rows, lens, q, [4, 1, 4], out, lse)
    out = cache.attend(0, q[:3], tables, ints(lens), longest=5000)
    cut = cache.attend(0, q[:3], tables, ints([5000, 3, 5000]), longest=5000)
    assert torch.equal(out, cut)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_attend_chunks_of_long_rows(kind, dtype):
    # many queries per row, each row's pages shared by many workgroups
    lens, counts = [15011, 3, 4000], [70, 2, 33]
    cache, rows, tables = filled(lens, 236, 310, 1, 64, kind)
    q = torch.randn(105, 4, 64, device="cuda").to(dtype)
    out, lse = cache.attend(0, q, tables, ints(lens), starts_of(counts), return_lse=True)
    check_attend(cache, HostCache(cache, 0), rows, lens, q, counts, out, lse)


@pytest.mark.parametrize("counts", [[1, 1], [6, 9], [100, 200]])
def test_attend_rows_do_not_depend_on_each_other(counts):
    lens = [1900, 300]
    cache, rows, tables = filled(lens, 30, 40, 1, 64, "int8")
    g = torch.Generator(device="cuda").manual_seed(11)
    q = torch.randn(sum(counts), 4, 64, generator=g, device="cuda").to(torch.float16)
    want = cache.attend(0, q, tables, ints(lens), starts_of(counts))
    for _ in range(2):
        q[:, 2] *= 100
        out = cache.attend(0, q, tables, ints(lens), starts_of(counts))
        assert torch.equal(out[:, [0, 1, 3]], want[:, [0, 1, 3]])


def test_attend_many_rows():
    # more rows than a wave has lanes, some of them empty, in every path
    r = np.random.RandomState(1)
    lens = [int(n) for n in r.randint(0, 300, 150)]
    lens[7] = lens[149] = 0
    lens[80] = 2000
    cache, rows, tables = filled(lens, 32, 520, 1, 64, "int8")
    host = HostCache(cache, 0)
    q = torch.randn(150, 2, 64, device="cuda").to(torch.bfloat16)
    out, lse = cache.attend(0, q, tables, ints(lens), return_lse=True)
    check_attend(cache, host, rows, lens, q, [1] * 150, out, lse)
    for most in (3, 60):
        counts = [min(n, int(c)) for n, c in zip(lens, r.randint(0, most, 150))]
        counts[3] = min(lens[3], most)
        q = torch.randn(sum(counts), 2, 64, device="cuda").to(torch.float16)
        out, lse = cache.attend(0, q, tables, ints(lens), starts_of(counts), return_lse=True)
        check_attend(cache, host, rows, lens, q, counts, out, lse)


def test_attend_queries_of_any_size():
    # float16 with one power of two per row: tiny, huge and mixed queries
    cache, rows, tables = filled([100] * 5, 2, 12, 1, 64, "int8")
    host = HostCache(cache, 0)
    g = torch.Generator(device="cuda").manual_seed(8)
    q = torch.randn(5, 2, 64, generator=g, device="cuda")
    q[1] *= 1e-20
    q[2] *= 1e-36
    q[3] *= 1e18
    q[4, :, ::2] *= 1e-6
    q = q.to(torch.bfloat16)
    out, lse = cache.attend(0, q, tables, ints([100] * 5), return_lse=True)
    for r in (0, 1, 2, 4):
        check_attend(cache, host, [rows[r]], [100], q[r:r + 1], [1], out[r:r + 1], lse[r:r + 1])
    assert torch.isfinite(out[3]).all()    # one key takes all
    q[0, 0, 3] = math.nan
    q[4, 1, 3] = math.inf
    bad = cache.attend(0, q, tables, ints([100] * 5))
    assert torch.isnan(bad[0, 0]).all() and torch.isnan(bad[4, 1]).all()
    assert torch.equal(bad[1:4], out[1:4]) and torch.equal(bad[0, 1], out[0, 1]) and torch.equal(bad[4, 0], out[4, 0])


def test_scores_past_float32s_fractions():
    # queries so large that one key takes all: several queries of a row, in both tilings
    cache, rows, tables = filled([90, 200], 4, 8, 1, 64, "int8")
    host = HostCache(cache, 0)
    for counts in ([2, 3], [60, 100]):
        q = (torch.randn(sum(counts), 2, 64, device="cuda") * 1e18).to(torch.bfloat16)
        out, lse = cache.attend(0, q, tables, ints([90, 200]), starts_of(counts), return_lse=True)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        t = 0
        for r, (n, c) in enumerate(zip([90, 200], counts)):
            k, v = host.row(rows[r], n)
            for i in range(c):
                x = q[t + i].double().cpu() @ k[:n - c + i + 1, 0].T          # [heads, keys]
                best = x.topk(2).values
                sure = best[:, 0] - best[:, 1] > 1e-5 * best[:, 0].abs()
                want = v[x.argmax(1), 0][sure]
                got = out[t + i].double().cpu()[sure]
                assert torch.all((got - want).abs() <= 2.0 ** -8 * want.abs())
            t += c


@pytest.mark.parametrize("kind", KINDS)
def test_scales_of_very_different_size(kind):
    # values of one block 1e6 times those of another: each block has its own scale
    cache = tq.KVCache(1, 6, 1, 64, kind)
    dirty(cache)
    rows, tables = table_of([200], 4, 6, 2)
    new = new_values([200], 1, 64, torch.float16, 3)
    size = torch.tensor([1.0, 1e-4, 100.0, 1e-2] * 4, device="cuda").repeat_interleave(16)[:200, None, None]
    v = (new[1].float() * size).to(torch.float16)
    cache.append(0, new[0], v, tables, ints([200]), starts_of([200]))
    q = torch.randn(1, 3, 64, device="cuda").to(torch.float16)
    out, lse = cache.attend(0, q, tables, ints([200]), return_lse=True)
    check_attend(cache, HostCache(cache, 0), rows, [200], q, [1], out, lse)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("length,count", [(200, 1), (200, 9), (200, 60), (2500, 1), (1100, 20)])
def test_scales_of_very_different_size_in_every_path(length, count, kind):
    # also blocks of zeros, and a first block far above or below the rest
    cache = tq.KVCache(1, 45, 1, 64, kind)
    dirty(cache)
    rows, tables = table_of([length], 40, 45, 2)
    new = new_values([length], 1, 64, torch.bfloat16, 3)
    r = np.random.RandomState(length)
    size = 10.0 ** r.uniform(-9, 3, length // 16 + 1)
    size[::5] = 0
    size[0] = 1e-12 if count % 2 else 1e6
    v = (new[1].float() * torch.tensor(size, device="cuda", dtype=torch.float32).repeat_interleave(16)[:length, None, None]).to(torch.bfloat16)
    cache.append(0, new[0], v, tables, ints([length]), starts_of([length]))
    q = torch.randn(count, 8, 64, device="cuda").to(torch.float16).to(torch.bfloat16)
    out, lse = cache.attend(0, q, tables, ints([length]), starts_of([count]), return_lse=True)
    check_attend(cache, HostCache(cache, 0), rows, [length], q, [count], out, lse)


def test_bad_page_ids_are_left_out():
    cache, rows, tables = filled([200], 4, 6, 1, 64, "int8")
    q = torch.randn(1, 2, 64, device="cuda").to(torch.float16)
    broken = tables.clone()
    broken[0, 1] = 6
    broken[0, 2] = -1
    out, lse = cache.attend(0, q, broken, ints([200]), return_lse=True)
    k, v = HostCache(cache, 0).row(rows[0], 200)
    keep = [i for i in range(200) if i // 64 in (0, 3)]
    ref, rl, size = attention64(q, k[keep], v[keep], [len(keep)], 1 / 8)
    assert torch.all((out.double().cpu() - ref).abs() <= 2.0 ** -10 * size + 2.0 ** -11 * ref.abs())
    with pytest.raises(RuntimeError, match="outside the pool"):
        cache.check()
    new = new_values([1], 1, 64, torch.float16, 9)
    before = cache.k.view(torch.int8).clone()
    cache.append(0, new[0], new[1], broken, ints([100]))
    assert torch.equal(cache.k.view(torch.int8), before)
    with pytest.raises(RuntimeError, match="outside the pool"):
        cache.check()


@pytest.mark.parametrize("counts", [[1, 1], [3, 50]])
def test_offsets_past_32_bits(counts):
    # pages at the far end of a 9 GB cache: the same results as in a small one
    lens, heads, d = [200, 130], 8, 128
    small, rows, tables = filled(lens, 4, 8, heads, d, "int8")
    far = 70000
    big = tq.KVCache(1, far, heads, d, "int8")
    assert far * heads * 64 * d > 2 ** 32
    moved = torch.where(tables >= 0, far - 8 + tables, tables)
    new = new_values(lens, heads, d, torch.float16, 100)
    big.append(0, new[0], new[1], moved, ints(lens), starts_of(lens))
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(sum(counts), 16, d, generator=g, device="cuda").to(torch.bfloat16)
    args = (ints(lens), None if counts == [1, 1] else starts_of(counts))
    assert torch.equal(big.attend(0, q, moved, *args), small.attend(0, q, tables, *args))
    # and a page copied from one end to the other
    state = tq.KVPages(2, 4, far)
    state.tables[0] = moved[0]
    state.lens[0] = 200
    state.refs[moved[0].long()] = 1
    state.fork(ints([0]), ints([1]), big)
    assert state.tables[1].tolist() == moved[0, :3].tolist() + [0]
    assert torch.equal(big.k[0, 0], big.k[0, moved[0, 3]]) and torch.equal(big.v_scale[0, 0, :, 0], big.v_scale[0, moved[0, 3], :, 0])


def test_calls_on_another_stream():
    cache, rows, tables = filled([300, 40], 5, 12, 2, 64, "fp8")
    lens = ints([301, 41])
    new = new_values([1, 1], 2, 64, torch.float16, 14)
    q = torch.randn(2, 4, 64, device="cuda").to(torch.float16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        cache.append(0, new[0], new[1], tables, lens)
        out, lse = cache.attend(0, q, tables, lens, return_lse=True)
    torch.cuda.current_stream().wait_stream(side)
    check_attend(cache, HostCache(cache, 0), rows, [301, 41], q, [1, 1], out, lse)


def test_refusals_of_the_binding():
    cache, rows, tables = filled([30], 2, 3, 2, 64, "int8")
    q = torch.randn(1, 4, 64, device="cuda").to(torch.float16)
    lens = ints([30])
    with pytest.raises(ValueError):
        cache.attend(0, q[:, :, :32], tables, lens)
    with pytest.raises(TypeError):
        cache.attend(0, q.float(), tables, lens)
    with pytest.raises(TypeError):
        cache.attend(0, q, tables.long(), lens)
    with pytest.raises(ValueError):
        cache.attend(0, q, tables, ints([30, 1]))
    with pytest.raises(ValueError):
        cache.attend(0, q, tables.expand(2, 2).t()[:1], lens)
    with pytest.raises(ValueError):
        cache.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2), tables, lens)
    with pytest.raises(ValueError):
        cache.attend(0, q, tables, lens, out=torch.empty(1, 4, 64, device="cuda", dtype=torch.float16)[:, :2])
    with pytest.raises(TypeError):
        cache.attend(0, q, tables.cpu(), lens)
    with pytest.raises(tq.TQError):
        cache.attend(1, q, tables, lens)
    with pytest.raises(tq.TQError):
        cache.attend(0, q[:, :3], tables, lens)
    with pytest.raises(tq.TQError):
        cache.attend(0, q, torch.zeros(1, 2000, dtype=torch.int32, device="cuda"), lens, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        cache.append(0, q, q, tables, lens)
    with pytest.raises(ValueError):
        tq.KVPages(1, 2, 3).fork(ints([0]), ints([0, 0]), cache)
    with pytest.raises(tq.TQError):
        tq.KVPages(1, 2, 4).compact(cache)


def test_graph_of_a_step():
    cache, rows, tables = filled([100, 40], 3, 8, 2, 64, "int8")
    lens = ints([101, 41])
    new = new_values([1, 1], 2, 64, torch.bfloat16, 12)
    q = torch.randn(2, 4, 64, device="cuda").to(torch.bfloat16)
    cache.append(0, new[0], new[1], tables, lens)
    eager = cache.attend(0, q, tables, lens)
    out = torch.empty_like(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append(0, new[0], new[1], tables, lens)
        cache.attend(0, q, tables, lens, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        cache.attend(0, q, tables, lens)


@pytest.mark.parametrize("counts", [None, [2, 1], [40, 90]])
@pytest.mark.parametrize("length", [-1, -70, -2 ** 31])
def test_negative_lengths_are_empty_rows(length, counts):
    cache, rows, tables = filled([30, 100], 30, 40, 2, 64, "int8")
    lens = ints([length, 100])
    starts = None if counts is None else starts_of(counts)
    counts = counts or [1, 1]
    before = HostCache(cache, 0)
    new = new_values(counts, 2, 64, torch.float16, 31)
    q = torch.randn(sum(counts), 4, 64, device="cuda").to(torch.float16)
    for longest in (0, 128):                     # long rows' path and that of short ones
        out, lse = cache.attend(0, q, tables, lens, starts, longest=longest, return_lse=True)
        check_attend(cache, before, rows, [0, 100], q, counts, out, lse)
    cache.append(0, new[0], new[1], tables, lens, starts)
    after = HostCache(cache, 0)
    for was, now in zip(before.codes + before.scales, after.codes + after.scales):
        assert np.array_equal(was[rows[0]], now[rows[0]], equal_nan=True)
    cache.check()


def test_queries_that_want_gradients_are_refused():
    cache, rows, tables = filled([30], 2, 3, 2, 64, "int8")
    q, lens = torch.randn(1, 4, 64, device="cuda").to(torch.float16).requires_grad_(), ints([30])
    new = new_values([1], 2, 64, torch.float16, 3)
    with pytest.raises(ValueError, match="requires a gradient"):
        cache.attend(0, q, tables, lens)
    with pytest.raises(ValueError, match="requires a gradient"):
        cache.append(0, new[0], new[1].requires_grad_(), tables, lens)
    with pytest.raises(ValueError, match="requires a gradient"):
        tq.attention(q, q.detach(), q.detach(), ints([0, 1]))
    with torch.no_grad():
        assert torch.equal(cache.attend(0, q, tables, lens), cache.attend(0, q.detach(), tables, lens))


@pytest.mark.parametrize("kind", KINDS)
def test_a_key_with_all_the_weight_gives_its_values(kind):
    # every key in turn, in the chunked kernel: its values, rounded once.  Weights of
    # 2^-12 next to the sum's would show where a value lies near the middle between two bfloat16.
    n, d = 200, 64
    cache, rows, tables = filled([n], 4, 8, 1, d, kind, seed=3)
    k, v = HostCache(cache, 0).row(rows[0], n)
    q = (k[:, 0] * 1e18).to(torch.bfloat16).cuda()[:, None].repeat(1, 2, 1)
    x = q[:, 0].double().cpu() @ k[:, 0].T
    x.masked_fill_(torch.arange(n)[None, :] > torch.arange(n)[:, None], -math.inf)
    best = x.topk(2).values
    sure = best[:, 0] - best[:, 1] > 1e-5 * best[:, 0].abs()
    assert sure.sum() > n // 2
    out = cache.attend(0, q, tables, ints([n]), starts_of([n]))
    got, want = out[:, 0].double().cpu()[sure], v[x.argmax(1), 0][sure]
    assert torch.all((got - want).abs() <= (2.0 ** -8 + 2.0 ** -18) * want.abs())
