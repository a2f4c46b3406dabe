"""Attention over packed prompts against the float64 form, row by row.

Tolerance: the weights are rounded to 16 bits (relative 2^-11 in float16, 2^-8
in bfloat16), the result once more, and a score of float32 products is off by
at most d 2^-24 sum|q k| < 2^-12 here (sum|q k| scale < 16), which moves its
weight by that factor: |err| <= w sum_j p_j |v_j| + e |out| with w = 2^-11 + 2^-12 and
2^-8 + 2^-12, e the half unit of the type."""
import math

import numpy as np
import pytest
import torch

import paper_2607_16973_amd as tq
from tests.reader import attention64, starts_of

pytestmark = pytest.mark.gpu
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def rows(counts, heads, d, dtype, seed, pad=0):
    """Packed vectors; pad: elements between tokens (odd strides)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(counts)
    x = torch.randn(n, heads * d + pad, generator=g, device="cuda").to(dtype)
    return x[:, pad:].reshape(n, heads, d) if pad == 0 else x[:, pad:].unflatten(1, (heads, d))


def check(q, k, v, counts, key_counts, out, lse, causal=True, scale=None):
    d = q.shape[2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    e = HALF[q.dtype]
    t = u = 0
    for n, m in zip(counts, key_counts):
        pos = [i + m - n if causal else m - 1 for i in range(n)]
        ref, rl, size = attention64(q[t:t + n], k[u:u + m], v[u:u + m], pos, scale)
        got, gl = out[t:t + n].double().cpu(), lse[t:t + n].double().cpu()
        assert torch.all((got - ref).abs() <= (e + 2.0 ** -12) * size + e * ref.abs() + 2.0 ** -24)
        assert torch.equal(torch.isinf(gl), torch.isinf(rl))
        fin = ~torch.isinf(rl)
        assert torch.all((gl - rl)[fin].abs() <= 2.0 ** -12 + 2.0 ** -20 * rl[fin].abs())
        t, u = t + n, u + m


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (6, 2), (7, 1)])
def test_lengths(heads, kv_heads, d, dtype):
    counts = [1, 0, 2, 63, 64, 65, 31, 129, 1, 200]
    q, k, v = (rows(counts, h, d, dtype, s) for h, s in ((heads, 1), (kv_heads, 2), (kv_heads, 3)))
    out, lse = tq.attention(q, k, v, starts_of(counts), return_lse=True)
    check(q, k, v, counts, counts, out, lse)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("causal", [True, False])
def test_keys_of_other_lengths(causal, dtype):
    # a prefix, fewer keys than queries (rows that see nothing), no keys, no queries
    counts, keys = [5, 70, 40, 3, 0, 130], [75, 70, 33, 0, 12, 129]
    q, k, v = rows(counts, 6, 64, dtype, 4), rows(keys, 3, 64, dtype, 5), rows(keys, 3, 64, dtype, 6)
    out, lse = tq.attention(q, k, v, starts_of(counts), starts_of(keys), causal=causal, scale=0.3, return_lse=True)
    check(q, k, v, counts, keys, out, lse, causal, 0.3)


@pytest.mark.parametrize("pad", [1, 8, 20])
@pytest.mark.parametrize("d", [64, 128])
def test_strides(d, pad):
    counts = [77, 130]
    q, k, v = (rows(counts, 3, d, torch.bfloat16, 10 + s, pad) for s in range(3))
    out, lse = tq.attention(q, k, v, starts_of(counts), return_lse=True)
    check(q, k, v, counts, counts, out, lse)
    # heads outermost: token stride d, head stride n d
    q, k, v = (rows(counts, 3, d, torch.float16, 20 + s).transpose(0, 1).contiguous().transpose(0, 1) for s in range(3))
    out, lse = tq.attention(q, k, v, starts_of(counts), return_lse=True)
    check(q, k, v, counts, counts, out, lse)
    # one key head read by all: head stride 0
    k1, v1 = k[:, :1].expand(-1, 3, -1), v[:, :1].expand(-1, 3, -1)
    out, lse = tq.attention(q, k1, v1, starts_of(counts), return_lse=True)
    check(q, k1, v1, counts, counts, out, lse)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_nonfinite_values_reach_only_who_sees_them(bad, dtype):
    counts = [100, 90, 80]
    q, k, v = (rows(counts, 2, 128, dtype, 30 + s) for s in range(3))
    clean = tq.attention(q, k, v, starts_of(counts))
    k2, v2 = k.clone(), v.clone()
    v2[100 + 70, :, 5] = bad          # row 1: queries from 70 on
    k2[190 + 79] = bad                # row 2: the last query
    out = tq.attention(q, k2, v2, starts_of(counts))
    assert torch.equal(out[:100], clean[:100]) and torch.equal(out[190:269], clean[190:269])
    assert torch.equal(out[100:170], clean[100:170])
    assert not torch.isfinite(out[170:190, :, 5]).any()
    other = [j for j in range(128) if j != 5]
    assert torch.equal(out[170:190][..., other], clean[170:190][..., other])


def test_large_scores_and_equal_ones():
    # one key far above the rest; all keys the same: the mean of the values
    counts = [150]
    q, k, v = (rows(counts, 2, 64, torch.bfloat16, 40 + s) for s in range(3))
    k[20] = 30 * q[60]
    out, lse = tq.attention(q, k, v, starts_of(counts), return_lse=True)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    assert torch.equal(out[60], v[20])
    k[:] = k[0, 0]
    out, lse = tq.attention(q, k, v, starts_of(counts), return_lse=True)
    mean = v.double().cumsum(0) / torch.arange(1, 151, device="cuda")[:, None, None]
    assert torch.all((out.double() - mean).abs() <= 2.0 ** -7 * (v.double().abs().max()))


@pytest.mark.parametrize("size", [1e4, 1e8, 1e18])
def test_scores_past_float32s_fractions(size):
    # one key takes all, whatever the scores' rounding: the others are hundreds below
    counts = [90]
    q, k, v = (rows(counts, 1, 64, torch.bfloat16, 45 + s) for s in range(3))
    out, lse = tq.attention(q * size, k, v, starts_of(counts), return_lse=True)
    x = (q * size)[:, 0].double() @ k[:, 0].double().T
    x.masked_fill_(torch.ones(90, 90, dtype=torch.bool, device="cuda").triu(1), -math.inf)
    best = x.topk(2).values
    sure = (best[:, 0] - best[:, 1] > 1e-5 * best[:, 0].abs() + 500)
    assert sure.sum() > 60
    assert torch.equal(out[sure, 0], v[x.argmax(1), 0][sure])
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


def test_repeats_are_equal_and_streams():
    counts = [300, 5, 211]
    q, k, v = (rows(counts, 8, 128, torch.bfloat16, 50 + s) for s in range(3))
    st = starts_of(counts)
    first = tq.attention(q, k, v, st)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = tq.attention(q, k, v, st)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)
    out = torch.full_like(first, 7)
    got = tq.attention(q, k, v, st, out=out, longest=300)
    assert got.data_ptr() == out.data_ptr() and torch.equal(out, first)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_rows_do_not_depend_on_each_other(dtype):
    # scores of one head far above the others': their results stay the same bits
    counts = [300]
    q, k, v = (rows(counts, h, 64, dtype, 90 + s) for s, h in enumerate((4, 1, 1)))
    want = tq.attention(q, k, v, starts_of(counts))
    for size in (20, 1e4):
        q2 = q.clone()
        q2[:, 1] *= size
        out = tq.attention(q2, k, v, starts_of(counts))
        assert torch.equal(out[:, [0, 2, 3]], want[:, [0, 2, 3]])


def test_longest_is_a_hint():
    counts = [700, 3, 0, 129, 1500]
    q, k, v = (rows(counts, h, 64, torch.float16, 80 + h) for h in (6, 2, 3))
    v = v[:, :2]
    st = starts_of(counts)
    want = tq.attention(q, k, v, st)
    for longest in (1500, 2000, 1499, 700, 40, 1):
        assert torch.equal(tq.attention(q, k, v, st, longest=longest), want)


def test_graph():
    counts = [64, 17]
    q, k, v = (rows(counts, 4, 64, torch.float16, 60 + s) for s in range(3))
    st = starts_of(counts)
    eager = tq.attention(q, k, v, st)
    out = torch.empty_like(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tq.attention(q, k, v, st, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager)
        q2 = q * 2
        del q2


def test_long_row_against_float64_samples():
    n, d = 5001, 128
    q, k, v = (rows([n], h, d, torch.bfloat16, 70 + h) for h in (8, 2, 3))
    v = v[:, :2]
    out, lse = tq.attention(q, k, v, starts_of([n]), return_lse=True)
    at = [0, 1, 63, 64, 2047, 4095, 5000] + np.random.RandomState(0).randint(0, n, 10).tolist()
    ref, rl, size = attention64(q[at], k, v, at, 1 / math.sqrt(d))
    got = out[at].double().cpu()
    e = HALF[torch.bfloat16]
    assert torch.all((got - ref).abs() <= (e + 2.0 ** -12) * size + e * ref.abs())
    assert torch.all((lse[at].double().cpu() - rl).abs() <= 2.0 ** -12)


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_scale_of_zero_weighs_all_keys_alike(d, scale):
    counts, keys = [70, 3, 130], [75, 2, 130]
    q, k, v = rows(counts, 4, d, torch.float16, 50), rows(keys, 2, d, torch.float16, 51), rows(keys, 2, d, torch.float16, 52)
    for causal in (True, False):
        out, lse = tq.attention(q, k, v, starts_of(counts), starts_of(keys), causal=causal, scale=scale, return_lse=True)
        check(q, k, v, counts, keys, out, lse, causal, scale)


@pytest.mark.parametrize("heads,kv_heads,most", [(4, 2, 3000), (40, 1, 300), (3, 3, 1500)])
def test_rows_of_any_lengths_as_each_alone(heads, kv_heads, most):
    # every tile of every row is somebody's, in whatever order they are taken
    r = np.random.RandomState(heads)
    counts = [int(n) for n in most * r.rand(90) ** 4]
    counts[5], counts[40], counts[-1] = most, 0, most // 2
    q, k, v = (rows(counts, h, 64, torch.bfloat16, s) for h, s in ((heads, 61), (kv_heads, 62), (kv_heads, 63)))
    out, lse = tq.attention(q, k, v, starts_of(counts), return_lse=True)
    t = 0
    for n in counts:
        one, one_lse = tq.attention(q[t:t + n], k[t:t + n], v[t:t + n], starts_of([n]), return_lse=True)
        assert torch.equal(out[t:t + n], one) and torch.equal(lse[t:t + n], one_lse)
        t += n
