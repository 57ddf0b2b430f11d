"""Softmax under a learned relative position bias, and its backward pass with the per-example table gradients, on the GPU against
plain 64-bit forms.

Tolerances, u = 2^-24 (half a step of fp32).  A logit t = scale s + b has one rounding; its distance to the largest, times log2 e, another and the
error of that constant; exp2 is good to a step: a probability is off by (|t| + 2 |t - max| + 4) u relative, the sum of K of them by (K / 8 + 32) u
more on top of the worst of those, and a division and a product by 4 u.  dz = p (d - dot): dot is off by (K + 2) u sum |p d|, the difference and
product by 3 u.  Results in bf16 add half a step, 2^-9 .. 2^-8 relative to the value: 2^-8 is used."""
import math

import numpy as np
import pytest
import torch

import paper_2109_12191_amd as dp

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
TINY = 2.0 ** -120               # below this an fp32 exponential may be flushed


def desc_of(n, heads, queries, keys, dtype=torch.float32, buckets=32, max_distance=128, bidirectional=1, causal=0, offset=0, scale=0.25, stride=0):
    return dp.BiasDesc(in_dtype=dp.DP_BF16 if dtype == torch.bfloat16 else dp.DP_F32, n=n, heads=heads, queries=queries, keys=keys, buckets=buckets,
                       max_distance=max_distance, bidirectional=bidirectional, causal=causal, query_offset=offset, scale=scale, row_stride=stride)


def places(desc, ql, kl):
    """[n, queries, keys]: buckets, and which places count."""
    lut = {}
    bucket = np.zeros((desc.n, desc.queries, desc.keys), dtype=np.int64)
    there = np.zeros(bucket.shape, dtype=bool)
    for i in range(desc.n):
        first = kl[i] - ql[i] if desc.query_offset < 0 else desc.query_offset
        d = first + np.arange(desc.queries)[:, None] - np.arange(desc.keys)[None, :]
        for v in np.unique(d):
            if v not in lut:
                lut[v] = dp.dp_bias_bucket(desc, int(v))
        bucket[i] = np.vectorize(lut.get)(d)
        there[i] = (np.arange(desc.queries)[:, None] < ql[i]) & (np.arange(desc.keys)[None, :] < kl[i])
        if desc.causal:
            there[i] &= d >= 0
    return bucket, there


def lengths(rng, n, most, ragged):
    v = np.full(n, most)
    if ragged:
        v = rng.integers(0, most + 1, n)
        v[0] = most
        if n > 1:
            v[1] = 0
        if n > 2:
            v[2] = 1
    return v


def rows(t, stride, start=0, fill=0.0):
    """A tensor [..., keys] as rows of `stride` elements that begin `start` elements in: (buffer, view)."""
    shape = tuple(t.shape[:-1])
    count = int(np.prod(shape))
    buf = torch.full((start + count * stride + 64,), fill, dtype=t.dtype, device="cuda:0")
    view = buf[start:start + count * stride].view(*shape, stride)[..., :t.shape[-1]]
    view.copy_(t)
    return buf, view


def device_lengths(v, ragged):
    return torch.from_numpy(v.astype(np.int32)).cuda() if ragged else None


CASES = [
    # n, heads, queries, keys, ragged, extra descriptor fields
    (1, 1, 1, 1, False, {}),
    (3, 2, 1, 300, True, dict(causal=1, offset=-1, bidirectional=0)),          # decoding
    (4, 3, 1, 5000, True, dict(causal=1, offset=-1, bidirectional=0)),
    (2, 3, 7, 9, False, {}),
    (3, 2, 33, 33, True, dict(causal=1)),
    (3, 2, 5, 260, True, dict(offset=-1)),
    (2, 2, 70, 513, True, dict(causal=1, offset=100, bidirectional=0)),
    (2, 2, 300, 300, False, {}),
    (2, 1, 300, 1100, True, dict(buckets=64, max_distance=512)),
    (1, 2, 257, 700, False, dict(causal=1, bidirectional=0, buckets=16, max_distance=64)),
    (1, 1, 40, 2049, False, dict(buckets=8, max_distance=4096)),
    (1, 1, 9, 9000, True, dict(offset=6000)),
    (1, 1, 3, 17001, False, dict(offset=9000)),
    (2, 1, 2, 32768, True, dict(causal=1, offset=-1)),
    (1, 2, 2, 32769, False, dict(offset=20000)),
    (1, 1, 2, 70002, False, dict(causal=1, offset=-1, bidirectional=0)),
    (2, 1, 20, 30, False, dict(buckets=2, max_distance=2, bidirectional=0)),
    (2, 1, 20, 30, False, dict(buckets=4, max_distance=9)),
    (2, 2, 150, 130, True, dict(stride=133)),
    (2, 2, 150, 130, True, dict(stride=136, causal=1)),
    # more than 16384 rows of at most 256 keys: several to a wave
    (10, 9, 210, 64, True, dict(causal=1)),
    (3, 19, 300, 128, False, {}),
    (4, 22, 200, 250, True, dict(buckets=8, max_distance=20)),
    (4, 22, 190, 201, True, dict(causal=1, bidirectional=0)),
    (30, 14, 40, 9, True, {}),
    (30, 14, 40, 6, True, dict(causal=1, offset=2)),
    (2, 33, 260, 256, True, dict(offset=-1)),
    (5, 24, 140, 120, True, dict(stride=124)),
    (5, 24, 140, 119, True, dict(stride=123, buckets=4, max_distance=4000)),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_softmax(case, dtype):
    n, heads, queries, keys, ragged, extra = case
    desc = desc_of(n, heads, queries, keys, dtype, **extra)
    rng = np.random.default_rng([n, queries, keys])
    s = torch.from_numpy(rng.standard_normal((n, heads, queries, keys)) * 8).to(dtype)
    table = torch.from_numpy(rng.standard_normal((desc.buckets, heads))).float()
    kl = lengths(rng, n, keys, ragged)
    ql = lengths(rng, n, queries, ragged and desc.query_offset >= 0)
    bucket, there = places(desc, ql, kl)
    t = s.double().numpy() * 0.25 + table.double().numpy()[bucket].transpose(0, 3, 1, 2)
    where = np.broadcast_to(there[:, None], t.shape)
    z = np.where(where, t, -math.inf)
    top = np.where(where.any(3, keepdims=True), z.max(3, keepdims=True), 0.0)
    e = np.exp(z - top)
    total = e.sum(3, keepdims=True)
    want = e / np.where(total == 0, 1.0, total)
    rel = (np.abs(t) + 2 * np.abs(t - top) + 4) * u
    worst = np.where(where, rel, 0.0).max(3, keepdims=True) + (keys / 8 + 36) * u
    bound = want * (rel + worst + (2.0 ** -8 if dtype == torch.bfloat16 else 0.0)) + TINY
    # places that do not count hold NaN, infinities and the type's lowest value
    dirty = s.clone()
    junk = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(dtype).min], dtype=dtype)
    hidden = torch.from_numpy(~where)
    dirty[hidden] = junk[torch.arange(int(hidden.sum())) % 4]
    stride = desc.row_stride or keys
    for start in ((0,) if stride == keys else (0, 3)):
        _, view = rows(dirty, stride, start, math.nan)
        out, probs = rows(torch.full_like(s, 5.0), stride, start, 9.0)
        dp.dp_bias_softmax(desc, view, table.cuda(), probs, query_lengths=device_lengths(ql, ragged and desc.query_offset >= 0),
                           key_lengths=device_lengths(kl, ragged))
        torch.cuda.synchronize()
        got = probs.double().cpu().numpy()
        assert np.isfinite(got).all()
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
        assert (got[~where] == 0.0).all()
        out[start:start + n * heads * queries * stride].view(-1, stride)[:, :keys] = 9.0
        assert (out == 9.0).all()                                  # nothing between rows, before or behind them was written
        dp.dp_bias_softmax(desc, view, table.cuda(), view, query_lengths=device_lengths(ql, ragged and desc.query_offset >= 0),
                           key_lengths=device_lengths(kl, ragged))        # in place
        assert np.array_equal(view.double().cpu().numpy(), got)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_softmax_of_rows_that_masks_leave_empty_or_nearly(dtype):
    """Masks added to the scores: -inf, and the type's lowest value; a row of them alone."""
    low = torch.finfo(dtype).min
    s = torch.zeros(1, 1, 5, 70, dtype=dtype)
    s[0, 0, 0] = -math.inf
    s[0, 0, 1, 3:] = -math.inf
    s[0, 0, 2] = low
    s[0, 0, 3, :69] = low
    s[0, 0, 4, 7] = 30.0
    desc = desc_of(1, 1, 5, 70, dtype, scale=1.0)
    table = torch.zeros(32, 1, device="cuda:0")
    probs = torch.empty(s.shape, dtype=dtype, device="cuda:0")
    dp.dp_bias_softmax(desc, s.cuda(), table, probs)
    got = probs.double().cpu().numpy()[0, 0]
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    assert (got[0] == 0).all()
    assert np.allclose(got[1, :3], 1 / 3, rtol=8 * u + half, atol=0) and (got[1, 3:] == 0).all()
    assert np.allclose(got[2], 1 / 70, rtol=64 * u + half, atol=0)          # all equal: uniform
    assert (got[3, :69] == 0).all() and got[3, 69] == 1.0
    assert abs(got[4].sum() - 1) <= 70 * u + half and got[4, 7] > 0.999


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(case, dtype):
    n, heads, queries, keys, ragged, extra = case
    desc = desc_of(n, heads, queries, keys, dtype, **extra)
    rng = np.random.default_rng([n, queries, keys, 1])
    kl = lengths(rng, n, keys, ragged)
    ql = lengths(rng, n, queries, ragged and desc.query_offset >= 0)
    bucket, there = places(desc, ql, kl)
    where = np.broadcast_to(there[:, None], (n, heads, queries, keys))
    e = np.where(where, np.exp(rng.standard_normal(where.shape)), 0.0)
    total = e.sum(3, keepdims=True)
    p = torch.from_numpy(e / np.where(total == 0, 1.0, total)).to(dtype)
    d = torch.from_numpy(rng.standard_normal(where.shape) * 0.01).to(dtype)
    pv, dv = p.double().numpy(), np.where(where, d.double().numpy(), 0.0)
    dot = (pv * dv).sum(3, keepdims=True)
    dz = pv * (dv - dot)
    off = pv * ((keys + 2) * u * np.abs(pv * dv).sum(3, keepdims=True) + 3 * u * np.abs(dv - dot))
    want = 0.25 * dz
    half = 2.0 ** -8 if dtype == torch.bfloat16 else u
    bound = 0.25 * off + half * (np.abs(want) + 0.25 * off) + 2.0 ** -130
    table, room = np.zeros((n, desc.buckets, heads)), np.zeros((n, desc.buckets, heads))
    for i in range(n):
        for h in range(heads):
            table[i, :, h] = np.bincount(bucket[i].ravel(), dz[i, h].ravel(), desc.buckets)
            # terms off by `off`, and sums of at most queries + keys + 64 of them in a row
            room[i, :, h] = np.bincount(bucket[i].ravel(), (off[i, h] + (queries + keys + 64) * u * np.abs(dz[i, h])).ravel(), desc.buckets)
    dirty = d.clone()
    hidden = torch.from_numpy(~where)
    junk = torch.tensor([math.nan, math.inf, -math.inf, torch.finfo(dtype).min], dtype=dtype)
    dirty[hidden] = junk[torch.arange(int(hidden.sum())) % 4]
    stride = desc.row_stride or keys
    g_stride = (desc.buckets * heads + 7) // 4 * 4
    need = dp.dp_bias_workspace_bytes(desc)
    kw = dict(query_lengths=device_lengths(ql, ragged and desc.query_offset >= 0), key_lengths=device_lengths(kl, ragged))
    seen = []
    for start in (0, 0) if stride == keys else (0, 3):
        _, pview = rows(p, stride, start, math.nan)
        _, dview = rows(dirty, stride, start, math.nan)
        out, ds = rows(torch.full_like(p, 5.0), stride, start, 9.0)
        g = torch.full((n, g_stride), -7.0, device="cuda:0")
        sq = torch.full((n + 1,), -7.0, device="cuda:0")
        ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda:0")
        dp.dp_bias_softmax_backward(desc, pview, dview, ds, g, sq, ws, g_stride=g_stride, ws_bytes=need, **kw)
        torch.cuda.synchronize()
        assert (ws[need:] == 0xA5).all() and sq[n] == -7.0 and (g[:, desc.buckets * heads:] == -7.0).all()
        got = ds.double().cpu().numpy()
        assert np.isfinite(got).all() and (got[~where] == 0.0).all()
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
        got_g = g[:, :desc.buckets * heads].reshape(n, desc.buckets, heads).double().cpu().numpy()
        assert (np.abs(got_g - table) <= room + 1e-300).all()
        exact = (got_g ** 2).sum((1, 2))
        assert (np.abs(sq[:n].double().cpu().numpy() - exact) <= (desc.buckets * heads / 4 + 16) * u * exact).all()
        out[start:start + n * heads * queries * stride].view(-1, stride)[:, :keys] = 9.0
        assert (out == 9.0).all()
        dp.dp_bias_softmax_backward(desc, pview, dview, dview, g, None, ws, g_stride=g_stride, ws_bytes=need, **kw)   # in place of dprobs
        assert np.array_equal(dview.double().cpu().numpy(), got)
        seen.append((got_g, got))
    if stride == keys:
        assert all(np.array_equal(a, b) for a, b in zip(*seen))


def test_table_gradient_by_differences():
    """L = sum of w * softmax(scale s + table): differences of it in 64 bits, against the table's gradient of forward and backward."""
    n, heads, queries, keys = 2, 2, 12, 20
    desc = desc_of(n, heads, queries, keys, torch.float32, buckets=8, max_distance=16)
    rng = np.random.default_rng(3)
    s, w = rng.standard_normal((n, heads, queries, keys)).astype(np.float32), rng.standard_normal((n, heads, queries, keys)).astype(np.float32)
    table = rng.standard_normal((8, heads)).astype(np.float32)
    kl, ql = np.full(n, keys), np.full(n, queries)
    bucket, _ = places(desc, ql, kl)
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    probs, ds = torch.empty(s.shape, device="cuda:0"), torch.empty(s.shape, device="cuda:0")
    g, sq = torch.empty(n, 8, heads, device="cuda:0"), torch.empty(n, device="cuda:0")
    ws = torch.empty(dp.dp_bias_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")
    dp.dp_bias_softmax(desc, dev(s), dev(table), probs)
    dp.dp_bias_softmax_backward(desc, probs, dev(w), ds, g, sq, ws)

    def loss(i, tab):
        z = s[i].astype(np.float64) * 0.25 + tab[bucket[i]].transpose(2, 0, 1)
        e = np.exp(z - z.max(2, keepdims=True))
        return (w[i] * e / e.sum(2, keepdims=True)).sum()
    step = 1e-5
    for i in range(n):
        for b in range(8):
            for h in range(heads):
                up, down = table.astype(np.float64), table.astype(np.float64)
                up[b, h] += step
                down[b, h] -= step
                slope = (loss(i, up) - loss(i, down)) / (2 * step)
                # differences: step^2 |L'''| / 6 <= 1e-10 sum |w|, rounding 1e-16 / step of it; fp32 probabilities: 64 u of sum |w p|
                assert abs(slope - float(g[i, b, h])) <= 2e-10 * np.abs(w[i]).sum() + 128 * u * np.abs(w[i]).sum()


def test_recorded_and_on_another_stream():
    n, heads, queries, keys = 3, 2, 130, 200
    desc = desc_of(n, heads, queries, keys, torch.bfloat16)
    s = torch.randn(n, heads, queries, keys, device="cuda:0").bfloat16()
    w = torch.randn_like(s)
    table = torch.randn(32, heads, device="cuda:0")
    probs, ds, g, sq = torch.empty_like(s), torch.empty_like(s), torch.empty(n, 32, heads, device="cuda:0"), torch.empty(n, device="cuda:0")
    ws = torch.empty(dp.dp_bias_workspace_bytes(desc), dtype=torch.uint8, device="cuda:0")

    def step():
        dp.dp_bias_softmax(desc, s, table, probs)
        dp.dp_bias_softmax_backward(desc, probs, w, ds, g, sq, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(4):
        s.copy_(torch.randn(s.shape, device="cuda:0"))
        step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in (probs, ds, g, sq)]
        for t in (probs, ds, g, sq):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (probs, ds, g, sq)))
