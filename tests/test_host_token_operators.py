"""CPU-only checks of the calls for token models (8-bit activation checkpoints, softmax under a relative position bias): what they
refuse, before anything could be launched, and their pure-host queries."""
import ctypes
import math
import os
from fractions import Fraction

import pytest
import torch

import paper_2109_12191_amd as dp
from paper_2109_12191_amd import binding as B

FAKE = 0x1000          # a non-null, 16-byte aligned "device pointer" that is never dereferenced
INT = B.DP_ERR_INVALID_ARG


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dp.lib_path()):
        from paper_2109_12191_amd.build import build
        build(verbose=False)
    return dp.load_library()


def _raises(status, fn, *a, **k):
    with pytest.raises(dp.DpError) as ei:
        fn(*a, **k)
    assert ei.value.status == status, str(ei.value)
    return str(ei.value)


def test_checkpoint_pitch(lib):
    assert [dp.dp_checkpoint_pitch(f) for f in (1, 31, 32, 33, 1003, 1 << 20)] == [32, 32, 32, 64, 1024, 1 << 20]
    for bad in (0, -1, (1 << 20) + 1):
        _raises(INT, dp.dp_checkpoint_pitch, bad)


def _c_write(x=FAKE, dtype=dp.DP_BF16, rows=4, features=48, stride=0, codes=FAKE, scales=FAKE):
    B._check(dp.load_library().dp_checkpoint_write(x, dtype, rows, features, stride, codes, scales, None))


def _c_read(x=FAKE, dtype=dp.DP_BF16, rows=4, features=48, stride=0, codes=FAKE, scales=FAKE):
    B._check(dp.load_library().dp_checkpoint_read(codes, scales, rows, features, x, dtype, stride, None))


@pytest.mark.parametrize("call", [_c_write, _c_read])
def test_checkpoint_calls_refuse(lib, call):
    for bad in (dict(x=None), dict(codes=None), dict(scales=None), dict(dtype=7), dict(features=0), dict(features=-5),
                dict(features=(1 << 20) + 1), dict(stride=47), dict(codes=FAKE + 8), dict(x=FAKE + 1), dict(x=FAKE + 2, dtype=dp.DP_F32)):
        assert _raises(INT, call, **bad)
    _raises(B.DP_ERR_UNSUPPORTED, call, rows=1 << 31)
    call(rows=0)                                     # no row: nothing to do, nothing launched


def test_checkpoint_binding_refuses_what_is_not_rows(lib):
    x = torch.zeros(4, 48)
    codes, scales = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    for fn in (lambda t, c=codes, s=scales: dp.dp_checkpoint_write(t, c, s, stream=0),
               lambda t, c=codes, s=scales: dp.dp_checkpoint_read(c, s, t, stream=0)):
        _raises(B.DP_ERR_UNSUPPORTED, fn, x.double())
        _raises(INT, fn, torch.zeros(48, 4).t())                       # features not consecutive
        _raises(INT, fn, torch.zeros(1, 48).expand(4, 48))             # rows on top of each other
        _raises(INT, fn, torch.zeros(4, 3, 48)[:, :2])                 # leading dimensions not evenly spaced
        _raises(INT, fn, x, codes[:3])
        _raises(INT, fn, x, codes, scales[:, :1])
        _raises(INT, fn, x, torch.zeros(4, 64, dtype=torch.int32))
    assert B._rows_of(torch.zeros(2, 3, 48)[..., :40]) == (dp.DP_F32, 6, 40, 48)
    assert B._rows_of(torch.zeros(5, 48, dtype=torch.bfloat16)[::2]) == (dp.DP_BF16, 3, 48, 96)
    assert B._rows_of(torch.zeros(48)) == (dp.DP_F32, 1, 48, 48)


def _desc(**k):
    d = dict(kind=dp.DP_DENSE, in_dtype=dp.DP_BF16, n=3, cin=48, cout=40, h=20, w=1, has_bias=1)
    d.update(k)
    return dp.LayerDesc(**d)


def test_checkpoint_gradients_refuse(lib):
    ws = dp.dp_checkpoint_workspace_bytes(_desc())
    assert ws >= 4 * 3

    def call(desc=_desc(), codes=FAKE, scales=FAKE, dy=FAKE, gw=FAKE, gb=FAKE, sq=FAKE, w=FAKE, wb=ws, lengths=None, gs=0):
        dp.dp_checkpoint_example_grad(desc, codes, scales, dy, gw, gb, sq, w, lengths=lengths, g_stride=gs, ws_bytes=wb, stream=0)
    for bad in (dict(codes=None), dict(scales=None), dict(dy=None), dict(codes=FAKE + 4), dict(dy=FAKE + 2), dict(gw=FAKE + 4),
                dict(lengths=FAKE + 2), dict(sq=FAKE + 2), dict(gw=None, gb=None, sq=None), dict(gb=None), dict(gw=None), dict(gs=6),
                dict(gs=8), dict(w=FAKE + 4), dict(desc=_desc(n=0)), dict(desc=_desc(h=0)), dict(desc=_desc(w=2)), dict(desc=_desc(in_dtype=9)),
                dict(desc=_desc(has_bias=0))):
        assert _raises(INT, call, **bad)
    for bad in (dict(wb=ws - 1), dict(w=None)):
        _raises(B.DP_ERR_WORKSPACE, call, **bad)
    conv = dp.LayerDesc(kind=dp.DP_CONV2D, n=2, cin=8, cout=8, h=8, w=8, kh=3, kw=3, stride=1, pad=1)
    for bad in (conv, _desc(cin=(1 << 20) + 1), _desc(n=65536), _desc(h=1 << 27, cin=1)):
        _raises(B.DP_ERR_UNSUPPORTED, call, desc=bad)
        assert dp.dp_checkpoint_workspace_bytes(bad) == 0
    assert dp.dp_checkpoint_workspace_bytes(_desc(), 5) == 0


def test_checkpoint_clip_accumulate_refuses(lib):
    big = _desc(n=64, h=512)                        # few tiles, many tokens: ranges of them meet in the workspace
    ws = dp.dp_checkpoint_workspace_bytes(big, dp.DP_WS_RECOMPUTE)
    assert ws > 0

    def call(desc=big, codes=FAKE, scales=FAKE, dy=FAKE, sq=FAKE, c=1.0, aw=FAKE, ab=FAKE, w=FAKE, wb=ws, lengths=None):
        dp.dp_checkpoint_clip_accumulate(desc, codes, scales, dy, sq, c, aw, ab, w, lengths=lengths, ws_bytes=wb, stream=0)
    for bad in (dict(codes=None), dict(scales=None), dict(dy=None), dict(sq=None), dict(aw=None), dict(ab=None), dict(c=0.0), dict(c=math.nan),
                dict(c=-1.0), dict(lengths=FAKE + 1), dict(aw=FAKE + 4), dict(codes=FAKE + 1), dict(desc=_desc(n=64, h=512, has_bias=0))):
        assert _raises(INT, call, **bad)
    for bad in (dict(wb=ws - 1), dict(w=None)):
        _raises(B.DP_ERR_WORKSPACE, call, **bad)


def _bias(**k):
    d = dict(in_dtype=dp.DP_BF16, n=2, heads=3, queries=5, keys=7, buckets=32, max_distance=128, bidirectional=1, causal=0, query_offset=0,
             scale=1.0, row_stride=0)
    d.update(k)
    return dp.BiasDesc(**d)


def test_bias_calls_refuse(lib):
    ws = dp.dp_bias_workspace_bytes(_bias())
    assert ws >= 2 * 3 * 32 * 4

    def forward(desc=_bias(), s=FAKE, table=FAKE, p=FAKE, ql=None, kl=None):
        dp.dp_bias_softmax(desc, s, table, p, query_lengths=ql, key_lengths=kl, stream=0)

    def backward(desc=_bias(), p=FAKE, d=FAKE, ds=FAKE, g=FAKE, sq=FAKE, w=FAKE, wb=ws, gs=0, ql=None, kl=None):
        dp.dp_bias_softmax_backward(desc, p, d, ds, g, sq, w, query_lengths=ql, key_lengths=kl, g_stride=gs, ws_bytes=wb, stream=0)
    for bad in (dict(s=None), dict(table=None), dict(p=None), dict(s=FAKE + 1), dict(table=FAKE + 2), dict(ql=FAKE + 1), dict(kl=FAKE + 3)):
        assert _raises(INT, forward, **bad)
    for bad in (dict(p=None), dict(d=None), dict(ds=None), dict(g=None), dict(g=FAKE + 4), dict(sq=FAKE + 1), dict(gs=95), dict(gs=98), dict(gs=92),
                dict(w=FAKE + 4), dict(kl=FAKE + 1)):
        assert _raises(INT, backward, **bad)
    for bad in (dict(wb=ws - 1), dict(w=None)):
        _raises(B.DP_ERR_WORKSPACE, backward, **bad)
    for k in (dict(n=0), dict(heads=0), dict(queries=0), dict(keys=-1), dict(in_dtype=4), dict(buckets=0), dict(buckets=2), dict(buckets=31),
              dict(bidirectional=0, buckets=1), dict(max_distance=8), dict(scale=math.inf), dict(scale=math.nan), dict(query_offset=-2),
              dict(row_stride=6)):
        bad = _bias(**k)
        assert _raises(INT, forward, desc=bad) and _raises(INT, backward, desc=bad) and _raises(INT, dp.dp_bias_bucket, bad, 0)
        assert dp.dp_bias_workspace_bytes(bad) == 0
    for k in (dict(max_distance=4097), dict(buckets=514), dict(n=65536), dict(queries=1 << 30), dict(n=65535, heads=65535)):
        bad = _bias(**k)
        _raises(B.DP_ERR_UNSUPPORTED, forward, desc=bad)
        _raises(B.DP_ERR_UNSUPPORTED, backward, desc=bad)


def test_null_descriptor(lib):
    assert lib.dp_bias_softmax(None, FAKE, FAKE, None, None, FAKE, None) == INT
    assert lib.dp_checkpoint_example_grad(None, FAKE, FAKE, FAKE, None, FAKE, FAKE, 0, FAKE, FAKE, ctypes.c_size_t(1 << 20), None) == INT


@pytest.mark.parametrize("buckets,max_distance,bidirectional", [(32, 128, 1), (32, 128, 0), (16, 64, 0), (64, 512, 1), (4, 8, 1), (2, 2, 0), (3, 20, 0),
                                                                (512, 4096, 1), (10, 81, 1), (128, 4096, 0)])
def test_buckets_against_whole_numbers(lib, buckets, max_distance, bidirectional):
    """The definition's floor of a quotient of logarithms, decided in whole numbers: (d / near)^span >= (max / near)^k."""
    desc = _bias(buckets=buckets, max_distance=max_distance, bidirectional=bidirectional)
    nb = buckets // 2 if bidirectional else buckets
    near, span = nb // 2, nb - nb // 2

    def mag(d):
        if d < near:
            return d
        k = 0
        while k < span - 1 and Fraction(d, near) ** span >= Fraction(max_distance, near) ** (k + 1):
            k += 1
        return near + k
    seen = [dp.dp_bias_bucket(desc, d) for d in range(max_distance + 3)]
    step = 1 if max_distance <= 512 else 37
    assert all(seen[d] == mag(d) for d in range(0, max_distance + 3, step))
    assert seen[max_distance] == nb - 1 and sorted(seen) == seen
    for d in (-1, -2, -near, -max_distance, -(1 << 31)):
        want = nb + (mag(-d) if -d <= max_distance else nb - 1) if bidirectional else 0
        assert dp.dp_bias_bucket(desc, d) == want
    assert dp.dp_bias_bucket(desc, (1 << 31) - 1) == nb - 1


def test_attention_block_refuses_other_shapes():
    with pytest.raises(ValueError):
        dp.PrivateAttention(2, 4, 32, 5, clip_c=1.0, sigma=1.0, total_batch=2, device="cpu")
    block = dp.PrivateAttention(2, 4, 32, 4, clip_c=1.0, sigma=1.0, total_batch=2, device="cpu")
    x = torch.zeros((2, 4, 32), dtype=torch.bfloat16)
    cache = torch.zeros((2, 4, 4, 8), dtype=torch.bfloat16)
    lengths = torch.zeros(2, dtype=torch.int32)
    for bad in (x.float(), x[:1], x[:, :3].contiguous(), x.transpose(0, 1), torch.zeros((2, 4, 33), dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            block.forward(bad)
        if bad.is_contiguous():
            with pytest.raises(ValueError):
                block.backward(bad)
    for bad in (lengths.long(), lengths[:1], torch.zeros((2, 2), dtype=torch.int32)):
        with pytest.raises(ValueError):
            block.forward(x, bad)
        with pytest.raises(ValueError):
            block.attend_last(x[:, 0].contiguous(), cache, cache, bad)
    for q, k, v in ((x[:, 0].contiguous(), cache[:, :, :3].contiguous(), cache), (x[:, 0].contiguous(), cache, cache.float()), (x[:1, 0].contiguous(), cache, cache)):
        with pytest.raises(ValueError):
            block.attend_last(q, k, v)
