"""CPU-only checks of what the token operators ask of their callers at the ends of their ranges."""
import os

import pytest
import torch

import paper_2109_12191_amd as dp


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(dp.lib_path()):
        from paper_2109_12191_amd.build import build
        build(verbose=False)
    return dp.load_library()


def _need(n, tokens, cin, cout, bias=0, dtype=dp.DP_BF16):
    desc = dp.LayerDesc(kind=dp.DP_DENSE, in_dtype=dtype, n=n, cin=cin, cout=cout, h=tokens, w=1, has_bias=bias)
    return dp.dp_checkpoint_workspace_bytes(desc, dp.DP_WS_RECOMPUTE)


@pytest.mark.parametrize("tokens,cin,cout,bias", [(64, 768, 768, 0), (512, 512, 512, 0), (512, 384, 384, 1), (100, 512, 512, 0), (16, 768, 768, 1), (256, 512, 512, 0),
                                                  (40, 100, 1000, 1), (17, 32, 40, 1), (700, 4096, 2048, 0)])
def test_workspace_of_a_clipped_sum_holds_every_part_of_it(tokens, cin, cout, bias):
    """Calls of more than 1024 examples go in launches of 1024 and one of the rest, each with the ranges that it takes by itself."""
    whole = _need(1024, tokens, cin, cout, bias)
    alone = {rest: _need(rest, tokens, cin, cout, bias) for rest in range(1, 1024)}
    for n in list(range(1025, 2048)) + [2049, 3000, 5000, 65535]:
        assert _need(n, tokens, cin, cout, bias) >= max(whole, alone.get(n % 1024, 0)), n


def test_attention_block_refuses_tensors_of_another_device(monkeypatch):
    """The calls take addresses: a tensor of another GPU, or a block on another than the current one, is refused before any of them."""
    block = dp.PrivateAttention(2, 4, 32, 4, clip_c=1.0, sigma=1.0, total_batch=2, device="cpu")

    class Elsewhere:
        """What the checks look at."""
        def __init__(self, shape, device, dtype=torch.bfloat16):
            self.shape, self.device, self.dtype = shape, torch.device(device), dtype

        def is_contiguous(self):
            return True

        def contiguous(self):
            return self
    block.theta = Elsewhere((4,), "cuda:0", torch.float32)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for call in (block.forward, block.backward):
        with pytest.raises(ValueError, match="cuda:1"):
            call(Elsewhere((2, 4, 32), "cuda:1"))
    with pytest.raises(ValueError, match="cuda:1"):
        block.forward(Elsewhere((2, 4, 32), "cuda:0"), Elsewhere((2,), "cuda:1", torch.int32))
    with pytest.raises(ValueError, match="cpu"):
        block.forward(torch.zeros((2, 4, 32), dtype=torch.bfloat16))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device is 1"):
        block.forward(Elsewhere((2, 4, 32), "cuda:0"))


def test_lengths_of_another_type_or_place_are_refused():
    """torch makes int64 of a list of numbers, on the host."""
    fake = 0x1000
    dense = dp.LayerDesc(kind=dp.DP_DENSE, in_dtype=dp.DP_BF16, n=3, cin=48, cout=40, h=20, w=1, has_bias=0)
    bias = dp.BiasDesc(in_dtype=dp.DP_BF16, n=3, heads=2, queries=5, keys=7, buckets=32, max_distance=128, bidirectional=1, causal=0, query_offset=0,
                       scale=1.0, row_stride=0)
    room = 1 << 30
    calls = [("lengths", lambda t: dp.dp_checkpoint_example_grad(dense, fake, fake, fake, None, None, fake, fake, lengths=t, ws_bytes=room, stream=0)),
             ("lengths", lambda t: dp.dp_checkpoint_clip_accumulate(dense, fake, fake, fake, fake, 1.0, fake, None, fake, lengths=t, ws_bytes=room, stream=0))]
    for which in ("query_lengths", "key_lengths"):
        calls.append((which, lambda t, w=which: dp.dp_bias_softmax(bias, fake, fake, fake, stream=0, **{w: t})))
        calls.append((which, lambda t, w=which: dp.dp_bias_softmax_backward(bias, fake, fake, fake, fake, None, fake, ws_bytes=room, stream=0, **{w: t})))
    for what, call in calls:
        for bad in (torch.tensor([1, 2, 3]), torch.zeros(3), torch.zeros(2, dtype=torch.int32), torch.zeros(6, dtype=torch.int32)[::2],
                    torch.zeros(3, dtype=torch.int32)):
            with pytest.raises(dp.DpError, match=what) as error:
                call(bad)
            assert error.value.status == dp.binding.DP_ERR_INVALID_ARG


def test_rows_of_views_with_dimensions_of_one():
    """Rows that are evenly spaced, whatever stride a dimension of one element has."""
    rows = dp.binding._rows_of
    x = torch.zeros(4, 6, 48)
    assert rows(x[:, 2:3]) == (dp.DP_F32, 4, 48, 6 * 48)                 # one token of each example
    assert rows(x[:, 2:3, :40]) == (dp.DP_F32, 4, 40, 6 * 48)
    assert rows(x[1:2]) == (dp.DP_F32, 6, 48, 48)
    assert rows(torch.zeros(2, 1, 3, 48).as_strided((2, 1, 3, 48), (144, 7, 48, 1))) == (dp.DP_F32, 6, 48, 48)
    assert rows(torch.zeros(5, 1, 1, 48)[::2]) == (dp.DP_F32, 3, 48, 96)
    assert rows(torch.zeros(1, 1, 48)) == (dp.DP_F32, 1, 48, 48) and rows(torch.zeros(3, 1)) == (dp.DP_F32, 3, 1, 1)
    assert rows(torch.zeros(1, 48).expand(1, 48)) == (dp.DP_F32, 1, 48, 48)
    assert rows(torch.zeros(0, 48))[1:3] == (0, 48) and rows(torch.zeros(4, 0, 48))[1:3] == (0, 48)
    for bad in (x[:, :2], x.transpose(0, 1), torch.zeros(1, 48).expand(3, 48), torch.zeros(48, 4).t(), torch.zeros(4, 0), x.expand(2, 4, 6, 48), torch.zeros(())):
        with pytest.raises(dp.DpError):
            rows(bad)
