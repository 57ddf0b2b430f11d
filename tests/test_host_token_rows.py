"""CPU-only checks of what the calls of the operators on either side of a token model's blocks take for their rows: tensors whose memory holds them where the
descriptor says they are.  Nothing is launched: a stand-in for the library notes the addresses."""
import pytest
import torch

import paper_2109_12191_amd as dp
from paper_2109_12191_amd import binding as B

N, TOKENS, WIDTH = 3, 5, 40


class OnDevice(torch.Tensor):
    """A host tensor that says it is on the device."""
    is_cuda = property(lambda self: True)


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def library(monkeypatch):
    stand_in = Library()
    monkeypatch.setattr(B, "load_library", lambda: stand_in)
    return stand_in


def make(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


def norm(row_stride=0, **k):
    return dp.NormDesc(**{**dict(in_dtype=dp.DP_BF16, n=N, tokens=TOKENS, features=WIDTH, rms=0, eps=1e-5, row_stride=row_stride), **k})


def logprob(row_stride=0, **k):
    return dp.LogprobDesc(**{**dict(in_dtype=dp.DP_BF16, n=N, tokens=TOKENS, vocab=WIDTH, top=0, scale=1.0, row_stride=row_stride), **k})


P = 0x1000


def calls_with(t, row_stride=0, **k):
    """Every place of a call that takes rows, as (call, position of the address in the library's call)."""
    d, e = norm(row_stride, **k), logprob(row_stride, **{("vocab" if key == "features" else key): v for key, v in k.items()})
    return [(lambda: dp.dp_layer_norm(d, t, None, None, P, stream=0), 1), (lambda: dp.dp_layer_norm(d, P, None, None, t, stream=0), 5),
            (lambda: dp.dp_layer_norm_backward(d, t, None, P, P, P, P, P, P, ws_bytes=1 << 20, stream=0), 1),
            (lambda: dp.dp_layer_norm_backward(d, P, None, t, P, P, P, P, P, ws_bytes=1 << 20, stream=0), 3),
            (lambda: dp.dp_layer_norm_backward(d, P, None, P, t, P, P, P, P, ws_bytes=1 << 20, stream=0), 5),
            (lambda: dp.dp_token_logprobs(e, t, P, P, None, None, None, None, P, ws_bytes=1 << 20, stream=0), 1),
            (lambda: dp.dp_token_logprobs_backward(e, t, P, None, P, P, P, ws_bytes=1 << 20, stream=0), 1),
            (lambda: dp.dp_token_logprobs_backward(e, P, P, None, P, t, P, ws_bytes=1 << 20, stream=0), 9)]


def wide(more):
    return make(N, TOKENS, WIDTH + more)


GOOD = {
    "packed": lambda: (make(N, TOKENS, WIDTH), 0),
    "packed, said so": lambda: (make(N, TOKENS, WIDTH), WIDTH),
    "rows alone": lambda: (make(N * TOKENS, WIDTH), 0),
    "heads": lambda: (make(N, TOKENS, 4, WIDTH // 4), 0),
    "memory": lambda: (make(N * TOKENS * WIDTH), 0),
    "memory with gaps": lambda: (make((N * TOKENS - 1) * 50 + WIDTH), 50),
    "more than is needed": lambda: (make(N + 2, TOKENS, WIDTH), 0),
    "columns of a wider tensor": lambda: (wide(8)[..., :WIDTH], WIDTH + 8),
    "later columns": lambda: (wide(9)[..., 9:], WIDTH + 9),
    "the wider tensor": lambda: (wide(8), WIDTH + 8),
    "every second token": lambda: (make(N, 2 * TOKENS, WIDTH)[:, ::2], 2 * WIDTH),
    "heads of one of three projections": lambda: (make(N, TOKENS, 3, 4, WIDTH // 4)[:, :, 1], 3 * WIDTH),
    "heads of the first examples": lambda: (make(N + 2, TOKENS, 4, WIDTH // 4), 0),
    "rows with room between them, as dimensions": lambda: (make(N, TOKENS, 2, WIDTH), 2 * WIDTH),
    "an example's values together": lambda: (make(N, TOKENS * WIDTH), 0),
    "an example's tokens as examples": lambda: (make(N * TOKENS, WIDTH + 3)[:, :WIDTH], WIDTH + 3),
}


@pytest.mark.parametrize("case", GOOD)
def test_rows_where_the_descriptor_says(library, case):
    t, row_stride = GOOD[case]()
    for call, place in calls_with(t, row_stride):
        call()
        assert library.calls[-1][1][place] == t.data_ptr()


BAD = {
    "packed, but rows are said to be further apart": lambda: (make(N, TOKENS, WIDTH), WIDTH + 8),
    "memory that ends in the last row": lambda: (make((N * TOKENS - 1) * 50 + WIDTH - 1), 50),
    "columns of a wider tensor, said to be packed": lambda: (wide(8)[..., :WIDTH], 0),
    "the wider tensor, said to be packed": lambda: (wide(8), 0),
    "columns, rows said to be nearer": lambda: (wide(8)[..., :WIDTH], WIDTH + 4),
    "columns, rows said to be further apart": lambda: (wide(8)[..., :WIDTH], WIDTH + 12),
    "tokens first": lambda: (make(TOKENS, N, WIDTH).transpose(0, 1), 0),
    "features first": lambda: (make(N, WIDTH, TOKENS).transpose(1, 2), 0),
    "every second feature": lambda: (make(N, TOKENS, 2 * WIDTH)[..., ::2], 2 * WIDTH),
    "heads first": lambda: (make(N, 4, TOKENS, WIDTH // 4).transpose(1, 2), 0),
    "twice the features, said to be packed": lambda: (make(N, TOKENS, 2 * WIDTH), 0),
    "one example for all": lambda: (make(1, TOKENS, WIDTH).expand(N, TOKENS, WIDTH), 0),
    "one token for all": lambda: (make(1, 1, WIDTH).expand(N, TOKENS, WIDTH), 0),
    "some tokens of longer examples": lambda: (make(N, TOKENS + 2, WIDTH)[:, :TOKENS], 0),
    "fewer features": lambda: (make(N, TOKENS, WIDTH + 8)[..., :WIDTH - 1], WIDTH + 8),
    "nothing": lambda: (make(0, TOKENS, WIDTH), 0),
    "another type": lambda: (make(N, TOKENS, WIDTH, dtype=torch.float32), 0),
}


@pytest.mark.parametrize("case", BAD)
def test_rows_elsewhere_are_refused(library, case):
    t, row_stride = BAD[case]()
    for call, _ in calls_with(t, row_stride):
        with pytest.raises(dp.DpError) as raised:
            call()
        assert raised.value.status == B.DP_ERR_INVALID_ARG
    assert not library.calls


def test_a_single_row_has_no_spacing(library):
    for t in (make(1, 1, WIDTH), make(WIDTH), make(1, 1, WIDTH + 7)[..., :WIDTH], make(4, 1, WIDTH)[2:3]):
        for row_stride in (0, WIDTH + 7, 1 << 30):
            for call, place in calls_with(t, row_stride, n=1, tokens=1):
                call()
                assert library.calls[-1][1][place] == t.data_ptr()


def test_rows_of_one_value(library):
    for t, row_stride in ((make(N, TOKENS, 1), 0), (make(N, TOKENS, 6)[..., 2:3], 6), (make(N, TOKENS, 6), 6), (make(N, TOKENS), 0)):
        for call, place in calls_with(t, row_stride, features=1):
            call()
            assert library.calls[-1][1][place] == t.data_ptr()


def gradient_calls(t, g_stride, n=N):
    def call(g_w, g_b):
        dp.dp_layer_norm_backward(norm(n=n), P, None, P, P, g_w, g_b, P, P, g_stride=g_stride, ws_bytes=1 << 20, stream=0)
    return [(lambda: call(t, P), 6), (lambda: call(P, t), 7)]


def grads(*shape):
    return make(*shape, dtype=torch.float32)


GOOD_GRADIENTS = {
    "packed": lambda: (grads(N, WIDTH), 0),
    "packed, said so": lambda: (grads(N, WIDTH), WIDTH),
    "with room behind each": lambda: (grads(N, WIDTH + 8), WIDTH + 8),
    "left columns": lambda: (grads(N, 2 * WIDTH)[:, :WIDTH], 2 * WIDTH),
    "right columns": lambda: (grads(N, 2 * WIDTH)[:, WIDTH:], 2 * WIDTH),
    "of more examples": lambda: (grads(N + 1, WIDTH), 0),
    "memory": lambda: (grads(N * WIDTH), 0),
    "memory with gaps": lambda: (grads((N - 1) * 64 + WIDTH), 64),
    "one of two for each example": lambda: (grads(N, 2, WIDTH)[:, 1], 2 * WIDTH),
    "scale and shift of each example": lambda: (grads(N, 2, WIDTH), 2 * WIDTH),
}


@pytest.mark.parametrize("case", GOOD_GRADIENTS)
def test_gradients_where_g_stride_says(library, case):
    t, g_stride = GOOD_GRADIENTS[case]()
    for call, place in gradient_calls(t, g_stride):
        call()
        assert library.calls[-1][1][place] == t.data_ptr()


BAD_GRADIENTS = {
    "packed, said to have room behind each": lambda: (grads(N, WIDTH), WIDTH + 8),
    "right columns, said to be left ones": lambda: (grads(N, WIDTH + 8)[:, 12:], WIDTH + 8),
    "with room behind each, said to be packed": lambda: (grads(N, WIDTH + 8), 0),
    "memory that ends in the last row": lambda: (grads((N - 1) * 64 + WIDTH - 1), 64),
    "one example for all": lambda: (grads(1, WIDTH).expand(N, WIDTH), 0),
    "features first": lambda: (grads(WIDTH, N).t(), 0),
    "fewer examples": lambda: (grads(N - 1, 2 * WIDTH), 2 * WIDTH),
    "one value": lambda: (grads(), 0),
    "another type": lambda: (make(N, WIDTH), 0),
}


@pytest.mark.parametrize("case", BAD_GRADIENTS)
def test_gradients_elsewhere_are_refused(library, case):
    t, g_stride = BAD_GRADIENTS[case]()
    for call, _ in gradient_calls(t, g_stride):
        with pytest.raises(dp.DpError) as raised:
            call()
        assert raised.value.status == B.DP_ERR_INVALID_ARG
    assert not library.calls


def test_a_single_example_has_no_spacing(library):
    for t in (grads(1, WIDTH), grads(WIDTH), grads(2, WIDTH)[1:]):
        for g_stride in (0, WIDTH, WIDTH + 64):
            for call, place in gradient_calls(t, g_stride, n=1):
                call()
                assert library.calls[-1][1][place] == t.data_ptr()
