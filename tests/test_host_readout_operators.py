"""CPU-only checks of the calls on either side of a token model's blocks (layer norm, log probabilities of tokens): what they refuse, before anything
could be launched, and their pure-host queries."""
import math
import os
import subprocess

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


def _norm(**k):
    d = dict(in_dtype=dp.DP_BF16, n=3, tokens=5, features=40, rms=0, eps=1e-5, row_stride=0)
    d.update(k)
    return dp.NormDesc(**d)


BAD_NORMS = [dict(in_dtype=5), dict(n=0), dict(tokens=0), dict(tokens=-1), dict(features=0), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan),
             dict(eps=math.inf), dict(eps=1e-31), dict(row_stride=39)]
WIDE_NORMS = [dict(features=(1 << 20) + 1), dict(n=1 << 16, tokens=1 << 15), dict(row_stride=1 << 40)]


def test_layer_norm_refuses(lib):
    def call(desc=_norm(), x=FAKE, gamma=FAKE, beta=FAKE, y=FAKE, lengths=None):
        dp.dp_layer_norm(desc, x, gamma, beta, y, lengths=lengths, stream=0)
    for bad in (dict(x=None), dict(y=None), dict(x=FAKE + 1), dict(y=FAKE + 1), dict(gamma=FAKE + 2), dict(beta=FAKE + 1), dict(lengths=FAKE + 2),
                dict(desc=_norm(in_dtype=dp.DP_F32), x=FAKE + 2), *(dict(desc=_norm(**b)) for b in BAD_NORMS)):
        assert _raises(INT, call, **bad)
    for bad in WIDE_NORMS:
        _raises(B.DP_ERR_UNSUPPORTED, call, desc=_norm(**bad))


def test_layer_norm_backward_refuses(lib):
    ws = dp.dp_layer_norm_workspace_bytes(_norm())
    assert ws >= 3 * 2 * 40 * 4

    def call(desc=_norm(), x=FAKE, gamma=FAKE, dy=FAKE, dx=FAKE, gw=FAKE, gb=FAKE, sq=FAKE, w=FAKE, wb=ws, lengths=None, gs=0):
        dp.dp_layer_norm_backward(desc, x, gamma, dy, dx, gw, gb, sq, w, lengths=lengths, g_stride=gs, ws_bytes=wb, stream=0)
    for bad in (dict(x=None), dict(dy=None), dict(x=FAKE + 1), dict(dy=FAKE + 1), dict(dx=FAKE + 1), dict(gamma=FAKE + 2), dict(lengths=FAKE + 1), dict(gw=FAKE + 4),
                dict(gb=FAKE + 8), dict(sq=FAKE + 2), dict(dx=None, gw=None, gb=None, sq=None), dict(gw=None), dict(gw=None, gb=None), dict(gw=None, sq=None),
                dict(gs=42), dict(gs=36), dict(w=FAKE + 8), *(dict(desc=_norm(**b)) for b in BAD_NORMS)):
        assert _raises(INT, call, **bad)
    for bad in (dict(wb=ws - 1), dict(w=None)):
        _raises(B.DP_ERR_WORKSPACE, call, **bad)
    for bad in WIDE_NORMS:
        _raises(B.DP_ERR_UNSUPPORTED, call, desc=_norm(**bad))
        assert dp.dp_layer_norm_workspace_bytes(_norm(**bad)) == 0


def _logprob(**k):
    d = dict(in_dtype=dp.DP_BF16, n=3, tokens=5, vocab=100, top=0, scale=1.0, row_stride=0)
    d.update(k)
    return dp.LogprobDesc(**d)


BAD_LOGPROBS = [dict(in_dtype=5), dict(n=0), dict(tokens=0), dict(vocab=0), dict(top=-1), dict(top=33), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                dict(scale=math.inf), dict(row_stride=99)]
WIDE_LOGPROBS = [dict(vocab=(1 << 24) + 1), dict(n=1 << 16, tokens=1 << 15), dict(row_stride=1 << 40)]


def test_token_logprobs_refuses(lib):
    few = _logprob(tokens=1, vocab=50000, top=4)             # rows that several workgroups share
    ws = dp.dp_token_logprobs_workspace_bytes(few)
    assert ws > 0

    def call(desc=few, logits=FAKE, targets=FAKE, logprobs=FAKE, entropy=FAKE, stats=FAKE, top=FAKE, tokens=FAKE, w=FAKE, wb=ws, lengths=None):
        dp.dp_token_logprobs(desc, logits, targets, logprobs, entropy, stats, top, tokens, w, lengths=lengths, ws_bytes=wb, stream=0)
    for bad in (dict(logits=None), dict(logits=FAKE + 1), dict(targets=None), dict(targets=FAKE + 2), dict(logprobs=FAKE + 1), dict(entropy=FAKE + 2),
                dict(stats=FAKE + 4), dict(top=FAKE + 2), dict(tokens=None), dict(tokens=FAKE + 1), dict(lengths=FAKE + 2), dict(w=FAKE + 4),
                dict(desc=_logprob(), top=None), dict(desc=_logprob(), tokens=None), *(dict(desc=_logprob(**b)) for b in BAD_LOGPROBS)):
        assert _raises(INT, call, **bad)
    _raises(INT, call, desc=_logprob(), top=None, tokens=None, logprobs=None, entropy=None, stats=None)
    for bad in (dict(wb=ws - 1), dict(w=None)):
        _raises(B.DP_ERR_WORKSPACE, call, **bad)
    for bad in WIDE_LOGPROBS:
        _raises(B.DP_ERR_UNSUPPORTED, call, desc=_logprob(**bad), top=None, tokens=None)
        assert dp.dp_token_logprobs_workspace_bytes(_logprob(**bad)) == 0


def test_token_logprobs_backward_refuses(lib):
    few = _logprob(tokens=1, vocab=50000)
    ws = dp.dp_token_logprobs_workspace_bytes(few)
    assert ws >= 3 * 12

    def call(desc=few, logits=FAKE, targets=FAKE, stats=FAKE, d=FAKE, out=FAKE, w=FAKE, entropy=FAKE, de=FAKE, lp=FAKE, lengths=None, wb=ws):
        dp.dp_token_logprobs_backward(desc, logits, targets, stats, d, out, w, entropy=entropy, d_entropy=de, logprobs=lp, lengths=lengths, ws_bytes=wb, stream=0)
    for bad in (dict(logits=None), dict(out=None), dict(out=FAKE + 1), dict(logits=FAKE + 1), dict(targets=None), dict(targets=FAKE + 1), dict(stats=FAKE + 4), dict(d=FAKE + 2),
                dict(de=FAKE + 2), dict(entropy=FAKE + 1), dict(lp=FAKE + 1), dict(lengths=FAKE + 3), dict(d=None, de=None), dict(entropy=None), dict(stats=None),
                dict(d=None, lp=FAKE, targets=None), dict(desc=_logprob(top=1)), dict(w=FAKE + 2), *(dict(desc=_logprob(**b)) for b in BAD_LOGPROBS)):
        assert _raises(INT, call, **bad)
    for bad in (dict(wb=ws - 1), dict(w=None)):
        _raises(B.DP_ERR_WORKSPACE, call, **bad)
    for bad in WIDE_LOGPROBS:
        _raises(B.DP_ERR_UNSUPPORTED, call, desc=_logprob(**bad))


def test_lengths_and_targets_have_to_be_int32_on_the_device(lib):
    for bad in (torch.zeros(15, dtype=torch.int64), torch.zeros(15, dtype=torch.float32), torch.zeros(15, dtype=torch.int32), torch.zeros(14, dtype=torch.int32)):
        _raises(INT, dp.dp_layer_norm, _norm(), FAKE, None, None, FAKE, lengths=bad, stream=0)
        _raises(INT, dp.dp_token_logprobs, _logprob(), FAKE, bad, FAKE, None, None, None, None, FAKE, stream=0)
        _raises(INT, dp.dp_token_logprobs_backward, _logprob(), FAKE, bad, None, FAKE, FAKE, FAKE, stream=0)


def test_tensors_have_to_be_what_the_descriptor_says(lib):
    """Of its type, with room enough, on the device: calls take addresses."""
    for bad in (torch.zeros(3, 5, 40), torch.zeros(3, 5, 40, dtype=torch.bfloat16), torch.zeros(3, 5, 40, dtype=torch.int16)):
        for names in ("x", "y"):
            _raises(INT, dp.dp_layer_norm, _norm(), bad if names == "x" else FAKE, None, None, bad if names == "y" else FAKE, stream=0)
        for place in range(3):
            t = [bad if i == place else FAKE for i in range(3)]
            _raises(INT, dp.dp_layer_norm_backward, _norm(), t[0], None, t[1], t[2], FAKE, FAKE, FAKE, FAKE, ws_bytes=1 << 20, stream=0)
        _raises(INT, dp.dp_token_logprobs, _logprob(), bad, FAKE, FAKE, None, None, None, None, FAKE, stream=0)
        _raises(INT, dp.dp_token_logprobs_backward, _logprob(), FAKE, FAKE, None, FAKE, bad, FAKE, stream=0)
    for bad in (torch.zeros(3, 40), torch.zeros(3, 40, dtype=torch.bfloat16), torch.zeros(2, 40)):
        for place in range(2):
            g = [bad if i == place else FAKE for i in range(2)]
            _raises(INT, dp.dp_layer_norm_backward, _norm(), FAKE, None, FAKE, FAKE, *g, FAKE, FAKE, ws_bytes=1 << 20, stream=0)
    for bad in (torch.zeros(15), torch.zeros(15, dtype=torch.bfloat16), torch.zeros(15, dtype=torch.int32)):
        _raises(INT, dp.dp_layer_norm, _norm(), FAKE, bad, None, FAKE, stream=0)
        _raises(INT, dp.dp_token_logprobs, _logprob(), FAKE, FAKE, bad, None, None, None, None, FAKE, stream=0)
        _raises(INT, dp.dp_token_logprobs, _logprob(), FAKE, FAKE, None, bad, None, None, None, FAKE, stream=0)
        _raises(INT, dp.dp_token_logprobs_backward, _logprob(), FAKE, FAKE, None, bad, FAKE, FAKE, stream=0)


def test_workspaces_of_every_size(lib):
    """Queries answer for the whole range, and grow with what they are for."""
    for features in (1, 7, 512, 1000, 8192, 16384, 16385, 1 << 20):
        for tokens in (1, 3, 1000):
            need = dp.dp_layer_norm_workspace_bytes(_norm(n=2, tokens=tokens, features=features))
            assert need >= 2 * 2 * features * 4 and need % 16 == 0
    for vocab in (1, 1000, 8192, 131072, 1 << 24):
        for tokens in (1, 1000):
            plain, top = (dp.dp_token_logprobs_workspace_bytes(_logprob(tokens=tokens, vocab=vocab, top=k)) for k in (0, 32))
            assert plain % 16 == 0 and top % 16 == 0
            assert plain > 0 or tokens == 1000 or vocab < 65536


def test_rows_are_taken_by_words_only_where_every_workgroup_begins_at_one(tmp_path):
    here, exe = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "token_words")
    subprocess.run(["g++", "-std=c++17", "-O1", "-I" + os.path.join(here, "..", "paper_2109_12191_amd", "csrc"), os.path.join(here, "token_words.cpp"), "-o", exe],
                   check=True)
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


def test_partial_results_of_shared_rows_begin_at_whole_16_bytes(lib):
    """They are stored and loaded by 16 bytes, so each row's room is a whole number of them, odd counts of workgroups and alternatives among them."""
    shared = 0
    for rows in (1, 2, 3, 5, 7, 100):
        for vocab in (33281, 36864, 45056, 60000, 131072):
            for top in range(33):
                need = dp.dp_token_logprobs_workspace_bytes(_logprob(n=rows, tokens=1, vocab=vocab, top=top))
                shared += need > 0
                if top:                                      # (without, a gradient's statistics are in there too)
                    assert need % (16 * rows) == 0, (rows, vocab, top, need)
    assert shared > 500
