"""The operators of token models -- 8-bit activation checkpoints with the per-example dense gradients that read them, and the softmax
of attention scores under a learned relative position bias with its gradient -- as cases that can be timed and compared.

Kinds of case ("op"):

  "write"     a layer's input activations into a checkpoint: e4m3 codes and one power-of-two scale for 32 features of a token
  "read"      the activations of a checkpoint as tensors again
  "grad"      per-example gradients of a dense layer from a checkpoint and dY: squared norms, and the gradients where "stored"
  "clip"      the clipped sum of those gradients, recomputed from the checkpoint, into a fresh accumulator (a step's first micro-step)
  "softmax"   probabilities of scores that a bucketed relative position bias is added to
  "backward"  gradient of the scores, and per example the gradient of the bias table with its squared norm

`own` False: the plain form, elementary torch operations.  `own` True: the calls of this repository's library.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
BLOCK = 32                       # features that share a scale
E4M3_MAX = 448.0
LOW_EXP, HIGH_EXP = -100, 119    # exponents that a scale may have
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CLIP = 1.0


# ---- cases ----------------------------------------------------------------------------------------------------------

def _checkpoint(op, rows, features, dtype, stride=0):
    """rows x features activations; stride: elements from one row of them to the next (0: features)."""
    return dict(op=op, rows=rows, features=features, dtype=dtype, stride=stride)


def _dense(op, n, tokens, cin, cout, dtype="bf16", bias=False, ragged=False, stored=False):
    """n examples of `tokens` tokens, cin -> cout; dtype: of dY; ragged: examples have lengths of their own, down to none."""
    return dict(op=op, n=n, tokens=tokens, cin=cin, cout=cout, dtype=dtype, bias=bias, ragged=ragged, stored=stored)


def _bias(op, n, heads, queries, keys, dtype="bf16", bidirectional=True, causal=False, at_end=False, ragged=False, buckets=32,
          max_distance=128):
    """Scores [n, heads, queries, keys]; at_end: the queries are the last of each example's keys (decoding from a cache)."""
    return dict(op=op, n=n, heads=heads, queries=queries, keys=keys, dtype=dtype, bidirectional=bidirectional, causal=causal,
                at_end=at_end, ragged=ragged, buckets=buckets, max_distance=max_distance)


def listed():
    return [
        # a few tokens of a micro-step with one short example: latency
        dict(name="write_few_tokens", **_checkpoint("write", 8, 768, "bf16")),
        # the inputs of a wide projection for a whole micro-step
        dict(name="write_micro_step", **_checkpoint("write", 32768, 2048, "bf16")),
        # activations of an odd width that lie in a wider tensor, read back as the fp32 they came from
        dict(name="read_odd_strided", **_checkpoint("read", 6000, 1003, "f32", stride=1017)),
        # norms of short examples in a batch: a classifier over sentences, lengths of their own
        dict(name="norms_short_ragged", **_dense("grad", 32, 64, 768, 768, bias=True, ragged=True)),
        # norms of long documents
        dict(name="norms_long", **_dense("grad", 8, 1024, 1024, 2048)),
        # a small layer whose gradients are kept for the clipped sum, fp32 gradients
        dict(name="stored_f32_odd", **_dense("grad", 12, 100, 250, 511, "f32", bias=True, stored=True)),
        # the clipped sum of the dense layer that the layer cases time
        dict(name="clip_tokens", **_dense("clip", 16, 128, 768, 768, bias=True)),
        # and of a wide projection over long examples
        dict(name="clip_long_ragged", **_dense("clip", 16, 512, 2048, 2048, ragged=True)),
        # decoding: one query for each example against caches of different lengths
        dict(name="softmax_decode", **_bias("softmax", 32, 12, 1, 4096, bidirectional=False, causal=True, at_end=True, ragged=True)),
        # an encoder's layer
        dict(name="softmax_encoder", **_bias("softmax", 16, 12, 512, 512)),
        # its backward pass
        dict(name="backward_encoder", **_bias("backward", 16, 12, 512, 512)),
        # a causal layer over long ragged examples, fp32
        dict(name="backward_causal_f32", **_bias("backward", 4, 8, 1500, 1500, "f32", bidirectional=False, causal=True, ragged=True)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6e12, w["flops"] / 1.2e15)


def draw(rng):
    while True:
        op = rng.choice(("write", "read", "grad", "grad", "clip", "clip", "softmax", "softmax", "backward", "backward"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if op in ("write", "read"):
            features = rng.choice((_log_int(rng, 16, 4096), 32 * _log_int(rng, 1, 128)))
            case = _checkpoint(op, _log_int(rng, 1, 32768), features, dtype, rng.choice((0, 0, features + _log_int(rng, 1, 64))))
        elif op in ("grad", "clip"):
            unit = rng.choice((1, 8, 64))
            cin, cout = (unit * _log_int(rng, max(1, 32 // unit), 2048 // unit) for _ in range(2))
            n, tokens = _log_int(rng, 1, 64), _log_int(rng, 1, 1024)
            stored = op == "grad" and n * cin * cout <= 1 << 25 and rng.random() < 0.5
            case = _dense(op, n, tokens, cin, cout, dtype, rng.random() < 0.5, rng.random() < 0.5, stored)
        else:
            decode = op == "softmax" and rng.random() < 0.4
            keys = _log_int(rng, 1, 8192)
            queries = 1 if decode else _log_int(rng, 1, 2048)
            causal = decode or rng.random() < 0.4
            buckets, max_distance = rng.choice(((32, 128), (32, 128), (16, 64), (64, 512)))
            case = _bias(op, _log_int(rng, 1, 32), _log_int(rng, 1, 16), queries, keys, dtype, rng.random() < 0.6, causal,
                         decode or rng.random() < 0.3, rng.random() < 0.5, buckets, max_distance)
        if _cost(case) <= max(_cost(c) for c in listed() if c["op"] == op):
            return case


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _pitch(features):
    return (features + BLOCK - 1) // BLOCK * BLOCK


def _activations(gen, rows, features):
    """What layers see: normal values, a few features that are far larger in every token."""
    x = torch.randn((rows, features), generator=gen, device=DEVICE)
    loud = torch.rand((features,), generator=gen, device=DEVICE) < 0.01
    return x.mul_(torch.where(loud, 20.0, 1.0))


def _lengths(gen, n, most, ragged):
    """int32 lengths of 0 .. most (one example of full length, and from four on one of none), or None."""
    if not ragged:
        return None
    v = torch.randint(1, most + 1, (n,), generator=gen, device=DEVICE, dtype=torch.int32)
    v[n // 2] = most
    if n >= 4:
        v[n // 4] = 0
    return v


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dtype, state = DTYPES[case["dtype"]], dict(case=case)
    if case["op"] in ("write", "read"):
        rows, features = case["rows"], case["features"]
        wide = torch.zeros((rows, case["stride"] or features), dtype=dtype, device=DEVICE)
        x = wide[:, :features]
        x.copy_(_activations(gen, rows, features))
        if case["op"] == "write":
            state["x"] = x
        else:
            state["codes"], state["scales"] = _encode(x)
            state["out"] = torch.zeros_like(wide)[:, :features]
        return state
    if case["op"] in ("grad", "clip"):
        n, tokens, cin, cout = (case[k] for k in ("n", "tokens", "cin", "cout"))
        state["codes"], state["scales"] = _encode(_activations(gen, n * tokens, cin))
        state["dy"] = torch.randn((n, tokens, cout), generator=gen, device=DEVICE).mul_(0.01).to(dtype)
        state["lengths"] = _lengths(gen, n, tokens, case["ragged"])
        if case["op"] == "clip":     # squared norms of the examples' whole gradients: most of them clipped
            state["sqnorm"] = torch.rand((n,), generator=gen, device=DEVICE).mul_(16.0).add_(0.25)
        return state
    n, heads, queries, keys = (case[k] for k in ("n", "heads", "queries", "keys"))
    state["key_lengths"] = _lengths(gen, n, keys, case["ragged"])
    state["query_lengths"] = None
    if case["ragged"] and not case["at_end"]:
        state["query_lengths"] = torch.clamp(state["key_lengths"], max=queries) if queries == keys else _lengths(gen, n, queries, True)
    state["scale"] = 0.125
    state["table"] = torch.randn((case["buckets"], heads), generator=gen, device=DEVICE).mul_(0.5)
    state["borders"] = torch.tensor(_borders(case), dtype=torch.int64, device=DEVICE)
    s = torch.randn((n, heads, queries, keys), generator=gen, device=DEVICE).mul_(8.0).to(dtype)
    if case["op"] == "softmax":
        state["scores"] = s
    else:
        state["probs"] = _softmax(case, s, state)
        state["dprobs"] = torch.randn((n, heads, queries, keys), generator=gen, device=DEVICE).mul_(0.01).to(dtype)
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _power(e):
    """2^e in fp32, e whole numbers of the normal range."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _encode(x):
    rows, features = x.shape
    v = torch.zeros((rows, _pitch(features)), dtype=torch.float32, device=x.device)
    v[:, :features] = x
    v = v.view(rows, -1, BLOCK)
    finite = torch.isfinite(v)
    top = torch.where(finite, v, 0.0).abs().amax(2)
    # smallest e with top <= 448 * 2^e = 1.75 * 2^(e + 8)
    bits = top.view(torch.int32)
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7FFFFF) > 0x600000).int()
    e = e.clamp(LOW_EXP, HIGH_EXP)
    scaled = (v * _power(-e)[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX)
    codes = torch.where(finite, scaled, float("nan")).to(torch.float8_e4m3fn).view(torch.uint8).view(rows, -1)
    return codes, (e + 127).to(torch.uint8)


def _decode(codes, scales, features):
    rows = codes.shape[0]
    v = codes.view(torch.float8_e4m3fn).float().view(rows, -1, BLOCK) * _power(scales.int() - 127)[:, :, None]
    return v.view(rows, -1)[:, :features]


def _kept_tokens(dy, lengths):
    """dY in 32 bits, zero where an example has no token."""
    d = dy.float()
    if lengths is None:
        return d
    there = torch.arange(d.shape[1], device=d.device)[None, :] < lengths[:, None]
    return torch.where(there[:, :, None], d, 0.0)


def _plain_grad(state):
    case = state["case"]
    n, tokens = case["n"], case["tokens"]
    x = _decode(state["codes"], state["scales"], case["cin"]).reshape(n, tokens, -1)
    dy = _kept_tokens(state["dy"], state["lengths"])
    g_w = torch.bmm(dy.transpose(1, 2), x)
    sq = g_w.double().square().sum((1, 2))
    out = {}
    g_b = None
    if case["bias"]:
        g_b = dy.sum(1)
        sq = sq + g_b.double().square().sum(1)
    out["sqnorm"] = sq.float()
    if case["stored"]:
        out["g_w"] = g_w
        if case["bias"]:
            out["g_b"] = g_b
    return out


def _plain_clip(state):
    case = state["case"]
    f = torch.clamp(CLIP / state["sqnorm"].sqrt(), max=1.0)
    x = _decode(state["codes"], state["scales"], case["cin"])
    dy = (_kept_tokens(state["dy"], state["lengths"]) * f[:, None, None]).reshape(x.shape[0], -1)
    out = {"acc_w": dy.t() @ x}
    if case["bias"]:
        out["acc_b"] = dy.sum(0)
    return out


def _borders(case):
    """Distances at which the buckets after the first e of a direction's nb begin: the smallest d with
    (nb - e) log(d / e) >= k log(max_distance / e), in whole numbers; k = 1 .. nb - e - 1."""
    nb = case["buckets"] // 2 if case["bidirectional"] else case["buckets"]
    e, far = nb // 2, case["max_distance"]
    span = nb - e
    reached = [max(k for k in range(span) if d ** span * e ** k >= far ** k * e ** span) for d in range(e, far + 1)]
    return [e + next(i for i, r in enumerate(reached) if r >= k) for k in range(1, span)]


def _buckets(case, distance, borders):
    """Buckets of whole-number distances query position - key position."""
    nb = case["buckets"] // 2 if case["bidirectional"] else case["buckets"]
    side = torch.where(distance < 0, nb, 0) if case["bidirectional"] else torch.zeros_like(distance)
    d = distance.abs() if case["bidirectional"] else distance.clamp(min=0)
    return side + torch.where(d < nb // 2, d, nb // 2 + torch.bucketize(d, borders, right=True))


def _positions(case, state):
    """(position of query 0, lengths of the queries, lengths of the keys) of every example, int64 [n]."""
    n = case["n"]
    full = lambda v: torch.full((n,), v, dtype=torch.int64, device=DEVICE)  # noqa: E731
    kl = full(case["keys"]) if state["key_lengths"] is None else state["key_lengths"].long()
    ql = full(case["queries"]) if state["query_lengths"] is None else state["query_lengths"].long()
    return (kl - ql if case["at_end"] else full(0)), ql, kl


def _distances_and_mask(case, state):
    """[n or 1, queries, keys]: distances, and which places count ([n, ...])."""
    first, ql, kl = _positions(case, state)
    q = torch.arange(case["queries"], device=DEVICE)
    k = torch.arange(case["keys"], device=DEVICE)
    if not case["at_end"]:
        first = first[:1]
    distance = first[:, None, None] + q[None, :, None] - k[None, None, :]
    there = (q[None, :, None] < ql[:, None, None]) & (k[None, None, :] < kl[:, None, None])
    if case["causal"]:
        there = there & (distance >= 0)
    return distance, there


def _softmax(case, scores, state):
    distance, there = _distances_and_mask(case, state)
    bias = state["table"][_buckets(case, distance, state["borders"])].permute(0, 3, 1, 2)
    z = torch.where(there[:, None], scores.float() * state["scale"] + bias, -math.inf)
    top = z.amax(3, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(3, keepdim=True)
    return (e / torch.where(total == 0, 1.0, total)).to(scores.dtype)


def _plain_backward(state):
    case = state["case"]
    n, heads, queries, keys = (case[k] for k in ("n", "heads", "queries", "keys"))
    _, there = _distances_and_mask(case, state)
    p = state["probs"].float()
    dp = torch.where(there[:, None], state["dprobs"].float(), 0.0)
    dz = p * (dp - (p * dp).sum(3, keepdim=True))
    # sums along the diagonals first: rows of queries + keys places, taken one place shorter, put equal distances under each other
    wide = torch.zeros((n, heads, queries, queries + keys), dtype=torch.float32, device=DEVICE)
    wide[..., :keys] = dz.flip(2)
    skewed = wide.view(n, heads, -1)[..., :queries * (queries + keys - 1)].view(n, heads, queries, -1)
    lines = skewed.sum(2)                                         # place j: key - query = j - (queries - 1)
    first, _, _ = _positions(case, state)
    distance = first[:, None] + (queries - 1) - torch.arange(queries + keys - 1, device=DEVICE)[None, :]
    which = torch.arange(case["buckets"], device=DEVICE)
    member = (_buckets(case, distance, state["borders"])[:, :, None] == which).float()
    g = torch.bmm(member.transpose(1, 2), lines.transpose(1, 2).contiguous())
    return {"dscores": (dz * state["scale"]).to(state["probs"].dtype), "g_table": g,
            "sqnorm": g.double().square().sum((1, 2)).float()}


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "write":
        codes, scales = _encode(state["x"])
        return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales}
    if op == "read":
        out = state["out"]
        out.copy_(_decode(state["codes"], state["scales"], state["case"]["features"]))
        return out
    if op == "grad":
        return _plain_grad(state)
    if op == "clip":
        return _plain_clip(state)
    if op == "softmax":
        return _softmax(state["case"], state["scores"], state)
    return _plain_backward(state)


def _plan(state):
    """What a program keeps from call to call: the descriptor, output buffers and the workspace."""
    import paper_2109_12191_amd as dp
    case, plan = state["case"], {}
    dtype = dp.DP_BF16 if case["dtype"] == "bf16" else dp.DP_F32
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=DEVICE)  # noqa: E731
    if case["op"] == "write":
        pitch = dp.dp_checkpoint_pitch(case["features"])
        plan["codes"] = empty(case["rows"], pitch, dtype=torch.uint8)
        plan["scales"] = empty(case["rows"], pitch // BLOCK, dtype=torch.uint8)
    elif case["op"] in ("grad", "clip"):
        use = dp.DP_WS_RECOMPUTE if case["op"] == "clip" else dp.DP_WS_PER_EXAMPLE_GRAD
        plan["desc"] = dp.LayerDesc(kind=dp.DP_DENSE, in_dtype=dtype, n=case["n"], cin=case["cin"], cout=case["cout"], h=case["tokens"],
                                    w=1, has_bias=case["bias"])
        plan["ws"] = empty(max(16, dp.dp_checkpoint_workspace_bytes(plan["desc"], use)), dtype=torch.uint8)
        rows = case["n"] if case["op"] == "grad" else 1
        kept = case["op"] == "clip" or case["stored"]
        plan["w"] = empty(rows, case["cout"], case["cin"]) if kept else None
        plan["b"] = empty(rows, case["cout"]) if kept and case["bias"] else None
        plan["sqnorm"] = empty(case["n"])
    elif case["op"] in ("softmax", "backward"):
        plan["desc"] = dp.BiasDesc(in_dtype=dtype, n=case["n"], heads=case["heads"], queries=case["queries"], keys=case["keys"],
                                   buckets=case["buckets"], max_distance=case["max_distance"], bidirectional=case["bidirectional"],
                                   causal=case["causal"], query_offset=dp.DP_QUERIES_AT_END if case["at_end"] else 0,
                                   scale=state["scale"])
        plan["out"] = torch.empty_like(state["scores"] if case["op"] == "softmax" else state["probs"])
        if case["op"] == "backward":
            plan["ws"] = empty(max(16, dp.dp_bias_workspace_bytes(plan["desc"])), dtype=torch.uint8)
            plan["g"] = empty(case["n"], case["buckets"], case["heads"])
            plan["sqnorm"] = empty(case["n"])
    return plan


def _run_own(state):
    import paper_2109_12191_amd as dp
    if "plan" not in state:
        state["plan"] = _plan(state)
    case, plan = state["case"], state["plan"]
    op = case["op"]
    if op == "write":
        dp.dp_checkpoint_write(state["x"], plan["codes"], plan["scales"])
        return {"codes": plan["codes"].view(torch.float8_e4m3fn), "scales": plan["scales"]}
    if op == "read":
        dp.dp_checkpoint_read(state["codes"], state["scales"], state["out"])
        return state["out"]
    if op == "grad":
        dp.dp_checkpoint_example_grad(plan["desc"], state["codes"], state["scales"], state["dy"], plan["w"], plan["b"],
                                      plan["sqnorm"], plan["ws"], lengths=state["lengths"])
        out = {"sqnorm": plan["sqnorm"]}
        if case["stored"]:
            out["g_w"] = plan["w"]
            if case["bias"]:
                out["g_b"] = plan["b"]
        return out
    if op == "clip":
        plan["w"].zero_()
        if case["bias"]:
            plan["b"].zero_()
        dp.dp_checkpoint_clip_accumulate(plan["desc"], state["codes"], state["scales"], state["dy"], state["sqnorm"], CLIP, plan["w"],
                                         plan["b"], plan["ws"], lengths=state["lengths"])
        out = {"acc_w": plan["w"][0]}
        if case["bias"]:
            out["acc_b"] = plan["b"][0]
        return out
    if op == "softmax":
        dp.dp_bias_softmax(plan["desc"], state["scores"], state["table"], plan["out"], query_lengths=state["query_lengths"],
                           key_lengths=state["key_lengths"])
        return plan["out"]
    dp.dp_bias_softmax_backward(plan["desc"], state["probs"], state["dprobs"], plan["out"], plan["g"], plan["sqnorm"], plan["ws"],
                                query_lengths=state["query_lengths"], key_lengths=state["key_lengths"])
    return {"dscores": plan["out"], "g_table": plan["g"], "sqnorm": plan["sqnorm"]}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    """Bytes read and written once, and multiply-adds as two operations; lengths counted as full."""
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] in ("write", "read"):
        rows, pitch = case["rows"], _pitch(case["features"])
        return {"bytes": rows * (case["features"] * size + pitch + pitch // BLOCK), "flops": 0}
    if case["op"] in ("grad", "clip"):
        n, t, cin, cout = (case[k] for k in ("n", "tokens", "cin", "cout"))
        pitch = _pitch(cin)
        nbytes = n * t * (pitch + pitch // BLOCK + cout * size) + 4 * n
        direct, gram = 2 * t * cin * cout, t * (t + 1) * (cin + cout)
        if case["op"] == "clip":
            return {"bytes": nbytes + 4 * cout * (cin + case["bias"]), "flops": n * direct}
        if case["stored"]:
            return {"bytes": nbytes + 4 * n * cout * (cin + case["bias"]), "flops": n * direct}
        return {"bytes": nbytes, "flops": n * min(direct, gram)}
    places = case["n"] * case["heads"] * case["queries"] * case["keys"]
    if case["op"] == "softmax":
        return {"bytes": 2 * size * places + 4 * case["buckets"] * case["heads"], "flops": 8 * places}
    return {"bytes": 3 * size * places + 4 * case["n"] * (case["buckets"] * case["heads"] + 1), "flops": 6 * places}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _two_to(e):
    """2^e in 64 bits, to the last bit."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(state, features):
    """Values of a checkpoint, in 64 bits."""
    codes, scales = state["codes"], state["scales"]
    s = _two_to(scales.long() - 127).repeat_interleave(BLOCK, dim=1)
    return (codes.view(torch.float8_e4m3fn).double() * s)[:, :features]


def _exact_encode(x):
    rows, features = x.shape
    pad = torch.zeros((rows, _pitch(features) - features), dtype=torch.float64, device=DEVICE)
    v = torch.cat((x.double(), pad), 1).view(rows, -1, BLOCK)
    top = v.abs().amax(2)
    _, e = torch.frexp(top / E4M3_MAX)                     # top / 448 = m 2^e, 0.5 <= m < 1: at most 2^e, and 2^(e-1) if m is 0.5
    e = torch.where(top == E4M3_MAX * _two_to(e - 1), e - 1, e)
    e = torch.where(top == 0, LOW_EXP, e).clamp(LOW_EXP, HIGH_EXP)
    y = v / _two_to(e)[:, :, None]
    # nearest of the values with four significant bits, none finer than 2^-9
    _, m = torch.frexp(y)
    step = _two_to((m - 4).clamp(min=-9))
    y = (torch.round(y / step) * step).clamp(-E4M3_MAX, E4M3_MAX)
    return {"codes": y.view(rows, -1), "scales": (e + 127).to(torch.uint8)}


def _exact_bucket(case, d):
    """Bucket of one distance, from the definition."""
    nb, side = case["buckets"], 0
    if case["bidirectional"]:
        nb //= 2
        side, d = (nb, -d) if d < 0 else (0, d)
    d, e, span = max(d, 0), nb // 2, nb - nb // 2
    if d < e:
        return side + d
    if d >= case["max_distance"]:
        return side + nb - 1
    k = math.floor(span * math.log(d / e) / math.log(case["max_distance"] / e) + 0.5)
    if d ** span * e ** k < case["max_distance"] ** k * e ** span:      # the border itself, in whole numbers
        k -= 1
    return side + min(nb - 1, e + k)


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "write":
        return _exact_encode(state["x"])
    if case["op"] == "read":
        return _exact_values(state, case["features"])
    if case["op"] in ("grad", "clip"):
        n, tokens = case["n"], case["tokens"]
        x = _exact_values(state, case["cin"]).reshape(n, tokens, -1)
        dy, out = state["dy"].double(), {}
        if state["lengths"] is not None:
            late = torch.arange(tokens, device=DEVICE)[None, :] >= state["lengths"][:, None]
            dy.masked_fill_(late[:, :, None], 0.0)
        if case["op"] == "clip":
            f = torch.clamp(CLIP / state["sqnorm"].double().sqrt(), max=1.0)
            acc = torch.zeros((case["cout"], case["cin"]), dtype=torch.float64, device=DEVICE)
            for i in range(n):
                acc += f[i] * (dy[i].t() @ x[i])
            out["acc_w"] = acc
            if case["bias"]:
                out["acc_b"] = (dy.sum(1) * f[:, None]).sum(0)
            return out
        each = [dy[i].t() @ x[i] for i in range(n)]
        sq = torch.stack([g.square().sum() for g in each])
        if case["bias"]:
            sq = sq + dy.sum(1).square().sum(1)
        out["sqnorm"] = sq
        if case["stored"]:
            out["g_w"] = torch.stack(each)
            if case["bias"]:
                out["g_b"] = dy.sum(1)
        return out
    n, queries, keys = case["n"], case["queries"], case["keys"]
    ql = torch.full((n,), queries) if state["query_lengths"] is None else state["query_lengths"].cpu()
    kl = torch.full((n,), keys) if state["key_lengths"] is None else state["key_lengths"].cpu()
    of = torch.tensor([_exact_bucket(case, d) for d in range(-queries - keys, queries + keys + 1)], device=DEVICE)
    q, k = torch.arange(queries, device=DEVICE)[:, None], torch.arange(keys, device=DEVICE)[None, :]
    shape = (n, case["heads"], queries, keys)
    res = torch.zeros(shape, dtype=torch.float64, device=DEVICE)
    g = torch.zeros((n, case["buckets"], case["heads"]), dtype=torch.float64, device=DEVICE)
    for i in range(n):
        first = int(kl[i]) - int(ql[i]) if case["at_end"] else 0
        distance = first + q - k
        there = (q < int(ql[i])) & (k < int(kl[i]))
        if case["causal"]:
            there = there & (distance >= 0)
        bucket = of[distance + queries + keys]
        if case["op"] == "softmax":
            z = state["scores"][i].double() * state["scale"] + state["table"].double()[bucket].permute(2, 0, 1)
            z = z.masked_fill(~there, -math.inf)
            res[i] = torch.nan_to_num(torch.softmax(z, 2), nan=0.0)
        else:
            p, d = state["probs"][i].double(), state["dprobs"][i].double().masked_fill(~there, 0.0)
            dz = p * (d - (p * d).sum(2, keepdim=True))
            res[i] = dz * state["scale"]
            lines = torch.stack([dz.masked_fill(bucket != b, 0.0).sum((1, 2)) for b in range(case["buckets"])])
            g[i] = lines
    if case["op"] == "softmax":
        return res
    return {"dscores": res, "g_table": g, "sqnorm": g.square().sum((1, 2))}
