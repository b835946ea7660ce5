"""Performance cases of what stands around the products of a decoder layer: the residual's addition and the norm with an INT8 output, the
gated activation with one, tokens sorted by expert and back, and attention of chunks of new tokens over the 4-bit cache.

A case is a dict of plain values.  Six kinds:

  norm      x + residual, its root-mean-square norm, INT8 codes with a scale a token; `y`: the norm's own result too, for a router
  swiglu    silu(gate) * up of rows [gate | up], INT8 codes with a scale a row
  dispatch  each token's row copied to a row for each of its experts, sorted by expert; `absent`: only half of the experts are here
  combine   the weighted sum of each token's rows, back in the tokens' order
  grads     its gradients: of the rows and of the weights
  chunks    attention of new tokens, any number of them a sequence, over the paged 4-bit cache that holds them already

INT8 codes are returned as the numbers that they stand for, in the type of what was quantised; rows of INT8 that are only moved as they are.

The plain forms are elementary torch operations in FP32 (FP64: the mean of the squares, and what follows from it alone, so that codes next to
a rounding border are the definition's).  A page of the cache holds, for each kv head, P tokens:
  P * D/2 bytes   key codes, row by row, element 2i in the low half of byte i;
  P * D/2 bytes   value codes: for four tokens at a time 16 column groups of D/16 elements, in each the token pairs (0, 1), (2, 3),
                  in each pair four elements at a time, two bytes for its first token and two for its second;
  4 P, 4 P bytes  a word for each token's keys, and one for its values: an FP32 scale whose low 12 bits are free, with the
                  zero point in the low four.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEVICE = "cuda"
EPS = 1e-6
SMALLEST = 2.0 ** -100  # of the cache's scales
WIDTHS = (2048, 4096, 4104, 5120, 8192, 8200)       # of the tokens' rows
INNER = (1536, 4096, 6912, 11008, 13824, 14336, 28672)  # of the activations between an MLP's products


def listed():
    return [
        # one token of a 7B model: the launch and the host's work are all there is
        _norm("norm_7b_t1", 1, 4096),
        # a prompt on a 70B model, an odd number of tokens; the router of a mixture of experts reads the norm's result too
        _norm("norm_70b_t4093", 4093, 8192, dtype="bfloat16", y=True),
        # a decode step of 16 tokens, two experts each
        _swiglu("swiglu_moe_t32", 32, 14336),
        # a prompt on a 70B model
        _swiglu("swiglu_70b_t2039", 2039, 28672, dtype="bfloat16"),
        # a decode step of 16 tokens goes to eight experts
        _dispatch("dispatch_moe_t16", 16, 2, 8, 4096, dtype="int8"),
        # a long prompt, eight of 64 experts a token, half of them on this GPU
        _dispatch("dispatch_moe_t8191", 8191, 8, 64, 4096, dtype="float16", absent=True),
        # the decode step's rows come back
        _combine("combine_moe_t16", 16, 2, 8, 4096),
        # and the long prompt's
        _combine("combine_moe_t8191", 8191, 8, 64, 4096, dtype="bfloat16", absent=True),
        # a router is trained: gradients of the experts' rows and of the weights
        _grads("grads_moe_t2047", 2047, 4, 16, 8192, dtype="bfloat16"),
        # the last few tokens of a short prompt on a 7B model: latency
        _chunks("chunk_7b_t17", 1, 17, 517, 32, 32),
        # a serving step: sequences that decode, and chunks of prompts between them; small pages
        _chunks("mixed_moe_b24", 24, 640, 4096, 32, 8, page=16, mixed=True),
        # chunks of two long prompts on a 70B model
        _chunks("chunks_70b_t4096", 2, 4096, 16384, 64, 8, dtype="bfloat16"),
    ]


def _norm(name, tokens, width, dtype="float16", residual=True, y=False):
    return _case(name, kind="norm", tokens=tokens, width=width, dtype=dtype, residual=residual, y=y)


def _swiglu(name, tokens, width, dtype="float16"):
    return _case(name, kind="swiglu", tokens=tokens, width=width, dtype=dtype)


def _dispatch(name, tokens, each, experts, width, dtype="float16", absent=False):
    return _case(name, kind="dispatch", tokens=tokens, each=each, experts=experts, width=width, dtype=dtype, absent=absent)


def _combine(name, tokens, each, experts, width, dtype="float16", absent=False):
    return _dispatch(name, tokens, each, experts, width, dtype, absent) | {"kind": "combine"}


def _grads(name, tokens, each, experts, width, dtype="float16", absent=False):
    return _dispatch(name, tokens, each, experts, width, dtype, absent) | {"kind": "grads"}


def _chunks(name, seqs, tokens, context, heads, kv_heads, dim=128, page=64, dtype="float16", mixed=False):
    return _case(name, kind="chunks", seqs=seqs, tokens=tokens, context=context, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                 dtype=dtype, mixed=mixed)


def _case(name, **values):
    return dict(name=name, **values) if name else values


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: any number of tokens, width, experts, head layout, page and type of the ranges above."""
    dtype, pick = rng.choice(("float16", "float16", "bfloat16")), rng.random()
    if pick < 0.2:
        return _norm("", _log_int(rng, 1, 8192), rng.choice(WIDTHS), dtype, rng.random() < 0.8, rng.random() < 0.4)
    if pick < 0.35:
        return _swiglu("", _log_int(rng, 1, 4096), rng.choice(INNER), dtype)
    if pick < 0.7:
        make = rng.choice((_dispatch, _combine, _grads))
        if make is _dispatch and rng.random() < 0.5:
            dtype = "int8"
        experts = rng.choice((4, 8, 16, 60, 64, 128))
        each = rng.choice([n for n in (1, 2, 2, 4, 6, 8) if n <= experts // 2])
        return make("", _log_int(rng, 1, 8192 // max(1, each // 2)), each, experts, rng.choice((2048, 4096, 5120, 8192)), dtype, rng.random() < 0.3)
    heads, kv_heads = rng.choice(((32, 32), (40, 40), (64, 8), (32, 8), (48, 8), (16, 4), (8, 1), (28, 4)))
    dim, page = rng.choice((128, 128, 128, 64)), rng.choice((16, 32, 64, 64, 128, 256))
    while True:
        seqs, mixed = _log_int(rng, 1, 32), rng.random() < 0.4
        c = _chunks("", seqs, _log_int(rng, 2 * seqs, 4096), _log_int(rng, 16, 32768), heads, kv_heads, dim, page, dtype, mixed)
        lens, most = _lengths(c), work(listed()[-1])
        there = seqs * heads * max(a for a, _ in lens) * max(b for _, b in lens)
        if there <= 2 * 64 * 2048 * 16384 and work(c)["flops"] <= most["flops"] and sum(b for _, b in lens) * kv_heads * dim <= 32 * 4096 * 32 * 128:
            return c


# ------------------------------------------------------------------------------ sizes
def _lengths(case):
    """(new tokens, tokens in the cache) of each sequence: lengths go by the case alone, so that work() knows them."""
    rng, n = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name"))), case["seqs"]
    if case["mixed"]:  # one new token each, but for a few that have the rest
        part = [rng.uniform(0.3, 1.0) if i % 8 == 3 or n < 4 else 0.0 for i in range(n)]
    else:
        part = [rng.uniform(0.7, 1.0) for _ in range(n)]
    new = [max(1, int((case["tokens"] - n) * p / (sum(part) or 1.0))) for p in part]
    new[part.index(max(part))] += max(0, case["tokens"] - sum(new))
    got = [(a, max(a, int(case["context"] * rng.uniform(0.2, 1.0)))) for a in new]
    got[0] = (got[0][0], max(got[0][0], case["context"]))
    return got


def work(case):
    t = case["tokens"]
    if case["kind"] == "chunks":
        heads, kv_heads, dim, lens = case["heads"], case["kv_heads"], case["dim"], _lengths(case)
        pairs = heads * sum(a * (b - a) + a * (a + 1) // 2 for a, b in lens)
        return {"bytes": sum(b for _, b in lens) * kv_heads * (dim + 8) + 4 * dim * heads * sum(a for a, _ in lens), "flops": 4 * dim * pairs}
    w = case["width"]
    if case["kind"] == "norm":  # (the numbers that the codes stand for come back, two bytes each)
        return {"bytes": t * w * (2 + 4 * case["residual"] + 2 * case["y"] + 1 + 2) + 4 * w + 4 * t, "flops": 8 * t * w}
    if case["kind"] == "swiglu":
        return {"bytes": t * w * (4 + 1 + 2) + 4 * t, "flops": 8 * t * w}
    pairs, size = t * case["each"], 1 if case["dtype"] == "int8" else 2
    kept = pairs // 2 if case["absent"] else pairs  # (about)
    if case["kind"] == "dispatch":
        return {"bytes": (t + kept) * w * size + 8 * pairs, "flops": pairs}
    if case["kind"] == "combine":
        return {"bytes": (t + kept) * w * 2 + 8 * pairs, "flops": 2 * kept * w}
    return {"bytes": (t + kept + pairs) * w * 2 + 12 * pairs, "flops": 3 * kept * w}


# ----------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _heads(gen, tokens, heads, dim, dtype, outliers=False):
    x = _normal(gen, tokens, heads, dim)
    if outliers:  # keys have channels that are several times as large as the rest, the same ones in every token
        x *= torch.exp(0.5 * _normal(gen, heads, dim)).clamp_(0.3, 4.0)
    return x.to(dtype)


def prepare(case, seed):
    gen, state = _generator(seed), {"case": case}
    dtype, t = getattr(torch, case["dtype"]), case["tokens"]
    if case["kind"] == "chunks":
        return state | _chunks_state(case, gen, dtype)
    w = case["width"]
    if case["kind"] == "norm":  # a stream whose channels differ, and what the layer before adds to it
        channels = torch.exp(0.5 * _normal(gen, w))
        state["x"] = (0.5 * _normal(gen, t, w)).to(dtype)
        state["residual"] = (2.0 * _normal(gen, t, w) * channels).to(dtype) if case["residual"] else None
        state["weight"] = 1.0 + 0.2 * _normal(gen, w)
        return state
    if case["kind"] == "swiglu":
        return state | {"x": (1.5 * _normal(gen, t, 2 * w)).to(dtype)}
    # a router's choice, some experts taken more often than others
    scores = _normal(gen, t, case["experts"]) + 0.7 * _normal(gen, case["experts"])
    best = scores.topk(case["each"], -1)
    state["experts"], state["weights"] = best.indices.to(torch.int32), torch.softmax(best.values, -1).contiguous()
    state["here"] = case["experts"]
    if case["absent"]:  # this GPU has the second and third quarter of the experts
        state["experts"], state["here"] = (state["experts"] - case["experts"] // 4).contiguous(), case["experts"] // 2
    rows = t * case["each"]
    if case["kind"] == "dispatch":
        if dtype is torch.int8:
            state["x"] = torch.randint(-127, 128, (t, w), generator=gen, device=DEVICE, dtype=torch.int32).to(torch.int8)
            state["scales"] = torch.rand(t, generator=gen, device=DEVICE) * 0.05 + 0.01
            state["out_scales"] = torch.zeros(rows, device=DEVICE)
        else:
            state["x"], state["scales"], state["out_scales"] = _normal(gen, t, w).to(dtype), None, None
        state["out"] = torch.zeros((rows, w), dtype=dtype, device=DEVICE)  # (rows that no pair takes stay as they are)
        return state
    state["offsets"], state["places"] = _plain_places(state["experts"], state["here"])
    state["rows"] = _normal(gen, rows, w).to(dtype)
    if case["kind"] == "grads":
        state["grad"] = (1e-2 * _normal(gen, t, w)).to(dtype)
    return state


def _chunks_state(case, gen, dtype):
    page, lens = case["page"], _lengths(case)
    need = [-(-b // page) for _, b in lens]
    order = torch.randperm(sum(need) + 1, generator=gen, device=DEVICE).to(torch.int32)
    table = torch.zeros((len(lens), max(need)), dtype=torch.int32, device=DEVICE)
    cache = torch.zeros((sum(need) + 1, case["kv_heads"], page * (case["dim"] + 8)), dtype=torch.uint8, device=DEVICE)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at: at + n]
        at += n
        for first in range(0, lens[b][1], 16384):
            j = torch.arange(first, min(lens[b][1], first + 16384), device=DEVICE)
            k = _heads(gen, len(j), case["kv_heads"], case["dim"], dtype, True)
            v = _heads(gen, len(j), case["kv_heads"], case["dim"], dtype)
            _plain_write(k, v, table[b][j // page] * page + j % page, cache)
    new = [a for a, _ in lens]
    q = _heads(gen, sum(new), case["heads"], case["dim"], dtype)
    return {"q": q, "cache": cache, "block_table": table, "context": torch.tensor([b for _, b in lens], dtype=torch.int32, device=DEVICE),
            "starts": torch.tensor([0, *new], device=DEVICE).cumsum(0).to(torch.int32), "most": max(new), "most_keys": max(b for _, b in lens)}


# ------------------------------------------------------------------------- the passes
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(s):
    from paper_2509_01229_amd import api

    kind, case = s["case"]["kind"], s["case"]
    if kind == "norm":
        q, scales, h, y = api.w4a8_norm_quantize(s["x"], s["weight"], residual=s["residual"], eps=EPS, want_y=case["y"])
        return {"values": _values(q, scales, s["x"].dtype), "scales": scales, "h": h, "y": y}
    if kind == "swiglu":
        q, scales = api.w4a8_swiglu_quantize(s["x"])
        return {"values": _values(q, scales, s["x"].dtype), "scales": scales}
    if kind == "dispatch":
        return api.moe_dispatch(s["x"], s["experts"], s["here"], act_scales=s["scales"], out=s["out"], out_scales=s["out_scales"])
    if kind == "combine":
        return api.moe_combine(s["rows"], s["places"], s["weights"])
    if kind == "grads":
        return api.moe_combine_backward(s["grad"], s["rows"], s["places"], s["weights"], row_offsets=s["offsets"])
    return api.kv4_attention_chunks(s["q"], s["cache"], s["block_table"], s["context"], s["starts"])


def _run_plain(s):
    kind, case = s["case"]["kind"], s["case"]
    if kind == "norm":
        return _plain_norm(s["x"], s["residual"], s["weight"], case["y"])
    if kind == "swiglu":
        gate, up = s["x"].float().split(case["width"], -1)
        q, scales = _plain_quantise(gate / (1.0 + torch.exp(-gate)) * up)
        return {"values": _values(q, scales, s["x"].dtype), "scales": scales}
    if kind == "dispatch":
        return _plain_dispatch(s)
    if kind == "combine":
        return _plain_combine(s["rows"], s["places"], s["weights"])
    if kind == "grads":
        return _plain_grads(s["grad"], s["rows"], s["places"], s["weights"])
    return _plain_chunks(s, case)


def _values(codes, scales, dtype):
    """The numbers that the codes stand for."""
    return torch.mul(codes, scales[:, None], out=torch.empty(codes.shape, dtype=dtype, device=codes.device))


def _plain_quantise(y):
    """INT8 codes (as FP32 numbers) and scales of the rows."""
    most = y.abs().amax(-1)
    scales = torch.where(most > 0, most / torch.full_like(most, 127.0), 1.0)  # (a number in its place is multiplied by its reciprocal)
    return torch.round(y / scales[:, None]).clamp(-127.0, 127.0), scales


def _plain_norm(x, residual, weight, want_y):
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    r = (1.0 / torch.sqrt(h.double().square().mean(-1, keepdim=True) + EPS)).float()
    y = h.float() * weight * r
    q, scales = _plain_quantise(y)
    return {"values": _values(q, scales, x.dtype), "scales": scales, "h": None if residual is None else h, "y": y.to(x.dtype) if want_y else None}


def _plain_places(experts, here):
    """The rows' first numbers for each expert and behind the last, and each pair's row (-1: its expert is not here)."""
    ids = experts.flatten()
    taken = ids == torch.arange(here, device=DEVICE, dtype=torch.int32)[:, None]
    before = taken.cumsum(-1, dtype=torch.int32)  # pairs of the expert up to this one
    offsets = torch.cat((torch.zeros(1, dtype=torch.int32, device=DEVICE), before[:, -1].cumsum(0, dtype=torch.int32)))
    places = torch.where(taken, offsets[:-1, None] + before - 1, 0).sum(0, dtype=torch.int32)
    return offsets, torch.where(taken.any(0), places, -1).view(experts.shape)


def _plain_dispatch(s):
    offsets, places = _plain_places(s["experts"], s["here"])
    pairs = (places.flatten() >= 0).nonzero().flatten()
    rows = places.flatten()[pairs].long()
    token = pairs // s["case"]["each"]
    s["out"][rows] = s["x"][token]
    if s["scales"] is not None:
        s["out_scales"][rows] = s["scales"][token]
    return s["out"], s["out_scales"], offsets, places


def _plain_combine(rows, places, weights):
    there = places >= 0
    x = rows[places.clamp(min=0).long()].float()
    return (x * torch.where(there, weights, 0.0)[..., None]).sum(1).to(rows.dtype)


def _plain_grads(grad, rows, places, weights):
    there, at = places >= 0, places.clamp(min=0).long()
    g = grad.float()[:, None]
    of_weights = torch.where(there, (rows[at].float() * g).sum(-1), 0.0)
    of_rows = torch.zeros_like(rows)
    of_rows[at[there]] = (weights[..., None] * g).to(rows.dtype)[there]
    return of_rows, of_weights


def _pages(cache, kv_heads, page, dim):
    """The four parts of the pages, as views: key bytes, value bytes, key words, value words."""
    n, half = cache.shape[0], page * dim // 2
    return (cache[..., :half].view(n, kv_heads, page, dim // 2),
            cache[..., half: 2 * half].view(n, kv_heads, page // 4, 16, 2, dim // 64, 2, 2),
            cache[..., 2 * half: 2 * half + 4 * page].view(torch.int32), cache[..., 2 * half + 4 * page:].view(torch.int32))


def _plain_codes(x):
    """4-bit codes (a byte each) and words of the last dimension's vectors."""
    x = x.float()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    bits = ((hi - lo) / torch.full_like(hi, 15.0)).view(torch.int32)
    bits = (bits + 0x7FF + ((bits >> 12) & 1)) & ~0xFFF  # to 12 significant bits, ties to even
    scale = bits.view(torch.float32).clamp(min=SMALLEST)
    zero = torch.round(-lo / scale)
    codes = (torch.round(x / scale[..., None]) + zero[..., None]).clamp(0.0, 15.0)
    return codes.to(torch.uint8), scale.view(torch.int32) | zero.to(torch.int32)


def _plain_write(k, v, slots, cache):
    dim = k.shape[-1]
    page = cache.shape[-1] // (dim + 8)
    keys, values, key_words, value_words = _pages(cache, k.shape[1], page, dim)
    at, j = slots.long() // page, slots.long() % page
    codes, key_words[at, :, j] = _plain_codes(k)
    keys[at, :, j] = codes[..., 0::2] | (codes[..., 1::2] << 4)
    codes, value_words[at, :, j] = _plain_codes(v)
    codes = (codes[..., 0::2] | (codes[..., 1::2] << 4)).view(*codes.shape[:2], 16, dim // 64, 2)
    values[at, :, j // 4, :, j % 4 // 2, :, j % 2] = codes


def _plain_read(cache, slots, case):
    page, dim = case["page"], case["dim"]
    keys, values, key_words, value_words = _pages(cache, case["kv_heads"], page, dim)
    at, j = slots.long() // page, slots.long() % page

    def numbers(codes, words):
        codes = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float()
        return (codes - (words & 15).float()[..., None]) * (words & ~0xFFF).view(torch.float32)[..., None]

    return (numbers(keys[at, :, j], key_words[at, :, j]),
            numbers(values[at, :, j // 4, :, j % 4 // 2, :, j % 2].flatten(-3), value_words[at, :, j]))


def _plain_chunks(s, case):
    page, dim, kv_heads, seqs = case["page"], case["dim"], case["kv_heads"], case["seqs"]
    group, most = case["heads"] // kv_heads, s["most"]
    j = torch.arange(s["most_keys"], device=DEVICE)
    slots = (s["block_table"].long()[:, j // page] * page + j % page).flatten()
    k, v = (x.view(seqs, -1, kv_heads, dim).transpose(1, 2).contiguous() for x in _plain_read(s["cache"], slots, case))
    first, new = s["starts"][:-1, None].long(), s["starts"].diff()[:, None]
    i = torch.arange(most, device=DEVICE)
    there = i < new
    q = s["q"][(first + i).clamp(max=s["q"].shape[0] - 1)].float().view(seqs, most, kv_heads, group, dim)
    q = q.permute(0, 2, 1, 3, 4).reshape(seqs, kv_heads, most * group, dim)
    scores = torch.matmul(q, k.transpose(-1, -2).contiguous()).div_(math.sqrt(dim)).view(seqs, kv_heads, most, group, -1)
    seen = j < (s["context"][:, None] - new + 1 + i)[..., None]
    scores = scores.masked_fill_(~seen[:, None, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores = scores.sub_(torch.where(top.isinf(), 0.0, top)).exp_().flatten(2, 3)
    o = torch.matmul(scores, v) / scores.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.view(seqs, kv_heads, most, group, dim).transpose(1, 2).reshape(seqs, most, case["heads"], dim)[there].to(s["q"].dtype)


# ------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s, case)
    if case["kind"] == "swiglu":
        w = case["width"]
        parts = []
        for x in s["x"].split(512):
            gate, up = x[:, :w].double(), x[:, w:].double()
            parts.append(_exact_codes(up * gate * torch.sigmoid(gate)))
        return {"values": torch.cat([a for a, _ in parts]), "scales": torch.cat([b for _, b in parts])}
    if case["kind"] == "dispatch":
        return _exact_dispatch(s)
    if case["kind"] == "chunks":
        return _exact_chunks(s, case)
    rows, places = s["rows"], s["places"].long()
    out, of_weights = torch.zeros((case["tokens"], case["width"]), dtype=torch.float64, device=DEVICE), torch.zeros(places.shape, dtype=torch.float64, device=DEVICE)
    of_rows = torch.zeros(rows.shape, dtype=torch.float64, device=DEVICE) if case["kind"] == "grads" else None
    for n in range(case["each"]):
        token = torch.nonzero(places[:, n] + 1).flatten()  # (all but -1)
        at, w = places[token, n], s["weights"][token, n].double()[:, None]
        if of_rows is None:
            out.index_add_(0, token, rows[at].double() * w)
        else:
            g = s["grad"][token].double()
            of_rows.index_add_(0, at, g * w)
            of_weights[token, n] = torch.linalg.vecdot(rows[at].double(), g)
    return out if of_rows is None else (of_rows, of_weights)


def _exact_dispatch(s):
    """The rows by a sort of the pairs; whole numbers have no value in 64 bits of their own."""
    ids = s["experts"].flatten().cpu()
    pairs = sorted((i for i in range(len(ids)) if 0 <= ids[i] < s["here"]), key=ids.tolist().__getitem__)
    token = torch.tensor(pairs, dtype=torch.long, device=DEVICE) // s["case"]["each"]

    def moved(x, out):
        got = out.double()
        got[: len(pairs)] = x.double()[token]
        return got

    if s["scales"] is None:
        return moved(s["x"], s["out"]), None, None, None
    return None, moved(s["scales"], s["out_scales"]), None, None


def _exact_codes(y):
    step = torch.linalg.vector_norm(y, math.inf, dim=-1) / 127
    step[step == 0] = 1.0
    return torch.round(y / step[:, None]) * step[:, None], step


def _exact_norm(s, case):
    h = s["x"].double()
    if case["residual"]:  # (rounded to its type: what the next layer adds to, and what the norm is of)
        h = (h + s["residual"].double()).to(s["x"].dtype).double()
    y = h / (torch.linalg.vector_norm(h, dim=-1, keepdim=True).square() / case["width"] + EPS).sqrt() * s["weight"].double()
    values, step = _exact_codes(y)
    return {"values": values, "scales": step, "h": h if case["residual"] else None, "y": y if case["y"] else None}


def _exact_pages(pages, case):
    """[pages, kv_heads, bytes] -> keys, values [pages * page, kv_heads, dim] in FP64."""
    page, dim = case["page"], case["dim"]
    d, j = torch.arange(dim, device=DEVICE), torch.arange(page, device=DEVICE)[:, None]
    width = dim // 16
    at_k = j * (dim // 2) + d // 2
    at_v = page * dim // 2 + (j // 4) * 2 * dim + (d // width) * (dim // 8) + (j % 4 // 2) * width + (d % width // 4) * 4 + (j % 2) * 2 + d % 4 // 2
    got = []
    for n, at in enumerate((at_k, at_v)):
        nibble = (pages[..., at] >> (4 * (d % 2)).to(torch.uint8)) & 15
        word = pages[..., page * (dim + 4 * n): page * (dim + 4 * n + 4)].reshape(*pages.shape[:2], page, 4).to(torch.int32)
        word = word[..., 0] | word[..., 1] << 8 | word[..., 2] << 16 | word[..., 3] << 24
        step = (word & -4096).view(torch.float32).double()[..., None]
        got.append(((nibble.double() - (word & 15).double()[..., None]) * step).transpose(1, 2).flatten(0, 1))
    return got


def _exact_chunks(s, case):
    out, q0 = [], 0
    for b, (new, n) in enumerate(_lengths(case)):
        pages = s["cache"][s["block_table"][b, : -(-n // case["page"])].long()]
        parts = [_exact_pages(p, case) for p in pages.split(max(1, 16384 // case["page"]))]
        k, v = (torch.cat([p[i] for p in parts])[:n] for i in (0, 1))
        got = torch.zeros((new, case["heads"], case["dim"]), dtype=torch.float64, device=DEVICE)
        j, i = torch.arange(n, device=DEVICE), torch.arange(new, device=DEVICE)[:, None]
        for h in range(case["heads"]):
            kv = h * case["kv_heads"] // case["heads"]
            x = s["q"][q0: q0 + new, h].double() @ k[:, kv].t().contiguous() / math.sqrt(case["dim"])
            got[:, h] = torch.softmax(torch.where(j <= i + n - new, x, -math.inf), -1) @ v[:, kv].contiguous()
        out.append(got)
        q0 += new
    return torch.cat(out)
