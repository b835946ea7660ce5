"""A decoder layer's operators one behind the other, as a serving program and a training step use them.

Serving: each operator's result against the definition applied to what the one before it returned, so that no tolerance adds up: codes of the norm, moved rows
and accumulators of the products bit for bit, the rest to its own tolerance (as in test_layer_gpu.py, test_chunks_gpu.py, test_grouped_gpu.py).
Training: the gradients of a mixture of FP16 experts against those of its formula in FP64, and against differences of it."""
import importlib.util
import os

import numpy as np
import pytest

import gpu_helpers as H
from oracle import attention_oracle as A
from oracle import layer_oracle as R
from oracle import lqq_oracle as O
from paper_2509_01229_amd import api
from paper_2509_01229_amd import workloads as WL
from test_attention_gpu import _close, _gpu, _np
from test_layer_gpu import _draw

pytestmark = pytest.mark.gpu


def _example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")
    spec = importlib.util.spec_from_file_location("decoder_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    return example


def test_example_runs():
    import torch

    got, want = _example().run(heads=4, kv_heads=2, experts=6, each=2, inner=256, prompt=150, chunk=32, others=2)
    assert got.shape == want.shape == (150, 512) and torch.isfinite(got).all() and torch.isfinite(want).all()


@pytest.mark.parametrize("prompt,chunk,others", [(150, 32, 2), (129, 64, 1), (70, 7, 3), (260, 200, 0)])
def test_example_in_chunks_is_the_example_in_one_piece(prompt, chunk, others):
    """Every token takes every expert, so that no choice hangs on a rounding.  Up to the attention both are the same bit for bit (the products' sums are whole numbers, a token's rows
    its own, the cache's codes those of the same keys).  The attention's results are off by 3e-4 of themselves each (FP16, weights rounded), 4.2e-4 together.  An INT8 row of them has
    steps of about 1/36 of its mean size (127 for 3.5 times that): a difference d of it moves one code in 36 d by a step, which is sqrt(d / 36) of the row; three of these one behind the other
    (output, first and second products) make 0.35%, 1%, 1.7% out of it, of which the last is only of the mixture's part.  Hence 2% of all, and 4% of a token, whose largest element may be less
    above the others; a wrong position, slot, start or context changes an attention result of mean size 0.1 to 1 altogether, in a stream of 1.4."""
    import torch

    got, want = (t.double() for t in _example().run(heads=4, kv_heads=2, experts=3, each=3, inner=256, prompt=prompt, chunk=chunk, others=others))
    off = torch.linalg.vector_norm(got - want, dim=1) / torch.linalg.vector_norm(want, dim=1)
    assert got.shape == (prompt, 512) and torch.isfinite(got).all() and (off <= 0.04).all(), float(off.max())
    assert float((got - want).norm() / want.norm()) <= 0.02, float((got - want).norm() / want.norm())


def test_the_operators_of_a_layer_one_behind_the_other():
    import torch

    E, each, heads, kv_heads, D, hidden, inner, page, g = 5, 2, 4, 2, 128, 512, 256, 16, 64
    rng = np.random.default_rng(1)
    weights = {name: [WL.make_weights(N, K, K ** -0.5, seed=i + 10 * e) for e in range(n)]
               for i, (name, n, N, K) in enumerate((("qkv", 1, 1024, 512), ("out", 1, 512, 512), ("up", E, 512, 512), ("down", E, 512, 256)))}
    oracle = {name: [O.quantize_weights(W, g) for W in Ws] for name, Ws in weights.items()}
    packs = {name: [api.liquidquant_pack_weights(W, g) for W in Ws] for name, Ws in weights.items()}
    blobs = {name: [_gpu(np.concatenate([p[i] for p in ps])) for i in (0, 1)] + [_gpu(np.stack([p[2] for p in ps]))] for name, ps in packs.items()}

    def product(name, x, s, offsets=None):
        (N, K), Ws = weights[name][0].shape, oracle[name]
        offs = [0, len(x)] if offsets is None else offsets
        if offsets is None:
            y = api.w4a8_gemm(x, s, blobs[name][0], blobs[name][1], blobs[name][2][0], N, K, g)
        else:
            y = api.w4a8_grouped_gemm(offsets, x, s, *blobs[name], N, K, g)[0]
        xs, ss = x.cpu().numpy(), s.cpu().numpy()
        acc, _ = O.grouped_w4a8_gemm(xs, ss, np.asarray(offs), Ws)
        s_w = np.concatenate([np.repeat(Ws[e]["s_w"][None], offs[e + 1] - offs[e], 0) for e in range(len(Ws))])
        H.assert_fp16_close(y.cpu().numpy(), acc.astype(np.float64) * ss.astype(np.float64)[:, None] * s_w.astype(np.float64), name)
        return y

    def norm(x, weight, residual):
        q, s, h, y = api.w4a8_norm_quantize(x, _gpu(weight), residual, want_y=True)
        want = R.norm_quantise(_np(x), _np(residual), weight, 1e-6, A.F16)
        assert np.array_equal(q.cpu().numpy(), want[0]) and np.array_equal(s.cpu().numpy(), want[1]) and np.array_equal(_np(h), want[2])
        assert np.array_equal(_np(y), A.round_to(want[3], A.F16))
        return q, s, h, y

    # a step: 37 tokens of a prompt that has 20, one token of a sequence of 70, nothing of a third
    new, before = np.array([37, 1, 0]), np.array([20, 69, 5])
    context, T = before + new, int(new.sum())
    starts = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
    table = rng.permutation(15).astype(np.int32).reshape(3, 5)
    cache = api.kv4_cache(15, page, kv_heads, D)
    held_k, held_v = [], []
    for b, n in enumerate(before):
        k, v = _draw(rng, (n, kv_heads, D), A.F16), _draw(rng, (n, kv_heads, D), A.F16)
        j = np.arange(n)
        api.kv4_write(_gpu(k, A.F16), _gpu(v, A.F16), _gpu((table[b, j // page] * page + j % page).astype(np.int32)), cache)
        held_k.append(k)
        held_v.append(v)
    sequence = np.repeat(np.arange(3), new)
    position = (np.arange(T) - starts[sequence] + before[sequence]).astype(np.int32)
    slots = (table[sequence, position // page] * page + position % page).astype(np.int32)
    rope = A.rope_table(100, D).astype(np.float32)
    norms = [(1 + 0.1 * rng.standard_normal(hidden)).astype(np.float32) for _ in range(2)]
    x, residual = _gpu(_draw(rng, (T, hidden), A.F16), A.F16), _gpu(_draw(rng, (T, hidden), A.F16, 2.0), A.F16)

    rows, s, residual, _ = norm(x, norms[0], residual)
    q, k, v = product("qkv", rows, s).view(T, heads + 2 * kv_heads, D).split((heads, kv_heads, kv_heads), 1)
    turned, turned_k = api.attn_qk_norm_rope(q, k, _gpu(position), _gpu(rope))
    q = api.kv4_append(q, k, v, _gpu(position), _gpu(rope), _gpu(slots), cache)
    assert torch.equal(q, turned)
    a = api.kv4_attention_chunks(q, cache, _gpu(table), _gpu(context.astype(np.int32)), _gpu(starts))
    for b in range(2):
        mine = slice(starts[b], starts[b + 1])
        ks, vs = (A.dequantise(*A.quantise(np.concatenate([held, _np(t)[mine]]))) for held, t in ((held_k[b], turned_k), (held_v[b], v)))
        want, spread = A.attention(_np(q)[mine], ks, vs, D ** -0.5, before[b] + 1 + np.arange(new[b]))
        _close(_np(a)[mine], want, spread, A.F16, 2.0 ** -11, f"sequence {b}")
    rows, s = api.w4a8_quantize_activations(a.view(T, hidden))
    rows, s, residual, y = norm(product("out", rows, s), norms[1], residual)
    router = _gpu(rng.standard_normal((hidden, E)).astype(np.float32) * np.float32(hidden ** -0.5))
    best = (y.float() @ router).topk(each, -1)
    experts, w = best.indices.to(torch.int32), torch.softmax(best.values, -1)
    experts[3, 0], experts[7, 1], experts[9] = E, -1, -1    # (another GPU's)
    moved, moved_s, offsets, places = api.moe_dispatch(rows, experts, E, act_scales=s)
    want_offsets, want_places, source = R.dispatch(experts.cpu().numpy(), E)
    assert np.array_equal(offsets.cpu().numpy(), want_offsets) and np.array_equal(places.cpu().numpy(), want_places)
    used = len(source)
    assert torch.equal(moved[:used], rows[_gpu(source)]) and torch.equal(moved_s[:used], s[_gpu(source)])
    offsets = offsets.tolist()
    gates = product("up", moved[:used], moved_s[:used], offsets)
    codes, s = api.w4a8_swiglu_quantize(gates)
    want, d = R.gated(_np(gates)), (4 + np.abs(_np(gates)[:, :inner])) * 2.0 ** -22
    step = s.cpu().numpy().astype(np.float64)[:, None]
    assert (np.abs(codes.cpu().numpy() * step - want) <= step * (0.5 + 127 * 2.0 ** -22) + d * np.abs(want)).all()
    results = product("down", codes, s, offsets)
    out = api.moe_combine(results, places, w)
    want, size = R.combine(_np(results), places.cpu().numpy(), w.cpu().numpy())
    assert (np.abs(_np(out) - want) <= A.UNIT[A.F16] * np.abs(want) + (each + 1) * 2.0 ** -24 * size + 2.0 ** -25).all()
    assert not out[9].any()


def test_gradients_of_a_mixture():
    """L = sum(c * out), out = sum_j w_j(x) (rows W_e) of FP16 rows: the gradients of x, of the weights w and of the experts' matrices, which one product for
    each expert makes from moe_combine_backward's rows.  Every tensor is rounded to FP16 where it is one; the tolerance counts each rounding (2^-11 of
    the term) on its way to a result."""
    import torch

    rng = np.random.default_rng(3)
    T, each, E, K, N = 41, 3, 6, 64, 48
    u = 2.0 ** -11
    x, W, c = _draw(rng, (T, K), A.F16), _draw(rng, (E, K, N), A.F16, 0.2), _draw(rng, (T, N), A.F16)
    ids = np.argsort(rng.random((T, E)), 1)[:, :each].astype(np.int32)
    ids[5, 1], ids[8] = -1, E
    w = rng.random((T, each)).astype(np.float32)
    there = (ids >= 0) & (ids < E)
    picked = W.astype(np.float64)[np.where(there, ids, 0)] * there[..., None, None]          # [T, each, K, N]
    # the formula's, FP64, and the sums of the terms' absolute values
    y = np.einsum("tk,tjkn->tjn", x.astype(np.float64), picked)
    want_w, size_w = (y * c[:, None]).sum(-1), np.einsum("tk,tjkn,tn->tj", np.abs(x), np.abs(picked), np.abs(c))
    g = w[..., None].astype(np.float64) * c[:, None]                                         # dL/dy
    want_x, size_x = np.einsum("tjn,tjkn->tk", g, picked), np.einsum("tjn,tjkn->tk", np.abs(g), np.abs(picked))
    # the operators
    rows, _, offsets, places = api.moe_dispatch(_gpu(x, A.F16), _gpu(ids), E)
    offs = offsets.tolist()
    results = torch.full((T * each, N), float("nan"), dtype=torch.float16, device="cuda")    # (rows behind the last expert's: nobody's)
    dW = _gpu(W).half()
    for e in range(E):
        results[offs[e]:offs[e + 1]] = rows[offs[e]:offs[e + 1]] @ dW[e]
    out = api.moe_combine(results, places, _gpu(w))
    of_results, of_w = api.moe_combine_backward(_gpu(c, A.F16), results, places, _gpu(w), row_offsets=offsets)
    of_rows = torch.zeros((T * each, K), dtype=torch.float16, device="cuda")
    of_W = np.zeros((E, K, N))
    for e in range(E):
        mine = slice(offs[e], offs[e + 1])
        of_rows[mine] = of_results[mine] @ dW[e].t().contiguous()
        of_W[e] = (rows[mine].double().t() @ of_results[mine].double()).cpu().numpy()
    of_x = api.moe_combine(of_rows, places)
    want_out, size_out = (y * w[..., None]).sum(1), np.einsum("tk,tjkn,tj->tn", np.abs(x), np.abs(picked), w)
    assert (np.abs(_np(out) - want_out) <= 1.1 * 2 * u * size_out + 2.0 ** -23).all()        # (results and out)
    assert (np.abs(of_w.cpu().numpy() - want_w) <= 1.1 * u * size_w + 2.0 ** -20).all()      # (results)
    assert (np.abs(_np(of_x) - want_x) <= 1.1 * 3 * u * size_x + 2.0 ** -22).all()           # (their gradients, the rows' and x's)
    assert not of_w[8].any() and not of_x[8].any() and not of_results[offs[-1]:].any()
    token, j = np.nonzero(there)
    want_W, size_W = np.zeros((2, E, K, N))
    for t, i in zip(token, j):
        want_W[ids[t, i]] += np.outer(x[t], g[t, i])
        size_W[ids[t, i]] += np.abs(np.outer(x[t], g[t, i]))
    assert (np.abs(of_W - want_W) <= 1.1 * u * size_W + 2.0 ** -20).all()
    # against differences of the formula: L is linear in w, and in x for given experts, so that they are exact in FP64
    loss = lambda x, w: float((np.einsum("tk,tjkn,tj->tn", x, picked, w * there) * c).sum())  # noqa: E731
    for t, i in ((0, 0), (5, 2), (40, 1)):
        step = np.zeros((T, each))
        step[t, i] = 0.5
        assert abs((loss(x.astype(np.float64), w + step) - loss(x.astype(np.float64), w - step)) - float(of_w[t, i])) <= 1.1 * u * size_w[t, i] + 2.0 ** -20
    for t, i in ((0, 3), (5, 63), (20, 17)):
        step = np.zeros((T, K))
        step[t, i] = 0.5
        assert abs((loss(x + step, w.astype(np.float64)) - loss(x - step, w.astype(np.float64))) - float(of_x[t, i])) <= 1.1 * 3 * u * size_x[t, i] + 2.0 ** -22
