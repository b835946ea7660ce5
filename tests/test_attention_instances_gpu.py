"""Kernel forms that only large batches reach, each at both head sizes and types against the definition: chunks that a kernel of its own
finds (blocks of four and of eight waves, one and two tiles of rows), many chunks joined in sets, and more prompts than a wave has lanes.
Tolerances as in test_attention_gpu.py."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from paper_2509_01229_amd import api
from test_attention_gpu import TYPES, _close, _draw, _filled, _gpu, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,longest,Hq,Hkv,new,long", [
    (140, 200, 8, 8, 1, {70: 5000, 139: 2500}),            # 16 rows at most, blocks of four waves
    (300, 60, 16, 4, 3, {0: 0, 299: 4000, 5: 65}),         # the same, 12 rows
    (70, 90, 32, 8, 5, {3: 3000, 4: 0}),                   # 20 rows, blocks of four waves
    (70, 60, 16, 8, 12, {0: 9000, 69: 20000, 33: 0}),      # 24 rows; more chunks than one set joins
    (40, 90, 32, 8, 5, {39: 2000, 7: 1}),                  # 20 rows, blocks of eight waves
    (36, 50, 16, 8, 10, {0: 20000, 20: 0, 35: 300}),       # the same, more chunks than one set
    (17, 130, 32, 2, 6, {3: 5000}),                        # 96 rows: three passes
])
def test_large_batches(dtype, D, n, longest, Hq, Hkv, new, long):
    import torch

    rng = np.random.default_rng(n + D)
    contexts = [int(x) for x in rng.integers(0, longest + 1, n)]
    for s, c in long.items():
        contexts[s] = c
    cache, table, keys, values = _filled(rng, contexts, 32, Hkv, D, dtype)
    q = _draw(rng, (n * new, Hq, D), dtype)
    args = (_gpu(q, dtype).unflatten(0, (n, new)), cache, _gpu(table), _gpu(np.array(contexts, dtype=np.int32)))
    ws = torch.zeros(int(api.lib().kv4_attention_workspace_size(n, new, Hq, Hkv, D)), dtype=torch.uint8, device="cuda")
    ws[32768:] = 255
    got = [_np(api.kv4_attention(*args, workspace=w)) for w in (ws, ws, ws[:16])]
    assert np.array_equal(got[0], got[1]) and not ws[:32768].any()
    for g in got[1:]:
        for b, c in enumerate(contexts):
            want, spread = A.attention(q[b * new:(b + 1) * new], keys[b], values[b], D ** -0.5, c - new + 1 + np.arange(new))
            _close(g[b], want, spread, dtype, 2.0 ** -11, f"sequence {b} of {c}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_many_prompts_of_wide_heads(dtype, causal):
    rng = np.random.default_rng(50)
    n, D, Hq, Hkv = 90, 128, 6, 2
    lens_q, lens_k = rng.integers(0, 60, n), rng.integers(0, 60, n)
    lens_q[45], lens_k[45], lens_k[89] = 300, 333, 200
    sq, sk = (np.concatenate(([0], np.cumsum(x))).astype(np.int32) for x in (lens_q, lens_k))
    q, k, v = _draw(rng, (sq[-1], Hq, D), dtype), _draw(rng, (sk[-1], Hkv, D), dtype, True), _draw(rng, (sk[-1], Hkv, D), dtype)
    got = _np(api.attn_prompt(*(_gpu(x, dtype) for x in (q, k, v)), _gpu(sq), _gpu(sk), causal=causal))
    for s in range(n):
        a, b = int(lens_q[s]), int(lens_k[s])
        if a:
            limits = np.arange(a) + b - a + 1 if causal else np.full(a, b)
            want, spread = A.attention(q[sq[s]:sq[s + 1]], k[sk[s]:sk[s + 1]], v[sk[s]:sk[s + 1]], D ** -0.5, limits)
            _close(got[sq[s]:sq[s + 1]], want, spread, dtype, A.UNIT[dtype], f"sequence {s}")
