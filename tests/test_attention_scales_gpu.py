"""Scales at and near zero, and queries of zeros and of the type's largest numbers, against the definition.

Tolerances as for the attention kernels elsewhere: one rounding of the result (u), one of each weight before the second product (w):
|error| <= 1.1 (u |o| + w sum_j p_j |v_j|) + 2^-24."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from paper_2509_01229_amd import api

pytestmark = pytest.mark.gpu
TYPES = (A.F16, A.BF16)


def _draw(rng, shape, dtype):
    return A.round_to(rng.standard_normal(shape, dtype=np.float32), dtype)


def _gpu(x, dtype=None):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to(getattr(torch, dtype)) if dtype else t


def _close(got, want, spread, dtype, weights, what=""):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), f"{what}: not finite"
    off = np.abs(got - want) / (1.1 * (A.UNIT[dtype] * np.abs(want) + weights * spread) + 2.0 ** -24)
    assert off.max() <= 1, f"{what}: {np.sum(off > 1)} of {off.size} off, worst {off.max():.2f} times the tolerance"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.0, 1e-38, -1e-38, 1e-42])
def test_prompts_keys_in_parts(dtype, D, scale):
    """Few queries, whose keys are split over blocks and joined; rows that see nothing of the first tile that their wave takes."""
    import torch

    rng = np.random.default_rng(40)
    lens, Hq, Hkv = [(70, 4000), (33, 2500)], 3, 1
    sq, sk = (np.concatenate(([0], np.cumsum([x[i] for x in lens]))).astype(np.int32) for i in (0, 1))
    q, k, v = _draw(rng, (sq[-1], Hq, D), dtype), _draw(rng, (sk[-1], Hkv, D), dtype), _draw(rng, (sk[-1], Hkv, D), dtype)
    need = int(api.lib().attn_prompt_workspace_size(len(lens), int(sq[-1]), int(sk[-1]), Hq, Hkv, D))
    assert need > 32768  # (the keys are split)
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    for workspace in (ws, ws[:16]):
        for causal in (True, False):
            got = api.attn_prompt(*(_gpu(x, dtype) for x in (q, k, v)), _gpu(sq), _gpu(sk), scale=scale, causal=causal, workspace=workspace)
            for s, (a, b) in enumerate(lens):
                limits = np.arange(a) + b - a + 1 if causal else np.full(a, b)
                want, spread = A.attention(q[sq[s]:sq[s + 1]], k[sk[s]:sk[s + 1]], v[sk[s]:sk[s + 1]], scale, limits)
                _close(got[sq[s]:sq[s + 1]], want, spread, dtype, A.UNIT[dtype], f"sequence {s}, causal {causal}")


def _decode(q, k, v, scale, dtype, page=16):
    """q [new, heads, D] over the keys and values of one sequence; the definition's result, and what its weights' errors multiply."""
    new, c, Hkv, D = len(q), len(k), k.shape[1], k.shape[2]
    pages = -(-c // page)
    cache = api.kv4_cache(pages, page, Hkv, D)
    api.kv4_write(_gpu(k, dtype), _gpu(v, dtype), _gpu(np.arange(c, dtype=np.int32)), cache)
    got = api.kv4_attention(_gpu(q[None], dtype), cache, _gpu(np.arange(pages, dtype=np.int32)[None]), _gpu(np.array([c], dtype=np.int32)), scale=scale)[0]
    k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
    return got, *A.attention(q, k, v, scale, c - new + 1 + np.arange(new))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,Hq,Hkv,new,c", [(128, 4, 2, 1, 70), (64, 8, 1, 5, 900), (128, 16, 2, 1, 3000), (128, 16, 2, 3, 3000)])
@pytest.mark.parametrize("scale", [0.0, 1e-30, -1e-30, 1e-42, 0.1])
def test_queries_of_zeros_over_the_cache(dtype, D, Hq, Hkv, new, c, scale):
    """They see the mean of the values whatever the scale; next to rows that are not zero."""
    rng = np.random.default_rng(41)
    q, k, v = _draw(rng, (new, Hq, D), dtype), _draw(rng, (c, Hkv, D), dtype), _draw(rng, (c, Hkv, D), dtype)
    q[:, 1] = 0
    q[-1, -1] = 0
    got, want, spread = _decode(q, k, v, scale, dtype)
    _close(got, want, spread, dtype, 2.0 ** -11)


@pytest.mark.parametrize("new", [1, 6])
def test_queries_of_zeros_alone(new):
    rng = np.random.default_rng(42)
    k, v = _draw(rng, (200, 1, 64), A.F16), _draw(rng, (200, 1, 64), A.F16)
    for scale in (0.0, 0.125):
        got, want, spread = _decode(np.zeros((new, 4, 64), np.float32), k, v, scale, A.F16)
        _close(got, want, spread, A.F16, 2.0 ** -11)


@pytest.mark.parametrize("size", [2.0 ** 113, 2.0 ** 118, 2.0 ** 124])
def test_queries_near_the_end_of_bf16(size):
    """With a scale that brings the scores back to ordinary numbers, and with one that leaves all weight to the key that fits best."""
    rng = np.random.default_rng(43)
    k, v = _draw(rng, (90, 1, 64), A.BF16), _draw(rng, (90, 1, 64), A.BF16)
    q = A.round_to(_draw(rng, (1, 2, 64), A.BF16) * np.float32(size), A.BF16)
    assert np.isfinite(q).all()
    got, want, spread = _decode(q, k, v, 0.125 / size, A.BF16)
    _close(got, want, spread, A.BF16, 2.0 ** -11)
    k[40, 0] = A.round_to(np.sign(q[0, 0]) * 3, A.BF16)
    k[17, 0] = A.round_to(np.sign(q[0, 1]) * 3, A.BF16)
    got, want, spread = _decode(q, k, v, 0.125, A.BF16)
    _close(got, want, spread, A.BF16, 2.0 ** -11)
