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
