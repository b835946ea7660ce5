"""Several host threads that call on one stream with one workspace: each gets what it gets alone.  Calls of two kernels (the attention of
many sequences, whose chunks are found beforehand, and products with K slices) next to calls of one that write to the workspace too."""
import threading

import numpy as np
import pytest

import gpu_helpers as H
from oracle import attention_oracle as A
from paper_2509_01229_amd import api

pytestmark = pytest.mark.gpu


def _decode(n, Hq, Hkv, new, D, seed):
    import torch

    rng = np.random.default_rng(seed)
    page, width = 16, 40
    contexts = rng.integers(0, page * width + 1, n).astype(np.int32)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    cache = api.kv4_cache(n * width, page, Hkv, D)
    kv = torch.randn((2, n * width * page, Hkv, D), generator=gen, device="cuda").half()
    api.kv4_write(kv[0], kv[1], torch.arange(n * width * page, dtype=torch.int32, device="cuda"), cache)
    q = torch.randn((n, new, Hq, D), generator=gen, device="cuda").half()
    table = torch.from_numpy(rng.permutation(n * width).astype(np.int32).reshape(n, width)).cuda()
    ctx = torch.from_numpy(contexts).cuda()
    # one sequence against the definition, so that "alone" is right in itself
    b = int(contexts.argmax())
    slots = (table[b, :, None] * page + torch.arange(page, dtype=torch.int32, device="cuda")).flatten()[: int(contexts[b])]
    k, v = (A.dequantise(*A.quantise(x[slots.long()].float().cpu().numpy())) for x in kv)
    want = A.attention(q[b].float().cpu().numpy(), k, v, D ** -0.5, contexts[b] - new + 1 + np.arange(new))
    return (q, cache, table, ctx), b, want


def test_threads_on_one_stream():
    import torch

    work = []
    for n, Hq, Hkv, new, D, seed in ((140, 8, 8, 1, 128, 1), (300, 8, 8, 1, 64, 2), (110, 32, 8, 5, 128, 3), (2, 32, 8, 1, 128, 4)):
        args, b, (want, spread) = _decode(n, Hq, Hkv, new, D, seed)
        run = lambda ws, args=args: api.kv4_attention(*args, workspace=ws)
        ws = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
        alone = run(ws)
        err = np.abs(alone[b].float().cpu().numpy() - want)
        assert (err <= 1.1 * 2.0 ** -11 * (np.abs(want) + spread) + 2.0 ** -24).all()
        work.append((run, alone))
    M, N, K, g = 256, 512, 16384, 64
    W = H.RandomWeights(N, K, g, seed=6)
    X, s = W.activations(M)
    product = W.product(X)
    for name in ("solo16_g2_m256_s4", "duo_m64_s2"):
        rows = M if "m256" in name else 64
        variant = api.w4a8_variant_names().index(name)
        run = lambda ws, variant=variant, rows=rows: api.w4a8_gemm_variant(variant, X[:rows], s[:rows], W.codes, W.gparams, W.scales, N, K, g,
                                                                           want_y=False, workspace=ws)[1]
        work.append((run, product[:rows]))
    torch.cuda.synchronize()

    shared = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    wrong, errors = [0] * len(work), []

    def go(i):
        run, alone = work[i]
        try:
            outs = [run(shared) for _ in range(40)]
            torch.cuda.current_stream().synchronize()
            wrong[i] = sum(not torch.equal(o, alone) for o in outs)
        except Exception as e:  # noqa: BLE001 (a thread's error fails the test)
            errors.append(e)

    threads = [threading.Thread(target=go, args=(i,)) for i in range(len(work))]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not errors and wrong == [0] * len(work)
    assert not shared[:32768].any()
