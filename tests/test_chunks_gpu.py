"""Attention of chunks of new tokens over the 4-bit cache against its definition (oracle/attention_oracle.py, FP64).

Tolerances as for the other attention kernels: a result is rounded once to its type (u = 2^-11 in FP16, 2^-8 in BF16), a weight times its value's scale
once to FP16 before the second product (w = 2^-11, which moves the result by at most w * sum_j p_j |v_j|); everything else is FP32 (below 2^-16 of
that).  Hence |error| <= 1.1 (u |o| + w sum_j p_j |v_j|) + 2^-24.  Weights under 2^-20 of the row's largest product of weight and scale have fewer bits in FP16, an
error of 2^-31 of that product each, times a code's 15 at most: 2^-13 of it for 16384 of them at once."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from paper_2509_01229_amd import api
from test_attention_gpu import TYPES, _close, _draw, _filled, _gpu, _np, _views

pytestmark = pytest.mark.gpu


def _starts(new, at=0):
    return np.concatenate(([at], at + np.cumsum(new))).astype(np.int32)


def _ints(x):
    return _gpu(np.asarray(x, dtype=np.int32))


def _check(got, q, starts, contexts, keys, values, dtype, scale=None, which=None):
    D = q.shape[-1]
    for s, c in enumerate(contexts):
        n = int(starts[s + 1] - starts[s])
        if not n or (which is not None and s not in which):
            continue
        want, spread = A.attention(q[starts[s]:starts[s + 1]], keys[s], values[s], D ** -0.5 if scale is None else scale, c - n + 1 + np.arange(n))
        _close(got[starts[s]:starts[s + 1]], want, spread, dtype, 2.0 ** -11, f"sequence {s}: {n} of {c}")


CHUNKS = [
    # new tokens and contexts of the sequences, page, Hq, Hkv
    ([1], [1], 16, 1, 1),
    ([17], [517], 64, 4, 4),
    ([1, 33, 1, 0, 64, 1], [100, 33, 64, 50, 65, 0], 16, 8, 2),       # single tokens, whole prompts, nothing new, an empty context
    ([5, 40, 3], [3, 20, 3], 32, 6, 2),                              # contexts shorter than the new tokens: rows without keys
    ([200, 129, 1], [263, 129, 700], 128, 28, 4),                    # groups of 7
    ([70, 257], [1000, 300], 256, 8, 1),                             # pages longer than a tile of keys
    ([300, 31], [300, 2000], 16, 24, 8),
    ([9, 2, 130], [3000, 4097, 2500], 64, 3, 1),                     # few queries, many keys: parts of the keys
    ([1], [9000], 16, 8, 2),                                         # few rows of one sequence: many parts
    ([8, 9, 32, 33], [1030, 2100, 31, 40], 256, 4, 1),               # 32 rows, 36, 128, 132: tiles with few rows behind full ones
    ([65, 64, 63, 1], [1100, 65, 1200, 2], 32, 4, 2),
    ([1, 2, 3, 4, 5], [33, 64, 129, 4, 2], 16, 32, 1),               # 32 rows a token
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(CHUNKS)))
def test_chunks(dtype, D, case):
    import torch

    new, contexts, page, Hq, Hkv = CHUNKS[case]
    rng = np.random.default_rng(case)
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
    starts = _starts(new, at=3)
    q = _draw(rng, (starts[-1] + 5, Hq, D), dtype) * np.float32(2.0)
    dq = _views((q,), dtype, pad=2)[0]
    assert not dq.is_contiguous()
    args = (cache, _gpu(table), _ints(contexts), _ints(starts))
    need = int(api.lib().kv4_attention_chunks_workspace_size(len(new), len(q), Hq, Hkv, D, page, table.shape[1]))
    ws = torch.zeros(max(need, 32768 + 16), dtype=torch.uint8, device="cuda")
    ws[32768:] = 255  # (what it holds does not matter)
    out = torch.full((len(q), Hq, D), 7.0, dtype=dq.dtype, device="cuda")
    assert api.kv4_attention_chunks(dq, *args, out=out, workspace=ws) is out
    got = _np(out)
    assert (got[:3] == 7.0).all() and (got[starts[-1]:] == 7.0).all()    # nobody's rows
    _check(got, q, starts, contexts, keys, values, dtype)
    assert not ws[:32768].any()
    again = api.kv4_attention_chunks(dq, *args, workspace=ws)
    kept = slice(3, int(starts[-1]))
    assert torch.equal(again[kept], out[kept]) and torch.equal(api.kv4_attention_chunks(dq, *args)[kept], out[kept])
    _check(_np(api.kv4_attention_chunks(dq, *args, workspace=ws[:16])), q, starts, contexts, keys, values, dtype)  # (too small: without parts)


def test_many_sequences_of_few_rows():
    """More sequences than a wave has lanes, each with one block for all of its keys."""
    rng = np.random.default_rng(71)
    D, Hq, Hkv, page, dtype = 128, 8, 2, 16, A.BF16
    new, contexts = rng.integers(1, 4, 70), rng.integers(1, 900, 70).tolist()
    contexts[3], new[3] = 5000, 1
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
    starts = _starts(new)
    q = _draw(rng, (starts[-1], Hq, D), dtype)
    got = _np(api.kv4_attention_chunks(_gpu(q, dtype), cache, _gpu(table), _ints(contexts), _ints(starts)))
    _check(got, q, starts, contexts, keys, values, dtype)


@pytest.mark.parametrize("n,longest", [(65, 40), (150, 90), (4500, 2)])
def test_many_sequences(n, longest):
    """More sequences than a wave has lanes, empty ones among them, a long one, and rows before the first and behind the last that are nobody's."""
    import torch

    rng = np.random.default_rng(n)
    D, Hq, Hkv, page, dtype = 64, 6, 2, 16, A.F16
    new = rng.integers(0, longest + 1, n)
    new[n // 2] = 300
    contexts = [int(a + rng.integers(0, 30)) if rng.random() < 0.9 else int(rng.integers(0, 20)) for a in new]
    contexts[n // 2] = 333
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
    starts = _starts(new, at=5)
    q = _draw(rng, (starts[-1] + 9, Hq, D), dtype)
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    got = _np(api.kv4_attention_chunks(_gpu(q, dtype), cache, _gpu(table), _ints(contexts), _ints(starts), out=out))
    assert (got[:5] == 7.0).all() and (got[starts[-1]:] == 7.0).all()
    _check(got, q, starts, contexts, keys, values, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 3, 40])
def test_the_same_as_the_attention_of_new_tokens(dtype, n):
    """Sequences with as many new tokens each: kv4_attention's results, to within both kernels' tolerances."""
    rng = np.random.default_rng(n)
    contexts, page, Hq, Hkv, D = [700, 64, 41, 300], 32, 8, 2, 128
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
    q = _draw(rng, (len(contexts) * n, Hq, D), dtype)
    starts = _starts([n] * len(contexts))
    one = _np(api.kv4_attention_chunks(_gpu(q, dtype), cache, _gpu(table), _ints(contexts), _ints(starts)))
    two = _np(api.kv4_attention(_gpu(q, dtype).unflatten(0, (len(contexts), n)), cache, _gpu(table), _ints(contexts))).reshape(one.shape)
    for got in (one, two):
        _check(got, q, starts, contexts, keys, values, dtype)


@pytest.mark.parametrize("n", [40, 7])
@pytest.mark.parametrize("dtype", TYPES)
def test_weights_of_all_sizes(dtype, n):
    """Scores far apart, in rising and falling order (the running maximum moves often, or never), and values whose scales differ by
    2^20 (FP16: 2^12) from token to token."""
    rng = np.random.default_rng(5)
    D, page, Hq, Hkv, c = 128, 32, 4, 2, 700
    for order in (1, -1):
        q = _draw(rng, (n, Hq, D), dtype)
        k = rng.standard_normal((c, Hkv, D)).astype(np.float32) * 0.1
        k += np.linspace(-1, 1, c, dtype=np.float32)[::order, None, None] * q[:1, ::2] * np.float32(3)
        v = rng.standard_normal((c, Hkv, D)).astype(np.float32) * np.exp2(rng.integers(-6 if dtype == A.F16 else -10, 7 if dtype == A.F16 else 11, (c, 1, 1))).astype(np.float32)
        k, v = A.round_to(k, dtype), A.round_to(v, dtype)
        cache = api.kv4_cache(22, page, Hkv, D)
        api.kv4_write(_gpu(k, dtype), _gpu(v, dtype), _ints(np.arange(c)), cache)
        got = api.kv4_attention_chunks(_gpu(q, dtype), cache, _ints(np.arange(22)[None]), _ints([c]), _ints([0, n]))
        k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
        _check(_np(got), q, [0, n], [c], [k], [v], dtype)


@pytest.mark.parametrize("n", [5, 70])
@pytest.mark.parametrize("split", [False, True])
def test_values_near_the_ends_of_bf16(split, n):
    """Values of 2^126 and of 2^-110, alone and next to rows of zeros (whose scale is 2^-100) and to each other; queries of 2^100 beside ones of 2^-20."""
    rng = np.random.default_rng(6)
    D, page, c = 64, 16, 400 if split else 40
    q, k = _draw(rng, (n, 2, D), A.BF16), _draw(rng, (c, 1, D), A.BF16)
    q = A.round_to(q * np.float32(2.0) ** np.resize(np.array([100, 98, 60, -20, 100], dtype=np.float32), n)[:, None, None], A.BF16)
    q[2] = 0
    for sizes in ([126], [-110], [126, None], [-110, None], [30, None, -60], [126, -90, None], [60, 20, None, -20]):
        v = _draw(rng, (c, 1, D), A.BF16).clip(-1.5, 1.5)
        for i, e in enumerate(sizes):
            v[i::len(sizes)] *= np.float32(0 if e is None else 2.0 ** e)
        v = A.round_to(v, A.BF16)
        pages = -(-c // page)
        cache = api.kv4_cache(pages, page, 1, D)
        api.kv4_write(_gpu(k, A.BF16), _gpu(v, A.BF16), _ints(np.arange(c)), cache)
        got = api.kv4_attention_chunks(_gpu(q, A.BF16), cache, _ints(np.arange(pages)[None]), _ints([c]), _ints([0, n]), scale=2.0 ** -103)
        kk, vv = (A.dequantise(*A.quantise(x)) for x in (k, v))
        want, spread = A.attention(q, kk, vv, 2.0 ** -103, c - n + 1 + np.arange(n))
        got = got.double().cpu().numpy()
        # A weight times its value's scale is an FP16 number whose step is 2^-24 at least, and the largest of a row's is 2^6 at least: half a step is 2^-31 of
        # it, and each key's moves a result by that times 15 at most.  (So a value that is 2^-31 of another's scale may vanish, also where that one's code is 0.)
        limit = c - n + 1 + np.arange(n)
        scores = np.where(np.arange(c) < limit[:, None, None], q.astype(np.float64) @ kk[:, 0].astype(np.float64).T * 2.0 ** -103, -np.inf)
        p = np.where(limit[:, None, None] > 0, np.exp(scores - np.maximum(scores.max(-1, keepdims=True), -1e300)), 0.0)
        largest = (p * A.quantise(v)[1].astype(np.float64).reshape(c)).max(-1) / np.maximum(p.sum(-1), 1.0)
        tol = 1.1 * (A.UNIT[A.BF16] * np.abs(want) + 2.0 ** -11 * spread) + (15 * 2.0 ** -31 * c * largest)[..., None]
        assert (np.abs(got - want) <= tol).all(), sizes


def test_places_that_nothing_was_written_to_count_as_zeros():
    rng = np.random.default_rng(21)
    D, page, Hq, Hkv, c, n = 128, 16, 4, 2, 90, 20
    k, v = _draw(rng, (c, Hkv, D), A.F16), _draw(rng, (c, Hkv, D), A.F16)
    skip = np.array([0, 5, 17, 80])
    slots = np.arange(c, dtype=np.int32)
    slots[skip] = -1
    cache = api.kv4_cache(6, page, Hkv, D)
    api.kv4_write(_gpu(k, A.F16), _gpu(v, A.F16), _gpu(slots), cache)
    kk, vv = (A.dequantise(*A.quantise(x)) for x in (k, v))
    kk[skip], vv[skip] = 0, 0
    q = _draw(rng, (n, Hq, D), A.F16)
    got = api.kv4_attention_chunks(_gpu(q, A.F16), cache, _ints(np.arange(6)[None]), _ints([c]), _ints([0, n]))
    _check(_np(got), q, [0, n], [c], [kk], [vv], A.F16)


@pytest.mark.parametrize("n", [80, 13])
@pytest.mark.parametrize("dtype", TYPES)
def test_nan_stays_with_those_that_see_it(dtype, n):
    """A key, or a value, that is not finite: only for the queries that see it; and a query that is not: only for itself."""
    rng = np.random.default_rng(7)
    D, page, Hq, Hkv, contexts, new = 128, 16, 4, 2, [190, 60], [n, 3]
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
    starts = _starts(new)
    q = _draw(rng, (starts[-1], Hq, D), dtype)
    call = lambda q, cache: _np(api.kv4_attention_chunks(_gpu(q, dtype), cache, _gpu(table), _ints(contexts), _ints(starts)))  # noqa: E731
    clean = call(q, cache)
    for which in (0, 1):
        for key in (5, 128, 150, 189):
            spoilt = cache.clone()
            at = page * D + which * 4 * page + 4 * (key % page)
            spoilt[int(table[0, key // page]), 1, at:at + 4] = _gpu(np.array([0x7FC00000], dtype="<u4").view(np.uint8))
            got = call(q, spoilt)
            sees = np.zeros(got.shape[:2], dtype=bool)
            sees[:n, 2:] = (190 - n + np.arange(n) >= key)[:, None]
            assert np.isnan(got[sees]).all() and np.array_equal(got[~sees], clean[~sees]), (which, key)
    for bad in (np.nan, np.inf):
        q2 = q.copy()
        q2[n // 2, 1, 9] = bad
        got = call(q2, cache)
        assert np.isnan(got[n // 2, 1]).all()
        got[n // 2, 1] = clean[n // 2, 1]
        assert np.array_equal(got, clean)


def test_tables_that_name_no_page():
    rng = np.random.default_rng(8)
    D, page, Hq, Hkv, contexts, new = 64, 16, 2, 1, [140, 100, 140, 40], [20, 30, 20, 4]
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, A.F16)
    starts = _starts(new)
    q = _gpu(_draw(rng, (starts[-1], Hq, D), A.F16), A.F16)
    good = _np(api.kv4_attention_chunks(q, cache, _gpu(table), _ints(contexts), _ints(starts)))
    table[0, 1], table[2, 8] = -1, cache.shape[0]
    got = _np(api.kv4_attention_chunks(q, cache, _gpu(table), _ints([140, 100, 140, 16 * table.shape[1] + 1]), _ints(starts)))
    assert np.isnan(got[:20]).all() and np.array_equal(got[20:50], good[20:50]) and np.isnan(got[50 + 8:]).all()


def test_tables_that_name_no_page_few_rows():
    """The same where each wave of a block has keys of its own: a page that one wave meets, pages behind the context, a context longer than the table."""
    rng = np.random.default_rng(80)
    D, page, Hq, Hkv, contexts, new = 128, 16, 2, 1, [1400, 100, 140, 40], [3, 5, 16, 4]
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, A.F16)
    starts = _starts(new)
    q = _gpu(_draw(rng, (starts[-1], Hq, D), A.F16), A.F16)
    good = _np(api.kv4_attention_chunks(q, cache, _gpu(table), _ints(contexts), _ints(starts)))
    _check(good, _np(q), starts, contexts, keys, values, A.F16)
    for at in (0, 37, 87):
        wrong = table.copy()
        wrong[0, at], wrong[2, 8] = -1, cache.shape[0]
        got = _np(api.kv4_attention_chunks(q, cache, _gpu(wrong), _ints([1400, 100, 140, 16 * table.shape[1] + 1]), _ints(starts)))
        assert np.isnan(got[:3]).all() and np.array_equal(got[3:8], good[3:8]) and np.isnan(got[8 + 4:]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 60])
def test_rows_of_unlike_size(dtype, n):
    """One query that is 2^6 to 2^14 times the others of its block, and elements of a row as far apart: the others keep their own accuracy.  (Its own
    scores are thousands, which FP32 holds to 2^-12: it is left out.)"""
    rng = np.random.default_rng(n)
    c, Hq, Hkv, D = 300, 4, 2, 64
    cache, table, keys, values = _filled(rng, [c], 16, Hkv, D, dtype)
    for bits in (6, 8, 9, 14):
        q = _draw(rng, (n, Hq, D), dtype) * np.float32(2.0 ** (3 - bits))
        q[n // 2, 1] *= np.float32(2.0 ** bits)
        q[n // 3, 2, ::2] *= np.float32(2.0 ** -5)
        q = A.round_to(q, dtype)
        scale = 2.0 ** (bits - 6)
        got = _np(api.kv4_attention_chunks(_gpu(q, dtype), cache, _gpu(table), _ints([c]), _ints([0, n]), scale=scale))
        want, spread = A.attention(q, keys[0], values[0], scale, c - n + 1 + np.arange(n))
        assert np.isfinite(got[n // 2, 1]).all()
        got[n // 2, 1] = want[n // 2, 1]
        _close(got, want, spread, dtype, 2.0 ** -11, f"2^{bits}")


@pytest.mark.parametrize("scale", [0.0, -0.11, 1e-30, 3.0])
@pytest.mark.parametrize("dtype", TYPES)
def test_scales_of_any_sign(scale, dtype):
    rng = np.random.default_rng(23)
    c, Hq, Hkv, D, n = 170, 4, 2, 128, 70
    cache, table, keys, values = _filled(rng, [c], 16, Hkv, D, dtype)
    q = _draw(rng, (n, Hq, D), dtype)
    if scale == 3.0:
        q = A.round_to(q * np.float32(0.125), dtype)
    got = api.kv4_attention_chunks(_gpu(q, dtype), cache, _gpu(table), _ints([c]), _ints([0, n]), scale=scale)
    _check(_np(got), q, [0, n], [c], keys, values, dtype, scale=scale)


def test_starts_outside_the_tensor_are_cut_off():
    import torch

    rng = np.random.default_rng(13)
    D, page, Hq, Hkv = 64, 16, 2, 1
    cache, table, keys, values = _filled(rng, [50, 60], page, Hkv, D, A.F16)
    q = _draw(rng, (30, Hq, D), A.F16)
    out = torch.full((30, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    got = _np(api.kv4_attention_chunks(_gpu(q, A.F16), cache, _gpu(table), _ints([50, 60]), _ints([-5, 12, 2 ** 31 - 1]), out=out))
    _check(got, q, [0, 12, 30], [50, 60], keys, values, A.F16)
    got = _np(api.kv4_attention_chunks(_gpu(q, A.F16), cache, _gpu(table), _ints([50, 60]), _ints([20, 10, 15]), out=out.fill_(7.0)))
    assert (got[:10] == 7.0).all() and (got[15:] == 7.0).all()
    _check(got[10:15], q[10:15], [0, 5], [60], keys[1:], values[1:], A.F16)


def test_a_cache_of_more_than_4_gib():
    """Pages on both sides of 4 GiB, from a table that goes back and forth."""
    import torch

    rng = np.random.default_rng(15)
    D, page, Hkv, Hq = 128, 256, 8, 8
    pages = (5 << 30) // (page * (D + 8) * Hkv)
    cache = api.kv4_cache(pages, page, Hkv, D)
    used = np.array([pages - 1, 3, pages // 2, pages - 2, 0, pages * 4 // 5 + 1], dtype=np.int32)
    c, n = 6 * page - 20, 50
    j = np.arange(c)
    k, v = _draw(rng, (c, Hkv, D), A.F16), _draw(rng, (c, Hkv, D), A.F16)
    api.kv4_write(_gpu(k, A.F16), _gpu(v, A.F16), _ints(used[j // page].astype(np.int64) * page + j % page), cache)
    k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
    q = _draw(rng, (n, Hq, D), A.F16)
    got = _np(api.kv4_attention_chunks(_gpu(q, A.F16), cache, _gpu(used[None]), _ints([c]), _ints([0, n])))
    del cache
    torch.cuda.empty_cache()
    _check(got, q, [0, n], [c], [k], [v], A.F16)


@pytest.mark.parametrize("many", [False, True])
def test_a_graph_follows_contexts_and_starts(many):
    """Captured with one batch and replayed with others, the allocator and other calls at work between the replays; two graphs that share a stream's
    workspace; and on a stream given as a number."""
    import torch

    D, page, width, Hq, Hkv, T = 64, 16, 40, 8, 2, 1200 if many else 60
    n = 80 if many else 5
    rng = np.random.default_rng(31)
    cache, table, _, _ = _filled(rng, [page * width] * n, page, Hkv, D, A.F16, garbage=False, spare=0)
    table, ctx, starts = _gpu(table), torch.ones(n, dtype=torch.int32, device="cuda"), torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    q = _gpu(_draw(rng, (T, Hq, D), A.F16), A.F16)
    step = lambda **a: api.kv4_attention_chunks(q, cache, table, ctx, starts, **a)  # noqa: E731
    side, graphs, captured = torch.cuda.Stream(), [], []
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            captured.append(step())
    for i in range(5):
        cuts = np.sort(rng.integers(0, T + 1, n - 1))
        new = np.diff(np.concatenate(([0], cuts, [T])))
        starts.copy_(_gpu(_starts(new)))
        ctx.copy_(_ints(np.minimum(new + rng.integers(0, 200, n), page * width)))
        torch.randn(1 << 20, device="cuda").sum().item()
        for g, c in zip(graphs, captured):
            c.fill_(float("nan"))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        want = step()
        assert torch.isfinite(want).all() and all(torch.equal(c, want) for c in captured)
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    there = step(stream=other.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(there, want)


def test_heads_and_tokens_that_share_their_queries():
    """Strides of zero: one query for all tokens, one for all heads."""
    rng = np.random.default_rng(16)
    D, Hq, Hkv, c, n = 128, 4, 2, 100, 37
    cache, table, keys, values = _filled(rng, [c], 16, Hkv, D, A.F16)
    q = _draw(rng, (n, Hq, D), A.F16)
    for shared in (q[:1].repeat(n, 0), q[:, :1].repeat(Hq, 1)):
        view = _gpu(q[:1], A.F16).expand(n, Hq, D) if shared is not None and (shared[0] == shared[-1]).all() else _gpu(q[:, :1], A.F16).expand(n, Hq, D)
        got = api.kv4_attention_chunks(view, cache, _gpu(table), _ints([c]), _ints([0, n]))
        _check(_np(got), shared, [0, n], [c], keys, values, A.F16)


def test_refusals():
    import torch

    q = torch.zeros((6, 4, 128), dtype=torch.float16, device="cuda")
    cache, pages, ctx, starts = api.kv4_cache(2, 16, 2, 128), torch.zeros((2, 2), dtype=torch.int32, device="cuda"), _ints([3, 3]), _ints([0, 3, 6])
    call = lambda **a: api.kv4_attention_chunks(*(a.get(n, d) for n, d in zip(("q", "cache", "pages", "ctx", "starts"), (q, cache, pages, ctx, starts))),  # noqa: E731
                                                **{n: v for n, v in a.items() if n not in ("q", "cache", "pages", "ctx", "starts")})
    call()
    for bad, error in [
            (dict(q=q.float()), TypeError), (dict(q=q.cpu()), TypeError), (dict(q=q[0]), ValueError), (dict(q=q[..., :64]), ValueError), (dict(q=q[:, :3]), api.LiquidGemmError),
            (dict(q=q.transpose(1, 2)), ValueError), (dict(cache=cache[:, :, :-16].contiguous()), ValueError), (dict(pages=pages[:1]), ValueError), (dict(pages=pages[:, :0]), api.LiquidGemmError),
            (dict(pages=pages.long()), TypeError), (dict(ctx=ctx[:1]), ValueError), (dict(ctx=ctx.long()), TypeError), (dict(starts=starts[:0]), ValueError),
            (dict(starts=starts.long()), TypeError), (dict(starts=starts[:2]), ValueError), (dict(scale=float("nan")), api.LiquidGemmError), (dict(out=q.bfloat16()), TypeError),
            (dict(out=q[:5]), ValueError), (dict(q=torch.zeros(6 * 4 * 128 + 1, dtype=torch.float16, device="cuda")[1:].view(6, 4, 128)), api.LiquidGemmError),
            (dict(q=torch.zeros((6, 4, 132), dtype=torch.float16, device="cuda")[..., :128]), api.LiquidGemmError), (dict(q=q.clone().requires_grad_()), ValueError)]:
        with pytest.raises(error):
            call(**bad)
    assert call(q=q[:0], starts=_ints([0, 0, 0])).shape == (0, 4, 128)
    assert call(q=q[:0], pages=pages[:0], ctx=ctx[:0], starts=_ints([0])).shape == (0, 4, 128)


def test_through_the_native_module_and_without(monkeypatch):
    import torch

    rng = np.random.default_rng(3)
    cache, table, _, _ = _filled(rng, [40, 300], 16, 2, 128, A.F16)
    q = _gpu(_draw(rng, (25, 4, 128), A.F16), A.F16)
    call = lambda: api.kv4_attention_chunks(q, cache, _gpu(table), _ints([40, 300]), _ints([0, 20, 25]))  # noqa: E731
    native, answers = api._native, []
    want = call()  # (makes this stream's workspace)

    class Watched:
        @staticmethod
        def chunks(*a):
            answers.append(native.chunks(*a))
            return answers[-1]

    class Nothing:
        chunks = staticmethod(lambda *a: None)

    for stands_in in (Watched, Nothing):
        monkeypatch.setattr(api, "_native", stands_in)
        assert torch.equal(call(), want)
    assert len(answers) == 1 and answers[0] is not None


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(8, 1), (8, 8)])
def test_fp16_results_of_few_rows_have_their_own_rounding_alone(D, Hq, Hkv):
    """Tiles of up to 32 rows multiply the weights as two FP16 numbers each where the result is FP16, as kv4_attention does.

    Queries are small whole numbers, so that the products with the codes and their sums are exact; a score (below 16) times its scale and the logarithm of the value's scale are off
    by 2^-19 at most, the second number of a weight leaves 2^-22 of it, sums of 60 terms in FP32 are off by 2^-18 of the terms: together below 2^-16 of sum_j p_j |v_j|.  Beside that, the
    matrix cores cut the products that they add up, of eight keys at a time, below 2^-24 of the largest, and a subnormal number counts as 2^-14 in that.  A weight's product with a code
    difference, which is the difference times 2^-24 in the even places of a dword (times 2^-20 in the odd ones), so loses up to 2^(24 - 14 - 24) = 2^-14 of the largest weight times its value's scale
    among the eight keys; these lie in sixteen consecutive ones, the rests of the weights lose 2^-11 of that.  Hence 16 * 2^-14 of the largest p_j s_j of every sixteen keys."""
    rng = np.random.default_rng(D + Hkv)
    new, contexts, page = [1, 2, 1, 4, 1, 3], [2, 5, 17, 33, 60, 3], 16
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, A.F16)
    starts = _starts(new)
    q = rng.integers(-2, 3, (starts[-1], Hq, D)).astype(np.float32)
    args = (cache, _gpu(table), _ints(contexts))
    got = _np(api.kv4_attention_chunks(_gpu(q, A.F16), *args, _ints(starts)))
    for s, c in enumerate(contexts):
        mine, limit = slice(starts[s], starts[s + 1]), c - new[s] + 1 + np.arange(new[s])
        want, spread = A.attention(q[mine], keys[s], values[s], D ** -0.5, limit)
        k, v = (np.repeat(x.astype(np.float64), Hq // Hkv, 1) for x in (keys[s], values[s]))
        scores = np.einsum("nhd,khd->nhk", q[mine].astype(np.float64), k) * D ** -0.5
        scores = np.where(np.arange(c) < limit[:, None, None], scores, -np.inf)
        p = np.exp(scores - scores.max(-1, keepdims=True))
        step = np.stack([[np.diff(np.unique(x)).min(initial=np.inf) for x in row] for row in v])                 # [keys, heads]: numbers are whole multiples of the scale apart
        step = np.where(np.isfinite(step), step, 0.0)
        weighed = p / p.sum(-1, keepdims=True) * step.T
        weighed = np.pad(weighed, ((0, 0), (0, 0), (0, -c % 16))).reshape(*p.shape[:2], -1, 16).max(-1).sum(-1)
        tol = 1.1 * (A.UNIT[A.F16] * np.abs(want) + 2.0 ** -16 * spread) + 2.0 ** -24 + 16 * 2.0 ** -14 * 1.001 * weighed[..., None]
        err = np.abs(got[mine] - want)
        assert (err <= tol).all(), f"sequence {s}: {new[s]} of {c}: {np.sum(err > tol)} of {err.size}, worst {np.max(err / tol):.2f} times the tolerance"
