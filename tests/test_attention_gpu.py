"""Rotary positions, the 4-bit cache and the attention kernels against their definitions (oracle/attention_oracle.py, FP64).

Tolerances: a result is rounded once to its type (relative error u = 2^-11 in FP16, 2^-8 in BF16), and the attention kernels
round each weight once before the second product (w = 2^-11, prompts in BF16: 2^-8), which moves the result by at most w * sum_j p_j |v_j|;
everything else is FP32 (below 2^-16 of that).  Hence |error| <= 1.1 (u |o| + w sum_j p_j |v_j|) + 2^-24."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from paper_2509_01229_amd import api

pytestmark = pytest.mark.gpu
TYPES = (A.F16, A.BF16)


def _draw(rng, shape, dtype, outliers=False):
    x = rng.standard_normal(shape, dtype=np.float32)
    if outliers:
        x *= np.exp(0.5 * rng.standard_normal(shape[1:], dtype=np.float32))
    return A.round_to(x, dtype)


def _gpu(x, dtype=None):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to(getattr(torch, dtype)) if dtype else t


def _np(t):
    return t.float().cpu().numpy()


def _views(x, dtype, pad=0):
    """The arrays side by side as views of one matrix, `pad` heads of NaN behind them."""
    import torch

    parts = [_gpu(a, dtype) for a in x]
    parts.append(torch.full((x[0].shape[0], pad, x[0].shape[2]), float("nan"), dtype=parts[0].dtype, device="cuda"))
    return torch.cat(parts, 1).split([p.shape[1] for p in parts], 1)[:-1]


def _close(got, want, spread, dtype, weights, what=""):
    tol = 1.1 * (A.UNIT[dtype] * np.abs(want) + weights * spread) + 2.0 ** -24
    err = np.abs(got.astype(np.float64) - want)
    assert np.isfinite(got).all(), f"{what}: not finite"
    assert (err <= tol).all(), f"{what}: {np.sum(err > tol)} of {err.size} off, worst {np.max(err / tol):.2f} times the tolerance"


# ------------------------------------------------------------------------------ norm and rotation
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 48)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv", [(1, 4, 1), (37, 7, 3)])
def test_rotation_is_exact(dtype, D, rot, interleaved, T, Hq, Hkv):
    rng = np.random.default_rng(D + rot + T)
    q, k = _draw(rng, (T, Hq, D), dtype), _draw(rng, (T, Hkv, D), dtype)
    table = A.rope_table(300, rot).astype(np.float32)
    pos = rng.integers(0, 300, T).astype(np.int32)
    dq, dk = _views((q, k), dtype, pad=2)
    got = api.attn_qk_norm_rope(dq, dk, _gpu(pos), _gpu(table), interleaved=interleaved)
    for g, x in zip(got, (q, k)):
        assert g.is_contiguous()
        want = A.round_to(A.rope(x, pos, table, interleaved), dtype)
        assert np.array_equal(_np(g), want)
    # in place, on views
    again = api.attn_qk_norm_rope(dq, dk, _gpu(pos), _gpu(table), interleaved=interleaved, out_q=dq, out_k=dk)
    assert again[0] is dq and again[1] is dk
    assert all(np.array_equal(_np(a), _np(g)) for a, g in zip(again, got))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,rot,interleaved", [(128, 128, False), (128, 32, True), (64, 64, False)])
def test_norm(dtype, D, rot, interleaved):
    rng = np.random.default_rng(D)
    T, Hq, Hkv, eps = 53, 5, 2, 1e-5
    q, k = _draw(rng, (T, Hq, D), dtype, True), A.round_to(_draw(rng, (T, Hkv, D), dtype) * np.float32(2.0 ** -6), dtype)
    q[3] = 0
    table = A.rope_table(99, rot).astype(np.float32)
    pos = rng.integers(0, 99, T).astype(np.int32)
    for qw, kw in ((True, True), (True, False), (False, True)):
        w = [rng.standard_normal(D).astype(np.float32) if use else None for use in (qw, kw)]
        got = api.attn_qk_norm_rope(_gpu(q, dtype), _gpu(k, dtype), _gpu(pos), _gpu(table), interleaved=interleaved, eps=eps,
                                    q_norm=None if w[0] is None else _gpu(w[0]), k_norm=None if w[1] is None else _gpu(w[1]))
        for g, x, wx in zip(got, (q, k), w):
            want = A.rope(x, pos, table, interleaved, wx, eps, np.float64)
            size = np.abs(want) + 2.0 ** -12 * np.abs(want).max(-1, keepdims=True)  # (FP32 sums of two products may cancel)
            assert (np.abs(_np(g) - want) <= 1.01 * A.UNIT[dtype] * size + 2.0 ** -24).all()


def test_positions_outside_the_table_give_nan():
    rng = np.random.default_rng(0)
    q, k = _draw(rng, (4, 2, 128), A.F16), _draw(rng, (4, 1, 128), A.F16)
    table = A.rope_table(10, 64).astype(np.float32)
    pos = np.array([0, -1, 10, 9], dtype=np.int32)
    for y, x in zip(api.attn_qk_norm_rope(_gpu(q, A.F16), _gpu(k, A.F16), _gpu(pos), _gpu(table)), (q, k)):
        y = _np(y)
        assert np.isfinite(y[[0, 3]]).all() and np.isnan(y[1:3, :, :64]).all() and np.array_equal(y[1:3, :, 64:], x[1:3, :, 64:])


# ---------------------------------------------------------------------------------------- the cache
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page,T,Hkv", [(16, 45, 3), (64, 1, 1), (256, 70, 2)])
def test_cache_bytes(dtype, D, page, T, Hkv):
    import torch

    rng = np.random.default_rng(page + T + D)
    k, v = _draw(rng, (T, Hkv, D), dtype, True), _draw(rng, (T, Hkv, D), dtype)
    if T > 8:
        k[0] = 0                                        # nothing to hold
        k[1] = np.abs(k[1]) + 1                         # no negative element: zero point 0
        v[2] = -np.abs(v[2]) - 1
        v[3] = v[3, :, :1]                              # constant
        k[4] = A.round_to(np.arange(D) % 31 * 0.5 - 4.0, dtype)  # ties
        v[5] *= np.float32(2.0 ** (-14 if dtype == A.F16 else -110))   # subnormal numbers; scales at their smallest
        v[6] *= np.float32(2.0 ** (13 if dtype == A.F16 else 120))
        k, v = A.round_to(k, dtype), A.round_to(v, dtype)
    pages = 5
    slots = rng.permutation(pages * page)[:T].astype(np.int32)
    if T > 8:
        slots[7], slots[8] = -1, pages * page           # not stored
    before = rng.integers(0, 256, (pages, Hkv, page * (D + 8)), dtype=np.uint8)
    want = before.copy()
    A.write(want, page, slots, k, v)
    cache = _gpu(before)
    dk, dv = _views((k, v), dtype, pad=1)
    assert api.kv4_write(dk, dv, _gpu(slots), cache) is cache
    assert np.array_equal(cache.cpu().numpy(), want)
    # and read back
    for out in (A.F16, A.BF16):
        got = api.kv4_read(cache, _gpu(slots), dtype=getattr(torch, out))
        for g, x in zip(got, (k, v)):
            values = A.round_to(A.dequantise(*A.quantise(x)), out)
            values[(slots < 0) | (slots >= pages * page)] = 0
            assert np.array_equal(_np(g), values)


def test_vectors_that_are_not_finite_read_back_as_nan():
    rng = np.random.default_rng(3)
    k, v = _draw(rng, (4, 2, 128), A.BF16), _draw(rng, (4, 2, 128), A.BF16)
    k[0, 0, 5], k[1, 1, 127], v[2, 0, 0], v[3, 1, 9] = np.nan, np.inf, -np.inf, np.nan
    v[1, 0, :2] = 3e38, -3e38
    k, v = A.round_to(k, A.BF16), A.round_to(v, A.BF16)
    cache = api.kv4_cache(1, 16, 2, 128)
    slots = _gpu(np.arange(4, dtype=np.int32))
    api.kv4_write(_gpu(k, A.BF16), _gpu(v, A.BF16), slots, cache)
    for got, x, bad in zip(api.kv4_read(cache, slots), (k, v), ({(0, 0), (1, 1)}, {(2, 0), (3, 1), (1, 0)})):
        got = _np(got)
        for t in range(4):
            for h in range(2):
                assert np.isnan(got[t, h]).all() if (t, h) in bad else np.isfinite(got[t, h]).all(), (t, h)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,rot,interleaved,norm", [(128, 128, False, False), (64, 32, True, True), (128, 64, False, True)])
def test_append_is_rotation_and_write(dtype, D, rot, interleaved, norm):
    rng = np.random.default_rng(rot)
    T, Hq, Hkv, page = 21, 6, 2, 32
    q, k, v = (_draw(rng, (T, h, D), dtype, True) for h in (Hq, Hkv, Hkv))
    pos, slots = rng.integers(0, 50, T).astype(np.int32), rng.permutation(4 * page)[:T].astype(np.int32)
    slots[4] = -5
    table = _gpu(A.rope_table(50, rot).astype(np.float32))
    w = {n: _gpu(rng.standard_normal(D).astype(np.float32)) for n in ("q_norm", "k_norm")} if norm else {}
    dq, dk, dv = _views((q, k, v), dtype)
    two, one = api.kv4_cache(4, page, Hkv, D), api.kv4_cache(4, page, Hkv, D)
    turned_q, turned_k = api.attn_qk_norm_rope(dq, dk, _gpu(pos), table, interleaved=interleaved, **w)
    api.kv4_write(turned_k, dv, _gpu(slots), two)
    got = api.kv4_append(dq, dk, dv, _gpu(pos), table, _gpu(slots), one, interleaved=interleaved, **w)
    assert np.array_equal(_np(got), _np(turned_q)) and np.array_equal(one.cpu().numpy(), two.cpu().numpy())
    assert one.any()


# -------------------------------------------------------------------------- attention over the cache
def _filled(rng, contexts, page, Hkv, D, dtype, garbage=True, spare=3):
    """A cache with pages in any order, what no token holds filled with bytes whose words are NaN; its table, and the keys and values."""
    need = [-(-c // page) for c in contexts]
    order = rng.permutation(sum(need) + spare).astype(np.int32)
    cache = api.kv4_cache(sum(need) + spare, page, Hkv, D)
    if garbage:
        cache.fill_(255)
    table = np.full((len(contexts), max(max(need), 1)), 2 ** 31 - 1, dtype=np.int32)  # (places that are not read)
    keys, values, at = [], [], 0
    for b, c in enumerate(contexts):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        k, v = _draw(rng, (c, Hkv, D), dtype, True), _draw(rng, (c, Hkv, D), dtype)
        if c:
            j = np.arange(c)
            slots = (table[b, j // page] * page + j % page).astype(np.int32)
            api.kv4_write(_gpu(k, dtype), _gpu(v, dtype), _gpu(slots), cache)
            k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
        keys.append(k)
        values.append(v)
    return cache, table, keys, values


DECODE = [
    # contexts, page, Hq, Hkv, new tokens
    ([1], 16, 1, 1, 1),
    ([517], 64, 4, 4, 1),
    ([0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 0], 16, 8, 2, 1),
    ([63, 64, 65, 1000, 2], 32, 16, 2, 1),
    ([300, 77, 5, 0, 3], 64, 16, 2, 4),            # 32 rows; contexts shorter than the new tokens
    ([200, 129], 128, 28, 4, 7),                   # 49 rows, groups of 7
    ([257, 4097], 256, 24, 1, 3),                  # 72 rows of one kv head
    ([9000], 16, 8, 1, 1),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_attention_over_the_cache(dtype, D, case):
    contexts, page, Hq, Hkv, new = DECODE[case]
    rng = np.random.default_rng(case)
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
    q = _draw(rng, (len(contexts) * new, Hq, D), dtype) * np.float32(2.0)
    dq = _views((q,), dtype, pad=2)[0].unflatten(0, (len(contexts), new))
    assert dq.shape[0] * new == 1 or not dq.is_contiguous()
    got = api.kv4_attention(dq, cache, _gpu(table), _gpu(np.array(contexts, dtype=np.int32)))
    got = _np(got)
    for b, c in enumerate(contexts):
        want, spread = A.attention(q[b * new:(b + 1) * new], keys[b], values[b], D ** -0.5, c - new + 1 + np.arange(new))
        _close(got[b], want, spread, dtype, 2.0 ** -11, f"sequence {b} of {c}")
    if new == 1:  # the form without the dimension of new tokens, a scale of its own, a given output
        import torch

        out = torch.empty((len(contexts), Hq, D), dtype=dq.dtype, device="cuda")
        assert api.kv4_attention(dq[:, 0], cache, _gpu(table), _gpu(np.array(contexts, dtype=np.int32)), scale=0.3, out=out) is out
        want, spread = A.attention(q[:1], keys[0], values[0], 0.3, [contexts[0]])
        _close(_np(out)[:1], want, spread, dtype, 2.0 ** -11)


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_weights_of_all_sizes(dtype):
    """Scores far apart, in rising and falling order (the running maximum moves often, or never), and values whose scales differ by
    2^20 (FP16: 2^12) from token to token."""
    rng = np.random.default_rng(5)
    D, page, Hq, Hkv, c = 128, 32, 4, 2, 700
    for order in (1, -1):
        q = _draw(rng, (1, Hq, D), dtype)
        k = rng.standard_normal((c, Hkv, D)).astype(np.float32) * 0.1
        k += np.linspace(-1, 1, c, dtype=np.float32)[::order, None, None] * q[:1, ::2] * np.float32(3)
        v = rng.standard_normal((c, Hkv, D)).astype(np.float32) * np.exp2(rng.integers(-6 if dtype == A.F16 else -10, 7 if dtype == A.F16 else 11, (c, 1, 1))).astype(np.float32)
        k, v = A.round_to(k, dtype), A.round_to(v, dtype)
        cache = api.kv4_cache(22, page, Hkv, D)
        slots = np.arange(c, dtype=np.int32)
        api.kv4_write(_gpu(k, dtype), _gpu(v, dtype), _gpu(slots), cache)
        got = api.kv4_attention(_gpu(q, dtype), cache, _gpu(np.arange(22, dtype=np.int32)[None]), _gpu(np.array([c], dtype=np.int32)))
        k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
        want, spread = A.attention(q, k, v, D ** -0.5, [c])
        _close(_np(got), want, spread, dtype, 2.0 ** -11)


def test_attention_values_near_the_end_of_bf16():
    rng = np.random.default_rng(6)
    D, page, c = 64, 16, 40
    q, k = _draw(rng, (1, 2, D), A.BF16), _draw(rng, (c, 1, D), A.BF16)
    for size in (2.0 ** 126, 2.0 ** -110):
        v = A.round_to(_draw(rng, (c, 1, D), A.BF16).clip(-1.5, 1.5) * np.float32(size), A.BF16)
        big = A.round_to(q * np.float32(2.0 ** 100), A.BF16)
        cache = api.kv4_cache(3, page, 1, D)
        api.kv4_write(_gpu(k, A.BF16), _gpu(v, A.BF16), _gpu(np.arange(c, dtype=np.int32)), cache)
        got = api.kv4_attention(_gpu(big, A.BF16), cache, _gpu(np.arange(3, dtype=np.int32)[None]), _gpu(np.array([c], dtype=np.int32)), scale=2.0 ** -103)
        kk, vv = (A.dequantise(*A.quantise(x)) for x in (k, v))
        want, spread = A.attention(big, kk, vv, 2.0 ** -103, [c])
        got = got.double().cpu().numpy()
        assert (np.abs(got - want) <= 1.1 * (A.UNIT[A.BF16] * np.abs(want) + 2.0 ** -11 * spread)).all()


def test_attention_nan_stays_with_those_that_see_it():
    rng = np.random.default_rng(7)
    D, page, Hq, Hkv, contexts, new = 128, 16, 4, 2, [90, 60], 3
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, A.F16)
    q = _draw(rng, (2 * new, Hq, D), A.F16)
    ctx = _gpu(np.array(contexts, dtype=np.int32))
    clean = _np(api.kv4_attention(_gpu(q, A.F16).unflatten(0, (2, new)), cache, _gpu(table), ctx))
    for which in (0, 1):  # a key, a value of sequence 0, kv head 1, the one before the last token
        spoilt = cache.clone()
        at = page * D + which * 4 * page + 4 * (88 % page)
        spoilt[int(table[0, 88 // page]), 1, at:at + 4] = _gpu(np.array([0x7FC00000], dtype="<u4").view(np.uint8))
        got = _np(api.kv4_attention(_gpu(q, A.F16).unflatten(0, (2, new)), spoilt, _gpu(table), ctx))
        sees = np.zeros((2, new, Hq), dtype=bool)
        sees[0, 1:, 2:] = True
        assert np.isnan(got[sees]).all() and np.array_equal(got[~sees], clean[~sees])


def test_attention_tables_that_name_no_page():
    rng = np.random.default_rng(8)
    D, page, Hq, Hkv, contexts = 64, 16, 2, 1, [40, 100, 40, 40]
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, A.F16)
    q = _gpu(_draw(rng, (4, Hq, D), A.F16), A.F16)
    good = _np(api.kv4_attention(q, cache, _gpu(table), _gpu(np.array(contexts, dtype=np.int32))))
    table[0, 1], table[2, 2] = -1, cache.shape[0]
    got = _np(api.kv4_attention(q, cache, _gpu(table), _gpu(np.array([40, 100, 40, 16 * table.shape[1] + 1], dtype=np.int32))))
    assert np.isnan(got[[0, 2, 3]]).all() and np.array_equal(got[1], good[1])


# ------------------------------------------------------------------------------ attention of prompts
PROMPT = [
    # (queries, keys) of the sequences, Hq, Hkv
    ([(1, 1)], 1, 1),
    ([(64, 64), (1, 1), (65, 65), (63, 63)], 2, 2),
    ([(128, 128), (129, 129), (300, 300), (0, 0), (31, 31)], 4, 2),
    ([(33, 500), (200, 263), (1, 700), (128, 129)], 4, 1),      # chunks behind what came before
    ([(50, 20), (0, 30), (40, 0), (3, 3)], 6, 2),               # rows without keys, sequences without queries or keys
    ([(513, 513), (97, 1000)], 7, 1),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_prompts(dtype, D, causal, case):
    lens, Hq, Hkv = PROMPT[case]
    rng = np.random.default_rng(case)
    sq, sk = (np.concatenate(([0], np.cumsum([x[i] for x in lens]))).astype(np.int32) for i in (0, 1))
    q, k, v = _draw(rng, (sq[-1], Hq, D), dtype) * np.float32(2.0), _draw(rng, (sk[-1], Hkv, D), dtype, True), _draw(rng, (sk[-1], Hkv, D), dtype)
    dq = _views((q,), dtype, pad=1)[0]
    dk, dv = _views((k, v), dtype, pad=3)
    got = api.attn_prompt(dq, dk, dv, _gpu(sq), _gpu(sk), causal=causal)
    assert got.is_contiguous()
    got = _np(got)
    for s, (a, b) in enumerate(lens):
        limits = np.arange(a) + b - a + 1 if causal else np.full(a, b)
        want, spread = A.attention(q[sq[s]:sq[s + 1]], k[sk[s]:sk[s + 1]], v[sk[s]:sk[s + 1]], D ** -0.5, limits)
        _close(got[sq[s]:sq[s + 1]], want, spread, dtype, A.UNIT[dtype], f"sequence {s}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_prompts_masked_keys_and_values_do_not_matter(dtype, D, bad):
    """Keys and values that are not finite: rows that do not see them are as they were, those that see them are not finite."""
    rng = np.random.default_rng(11)
    n, Hq, Hkv = 200, 2, 1
    q, k, v = (_draw(rng, (n + 40, h, D), dtype) for h in (Hq, Hkv, Hkv))
    starts = _gpu(np.array([0, n, n + 40], dtype=np.int32))
    clean = _np(api.attn_prompt(_gpu(q, dtype), _gpu(k, dtype), _gpu(v, dtype), starts))
    for j in (0, 63, 64, 100, 127, 130, 199, n + 3):
        for which in ("k", "v"):
            kv = {"k": k.copy(), "v": v.copy()}
            kv[which][j, 0, 7] = bad
            got = _np(api.attn_prompt(_gpu(q, dtype), _gpu(kv["k"], dtype), _gpu(kv["v"], dtype), starts))
            i = np.arange(n + 40)
            sees = (i >= j) & ((i < n) == (j < n))
            assert np.array_equal(got[~sees], clean[~sees]), (j, which)
            if which == "v":
                assert not np.isfinite(got[sees][..., 7]).any(), j
                assert np.array_equal(np.delete(got[sees], 7, -1), np.delete(clean[sees], 7, -1)), j
            elif np.isnan(bad):
                assert np.isnan(got[sees]).all(), j


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_few_queries_over_many_keys(dtype, D):
    """Keys split over blocks and joined: with a workspace, without one (one block a tile), twice on the same tickets; a value
    that is not finite in a part that some rows do not see."""
    import torch

    rng = np.random.default_rng(17)
    lens, Hq, Hkv = [(70, 4000), (130, 2500), (1, 3000), (5, 3)], 3, 1
    sq, sk = (np.concatenate(([0], np.cumsum([x[i] for x in lens]))).astype(np.int32) for i in (0, 1))
    q, k, v = _draw(rng, (sq[-1], Hq, D), dtype) * np.float32(2.0), _draw(rng, (sk[-1], Hkv, D), dtype, True), _draw(rng, (sk[-1], Hkv, D), dtype)
    args = [_gpu(x, dtype) for x in (q, k, v)] + [_gpu(sq), _gpu(sk)]
    need = int(api.lib().attn_prompt_workspace_size(len(lens), int(sq[-1]), int(sk[-1]), Hq, Hkv, D))
    assert need > 32768
    for causal in (True, False):
        ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
        ws[32768:] = 255  # (what it holds does not matter)
        got = api.attn_prompt(*args, causal=causal, workspace=ws)
        assert torch.equal(got, api.attn_prompt(*args, causal=causal, workspace=ws)) and torch.equal(got, api.attn_prompt(*args, causal=causal))
        assert not ws[:32768].any()
        for g in (got, api.attn_prompt(*args, causal=causal, workspace=ws[:16])):
            for s, (a, b) in enumerate(lens):
                limits = np.arange(a) + b - a + 1 if causal else np.full(a, b)
                want, spread = A.attention(q[sq[s]:sq[s + 1]], k[sk[s]:sk[s + 1]], v[sk[s]:sk[s + 1]], D ** -0.5, limits)
                _close(_np(g)[sq[s]:sq[s + 1]], want, spread, dtype, A.UNIT[dtype], f"sequence {s}")
    clean = _np(api.attn_prompt(*args))
    args[2][3980, 0, 5] = float("nan")  # (queries 50 .. of the first sequence see it)
    got = _np(api.attn_prompt(*args))
    assert np.isnan(got[50:70, :, 5]).all()
    got[50:70, :, 5] = clean[50:70, :, 5]
    assert np.array_equal(got, clean)


@pytest.mark.parametrize("n,longest", [(65, 40), (150, 90), (4500, 3)])
def test_prompts_many_sequences(n, longest):
    """More sequences than a wave has lanes, empty ones among them, a long one, and rows before the first and behind the last that
    are nobody's."""
    rng = np.random.default_rng(n)
    D, Hq, Hkv, dtype = 64, 6, 2, A.F16
    lens_q, lens_k = rng.integers(0, longest + 1, n), rng.integers(0, longest + 1, n)
    lens_q[n // 2], lens_k[n // 2], lens_k[n - 1] = 300, 333, 200
    sq, sk = (np.concatenate(([at], at + np.cumsum(x))).astype(np.int32) for at, x in ((5, lens_q), (3, lens_k)))
    q, k, v = _draw(rng, (sq[-1] + 9, Hq, D), dtype), _draw(rng, (sk[-1] + 2, Hkv, D), dtype, True), _draw(rng, (sk[-1] + 2, Hkv, D), dtype)
    import torch

    args = [_gpu(x, dtype) for x in (q, k, v)] + [_gpu(sq), _gpu(sk)]
    for causal in (True, False):
        out = torch.full_like(args[0], 7.0)
        got = _np(api.attn_prompt(*args, causal=causal, out=out))
        assert (got[:5] == 7.0).all() and (got[sq[-1]:] == 7.0).all()
        for s in range(n):
            a, b = int(lens_q[s]), int(lens_k[s])
            if not a:
                continue
            limits = np.arange(a) + b - a + 1 if causal else np.full(a, b)
            want, spread = A.attention(q[sq[s]:sq[s + 1]], k[sk[s]:sk[s + 1]], v[sk[s]:sk[s + 1]], D ** -0.5, limits)
            _close(got[sq[s]:sq[s + 1]], want, spread, dtype, A.UNIT[dtype], f"sequence {s}")


def test_prompts_scores_far_apart():
    rng = np.random.default_rng(12)
    n, D = 400, 128
    for order in (1, -1):
        q, k, v = (_draw(rng, (n, 1, D), A.F16) for _ in range(3))
        k += q[:1] * np.linspace(-4, 4, n, dtype=np.float32)[::order, None, None]
        q = A.round_to(q * 0.2 + q[:1], A.F16)
        k = A.round_to(k, A.F16)
        starts = _gpu(np.array([0, n], dtype=np.int32))
        got = _np(api.attn_prompt(_gpu(q, A.F16), _gpu(k, A.F16), _gpu(v, A.F16), starts, scale=0.2))
        want, spread = A.attention(q, k, v, 0.2, np.arange(n) + 1)
        _close(got, want, spread, A.F16, A.UNIT[A.F16])


def test_prompt_starts_outside_the_tensors_are_cut_off():
    rng = np.random.default_rng(13)
    q, k, v = (_draw(rng, (100, 2, 64), A.F16) for _ in range(3))
    d = [_gpu(x, A.F16) for x in (q, k, v)]
    import torch

    out = torch.full_like(d[0], 7.0)
    api.attn_prompt(*d, _gpu(np.array([-5, 30, 1000], dtype=np.int32)), out=out)
    for a, b in ((0, 30), (30, 100)):
        want, spread = A.attention(q[a:b], k[a:b], v[a:b], 64 ** -0.5, np.arange(b - a) + 1)
        _close(_np(out)[a:b], want, spread, A.F16, A.UNIT[A.F16])
    out.fill_(7.0)
    api.attn_prompt(*d, _gpu(np.array([40, 60], dtype=np.int32)), out=out)  # rows of no sequence
    assert (out[:40] == 7).all() and (out[60:] == 7).all() and not (out[40:60] == 7).all()


def test_a_cache_of_more_than_4_gib():
    """Pages whose places pass 32 bits: written, read back and attended to."""
    import torch

    rng = np.random.default_rng(20)
    D, page, Hkv, Hq, pages, c = 128, 256, 8, 16, 16000, 900
    cache = torch.empty((pages, Hkv, page * (D + 8)), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    table = np.array([[15999, 3, 15500, 15421]], dtype=np.int32)  # (15421 * 278528 just above 2^32)
    j = np.arange(c)
    slots = (table[0, j // page] * page + j % page).astype(np.int32)
    k, v, q = _draw(rng, (c, Hkv, D), A.F16, True), _draw(rng, (c, Hkv, D), A.F16), _draw(rng, (1, Hq, D), A.F16)
    api.kv4_write(_gpu(k, A.F16), _gpu(v, A.F16), _gpu(slots), cache)
    k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
    for got, x in zip(api.kv4_read(cache, _gpu(slots)), (k, v)):
        assert np.array_equal(_np(got), A.round_to(x, A.F16))
    got = api.kv4_attention(_gpu(q, A.F16), cache, _gpu(table), _gpu(np.array([c], dtype=np.int32)))
    want, spread = A.attention(q, k, v, D ** -0.5, [c])
    _close(_np(got), want, spread, A.F16, 2.0 ** -11)


def test_keys_and_values_that_heads_or_tokens_share():
    """Strides of zero: heads that are one head expanded, tokens that are one token."""
    rng = np.random.default_rng(21)
    n, Hq, Hkv, D = 150, 4, 2, 64
    q, k, v = _draw(rng, (n, Hq, D), A.BF16), _draw(rng, (n, 1, D), A.BF16), _draw(rng, (1, Hkv, D), A.BF16)
    starts = _gpu(np.array([0, n], dtype=np.int32))
    dk, dv = _gpu(k, A.BF16).expand(n, Hkv, D), _gpu(v, A.BF16).expand(n, Hkv, D)
    got = _np(api.attn_prompt(_gpu(q, A.BF16), dk, dv, starts))
    assert np.array_equal(got, _np(api.attn_prompt(_gpu(q, A.BF16), dk.contiguous(), dv.contiguous(), starts)))
    want, spread = A.attention(q, np.repeat(k, Hkv, 1), np.repeat(v, n, 0), D ** -0.5, np.arange(n) + 1)
    _close(got, want, spread, A.BF16, A.UNIT[A.BF16])
    one, two = api.kv4_cache(10, 16, Hkv, D), api.kv4_cache(10, 16, Hkv, D)
    slots = _gpu(np.arange(n, dtype=np.int32))
    assert np.array_equal(api.kv4_write(dk, dv, slots, one).cpu().numpy(), api.kv4_write(dk.contiguous(), dv.contiguous(), slots, two).cpu().numpy())


def test_attention_of_many_sequences():
    """More sequences than a wave has lanes, of all lengths, empty ones among them; the same without a workspace, bit for bit where
    an item is not split."""
    import torch

    rng = np.random.default_rng(22)
    contexts = [int(x) for x in rng.integers(0, 300, 150)]
    contexts[70], contexts[149] = 5000, 2500
    D, page, Hq, Hkv = 64, 16, 4, 2
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, A.F16)
    q = _draw(rng, (len(contexts), Hq, D), A.F16)
    args = (_gpu(q, A.F16), cache, _gpu(table), _gpu(np.array(contexts, dtype=np.int32)))
    ws = torch.zeros(int(api.lib().kv4_attention_workspace_size(len(contexts), 1, Hq, Hkv, D)), dtype=torch.uint8, device="cuda")
    ws[32768:] = 255
    got = [_np(api.kv4_attention(*args, workspace=w)) for w in (ws, ws, ws[:16])]
    assert np.array_equal(got[0], got[1]) and not ws[:32768].any()
    for g in got[1:]:
        for b, c in enumerate(contexts):
            want, spread = A.attention(q[b:b + 1], keys[b], values[b], D ** -0.5, [c])
            _close(g[b:b + 1], want, spread, A.F16, 2.0 ** -11, f"sequence {b} of {c}")


@pytest.mark.parametrize("n,longest,Hq,Hkv,new,long", [
    (140, 300, 8, 8, 1, {70: 5000, 139: 2500}),        # split ones among many
    (70, 90, 32, 8, 5, {3: 3000, 4: 0}),               # 20 rows
    (1100, 40, 2, 2, 1, {0: 0, 1099: 1500, 500: 129}),  # more sequences than a block has threads
    (520, 0, 2, 2, 1, {}),                             # nothing but empty ones
])
def test_attention_of_more_items_than_run_at_once(n, longest, Hq, Hkv, new, long):
    """The chunks are found before the blocks start, long ones first; all the same twice, and the tickets are back at zero."""
    import torch

    rng = np.random.default_rng(n)
    contexts = [int(x) for x in rng.integers(0, longest + 1, n)]
    for s, c in long.items():
        contexts[s] = c
    D, page, dtype = 64, 16, A.BF16
    cache, table, keys, values = _filled(rng, contexts, page, Hkv, D, dtype)
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


@pytest.mark.parametrize("scale", [0.0, -0.11, 1e-30])
def test_scales_of_any_sign(scale):
    rng = np.random.default_rng(23)
    c, Hq, Hkv, D = 70, 4, 2, 128
    q, k, v = _draw(rng, (c, Hq, D), A.F16), _draw(rng, (c, Hkv, D), A.F16), _draw(rng, (c, Hkv, D), A.F16)
    got = api.attn_prompt(_gpu(q, A.F16), _gpu(k, A.F16), _gpu(v, A.F16), _gpu(np.array([0, c], dtype=np.int32)), scale=scale)
    want, spread = A.attention(q, k, v, scale, np.arange(c) + 1)
    _close(_np(got), want, spread, A.F16, 2.0 ** -11)
    cache = api.kv4_cache(5, 16, Hkv, D)
    api.kv4_write(_gpu(k, A.F16), _gpu(v, A.F16), _gpu(np.arange(c, dtype=np.int32)), cache)
    k, v = (A.dequantise(*A.quantise(x)) for x in (k, v))
    got = api.kv4_attention(_gpu(q[None, -3:], A.F16), cache, _gpu(np.arange(5, dtype=np.int32)[None]), _gpu(np.array([c], dtype=np.int32)), scale=scale)
    want, spread = A.attention(q[-3:], k, v, scale, c - 2 + np.arange(3))
    _close(_np(got)[0], want, spread, A.F16, 2.0 ** -11)


def test_example_layer():
    """Prompts, then steps from a graph.  4 bits hold a vector to a step of a fifteenth of its range, 0.35 of its standard deviation or
    so for 128 elements: errors of 0.1 of it in keys and values, each of which moves the result by about 0.1 of itself."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
    spec = importlib.util.spec_from_file_location("attention_layer", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    got, want = (x.float().cpu().numpy() for x in example.run(8, 2, (150, 33, 64), steps=5))
    assert got.shape == want.shape == (3, 5, 1024)
    assert 0.01 < np.linalg.norm(got - want) / np.linalg.norm(want) < 0.25


# --------------------------------------------------------------------------- streams, graphs, refusals
def test_another_stream_and_a_graph():
    """A decode step (append, attention) captured and replayed with other inputs between the replays, the allocator in use beside it;
    and the same calls on a stream handed over as a number."""
    import torch

    rng = np.random.default_rng(14)
    B, Hq, Hkv, D, page, width = 3, 8, 2, 128, 16, 12
    cache, table, _, _ = _filled(rng, [150, 20, 64], page, Hkv, D, A.F16, garbage=False, spare=40)
    free = [p for p in range(cache.shape[0]) if p not in table]
    wide = np.zeros((B, width), dtype=np.int32)
    wide[:, :table.shape[1]] = np.where(table == 2 ** 31 - 1, 0, table)
    for b, c in enumerate((150, 20, 64)):
        for i in range(-(-c // page), width):
            wide[b, i] = free.pop()
    rope = _gpu(A.rope_table(400, D).astype(np.float32))
    qkv = torch.zeros((B, Hq + 2 * Hkv, D), dtype=torch.float16, device="cuda")
    q, k, v = qkv.split((Hq, Hkv, Hkv), 1)
    pos, slots, ctx = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    d_table = _gpu(wide)
    lens = np.array([150, 20, 64])

    def feed(step):
        n = lens + step
        qkv.copy_(_gpu(_draw(np.random.default_rng(step), qkv.shape, A.F16), A.F16))
        pos.copy_(_gpu(n.astype(np.int32)))
        slots.copy_(_gpu((wide[np.arange(B), n // page] * page + n % page).astype(np.int32)))
        ctx.copy_(_gpu((n + 1).astype(np.int32)))

    def step(stream=None):
        turned = api.kv4_append(q, k, v, pos, rope, slots, cache, stream=stream)
        return api.kv4_attention(turned, cache, d_table, ctx, stream=stream)

    feed(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()  # (makes this stream's workspace)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for i in range(4):
        feed(i)
        torch.randn(1 << 20, device="cuda").sum().item()
        captured.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = captured.clone()
        assert torch.equal(got, step()) and torch.isfinite(got).all()
        torch.cuda.synchronize()
        other = torch.cuda.Stream()
        there = step(stream=other.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got, there)
    starts = _gpu(np.array([0, 1, 3], dtype=np.int32))
    here = api.attn_prompt(q, k, v, starts)
    torch.cuda.synchronize()
    there = api.attn_prompt(q, k, v, starts, stream=other.cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(here, there)


@pytest.mark.parametrize("n,Hq,Hkv,new", [(140, 8, 8, 1), (40, 32, 8, 5), (6, 16, 2, 4)])
def test_a_graph_follows_the_contexts(n, Hq, Hkv, new):
    """Attention captured with short contexts and replayed with others: what each block does is found anew in every replay."""
    import torch

    D, page, width = 64, 16, 20
    rng = np.random.default_rng(31)
    full = [page * width] * n
    cache, table, _, _ = _filled(rng, full, page, Hkv, D, A.F16, garbage=False, spare=0)
    table, ctx = _gpu(table), torch.ones(n, dtype=torch.int32, device="cuda")
    q = _gpu(_draw(rng, (n * new, Hq, D), A.F16), A.F16).unflatten(0, (n, new))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        api.kv4_attention(q, cache, table, ctx)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        captured = api.kv4_attention(q, cache, table, ctx)
    for i in range(5):
        lens = rng.integers(0, page * width + 1, n) if i % 2 else np.where(rng.random(n) < 0.1, page * width, i)
        ctx.copy_(_gpu(lens.astype(np.int32)))
        torch.randn(1 << 20, device="cuda").sum().item()
        captured.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = captured.clone()
        assert torch.equal(got, api.kv4_attention(q, cache, table, ctx)) and torch.isfinite(got).all()


def test_refusals():
    import torch

    q, k, v = (torch.zeros((4, h, 128), dtype=torch.float16, device="cuda") for h in (4, 2, 2))
    pos, table = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros((8, 128), device="cuda")
    cache = api.kv4_cache(2, 16, 2, 128)
    pages, ctx = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    rope = lambda **a: api.attn_qk_norm_rope(*(a.get(n, d) for n, d in zip(("q", "k", "pos", "table"), (q, k, pos, table))),
                                             **{n: x for n, x in a.items() if n not in ("q", "k", "pos", "table")})
    rope(), api.kv4_write(k, v, pos, cache), api.kv4_attention(q, cache, pages, ctx), api.attn_prompt(q, k, v, starts)
    for bad, error in [
            (lambda: rope(q=q.float()), TypeError), (lambda: rope(k=k.bfloat16()), TypeError), (lambda: rope(q=q.cpu()), TypeError),
            (lambda: rope(k=k[:3]), ValueError), (lambda: rope(pos=pos.long()), TypeError), (lambda: rope(pos=pos[:3]), ValueError),
            (lambda: rope(table=table.half()), TypeError), (lambda: rope(table=table[0]), ValueError),
            (lambda: rope(q_norm=torch.ones(64, device="cuda")), ValueError), (lambda: rope(q=q.transpose(1, 2)), ValueError),
            (lambda: rope(out_q=torch.empty_like(k)), ValueError), (lambda: rope(table=torch.zeros((8, 24), device="cuda")), api.LiquidGemmError),
            (lambda: rope(table=torch.zeros((8, 144), device="cuda")), api.LiquidGemmError), (lambda: rope(table=table[:0]), api.LiquidGemmError),
            (lambda: rope(k_norm=torch.ones(128, device="cuda"), eps=0.0), api.LiquidGemmError),
            (lambda: api.attn_qk_norm_rope(q[..., :96], k[..., :96], pos, table), api.LiquidGemmError),
            (lambda: rope(q=torch.zeros(4 * 4 * 128 + 1, dtype=torch.float16, device="cuda")[1:].view(4, 4, 128)), api.LiquidGemmError),
            (lambda: rope(q=torch.zeros((4, 4, 132), dtype=torch.float16, device="cuda")[..., :128]), api.LiquidGemmError),
            (lambda: api.kv4_write(k, v[:, :1], pos, cache), ValueError), (lambda: api.kv4_write(k, v, pos, cache[:, :1].contiguous()), ValueError),
            (lambda: api.kv4_write(k, v, pos, cache[:, :, :-16].contiguous()), ValueError), (lambda: api.kv4_write(k, v, pos, cache[:, :, ::2]), ValueError),
            (lambda: api.kv4_write(k, v, pos.long(), cache), TypeError), (lambda: api.kv4_read(cache, pos, dtype=torch.float32), TypeError),
            (lambda: api.kv4_attention(q[..., :64], cache, pages, ctx), ValueError), (lambda: api.kv4_attention(q[:, :3], cache, pages, ctx), api.LiquidGemmError),
            (lambda: api.kv4_attention(q, cache, pages[:3], ctx), ValueError), (lambda: api.kv4_attention(q, cache, pages, ctx[:3]), ValueError),
            (lambda: api.kv4_attention(q, cache, pages[:, :0], ctx), api.LiquidGemmError), (lambda: api.kv4_attention(q, cache, pages.long(), ctx), TypeError),
            (lambda: api.kv4_attention(q, cache, pages, ctx, scale=float("nan")), api.LiquidGemmError),
            (lambda: api.kv4_attention(q, cache, pages, ctx, out=q.bfloat16()), TypeError),
            (lambda: api.attn_prompt(q, k, v[:3], starts), ValueError), (lambda: api.attn_prompt(q, k[..., :64], v[..., :64], starts), ValueError),
            (lambda: api.attn_prompt(q[:, :3], k, v, starts), api.LiquidGemmError), (lambda: api.attn_prompt(q, k, v, starts.long()), TypeError),
            (lambda: api.attn_prompt(q, k, v, starts, starts[:1]), ValueError), (lambda: api.attn_prompt(q, k, v, starts, scale=float("inf")), api.LiquidGemmError),
            (lambda: api.kv4_cache(0, 16, 1, 128), ValueError), (lambda: api.kv4_cache(1, 24, 1, 128), ValueError), (lambda: api.kv4_cache(1, 16, 1, 96), ValueError)]:
        with pytest.raises(error):
            bad()
    # nothing to do
    none = q[:0]
    assert rope(q=none, k=k[:0], pos=pos[:0])[0].shape == (0, 4, 128)
    assert api.kv4_attention(none, cache, pages[:0], ctx[:0]).shape == none.shape
    assert api.attn_prompt(none, k, v, torch.zeros(1, dtype=torch.int32, device="cuda")).shape == none.shape
    api.kv4_write(k[:0], v[:0], pos[:0], cache)
    assert api.kv4_read(cache, pos[:0])[0].shape == (0, 2, 128)
