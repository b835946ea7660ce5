"""The norm and the gated activation with INT8 outputs, tokens sorted by expert and back, against their definitions (oracle/layer_oracle.py).

The norm's results and the gradients of the rows are determined bit for bit (single FP32 roundings after FP64 sums), and so are places and moved
rows.  The gated activation's FP32 values are within d = (4 + |gate|) 2^-22 of themselves: its codes q and scale s hold
|q s - y| <= s / 2 + d |y| + 2^-22 * 127 s (q s is compared in FP64; y / s and s are rounded), and s itself is within d + 2^-23 of max |y| / 127.  Sums of k
FP32 products are within (k + 1) 2^-24 of the sum of their absolute values, and a result in its type is rounded once (u = 2^-11 in FP16, 2^-8 in BF16)."""
import numpy as np
import pytest

from oracle import attention_oracle as A
from oracle import layer_oracle as R
from paper_2509_01229_amd import api

pytestmark = pytest.mark.gpu
TYPES = (A.F16, A.BF16)


def _draw(rng, shape, dtype, size=1.0):
    return A.round_to(rng.standard_normal(shape, dtype=np.float32) * np.float32(size), dtype)


def _gpu(x, dtype=None):
    import torch

    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to(getattr(torch, dtype)) if dtype else t


def _np(t):
    return t.float().cpu().numpy()


def _rows(x, dtype, stride=0):
    """x on the GPU, its rows `stride` elements apart with NaN between."""
    import torch

    t = torch.full((x.shape[0], x.shape[1] + stride), float("nan"), dtype=getattr(torch, dtype), device="cuda")
    t[:, :x.shape[1]] = _gpu(x, dtype)
    return t[:, :x.shape[1]]


# ------------------------------------------------------------------------------------------- norm
SHAPES = [(1, 8), (1, 4096), (3, 520), (130, 2048), (67, 2056), (5, 4104), (600, 4096), (20, 5120), (33, 8200), (2, 16392), (3, 28672), (2, 32776), (1, 70008)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M,K", SHAPES)
def test_norm_is_exact(dtype, residual, M, K):
    import torch

    rng = np.random.default_rng(M + K)
    x, w = _draw(rng, (M, K), dtype), (1 + 0.3 * rng.standard_normal(K)).astype(np.float32)
    res = _draw(rng, (M, K), dtype, 3.0) * np.exp2(rng.integers(-3, 4, K)).astype(np.float32) if residual else None
    res = A.round_to(res, dtype) if residual else None
    if M > 2:
        x[0] = 0
        if residual:
            res[0], res[1] = 0, -x[1]                # rows of zeros
        x[2] = A.round_to(x[2] * np.float32(2.0 ** -20), dtype)  # (in FP16 subnormal numbers)
    for weight, want_y, stride in ((w, True, 0), (None, False, 24)):
        got = api.w4a8_norm_quantize(_rows(x, dtype, stride), None if weight is None else _gpu(weight), eps=1e-6, want_y=want_y,
                                     residual=_rows(res, dtype, 2 * stride) if residual else None)
        q, s, h, y = R.norm_quantise(x, res, weight, 1e-6, dtype)
        assert got[0].dtype == torch.int8 and np.array_equal(got[1].cpu().numpy().view(np.uint32), s.view(np.uint32))
        assert np.array_equal(got[0].cpu().numpy(), q)
        assert (got[2] is None) == (not residual) and (got[3] is None) == (not want_y)
        if residual:
            assert np.array_equal(_np(got[2]), h)
        if want_y:
            assert np.array_equal(_np(got[3]), A.round_to(y, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [1024, 8192, 40000])
def test_norm_in_place(dtype, K):
    """h in the place of the residual, or of x; outputs that are given."""
    import torch

    rng = np.random.default_rng(K)
    x, res = _draw(rng, (9, K), dtype), _draw(rng, (9, K), dtype)
    q, s, h, y = R.norm_quantise(x, res, None, 1e-5, dtype)
    for name in ("residual", "x"):
        t = {"x": _gpu(x, dtype), "residual": _gpu(res, dtype)}
        out = {"out_q": torch.empty((9, K), dtype=torch.int8, device="cuda"), "out_scales": torch.empty(9, device="cuda"), "out_y": torch.empty_like(t["x"]), "out_h": t[name]}
        got = api.w4a8_norm_quantize(t["x"], residual=t["residual"], eps=1e-5, **out)
        assert [a is b for a, b in zip(got, (out["out_q"], out["out_scales"], out["out_h"], out["out_y"]))] == [True] * 4
        assert np.array_equal(got[0].cpu().numpy(), q) and np.array_equal(got[1].cpu().numpy(), s)
        assert np.array_equal(_np(got[2]), h) and np.array_equal(_np(got[3]), A.round_to(y, dtype))


def test_norm_of_numbers_near_the_ends():
    """Squares that overflow FP32 and ones that vanish in it; a row that is not finite spoils no other."""
    import torch

    rng = np.random.default_rng(4)
    K = 512
    x = np.stack([_draw(rng, K, A.BF16, 1.0) * np.float32(f) for f in (2.0 ** 120, 2.0 ** 64, 2.0 ** -70, 2.0 ** -120, 1.0, 1.0)])
    x = A.round_to(x, A.BF16)
    q, s, _, y = R.norm_quantise(x, None, None, 1e-30, A.BF16)
    got = api.w4a8_norm_quantize(_gpu(x, A.BF16), eps=1e-30, want_y=True)
    assert np.array_equal(got[0].cpu().numpy(), q) and np.array_equal(got[1].cpu().numpy(), s) and np.array_equal(_np(got[3]), A.round_to(y, A.BF16))
    for bad in (np.nan, np.inf):
        x[4, 77] = bad
        again = api.w4a8_norm_quantize(_gpu(x, A.BF16), eps=1e-30, want_y=True)
        keep = [0, 1, 2, 3, 5]
        for a, b in zip(again, got):
            assert a is None or torch.equal(a[keep], b[keep])


# ------------------------------------------------------------------------------- gated activation
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,K", [(1, 8), (1, 1536), (7, 2056), (65, 4096), (3, 6912), (300, 11008), (2, 14336), (3, 28672), (2, 32776), (1, 65544)])
def test_swiglu(dtype, M, K):
    rng = np.random.default_rng(M + K)
    x = _draw(rng, (M, 2 * K), dtype, 2.0)
    x[0, :K] = A.round_to(np.linspace(-16, 16, K), dtype)
    if M > 2:
        x[1] = 0
        x[2, K:] = 0
    for stride in (0, 40):
        q, s = (t.cpu().numpy().astype(np.float64) for t in api.w4a8_swiglu_quantize(_rows(x, dtype, stride)))
        y = R.gated(x)
        d = (4 + np.abs(x[:, :K].astype(np.float64))) * 2.0 ** -22
        most = np.abs(y).max(-1)
        assert (s[most == 0] == 1).all()
        assert (np.abs(s * 127 - most) <= (d * np.abs(y)).max(-1) + 2.0 ** -23 * most)[most > 0].all()
        assert (np.abs(q * s[:, None] - y) <= s[:, None] * (0.5 + 127 * 2.0 ** -22) + d * np.abs(y)).all()
        assert (np.abs(q).max(-1)[most > 0] == 127).all()


def test_swiglu_of_large_gates():
    """Gates whose exponential is infinite or vanishes: zero, and the gate itself."""
    x = np.zeros((2, 32), dtype=np.float32)
    x[0, :16], x[0, 16:] = [-60000, -200, -100, -89, 100, 200, 500, 1000] * 2, 1
    x[1, :16], x[1, 16:] = [-88.5, -50, 30, 88, 89, -30, 0, 40] * 2, 2
    q, s = (t.cpu().numpy().astype(np.float64) for t in api.w4a8_swiglu_quantize(_gpu(x, A.F16)))
    x = A.round_to(x, A.F16)
    y = R.gated(x)
    assert np.isfinite(s).all() and (np.abs(q * s[:, None] - y) <= s[:, None] * 0.50001 + (4 + np.abs(x[:, :16])) * 2.0 ** -22 * np.abs(y)).all()


# ------------------------------------------------------------------------- tokens sorted by expert
ROUTES = [
    # tokens, experts a token, experts
    (1, 1, 1), (1, 2, 8), (16, 2, 8), (37, 8, 64), (512, 2, 8), (513, 2, 8), (128, 8, 256), (1000, 3, 5), (4099, 1, 17), (700, 64, 200), (2500, 8, 128),
    (64, 2, 8), (43, 3, 8), (1024, 2, 20), (683, 3, 20),  # on both sides of 128 and 2048 pairs
    (4096, 4, 3), (4097, 4, 3), (9001, 4, 6), (4500, 8, 256), (20000, 1, 128),  # several blocks an expert, and one for several batches of pairs
]


def _route(rng, T, each, E, style):
    if style == "same":
        return np.full((T, each), E // 2, dtype=np.int32)
    ids = rng.integers(0, E, (T, each)).astype(np.int32)
    if style == "skewed":
        ids = np.minimum(ids, rng.integers(0, E, (T, each))).astype(np.int32)
    if style == "absent":
        ids = np.where(rng.random((T, each)) < 0.4, rng.choice([-1, -2 ** 31, E, 2 ** 31 - 1], (T, each)), ids).astype(np.int32)
    if style == "nobody":
        ids[:] = -1
    return ids


@pytest.mark.parametrize("style", ["skewed", "same", "absent", "nobody"])
@pytest.mark.parametrize("T,each,E", ROUTES)
def test_dispatch(T, each, E, style):
    import torch

    rng = np.random.default_rng(T + E)
    ids = _route(rng, T, each, E, style)
    offsets, places, tokens = R.dispatch(ids, E)
    for dtype, K, stride in ((torch.int8, 48, 16), (torch.float16, 2056, 0), (torch.bfloat16, 8, 8)):
        if T * each > 8192 and K > 1000:
            K = 264
        x = _gpu(rng.integers(-127, 128, (T, K + stride)).astype(np.int8)).to(dtype)[:, :K]
        scales = _gpu(rng.random(T).astype(np.float32)) if dtype == torch.int8 else None
        out = torch.full((T * each, K), 99, dtype=dtype, device="cuda")
        out_scales = torch.full((T * each,), -1.0, device="cuda") if scales is not None else None
        got = api.moe_dispatch(x, _gpu(ids), E, act_scales=scales, out=out, out_scales=out_scales)
        assert got[0] is out and got[1] is out_scales
        assert got[2].dtype == got[3].dtype == torch.int32 and np.array_equal(got[2].cpu().numpy(), offsets) and np.array_equal(got[3].cpu().numpy(), places)
        n, source = len(tokens), _gpu(tokens)
        assert torch.equal(out[:n], x[source]) and (out[n:] == 99).all()
        if scales is not None:
            assert torch.equal(out_scales[:n], scales[source]) and (out_scales[n:] == -1).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,each,E,N", [(1, 1, 4, 8), (16, 2, 8, 4096), (37, 8, 64, 2056), (300, 3, 7, 1032), (2, 64, 200, 24), (513, 6, 60, 264)])
@pytest.mark.parametrize("style", ["skewed", "absent"])
def test_combine_and_its_gradients(dtype, T, each, E, N, style):
    import torch

    rng = np.random.default_rng(T + N)
    offsets, places, tokens = R.dispatch(_route(rng, T, each, E, style), E)
    rows, u = T * each, A.UNIT[dtype]
    Y, grad, w = _draw(rng, (rows, N), dtype), _draw(rng, (T, N), dtype), rng.random((T, each)).astype(np.float32)
    Y[len(tokens):] = np.nan                             # (rows that no pair has are not looked at)
    w[places < 0] = np.nan
    dY, dg, dp = _rows(Y, dtype, 16), _rows(grad, dtype, 8), _gpu(places)
    for weights in (w, None):
        got = _np(api.moe_combine(dY, dp, None if weights is None else _gpu(weights)))
        want, size = R.combine(Y, places, weights)
        assert (np.abs(got - want) <= u * np.abs(want) * 1.001 + (each + 1) * 2.0 ** -24 * size + 2.0 ** -25).all()
    of_rows, of_weights, size = R.combine_backward(grad, Y, places, w, dtype)
    for row_offsets in (_gpu(offsets), None):
        out = torch.full((rows, N), 7.0, dtype=dY.dtype, device="cuda")
        for given in ({}, {"out_Y": out, "out_weights": torch.empty((T, each), device="cuda")}):
            gY, gw = api.moe_combine_backward(dg, dY, dp, _gpu(w), row_offsets=row_offsets, **given)
            assert not given or (gY is out and gw is given["out_weights"])
            assert np.array_equal(_np(gY)[:len(tokens)], of_rows[:len(tokens)])
            assert (gY[len(tokens):] == (7.0 if given and row_offsets is None else 0.0)).all()
            assert gw.dtype == torch.float32 and (np.abs(gw.double().cpu().numpy() - of_weights) <= (N / 256 + 16) * 2.0 ** -24 * size).all()


def test_gradients_against_differences():
    """moe_combine_backward, and moe_combine as the gradient of moe_dispatch, against differences of what they are the gradients of.  The functions are
    linear in each of their arguments, and the differences are taken of results that are exact: small whole numbers."""
    import torch

    rng = np.random.default_rng(8)
    T, each, E, N = 6, 3, 5, 16
    ids = _route(rng, T, each, E, "absent")
    offsets, places, tokens = R.dispatch(ids, E)
    whole = lambda *shape: rng.integers(-4, 5, shape).astype(np.float32)  # noqa: E731
    Y, w, grad, X = whole(T * each, N), whole(T, each), whole(T, N), whole(T, N)
    dp = _gpu(places)
    forward = lambda Y, w: (_np(api.moe_combine(_gpu(Y, A.F16), dp, _gpu(w))).astype(np.float64) * grad).sum()  # noqa: E731
    gY, gw = (_np(t) for t in api.moe_combine_backward(_gpu(grad, A.F16), _gpu(Y, A.F16), dp, _gpu(w), row_offsets=_gpu(offsets)))
    base = forward(Y, w)
    for _ in range(25):
        r, n, t, j = rng.integers(T * each), rng.integers(N), rng.integers(T), rng.integers(each)
        Y2, w2 = Y.copy(), w.copy()
        Y2[r, n] += 1
        w2[t, j] += 1
        assert forward(Y2, w) - base == gY[r, n] and forward(Y, w2) - base == gw[t, j]
    rows_grad = whole(T * each, N)
    out = lambda X: api.moe_dispatch(_gpu(X, A.F16), _gpu(ids), E, out=torch.zeros((T * each, N), dtype=torch.float16, device="cuda"))[0]  # noqa: E731
    of = lambda X: (_np(out(X)).astype(np.float64) * rows_grad).sum()  # noqa: E731
    gX, base = _np(api.moe_combine(_gpu(rows_grad, A.F16), dp)), of(X)
    for _ in range(25):
        t, n = rng.integers(T), rng.integers(N)
        X2 = X.copy()
        X2[t, n] += 1
        assert of(X2) - base == gX[t, n]


def test_places_outside_the_rows_and_the_same_row_twice():
    """Places that moe_dispatch does not give: outside the rows they add nothing, a row may count twice."""
    rng = np.random.default_rng(9)
    Y, w = _draw(rng, (5, 64), A.F16), rng.random((4, 3)).astype(np.float32)
    places = np.array([[0, 0, 4], [5, 2 ** 31 - 1, -2 ** 31], [-1, 3, 3], [1, 2, -7]], dtype=np.int32)
    got = _np(api.moe_combine(_gpu(Y, A.F16), _gpu(places), _gpu(w)))
    want, size = R.combine(Y, places, w)
    assert (np.abs(got - want) <= 1.001 * 2.0 ** -11 * np.abs(want) + 4 * 2.0 ** -24 * size + 2.0 ** -25).all() and (got[1] == 0).all()
    assert (api.moe_combine(_gpu(Y[:0], A.F16), _gpu(places), _gpu(w)) == 0).all()


# -------------------------------------------------------------------------- streams, graphs, refusals
def test_a_graph_follows_its_inputs():
    """All of them captured together, small and large, and replayed with other inputs between the replays; and on a stream given as a number."""
    import torch

    rng = np.random.default_rng(10)
    for T in (20, 900):
        K, E, each = 512, 8, 2
        x, res, grad = (torch.empty((T, K), dtype=torch.float16, device="cuda") for _ in range(3))
        ids, w = torch.zeros((T, each), dtype=torch.int32, device="cuda"), torch.empty((T, each), device="cuda")
        rows = torch.zeros((T * each, K), dtype=torch.int8, device="cuda")
        row_scales = torch.zeros(T * each, device="cuda")

        def feed(i):
            for t in (x, res, grad):
                t.copy_(_gpu(_draw(rng, (T, K), A.F16)))
            ids.copy_(_gpu(_route(rng, T, each, E, ("skewed", "absent", "same")[i % 3])))
            w.copy_(_gpu(rng.random((T, each)).astype(np.float32)))

        def step():
            q, s, h, y = api.w4a8_norm_quantize(x, residual=res, want_y=True)
            _, _, offsets, places = api.moe_dispatch(q, ids, E, act_scales=s, out=rows, out_scales=row_scales)
            q2, s2 = api.w4a8_swiglu_quantize(y)
            Y = y[:, None].expand(T, each, K).reshape(T * each, K)
            out = api.moe_combine(Y, places, w)
            return [q, s, h, y, offsets, places, q2, s2, out, *api.moe_combine_backward(grad, Y, places, w, row_offsets=offsets)]

        feed(0)
        step()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            captured = step()
        for i in range(4):
            feed(i)
            torch.randn(1 << 20, device="cuda").sum().item()
            for t in captured:
                t.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in captured]
            kept = rows.clone(), row_scales.clone()
            want = step()
            n = int(want[4][-1])
            for a, b in zip(got, want):
                assert torch.equal(a, b)
            assert torch.equal(kept[0][:n], rows[:n]) and torch.equal(kept[1][:n], row_scales[:n])
        other = torch.cuda.Stream()
        torch.cuda.synchronize()
        q, s, h, y = api.w4a8_norm_quantize(x, residual=res, want_y=True, stream=other.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(q, want[0]) and torch.equal(s, want[1]) and torch.equal(h, want[2]) and torch.equal(y, want[3])


def test_more_rows_than_the_calls_count():
    """(Rows that are one row in memory.)"""
    import torch

    row = torch.ones((1, 8), dtype=torch.float16, device="cuda")
    for rows in (2 ** 31, 2 ** 32 + 3):
        many = row.expand(rows, 8)
        for call in (lambda: api.w4a8_norm_quantize(many), lambda: api.w4a8_swiglu_quantize(row.repeat(1, 2).expand(rows, 16)),
                     lambda: api.moe_combine(many, _gpu(np.zeros((1, 1), dtype=np.int32)))):
            with pytest.raises(ValueError, match="too large"):
                call()


def test_gradients_on_another_stream():
    """What no place names is zeroed on the stream that the call is given, not on the current one, which is at work."""
    import torch

    rng = np.random.default_rng(30)
    Y, grad = _gpu(_draw(rng, (9, 64), A.F16), A.F16), _gpu(_draw(rng, (3, 64), A.F16), A.F16)
    places, w = _gpu(np.array([[0, 4], [8, -1], [2, 7]], dtype=np.int32)), _gpu(rng.random((3, 2)).astype(np.float32))
    want = api.moe_combine_backward(grad, Y, places, w)
    side = torch.cuda.Stream()
    for _ in range(2):
        torch.cuda.synchronize()
        big = torch.zeros(1 << 28, device="cuda")
        for _ in range(20):
            big.add_(1.0)                                   # (milliseconds)
        got = api.moe_combine_backward(grad, Y, places, w, stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[0][[1, 3, 5, 6]].any()


def test_refusals():
    import torch

    x, ids, w = torch.zeros((4, 64), dtype=torch.float16, device="cuda"), torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    q8, s8, odd = x.to(torch.int8), torch.ones(4, device="cuda"), torch.zeros(4 * 64 + 1, dtype=torch.float16, device="cuda")[1:].view(4, 64)
    Y = torch.zeros((8, 64), dtype=torch.float16, device="cuda")
    offsets = torch.zeros(3, dtype=torch.int32, device="cuda")
    weight = torch.ones(64, device="cuda")
    norm, back = api.w4a8_norm_quantize, lambda **a: api.moe_combine_backward(*(a.get(n, d) for n, d in zip(("grad", "Y", "places", "weights"), (x, Y, ids, w))),
                                                                              **{n: v for n, v in a.items() if n not in ("grad", "Y", "places", "weights")})
    norm(x, weight), api.w4a8_swiglu_quantize(x), api.moe_dispatch(q8, ids, 2, act_scales=s8), api.moe_combine(Y, ids, w), back(row_offsets=offsets)
    E = api.LiquidGemmError
    for bad, error in [
            (lambda: norm(x.float()), TypeError), (lambda: norm(x[0]), ValueError), (lambda: norm(x.t()), ValueError), (lambda: norm(x, weight.half()), TypeError),
            (lambda: norm(x, weight[:32]), ValueError), (lambda: norm(x, residual=x.bfloat16()), TypeError), (lambda: norm(x, residual=x[:3]), ValueError),
            (lambda: norm(x, eps=0.0), E), (lambda: norm(x, eps=float("nan")), E), (lambda: norm(x, out_h=x), ValueError), (lambda: norm(x, out_y=Y), ValueError),
            (lambda: norm(x, residual=x, out_h=Y[::2]), ValueError), (lambda: norm(x[:, :60]), E), (lambda: norm(odd), E), (lambda: norm(x, out_q=q8[:3]), ValueError),
            (lambda: norm(torch.zeros((4, 68), dtype=torch.float16, device="cuda")[:, :64]), E), (lambda: norm(x, out_scales=s8.double()), TypeError),
            (lambda: api.w4a8_swiglu_quantize(x.float()), TypeError), (lambda: api.w4a8_swiglu_quantize(x[:, :24]), E), (lambda: api.w4a8_swiglu_quantize(x[:, :33]), ValueError),
            (lambda: api.w4a8_swiglu_quantize(odd), E), (lambda: api.w4a8_swiglu_quantize(x, out_q=q8), ValueError),
            (lambda: api.moe_dispatch(x.float(), ids, 2), TypeError), (lambda: api.moe_dispatch(x, ids.long(), 2), TypeError), (lambda: api.moe_dispatch(x, ids[:3], 2), ValueError),
            (lambda: api.moe_dispatch(x, ids[:, 0], 2), ValueError), (lambda: api.moe_dispatch(x, ids, 0), ValueError), (lambda: api.moe_dispatch(x, ids, 257), ValueError),
            (lambda: api.moe_dispatch(x, ids[:, :0], 2), E), (lambda: api.moe_dispatch(q8[:, :24].contiguous(), ids, 2), E), (lambda: api.moe_dispatch(x, ids, 2, out=Y[:7]), ValueError),
            (lambda: api.moe_dispatch(x, ids, 2, out_scales=torch.zeros(8, device="cuda")), ValueError), (lambda: api.moe_dispatch(q8, ids, 2, act_scales=s8[:3]), ValueError),
            (lambda: api.moe_dispatch(x, ids.repeat(1, 33).contiguous(), 2), E), (lambda: api.moe_dispatch(x, ids.repeat(1, 2)[:, ::2], 2), ValueError),
            (lambda: api.moe_combine(Y.float(), ids, w), TypeError), (lambda: api.moe_combine(Y, ids.long(), w), TypeError), (lambda: api.moe_combine(Y, ids, w[:, :1]), ValueError),
            (lambda: api.moe_combine(Y, ids[0], w), ValueError), (lambda: api.moe_combine(Y[:, :12], ids, w), E), (lambda: api.moe_combine(Y, ids, w, out=Y), ValueError),
            (lambda: back(grad=x[:3]), ValueError), (lambda: back(grad=x.bfloat16()), TypeError), (lambda: back(weights=None), ValueError), (lambda: back(row_offsets=offsets.long()), TypeError),
            (lambda: back(row_offsets=offsets[:0]), ValueError), (lambda: back(out_Y=Y[:, :32]), ValueError), (lambda: back(out_weights=w.half()), TypeError)]:
        with pytest.raises(error):
            bad()
    # nothing to do
    assert norm(x[:0])[0].shape == (0, 64) and api.w4a8_swiglu_quantize(x[:0])[0].shape == (0, 32)
    rows, _, offsets, places = api.moe_dispatch(x[:0], ids[:0], 2)
    assert rows.shape == (0, 64) and places.shape == (0, 2) and offsets.tolist() == [0, 0, 0]
    assert api.moe_combine(Y, ids[:0], w[:0]).shape == (0, 64)
    gY, gw = back(grad=x[:0], places=ids[:0], weights=w[:0], row_offsets=offsets)
    assert (gY == 0).all() and gw.shape == (0, 2)


def test_what_asks_for_a_gradient_is_refused():
    import torch

    x, Y = torch.randn((4, 64), device="cuda").half(), torch.randn((8, 64), device="cuda").half()
    ids, w, weight = torch.tensor([[0, 1]] * 4, dtype=torch.int32, device="cuda"), torch.rand((4, 2), device="cuda"), torch.rand(64, device="cuda")
    made = {"x": x, "residual": x.clone(), "weight": weight, "X": x, "Y": Y, "weights": w, "grad": x}
    for names, call in [(("x", "weight", "residual"), lambda x, weight, residual: api.w4a8_norm_quantize(x, weight, residual)), (("x",), api.w4a8_swiglu_quantize),
                        (("X",), lambda X: api.moe_dispatch(X, ids, 2)), (("Y", "weights"), lambda Y, weights: api.moe_combine(Y, ids, weights)),
                        (("grad", "Y", "weights"), lambda grad, Y, weights: api.moe_combine_backward(grad, Y, ids, weights))]:
        call(*(made[n] for n in names))
        for name in names:
            args = [made[n].clone().requires_grad_() if n == name else made[n] for n in names]
            with pytest.raises(ValueError, match=name):
                call(*args)
            with torch.no_grad():
                call(*args)
            with torch.inference_mode():
                call(*args)


def test_through_the_native_module_and_without(monkeypatch):
    """The native module answers the plain calls, and with the same bytes as the path behind it."""
    import torch

    api.lib()
    native = api._native
    x, ids, w = torch.randn((40, 256), device="cuda").half(), torch.randint(-1, 5, (40, 2), device="cuda").int(), torch.rand((40, 2), device="cuda")
    wide, weight, Y = torch.randn((40, 528), device="cuda").bfloat16()[:, :512], torch.rand(256, device="cuda"), torch.randn((80, 256), device="cuda").half()
    q8, s8 = api.w4a8_swiglu_quantize(wide)
    kept = torch.zeros((80, 256), dtype=torch.int8, device="cuda"), torch.zeros(80, device="cuda")
    places, offsets = api.moe_dispatch(x, ids, 4)[3], api.moe_dispatch(x, ids, 4)[2]
    now = torch.cuda.current_stream().cuda_stream
    calls = [lambda: api.w4a8_norm_quantize(x, weight, residual=x, want_y=True), lambda: api.w4a8_norm_quantize(wide, eps=1e-5, stream=now),
             lambda: api.w4a8_swiglu_quantize(wide), lambda: api.moe_dispatch(q8, ids, 4, act_scales=s8, out=kept[0], out_scales=kept[1]),
             lambda: api.moe_combine(Y, places, w), lambda: api.moe_combine(Y, places), lambda: api.moe_combine_backward(x, Y, places, w, row_offsets=offsets)]
    for call in calls:
        answers = []

        class Watched:
            def __getattr__(self, name):
                def run(*a):
                    answers.append(getattr(native, name)(*a))
                    return answers[-1]
                return run

        class Nothing:
            def __getattr__(self, name):
                return lambda *a: None

        monkeypatch.setattr(api, "_native", Watched())
        fast = call()
        assert len(answers) == 1 and answers[0] is not None
        fast = [t if t is None else t.clone() for t in (fast if isinstance(fast, tuple) else (fast,))]
        monkeypatch.setattr(api, "_native", Nothing())
        general = call()
        general = general if isinstance(general, tuple) else (general,)
        monkeypatch.setattr(api, "_native", native)
        assert len(fast) == len(general)
        for f, g in zip(fast, general):
            assert (f is None) == (g is None)
            if f is not None:
                assert f.dtype == g.dtype and f.shape == g.shape and torch.equal(f.view(torch.uint8), g.view(torch.uint8))


# ------------------------------------------------------------------------------- millions of tokens
def test_dispatch_of_millions_of_tokens():
    """More tokens than one launch holds where a row has 1024 threads.  Nearly all of them go to experts that are elsewhere, so that the rows are few; the tokens' rows overlap
    in memory, eight elements apart."""
    import ctypes

    import torch

    T, each, E, K = 2 ** 22 + 5, 2, 3, 4104
    rng = np.random.default_rng(40)
    ids = torch.full((T, each), -1, dtype=torch.int32)
    tokens = sorted({0, 1, 2 ** 21 - 1, 2 ** 21, 2 ** 21 + 1, 2 ** 22 - 1, 2 ** 22, T - 1, *rng.integers(0, T, 50).tolist()})
    ids[tokens] = torch.from_numpy(rng.integers(-1, E + 1, (len(tokens), each)).astype(np.int32))
    offsets, places, source = R.dispatch(ids.numpy(), E)
    buffer = torch.randn(8 * T + K, device="cuda").half()
    scales, ids = torch.rand(T, device="cuda"), ids.cuda()
    rows, row_scales = torch.full((len(source) + 2, K), 99.0, dtype=torch.float16, device="cuda"), torch.full((len(source) + 2,), 99.0, device="cuda")
    got_offsets, got_places = torch.empty(E + 1, dtype=torch.int32, device="cuda"), torch.empty((T, each), dtype=torch.int32, device="cuda")
    pointer = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    rc = api.lib().moe_dispatch(api.LQ_F16, T, each, E, K, pointer(buffer), 8, pointer(scales), pointer(ids), pointer(rows), pointer(row_scales),
                                pointer(got_offsets), pointer(got_places), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    assert np.array_equal(got_offsets.cpu().numpy(), offsets) and np.array_equal(got_places.cpu().numpy(), places)
    n, source = len(source), _gpu(source)
    assert torch.equal(rows[:n], buffer.as_strided((T, K), (8, 1))[source]) and (rows[n:] == 99).all()
    assert torch.equal(row_scales[:n], scales[source]) and (row_scales[n:] == 99).all()


@pytest.mark.parametrize("T,N,weighted", [(2 ** 23 + 9, 8, True), (2 ** 22 + 7, 2056, False)])
def test_combine_of_millions_of_tokens(T, N, weighted):
    """More blocks than one launch holds; nearly all tokens have no row."""
    import torch

    rng = np.random.default_rng(41)
    tokens = sorted({0, 1, 2 ** 21, 2 ** 22 - 1, 2 ** 22, T - 10, T - 9, T - 8, T - 1, *rng.integers(0, T, 40).tolist()})
    Y, places, w = _draw(rng, (30, N), A.BF16), torch.full((T, 2), -1, dtype=torch.int32), torch.from_numpy(rng.random((T, 2)).astype(np.float32))
    places[tokens] = torch.from_numpy(rng.integers(0, 30, (len(tokens), 2)).astype(np.int32))
    out = torch.full((T, N), 7.0, dtype=torch.bfloat16, device="cuda")
    assert api.moe_combine(_gpu(Y, A.BF16), places.cuda(), w.cuda() if weighted else None, out=out) is out
    want, size = R.combine(Y, places[tokens].numpy(), w[tokens].numpy() if weighted else None)
    at = _gpu(np.array(tokens))
    assert (np.abs(_np(out[at]) - want) <= A.UNIT[A.BF16] * np.abs(want) * 1.001 + 3 * 2.0 ** -24 * size + 2.0 ** -25).all()
    out[at] = 0
    assert not out.any()


@pytest.mark.parametrize("T,N", [(2 ** 22 + 5, 4104), (2 ** 23 - 1, 8)])
def test_gradients_of_millions_of_tokens(T, N):
    """The same of the gradients (whose rows overlap in memory, eight elements apart)."""
    import torch

    rng = np.random.default_rng(42)
    ids = torch.full((T, 2), -1, dtype=torch.int32)
    tokens = sorted({0, 1, 2 ** 21, 2 ** 22 - 1, 2 ** 22, T - 2, T - 1, *rng.integers(0, T, 40).tolist()})
    ids[tokens] = torch.from_numpy(rng.integers(-1, 4, (len(tokens), 2)).astype(np.int32))
    offsets, places, source = R.dispatch(ids.numpy(), 3)
    rows = len(source) + 3
    grad, Y, w = torch.randn(8 * T + N, device="cuda").half().as_strided((T, N), (8, 1)), _draw(rng, (rows, N), A.F16), torch.rand((T, 2), device="cuda")
    gY, gw = api.moe_combine_backward(grad, _gpu(Y, A.F16), _gpu(places), w, row_offsets=_gpu(offsets))
    at = _gpu(np.array(tokens))
    of_rows, of_weights, size = R.combine_backward(_np(grad[at]), Y, places[tokens], w[at].cpu().numpy(), A.F16)
    assert np.array_equal(_np(gY)[:len(source)], of_rows[:len(source)]) and not gY[len(source):].any()
    assert (np.abs(gw[at].double().cpu().numpy() - of_weights) <= (N / 256 + 16) * 2.0 ** -24 * size).all()
    gw[at] = 0
    assert not gw.any()


# ------------------------------------------------------------------- gates and rows at the ends of FP32
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K", [64, 33000])
def test_swiglu_of_gates_whose_exponential_overflows(dtype, K):
    """exp(-gate) overflows FP32 from a gate of -88.7 on, where gate * exp(gate) * up is still an ordinary number if up is large: rows of such gates alone, and of some next to
    others.  A subnormal result is rounded to 2^-149, and so is the scale, which 127 times that is an error of a value; hence the absolute term."""
    rng = np.random.default_rng(K)
    ranges = [(-81, -79), (-89, -86), (-90, -89), (-96, -90), (-104, -96), (-115, -104)] + ([(-150, -115), (-180, -150), (-192, -180)] if dtype == A.BF16 else [])
    gate = np.stack([rng.uniform(a, b, K) for a, b in ranges] + [np.where(np.arange(K) % 5 == 2, rng.uniform(-100, -70, K), rng.standard_normal(K))])
    up = np.exp2(rng.uniform(110, 127, gate.shape) if dtype == A.BF16 else rng.uniform(5, 15.9, gate.shape)) * rng.choice([-1, 1], gate.shape)
    up[-1] = np.where(gate[-1] < -60, up[-1], 2.0 ** -30)
    x = A.round_to(np.concatenate([gate, up], 1).astype(np.float32), dtype)
    q, s = (t.cpu().numpy().astype(np.float64) for t in api.w4a8_swiglu_quantize(_gpu(x, dtype)))
    y, least = R.gated(x), 128 * 2.0 ** -149
    d = (4 + np.abs(x[:, :K].astype(np.float64))) * 2.0 ** -22
    most = np.abs(y).max(-1)
    assert (most > 2 * least).sum() >= len(x) - 1
    assert (np.abs(s * 127 - most) <= (d * np.abs(y)).max(-1) + 2.0 ** -23 * most + least)[most > 2 * least].all()
    assert (np.abs(q * s[:, None] - y) <= s[:, None] * (0.5 + 127 * 2.0 ** -22) + d * np.abs(y) + least).all()
    one = api.w4a8_swiglu_quantize(_gpu(x[:, np.r_[0:8, K:K + 8]], dtype))    # (whatever stands next to a gate)
    assert np.isfinite(one[1].cpu().numpy()).all()


def test_rows_whose_scale_is_subnormal():
    """Rows so small that the scale has few bits, or none: codes are those of the division by the scale, up to 127 (and of a row without a scale 0, with scale 1)."""
    rng = np.random.default_rng(50)
    K, sizes = 256, np.array([2.0 ** -e for e in (120, 125, 126, 127, 130, 133, 136, 138, 139, 140, 141, 142, 143, 144, 146, 149)], dtype=np.float32)
    x = _draw(rng, (len(sizes), K), A.BF16)
    x[:, 0] = 0
    for weight in (sizes[:, None] * np.float32(1.0) * np.ones((1, K), dtype=np.float32)):
        q, s, _, y = R.norm_quantise(x, None, weight, 1e-6, A.BF16)
        got = api.w4a8_norm_quantize(_gpu(x, A.BF16), _gpu(weight), eps=1e-6)
        assert np.array_equal(got[1].cpu().numpy().view(np.uint32), s.view(np.uint32)) and np.array_equal(got[0].cpu().numpy(), q), weight[0]
    # gates of 64, whose logistic is 1 in FP32; ups as small as the type has them
    up = A.round_to(rng.standard_normal((len(sizes), K)).astype(np.float32) * sizes[:, None] * np.float32(2.0 ** -6), A.BF16)
    up[:, 1] = 0
    q, s = R.quantise_rows((np.float32(64) * up).astype(np.float32))
    got = api.w4a8_swiglu_quantize(_gpu(np.concatenate([np.full_like(up, 64), up], 1), A.BF16))
    assert np.array_equal(got[1].cpu().numpy().view(np.uint32), s.view(np.uint32)) and np.array_equal(got[0].cpu().numpy(), q)


# -------------------------------------------------------------------------- rows that a block goes through more than once
@pytest.mark.parametrize("dtype,K", [("float16", 4096), ("bfloat16", 4104), ("float16", 8200), ("bfloat16", 16392), ("int8", 8192), ("int8", 8208), ("int8", 16400), ("int8", 32784)])
def test_dispatch_of_long_rows(dtype, K):
    """More than 2048 pairs, rows of up to 512 pieces of 16 bytes and of more: one, two and three pieces a thread."""
    import torch

    rng = np.random.default_rng(K)
    T, each, E = 750, 3, 5
    ids = _route(rng, T, each, E, "absent")
    offsets, places, tokens = R.dispatch(ids, E)
    x = _gpu(rng.integers(-127, 128, (T, K + 16)).astype(np.int8)).to(getattr(torch, dtype))[:, :K]
    out = torch.full((T * each, K), 99, dtype=x.dtype, device="cuda")
    got = api.moe_dispatch(x, _gpu(ids), E, out=out)
    n = len(tokens)
    assert np.array_equal(got[2].cpu().numpy(), offsets) and np.array_equal(got[3].cpu().numpy(), places)
    assert torch.equal(out[:n], x[_gpu(tokens)]) and (out[n:] == 99).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N", [2048, 2056, 4104, 8192, 8200, 12296])
def test_gradients_of_long_rows(dtype, N):
    """One to four pieces a thread, whole turns of the block and remainders; six rows a token, in two lots."""
    rng = np.random.default_rng(N)
    T, each, E = 23, 6, 7
    offsets, places, tokens = R.dispatch(_route(rng, T, each, E, "absent"), E)
    Y, grad, w = _draw(rng, (T * each, N), dtype), _draw(rng, (T, N), dtype), rng.random((T, each)).astype(np.float32)
    gY, gw = api.moe_combine_backward(_rows(grad, dtype, 8), _rows(Y, dtype, 24), _gpu(places), _gpu(w), row_offsets=_gpu(offsets))
    of_rows, of_weights, size = R.combine_backward(grad, Y, places, w, dtype)
    assert np.array_equal(_np(gY)[:len(tokens)], of_rows[:len(tokens)]) and not gY[len(tokens):].any()
    assert (np.abs(gw.double().cpu().numpy() - of_weights) <= (N / 256 + 16) * 2.0 ** -24 * size).all()
    got = _np(api.moe_combine(_rows(Y, dtype, 24), _gpu(places), _gpu(w)))
    want, size = R.combine(Y, places, w)
    assert (np.abs(got - want) <= A.UNIT[dtype] * np.abs(want) * 1.001 + (each + 1) * 2.0 ** -24 * size + 2.0 ** -25).all()


@pytest.mark.parametrize("T,N", [(700, 1000), (300, 4104)])
def test_many_rows_that_no_expert_has_are_cleared(T, N):
    """More of them than the blocks that clear take at once."""
    import torch

    rng = np.random.default_rng(T)
    each = 4
    ids = np.full((T, each), -1, dtype=np.int32)
    ids[rng.integers(0, T, 9), rng.integers(0, each, 9)] = 2
    offsets, places, tokens = R.dispatch(ids, 3)
    assert (T * each - len(tokens)) * N // 8 > 256 * 512
    Y, grad, w = _draw(rng, (T * each, N), A.BF16), _draw(rng, (T, N), A.BF16), rng.random((T, each)).astype(np.float32)
    out = torch.full((T * each, N), 7.0, dtype=torch.bfloat16, device="cuda")
    gY, gw = api.moe_combine_backward(_gpu(grad, A.BF16), _gpu(Y, A.BF16), _gpu(places), _gpu(w), row_offsets=_gpu(offsets), out_Y=out)
    of_rows, of_weights, size = R.combine_backward(grad, Y, places, w, A.BF16)
    assert gY is out and np.array_equal(_np(gY)[:len(tokens)], of_rows[:len(tokens)]) and not gY[len(tokens):].any()
    assert (np.abs(gw.double().cpu().numpy() - of_weights) <= (N / 256 + 16) * 2.0 ** -24 * size).all()


def test_norm_and_swiglu_of_millions_of_rows():
    """More rows than one launch takes, with strides of their own."""
    M, K, period = 2 ** 21 + 70001, 16, 997
    rng = np.random.default_rng(60)
    x, res = _draw(rng, (period, K), A.F16), _draw(rng, (period, K), A.F16)
    at = np.arange(M) % period
    # (the rows repeat, the last of a period next to the first of the next: an odd number of them, so that no launch begins where one does)
    many = lambda a, pad: _rows(a, A.F16, pad)[_gpu(at)] if not pad else _rows(a[at], A.F16, pad)  # noqa: E731
    q, s, h, y = api.w4a8_norm_quantize(many(x, 8), residual=many(res, 0), want_y=True)
    want = R.norm_quantise(x, res, None, 1e-6, A.F16)
    for got, one in ((q, want[0]), (s, want[1]), (h, want[2]), (y, A.round_to(want[3], A.F16))):
        assert np.array_equal(got.cpu().numpy().astype(np.float32), one.astype(np.float32)[at])
    q, s = api.w4a8_swiglu_quantize(many(x, 8))
    one_q, one_s = (t.cpu().numpy() for t in api.w4a8_swiglu_quantize(_gpu(x, A.F16)))
    assert np.array_equal(q.cpu().numpy(), one_q[at]) and np.array_equal(s.cpu().numpy(), one_s[at])


@pytest.mark.parametrize("T,each,E", [(3000, 1, 1), (70000, 2, 1), (40000, 1, 256), (2048, 1, 1), (1025, 2, 255)])
def test_dispatch_of_one_expert_and_of_all(T, each, E):
    """As many blocks an expert as there are, or one each."""
    import torch

    rng = np.random.default_rng(T)
    ids = _route(rng, T, each, E, "absent")
    offsets, places, tokens = R.dispatch(ids, E)
    x = _gpu(rng.integers(-127, 128, (T, 16)).astype(np.int8))
    rows, _, got_offsets, got_places = api.moe_dispatch(x, _gpu(ids), E)
    assert np.array_equal(got_offsets.cpu().numpy(), offsets) and np.array_equal(got_places.cpu().numpy(), places)
    assert torch.equal(rows[:len(tokens)], x[_gpu(tokens)])
