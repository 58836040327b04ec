"""GPU tests of layer norm and its gradients against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as O
from gpu_util import U32, device, gamma, to_dev

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _lsgd():
    from paper_1808_07217_amd import lsgd as L
    return L


def _np(t):
    return t.to(torch.float32).cpu().numpy().astype(np.float64)


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _rounded(bound, ref, dtype):
    """With the rounding of a bf16 result."""
    return bound + 2.0 ** -8 * (np.abs(ref) + bound) if dtype == torch.bfloat16 else bound


def _check_forward(got, X, w, b):
    """The mean is rounded once. d = (x - hi) - lo rounds twice (the first time a value next to
    d: |lo| <= u |mean|), its square's mean to 4 u, rstd once more: n = d rstd is off by
    2 + 3 + 1 u, and y = n w + b rounds once, then to its type."""
    y, mean, rstd = got
    ry, rm, rr = O.layer_norm(X, w, b, EPS)
    assert np.all(np.abs(_np(mean) - rm) <= 1.01 * U32 * np.abs(rm) + 2.0 ** -50 * np.abs(X).mean(2))
    assert np.all(np.abs(_np(rstd) - rr) <= 4 * U32 * rr)
    n = np.abs((X - rm[..., None]) * rr[..., None])
    # what is left of the mean's own rounding, from fp64 sums in any order and from `lo`
    rest = (2.0 ** -46 * np.abs(rm) + 2.0 ** -50 * np.abs(X).mean(2)) * rr
    bound = (8 * U32 * n + rest[..., None]) * np.abs(w)[:, None] + 1.01 * U32 * np.abs(ry) + 2.0 ** -140
    err = np.abs(_np(y) - ry)
    bound = _rounded(bound, ry, y.dtype)
    assert np.all(err <= bound), np.max(err / bound)


def _check_backward(got, dY, X, mean, rstd, w):
    """n rounds twice, e = dy w once. A row's sums are added along at most 40 + N / 1024
    terms one after the other, a column's along the rows that a thread takes of a strip (at most 16,
    or a 256th of all groups' rows) and up to 64 threads'. Rows of up to 8 columns are
    computed in fp64."""
    dx, dw, db = got
    G, M, N = X.shape
    rx, rw, rb = O.layer_norm_backward(dY, X, mean, rstd, w)
    r = rstd[..., None]
    n, e = (X - mean[..., None]) * r, dY * w[:, None]
    a = lambda t: np.abs(t)  # noqa: E731
    c1, c2 = e.mean(2, keepdims=True), (e * n).mean(2, keepdims=True)
    if N <= 8:
        bound = 2.0 ** -45 * r * (a(e) + a(c1) + a(n * c2)) + 1.01 * U32 * a(rx) + 2.0 ** -140
    else:
        D = 46 + N // 1024
        e1, e2 = gamma(D) * a(e).mean(2, keepdims=True), gamma(D) * a(e * n).mean(2, keepdims=True)
        bound = a(r) * (U32 * a(e) + e1 + a(n) * e2 + 2.1 * U32 * a(n * c2)
                        + 4 * U32 * (a(e) + a(c1) + a(n * c2))) + 1.01 * U32 * a(rx) + 2.0 ** -140
    err, bound = np.abs(_np(dx) - rx), _rounded(bound, rx, dx.dtype)
    assert np.all(err <= bound), np.max(err / bound)
    if dw is None:
        return
    R = min(M, -(-M // max(1, 256 // G)) + 16) + 64
    assert np.all(np.abs(_np(dw) - rw) <= gamma(R + 3) * np.abs(dY * n).sum(1) + 2.0 ** -140)
    assert np.all(np.abs(_np(db) - rb) <= gamma(R) * np.abs(dY).sum(1) + 2.0 ** -140)


def _inputs(shape, xt, yt, seed=None, far=3.0):
    rng = np.random.default_rng(sum(shape) if seed is None else seed)
    G, M, N = shape
    X = rng.standard_normal(shape) * np.exp(rng.standard_normal((G, M, 1))) + far * rng.standard_normal((G, M, 1))
    X, dY = to_dev(X.astype(np.float32)).to(xt), to_dev(rng.standard_normal(shape).astype(np.float32)).to(yt)
    w, b = (to_dev(rng.standard_normal((G, N)).astype(np.float32)) for _ in range(2))
    return X, dY, w, b


# each number of threads and vectors a row takes, narrow rows, one row, many strips
SHAPES = [(1, 1, 1), (2, 5, 1), (3, 7, 2), (2, 300, 3), (1, 33, 8), (2, 5, 9), (3, 17, 128), (2, 16, 129),
          (1, 65, 512), (2, 9, 513), (1, 6, 1024), (1, 5, 1027), (2, 3, 2049), (1, 3, 4096), (1, 3, 4099),
          (1, 2, 8192), (1, 3, 8195), (1, 2, 16384), (1, 5, 16385), (2, 2, 40003), (1, 5000, 33),
          (3, 1537, 771), (300, 1, 130), (40, 70, 20), (2, 50, 13), (1, 77, 63), (2, 400, 64), (2, 40, 300),
          (1, 30, 256), (3, 999, 16), (2, 260, 32), (2, 37, 1530), (1, 41, 1537), (3, 45, 2303), (2, 29, 5555),
          (2, 11, 12001), (1, 7, 12289), (1, 9, 383), (1, 9001, 1100), (1, 5001, 2063), (1, 1100, 8200)]


@pytest.mark.parametrize("types", ["fp32 fp32", "bf16 bf16", "fp32 bf16", "bf16 fp32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_matches_oracle(shape, types):
    L = _lsgd()
    print(f"layer norm {shape} {types}", flush=True)
    xt, yt = map(_dt, types.split())
    X, dY, w, b = _inputs(shape, xt, yt)
    got = L.layer_norm(X, w, b, eps=EPS, out_dtype=yt)
    assert got[0].dtype == yt
    _check_forward(got, _np(X), _np(w), _np(b))
    _, mean, rstd = got
    back = L.layer_norm_backward(dY, X, mean, rstd, w)
    assert back[0].dtype == xt
    _check_backward(back, _np(dY), _np(X), _np(mean), _np(rstd), _np(w))
    # the same bits again, and with the parameters' gradients left out
    again = L.layer_norm_backward(dY, X, mean, rstd, w)
    assert all(torch.equal(p, q) for p, q in zip(back, again))
    alone = L.layer_norm_backward(dY, X, mean, rstd, w, parameters=False)
    assert torch.equal(alone[0], back[0]) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("shape", [(2, 5, 33), (1, 3, 20000)])
def test_without_weight_and_bias(shape):
    L = _lsgd()
    print(f"layer norm bare {shape}", flush=True)
    X, dY, w, b = _inputs(shape, torch.float32, torch.float32)
    one, zero = np.ones((shape[0], shape[2])), np.zeros((shape[0], shape[2]))
    _check_forward(L.layer_norm(X), _np(X), one, zero)
    _check_forward(L.layer_norm(X, w), _np(X), _np(w), zero)
    _check_forward(L.layer_norm(X, None, b), _np(X), one, _np(b))
    _, mean, rstd = L.layer_norm(X)
    _check_backward(L.layer_norm_backward(dY, X, mean, rstd), _np(dY), _np(X), _np(mean), _np(rstd), one)


def test_rows_far_from_zero_and_large_ones():
    """Means of 10^4 deviations, values whose squares leave fp32's range, constant rows, and
    rows of zeros: the statistics are those of the values."""
    L = _lsgd()
    print("layer norm extremes", flush=True)
    rng = np.random.default_rng(3)
    for N in (40, 700, 5000, 20000):
        X = rng.standard_normal((1, 6, N))
        X[0, 0] += 1e4
        X[0, 1] = 1e4 + 1e-2 * X[0, 1]
        X[0, 2] *= 1e25
        X[0, 3] *= 1e-30
        X[0, 4] = -77.25
        X[0, 5] = 0
        Xd = to_dev(X.astype(np.float32))
        w, b = (to_dev(rng.standard_normal((1, N)).astype(np.float32)) for _ in range(2))
        got = L.layer_norm(Xd, w, b)
        _check_forward(got, _np(Xd), _np(w), _np(b))
        assert torch.equal(got[0][0, 4:], b.expand(2, N))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_one_column_and_equal_gradients(dtype):
    """A row of one value, and rows whose dy w is one number throughout (a power of two, whose sums
    are exact): no gradient at all, not even a rounding of one."""
    L = _lsgd()
    print(f"layer norm one column {dtype}", flush=True)
    dt = _dt(dtype)
    X, dY, w, _ = _inputs((3, 200, 1), dt, dt)
    y, mean, rstd = L.layer_norm(X, w)
    dx, dw, db = L.layer_norm_backward(dY, X, mean, rstd, w)
    assert not dx.any() and not dw.any() and not y.any()
    for N in (4, 32, 64, 1024, 8192):
        X = to_dev(np.tile([1.5, -1.5], (1, 5, N // 2)).astype(np.float32)).to(dt)
        _, mean, rstd = L.layer_norm(X)
        dx, dw, db = L.layer_norm_backward(torch.full_like(X, 0.25), X, mean, rstd)
        assert not dx.any() and torch.equal(db, torch.full_like(db, 1.25)), N


def test_rows_that_are_not_finite():
    """A NaN or an infinity makes its own row NaN and reaches the gradients of its columns;
    other rows keep their bits."""
    L = _lsgd()
    print("layer norm specials", flush=True)
    for shape in ((2, 6, 40), (1, 6, 3000), (1, 6, 17000)):
        X, dY, w, b = _inputs(shape, torch.float32, torch.float32)
        want = L.layer_norm(X, w, b)
        dx = L.layer_norm_backward(dY, X, *want[1:], w)[0]
        Z = X.clone()
        Z[0, 1, 3], Z[0, 3, 0], Z[0, 4, 30] = float("nan"), float("inf"), float("-inf")
        y, mean, rstd = L.layer_norm(Z, w, b)
        ok = [0, 2, 5]
        assert torch.isnan(y[0, [1, 3, 4]]).all() and torch.equal(y[0, ok], want[0][0, ok])
        got = L.layer_norm_backward(dY, Z, mean, rstd, w)
        assert torch.isnan(got[0][0, [1, 3, 4]]).all() and torch.equal(got[0][0, ok], dx[0, ok])
        assert torch.isnan(got[1][0]).all() and not torch.isnan(got[2]).any()


def test_strided_views_and_shared_tensors():
    """Rows and groups of views, parameters inside flat rows, one parameter for all groups;
    nothing beside the results changes."""
    L = _lsgd()
    print("layer norm strided", flush=True)
    rng = np.random.default_rng(5)
    K, M, N = 3, 37, 131
    for dt in (torch.float32, torch.bfloat16):
        room = to_dev(rng.standard_normal((K, M + 3, N + 9)).astype(np.float32)).to(dt)
        X, dY = room[:, 2:M + 2, 5:N + 5], room[:, :M, 1:N + 1]
        flat = to_dev(rng.standard_normal((K, 500)).astype(np.float32))
        w, b = flat[:, 7:7 + N], flat[:1, 200:200 + N].expand(K, N)
        out = torch.full((M, K, N + 3), 7.0, device=device(), dtype=dt)
        y = out[:, :, 1:N + 1].transpose(0, 1)
        got = L.layer_norm(X, w, b, out=y)
        assert got[0] is y
        _check_forward((y.contiguous(), *got[1:]), _np(X), _np(w), _np(b))
        y.fill_(7.0)
        assert (out == 7.0).all()
        grads = torch.full((K, 500), 7.0, device=device())
        dxs = torch.full((K, M + 1, N + 2), 7.0, device=device(), dtype=dt)
        dw, db, dx = grads[:, 7:7 + N], grads[:, 200:200 + N], dxs[:, 1:, 1:N + 1]
        res = L.layer_norm_backward(dY, X, *got[1:], w, out=dx, dweight=dw, dbias=db)
        assert res[0] is dx and res[1] is dw and res[2] is db
        _check_backward((dx.contiguous(), dw.contiguous(), db.contiguous()), _np(dY), _np(X),
                        _np(got[1]), _np(got[2]), _np(w))
        for t in (dw, db, dx):
            t.fill_(7.0)
        assert (grads == 7.0).all() and (dxs == 7.0).all()
    # one matrix for every group
    X = X[:1].expand(K, M, N)
    _check_forward(L.layer_norm(X, w, b), _np(X), _np(w), _np(b))


def test_refusals_of_the_binding():
    L = _lsgd()
    X, dY, w, b = _inputs((2, 5, 33), torch.float32, torch.float32)
    _, mean, rstd = L.layer_norm(X, w, b)
    for bad in (dict(out=X), dict(out=X[:, :4]), dict(weight=w[:1]), dict(bias=b.double()),
                dict(weight=w.t().contiguous().t()), dict(out_dtype=torch.float16)):
        with pytest.raises(ValueError):
            L.layer_norm(X, **{"weight": w, "bias": b, **bad})
    with pytest.raises(L.LsgdError):
        L.layer_norm(X, w, b, eps=0.0)
    for bad in (dict(out=X), dict(out=dY), dict(dweight=w), dict(dbias=mean[:, :1].expand(2, 33)),
                dict(dweight=b, dbias=b), dict(parameters=False, dbias=b), dict(out=X.bfloat16())):
        with pytest.raises((ValueError, L.LsgdError)):
            L.layer_norm_backward(dY, X, mean, rstd, w, **bad)
    for bad in ((dY[:1], X, mean, rstd), (dY, X, mean[:, :4], rstd), (dY, X, mean, rstd.double()),
                (dY, X, mean.cpu(), rstd), (dY, X, mean, rstd.t().contiguous().t())):
        with pytest.raises((ValueError, L.LsgdError)):
            L.layer_norm_backward(*bad, w)


@pytest.mark.parametrize("shape", [(2, 6, 9), (1, 5, 200), (1, 4, 3000), (1, 3, 17000)])
def test_gradients_against_differences(shape):
    """The kernels' gradients against quotients of the loss sum(y dy) of the formula in float64 at
    the kernels' inputs: h^2 of the third derivative and the rounding of two sums over 2 h
    are far below fp32's rounding of the gradients, which is what the bound holds."""
    L = _lsgd()
    print(f"layer norm differences {shape}", flush=True)
    X, dY, w, b = _inputs(shape, torch.float32, torch.float32, far=0.5)
    _, mean, rstd = L.layer_norm(X, w, b)
    grads = [_np(t) for t in L.layer_norm_backward(dY, X, mean, rstd, w)]
    args = [_np(X), _np(w), _np(b)]
    d = _np(dY)
    rng = np.random.default_rng(1)
    h = 1e-4
    for i, g in enumerate(grads):
        for at in [tuple(rng.integers(0, n) for n in g.shape) for _ in range(12)]:
            terms = []
            for s in (h, -h):
                a = [v.copy() for v in args]
                a[i][at] += s
                terms.append(O.layer_norm(a[0], a[1], a[2], EPS)[0] * d)
            quotient = (terms[0] - terms[1]).sum() / (2 * h)
            size = np.abs(g).max()
            assert abs(quotient - g[at]) <= 2e-5 * size, (i, at)


def test_on_a_side_stream_and_in_a_graph():
    L = _lsgd()
    print("layer norm stream and graph", flush=True)
    X, dY, w, b = _inputs((2, 3000, 300), torch.float32, torch.float32)

    def step():
        y, mean, rstd = L.layer_norm(X, w, b)
        return (y, mean, rstd) + L.layer_norm_backward(dY, X, mean, rstd, w)

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        X.copy_(torch.randn(X.shape, device=device()) + k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))


@pytest.mark.parametrize("shape", [(1, 40000, 33), (2, 3000, 700), (1, 140, 17000)])
def test_whatever_the_workspace_holds(shape):
    """The caller's own workspace of exactly the size asked for: the same bits, and nothing
    behind its end written."""
    L = _lsgd()
    print(f"layer norm workspace {shape}", flush=True)
    G, M, N = shape
    X, dY, w, b = _inputs(shape, torch.float32, torch.float32)
    _, mean, rstd = L.layer_norm(X, w, b)
    dx, dw, db = L.layer_norm_backward(dY, X, mean, rstd, w)
    nb = L._norm_workspace(G, M, N)
    assert nb > 0
    ws = torch.empty(nb + 64, device=device(), dtype=torch.uint8)
    for fill in (0, 255):
        ws.fill_(fill)
        ws[nb:] = 77
        x2, w2, b2 = torch.full_like(dx, 7.0), torch.full_like(dw, 7.0), torch.full_like(db, 7.0)
        assert L._lib.lsgd_layer_norm_backward(
            0, 0, G, M, N, dY.data_ptr(), N, M * N, X.data_ptr(), N, M * N, mean.data_ptr(),
            rstd.data_ptr(), w.data_ptr(), N, x2.data_ptr(), N, M * N, w2.data_ptr(), N, b2.data_ptr(),
            N, ws.data_ptr(), nb, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(x2, dx) and torch.equal(w2, dw) and torch.equal(b2, db)
        assert (ws[nb:] == 77).all()


@pytest.mark.parametrize("N", [33000, 1000])
def test_past_32_bit_offsets(N):
    """More than 2^31 elements: the last rows are those of the same rows alone, and the
    parameters' gradients the sum of the halves'."""
    L = _lsgd()
    print(f"layer norm past 32 bits {N}", flush=True)
    gen = torch.Generator(device=device()).manual_seed(4)
    M = 2 ** 31 // N + 77
    X = torch.randn(1, M, N, generator=gen, device=device(), dtype=torch.bfloat16)
    dY = torch.randn(1, M, N, generator=gen, device=device(), dtype=torch.bfloat16)
    w, b = (torch.randn(1, N, generator=gen, device=device()) for _ in range(2))
    y, mean, rstd = L.layer_norm(X, w, b)
    tail = L.layer_norm(X[:, -65:], w, b)
    assert torch.equal(y[:, -65:], tail[0]) and torch.equal(mean[:, -65:], tail[1])
    assert torch.equal(rstd[:, -65:], tail[2])
    del y
    dx, dw, db = L.layer_norm_backward(dY, X, mean, rstd, w)
    end = L.layer_norm_backward(dY[:, -65:], X[:, -65:], *tail[1:], w)
    assert torch.equal(dx[:, -65:], end[0])
    del dx
    sums, size = torch.zeros(N, dtype=torch.float64, device=device()), torch.zeros(N, device=device())
    for m in range(0, M, 8192):
        sums += dY[0, m:m + 8192].sum(0, dtype=torch.float64)
        size += dY[0, m:m + 8192].abs().sum(0, dtype=torch.float32)
    assert bool(((db[0] - sums).abs() <= gamma(M // 256 + 60) * size).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("N", [5, 40, 64, 100, 700, 1100, 2000, 4000, 5000, 7000, 8192, 9000, 16384, 20001])
def test_constant_rows_far_out(N, dtype):
    """One value throughout, so far from zero that it leaves fp32's range in deviations of
    eps: no deviations, and the gradient that is left."""
    L = _lsgd()
    print(f"layer norm constant rows {N} {dtype}", flush=True)
    dt = _dt(dtype)
    rng = np.random.default_rng(N)
    X = np.repeat(np.array([2e36, -3e37, 1.0, 3e38])[None, :, None], N, 2)
    X = to_dev(X.astype(np.float32)).to(dt)
    dY, w, b = (to_dev(rng.standard_normal(s).astype(np.float32)) for s in ((1, 4, N), (1, N), (1, N)))
    dY = (dY * 1e-3).to(dt)
    for eps in (1e-5, 1e-12):
        y, mean, rstd = L.layer_norm(X, w, b, eps=eps)
        assert torch.equal(y[0], b.to(dt).expand(4, N)) and torch.equal(mean[0], X[0, :, 0].float())
        got = L.layer_norm_backward(dY, X, mean, rstd, w)
        assert not got[1].any()
        _check_backward(got, _np(dY), _np(X), _np(mean), _np(rstd), _np(w))


@pytest.mark.parametrize("types", ["fp32 fp32", "fp32 bf16"])
@pytest.mark.parametrize("N", [2, 5, 9, 40, 100, 130, 400, 700, 1100, 1500, 2000, 2500, 4000, 5000, 8000, 9000,
                               16000, 20001])
def test_gradients_of_rows_far_from_zero(N, types):
    """Means of 10^4 and 10^6 deviations: the gradients of the values' own mean, which the fp32 one
    that is handed over misses by up to 6% of a deviation. x - mean as it was written is rounded to u,
    times rstd once more; what is taken off is the mean of those, rounded, as is the difference."""
    L = _lsgd()
    print(f"layer norm far rows {N} {types}", flush=True)
    xt, yt = map(_dt, types.split())
    rng = np.random.default_rng(N)
    M = 21
    X = rng.standard_normal((1, M, N))
    X[0, 0:5] += 1e4
    X[0, 5:10] -= 1e6
    X[0, 10:13] = 1e4 + 1e-2 * X[0, 10:13]
    X[0, 13:15] = 1e9 + 1e4 * X[0, 13:15]
    X[0, 15:16] = 1e34 + 1e29 * X[0, 15:16]
    X = to_dev(X.astype(np.float32)).to(xt)
    dY, w = (to_dev(rng.standard_normal(s).astype(np.float32)) for s in ((1, M, N), (1, N)))
    dY = dY.to(yt)
    _, mean, rstd = L.layer_norm(X, w)
    dx, dw, db = L.layer_norm_backward(dY, X, mean, rstd, w)
    x, d, r = _np(X), _np(dY), _np(rstd)[..., None]
    own = x.mean(2)
    far = np.abs(own) * r[..., 0] >= 2100
    assert far[0, :13].sum() >= 10 and not far[0, 16:].any()
    own = np.where(far, own, _np(mean))
    rx, rw, rb = O.layer_norm_backward(d, x, own, _np(rstd), _np(w))
    a = lambda t: np.abs(t)  # noqa: E731
    av = lambda t: t.mean(2, keepdims=True)  # noqa: E731
    n, e, off = (x - own[..., None]) * r, d * _np(w)[:, None], 2.0 ** -24 * a(own[..., None]) * r
    en = U32 * (4 * (a(n) + off) + np.where(far[..., None], 4 * (av(a(n)) + off), 0))
    D = 46 + N // 1024
    bound = r * (a(av(e * n)) * en + (a(n) + en) * (av(a(e) * en) + gamma(D) * av(a(e) * (a(n) + off)))
                 + gamma(D) * av(a(e)) + 6 * U32 * (a(e) + a(av(e)) + a(n * av(e * n)))) + 1.01 * U32 * a(rx)
    err, bound = a(_np(dx) - rx), _rounded(bound, rx, dx.dtype)
    assert np.all(err <= bound), np.max(err / bound)
    assert np.all(a(_np(dw) - rw) <= (a(d) * en).sum(1) + gamma(M + 3) * a(d * n).sum(1))
    assert np.all(a(_np(db) - rb) <= gamma(M + 3) * a(d).sum(1))


# of each the roundings of a column's sum one after the other: kept over four rows and joined in
# fp64 (a thread's three, its workgroup's slot, its strip and the result), or over 32 rows
@pytest.mark.parametrize("shape, D", [((129, 80000, 500), 6), ((129, 4000, 8000), 6), ((1, 60000, 8000), 6),
                                      ((129, 200000, 40), 6), ((300, 100000, 6), 6), ((129, 4000, 17000), 6),
                                      ((129, 40000, 1100), 34), ((200, 8000, 4200), 34), ((129, 6000, 9000), 34)])
def test_sums_over_any_number_of_rows(shape, D):
    """Columns of one sign, whose sums every rounding moves, in groups that share them: no more of
    them for more rows or groups."""
    L = _lsgd()
    print(f"layer norm sums {shape}", flush=True)
    G, M, N = shape
    gen = torch.Generator(device=device()).manual_seed(sum(shape))
    sign = torch.where(torch.arange(N, device=device()) % 2 == 0, 1.0, -1.0)
    X = (torch.randn((1, M, N), generator=gen, device=device()) * 0.1 + sign).bfloat16()
    dY = torch.rand((1, M, N), generator=gen, device=device()) * 0.1 + 0.05
    _, mean, rstd = L.layer_norm(X)
    mean, rstd = (t.repeat(G, 1) for t in (mean, rstd))
    dx, dw, db = L.layer_norm_backward(dY.expand(shape), X.expand(shape), mean, rstd)
    del dx
    want, size, sums = (torch.zeros(N, device=device(), dtype=torch.float64) for _ in range(3))
    for m in range(0, M, 5000):
        at = slice(m, m + 5000)
        d = dY[0, at].double()
        dn = d * ((X[0, at].double() - mean[0, at, None].double()) * rstd[0, at, None].double())
        want += dn.sum(0)
        size += dn.abs().sum(0)
        sums += d.sum(0)
    # (n is rounded twice, its product with dy once more)
    assert bool(((dw.double() - want).abs() <= gamma(D + 3) * size).all())
    assert bool(((db.double() - sums).abs() <= gamma(D) * sums).all())
    assert torch.equal(dw, dw[:1].expand(G, N)) and torch.equal(db, db[:1].expand(G, N))


@pytest.mark.parametrize("N", [16385, 40003, 2 ** 24 + 5])
def test_statistics_of_long_rows(N):
    """One gradient throughout: its mean is itself, whatever the length, to the roundings of eight terms
    and a few more."""
    L = _lsgd()
    print(f"layer norm long rows {N}", flush=True)
    gen = torch.Generator(device=device()).manual_seed(N)
    X = torch.randn(1, 2, N, generator=gen, device=device())
    dY = torch.full_like(X, 0.1)
    _, mean, rstd = L.layer_norm(X)
    dx, _, _ = L.layer_norm_backward(dY, X, mean, rstd)
    n = (X - mean[..., None]) * rstd[..., None]
    # (sum n is that of the mean's rounding and of n's own, u |x| and 2 u |n| a term)
    size = 0.1 * (1 + n.abs() * n.abs().mean(2, keepdim=True))
    assert bool((dx.abs() <= gamma(16) * rstd[..., None] * size).all())


@pytest.mark.parametrize("N", [4, 40, 64, 100, 400, 700, 1100, 2000, 4000, 5000, 8000, 9000, 16000, 20001])
def test_rows_as_wide_as_fp32(N):
    """Finite rows whose values lie further from their mean than fp32 reaches, or whose
    deviation's inverse is subnormal: results as exact as others', but for rstd's own lost bits."""
    L = _lsgd()
    print(f"layer norm wide rows {N}", flush=True)
    big = float(np.finfo(np.float32).max)
    rng = np.random.default_rng(N)
    X = np.empty((1, 8, N))
    X[0, 0] = -3e38
    X[0, 0, ::4] = 3e38
    X[0, 1] = big
    X[0, 1, N // 3] = -big
    X[0, 2] = np.where(np.arange(N) % 2, big, -big)
    X[0, 3] = rng.uniform(-big, big, N)
    X[0, 4] = big
    X[0, 5] = 1e-40
    X[0, 5, 1] = -3e38
    X[0, 6] = 1e38 + 1e37 * rng.standard_normal(N)
    X[0, 7] = rng.standard_normal(N)
    X = to_dev(X.astype(np.float32))
    dY, w, b = (to_dev(rng.standard_normal(s).astype(np.float32)) for s in ((1, 8, N), (1, N), (1, N)))
    y, mean, rstd = L.layer_norm(X, w, b)
    x, wd = _np(X), _np(w)
    ry, rm, rr = O.layer_norm(x, wd, _np(b), EPS)
    assert np.all(np.abs(_np(mean) - rm) <= 1.01 * U32 * np.abs(rm) + 2.0 ** -50 * np.abs(x).mean(2))
    assert np.all(np.abs(_np(rstd) - rr) <= 4 * U32 * rr + 1.01 * 2.0 ** -150)
    n = np.abs((x - rm[..., None]) * rr[..., None])
    rest = (2.0 ** -46 * np.abs(rm) + 2.0 ** -50 * np.abs(x).mean(2)) * rr
    bound = (8 * U32 * n + rest[..., None]) * np.abs(wd)[:, None] + 1.01 * U32 * np.abs(ry)
    assert np.all(np.abs(_np(y) - ry) <= bound), np.max(np.abs(_np(y) - ry) / bound)
    _check_backward(L.layer_norm_backward(dY, X, mean, rstd, w), _np(dY), x, _np(mean), _np(rstd), wd)


def test_sizes_past_32_bits_are_refused():
    """Groups, rows or columns past the ABI's integers, in views of a few values: refused before
    anything is made."""
    L = _lsgd()
    print("layer norm refused sizes", flush=True)
    x = torch.ones(1, 1, 1, device=device())
    n = 2 ** 32 + 1
    for X in (x.expand(n, 1, 1), x.expand(1, n, 1)):
        for call in (L.layer_norm, L.quantise_rows, L.quantise_blocks, L.orthogonalise,
                     lambda X: L.layer_norm_backward(X, X, X[..., 0], X[..., 0])):
            with pytest.raises(ValueError, match="2\\^31"):
                call(X)
    for call in (L.gradient_norm, lambda t: L.clip_gradients(t, 1.0)):
        with pytest.raises(ValueError, match="2\\^31"):
            call([x.expand(n, 1, 1)])


@pytest.mark.parametrize("N", [7, 40, 700, 1100, 2500, 8000, 9000, 20001])
def test_far_rows_in_strided_views(N):
    """Rows far from zero among others, with pitches, without weights and without parameters' gradients:
    the bits of contiguous ones."""
    L = _lsgd()
    print(f"layer norm far strided {N}", flush=True)
    gen = torch.Generator(device=device()).manual_seed(N)
    G, M = 3, 37
    room = torch.randn(G, M + 2, N + 5, generator=gen, device=device())
    room[:, ::3] += 3e4
    room[:, 1::7] -= 1e32
    more = torch.randn(M, G, N + 3, generator=gen, device=device()).bfloat16()
    X, dY = room[:, 1:M + 1, 3:N + 3], more[:, :, 1:N + 1].transpose(0, 1)
    w = torch.randn(1, N, generator=gen, device=device()).expand(G, N)
    for weight in (None, w):
        _, mean, rstd = L.layer_norm(X, weight)
        want = L.layer_norm_backward(dY.contiguous(), X.contiguous(), mean, rstd, weight)
        got = L.layer_norm_backward(dY, X, mean, rstd, weight)
        assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(got, want))
        alone = L.layer_norm_backward(dY, X, mean, rstd, weight, parameters=False)
        assert torch.equal(alone[0], want[0])
