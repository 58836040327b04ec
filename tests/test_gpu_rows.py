"""GPU tests of tensors in 8-bit integers with a scale for each row and their grouped
product against the float64 oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import layer_oracle as O
from gpu_util import U32, device, to_dev

pytestmark = pytest.mark.gpu


def _lsgd():
    from paper_1808_07217_amd import lsgd as L
    return L


def _np(t):
    return t.to(torch.float32).cpu().numpy().astype(np.float64)


def _dt(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _check_rows(got, X):
    """Bit for bit the oracle's integers and scales, padding included."""
    q, s = O.quantise_rows(X)
    assert got.n == X.shape[2]
    assert tuple(got.q.shape) == q.shape and tuple(got.scale.shape) == s.shape
    np.testing.assert_array_equal(_np(got.scale), s)
    np.testing.assert_array_equal(got.q.cpu().numpy().astype(np.float64), q)


# each number of threads and vectors a row takes, and sizes on both sides of a tile's edge
SHAPES = [(1, 1, 1), (2, 1, 7), (3, 5, 1), (2, 16, 128), (1, 64, 512), (2, 129, 127), (3, 130, 257),
          (1, 17, 1025), (1, 700, 9), (2, 127, 641), (2, 3, 2049), (1, 5, 4097), (1, 3, 8191), (1, 2, 16384),
          (1, 3, 16385), (1, 2, 40001), (1, 1030, 3), (2, 513, 513), (300, 1, 130), (2, 9, 1530), (3, 9, 1537),
          (3, 13, 2303), (2, 7, 5555), (1, 5, 12001), (1, 5, 12289)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantise_matches_oracle(shape, dtype):
    L = _lsgd()
    print(f"quantise rows {shape} {dtype}", flush=True)
    rng = np.random.default_rng(sum(shape))
    X = rng.standard_normal(shape) * np.exp(3 * rng.standard_normal((1, shape[1], 1)))
    Xd = to_dev(X.astype(np.float32)).to(_dt(dtype))
    X = _np(Xd)
    _check_rows(L.quantise_rows(Xd), X)
    both, t = L.quantise_rows(Xd, both=True)
    _check_rows(both, X)
    _check_rows(t, X.transpose(0, 2, 1))


def test_quantise_extremes():
    """Ties, neighbours of ties, zeros, subnormals, the largest values, and rows and columns
    with infinities and NaN."""
    L = _lsgd()
    print("quantise rows extremes", flush=True)
    n = np.arange(300)
    X = np.zeros((1, 12, 300), np.float32)
    X[0, 0] = n % 127 + 0.5          # scale 1: ties
    X[0, 0, 0] = 127
    X[0, 1] = np.nextafter(X[0, 0], np.float32(1e9))
    X[0, 1, 0] = 127
    X[0, 2] = np.nextafter(X[0, 0], np.float32(0))
    X[0, 2, 0] = -127
    X[0, 3] = (n % 127 + 0.5) * np.float32(0.1 / 127)   # ties of a scale that is not exact
    X[0, 3, 0] = 0.1
    X[0, 4] = (n - 150) * 1e-45
    X[0, 5] = np.finfo(np.float32).max * (1 - n / 400)
    X[0, 6] = 2.0 ** -126 * (n - 20.0)
    X[0, 7, 250] = 1e-45
    X[0, 8] = n - 150
    X[0, 8, 3] = np.inf
    X[0, 9] = n - 150
    X[0, 9, 299] = np.nan
    X[0, 10] = -np.inf
    for dt in (torch.float32, torch.bfloat16):
        Xd = to_dev(X).to(dt)
        got, t = L.quantise_rows(Xd, both=True)
        _check_rows(got, _np(Xd))
        _check_rows(L.quantise_rows(Xd), _np(Xd))
        _check_rows(t, _np(Xd).transpose(0, 2, 1))
        assert torch.isnan(got.scale[0, 8:11]).all() and torch.isnan(t.scale).all()


@pytest.mark.parametrize("N", [5, 100, 128])
def test_quantise_specials_in_one_tile(N):
    """Matrices of a single tile, some of them with zeros, subnormals, the largest value, infinities
    and NaN; a column's special leaves the other columns as they are."""
    L = _lsgd()
    print(f"quantise rows one tile {N}", flush=True)
    rng = np.random.default_rng(N)
    X = rng.standard_normal((4, 90, N)).astype(np.float32)
    X[0, 3], X[0, 4], X[0, 5, N - 1] = 0, 1e-42, np.finfo(np.float32).max
    X[1, 89, 0], X[1, 7, N - 1] = np.nan, -np.inf
    X[2] = 0
    for dt in (torch.float32, torch.bfloat16):
        Xd = to_dev(X).to(dt)
        q, t = L.quantise_rows(Xd, both=True)
        _check_rows(q, _np(Xd))
        _check_rows(t, _np(Xd).transpose(0, 2, 1))


@pytest.mark.parametrize("shape", [(2, 300, 700), (1, 5000, 90), (1, 129, 3)])
def test_quantise_whatever_the_workspace_holds(shape):
    """The caller's own workspace of exactly the size asked for: the same bits, nothing behind its end
    or the results' written."""
    L = _lsgd()
    print(f"quantise rows workspace {shape}", flush=True)
    G, M, N = shape
    X = to_dev(np.random.default_rng(1).standard_normal(shape).astype(np.float32))
    q, t = L.quantise_rows(X, both=True)
    nb = L._rows_workspace(G, M, N)
    assert nb > 0
    for fill in (0, 255):
        room = [torch.full((n + 64,), 77, device=device(), dtype=torch.uint8)
                for n in (q.q.numel(), 4 * q.scale.numel(), t.q.numel(), 4 * t.scale.numel(), nb)]
        room[4][:nb] = fill
        assert L._lib.lsgd_quantise_rows(
            0, G, M, N, X.data_ptr(), N, M * N, *[r.data_ptr() for r in room], nb,
            torch.cuda.current_stream().cuda_stream) == 0
        for r, want in zip(room, (q.q, q.scale, t.q, t.scale)):
            assert torch.equal(r[:-64], want.flatten().view(torch.uint8)) and (r[-64:] == 77).all()
        assert (room[4][nb:] == 77).all()


@pytest.mark.parametrize("M,N,dtype", [(7000, 8300, "fp32"), (2 ** 24 + 5, 7, "bf16"),
                                       (700001, 123, "fp32")])
def test_quantise_tensors_past_the_caches(M, N, dtype):
    """Hundreds of MB, whose integers are streamed past the caches: rows and columns as on their own."""
    L = _lsgd()
    print(f"quantise rows streamed {M} {N} {dtype}", flush=True)
    gen = torch.Generator(device=device()).manual_seed(3)
    X = torch.randn(1, M, N, generator=gen, device=device()).to(_dt(dtype))
    q, t = L.quantise_rows(X, both=True)
    alone = L.quantise_rows(X)
    assert torch.equal(alone.q, q.q) and torch.equal(alone.scale, q.scale)
    _check_rows(L.Rows(q.q[:, -40:].contiguous(), q.scale[:, -40:].contiguous(), N), _np(X[:, -40:]))
    for n in (0, N // 2, N - 1):
        column = L.quantise_rows(X[:, :, n].unsqueeze(1).contiguous())
        assert torch.equal(column.q[0, 0], t.q[0, n]) and torch.equal(column.scale[0], t.scale[0, n:n + 1])


def test_quantise_every_quotient():
    """All 2^16 bfloat16 values against scales whose quotients fall near ties, and fp32
    neighbours of every tie of odd scales."""
    L = _lsgd()
    print("quantise rows ties", flush=True)
    bits = torch.arange(0x4000, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    top = bits.max()
    X = torch.stack([torch.cat([bits[-4000:], torch.tensor([float(top) * f], dtype=torch.bfloat16)])
                     for f in (1.0, 1.5, 2.0)])[None].to(device())
    _check_rows(L.quantise_rows(X), _np(X))
    rng = np.random.default_rng(6)
    rows = []
    for _ in range(64):
        top = np.float32(np.exp(rng.uniform(-60, 60)))
        s = np.float32(top / np.float32(127))
        ties = ((np.arange(127) + 0.5) * float(s)).astype(np.float32)
        rows.append(np.concatenate([[top], ties, np.nextafter(ties, np.float32(0)),
                                    np.nextafter(ties, top)]).clip(0, top))
    X = to_dev(np.stack(rows)[None].astype(np.float32))
    _check_rows(L.quantise_rows(X), _np(X))
    _check_rows(L.quantise_rows(-X, both=True)[0], _np(-X))


def test_quantise_strided_and_shared_inputs():
    L = _lsgd()
    rng = np.random.default_rng(5)
    for dt in (torch.float32, torch.bfloat16):
        flat = to_dev(rng.standard_normal(3 * 5000).astype(np.float32)).to(dt)
        X = flat[3:].as_strided((3, 33, 131), (4001, 139, 1), 3)
        print(f"quantise rows strided {dt}", flush=True)
        got, t = L.quantise_rows(X, both=True)
        _check_rows(got, _np(X))
        _check_rows(t, _np(X).transpose(0, 2, 1))
        E = X[:1].expand(4, 33, 131)
        _check_rows(L.quantise_rows(E), _np(E))
        q, t = L.quantise_rows(E, both=True)
        _check_rows(q, _np(E))
        _check_rows(t, _np(E).transpose(0, 2, 1))
        rows = X[0, :1].unsqueeze(0).expand(2, 7, 131)  # one row again and again
        with pytest.raises(L.LsgdError):  # (rows that overlap: a pitch below the columns)
            L.quantise_rows(rows)


def _operands(L, rng, G, M, N, K):
    A = rng.standard_normal((G, M, K)) * np.exp(rng.standard_normal((1, M, 1)))
    Bm = rng.standard_normal((G, N, K)) * np.exp(rng.standard_normal((1, N, 1)))
    return L.quantise_rows(to_dev(A.astype(np.float32))), L.quantise_rows(to_dev(Bm.astype(np.float32)))


def _bound(exact, bias, out):
    """The sum is exact: rounded to fp32, times one scale, and times the other with the bias in
    one rounding: three roundings of the product, the last of the result with it; a bf16
    result rounds once more (2^-8). And fp32's subnormal range."""
    u = U32
    bound = 2.01 * u * np.abs(exact) + 1.01 * u * np.abs(exact + bias) + 2.0 ** -148
    return bound if out != torch.bfloat16 else bound + 2.0 ** -8 * (np.abs(exact + bias) + bound)


def _check_product(C, a, b, bias=None):
    exact = O.product(a.q.cpu().numpy().astype(np.float64), _np(a.scale),
                      b.q.cpu().numpy().astype(np.float64), _np(b.scale))
    add = 0.0 if bias is None else _np(bias)[:, None]
    err = np.abs(_np(C) - (exact + add))
    bound = _bound(exact, add, C.dtype)
    assert np.all(err <= bound), np.max(err / bound)


PRODUCTS = [(1, 1, 1, 1), (2, 3, 5, 7), (1, 16, 16, 128), (1, 1, 300, 1000), (2, 64, 64, 256),
            (2, 65, 63, 129), (3, 33, 130, 640), (1, 128, 256, 512), (1, 257, 129, 300),
            (4, 128, 128, 128), (1, 5, 2050, 4100), (1, 300, 520, 1030), (16, 128, 512, 512)]


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_product_error_bound(shape, out):
    L = _lsgd()
    print(f"rows product {shape} {out}", flush=True)
    rng = np.random.default_rng(sum(shape))
    a, b = _operands(L, rng, *shape)
    _check_product(L.grouped_gemm_rows(a, b, out_dtype=_dt(out)), a, b)
    bias = to_dev(rng.standard_normal((shape[0], shape[2])).astype(np.float32))
    _check_product(L.grouped_gemm_rows(a, b, bias, out_dtype=_dt(out)), a, b, bias)


@pytest.mark.parametrize("shape", [(1, 64, 64, 8192), (2, 3, 130, 20001), (1, 70, 33, 4100),
                                   (2, 1, 66, 150000), (1, 130, 129, 262145)])
def test_product_split_over_the_inner_dimension(shape):
    """Few results and a long inner dimension, and one whose sums leave 32 bits: ranges joined
    by a second launch, whatever the workspace held, the same bits each time."""
    L = _lsgd()
    print(f"rows product split {shape}", flush=True)
    G, M, N, K = shape
    rng = np.random.default_rng(5)
    a, b = _operands(L, rng, *shape)
    bias = to_dev(rng.standard_normal((G, N)).astype(np.float32))
    nb = L._gemm_rows_workspace(0, G, M, N, K)
    assert nb > 0
    for dt, code in ((torch.float32, 0), (torch.bfloat16, 1)):
        C = L.grouped_gemm_rows(a, b, bias, out_dtype=dt)
        _check_product(C, a, b, bias)
        ws = torch.empty(nb + 64, device=device(), dtype=torch.uint8)
        for fill in (0, 255):
            ws.fill_(fill)
            ws[nb:] = 77
            D = torch.full_like(C, 7.0)
            assert L._lib.lsgd_grouped_gemm_rows(
                code, G, M, N, K, a.q.data_ptr(), a.q.stride(0), a.scale.data_ptr(), M, b.q.data_ptr(),
                b.q.stride(0), b.scale.data_ptr(), N, bias.data_ptr(), N, D.data_ptr(), N, M * N,
                ws.data_ptr(), nb, torch.cuda.current_stream().cuda_stream) == 0
            assert torch.equal(C, D) and (ws[nb:] == 77).all()


@pytest.mark.parametrize("K", [131071, 131072, 140000, 300000])
def test_product_of_the_largest_integers(K):
    """Every integer -128 or 127: sums at the ends of 32 bits and past them."""
    L = _lsgd()
    print(f"rows product largest {K}", flush=True)
    Lq = O.up(K, 128)
    q = torch.zeros(1, 3, Lq, dtype=torch.int8, device=device())
    q[0, 0, :K], q[0, 1, :K], q[0, 2, :K] = -128, 127, -127
    s = torch.tensor([[1.0, 2.0 ** -20, 0.3]], device=device())
    x = L.Rows(q, s, K)
    _check_product(L.grouped_gemm_rows(x, x), x, x)
    _check_product(L.grouped_gemm_rows(x, x, out_dtype=torch.bfloat16), x, x)


def test_product_of_the_longest_inner_dimension():
    """2^22 products a sum, in 33 ranges."""
    L = _lsgd()
    print("rows product longest", flush=True)
    K = 2 ** 22
    gen = torch.Generator(device=device()).manual_seed(3)
    a, b = (L.Rows(torch.randint(-127, 128, (1, n, K), generator=gen, device=device(),
                                 dtype=torch.int8), torch.rand(1, n, generator=gen, device=device()), K)
            for n in (3, 5))
    C = L.grouped_gemm_rows(a, b)
    # (exact in float64: below 2^36)
    exact = (a.q[0].double() @ b.q[0].double().t().contiguous()
             * a.scale[0].double()[:, None] * b.scale[0].double())
    assert bool(((C[0].double() - exact).abs() <= 3.1 * U32 * exact.abs()).all())
    bad = L.Rows(torch.zeros(1, 1, K + 128, dtype=torch.int8, device=device()),
                 torch.ones(1, 1, device=device()), K + 1)
    with pytest.raises(L.LsgdError):
        L.grouped_gemm_rows(bad, bad)


# (G, M, N): the cut that a product of theirs takes: the tile's side, and its stages of loads
CUTS = {(3, 150, 331): (64, 4), (1, 1501, 1487): (128, 4), (1, 2503, 2291): (128, 2),
        (10, 378, 2492): (256, 2)}


@pytest.mark.parametrize("out", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", CUTS)
def test_product_cuts(shape, out):
    """Every tile over one step to nine (each remainder of the unrolled loop), into a view of
    padded rows; every element against float64, in which the sums are exact."""
    L = _lsgd()
    G, M, N = shape
    dt = _dt(out)
    cut = (ctypes.c_int32 * 3)()
    gen = torch.Generator(device=device()).manual_seed(M)
    rand = lambda *s: torch.randn(*s, generator=gen, device=device())  # noqa: E731
    for K in (100, 250, 384, 500, 600, 1037):
        print(f"rows product cut {shape} {K} {out}", flush=True)
        assert L._lib.lsgd_grouped_gemm_rows_cut(int(out == "bf16"), G, M, N, K, cut) == 0
        assert tuple(cut) == (*CUTS[shape], 1)
        a, b = L.quantise_rows(rand(G, M, K) * torch.exp(rand(1, M, 1))), L.quantise_rows(rand(G, N, K))
        bias = rand(G, N)
        room = torch.full((G, M + 1, N + 3), 7.0, device=device(), dtype=dt)
        C = L.grouped_gemm_rows(a, b, bias, out=room[:, 1:, 2:N + 2])
        exact = (a.q.double() @ b.q.double().transpose(1, 2).contiguous()
                 * a.scale.double()[:, :, None] * b.scale.double()[:, None])
        add = bias.double()[:, None]
        bound = 2.01 * U32 * exact.abs() + 1.01 * U32 * (exact + add).abs() + 2.0 ** -148
        if out == "bf16":
            bound = bound + 2.0 ** -8 * ((exact + add).abs() + bound)
        assert bool(((C.double() - exact - add).abs() <= bound).all()), K
        C.fill_(7.0)
        assert bool((room == 7.0).all())


# (M, N, K): the cut: past 32-bit sums in each tile of 128 and 256, and a long one in ranges
RANGES = {(1300, 1250, 131200): (128, 4, 2), (2500, 4200, 131200): (128, 2, 2),
          (4000, 4090, 131200): (256, 2, 2), (1024, 1000, 65536): (128, 4, 4)}


@pytest.mark.parametrize("M,N,K", RANGES)
def test_large_products_in_ranges(M, N, K):
    """Sums by way of the workspace, checked at some rows and columns."""
    L = _lsgd()
    print(f"rows product ranges {M} {N} {K}", flush=True)
    cut = (ctypes.c_int32 * 3)()
    assert L._lib.lsgd_grouped_gemm_rows_cut(0, 1, M, N, K, cut) == 0
    assert tuple(cut) == RANGES[M, N, K]
    gen = torch.Generator(device=device()).manual_seed(M)
    a = L.quantise_rows(torch.randn(1, M, K, generator=gen, device=device(), dtype=torch.bfloat16))
    b = L.quantise_rows(torch.randn(1, N, K, generator=gen, device=device(), dtype=torch.bfloat16))
    bias = torch.randn(1, N, generator=gen, device=device())
    C = L.grouped_gemm_rows(a, b, bias)
    for rows, cols in ((slice(0, 70), slice(0, N)), (slice(M - 70, M), slice(0, N)),
                       (slice(0, M), slice(N - 40, N))):
        exact = (a.q[0, rows].double() @ b.q[0, cols].double().t().contiguous()
                 * a.scale[0, rows, None].double() * b.scale[0, None, cols].double())
        add = bias[0, cols].double()
        bound = 2.01 * U32 * exact.abs() + 1.01 * U32 * (exact + add).abs()
        assert bool(((C[0, rows, cols].double() - exact - add).abs() <= bound).all())


def test_product_scales_at_both_ends_and_not_finite():
    """Scales far apart whose product alone leaves fp32's range, and rows that held a NaN or an
    infinity: they show in their row or column alone."""
    L = _lsgd()
    print("rows product scales", flush=True)
    A = np.ones((1, 5, 200), np.float32)
    A[0] *= np.float32([[1], [2.0 ** 120], [2.0 ** -100], [3e-22], [1]])
    Bm = np.ones((1, 6, 200), np.float32)
    Bm[0] *= np.float32([[1], [2.0 ** -110], [2.0 ** 90], [4e-23], [1e-38], [1]])
    a, b = L.quantise_rows(to_dev(A)), L.quantise_rows(to_dev(Bm))
    C = _np(L.grouped_gemm_rows(a, b))[0]
    exact = O.product(a.q.cpu().numpy().astype(np.float64), _np(a.scale),
                      b.q.cpu().numpy().astype(np.float64), _np(b.scale))[0]
    fine = np.abs(exact) < 3.4e38
    assert np.all(np.abs(C - exact)[fine] <= _bound(exact, 0.0, None)[fine])
    assert np.isinf(C[~fine]).all() and (~fine).sum() == 1
    A[0, 4, 17], Bm[0, 5, 3] = np.inf, np.nan
    bias = torch.ones(1, 6, device=device())
    for dt in (torch.float32, torch.bfloat16):
        a, b = L.quantise_rows(to_dev(A)), L.quantise_rows(to_dev(Bm))
        C = _np(L.grouped_gemm_rows(a, b, bias, out_dtype=dt))[0]
        assert np.isnan(C[4]).all() and np.isnan(C[:, 5]).all() and not np.isnan(C[:4, :5]).any()


def test_product_shared_operands_and_strided_output():
    L = _lsgd()
    print("rows product shared", flush=True)
    rng = np.random.default_rng(8)
    a, b = _operands(L, rng, 3, 40, 70, 200)
    bs = L.Rows(b.q[:1].expand(3, -1, -1), b.scale[:1].expand(3, -1), b.n)
    bias = to_dev(rng.standard_normal((1, 70)).astype(np.float32)).expand(3, 70)
    for dt in (torch.float32, torch.bfloat16):
        room = torch.full((3, 44, 77), 7.0, device=device(), dtype=dt)
        out = room[:, 2:42, 3:73]
        assert L.grouped_gemm_rows(a, bs, bias, out=out) is out
        _check_product(out.contiguous(), a, bs, bias)
        out.fill_(7.0)
        assert (room == 7.0).all()
        side = torch.full((40, 3, 73), 7.0, device=device(), dtype=dt)
        _check_product(L.grouped_gemm_rows(a, bs, out=side[:, :, :70].transpose(0, 1)), a, bs)
        assert (side[:, :, 70:] == 7.0).all()
    part = L.Rows(a.q[1:2, 5:9], a.scale[1:2, 5:9], a.n)
    other = L.Rows(b.q[1:2, 3:], b.scale[1:2, 3:], b.n)
    _check_product(L.grouped_gemm_rows(part, other), part, other)
    for bad in (dict(out=a.scale[:, :, None].expand(3, 40, 70)), dict(bias=bias[:2]),
                dict(bias=bias.double()), dict(out_dtype=torch.float16)):
        with pytest.raises((ValueError, L.LsgdError)):
            L.grouped_gemm_rows(a, b, **bad)


def test_layer_gradients():
    """A layer's three products from tensors written both ways against the formulas on what the
    rows stand for."""
    L = _lsgd()
    print("rows layer gradients", flush=True)
    rng = np.random.default_rng(11)
    G, T, I, F = 2, 50, 96, 130
    x, w, dy = (to_dev(rng.standard_normal(s).astype(np.float32))
                for s in ((G, T, I), (G, I, F), (G, T, F)))
    (xq, xt), (wq, wt), (dq, dt) = (L.quantise_rows(t, both=True) for t in (x, w, dy))
    _check_product(L.grouped_gemm_rows(xq, wt), xq, wt)
    _check_product(L.grouped_gemm_rows(dq, wq), dq, wq)
    dw = L.grouped_gemm_rows(xt, dt)
    _check_product(dw, xt, dt)
    # rounding moves an element by at most half of its column's scale
    va, vd = np.abs(_np(x)), np.abs(_np(dy))
    ea, ed = va.max(1, keepdims=True) / 254, vd.max(1, keepdims=True) / 254
    exact = _np(x).transpose(0, 2, 1) @ _np(dy)
    bound = ((va + ea).transpose(0, 2, 1) @ (vd + ed)) - va.transpose(0, 2, 1) @ vd
    assert np.all(np.abs(_np(dw) - exact) <= 1.0001 * bound)


def test_rows_on_a_side_stream_and_in_a_graph():
    L = _lsgd()
    print("rows stream and graph", flush=True)
    rng = np.random.default_rng(13)
    X = to_dev(rng.standard_normal((1, 6, 3000)).astype(np.float32))
    W = to_dev(rng.standard_normal((1, 3000, 700)).astype(np.float32))
    bias = to_dev(rng.standard_normal((1, 700)).astype(np.float32))

    def step():
        q, t = L.quantise_rows(X, both=True)
        return L.grouped_gemm_rows(q, L.quantise_rows(W, both=True)[1], bias), t.q, t.scale

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
        X.copy_(to_dev(rng.standard_normal((1, 6, 3000)).astype(np.float32)))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step()))


def test_rows_past_32_bit_offsets():
    """Inputs, integers and results of more than 2^32 bytes and 2^31 elements: the last rows are
    those of the same rows alone."""
    L = _lsgd()
    print("rows past 32 bits", flush=True)
    gen = torch.Generator(device=device()).manual_seed(4)
    X = torch.randn(1, 131200, 33000, generator=gen, device=device(), dtype=torch.bfloat16)
    a, t = L.quantise_rows(X, both=True)
    alone = L.quantise_rows(X)
    assert a.q.numel() > 2 ** 32 and t.q.numel() > 2 ** 32
    assert torch.equal(alone.q, a.q) and torch.equal(alone.scale, a.scale)
    del alone
    tail = L.Rows(a.q[:, -65:].contiguous(), a.scale[:, -65:].contiguous(), a.n)
    _check_rows(tail, _np(X[:, -65:]))
    _check_rows(L.Rows(t.q[:, -65:].contiguous(), t.scale[:, -65:].contiguous(), t.n),
                _np(X[:, :, -65:]).transpose(0, 2, 1))
    b = L.quantise_rows(X[:, :70])
    del X
    _check_product(L.grouped_gemm_rows(a, b)[:, -65:], tail, b)
    del t
    rows = L.Rows(a.q[:, :49000, :128].contiguous(), a.scale[:, :49000].contiguous(), 128)
    end = L.Rows(rows.q[:, -65:].contiguous(), rows.scale[:, -65:].contiguous(), 128)
    del a
    for out in (torch.bfloat16, torch.float32):
        C = L.grouped_gemm_rows(rows, rows, out_dtype=out)
        _check_product(C[:, -65:, -65:], end, end)
