"""CPU tests of the large-layer operators: the numpy oracle against torch's own
8-bit types and against known properties, and every refusal of the entry
points (nothing is launched)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import blocks_oracle as B

TORCH = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_rounds_as_torch_does(fmt):
    """Every value of the format, every midpoint between neighbours (ties), and
    their fp32 neighbours on both sides."""
    codes = torch.arange(256, dtype=torch.uint8).view(TORCH[fmt]).to(torch.float64)
    v = np.unique(codes[torch.isfinite(codes)].numpy())
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid.astype(np.float32), np.float32(1e9)),
                        np.nextafter(mid.astype(np.float32), np.float32(-1e9))]).astype(np.float32)
    want = torch.from_numpy(x).to(TORCH[fmt]).to(torch.float64).numpy()
    assert np.array_equal(B.round_format(x.astype(np.float64), fmt), want)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_oracle_scale_is_the_smallest_that_fits(fmt):
    top = B.FORMATS[fmt][0]
    for amax, e in ((top, 0), (np.nextafter(np.float32(top), np.float32(1e9)), 1), (top / 2, -1),
                    (1e-45, -127), (np.finfo(np.float32).max, 120 if fmt == "e4m3" else 113),
                    (0.0, 0)):
        X = np.zeros((1, 1, 130))
        X[0, 0, 3] = -float(amax)
        q, s = B.quantise(X, fmt)
        assert s[0, 0].tolist() == [2.0 ** e, 1.0, 1.0, 1.0], (amax, s)
        assert np.abs(q).max() <= top
        if 1e-38 < amax:
            assert abs(B.values(q, s)[0, 0, 3] + amax) <= amax * 2.0 ** -(B.FORMATS[fmt][1] + 1)


def test_oracle_orthogonalises():
    """Singular values of a well-conditioned matrix land where five steps of the
    scalar iteration take them, singular vectors stay."""
    rng = np.random.default_rng(0)
    X = rng.standard_normal((1, 12, 7))
    u, s, vt = np.linalg.svd(X[0], full_matrices=False)
    t = s / (np.linalg.norm(X) + float(np.float32(1e-7)))
    a, b, c = (float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))
    for _ in range(5):
        t = t * (a + b * t ** 2 + c * t ** 4)
    np.testing.assert_allclose(B.newton_schulz(X)[0], (u * t) @ vt, atol=1e-12)
    assert 0.6 < t.min() and t.max() < 1.3


def _lib():
    from paper_1808_07217_amd import lsgd as L
    return L._lib


P = ctypes.c_void_p


def test_quantise_refusals():
    f = P(4096)
    ok = [0, 0, 2, 3, 5, f, 5, 15, f, f, f, f, None]

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return _lib().lsgd_quantise_blocks(*a)

    for bad in (dict(_0=2), dict(_0=-1), dict(_1=2), dict(_1=-1), dict(_2=0), dict(_2=65536),
                dict(_3=0), dict(_4=0), dict(_4=-3), dict(_5=None), dict(_5=P(4098)), dict(_6=4),
                dict(_7=-1), dict(_8=None), dict(_9=None), dict(_10=None), dict(_11=None),
                dict(_8=None, _9=None, _10=None, _11=None), dict(_8=P(4104)), dict(_10=P(4097)),
                # more tiles than a launch can number
                dict(_2=65535, _3=2**31 - 1, _4=2**31 - 1, _6=2**31, _8=None, _9=None)):
        assert call(**bad) == 1, bad


def test_grouped_gemm_blocks_refusals():
    f, nb = P(4096), ctypes.c_size_t()
    lib = _lib()
    assert lib.lsgd_grouped_gemm_blocks_workspace_bytes(0, 2, 3, 4, 5, None) == 1
    assert lib.lsgd_grouped_gemm_blocks_workspace_bytes(2, 2, 3, 4, 5, ctypes.byref(nb)) == 1
    for bad in ((0, 3, 4, 5), (2, 3, 4, 2**22 + 1), (2, 0, 4, 5), (2, 3, 0, 5), (2, 3, 4, 0), (65536, 3, 4, 5)):
        assert lib.lsgd_grouped_gemm_blocks_workspace_bytes(0, *bad, ctypes.byref(nb)) == 1
    ok = [0, 0, 0, 2, 3, 4, 5, f, 384, f, 12, f, 512, f, 16, f, 4, 12, f, 1 << 40, None]

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.lsgd_grouped_gemm_blocks(*a)

    for bad in (dict(_0=2), dict(_1=-1), dict(_2=2), dict(_3=0), dict(_3=65536), dict(_4=0),
                dict(_5=0), dict(_6=0), dict(_6=2**22 + 1), dict(_7=None), dict(_7=P(4104)), dict(_8=-16),
                dict(_8=8), dict(_9=None), dict(_9=P(4098)), dict(_10=-4), dict(_10=3),
                dict(_11=None), dict(_11=P(4097)), dict(_12=24), dict(_13=None), dict(_13=P(4097)),
                dict(_14=6), dict(_15=None), dict(_15=P(4098)), dict(_16=3), dict(_17=11)):
        assert call(**bad) == 1, bad
    # a product that wants a workspace, without one and with one too small
    assert lib.lsgd_grouped_gemm_blocks_workspace_bytes(0, 1, 64, 64, 65536, ctypes.byref(nb)) == 0
    assert nb.value > 0
    big = dict(_3=1, _4=64, _5=64, _6=65536, _16=64)
    assert call(**big, _18=None) == 1
    assert call(**big, _18=P(4100)) == 1
    assert call(**big, _19=nb.value - 1) == 2


def test_blocks_refuse_more_rows_than_an_int_holds_tiles_of():
    f, nb, lib = P(4096), ctypes.c_size_t(), _lib()
    top = 2**31 - 1
    for M, N in ((2**30 + 1, 1), (1, 2**30 + 1), (top, 1), (1, top)):
        assert lib.lsgd_quantise_blocks(0, 0, 1, M, N, f, N, 0, f, f, None, None, None) == 1
        assert lib.lsgd_quantise_blocks(0, 0, 1, M, N, f, N, 0, None, None, f, f, None) == 1
        size = lib.lsgd_grouped_gemm_blocks_workspace_bytes
        assert size(1, 1, M, N, 5, ctypes.byref(nb)) == 1
        assert lib.lsgd_grouped_gemm_blocks(0, 0, 1, 1, M, N, 5, f, 0, f, 0, f, 0, f, 0, f, N, 0,
                                            f, 1 << 40, None) == 1
    assert size(1, 1, 2**30, 2**30, 5, ctypes.byref(nb)) == 0
    # sizes that are allowed, but more tiles than a launch can number
    M = N = 2**30
    assert lib.lsgd_quantise_blocks(0, 0, 1, M, N, f, N, 0, f, f, None, None, None) == 1
    assert lib.lsgd_grouped_gemm_blocks(0, 0, 1, 1, M, N, 5, f, 0, f, 0, f, 0, f, 0, f, N, 0, f,
                                        1 << 40, None) == 1


CO = (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315)


def test_orthogonalise_refusals():
    f, nb = P(4096), ctypes.c_size_t()
    lib = _lib()
    size = lib.lsgd_orthogonalise_workspace_bytes
    assert size(0, 2, 3, 5, None) == 1
    for bad in ((2, 2, 3, 5), (0, 0, 3, 5), (0, 65536, 3, 5), (0, 2, 0, 5), (0, 2, 3, 0),
                (0, 1, 1 << 16, 1 << 16), (0, 1, 2**20 + 1, 1), (0, 1, 2**31 - 1, 1), (1, 1, 2**31 - 1, 2**31 - 1)):
        assert size(*bad, ctypes.byref(nb)) == 1, bad
    assert size(0, 2, 3, 5, ctypes.byref(nb)) == 0
    # (150 x 200: larger than one launch takes, so there is a workspace)
    assert size(0, 2, 150, 200, ctypes.byref(nb)) == 0 and nb.value > 0
    inf, nan = float("inf"), float("nan")

    def co(*v):
        return (ctypes.c_float * 3)(*v)

    M, N, S = 150, 200, 150 * 200
    ok = [0, 2, M, N, f, N, S, f, N, S, 5, CO, ctypes.c_float(1e-7), f, nb.value, None]

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.lsgd_orthogonalise(*a)

    for bad in (dict(_0=2), dict(_1=0), dict(_2=0), dict(_3=0), dict(_4=None), dict(_4=P(4098)),
                dict(_5=N - 1), dict(_6=-1), dict(_7=None), dict(_7=P(4097)), dict(_8=N - 1),
                dict(_9=S - 1), dict(_9=-S), dict(_9=0), dict(_8=2 * N - 1, _9=N), dict(_10=0),
                dict(_10=65),
                dict(_11=None), dict(_11=co(inf, 0, 0)), dict(_11=co(1, nan, 0)),
                dict(_11=co(40, 0, 0)), dict(_11=co(3, 0, 0)), dict(_12=ctypes.c_float(0.0)),
                dict(_12=ctypes.c_float(-1e-7)), dict(_12=ctypes.c_float(nan)),
                dict(_12=ctypes.c_float(inf)), dict(_13=None), dict(_13=P(4096 + 128))):
        assert call(**bad) == 1, bad
    assert call(_14=nb.value - 1) == 2


def test_orthogonal_update_refusals():
    f, nb = P(4096), ctypes.c_size_t()
    lib = _lib()
    M, N, S = 150, 200, 150 * 200
    assert lib.lsgd_orthogonalise_workspace_bytes(0, 2, M, N, ctypes.byref(nb)) == 0
    c = ctypes.c_float
    ok = [0, 2, M, N, f, N, S, f, N, S, f, N, S, c(0.1), c(0.9), c(0.01), 0, c(1.0), 5, CO,
          c(1e-7), f, nb.value, None]

    def call(**kw):
        a = list(ok)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return lib.lsgd_orthogonal_update(*a)

    nan = float("nan")
    for bad in (dict(_0=2), dict(_1=0), dict(_2=0), dict(_3=0), dict(_4=None), dict(_5=N - 1),
                dict(_6=S - 1), dict(_6=0), dict(_7=None), dict(_7=P(4098)), dict(_8=N - 1),
                dict(_9=N - 1), dict(_10=None), dict(_11=N - 1), dict(_12=-1), dict(_13=c(nan)), dict(_14=c(1.0)),
                dict(_14=c(-0.1)), dict(_14=c(nan)), dict(_15=c(nan)), dict(_16=2),
                dict(_17=c(nan)), dict(_18=0), dict(_19=None), dict(_20=c(0.0)), dict(_21=None)):
        assert call(**bad) == 1, bad
    assert call(_22=nb.value - 1) == 2


def test_binding_refuses_host_tensors_and_shapes():
    from paper_1808_07217_amd import lsgd as L
    x = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError, match="CUDA"):
        L.quantise_blocks(x)
    with pytest.raises(ValueError):
        L.quantise_blocks(x[0])
    with pytest.raises(ValueError):
        L.quantise_blocks(x.half())
    with pytest.raises(ValueError, match="CUDA"):
        L.orthogonalise(x)
    with pytest.raises(ValueError, match="CUDA"):
        L.orthogonal_update(x, x, x, 0.1, 0.9)
    q = torch.zeros(2, 3, 128, dtype=torch.uint8).view(torch.float8_e4m3fn)
    s = torch.zeros(2, 3, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for bad in (L.Blocks(q, s, 129), L.Blocks(q, s, 0), L.Blocks(q[:, :2], s, 5),
                L.Blocks(q.view(torch.uint8), s, 5), L.Blocks(q, s.view(torch.uint8), 5),
                L.Blocks(q, s, 5)):
        with pytest.raises(ValueError):
            L.grouped_gemm_blocks(bad, bad)


def test_product_refuses_groups_that_overlap():
    """Group strides that would let two groups of C share an element; nothing is
    launched."""
    f, lib = P(4096), _lib()
    M, N, ld = 3, 4, 6

    def call(G, ldc, sC):
        return lib.lsgd_grouped_gemm_blocks(0, 0, 0, G, M, N, 5, f, 384, f, 12, f, 512, f, 16, f,
                                            ldc, sC, f, 1 << 40, None)

    for G, ldc, sC in ((2, ld, 2 * ld + N - 1), (2, ld, 3), (2, ld, 0), (2, ld, -ld * M),
                       (2, 2 * N - 1, N), (3, 3 * N - 1, N), (2, ld, ld)):
        assert call(G, ldc, sC) == 1, (G, ldc, sC)


def test_binding_finds_overlaps_exactly():
    """Random pairs of views into one buffer, of any pitches and strides, types and shared
    groups, against the set of their bytes."""
    from paper_1808_07217_amd import lsgd as L
    rng = np.random.default_rng(1)
    buf = torch.zeros(4096, dtype=torch.uint8)
    seen = {False: 0, True: 0}

    def view():
        t = buf.view([torch.float32, torch.bfloat16, torch.float8_e4m3fn][rng.integers(3)])
        G, M, N = (int(v) for v in rng.integers(1, 6, 3))
        ld = N + int(rng.integers(0, 30)) * int(rng.integers(0, 2))
        s = int(rng.choice([0, N, M * ld, M * ld + 40, (M - 1) * ld + N, 90]))
        extent = (G - 1) * s + (M - 1) * ld + N
        return t.as_strided((G, M, N), (s, ld, 1), int(rng.integers(0, t.numel() - extent + 1)))

    def bytes_of(t):
        e = t.element_size()
        return {t.data_ptr() + e * (g * t.stride(0) + m * t.stride(1) + n) + k
                for g in range(t.shape[0]) for m in range(t.shape[1]) for n in range(t.shape[2])
                for k in range(e)}

    for _ in range(3000):
        a, b = view(), view()
        want = bool(bytes_of(a) & bytes_of(b))
        assert L._overlap(a, b) == want == L._overlap(b, a)
        size = lambda t: max(bytes_of(t)) + 1 - t.data_ptr()  # noqa: E731
        apart = L._apart(a.data_ptr(), size(a), b.data_ptr(), size(b))
        assert not (apart and want)
        seen[want] += not apart
    # of both kinds among pairs whose spans are not apart
    assert min(seen.values()) > 100, seen


def test_product_cut_refusals():
    cut, lib = (ctypes.c_int32 * 3)(), _lib()
    f = lib.lsgd_grouped_gemm_blocks_cut
    assert f(0, 1, 2, 3, 4, None) == 1
    for bad in ((2, 1, 2, 3, 4), (0, 0, 2, 3, 4), (0, 1, 0, 3, 4), (0, 1, 2, 2**31 - 1, 4),
                (1, 1, 2, 3, 2**22 + 1)):
        assert f(*bad, cut) == 1, bad
    assert f(1, 1, 2, 3, 4, cut) == 0 and list(cut) == [64, 4, 1]


def test_every_cut_of_the_orthogonalisation_is_tested():
    """The shapes of the GPU tests, which run each in both precisions, against all the cuts that
    matrices of up to 32 x 32 tiles of 64, in any number up to 800, take."""
    import test_gpu_ortho as T
    cut, f = (ctypes.c_int32 * 7)(), _lib().lsgd_orthogonalise_cut

    def cuts(shapes):
        seen = set()
        for G, M, N in shapes:
            for dtype in (0, 1):
                assert f(dtype, G, M, N, cut) == 0
                if cut[0]:
                    seen |= {(cut[0], i, cut[i], cut[i + 1]) for i in (1, 3, 5)}
        return seen

    tested = cuts(T.SHAPES + T.LARGE + T.CUTS)
    tiles = (1, 2, 3, 4, 5, 6, 7, 8, 9, 11, 14, 18, 24, 32)
    assert tested == cuts((G, 64 * m, 64 * n + 600 * (n == 1)) for m in tiles for n in tiles
                          for G in (*range(1, 60), *range(60, 800, 7)))
    assert len(tested) == 35

    assert f(2, 1, 64, 64, cut) == 1 and f(0, 0, 64, 64, cut) == 1 and f(0, 1, 64, 0, cut) == 1
    assert f(0, 1, 64, 64, None) == 1
    assert f(0, 1, 64, 64, cut) == 0 and list(cut) == [0] * 7


def test_few_rows_keep_two_sums():
    """X X^T of matrices of fewer than 385 rows never takes the tiles that keep one sum."""
    cut, f = (ctypes.c_int32 * 7)(), _lib().lsgd_orthogonalise_cut
    one = 0
    for m in range(64, 449, 64):
        for n in (m, 600, 4096):
            for G in range(1, 700, 3):
                assert f(0, G, m, n, cut) == 0
                one += cut[3] == 256
                assert m >= 385 or cut[1] < 256, (G, m, n)
    assert one > 0


def test_update_refuses_factors_that_overflow():
    f, c = P(4096), ctypes.c_float
    for lr, wd, scale in ((1e30, 0.0, 1e30), (1e30, 1e30, 1.0), (-3e38, 0.0, 2.0)):
        assert _lib().lsgd_orthogonal_update(
            0, 1, 3, 4, f, 4, 0, f, 4, 0, f, 4, 0, c(lr), c(0.9), c(wd), 0, c(scale), 5, CO,
            c(1e-7), None, 0, None) == 1
