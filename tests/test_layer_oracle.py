"""The oracle of the operators around a large layer against torch on the CPU, and the
refusals of their entry points. Nothing is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import layer_oracle as O

P = ctypes.c_void_p


def _lib():
    from paper_1808_07217_amd import lsgd as L
    return L._lib


# ------------------------------------------------------------------ oracle
def test_oracle_rows_are_the_nearest_integers():
    rng = np.random.default_rng(0)
    X = rng.standard_normal((2, 5, 130)).astype(np.float32).astype(np.float64)
    X[0, 1] = 0
    q, s = O.quantise_rows(X)
    assert q.shape == (2, 5, 256) and not q[:, :, 130:].any()
    assert s[0, 1] == 1.0 and not q[0, 1].any()
    assert np.abs(q).max() == 127
    assert (np.abs(q[:, :, :130] * s[..., None] - X) <= s[..., None] / 2).all()
    # ties to even, and a scale that is exact
    q, s = O.quantise_rows(np.array([[[127.0, 0.5, 1.5, -2.5, 126.5]]]))
    assert s[0, 0] == 1.0 and list(q[0, 0, :5]) == [127, 0, 2, -2, 126]


def test_oracle_layer_norm_is_torch_s():
    rng = np.random.default_rng(1)
    X, dY = (torch.from_numpy(rng.standard_normal((1, 7, 33))).requires_grad_() for _ in range(2))
    w, b = (torch.from_numpy(rng.standard_normal(33)).requires_grad_() for _ in range(2))
    eps = float(np.float32(1e-5))
    y = torch.nn.functional.layer_norm(X, (33,), w, b, eps)
    y.backward(dY.detach())
    f = lambda t: t.detach().numpy()  # noqa: E731
    got, mean, rstd = O.layer_norm(f(X), f(w)[None], f(b)[None], eps)
    np.testing.assert_allclose(got, f(y), rtol=1e-12, atol=1e-13)
    dx, dw, db = O.layer_norm_backward(f(dY), f(X), mean, rstd, f(w)[None])
    for a, c in ((dx, X.grad), (dw[0], w.grad), (db[0], b.grad)):
        np.testing.assert_allclose(a, c.numpy(), rtol=1e-11, atol=1e-12)


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(2)
    X, dY = rng.standard_normal((2, 3, 9)), rng.standard_normal((2, 3, 9))
    w, b = rng.standard_normal((2, 9)), rng.standard_normal((2, 9))
    loss = lambda X, w, b: (O.layer_norm(X, w, b, 1e-5)[0] * dY).sum()  # noqa: E731
    _, mean, rstd = O.layer_norm(X, w, b, 1e-5)
    grads = O.layer_norm_backward(dY, X, mean, rstd, w)
    h = 1e-6
    for i, g in enumerate(grads):
        for at in [tuple(rng.integers(0, n) for n in g.shape) for _ in range(8)]:
            args = [[X, w, b], [X, w, b]]
            for sign, a in zip((1, -1), args):
                a[i] = a[i].copy()
                a[i][at] += sign * h
            quotient = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            # h^2 of the third derivative, and the rounding of two sums over 2 h
            assert abs(quotient - g[at]) <= 1e-7 * (1 + abs(g[at]))


def test_oracle_clips_as_torch_does():
    rng = np.random.default_rng(3)
    ts = [rng.standard_normal((1, 4, 5)), rng.standard_normal((1, 7))]
    ps = [torch.nn.Parameter(torch.zeros(t.shape, dtype=torch.float64)) for t in ts]
    for p, t in zip(ps, ts):
        p.grad = torch.from_numpy(t.copy())
    norm, out = O.clip(ts, 0.5)
    got = torch.nn.utils.clip_grad_norm_(ps, 0.5)
    assert abs(float(got) - norm[0]) < 1e-12
    for p, t in zip(ps, out):  # (torch adds 1e-6 to the norm)
        np.testing.assert_allclose(p.grad.numpy(), t, rtol=1e-6)
    norm, out = O.clip([np.array([[3.0, 4.0], [0.3, 0.4], [np.inf, 1.0]])], 1.0)
    np.testing.assert_allclose(norm, [5.0, 0.5, np.inf])
    np.testing.assert_allclose(out[0][:2], [[0.6, 0.8], [0.3, 0.4]])
    assert np.isinf(out[0][2, 0]) and out[0][2, 1] == 1.0


# ---------------------------------------------------------------- refusals
def _refuses(f, ok, bads):
    for bad in bads:
        a = list(ok)
        for k, v in bad.items():
            a[int(k[1:])] = v
        assert f(*a) == 1, bad


def test_quantise_rows_refusals():
    f, nb, lib = P(4096), ctypes.c_size_t(), _lib()
    size = lib.lsgd_quantise_rows_workspace_bytes
    assert size(2, 3, 5, None) == 1
    for bad in ((0, 3, 5), (65536, 3, 5), (2, 0, 5), (2, 3, 0), (2, 2**30 + 1, 5), (2, 3, 2**30 + 1)):
        assert size(*bad, ctypes.byref(nb)) == 1, bad
    assert size(2, 3, 5, ctypes.byref(nb)) == 0 and nb.value == 0  # (a single tile)
    assert size(2, 3, 500, ctypes.byref(nb)) == 0 and nb.value > 0
    ok = [0, 2, 3, 500, f, 500, 1500, f, f, f, f, f, nb.value, None]
    _refuses(lib.lsgd_quantise_rows, ok, (
        dict(_0=2), dict(_0=-1), dict(_1=0), dict(_1=65536), dict(_2=0), dict(_3=0), dict(_4=None),
        dict(_4=P(4098)), dict(_5=499), dict(_6=-1), dict(_7=None), dict(_7=P(4104)), dict(_8=None),
        dict(_8=P(4098)), dict(_9=None), dict(_9=P(4104)), dict(_10=None), dict(_10=P(4097)),
        dict(_11=None), dict(_11=P(4098)), dict(_2=2**30 + 1), dict(_3=2**30 + 1, _5=2**31),
        # sizes that are allowed, but more rows or tiles than a launch can number
        dict(_1=65535, _2=2**30, _9=None, _10=None), dict(_1=1, _2=2**30, _3=2**30, _5=2**30, _12=1 << 62)))
    ok[12] = nb.value - 1
    assert lib.lsgd_quantise_rows(*ok) == 2


def test_grouped_gemm_rows_refusals():
    f, nb, lib = P(4096), ctypes.c_size_t(), _lib()
    size = lib.lsgd_grouped_gemm_rows_workspace_bytes
    assert size(0, 2, 3, 4, 5, None) == 1
    for bad in ((2, 2, 3, 4, 5), (0, 0, 3, 4, 5), (0, 65536, 3, 4, 5), (0, 2, 0, 4, 5), (0, 2, 3, 0, 5),
                (0, 2, 3, 4, 0), (0, 2, 3, 4, 2**22 + 1), (0, 2, 2**30 + 1, 4, 5),
                (0, 2, 3, 2**31 - 1, 5)):
        assert size(*bad, ctypes.byref(nb)) == 1, bad
        assert lib.lsgd_grouped_gemm_rows_cut(*bad, (ctypes.c_int32 * 3)()) == 1, bad
    assert lib.lsgd_grouped_gemm_rows_cut(0, 2, 3, 4, 5, None) == 1
    assert size(0, 2, 3, 4, 5, ctypes.byref(nb)) == 0 and nb.value == 0
    # A 3 x 5, B 4 x 5, C 3 x 4
    ok = [0, 2, 3, 4, 5, f, 384, f, 3, f, 512, f, 4, f, 4, f, 4, 12, None, 0, None]
    bads = (dict(_0=2), dict(_1=0), dict(_1=65536), dict(_2=0), dict(_3=0), dict(_4=0),
            dict(_4=2**22 + 1), dict(_5=None), dict(_5=P(4104)), dict(_6=-16), dict(_6=8),
            dict(_7=None), dict(_7=P(4098)), dict(_8=-1), dict(_9=None), dict(_9=P(4097)),
            dict(_10=24), dict(_11=None), dict(_11=P(4097)), dict(_12=-1), dict(_13=P(4098)),
            dict(_14=-1), dict(_15=None), dict(_15=P(4098)), dict(_16=3), dict(_17=11), dict(_17=0),
            dict(_17=3), dict(_16=7, _17=4),
            dict(_1=1, _2=2**30, _3=2**30, _4=5, _16=2**30))
    _refuses(lib.lsgd_grouped_gemm_rows, ok, bads)
    # with a workspace, for few results and for a long inner dimension
    for M, N, K in ((64, 64, 65536), (2000, 2000, 2**17)):
        assert size(0, 1, M, N, K, ctypes.byref(nb)) == 0 and nb.value > 0
        big = [0, 1, M, N, K, f, 0, f, 0, f, 0, f, 0, f, 0, f, N, 0, f, nb.value, None]
        _refuses(lib.lsgd_grouped_gemm_rows, big, (dict(_18=None), dict(_18=P(4100))))
        big[19] -= 1
        assert lib.lsgd_grouped_gemm_rows(*big) == 2


def test_long_products_never_sum_past_32_bits():
    """The ranges of every inner dimension: at most 2^17 - 1 products of up to 2^14 each."""
    cut, lib = (ctypes.c_int32 * 3)(), _lib()
    for K in (1, 128, 2**17 - 1, 2**17, 2**18 + 1, 2**20, 2**22):
        for M, N in ((1, 1), (64, 64), (3000, 5000), (2**16, 2**16)):
            for G in (1, 7):
                assert lib.lsgd_grouped_gemm_rows_cut(0, G, M, N, K, cut) == 0
                steps = -(-K // 128)
                chunk = -(-steps // cut[2])
                assert min(chunk * 128, K) * 2**14 < 2**31 and (cut[2] - 1) * chunk < steps


def test_layer_norm_refusals():
    f, lib, c = P(4096), _lib(), ctypes.c_float
    ok = [0, 0, 2, 3, 5, f, 5, 15, f, 5, f, 5, c(1e-5), f, 5, 15, f, f, None]
    inf = float("inf")
    _refuses(lib.lsgd_layer_norm, ok, (
        dict(_0=2), dict(_1=-1), dict(_2=0), dict(_2=65536), dict(_3=0), dict(_4=0),
        dict(_3=2**30 + 1), dict(_4=2**30 + 1, _6=2**31, _14=2**31, _15=2**40), dict(_5=None),
        dict(_5=P(4098)), dict(_6=4), dict(_7=-1), dict(_8=P(4098)), dict(_9=-1), dict(_10=P(4097)),
        dict(_11=-1), dict(_12=c(0.0)), dict(_12=c(-1e-5)), dict(_12=c(inf)),
        dict(_12=c(float("nan"))), dict(_13=None), dict(_13=P(4098)), dict(_14=4), dict(_15=14),
        dict(_15=0), dict(_16=None), dict(_16=P(4098)), dict(_17=None), dict(_17=P(4098)),
        # rows past what registers hold, more of them than a launch can number
        dict(_2=65535, _3=2**20, _4=20000, _6=20000, _7=0, _14=20000, _15=2**40)))


def test_layer_norm_backward_refusals():
    f, nb, lib = P(4096), ctypes.c_size_t(), _lib()
    size = lib.lsgd_layer_norm_backward_workspace_bytes
    assert size(2, 3, 5, None) == 1
    for bad in ((0, 3, 5), (65536, 3, 5), (2, 0, 5), (2, 3, 0), (2, 2**30 + 1, 5), (2, 3, 2**30 + 1)):
        assert size(*bad, ctypes.byref(nb)) == 1, bad
    M = 40000
    assert size(2, M, 5, ctypes.byref(nb)) == 0 and nb.value > 0
    S = 5 * M
    ok = [0, 0, 2, M, 5, f, 5, S, f, 5, S, f, f, f, 5, f, 5, S, f, 5, f, 5, f, nb.value, None]
    _refuses(lib.lsgd_layer_norm_backward, ok, (
        dict(_0=2), dict(_1=2), dict(_2=0), dict(_2=65536), dict(_3=0), dict(_4=0), dict(_5=None),
        dict(_5=P(4098)), dict(_6=4), dict(_7=-1), dict(_8=None), dict(_8=P(4097)), dict(_9=4),
        dict(_10=-1), dict(_11=None), dict(_11=P(4098)), dict(_12=None), dict(_12=P(4097)),
        dict(_13=P(4098)), dict(_14=-1), dict(_15=None), dict(_15=P(4098)), dict(_16=4),
        dict(_17=S - 1), dict(_18=None), dict(_18=P(4098)), dict(_19=4), dict(_20=None),
        dict(_20=P(4098)), dict(_21=4), dict(_21=-5), dict(_22=None), dict(_22=P(4104))))
    ok[23] = nb.value - 1
    assert lib.lsgd_layer_norm_backward(*ok) == 2


def _table(*rows):
    return (ctypes.c_int64 * (6 * len(rows)))(*[v for r in rows for v in r])


def test_clip_refusals():
    f, nb, lib, d = P(4096), ctypes.c_size_t(), _lib(), ctypes.c_double
    size, clip, norm = (lib.lsgd_gradient_norm_workspace_bytes, lib.lsgd_clip_gradients,
                        lib.lsgd_gradient_norm)
    good = (8192, 3, 5, 5, 15, 0)
    one = _table(good)
    assert size(2, 1, one, None) == 1
    assert size(2, 1, one, ctypes.byref(nb)) == 0 and nb.value == 0  # (few values)
    for bad in ((0, 1, one), (65536, 1, one), (2, 0, one), (2, 65537, one), (2, 1, None)):
        assert size(*bad, ctypes.byref(nb)) == 1, bad
        assert norm(*bad, f, f, 1 << 20, None) == 1, bad
        assert clip(*bad, d(1.0), f, f, 1 << 20, None) == 1, bad
    # (the last: a column past 32-bit numbers, in rows of a pitch)
    for k, v in ((0, 0), (0, 8194), (1, 0), (1, 2**44), (2, 0), (2, -5), (3, 4), (3, 2**50), (4, -1),
                 (4, 2**50), (5, 2), (5, 1 << 32), ((2, 2**30 + 1), (3, 2**30 + 2))):
        row = list(good)
        for k, v in ((k, v),) if isinstance(k, int) else (k, v):
            row[k] = v
        for t in (_table(row), _table(good, row)):
            n = len(t) // 6
            assert size(2, n, t, ctypes.byref(nb)) == 1, (k, v)
            assert norm(2, n, t, f, f, 1 << 20, None) == 1, (k, v)
            assert clip(2, n, t, d(1.0), f, f, 1 << 20, None) == 1, (k, v)
    # replicas that overlap: the norm reads them, a clip would scale a value twice
    for s in (14, 5, 0, 4):
        assert size(2, 1, _table((8192, 3, 5, 5, s, 0)), ctypes.byref(nb)) == 0
        assert clip(2, 1, _table((8192, 3, 5, 5, s, 0)), d(1.0), f, f, 1 << 20, None) == 1, s
    inf = float("inf")
    for bound in (0.0, -1.0, inf, float("nan")):
        assert clip(2, 1, one, d(bound), f, f, 1 << 20, None) == 1, bound
    one = _table((8192, 300, 500, 500, 150000, 0))
    assert size(2, 1, one, ctypes.byref(nb)) == 0 and nb.value > 0
    for p, ws, n, want in ((None, f, nb.value, 1), (P(4098), f, nb.value, 1), (f, None, nb.value, 1),
                           (f, P(4100), nb.value, 1), (f, f, nb.value - 1, 2)):
        assert clip(2, 1, one, d(1.0), p, ws, n, None) == want
        assert norm(2, 1, one, p, ws, n, None) == want


def test_binding_refuses_host_tensors_and_shapes():
    from paper_1808_07217_amd import lsgd as L
    x, v = torch.zeros(2, 3, 4), torch.zeros(2, 4)
    for call in (lambda: L.quantise_rows(x), lambda: L.layer_norm(x, v, v),
                 lambda: L.layer_norm_backward(x, x, v[:, :3], v[:, :3], v),
                 lambda: L.gradient_norm([x]), lambda: L.clip_gradients([x], 1.0)):  # (host tensors)
        with pytest.raises(ValueError, match="CUDA"):
            call()
    for bad in (x[0], x.half(), x[:, :, :0], x.int()):
        for call in (L.quantise_rows, L.layer_norm):
            with pytest.raises(ValueError):
                call(bad)
    q, s = torch.zeros(2, 3, 128, dtype=torch.int8), torch.zeros(2, 3)
    for bad in (L.Rows(q, s, 129), L.Rows(q, s, 0), L.Rows(q[:, :2], s, 5), L.Rows(q.float(), s, 5),
                L.Rows(q, s.double(), 5), L.Rows(q, s[0], 5), L.Rows(q[0], s, 5), L.Rows(q, s, 5)):
        with pytest.raises(ValueError):
            L.grouped_gemm_rows(bad, bad)
    for bad in ([], x, [x.half()], [x[:0]], [torch.tensor(1.0)]):
        for call in (L.gradient_norm, lambda t: L.clip_gradients(t, 1.0)):
            with pytest.raises(ValueError):
                call(bad)


def _apart(K, rows):
    out = ctypes.c_int32(-1)
    assert _lib().lsgd_tensors_apart(K, len(rows), _table(*rows), ctypes.byref(out)) == 0
    return bool(out.value)


def test_overlapping_tensors_are_found_exactly():
    """Random lists of views into one buffer against the set of their bytes; those that overlap
    are refused."""
    lib, rng, f = _lib(), np.random.default_rng(4), P(1 << 40)
    seen = {False: 0, True: 0}
    for _ in range(3000):
        K, table, used, clash = int(rng.integers(1, 4)), [], set(), False
        pitch = int(rng.choice([0, 0, 40, 64, 200]))
        for _ in range(int(rng.integers(2, 5))):
            d, M, N = (int(v) for v in (rng.integers(0, 2), rng.integers(1, 4), rng.integers(1, 6)))
            ld = N + int(rng.integers(0, 2)) * int(rng.integers(0, 9))
            ld = N if M == 1 else ld
            s = max(pitch, (M - 1) * ld + N) if K > 1 else 0
            p = 4096 + 4 * int(rng.integers(0, 150))
            e = (4, 2)[d]
            mine = {p + e * (k * s + m * ld + n) + b for k in range(K) for m in range(M)
                    for n in range(N) for b in range(e)}
            clash |= bool(mine & used)
            used |= mine
            table.append((p, M, N, ld, s, d))
        assert _apart(K, table) == (not clash), table
        if clash:
            assert lib.lsgd_clip_gradients(K, len(table), _table(*table), ctypes.c_double(1.0), f, f,
                                           1 << 20, None) == 1
        seen[clash] += 1
    assert min(seen.values()) > 300, seen
    # tensors of flat rows side by side, in any order
    row = [(4096, 4, 6, 6, 64, 0), (4096 + 4 * 24, 1, 6, 6, 64, 0), (4096 + 4 * 30, 2, 17, 17, 64, 0)]
    assert _apart(5, row) and _apart(5, row[::-1])
    assert not _apart(5, row + [(4096 + 4 * 63, 1, 2, 2, 64, 0)])
    # two interleaved matrices of too many rows to look at
    many = [(4096, 1 << 24, 3, 8, 0, 0), (4096 + 12, 1 << 24, 3, 8, 0, 0)]
    assert not _apart(1, many) and _apart(1, [(p, 1 << 20, *r) for p, _, *r in many])
    one = ctypes.c_int32()
    assert lib.lsgd_tensors_apart(5, 3, _table(*row), None) == 1
    assert lib.lsgd_tensors_apart(0, 3, _table(*row), ctypes.byref(one)) == 1
    assert lib.lsgd_tensors_apart(5, 3, None, ctypes.byref(one)) == 1
    assert lib.lsgd_tensors_apart(5, 1, _table((4096, 4, 6, 6, 20, 0)), ctypes.byref(one)) == 1


def test_the_most_values_to_clip():
    """The workspace's query, the norm and the clip have one limit, of all values together."""
    lib, f, nb, d = _lib(), P(1 << 40), ctypes.c_size_t(), ctypes.c_double
    huge = (1 << 40, 2**20, 2**24, 2**24, 0, 0)  # 2^44 values, one tensor for every replica
    for K, n, want in ((2**13 + 1, 2, 0), (2**15 + 1, 2, 1), (2**13, 8, 0), (2**13 + 1, 8, 1)):
        t = _table(*[huge] * n)
        assert lib.lsgd_gradient_norm_workspace_bytes(K, n, t, ctypes.byref(nb)) == want, (K, n)
        # (with no workspace at all: refused as such, or before)
        assert lib.lsgd_gradient_norm(K, n, t, f, None, 0, None) == 1
        assert lib.lsgd_gradient_norm(K, n, t, f, f, 0, None) == (1 if want else 2)
    # rows of a pitch count in eights
    narrow = (1 << 40, 2**41, 1, 2, 0, 0)
    for K, want in ((2**16 - 1, 0), (2**15, 0)):
        assert lib.lsgd_gradient_norm_workspace_bytes(K, 1, _table(narrow), ctypes.byref(nb)) == want
    for n, want in ((1, 0), (2, 1)):
        t = _table(*[narrow] * n)
        assert lib.lsgd_gradient_norm_workspace_bytes(2**16 - 1, n, t, ctypes.byref(nb)) == want
    # every list of small tensors for every replica
    many = _table(*[(4096 + 4 * i, 1, 1, 1, 65536, 0) for i in range(65536)])
    assert lib.lsgd_gradient_norm_workspace_bytes(65535, 65536, many, ctypes.byref(nb)) == 0
    assert nb.value == (65536 + 1) * 65535 * 8
    assert lib.lsgd_clip_gradients(65535, 65536, many, d(1.0), f, f, nb.value - 1, None) == 2


def test_binding_refuses_sizes_past_32_bits():
    """Not the call of their last 32 bits. (Expanded tensors: nothing of that size is held.)"""
    from paper_1808_07217_amd import lsgd as L
    n = 2**32 + 1
    for call in (lambda: L._int32(3, n), lambda: L._int32(2**31),
                 lambda: L._geometry((n, 3), (0, 1), torch.float32),
                 lambda: L.replica_average(torch.empty(n, 0)),
                 lambda: L.replica_average_blocks(torch.empty(n, 0), 1),
                 lambda: L.grouped_gemm(torch.empty(n, 0, 1), torch.empty(n, 1, 0))):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
    L._int32(2**31 - 1, 1)
    q, s = torch.zeros(1, 1, 128, dtype=torch.int8), torch.zeros(1, 1)
    wide = L.Rows(q.expand(n, 1, 128), s.expand(n, 1), 5)
    with pytest.raises(ValueError, match="2\\^31"):
        L.grouped_gemm_rows(wide, wide)
    b = L.Blocks(q.to(torch.float8_e4m3fn).expand(n, 1, 128),
                 torch.zeros(1, 1, 4).to(torch.float8_e8m0fnu).expand(n, 1, 4), 5)
    with pytest.raises(ValueError, match="2\\^31"):
        L.grouped_gemm_blocks(b, b)
