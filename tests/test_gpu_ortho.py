"""GPU tests of the orthogonalised momentum against the float64 oracle.

Tolerance: the oracle run with the roundings of the kernels' precision (fp16
pieces, fp32 sums) lands at some distance from the exact result; a kernel of
that precision, whose sums run in another order, may be four times as far, in
norm and at the worst entry, plus its output's own rounding (half a step). With
few values that distance is one sample of a random sum and may come out near zero,
so a floor stands beside it: the last step's three terms a s, b s^3, c s^5 add to
(3.44 + 4.78 1.45 + 2.03 2.1) 1.2 = 17.6 at the largest s = 1.2, and each is rounded to 24
bits twice at least (as pieces and as a sum), 35 2^-24 in all of a result near 1."""
import numpy as np
import pytest
import torch

from oracle import blocks_oracle as B
from gpu_util import device, to_dev

pytestmark = pytest.mark.gpu


def _lsgd():
    from paper_1808_07217_amd import lsgd as L
    return L


def _np(t):
    return t.to(torch.float32).cpu().numpy().astype(np.float64)


def _matrices(rng, G, M, N, low=False):
    x = rng.standard_normal((G, M, N))
    r = max(1, min(M, N) // 16)
    part = rng.standard_normal((G, M, r)) @ rng.standard_normal((G, r, N))
    return (x * 0.02 + part) if low else x + part / np.sqrt(r)


def _check(got, X, bf16, **kw):
    want = B.newton_schulz(X, **kw)
    near = B.newton_schulz_rounded(X, 1 if bf16 else 2, **kw)
    half = 2.0 ** -8 if bf16 else 2.0 ** -24
    for g in range(X.shape[0]):
        e, d, w = np.abs(got[g] - want[g]), np.abs(near[g] - want[g]), np.abs(want[g])
        floor = half + 35 * 2.0 ** -24
        tol = 4 * np.linalg.norm(d) + floor * np.linalg.norm(w)
        assert np.linalg.norm(e) <= tol, (g, np.linalg.norm(e), tol)
        tol = 4 * d.max() + floor * w.max()
        assert e.max() <= tol, (g, e.max(), tol)


SHAPES = [(1, 1, 1), (2, 1, 7), (3, 5, 1), (2, 16, 16), (4, 64, 64), (2, 65, 63), (2, 128, 100),
          (2, 129, 130), (1, 130, 257), (3, 257, 100), (1, 200, 1000), (1, 700, 64), (2, 512, 512),
          (1, 33, 3000), (1, 640, 900)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("low", [False, True])
def test_orthogonalise_matches_oracle(shape, dtype, low):
    L = _lsgd()
    print(f"orthogonalise {shape} {dtype} low={low}", flush=True)
    X = _matrices(np.random.default_rng(sum(shape)), *shape, low=low)
    Xd = to_dev(X.astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    Y = L.orthogonalise(Xd)
    assert Y.dtype == Xd.dtype and Y.shape == Xd.shape
    _check(_np(Y), _np(Xd), dtype == "bf16")


@pytest.mark.parametrize("steps,co", [(1, (3.4445, -4.7750, 2.0315)), (2, (1.5, -0.5, 0.0)),
                                      (12, (1.875, -1.25, 0.375)), (3, (0.5, 0.0, 0.0)),
                                      (64, (1.5, -0.5, 0.0)), (4, (2.0, -1.5, 0.5))])
def test_orthogonalise_steps_and_coefficients(steps, co):
    L = _lsgd()
    print(f"orthogonalise {steps} {co}", flush=True)
    X = _matrices(np.random.default_rng(steps), 2, 70, 150)
    for dt in (torch.float32, torch.bfloat16):
        Xd = to_dev(X.astype(np.float32)).to(dt)
        Y = L.orthogonalise(Xd, steps=steps, coefficients=co)
        _check(_np(Y), _np(Xd), dt == torch.bfloat16, steps=steps, coefficients=co)


@pytest.mark.parametrize("shape", [(2, 40, 60), (1, 150, 200)])
@pytest.mark.parametrize("size", [1e30, 1e-9, 1e-13, 1e-25])
def test_orthogonalise_sizes(size, shape):
    """Norms whose square leaves fp32's range, and norms far below eps, where the
    result is a small multiple of X (with its precision all the same)."""
    L = _lsgd()
    print(f"orthogonalise {shape} times {size}", flush=True)
    X = (_matrices(np.random.default_rng(4), *shape) * size).astype(np.float32)
    got = _np(L.orthogonalise(to_dev(X)))
    want = B.newton_schulz(X.astype(np.float64))
    # as the fp32 cases of ordinary size, whose distance is below 2e-6
    e = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert e <= 1e-5, e


def test_orthogonalise_zeros_and_specials():
    """A zero matrix stays zero; one NaN or infinity makes its own matrix NaN and
    leaves the other groups' bits alone."""
    L = _lsgd()
    for shape in ((4, 20, 30), (4, 200, 150)):
        print(f"orthogonalise specials {shape}", flush=True)
        X = _matrices(np.random.default_rng(6), *shape).astype(np.float32)
        clean = L.orthogonalise(to_dev(X))
        X[1] = 0
        X[2, 3, 5] = np.nan
        X[3, 0, 0] = np.inf
        Y = L.orthogonalise(to_dev(X))
        assert torch.equal(Y[0], clean[0])
        assert (Y[1] == 0).all()
        assert torch.isnan(Y[2]).all() and torch.isnan(Y[3]).all()


def test_orthogonalise_views_in_place_and_shared():
    """Views at odd offsets with padded rows, groups side by side in a row, out = X,
    one matrix for all groups: the same bits as contiguous tensors, and nothing
    written outside."""
    L = _lsgd()
    rng = np.random.default_rng(7)
    for dt in (torch.float32, torch.bfloat16):
        for M, N in ((30, 41), (150, 141), (141, 300)):
            print(f"orthogonalise views {dt} {M} {N}", flush=True)
            room = to_dev(rng.standard_normal((3, M + 3, N + 5)).astype(np.float32)).to(dt)
            X = room[:, 1:M + 1, 3:N + 3]
            want = L.orthogonalise(X.contiguous())
            keep = room.clone()
            out = torch.full((M, 3, N + 2), 9.0, device=device(), dtype=dt)
            L.orthogonalise(X, out=out[:, :, :N].transpose(0, 1))
            assert torch.equal(out[:, :, :N].transpose(0, 1), want) and (out[:, :, N:] == 9.0).all()
            L.orthogonalise(X, out=X)
            assert torch.equal(X, want)
            keep[:, 1:M + 1, 3:N + 3] = want
            assert torch.equal(room, keep)
            E = keep[:1, 1:M + 1, 3:N + 3].expand(3, M, N)
            Y = L.orthogonalise(E)
            assert torch.equal(Y[0], Y[2])


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("shape", [(3, 24, 40), (2, 100, 100), (4, 130, 70), (2, 150, 260)])
def test_orthogonal_update_matches_oracle(shape, nesterov):
    """The update of a layer inside flat rows (as the replicas hold it), at an
    offset that is no multiple of four; the rest of the rows stays."""
    L = _lsgd()
    print(f"update {shape} nesterov={nesterov}", flush=True)
    K, M, N = shape
    rng = np.random.default_rng(sum(shape))
    Pn = M * N + 77
    flat = rng.standard_normal((2, K, Pn)).astype(np.float32)
    W, U = to_dev(flat[0]), to_dev(flat[1])
    G = to_dev(_matrices(rng, K, M, N).astype(np.float32))
    view = lambda t: t[:, 13:13 + M * N].view(K, M, N)  # noqa: E731
    w0, u0 = _np(view(W)), _np(view(U))
    lr, m, wd, scale = 0.05, 0.9, 0.1, 1.7
    L.orthogonal_update(view(W), view(U), G, lr, m, wd, nesterov=nesterov, scale=scale)
    w, u, o = B.orthogonal_update(w0, u0, _np(G), lr, m, wd, nesterov, scale)
    got_u, got_w = _np(view(U)), _np(view(W))
    # u = m u + g and w = keep w + step o: two roundings each
    assert np.all(np.abs(got_u - u) <= 2 * 2.0 ** -24 * (np.abs(u0) + np.abs(_np(G))))
    f = np.float32
    d = (_np(G) + float(f(m)) * u) if nesterov else u
    near = np.abs(B.newton_schulz_rounded(d, 2) - o).max()
    tol = 3 * 2.0 ** -24 * (np.abs(w0) + lr * scale * np.abs(o)) + lr * scale * (
        4 * near + 2 * 2.0 ** -24 * np.abs(o).max())
    assert np.all(np.abs(got_w - w) <= tol), np.max(np.abs(got_w - w) / tol)
    for t, want in ((W, flat[0]), (U, flat[1])):
        t = t.cpu().numpy()
        assert np.array_equal(t[:, :13], want[:, :13])
        assert np.array_equal(t[:, 13 + M * N:], want[:, 13 + M * N:])


def test_orthogonal_update_in_bf16_precision():
    L = _lsgd()
    print("update bf16 precision", flush=True)
    rng = np.random.default_rng(21)
    for K, M, N in ((2, 48, 64), (2, 200, 160)):
        W0 = rng.standard_normal((K, M, N)).astype(np.float32)
        U0 = rng.standard_normal((K, M, N)).astype(np.float32)
        G0 = _matrices(rng, K, M, N).astype(np.float32)
        W, U = to_dev(W0), to_dev(U0)
        L.orthogonal_update(W, U, to_dev(G0), 0.1, 0.9, gemm_dtype=torch.bfloat16)
        w, u, o = B.orthogonal_update(W0.astype(np.float64), U0.astype(np.float64),
                                      G0.astype(np.float64), 0.1, 0.9, 0.0, False, 1.0)
        near = np.abs(B.newton_schulz_rounded(u, 1) - o).max()
        assert np.abs(_np(W) - w).max() <= 0.1 * 4 * near + 2.0 ** -22 * np.abs(w).max()


def test_orthogonal_update_refuses_one_tensor_twice():
    L = _lsgd()
    a, b = (torch.ones(2, 3, 4, device=device()) for _ in range(2))
    for bad in ((a, a, b), (a, b, a), (a, b, b)):
        with pytest.raises(ValueError, match="overlap"):
            L.orthogonal_update(*bad, 0.1, 0.9)
    assert (a == 1).all() and (b == 1).all()


def test_updates_on_streams_and_in_graphs():
    """Two captured graphs with a workspace each, replayed in turn with eager calls
    between them, and a call on a side stream: the eager bits every time."""
    L = _lsgd()
    print("update streams and graphs", flush=True)
    rng = np.random.default_rng(31)
    for K, M, N in ((2, 60, 90), (2, 140, 190)):
        W = [to_dev(rng.standard_normal((K, M, N)).astype(np.float32)) for _ in range(2)]
        U = [torch.zeros_like(W[0]) for _ in range(2)]
        G = to_dev(rng.standard_normal((K, M, N)).astype(np.float32))
        eager = [(w.clone(), u.clone()) for w, u in zip(W, U)]
        ws = [L.orthogonalise_workspace(K, M, N) for _ in range(2)]
        args = (0.1, 0.9, 0.01)
        graphs = []
        for i in range(2):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[i]):
                L.orthogonal_update(W[i], U[i], G, *args, workspace=ws[i])
        for k in range(3):
            for i in range(2):
                graphs[i].replay()
                L.orthogonal_update(*eager[i], G, *args)
            torch.cuda.synchronize()
            for i in range(2):
                assert torch.equal(W[i], eager[i][0]) and torch.equal(U[i], eager[i][1])
            G.copy_(to_dev(rng.standard_normal((K, M, N)).astype(np.float32)))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        want = L.orthogonalise(G)
        with torch.cuda.stream(side):
            got = L.orthogonalise(G)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_local_step_of_a_large_layer():
    """The operators together, as a round uses them: K replicas of one linear
    layer fit a target by products in 8 bits, orthogonalised updates and the
    replica average; every quantity against the formulas in float64 on the same
    8-bit values, step by step."""
    L = _lsgd()
    print("local step of a large layer", flush=True)
    rng = np.random.default_rng(41)
    K, T, I, O = 3, 64, 96, 80
    flat = to_dev(np.repeat(0.1 * rng.standard_normal((1, I * O)), K, axis=0).astype(np.float32))
    W = flat.view(K, I, O)
    U = torch.zeros_like(W)
    for step in range(3):
        x = to_dev(rng.standard_normal((K, T, I)).astype(np.float32))
        target = to_dev(rng.standard_normal((K, T, O)).astype(np.float32))
        xq, xt = L.quantise_blocks(x, both=True)
        _, wt = L.quantise_blocks(W, both=True)
        y = L.grouped_gemm_blocks(xq, wt)
        _, dt = L.quantise_blocks((y - target) / T, "e5m2", both=True)
        dw = L.grouped_gemm_blocks(xt, dt)
        val = lambda t: B.values(_np(t.q), _np(t.scale))  # noqa: E731
        exact_dw = (val(xt) @ val(dt).transpose(0, 2, 1))
        assert np.abs(_np(dw) - exact_dw).max() <= 1e-5 * np.abs(exact_dw).max()
        w0, u0 = _np(W), _np(U)
        L.orthogonal_update(W, U, dw, 0.02, 0.95, 0.01, nesterov=True)
        w, u, o = B.orthogonal_update(w0, u0, _np(dw), 0.02, 0.95, 0.01, True, 1.0)
        assert np.abs(_np(U) - u).max() <= 1e-6 * np.abs(u).max()
        assert np.abs(_np(W) - w).max() <= 0.02 * 1e-4 * np.abs(o).max() + 1e-6 * np.abs(w).max()
    mean = _np(flat).mean(axis=0)
    L.replica_average(flat)
    assert np.abs(_np(flat) - mean).max() <= 1e-6 * np.abs(mean).max()


def _steps_on_device(X, pieces, eps=1e-7, coefficients=(3.4445, -4.7750, 2.0315), steps=5):
    """The oracle's two functions for matrices too large for the host: exact in float64
    (pieces = 0), or with the roundings of that many fp16 pieces and fp32 sums."""
    a, b, c = (float(np.float32(v)) for v in coefficients)

    def split(x, scale, n):
        x = x * scale
        hi = x.half().float()
        return [hi, (x - hi).half().float()][:n]

    def product(p, q):
        r = p[0] @ q[0]
        return r if min(len(p), len(q)) == 1 else r + (p[0] @ q[1] + p[1] @ q[0])

    out = torch.empty(X.shape, device=X.device, dtype=torch.float64)
    for g in range(X.shape[0]):
        x = X[g].double()
        flip = x.shape[0] > x.shape[1]
        x = (x.T if flip else x).contiguous()
        x = x / (x.norm() + float(np.float32(eps)))
        if pieces == 0:
            for _ in range(steps):
                A = x @ x.T.contiguous()
                x = a * x + (b * A + c * (A @ A)) @ x
        else:
            S, Sa, Sb = 2.0 ** np.floor(np.log2(np.sqrt(x.numel()))), 2.0 ** 15, 2.0 ** 14
            X2 = split(x.float(), S, 2)
            for _ in range(steps):
                Xp = X2[:pieces]
                A = split(product(Xp, [p.T.contiguous() for p in Xp]) * (Sa / S / S), 1.0, pieces)
                Bm = split((b * sum(A) + c * (product(A, A) / Sa)) / Sa, Sb, pieces)
                y = product(Bm, Xp) / Sb + a * sum(X2)
                X2 = split(y, 1.0, 2)
            x = y.double() / S
        out[g] = x.T if flip else x
    return out


# Ragged edges and the result's rows along either side: few or many matrices of hundreds of
# rows, of thousands. (SHAPES, these and CUTS take every cut that the products have.)
LARGE = [(100, 190, 200), (16, 500, 510), (2, 2040, 2030), (1, 4090, 1500), (1, 8190, 2040),
         (1, 4000, 4090), (1, 4300, 4400), (4, 1500, 1490), (1, 1900, 4500)]


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", LARGE)
def test_large_matrices_match_float64(shape, precision):
    """orthogonalise, and the update (whose result is not rounded to bf16), within the
    module's tolerance."""
    L = _lsgd()
    print(f"large {shape} {precision}", flush=True)
    K, M, N = shape
    dt = torch.bfloat16 if precision == "bf16" else torch.float32
    gen = torch.Generator(device=device()).manual_seed(M + N)
    rand = lambda *s: torch.randn(*s, generator=gen, device=device())  # noqa: E731
    r = max(1, min(M, N) // 16)
    X = (rand(K, M, N) + torch.stack([rand(M, r) @ rand(r, N) for _ in range(K)]) / r ** 0.5).to(dt)
    W, U = torch.zeros(K, M, N, device=device()), torch.zeros(K, M, N, device=device())
    L.orthogonal_update(W, U, X.float(), -1.0, 0.0, gemm_dtype=dt)
    assert torch.equal(U, X.float())
    Y = L.orthogonalise(X)
    pieces = 1 if precision == "bf16" else 2
    for g in range(0, K, max(1, K // 3)):
        want = _steps_on_device(X[g:g + 1], 0)[0]
        near = (_steps_on_device(X[g:g + 1], pieces)[0] - want).abs()
        # W = 0 * 1 + 1 * O rounds once, as orthogonalise's fp32 result does
        for got, half in ((Y[g], torch.finfo(dt).eps / 2), (W[g], 2.0 ** -24)):
            e, floor = (got.double() - want).abs(), half + 35 * 2.0 ** -24
            tol = 4 * near.norm() + floor * want.norm()
            assert e.norm() <= tol, (g, float(e.norm()), float(tol))
            tol = 4 * near.max() + floor * want.abs().max()
            assert e.max() <= tol, (g, float(e.max()), float(tol))


def test_update_in_bf16_precision_of_a_large_layer_in_flat_rows():
    """Momentum, decay and Nesterov on matrices that take the one-piece products, inside
    rows that are longer than them."""
    L = _lsgd()
    print("update large flat", flush=True)
    K, M, N = 2, 600, 401
    gen = torch.Generator(device=device()).manual_seed(5)
    flat = [torch.randn(K, M * N + 9, generator=gen, device=device()) for _ in range(3)]
    W, U, G = (t[:, 5:5 + M * N].view(K, M, N) for t in flat)
    kept = [(t[:, :5].clone(), t[:, 5 + M * N:].clone()) for t in flat]
    f = lambda v: float(np.float32(v))  # noqa: E731
    lr, m, wd = 0.05, 0.9, 0.1
    w0, u0, g0 = W.double(), U.double(), G.double()
    L.orthogonal_update(W, U, G, lr, m, wd, nesterov=True, gemm_dtype=torch.bfloat16)
    u = f(m) * u0 + g0
    d = g0 + f(m) * u
    o = _steps_on_device(d, 0)
    near = (_steps_on_device(d, 1) - o).abs().max()
    w = (1 - f(lr) * f(wd)) * w0 - f(lr) * o
    assert ((U.double() - u).abs() <= 2 * 2.0 ** -24 * (u0.abs() + g0.abs())).all()
    tol = 3 * 2.0 ** -24 * (w0.abs() + lr * o.abs()) + lr * (
        4 * near + 36 * 2.0 ** -24 * o.abs().max())
    assert ((W.double() - w).abs() <= tol).all()
    for t, (a, b) in zip(flat, kept):
        assert torch.equal(t[:, :5], a) and torch.equal(t[:, 5 + M * N:], b)


def test_groups_past_32_bit_offsets():
    """Three tall matrices, 3.2e9 elements: the last of them as a matrix alone."""
    L = _lsgd()
    print("orthogonalise past 32 bits", flush=True)
    gen = torch.Generator(device=device()).manual_seed(6)
    X = torch.randn(3, 2 ** 20, 1024, generator=gen, device=device(), dtype=torch.bfloat16)
    Y = L.orthogonalise(X)[2:]
    X = X[2:].clone()
    want = L.orthogonalise(X)
    # (the cut of the products may differ, and with it the order of their sums: two results
    # of one precision are each within the tolerance of the exact one)
    exact, near = _steps_on_device(X, 0), _steps_on_device(X, 1)
    tol = 4 * (near - exact).norm() + (2.0 ** -8 + 35 * 2.0 ** -24) * exact.norm()
    for got in (Y, want):
        assert (got.double() - exact).norm() <= tol


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(2 ** 20, 1024), (1024, 2 ** 20)])
def test_one_entry_holds_the_norm_of_the_largest_matrix(shape, dtype):
    """2^30 elements, all but one of them zero: that one is held as high as any entry can be,
    and the result is its singular value's course, s := s (a + b s^2 + c s^4), at its place.

    From 1 on the course is 0.70, 1.11, 0.72, 1.09, 0.70, and an error of one step grows by
    |a + 3 b s^2 + 5 c s^4| <= 1.3 in each of the next, to below 2 in all. One step's own: in
    fp32 precision 35 2^-24 (see the top); with operands of 11 bits, off by u = 2^-11, A is off
    by 3 u (two X, A itself), A A by 6 u, B by one more, B X by yet another, so at s = 1.12
    5 |b| s^3 + 8 |c| s^5 = 62 u."""
    L = _lsgd()
    print(f"one entry {shape} {dtype}", flush=True)
    M, N = shape
    X = torch.zeros(1, M, N, device=device(),
                    dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    X[0, M - 3, 7] = -1.0
    Y = L.orthogonalise(X)
    s = -1.0 / (1.0 + float(np.float32(1e-7)))
    a, b, c = (float(np.float32(v)) for v in (3.4445, -4.7750, 2.0315))
    for _ in range(5):
        s = s * (a + b * s ** 2 + c * s ** 4)
    got = float(Y[0, M - 3, 7])
    step = 35 * 2.0 ** -24 if dtype == "fp32" else 62 * 2.0 ** -11 + 2.0 ** -8
    assert abs(got - s) <= 5 * 2 * step, (got, s)
    Y[0, M - 3, 7] = 0
    assert bool((Y == 0).all())


@pytest.mark.parametrize("shape", [(4, 20, 30), (4, 200, 150), (4, 400, 500)])
@pytest.mark.parametrize("bits", [0x7FC0, 0x7FFF, -1, 0x7F81, 0x7F80])
def test_specials_in_bf16(shape, bits):
    """A NaN of any pattern or an infinity makes its own bf16 matrix NaN in every entry,
    whichever kernels it takes, and leaves the other groups' bits alone; zeros stay."""
    L = _lsgd()
    print(f"specials bf16 {shape} {bits:x}", flush=True)
    X = to_dev(_matrices(np.random.default_rng(6), *shape).astype(np.float32)).to(torch.bfloat16)
    clean = L.orthogonalise(X)
    X[1] = 0
    X.view(torch.int16)[2, 3, 5] = bits
    Y = L.orthogonalise(X)
    assert torch.equal(Y[0], clean[0]) and torch.equal(Y[3], clean[3])
    assert (Y[1] == 0).all()
    assert torch.isnan(Y[2]).all()


def test_overlapping_tensors_are_refused():
    """Views that share some elements, and an ``out`` that is neither X itself nor apart from
    it: refused before anything is written. Rows that lie between each other's are not."""
    L = _lsgd()
    print("overlaps", flush=True)
    buf = torch.ones(2, 200, device=device())
    view = lambda at: buf[:, at:at + 60].view(2, 6, 10)  # noqa: E731
    for at in ((0, 59, 130), (0, 70, 129), (70, 129, 0), (5, 70, 0)):
        with pytest.raises(ValueError, match="overlap"):
            L.orthogonal_update(*(view(v) for v in at), 0.1, 0.9)
    for bad in (view(59), buf[:1, :60].view(1, 6, 10).expand(2, 6, 10),
                buf.as_strided((2, 6, 10), (100, 11, 1))):
        with pytest.raises(ValueError, match="overlap"):
            L.orthogonalise(view(0), out=bad)
    blocks = L.quantise_blocks(view(0))
    room = torch.zeros(2, 6, 128, device=device(), dtype=torch.uint8)
    inside = L.Blocks(room.view(torch.float8_e4m3fn), blocks.scale, 10)
    with pytest.raises(ValueError, match="overlap"):
        L.grouped_gemm_blocks(inside, blocks, out=room.view(torch.float32)[:, :, :6])
    assert (buf == 1).all() and (room == 0).all()
    G = to_dev(_matrices(np.random.default_rng(3), 2, 6, 10).astype(np.float32))
    W, U = view(0), view(60)
    want = [W.clone(), U.clone()]
    L.orthogonal_update(*want, G, 0.1, 0.9)
    L.orthogonal_update(W, U, G, 0.1, 0.9)
    assert torch.equal(W, want[0]) and torch.equal(U, want[1])


# Few wide or many small matrices, whose products take 64 x 64 tiles of three or four stages
CUTS = [(15, 18, 2318), (15, 2318, 18), (26, 400, 448), (26, 448, 400), (1, 450, 500)]


@pytest.mark.parametrize("precision", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", CUTS)
def test_small_tiles_match_float64(shape, precision):
    test_large_matrices_match_float64(shape, precision)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 141, 300), (2, 450, 390)])
def test_whatever_the_workspace_holds(shape, dtype):
    """Full of NaN, of zeros, or of what a call on another matrix left: the same bits."""
    L = _lsgd()
    print(f"workspace {shape} {dtype}", flush=True)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.default_rng(9)
    X, other = (to_dev(_matrices(rng, *shape).astype(np.float32)).to(dt) for _ in range(2))
    want = L.orthogonalise(X)
    ws = L.orthogonalise_workspace(*shape, dtype=dt)
    assert ws.numel() > 0
    for before in (lambda: ws.fill_(255), lambda: ws.zero_(),
                   lambda: L.orthogonalise(other, workspace=ws),
                   lambda: L.orthogonalise(other * float("nan"), workspace=ws)):
        before()
        assert torch.equal(L.orthogonalise(X, workspace=ws), want)


def test_precision_does_not_depend_on_the_number_of_matrices():
    """Few long rows, alone and as one of many, where the products take other tiles: sums of as
    many roundings, in another order, are off by as much (their rms over 10^6 results; a
    quarter for chance. With one sum in place of two X X^T alone would round sqrt(3) times
    as far)."""
    L = _lsgd()
    print("precision in a crowd", flush=True)
    gen = torch.Generator(device=device()).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen, device=device())  # noqa: E731
    X = rand(1, 256, 4096) + 0.5 * rand(1, 256, 16) @ rand(1, 16, 4096)
    want = _steps_on_device(X, 0)
    alone = (L.orthogonalise(X).double() - want).norm()
    for G in (200, 256):
        many = (L.orthogonalise(X.expand(G, 256, 4096))[G - 1:].double() - want).norm()
        assert many <= 1.25 * alone, (G, float(many / alone))


@pytest.mark.parametrize("shape", [(3, 30, 41), (3, 150, 141)])
def test_update_with_a_shared_gradient_and_replicas_side_by_side(shape):
    """One gradient for every replica (expand), W and U in rows that hold all replicas' rows:
    the bits of separate contiguous tensors."""
    L = _lsgd()
    print(f"update shared {shape}", flush=True)
    K, M, N = shape
    rng = np.random.default_rng(2)
    room = to_dev(rng.standard_normal((2, M, K, N + 2)).astype(np.float32))
    W, U = (t[:, :, 1:N + 1].transpose(0, 1) for t in room)
    g = to_dev(_matrices(rng, 1, M, N).astype(np.float32))
    w, u, before = W.contiguous(), U.contiguous(), room.clone()
    L.orthogonal_update(w, u, g.expand(K, M, N).contiguous(), 0.1, 0.9, 0.01, nesterov=True)
    L.orthogonal_update(W, U, g.expand(K, M, N), 0.1, 0.9, 0.01, nesterov=True)
    assert torch.equal(W, w) and torch.equal(U, u)
    for i, t in enumerate((w, u)):
        before[i][:, :, 1:N + 1] = t.transpose(0, 1)
    assert torch.equal(room, before)
