"""The operators of a large matrix layer's local step, one by one: writing a
tensor in 8 bits with a scale for each block of 128 (``quantise_blocks``), the
grouped product of two such tensors (``grouped_gemm_blocks``), and the update
by an orthogonalised momentum (``orthogonalise``, ``orthogonal_update``).

A tensor in blocks is a matrix [G][M][N] of 8-bit floats (e4m3: four exponent
bits, largest value 448; e5m2: five, 57344), its rows padded with zeros to a
multiple of 128, and one power of two for each row and 128 columns: the
smallest 2^e, -127 <= e <= 127, with max |x| <= 2^e times the largest 8-bit value
(1 for a block of zeros). Scales are held as e + 127 in a byte, their rows
padded with 1 to a multiple of four. An element is q 2^e, q the nearest 8-bit
float to x 2^-e, ties to even.

The product is C[g] = A[g] B[g]^T, both operands in blocks along the
contracted dimension: y = x w takes w^T, dx = dy w^T takes dy and w, and
dw = x^T dy takes x^T and dy^T, so a tensor that is read both ways is written
both ways in one call.

Orthogonalising maps X = U S V^T towards U V^T by the Newton-Schulz steps
X := a X + (b A + c A A) X, A = X X^T, from X / (|X|_F + eps), on the
transposed matrix where that has fewer rows. The update is
u = m u + g, d = g + m u (Nesterov) or u, w = (1 - lr wd) w - lr s O(d).

``run`` computes the plain forms on torch unless ``own`` is set, ``exact`` the
definitions in 64 bits.
"""
import math

import torch

own = False

STEPS, EPS = 5, 1e-7
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01
FORMATS = {"e4m3": (torch.float8_e4m3fn, 9, 3, -6), "e5m2": (torch.float8_e5m2, 16, 2, -14)}


def _quantise(name, G, M, N, dtype, fmt, both):
    return dict(name=name, kind="quantise", G=G, M=M, N=N, dtype=dtype, fmt=fmt, both=both)


def _product(name, G, M, N, K, out, fmt_a="e4m3", fmt_b="e4m3"):
    return dict(name=name, kind="product", G=G, M=M, N=N, K=K, out=out, fmt_a=fmt_a, fmt_b=fmt_b)


def _orthogonalise(name, G, M, N, dtype):
    return dict(name=name, kind="orthogonalise", G=G, M=M, N=N, dtype=dtype)


def _update(name, G, M, N, nesterov):
    return dict(name=name, kind="update", G=G, M=M, N=N, nesterov=nesterov)


def listed():
    return [
        # one worker's mini-batch of 64 hidden states, written for the next layer's product alone
        _quantise("quantise_batch", 1, 64, 512, "bf16", "e4m3", False),
        # gradients of an odd layer, whose rows and columns both end inside a block, both ways
        _quantise("quantise_ragged", 3, 1537, 771, "fp32", "e5m2", True),
        # a large batch's activations, both ways: the forward product and the weight gradient
        _quantise("quantise_tokens", 1, 16384, 8192, "bf16", "e4m3", True),
        # the hidden layer of the 512-wide MLP on its 16 replicas, batch 128
        _product("product_mlp_512", 16, 128, 512, 512, "fp32"),
        # one token through a large layer: the weights' bytes are all there is
        _product("product_token", 1, 1, 8192, 8192, "bf16"),
        # a weight gradient of ragged sizes, e4m3 activations with e5m2 gradients
        _product("product_wgrad_ragged", 3, 1537, 771, 1000, "fp32", "e4m3", "e5m2"),
        # a large batch through a large layer: the matrix cores' rate
        _product("product_tokens", 1, 8192, 8192, 8192, "bf16"),
        # four replicas of a small square layer: launches and latency
        _orthogonalise("orthogonalise_64", 4, 64, 64, "fp32"),
        # a layer of 1000 to 333 units, no multiple of a tile, more rows than columns
        _orthogonalise("orthogonalise_ragged", 5, 1000, 333, "fp32"),
        # a large layer from bf16 gradients
        _orthogonalise("orthogonalise_wide", 1, 4096, 8192, "bf16"),
        # the hidden layer of the 512-wide MLP on its 16 replicas, inside their flat parameter rows
        _update("update_mlp_512", 16, 512, 512, True),
        # the hidden layer of the 2048-wide MLP on eight replicas
        _update("update_wide_2048", 8, 2048, 2048, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    u = rng.random()
    if u < 0.25:
        while True:
            G, M, N = _log(rng, 1, 32), _log(rng, 1, 16384), _log(rng, 1, 16384)
            if G * M * N <= 1 << 26:
                break
        c = _quantise("", G, M, N, rng.choice(["fp32", "bf16"]), rng.choice(["e4m3", "e5m2"]),
                      rng.random() < 0.6)
    elif u < 0.6:
        while True:
            G, M = _log(rng, 1, 32), _log(rng, 1, 8192)
            N, K = _log(rng, 16, 8192), _log(rng, 16, 8192)
            if G * M * N * K <= 1 << 38 and G * max(M * N, N * K, M * K) <= 1 << 26:
                break
        c = _product("", G, M, N, K, rng.choice(["fp32", "bf16"]), rng.choice(["e4m3", "e4m3", "e5m2"]),
                     rng.choice(["e4m3", "e4m3", "e5m2"]))
    else:
        while True:
            G, M, N = _log(rng, 1, 16), _log(rng, 16, 4096), _log(rng, 16, 4096)
            if G * M * N <= 1 << 24:
                break
        if u < 0.8:
            c = _orthogonalise("", G, M, N, rng.choice(["fp32", "bf16"]))
        else:
            c = _update("", G, M, N, rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------- layout
def _up(n, m):
    return (n + m - 1) // m * m


def _blocks(n):
    return (n + 127) // 128


def _dtype(name):
    return torch.float32 if name == "fp32" else torch.bfloat16


def work(case):
    G, M, N = case["G"], case["M"], case["N"]
    if case["kind"] == "quantise":
        one = M * (_up(N, 128) + _up(_blocks(N), 4))
        two = N * (_up(M, 128) + _up(_blocks(M), 4)) if case["both"] else 0
        return {"bytes": G * (M * N * (4 if case["dtype"] == "fp32" else 2) + one + two),
                "flops": 2.0 * G * M * N}
    if case["kind"] == "product":
        K = case["K"]
        return {"bytes": G * ((M + N) * (K + _blocks(K)) + M * N * (4 if case["out"] == "fp32" else 2)),
                "flops": 2.0 * G * M * N * K}
    # X X^T and A A are symmetric: half of their products do
    m, n = min(M, N), max(M, N)
    flops = STEPS * G * (3.0 * m * m * n + 1.0 * m * m * m)
    if case["kind"] == "orthogonalise":
        return {"bytes": 2 * G * M * N * (4 if case["dtype"] == "fp32" else 2), "flops": flops}
    return {"bytes": 5 * 4 * G * M * N, "flops": flops}


# ---------------------------------------------------------------- plain forms
def _quantise_rows(X, fmt):
    """The rows of X [G][M][N] in blocks of 128: (q, scales) in the padded layout."""
    kind, top, _, _ = FORMATS[fmt]
    G, M, N = X.shape
    nb = _blocks(N)
    x = torch.zeros((G, M, nb * 128), device=X.device)
    x[:, :, :N] = X
    x = x.view(G, M, nb, 128)
    amax = x.abs().amax(3)
    mant, e = torch.frexp(amax)
    e = torch.where(mant > 0.875, e - top + 1, e - top)  # the largest value is 0.875 2^top
    e = torch.where(amax == 0, torch.zeros_like(e), e.clamp(-127, 127))
    q = torch.ldexp(x, -e[..., None]).to(kind).view(G, M, nb * 128)
    s = torch.full((G, M, _up(nb, 4)), 127, dtype=torch.uint8, device=X.device)
    s[:, :, :nb] = (e + 127).to(torch.uint8)
    return q, s.view(torch.float8_e8m0fnu)


def _values(q, s, dtype=torch.float32):
    """What a tensor in blocks stands for, padding included."""
    G, M, L = q.shape
    f = s.view(torch.uint8)[:, :, :L // 128].to(torch.int32) - 127
    return torch.ldexp(q.to(dtype).view(G, M, L // 128, 128), f[..., None]).view(G, M, L)


def _newton_schulz(X):
    a, b, c = COEFFICIENTS
    x = X.transpose(1, 2).contiguous() if X.shape[1] > X.shape[2] else X
    norm = x.double().square().sum((1, 2), keepdim=True).sqrt()  # a long sum
    x = (x.double() / (norm + EPS)).float()
    for _ in range(STEPS):
        A = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * A + c * torch.matmul(A, A), x)
    return x.transpose(1, 2) if X.shape[1] > X.shape[2] else x


def _shape_scale(M, N):
    """Weights are [inputs][outputs]."""
    return math.sqrt(max(1.0, N / M))


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "quantise":
        out = _quantise_rows(s["X"].float(), c["fmt"])
        if c["both"]:
            out += _quantise_rows(s["X"].float().transpose(1, 2), c["fmt"])
        return out
    if c["kind"] == "product":
        A, B = _values(*s["A"]), _values(*s["B"])
        return torch.matmul(A, B.transpose(1, 2).contiguous()).to(_dtype(c["out"]))
    if c["kind"] == "orthogonalise":
        return _newton_schulz(s["X"].float()).to(_dtype(c["dtype"])).contiguous()
    W, U, g = s["W"], s["U"], s["g"]
    U.mul_(MOMENTUM).add_(g)
    d = g + MOMENTUM * U if c["nesterov"] else U
    O = _newton_schulz(d)
    W.mul_(1.0 - LR * DECAY).sub_(LR * _shape_scale(c["M"], c["N"]) * O)
    return {"W": W, "U": U}


def _run_own(s):
    from paper_1808_07217_amd import lsgd as L
    c = s["case"]
    if c["kind"] == "quantise":
        if not c["both"]:
            q = L.quantise_blocks(s["X"], c["fmt"])
            return q.q, q.scale
        q, t = L.quantise_blocks(s["X"], c["fmt"], both=True)
        return q.q, q.scale, t.q, t.scale
    if c["kind"] == "product":
        return L.grouped_gemm_blocks(L.Blocks(*s["A"], c["K"]), L.Blocks(*s["B"], c["K"]),
                                     out_dtype=_dtype(c["out"]))
    if c["kind"] == "orthogonalise":
        return L.orthogonalise(s["X"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
    L.orthogonal_update(s["W"], s["U"], s["g"], LR, MOMENTUM, DECAY, nesterov=c["nesterov"],
                        scale=_shape_scale(c["M"], c["N"]), steps=STEPS,
                        coefficients=COEFFICIENTS, eps=EPS)
    return {"W": s["W"], "U": s["U"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _activations(gen, G, M, N):
    """Hidden states: a normal bulk, and a few columns far above it."""
    x = torch.randn((G, M, N), generator=gen, device="cuda")
    loud = torch.rand((G, 1, N), generator=gen, device="cuda") < 0.01
    return torch.where(loud, x * 20.0, x)


def _gradients(gen, G, M, N):
    """Noise, and a part of low rank above it, as a batch's gradients have."""
    r = max(1, min(M, N) // 16)
    left = torch.randn((G, M, r), generator=gen, device="cuda")
    right = torch.randn((G, r, N), generator=gen, device="cuda")
    left = left * torch.logspace(0, -1, r, device="cuda")
    x = torch.randn((G, M, N), generator=gen, device="cuda")
    return 1e-3 * (x + torch.matmul(left, right) * (2.0 / math.sqrt(r)))


def prepare(case, seed):
    gen = _generator(seed)
    c = dict(case)
    G, M, N = c["G"], c["M"], c["N"]
    s = {"case": c}
    if c["kind"] == "quantise":
        make = _activations if c["fmt"] == "e4m3" else _gradients
        s["X"] = make(gen, G, M, N).to(_dtype(c["dtype"]))
    elif c["kind"] == "product":
        make = {"e4m3": _activations, "e5m2": _gradients}
        s["A"] = _quantise_rows(make[c["fmt_a"]](gen, G, M, c["K"]), c["fmt_a"])
        s["B"] = _quantise_rows(make[c["fmt_b"]](gen, G, N, c["K"]) / math.sqrt(c["K"]), c["fmt_b"])
    elif c["kind"] == "orthogonalise":
        s["X"] = _gradients(gen, G, M, N).to(_dtype(c["dtype"]))
    else:
        # the layer's weights and momentum buffer inside each replica's flat row, as
        # the replicas hold them: weight, then bias, rows a multiple of 64 elements
        P = _up(M * N + N, 64)
        for name in ("W", "U"):
            s[name] = torch.zeros((G, P), device="cuda")[:, :M * N].view(G, M, N)
        s["W"].copy_(torch.randn((G, M, N), generator=gen, device="cuda") / math.sqrt(M))
        s["U"].copy_(10.0 * _gradients(gen, G, M, N))
        s["g"] = _gradients(gen, G, M, N)
    return s


# ---------------------------------------------------------------- 64 bits
def _exact_blocks(X, fmt):
    _, top, bits, low = FORMATS[fmt]
    G, M, N = X.shape
    nb = _blocks(N)
    x = torch.nn.functional.pad(X, (0, nb * 128 - N)).reshape(G, M, nb, 128)
    amax = x.abs().max(dim=3, keepdim=True).values
    most = 0.875 * 2.0 ** top
    e = torch.ceil(torch.log2(amax / most))
    # the logarithm may land on the wrong side of a power of two
    e = torch.where(amax > most * torch.exp2(e), e + 1, e)
    e = torch.where(amax <= most * torch.exp2(e - 1), e - 1, e)
    e = torch.where(amax == 0, torch.zeros_like(e), e.clamp(-127.0, 127.0))
    y = x / torch.exp2(e)
    # the spacing of 8-bit floats around y, that of the subnormal ones at least
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** low))).clamp_min(low) - bits)
    q = (torch.round(y / step) * step).reshape(G, M, nb * 128)
    s = torch.nn.functional.pad(torch.exp2(e[..., 0]), (0, _up(nb, 4) - nb), value=1.0)
    return q, s


def _exact_orthogonal(X):
    a, b, c = COEFFICIENTS
    flip = X.shape[1] > X.shape[2]
    x = X.mT.contiguous() if flip else X
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + EPS)
    for _ in range(STEPS):
        gram = x @ x.mT.contiguous()
        ax = gram @ x
        x = a * x + b * ax + c * (gram @ ax)
    return x.mT.contiguous() if flip else x


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "quantise":
        X = s["X"].double()
        out = _exact_blocks(X, c["fmt"])
        return out + _exact_blocks(X.mT, c["fmt"]) if c["both"] else out
    if c["kind"] == "product":
        def values(q, scale):
            f = scale.to(torch.float64)[:, :, :q.shape[2] // 128]
            return q.to(torch.float64) * f.repeat_interleave(128, dim=2)
        return values(*s["A"]) @ values(*s["B"]).mT.contiguous()
    if c["kind"] == "orthogonalise":
        return _exact_orthogonal(s["X"].double())
    W, U, g = (s[k].double() for k in ("W", "U", "g"))
    U = MOMENTUM * U + g
    d = g + MOMENTUM * U if c["nesterov"] else U
    return {"W": W - LR * (DECAY * W + _shape_scale(c["M"], c["N"]) * _exact_orthogonal(d)), "U": U}
