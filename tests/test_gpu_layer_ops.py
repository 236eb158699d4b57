"""Layer operators on the GPU: norms, linear layers and their gradients against a plain implementation in 64 bits.

Tolerances, derived before any run.  u = 2^-9 (bf16) or 2^-24 (fp32) is the relative error of one
rounding; a product or sum in fp32 adds at most 2^-23 of its size (the tensor cores truncate where
the others round), so a sum of n products is off by at most n 2^-23 of the sum S of the products' magnitudes.

* linear, forward: z is off by (in + 2) 2^-23 S with S = |x| |w|^T + |bias|.  The activations' slopes
  are at most 1.13; their own evaluation is good to 2^-18 of |z| (a fast exponential's 2 ulp, an argument's
  rounding times a slope of 0.8 z at |z| < 10).  Then one rounding, u |y|.
* linear, backward: dz is off by 2^-17 |dy| |mul| (1 + |z|) from the derivative's evaluation and, as an operand of
  the products in bf16, by u |dz|; a product with it by those of S plus (n + 2) 2^-23 S; one rounding.
* norms: statistics are sums of cols terms: cols 2^-23 relative for sums of squares (all of one
  sign), so half of that for rstd; the mean is off by cols 2^-23 of mean |x|.  y and dx follow by their formulas.

A test takes the bound with a factor of 2 for what these first-order terms leave out.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -9, "fp32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
E = 2.0 ** -23
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


@pytest.fixture(scope="module")
def mp():
    import paper_2605_29489_gb300 as m

    return m


def act_id(mp, a):
    return {"none": mp.MP_ACT_NONE, "relu": mp.MP_ACT_RELU, "silu": mp.MP_ACT_SILU, "gelu": mp.MP_ACT_GELU,
            "gelu_tanh": mp.MP_ACT_GELU_TANH}[a]


def make(shape, dtype, seed, scale=1.0, pad=0, shift=0):
    """a random matrix (or vector) on the GPU: rows `pad` elements further apart than they are long, the first element
    `shift` elements into its buffer; everything around it is NaN"""
    g = torch.Generator().manual_seed(seed)
    v = (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(DT[dtype])
    if not pad and not shift:
        return v.cuda()
    rows, cols = shape
    buf = torch.full((shift + rows * (cols + pad) + 64,), float("nan"), dtype=DT[dtype], device="cuda")
    m = buf[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(v)
    return m


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def erf(z):
    return torch.erf(torch.from_numpy(np.asarray(z))).numpy()


def act(z, a):
    if a == "relu":
        return np.where(z > 0, z, 0.0)
    if a == "silu":
        return z / (1 + np.exp(-z))
    if a == "gelu":
        return 0.5 * z * (1 + erf(z / math.sqrt(2)))
    if a == "gelu_tanh":
        return 0.5 * z * (1 + np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def act_grad(z, a):
    if a == "relu":
        return (z > 0).astype(float)
    if a == "silu":
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    if a == "gelu":
        return 0.5 * (1 + erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if a == "gelu_tanh":
        t = np.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def near(got, want, bound, what):
    got = f64(got)
    assert got.shape == want.shape, what
    assert np.isfinite(got).all(), what
    worst = np.max(np.abs(got - want) - 2 * bound) if want.size else -1.0
    assert worst <= 0, (what, worst, float(np.max(np.abs(got - want))))


# ---- norms --------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (1, 896), (3, 8), (5, 7), (2, 33), (9, 257), (130, 128), (64, 1024), (33, 2056), (700, 1537),
               (17, 4096), (3, 5003), (5, 8192), (2, 8200), (3, 12288), (2, 16384), (2, 16400), (1, 20001), (1201, 64),
               # many rows of whole vectors: the backward pass's ring, of every width and number of slots
               (700, 1024), (1300, 1032), (611, 2056), (777, 4096), (640, 8192), (3001, 256), (900, 512), (1000, 520), (2000, 896),
               # short rows, several to a warp, whole CTAs of them and one too many
               (1, 64), (15, 128), (16, 128), (17, 120), (5000, 72), (4097, 128), (129, 33), (1000, 3)]


@pytest.mark.parametrize("shape", NORM_SHAPES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norm_and_its_gradients(mp, shape, kind, dtype):
    rows, cols = shape
    layer, u = kind == "layer", U[dtype]
    pad, shift = ((0, 0), (8, 8), (3, 1))[(rows + cols) % 3]
    x = make(shape, dtype, 1, 2.0, pad, shift)
    x += 0.5
    dy, add = make(shape, dtype, 2, 0.1, pad), make(shape, dtype, 3, 0.1)
    w, b = make((cols,), dtype, 4), make((cols,), dtype, 5) if layer else None
    k = mp.MP_NORM_LAYER if layer else mp.MP_NORM_RMS
    y, mean, rstd = mp.mp_norm(x, w, b, eps=1e-5, kind=k)
    dx, dw, db = mp.mp_norm_backward(dy, x, w, mean, rstd, kind=k, bias=layer, add=add)

    X, W, G, A = f64(x), f64(w), f64(dy), f64(add)
    mu = X.mean(1, keepdims=True) if layer else np.zeros((rows, 1))
    var = ((X - mu) ** 2).mean(1, keepdims=True)
    r = 1 / np.sqrt(var + 1e-5)
    e_mu = (cols + 2) * E * np.abs(X).mean(1, keepdims=True) if layer else np.zeros((rows, 1))
    # the centred values are off by e_mu and a rounding of theirs, the variance by its terms' and its sum's errors
    e_c = e_mu + E * np.abs(X - mu)
    e_r = r * (0.5 * (cols + 8) * E + r * e_c.mean(1, keepdims=True) + r ** 2 * e_c.mean(1, keepdims=True) ** 2)
    h = (X - mu) * r
    e_h = r * e_c + np.abs(X - mu) * e_r + E * np.abs(h)
    want = h * W + (f64(b) if layer else 0.0)
    near(rstd, r[:, 0], e_r[:, 0] + E * r[:, 0], "rstd")
    if layer:
        near(mean, mu[:, 0], e_mu[:, 0] + E * np.abs(mu[:, 0]), "mean")
    near(y, want, np.abs(W) * e_h + 2 * E * (np.abs(h * W) + np.abs(want)) + u * np.abs(want), "y")

    g = G * W
    p1, p2 = (g * h).mean(1, keepdims=True), g.mean(1, keepdims=True) if layer else 0.0
    want = r * (g - p2 - h * p1) + A
    s1 = (np.abs(g) * (np.abs(h) * (cols + 4) * E + e_h)).mean(1, keepdims=True)
    s2 = (cols + 4) * E * np.abs(g).mean(1, keepdims=True) if layer else 0.0
    inner = np.abs(g) + np.abs(p2) + np.abs(h * p1)
    bound = r * (s2 + np.abs(h) * s1 + e_h * np.abs(p1) + 4 * E * inner) + e_r * inner + 2 * E * (np.abs(want) + np.abs(A))
    near(dx, want, bound + u * np.abs(want), "dx")
    want = (G * h).sum(0)
    near(dw, want, (np.abs(G) * (e_h + (rows + 2) * E * np.abs(h))).sum(0) + u * np.abs(want), "dw")
    if layer:
        want = G.sum(0)
        near(db, want, (rows + 2) * E * np.abs(G).sum(0) + u * np.abs(want), "db")


def test_norm_without_weight_in_place_and_on_no_rows(mp):
    x = make((6, 96), "fp32", 1)
    want, _, _ = mp.mp_norm(x, kind=mp.MP_NORM_LAYER)
    y, mean, rstd = mp.mp_norm(x, kind=mp.MP_NORM_LAYER, out=x)
    assert y is x and torch.equal(x, want)
    x, dy = make((6, 96), "fp32", 1), make((6, 96), "fp32", 2)
    dx, dw, db = mp.mp_norm_backward(dy, x, None, mean, rstd, kind=mp.MP_NORM_LAYER)
    one, _, _ = mp.mp_norm_backward(dy, x, torch.ones(96, device="cuda"), mean, rstd, kind=mp.MP_NORM_LAYER)
    assert dw is None and db is None and torch.equal(dx, one)
    e = torch.empty((0, 96), device="cuda")
    y, mean, rstd = mp.mp_norm(e, torch.ones(96, device="cuda"), kind=mp.MP_NORM_LAYER)
    assert y.shape == (0, 96) and mean.shape == rstd.shape == (0,)
    dx, dw, db = mp.mp_norm_backward(e, e, torch.ones(96, device="cuda"), mean, rstd, kind=mp.MP_NORM_LAYER, bias=True)
    assert dx.shape == (0, 96) and not dw.any() and not db.any()


def test_norm_of_extreme_rows(mp):
    """constant and zero rows (no variance), large values in one row, NaN and infinity staying in theirs"""
    x = torch.zeros((6, 256), device="cuda")
    x[1] = 3.0
    x[2] = 1e15 * torch.sign(torch.arange(256, device="cuda") - 127.5)
    x[3, 17] = float("nan")
    x[4, 200] = float("inf")
    x[5] = torch.arange(256, device="cuda") / 64 + 1e4
    y, mean, rstd = mp.mp_norm(x, kind=mp.MP_NORM_LAYER, eps=1e-5)
    assert not y[0].any() and not y[1].any() and abs(rstd[0].item() - 1e-5 ** -0.5) < 1e-3
    assert torch.allclose(y[2].abs(), torch.ones(256, device="cuda"))
    assert y[3].isnan().all() and not y[4].isfinite().any() and y[5].isfinite().all()
    want = f64(x[5]) - f64(x[5]).mean()
    want /= np.sqrt((want ** 2).mean() + 1e-5)
    # the mean is a sum of 16 terms per thread and a tree: 23 2^-24 of 1e4 at most, over the deviation of 1.15
    assert np.max(np.abs(f64(y[5]) - want)) < 2e-2


def test_norm_gradients_against_differences(mp):
    """dx, dweight and dbias are the slopes of sum(y * dy) along random directions (central differences in fp32 of
    a function whose third derivative is of the order of one: h^2 = 1e-4 and 2^-23 of sums of 600 terms over h)"""
    x, w, b = make((4, 150), "fp32", 1), make((150,), "fp32", 2), make((150,), "fp32", 3)
    dy = make((4, 150), "fp32", 4)
    k = mp.MP_NORM_LAYER
    _, mean, rstd = mp.mp_norm(x, w, b, kind=k)
    dx, dw, db = mp.mp_norm_backward(dy, x, w, mean, rstd, kind=k, bias=True)
    for n, (t, grad) in enumerate(((x, dx), (w, dw), (b, db))):
        v = make(tuple(t.shape), "fp32", 10 + n)
        v /= v.norm()
        h = 1e-2
        args = [[x, w, b], [x, w, b]]
        args[0][n], args[1][n] = t + h * v, t - h * v
        up, down = (f64(mp.mp_norm(*a, kind=k)[0]) * f64(dy) for a in args)
        assert abs((up.sum() - down.sum()) / (2 * h) - (f64(grad) * f64(v)).sum()) < 5e-3


def test_norm_is_the_same_every_time(mp):
    x, dy, w = make((999, 1024), "bf16", 1), make((999, 1024), "bf16", 2), make((1024,), "bf16", 3)
    _, _, rstd = mp.mp_norm(x, w)
    first = mp.mp_norm_backward(dy, x, w, None, rstd)[:2]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, mp.mp_norm_backward(dy, x, w, None, rstd)[:2]))


# ---- linear layers --------------------------------------------------------------------------------

# rows, in, out: single tokens, a few, ragged ones; inner dimensions below and above one stage; tiles cut short;
# both kernels of the tensor cores
LINEAR_SHAPES = [(1, 1, 1), (1, 64, 128), (1, 896, 1152), (1, 901, 77), (2, 8, 8), (7, 333, 130), (16, 2048, 512),
                 (17, 1000, 129), (33, 72, 1000), (65, 640, 264), (128, 512, 384), (129, 100, 131), (300, 1151, 901),
                 (513, 256, 1024), (1024, 320, 2304), (2000, 136, 4104), (2600, 1000, 2568)]
F32_SHAPES = [(1, 1, 1), (1, 512, 512), (3, 17, 65), (64, 64, 64), (65, 130, 67), (200, 333, 129)]


def linear_case(dtype, shape, seed, mul=False, res=False, bias=False, pad=0, shift=0):
    m, k, n = shape
    return dict(x=make((m, k), dtype, seed, 1.0, pad, shift), w=make((n, k), dtype, seed + 1, k ** -0.5, pad, shift),
                b=make((n,), dtype, seed + 2) if bias else None,
                mul=make((m, n), dtype, seed + 3, 1.0, pad, shift) if mul else None,
                res=make((m, n), dtype, seed + 4, 1.0, pad) if res else None)


def check_forward(mp, dtype, shape, a, mul, res, bias, pad=0, shift=0):
    c = linear_case(dtype, shape, 7, mul, res, bias, pad, shift)
    y, pre = mp.mp_linear(c["x"], c["w"], c["b"], act=act_id(mp, a), mul=c["mul"], residual=c["res"], keep_pre=True)
    u = U[dtype]
    X, W = f64(c["x"]), f64(c["w"])
    B = f64(c["b"]) if bias else 0.0
    M = f64(c["mul"]) if mul else np.ones(())
    R = f64(c["res"]) if res else np.zeros(())
    z = X @ W.T + B
    e_z = (shape[1] + 2) * E * (np.abs(X) @ np.abs(W).T + np.abs(B))
    near(pre, z, e_z + u * np.abs(z), "pre")
    v = act(z, a)
    e_v = 1.13 * e_z + (2.0 ** -18 * np.abs(z) if a not in ("none", "relu") else 0.0)
    want = v * M + R
    near(y, want, np.abs(M) * e_v + 2 * E * (np.abs(v * M) + np.abs(R)) + u * np.abs(want), "y")
    plain, none = mp.mp_linear(c["x"], c["w"], c["b"], act=act_id(mp, a), mul=c["mul"], residual=c["res"])
    assert none is None and torch.equal(plain, y)


@pytest.mark.parametrize("shape", LINEAR_SHAPES)
@pytest.mark.parametrize("form", range(4))
def test_linear_bf16(mp, shape, form):
    a = ACTS[(shape[0] + form) % 5]
    pad, shift = ((0, 0), (8, 8), (5, 3), (0, 1))[form]
    check_forward(mp, "bf16", shape, a, form in (1, 3), form in (2, 3), form % 2 == 0, pad, shift)


@pytest.mark.parametrize("shape", F32_SHAPES)
@pytest.mark.parametrize("form", range(4))
def test_linear_fp32(mp, shape, form):
    a = ACTS[(shape[1] + form) % 5]
    pad, shift = ((0, 0), (4, 4), (5, 3), (0, 1))[form]
    check_forward(mp, "fp32", shape, a, form in (1, 3), form in (2, 3), form % 2 == 0, pad, shift)


@pytest.mark.parametrize("a", ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_activation(mp, a, dtype):
    check_forward(mp, dtype, (70, 200, 136), a, True, True, True)
    check_backward(mp, dtype, (70, 200, 136), a, True, True)


def check_backward(mp, dtype, shape, a, mul, bias, pad=0, shift=0, add=False):
    m, k, n = shape
    u = U[dtype]
    c = linear_case(dtype, shape, 27, mul, False, False, pad, shift)
    dy, pre = make((m, n), dtype, 40, 0.5, pad, shift), make((m, n), dtype, 41, 1.5, pad)
    dxa, dwa = (make((m, k), dtype, 42), make((n, k), dtype, 43)) if add else (None, None)
    dx, dw, db, dm = mp.mp_linear_backward(dy, c["x"], c["w"], pre=pre, act=act_id(mp, a), mul=c["mul"], bias=bias,
                                           dx_add=dxa, dw_add=dwa)
    G, Z, X, W = f64(dy), f64(pre), f64(c["x"]), f64(c["w"])
    M = f64(c["mul"]) if mul else np.ones((m, n))
    dz = G * M * act_grad(Z, a)
    e_dz = 2.0 ** -17 * np.abs(G * M) * (1 + np.abs(Z)) + 2 * E * np.abs(dz)
    if not mul and a == "none":
        e_dz = np.zeros_like(dz)
    e_op = e_dz + (u * np.abs(dz) if dtype == "bf16" else 0.0)
    want = dz @ W + (f64(dxa) if add else 0.0)
    near(dx, want, e_op @ np.abs(W) + (n + 3) * E * (np.abs(dz) @ np.abs(W) + np.abs(want)) + u * np.abs(want), "dx")
    want = dz.T @ X + (f64(dwa) if add else 0.0)
    near(dw, want, e_op.T @ np.abs(X) + (m + 3) * E * (np.abs(dz).T @ np.abs(X) + np.abs(want)) + u * np.abs(want), "dw")
    if bias:
        want = dz.sum(0)
        near(db, want, e_dz.sum(0) + (m + 2) * E * np.abs(dz).sum(0) + u * np.abs(want), "db")
    else:
        assert db is None
    if mul:
        want = G * act(Z, a)
        near(dm, want, np.abs(G) * 2.0 ** -17 * np.abs(Z) + 2 * E * np.abs(want) + u * np.abs(want), "dmul")
    else:
        assert dm is None


@pytest.mark.parametrize("shape", LINEAR_SHAPES)
@pytest.mark.parametrize("form", range(4))
def test_linear_backward_bf16(mp, shape, form):
    a = ACTS[(shape[0] + form + 1) % 5]
    pad, shift = ((0, 0), (8, 8), (5, 3), (0, 1))[form]
    check_backward(mp, "bf16", shape, a, form in (1, 2), form % 2 == 0, pad, shift, form == 1)


@pytest.mark.parametrize("shape", F32_SHAPES)
@pytest.mark.parametrize("form", range(4))
def test_linear_backward_fp32(mp, shape, form):
    a = ACTS[(shape[0] + form + 1) % 5]
    pad, shift = ((0, 0), (4, 4), (5, 3), (0, 1))[form]
    check_backward(mp, "fp32", shape, a, form in (1, 2), form % 2 == 0, pad, shift, form == 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_linear_backward_of_parts(mp, dtype):
    """outputs asked for one at a time are those of the whole call; sums onto themselves; no activation
    and no factor, where dz is dy"""
    c = linear_case(dtype, (50, 96, 80), 3, mul=True)
    dy, pre = make((50, 80), dtype, 8), make((50, 80), dtype, 9)
    s = mp.MP_ACT_SILU
    dx, dw, db, dm = mp.mp_linear_backward(dy, c["x"], c["w"], pre=pre, act=s, mul=c["mul"], bias=True)
    only = mp.mp_linear_backward(dy, c["x"], c["w"], pre=pre, act=s, mul=c["mul"], need_dw=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None and torch.equal(only[3], dm)
    only = mp.mp_linear_backward(dy, c["x"], c["w"], pre=pre, act=s, mul=c["mul"], need_dx=False, need_dw=False, bias=True)
    assert only[0] is None and only[1] is None and torch.equal(only[2], db) and torch.equal(only[3], dm)
    gx, gw = make((50, 96), dtype, 10), make((80, 96), dtype, 11)
    want = mp.mp_linear_backward(dy, c["x"], c["w"], dx_add=gx, dw_add=gw)
    same = mp.mp_linear_backward(dy, c["x"], c["w"], dx_add=gx, dw_add=gw, dx=gx, dw=gw)
    assert same[0] is gx and same[1] is gw and torch.equal(gx, want[0]) and torch.equal(gw, want[1])


def test_linear_in_place_and_side_by_side(mp):
    """y onto the residual or the factor, operands and results as columns of one wider matrix, one row"""
    c = linear_case("bf16", (40, 128, 64), 3, mul=True, res=True)
    want, _ = mp.mp_linear(c["x"], c["w"], mul=c["mul"], residual=c["res"])
    for name in ("mul", "res"):
        d = {k: None if v is None else v.clone() for k, v in c.items()}
        y, _ = mp.mp_linear(d["x"], d["w"], mul=d["mul"], residual=d["res"], out=d[name])
        assert y is d[name] and torch.equal(y, want)
    wide = torch.full((40, 256), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, :128], wide[:, 192:] = c["x"], c["res"]
    mp.mp_linear(wide[:, :128], c["w"], mul=c["mul"], residual=wide[:, 192:], out=wide[:, 128:192])
    assert torch.equal(wide[:, 128:192], want) and torch.equal(wide[:, :128], c["x"]) and torch.equal(wide[:, 192:], c["res"])


def test_linear_on_no_rows(mp):
    for dtype in ("bf16", "fp32"):
        w, e = make((24, 40), dtype, 1), torch.empty((0, 40), dtype=DT[dtype], device="cuda")
        y, pre = mp.mp_linear(e, w, keep_pre=True)
        assert y.shape == pre.shape == (0, 24)
        dx, dw, db, _ = mp.mp_linear_backward(y, e, w, bias=True)
        assert dx.shape == (0, 40) and not dw.any() and not db.any()
        g = make((24, 40), dtype, 2)
        assert torch.equal(mp.mp_linear_backward(y, e, w, dw_add=g)[1], g)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [5, 300])
def test_linear_nonfinite_values_stay_where_they_belong(mp, rows, dtype):
    """a NaN or an infinity in a row of x reaches that row of y alone, one in a row of w that column; extreme
    activations' arguments give their limits"""
    x, w = make((rows, 200), dtype, 1), make((136, 200), dtype, 2, 0.05)
    clean, _ = mp.mp_linear(x, w)
    x[1, 7], w[130, 199] = float("nan"), float("inf")
    y, _ = mp.mp_linear(x, w)
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[1, :] = False
    keep[:, 130] = False
    assert torch.equal(y[keep], clean[keep]) and y[1].isnan().all() and not y[:, 130].isfinite().any()
    one = torch.eye(16, dtype=DT[dtype], device="cuda")
    z = torch.tensor([0.0, -0.0, 1e-30, 80.0, -80.0, 100.0, -100.0, 1e4, -1e4, 1e30, -1e30, 9.0, -9.0, 3.0, -3.0, 0.5],
                     dtype=DT[dtype], device="cuda").view(1, 16)
    for a in ACTS[1:]:
        y, _ = mp.mp_linear(z, one, act=act_id(mp, a))
        with np.errstate(over="ignore"):
            want = act(f64(z), a)
        assert y.isfinite().all(), a
        assert np.all(np.abs(f64(y) - want) <= U[dtype] * 2 * np.abs(want) + 2.0 ** -16), a
        dx, _, _, _ = mp.mp_linear_backward(torch.ones_like(z), z, one, pre=z, act=act_id(mp, a), need_dw=False)
        assert dx.isfinite().all(), a
        with np.errstate(over="ignore", invalid="ignore"):
            want = np.nan_to_num(act_grad(f64(z), a), nan=0.0)
        assert np.all(np.abs(f64(dx) - want) <= U[dtype] * 4 + 2.0 ** -16), a


def test_linear_gradients_against_differences(mp):
    """dx, dw, db and dmul are the slopes of sum(y * dy): central differences, as for the norms"""
    c = linear_case("fp32", (6, 40, 30), 3, mul=True, bias=True)
    dy, s = make((6, 30), "fp32", 9), mp.MP_ACT_GELU_TANH
    _, pre = mp.mp_linear(c["x"], c["w"], c["b"], act=s, mul=c["mul"], keep_pre=True)
    grads = mp.mp_linear_backward(dy, c["x"], c["w"], pre=pre, act=s, mul=c["mul"], bias=True)
    for name, grad in zip(("x", "w", "b", "mul"), grads):
        v = make(tuple(c[name].shape), "fp32", 20)
        v /= v.norm()
        h, out = 1e-2, []
        for sign in (1, -1):
            d = dict(c)
            d[name] = c[name] + sign * h * v
            out.append((f64(mp.mp_linear(d["x"], d["w"], d["b"], act=s, mul=d["mul"])[0]) * f64(dy)).sum())
        assert abs((out[0] - out[1]) / (2 * h) - (f64(grad) * f64(v)).sum()) < 5e-3, name


@pytest.mark.parametrize("rows", [3, 40, 1000])
def test_linear_is_the_same_every_time(mp, rows):
    c = linear_case("bf16", (rows, 2048, 1536), 3, mul=True)
    first, pre = mp.mp_linear(c["x"], c["w"], act=mp.MP_ACT_SILU, mul=c["mul"], keep_pre=True)
    grads = mp.mp_linear_backward(first, c["x"], c["w"], pre=pre, act=mp.MP_ACT_SILU, mul=c["mul"], bias=True)
    for _ in range(3):
        assert torch.equal(mp.mp_linear(c["x"], c["w"], act=mp.MP_ACT_SILU, mul=c["mul"])[0], first)
        again = mp.mp_linear_backward(first, c["x"], c["w"], pre=pre, act=mp.MP_ACT_SILU, mul=c["mul"], bias=True)
        assert all(torch.equal(a, b) for a, b in zip(grads, again))


def test_streams_and_graphs(mp):
    """calls on two streams at once, and a step captured into a graph and replayed on new contents"""
    c = linear_case("bf16", (77, 901, 1151), 3, bias=True)
    w1 = make((1151,), "bf16", 30)

    def step():
        y, pre = mp.mp_linear(c["x"], c["w"], c["b"], act=mp.MP_ACT_SILU, keep_pre=True)
        n, _, rstd = mp.mp_norm(y, w1)
        dn, dw1, _ = mp.mp_norm_backward(n, y, w1, None, rstd)
        return (y, n, dw1, *mp.mp_linear_backward(dn, c["x"], c["w"], pre=pre, act=mp.MP_ACT_SILU, bias=True)[:3])

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(step())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for out in got for a, b in zip(out, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(2):
        c["x"].copy_(make((77, 901), "bf16", 50))
        graph.replay()
        torch.cuda.synchronize()
        now = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(now, step()))
    mp.mp_layer_status()


def test_a_stream_that_is_not_the_current_one(mp):
    """results of calls on another stream: dropped at once, they are not handed out again before that stream is done
    with them: a fill on the current stream right after does not reach them, nor they it"""
    c = linear_case("bf16", (2048, 2048, 2048), 3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        for _ in range(20):
            y, pre = mp.mp_linear(c["x"], c["w"], keep_pre=True, stream=stream)
            del y, pre
            z = torch.zeros((2048, 2048), dtype=torch.bfloat16, device="cuda")
            torch.cuda.synchronize()
            assert not z.any()
    want, _ = mp.mp_linear(c["x"], c["w"])
    torch.cuda.synchronize()
    big = torch.empty(1 << 30, dtype=torch.uint8, device="cuda")
    for _ in range(5):  # memory that the current stream still has to write is not a result's
        z = torch.empty((2048, 2048), dtype=torch.bfloat16, device="cuda")
        for _ in range(50):
            big.zero_()
        z.zero_()
        del z
        got, _ = mp.mp_linear(c["x"], c["w"], stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_calls_from_many_threads(mp):
    """threads whose products take different amounts of shared memory, each on a stream of its own"""
    import concurrent.futures as cf

    shapes = [(1, 4096, 512), (24, 1024, 300), (100, 700, 640), (300, 512, 2000), (1200, 256, 4096), (700, 4096, 64)]
    cases = [linear_case("bf16", s, 3 + i) for i, s in enumerate(shapes)]
    want = [mp.mp_linear(c["x"], c["w"])[0] for c in cases]
    x, dy = make((900, 4096), "bf16", 1), make((900, 4096), "bf16", 2)
    _, _, rstd = mp.mp_norm(x)
    norm = mp.mp_norm_backward(dy, x, None, None, rstd)[0]
    torch.cuda.synchronize()

    def work(k):
        s = torch.cuda.Stream()
        for i in range(40):
            c, w = cases[(i + k) % len(cases)], want[(i + k) % len(cases)]
            with torch.cuda.stream(s):
                y, _ = mp.mp_linear(c["x"], c["w"])
                n = mp.mp_norm_backward(dy, x, None, None, rstd)[0] if i % 8 == 0 else norm
            s.synchronize()
            if not torch.equal(y, w) or not torch.equal(n, norm):
                return (k, i)
        return None

    with cf.ThreadPoolExecutor(6) as ex:
        assert [r for r in ex.map(work, range(6)) if r] == []
    mp.mp_layer_status()


def test_linear_far_into_large_matrices(mp):
    """rows beyond 2^32 bytes and 2^31 elements: the last rows of a tall bf16 matrix, forward and backward"""
    rows, k, n = (1 << 31) // 64 + 300, 64, 8
    x = torch.empty((rows, k), dtype=torch.bfloat16, device="cuda")
    x.fill_(0.5)
    tail = make((700, k), "bf16", 1)
    x[-700:] = tail
    w = make((n, k), "bf16", 2)
    y, _ = mp.mp_linear(x, w)
    want, _ = mp.mp_linear(tail, w)
    assert torch.equal(y[-700:], want)
    z, _, rstd = mp.mp_norm(x)
    assert torch.equal(z[-700:], mp.mp_norm(tail)[0])
    dx, _, _, _ = mp.mp_linear_backward(y, x, w, need_dw=False)
    assert torch.equal(dx[-700:], mp.mp_linear_backward(want, tail, w, need_dw=False)[0])


# ---- merge coefficients ----------------------------------------------------------------------------


def coef_family(mp, dtype, sizes, block, K, active, seed):
    """a family with gaps between its tensors, experts equal to the base outside their active blocks"""
    rng = np.random.default_rng(seed)
    es = 2 if dtype == "bf16" else 4
    offs, at = [], 16
    for s in sizes:
        offs.append(at)
        at = (at + s + 40) // (16 // es) * (16 // es)
    total = at + 64
    base = (rng.standard_normal(total) * 0.02).astype(np.float32)
    experts, mask = [], []
    for i in range(K):
        e = base.copy()
        for o, s in zip(offs, sizes):
            for b in range(0, s, block):
                if rng.random() < active:
                    n = min(block, s - b)
                    e[o + b:o + b + n] += (rng.standard_normal(n) * 10.0 ** rng.uniform(-3, -2)).astype(np.float32)
        experts.append(e)
    T = lambda a: torch.from_numpy(a).to(DT[dtype]).cuda()  # noqa: E731
    b, ex = T(base), [T(e) for e in experts]
    g = T((rng.standard_normal(total) * 1e-2).astype(np.float32))
    fam = mp.family(list(zip(offs, sizes)), b, ex, block, mp.MP_BF16 if dtype == "bf16" else mp.MP_F32, 0)
    return fam, b, ex, g


def coef_reference(fam, b, ex, g, block, mask):
    B, G = f64(b), f64(g)
    want, size = np.zeros((fam.K, len(fam.tensors))), np.zeros((fam.K, len(fam.tensors)))
    for i in range(fam.K):
        X, blk = f64(ex[i]), 0
        for t, (o, s) in enumerate(fam.tensors):
            for a in range(0, s, block):
                n = min(block, s - a)
                if mask[blk] >> i & 1:
                    p = (X[o + a:o + a + n] - B[o + a:o + a + n]) * G[o + a:o + a + n]
                    want[i, t] += p.sum()
                    size[i, t] += np.abs(p).sum()
                blk += 1
    return want, size


@pytest.mark.parametrize("dtype,sizes,block,K,active,budget", [
    ("bf16", [1], 256, 1, 1.0, 1.0), ("bf16", [7, 256, 300, 5000], 256, 3, 0.5, 1.0),
    ("bf16", [70001, 4096, 300, 20000], 4096, 3, 0.5, 0.4), ("bf16", [400000, 31, 16384, 16385], 65536, 8, 0.4, 0.5),
    ("bf16", [200000, 77], 16384, 32, 0.7, 0.6), ("fp32", [9, 8200, 40000], 4096, 5, 0.6, 0.3),
    ("fp32", [3, 131072 + 5], 131072, 17, 1.0, 1.0), ("bf16", [5000, 600], 1024, 4, 0.5, 0.0)])
def test_coef_grad(mp, dtype, sizes, block, K, active, budget):
    """against sums in 64 bits over the plan's blocks: fp32 differences and products of up to 64 + 13 terms per thread
    and tree, then fp64, then one rounding: 80 2^-24 of the sum of magnitudes.  Blocks that the plan leaves
    out are not read: NaN in them changes nothing"""
    fam, b, ex, g = coef_family(mp, dtype, sizes, block, K, active, 5)
    op = mp.make_op(mp.MP_OP_TA, alpha=[0.3] * K)
    idx = mp.mp_index_blocks(fam, op)
    plan = mp.mp_plan(idx, op, mp.mp_budget_from_fraction(fam, budget))
    mask = mp.mp_plan_info(plan, idx)["mask"]
    want, size = coef_reference(fam, b, ex, g, block, mask)
    got = mp.mp_coef_grad(fam, idx, plan, g)
    assert np.all(np.abs(f64(got) - want) <= 2 * (80 * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want)))
    blk = 0
    for o, s in fam.tensors:
        for a in range(0, s, block):
            n = min(block, s - a)
            for i in range(K):
                if not mask[blk] >> i & 1:
                    ex[i][o + a:o + a + n] = float("nan")
            if not mask[blk]:
                b[o + a:o + a + n] = float("nan")
                g[o + a:o + a + n] = float("nan")
            blk += 1
    end = fam.tensors[-1][0] + fam.tensors[-1][1]
    g[end:], g[:fam.tensors[0][0]] = float("nan"), float("nan")
    out = torch.full_like(got, float("nan"))
    assert mp.mp_coef_grad(fam, idx, plan, g, out=out) is out and torch.equal(out, got)


def test_coef_grad_against_differences(mp):
    """the slope of L(alpha) = sum(merged * g) in each alpha, from two merges in fp32: linear in alpha, so that only
    roundings count (2^-24 of weights of 0.1, their products with g summed, over a step of 0.5)"""
    fam, b, ex, g = coef_family(mp, "fp32", [3000, 5000], 1024, 3, 0.7, 8)

    def merged(alpha):
        op = mp.make_op(mp.MP_OP_TA, alpha=alpha)
        idx = mp.mp_index_blocks(fam, op)
        plan = mp.mp_plan(idx, op, mp.mp_budget_from_fraction(fam, 1.0))
        out = b.clone()
        mp.mp_merge(fam, idx, plan, out)
        return idx, plan, out

    idx, plan, _ = merged([0.3, 0.2, 0.1])
    got = f64(mp.mp_coef_grad(fam, idx, plan, g)).sum(1)
    for i in range(3):
        up, down = [0.3, 0.2, 0.1], [0.3, 0.2, 0.1]
        up[i] += 0.5
        down[i] -= 0.5
        slope = ((f64(merged(up)[2]) - f64(merged(down)[2])) * f64(g)).sum()
        assert abs(slope - got[i]) < 8000 * 2.0 ** -24 * 0.1 * 1e-2 * 8


def test_coef_grad_in_a_graph_and_after_the_handles_are_freed(mp):
    fam, b, ex, g = coef_family(mp, "bf16", [300000, 5000], 4096, 4, 0.6, 9)
    op = mp.make_op(mp.MP_OP_AVG, alpha=[0.25] * 4)
    idx = mp.mp_index_blocks(fam, op)
    plan = mp.mp_plan(idx, op, mp.mp_budget_from_fraction(fam, 0.7))
    want = mp.mp_coef_grad(fam, idx, plan, g).clone()
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mp.mp_coef_grad(fam, idx, plan, g, out=out)
    g *= 2
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, 2 * want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = mp.mp_coef_grad(fam, idx, plan, g)
    plan.free()
    idx.free()
    torch.cuda.synchronize()
    assert torch.equal(out, 2 * want)


# ---- refusals and failures ---------------------------------------------------------------------------


def test_refusals(mp):
    x, w = make((4, 16), "bf16", 1), make((8, 16), "bf16", 2)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        mp.mp_linear(x.half(), w.half())
    with pytest.raises(ValueError, match="w must be"):
        mp.mp_linear(x, w.float())
    with pytest.raises(ValueError, match="contiguous"):
        mp.mp_linear(x.t(), make((8, 4), "bf16", 2))
    with pytest.raises(ValueError, match="mul must be"):
        mp.mp_linear(x, w, mul=x)
    with pytest.raises(ValueError, match="GPU"):
        mp.mp_linear(x, w.cpu())
    with pytest.raises(ValueError, match="bias must be"):
        mp.mp_linear(x, w, bias=w[:, 0])
    with pytest.raises(ValueError, match="two dimensions"):
        mp.mp_norm(x[0])

    def refused(text, f, *a, **k):
        with pytest.raises(mp.MergePipeError, match=text) as e:
            f(*a, **k)
        assert e.value.status == -1

    refused("overlaps x", mp.mp_linear, x, w, out=x[:, :8])
    refused("overlaps w", mp.mp_linear, x, w, out=w[:4, :8])
    big = x.new_zeros(64)
    refused("overlaps residual", mp.mp_linear, x, w, residual=big[8:40].view(4, 8), out=big[:32].view(4, 8))
    refused("row stride", mp.mp_linear, x[:1].expand(4, 16), w)
    refused("unknown activation", mp.mp_linear, x, w, act=9)
    refused("unknown norm kind", mp.mp_norm, x, kind=5)
    refused("no bias", mp.mp_norm, x, bias=x[0])
    refused("eps", mp.mp_norm, x, eps=-1.0)
    refused("eps", mp.mp_norm, x, eps=float("nan"))
    _, _, rstd = mp.mp_norm(x)
    refused("mean is NULL", mp.mp_norm_backward, x, x, None, None, rstd, kind=mp.MP_NORM_LAYER)
    refused("overlaps x", mp.mp_norm_backward, x.clone(), x, None, None, rstd, dx=x)
    refused("pre is needed", mp.mp_linear_backward, make((4, 8), "bf16", 3), x, w, act=mp.MP_ACT_SILU)
    refused("overlaps dx", mp.mp_linear_backward, make((4, 8), "bf16", 3), x, w, dx=(v := x.new_zeros(512)).as_strided((4, 16), (16, 1)),
            dw=v.as_strided((8, 16), (16, 1)))
    with pytest.raises(mp.MergePipeError, match="args is NULL"):
        mp._check(mp.lib().mp_norm(None, None))


def test_coef_refusals(mp):
    fam, b, ex, g = coef_family(mp, "bf16", [3000, 600], 1024, 2, 1.0, 3)

    def handles(op):
        idx = mp.mp_index_blocks(fam, op)
        return idx, mp.mp_plan(idx, op, mp.mp_budget_from_fraction(fam, 1.0))

    ta = handles(mp.make_op(mp.MP_OP_TA, alpha=[0.5, 0.5]))
    other = handles(mp.make_op(mp.MP_OP_TA, alpha=[0.5, 0.4]))
    for op in (mp.make_op(mp.MP_OP_TIES), mp.make_op(mp.MP_OP_DARE, alpha=[0.5, 0.5], drop_p=0.5),
               mp.make_op(mp.MP_OP_AVG_RENORM, alpha=[0.5, 0.5])):
        with pytest.raises(mp.MergePipeError, match="AVG or TA") as e:
            mp.mp_coef_grad(fam, *handles(op), g)
        assert e.value.status == -7
    with pytest.raises(mp.MergePipeError, match="different index") as e:
        mp.mp_coef_grad(fam, ta[0], other[1], g)
    assert e.value.status == -8
    with pytest.raises(ValueError, match="spans"):
        mp.mp_coef_grad(fam, *ta, g[:1000])
    with pytest.raises(ValueError, match="spans"):
        mp.mp_coef_grad(fam, *ta, g.float())
    with pytest.raises(mp.MergePipeError, match="16-byte aligned"):
        mp.mp_coef_grad(fam, *ta, torch.cat([g, g])[1:])
    with pytest.raises(mp.MergePipeError, match="overlaps"):
        mp.mp_coef_grad(fam, *ta, g, out=g[:8].view(torch.float32).view(2, 2))
    host = mp.family(fam.tensors, b, [e.cpu().pin_memory() for e in ex], 1024)
    idx = mp.mp_index_blocks(host, mp.make_op(mp.MP_OP_TA, alpha=[0.5, 0.5]))
    plan = mp.mp_plan(idx, mp.make_op(mp.MP_OP_TA, alpha=[0.5, 0.5]), 1 << 20)
    with pytest.raises(mp.MergePipeError, match="device memory") as e:
        mp.mp_coef_grad(host, idx, plan, g)
    assert e.value.status == -7


def test_failed_scratch_and_calls_after_it(mp):
    """the n-th allocation of a call fails: MP_ERR_OOM, nothing left behind, the next call is right"""
    c = linear_case("bf16", (5, 33, 17), 3)
    dy = make((5, 17), "bf16", 4)
    want = mp.mp_linear_backward(dy, c["x"], c["w"], bias=True)
    n = 0
    for n in range(1, 10):
        mp.mp_debug_inject_fault(mp.MP_FAULT_ALLOC, n)
        try:
            mp.mp_linear_backward(dy, c["x"], c["w"], bias=True)
        except mp.MergePipeError as e:
            assert e.status == -3 and "injected" in str(e)
            continue
        break
    mp.mp_debug_inject_fault(mp.MP_FAULT_ALLOC, 0)
    assert n >= 2
    got = mp.mp_linear_backward(dy, c["x"], c["w"], bias=True)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
    mp.mp_layer_status()


@pytest.mark.parametrize("rows", [4, 2048])
def test_a_wait_that_runs_out_is_reported(mp, rows):
    """the first stage of each CTA is never filled (test hook): the kernels give up, mp_layer_status says so once, and
    the next call is right"""
    c = linear_case("bf16", (rows, 512, 2048), 3)
    want, _ = mp.mp_linear(c["x"], c["w"])
    mp.mp_layer_status()
    mp.mp_debug_stall_pipeline(2000)
    try:
        mp.mp_linear(c["x"], c["w"])
        torch.cuda.synchronize()
    finally:
        mp.mp_debug_stall_pipeline(0)
    with pytest.raises(mp.MergePipeError) as e:
        mp.mp_layer_status()
    assert e.value.status == -6
    mp.mp_layer_status()
    assert torch.equal(mp.mp_linear(c["x"], c["w"])[0], want)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_a_norm_whose_ring_is_not_filled_is_reported(mp, kind):
    x, dy, w = make((900, 4096), "bf16", 1), make((900, 4096), "bf16", 2), make((4096,), "bf16", 3)
    k = mp.MP_NORM_LAYER if kind == "layer" else mp.MP_NORM_RMS
    _, mean, rstd = mp.mp_norm(x, w, kind=k)
    want = mp.mp_norm_backward(dy, x, w, mean, rstd, kind=k)
    mp.mp_layer_status()
    mp.mp_debug_stall_pipeline(2000)
    try:
        mp.mp_norm_backward(dy, x, w, mean, rstd, kind=k)
        torch.cuda.synchronize()
    finally:
        mp.mp_debug_stall_pipeline(0)
    with pytest.raises(mp.MergePipeError) as e:
        mp.mp_layer_status()
    assert e.value.status == -6
    got = mp.mp_norm_backward(dy, x, w, mean, rstd, kind=k)
    mp.mp_layer_status()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_trace_ranges(mp):
    c = linear_case("bf16", (8, 64, 64), 3)
    mp.mp_trace_start(16)
    y, _ = mp.mp_linear(c["x"], c["w"])
    _, _, rstd = mp.mp_norm(y)
    kinds = [r["kind"] for r in mp.mp_trace_stop()]
    assert kinds == [mp.MP_TRACE_LINEAR, mp.MP_TRACE_NORM]


def test_checked_build_of_the_coefficients_gradient():
    """blocks of many items, ragged ends and omitted blocks through the checked library: no check fails, the same result"""
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = ("import sys; sys.path.insert(0, 'tests'); import torch, test_gpu_layer_ops as t, paper_2605_29489_gb300 as mp\n"
            "fam, b, ex, g = t.coef_family(mp, 'bf16', [400000, 31, 16384, 16385], 65536, 8, 0.4, 5)\n"
            "op = mp.make_op(mp.MP_OP_TA, alpha=[0.3] * 8)\n"
            "idx = mp.mp_index_blocks(fam, op)\n"
            "plan = mp.mp_plan(idx, op, mp.mp_budget_from_fraction(fam, 0.5))\n"
            "out = mp.mp_coef_grad(fam, idx, plan, g)\n"
            "mp.mp_layer_status()\n"
            "print(mp.mp_version(), [v.hex() for v in out.flatten().tolist()])\n")
    got = []
    for checked in ("0", "1"):
        r = subprocess.run([sys.executable, "-c", code], cwd=root, env=dict(os.environ, MERGEPIPE_CHECKED=checked),
                           capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stdout + r.stderr
        got.append(r.stdout)
    assert "checked" in got[1] and got[0].split("[")[1] == got[1].split("[")[1]
