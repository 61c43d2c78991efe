"""The operators of a worker's local step on the GPU, against the definitions in 64 bits and against differences."""
import math

import pytest
import torch

import _train_ref as R
from _train_ref import EPS, TYPES, close, empty, gen, matrix, untouched

pytestmark = pytest.mark.gpu
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]


@pytest.fixture(scope="module")
def P():
    import paper_1709_09393_b200 as pkg
    assert torch.cuda.is_available()
    return pkg


def ws_of(size):
    return torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------ layer norm

LN_SHAPES = [(1, 1), (3, 2), (2, 31), (5, 33), (9, 256), (17, 257), (40, 1000), (300, 1003), (33, 1024), (6, 1032),
             (3, 2048), (700, 2049), (5, 4096), (4, 4104), (650, 8192), (3, 8200), (2, 16384), (3, 16385), (35, 20000)]


def ln_forward(P, x, gamma, beta, eps, pad=0, offset=0):
    rows, dim = x.shape
    y, flat = empty(rows, dim, x.dtype, pad, offset)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    P.slimdp_layernorm_forward(x, gamma, beta, eps, y, mean, rstd)
    assert untouched(y, flat)
    return y, mean, rstd


def ln_check(x, gamma, beta, eps, y, mean, rstd):
    ref, rmean, rrstd, h = R.layernorm(x, gamma, beta, eps)
    xd = x.double()
    size = xd.abs().mean(1)
    # a sum over dim in blocks and trees: 64 roundings in the longest chain of additions are more than enough up to
    # 65536 elements (64 a thread at most, then two trees of five levels)
    close(mean, rmean, 80 * EPS * size, "mean")
    dmu = 80 * EPS * size * rrstd                           # the mean's error in units of the deviation
    rel = 100 * EPS + dmu * (dmu + 2 * EPS) + 4 * EPS       # its square and the sum of squares
    close(rstd, rrstd, rel * rrstd, "rstd")
    g = torch.ones_like(ref) if gamma is None else gamma.double().abs().expand_as(ref)
    tol = R.rounding(ref, x.dtype) + g * (dmu[:, None] + (rel[:, None] + 8 * EPS) * h.abs()) + 4 * EPS * ref.abs() \
        + 4 * EPS * (0 if beta is None else beta.double().abs())
    close(y, ref, tol, "y")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", LN_SHAPES)
def test_layernorm_forward(P, dtype, rows, dim):
    g = gen(rows * 7 + dim)
    x = matrix(rows, dim, dtype, g, 2.0) + torch.randn(rows, 1, generator=g, device="cuda").to(dtype)
    flat = torch.randn(2 * dim + 1, generator=g, device="cuda")
    for gamma, beta in [(flat[1:1 + dim], flat[1 + dim:]), (None, flat[:dim]), (None, None)]:
        ln_check(x, gamma, beta, 1e-5, *ln_forward(P, x, gamma, beta, 1e-5))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(8, 0), (0, 8), (3, 0), (0, 1), (5, 3)])
def test_layernorm_forward_rows_of_any_alignment(P, dtype, pad, offset):
    for dim in (24, 1000, 4096):
        g = gen(dim + pad)
        x = matrix(11, dim, dtype, g, 1.0, pad, offset)
        ln_check(x, None, None, 1e-6, *ln_forward(P, x, None, None, 1e-6, pad, offset))
        ln_check(x, None, None, 1e-6, *ln_forward(P, x, None, None, 1e-6))


def test_layernorm_forward_of_hard_rows(P):
    for dim in (64, 1536, 9000, 17000):
        x = torch.zeros(6, dim, device="cuda")
        x[1] = 3.25                                      # no variance: rstd = 1 / sqrt(eps)
        x[2] = torch.randn(dim, generator=gen(1), device="cuda") + 1.0e4   # a mean far above the deviation
        x[3] = torch.randn(dim, generator=gen(2), device="cuda")
        x[3, 0] = 1.0e4                                  # one entry far above the rest
        x[4] = torch.randn(dim, generator=gen(3), device="cuda")
        x[4, dim // 2] = math.nan                        # stays in its row
        x[5] = torch.randn(dim, generator=gen(4), device="cuda") * 1.0e-6
        y, mean, rstd = ln_forward(P, x, None, None, 1e-5)
        keep = [0, 1, 2, 3, 5]
        ln_check(x[keep], None, None, 1e-5, y[keep], mean[keep], rstd[keep])
        assert y[4].isnan().all() and mean[4].isnan() and rstd[4].isnan()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", LN_SHAPES)
def test_layernorm_backward(P, dtype, rows, dim):
    g = gen(rows * 5 + dim)
    pad, offset = (0, 0) if dim % 2 == 0 else (2, 1)
    x, dy = matrix(rows, dim, dtype, g, 1.5, pad, offset), matrix(rows, dim, dtype, g, 0.1)
    gamma = torch.randn(dim, generator=g, device="cuda")
    _, mean, rstd, _ = R.layernorm(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    dx, flat = empty(rows, dim, dtype, pad, 0)
    delta = torch.full((2 * dim + 2,), -77.0, device="cuda")
    dgamma, dbeta = delta[1:1 + dim], delta[1 + dim:1 + 2 * dim]
    ws = ws_of(P.layernorm_workspace_bytes(rows, dim))
    P.slimdp_layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws)
    assert untouched(dx, flat) and delta[0] == -77.0 and delta[-1] == -77.0
    rdx, rdg, rdb, h, gg, r = R.layernorm_grad(dy, x, gamma, mean, rstd)
    # h is off by its own rounding and by that of x - mean; the two averages are sums of dim terms
    dh = 4 * EPS * (h.abs() + r * mean.double().abs()[:, None])
    avg = gg.abs().mean(1, keepdim=True)
    avg_h = (gg.abs() * (h.abs() + 1)).mean(1, keepdim=True)
    tol = R.rounding(rdx, dtype) + r * (8 * EPS * gg.abs() + 80 * EPS * avg + h.abs() * 90 * EPS * avg_h +
                                        dh * avg_h + h.abs() * (gg.abs() * dh).mean(1, keepdim=True))
    close(dx, rdx, tol, "dx")
    d = dy.double().abs()
    tol_g, tol_b = (rows + 8) * EPS * (d * h.abs()).sum(0) + (d * dh).sum(0), (rows + 8) * EPS * d.sum(0)
    close(dgamma, rdg, tol_g, "dgamma")
    close(dbeta, rdb, tol_b, "dbeta")
    once = delta.clone()
    P.slimdp_layernorm_backward(dy, x, gamma, mean, rstd, dx, dgamma, dbeta, ws, accumulate=True)
    close(dgamma, once[1:1 + dim].double() * 2, 2 * EPS * rdg.abs() + tol_g, "dgamma, added")
    assert torch.equal(dbeta, once[1 + dim:1 + 2 * dim] * 2)          # doubling is exact
    only = torch.empty_like(dx)
    P.slimdp_layernorm_backward(dy, x, gamma, mean, rstd, only, None, None, None)
    assert torch.equal(only, dx)
    P.slimdp_layernorm_backward(dy, x, gamma, mean, rstd, dx, None, dbeta, ws)
    assert torch.equal(dbeta, once[1 + dim:1 + 2 * dim])


# rows on 4-byte boundaries only, and rows too long for registers, for the ring or for column sums in shared memory
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,dim", [(5, 34), (333, 1002), (170, 4090), (3, 8198), (2, 16382), (400, 16390), (310, 20008),
                                      (160, 24584), (7, 26001), (330, 30000), (3, 40000), (5, 65536)])
def test_layernorm_of_even_and_of_long_rows(P, dtype, rows, dim):
    test_layernorm_forward(P, dtype, rows, dim)
    test_layernorm_backward(P, dtype, rows, dim)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(2, 0), (0, 2), (6, 4)])
def test_layernorm_forward_rows_on_4_byte_boundaries(P, dtype, pad, offset):
    for dim in (24, 1002, 4096):
        x = matrix(11, dim, dtype, gen(dim + pad + offset), 1.0, pad, offset)
        ln_check(x, None, None, 1e-6, *ln_forward(P, x, None, None, 1e-6, pad, offset))


def test_layernorm_of_no_rows(P):
    x = torch.empty(0, 96, device="cuda")
    stats = torch.empty(0, device="cuda")
    P.slimdp_layernorm_forward(x, None, None, 1e-5, torch.empty_like(x), stats, stats)
    dg, db = torch.full((96,), 5.0, device="cuda"), torch.full((96,), 5.0, device="cuda")
    ws = ws_of(P.layernorm_workspace_bytes(0, 96))
    P.slimdp_layernorm_backward(x, x, None, stats, stats, torch.empty_like(x), dg, db, ws, accumulate=True)
    assert (dg == 5).all() and (db == 5).all()
    P.slimdp_layernorm_backward(x, x, None, stats, stats, torch.empty_like(x), dg, db, ws)
    assert (dg == 0).all() and (db == 0).all()


def test_layernorm_gradient_against_differences(P):
    rows, dim, step = 6, 200, 2.0 ** -7
    g = gen(3)
    x, c = matrix(rows, dim, torch.float32, g), matrix(rows, dim, torch.float32, g)
    gamma, beta = torch.randn(2, dim, generator=g, device="cuda").unbind(0)
    y, mean, rstd = ln_forward(P, x, gamma, beta, 1e-3)
    dx, dg, db = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    P.slimdp_layernorm_backward(c, x, gamma, mean, rstd, dx, dg, db, ws_of(P.layernorm_workspace_bytes(rows, dim)))

    def value(xx, gg, bb):
        return (ln_forward(P, xx, gg, bb, 1e-3)[0].double() * c.double()).sum().item()

    ux, ug, ub = torch.randn_like(x), torch.randn_like(gamma), torch.randn_like(beta)
    for at, u, grad in [(0, ux, dx), (1, ug, dg), (2, ub, db)]:
        v = [x, gamma, beta]
        plus, minus = list(v), list(v)
        plus[at], minus[at] = v[at] + step * u, v[at] - step * u
        diff = (value(*plus) - value(*minus)) / (2 * step)
        along = (grad.double() * u.double()).sum().item()
        # rounding of y, 16 EPS |y| |c| summed at random, over the step; the third derivative, about 4 |u|^3 |c| step^2
        noise = 16 * EPS * (y.double() * c.double()).norm().item() * 4 / step
        third = step ** 2 * 4 * (u.double().abs().pow(3).mean().item()) * c.double().abs().sum().item() / 6
        assert abs(diff - along) <= noise + third


# ------------------------------------------------------------------------------------------ product

LINEAR_SHAPES = [(1, 1, 1), (1, 64, 64), (2, 3, 5), (5, 128, 72), (17, 200, 96), (64, 64, 512), (128, 256, 64),
                 (129, 257, 65), (130, 100, 1000), (200, 513, 136), (257, 136, 2050), (1000, 72, 40), (3, 1500, 1032),
                 (384, 640, 320)]


def linear_operands(m, n, k, dtype, pad, seed):
    g = gen(seed)
    return (matrix(m, k, dtype, g, 1.0, pad), matrix(n, k, dtype, g, 1.0 / math.sqrt(k), pad),
            matrix(m, n, dtype, g, 1.0, pad), matrix(m, k, dtype, g, 1.0, pad), g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", LINEAR_SHAPES)
def test_linear_forward(P, dtype, m, n, k):
    ws = ws_of(P.linear_workspace_bytes(m, n, k, dtype))
    for pad, act in [(0, "none"), (0, "gelu"), (8, "silu"), (3, "gelu_tanh"), (1, "relu")]:
        x, w, res, _, g = linear_operands(m, n, k, dtype, pad, m + n + k + pad)
        bias = torch.randn(n + 1, generator=g, device="cuda")[1:]
        ref_z, tol_z = R.product(x, w)
        for b, r, keep in [(bias, res, True), (None, None, False), (bias, None, True)]:
            y, yflat = empty(m, n, dtype, pad)
            z, zflat = empty(m, n, dtype, pad) if keep else (None, None)
            P.slimdp_linear_forward(x, w, b, y, ws, activation=act, residual=r, z=z)
            assert untouched(y, yflat) and (not keep or untouched(z, zflat))
            rz = ref_z + (0 if b is None else b.double())
            tz = tol_z + 2 * EPS * rz.abs()
            if keep:
                close(z, rz, tz + R.rounding(rz, dtype), "z")
            ry = R.act(rz, act)
            # slopes of the activations are below 1.13; their own evaluation is a few roundings of |z| + |y|
            ty = 1.13 * tz + 16 * EPS * (rz.abs() + ry.abs())
            if r is not None:
                ry = ry + r.double()
                ty = ty + EPS * ry.abs()
            close(y, ry, ty + R.rounding(ry, dtype), f"y, {act}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", LINEAR_SHAPES)
def test_linear_backward_input(P, dtype, m, n, k):
    ws = ws_of(P.linear_workspace_bytes(m, n, k, dtype))
    for pad, act in [(0, "none"), (0, "gelu"), (8, "silu"), (3, "gelu_tanh"), (1, "relu")]:
        z, w, dy, add, _ = linear_operands(m, n, k, dtype, pad, m + n + k + pad)
        ref, tol = R.product(dy, w.t())
        slope = R.act_slope(z.double(), act)
        for a in (None, add):
            dx, flat = empty(m, k, dtype, pad)
            P.slimdp_linear_backward_input(dy, w, dx, ws, activation=act, z=None if act == "none" else z, add=a)
            assert untouched(dx, flat)
            r = ref * slope
            # the slope itself: a few roundings of terms up to |z| + 2
            t = tol * slope.abs() + 16 * EPS * ref.abs() * (2 + z.double().abs()) + EPS * r.abs()
            if a is not None:
                r = r + a.double()
                t = t + EPS * r.abs()
            close(dx, r, t + R.rounding(r, dtype), f"dx, {act}")


# few rows against wide, tall and tiny matrices; long summed axes of few results
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (2, 1, 3000), (1, 5000, 700), (3, 40000, 36), (4, 270, 2052), (5, 33, 1030),
                                   (7, 16, 5000), (8, 4099, 516), (8, 1000, 4096), (9, 2000, 640), (16, 700, 1028),
                                   (17, 5001, 516), (32, 3000, 260), (31, 333, 77), (33, 400, 300), (1, 700, 4098),
                                   (2, 333, 1002), (4, 1000, 94), (5, 600, 1002)])
def test_linear_of_few_rows(P, dtype, m, n, k):
    test_linear_forward(P, dtype, m, n, k)
    test_linear_backward_input(P, dtype, m, n, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(40, 130, 20000), (130, 20000, 70), (20000, 70, 130)])
def test_linear_of_long_sums_and_few_results(P, dtype, m, n, k):
    test_linear_forward(P, dtype, m, n, k)
    test_linear_backward_input(P, dtype, m, n, k)
    test_linear_backward_weight(P, dtype, m, n, k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", LINEAR_SHAPES)
def test_linear_backward_weight(P, dtype, m, n, k):
    ws = ws_of(P.linear_workspace_bytes(m, n, k, dtype))
    for pad in (0, 8, 3):
        x, _, dy, _, _ = linear_operands(m, n, k, dtype, pad, m + n + k + pad)
        delta = torch.full((n * k + n + 2,), -77.0, device="cuda")
        dw, db = delta[1:1 + n * k].view(n, k), delta[1 + n * k:1 + n * k + n]
        P.slimdp_linear_backward_weight(dy, x, dw, db, ws)
        assert delta[0] == -77.0 and delta[-1] == -77.0
        ref, tol = R.product(dy.t(), x.t())
        close(dw, ref, tol, "dw")
        rb, tb = dy.double().sum(0), (m + 8) * EPS * dy.double().abs().sum(0)
        close(db, rb, tb, "db")
        first = delta.clone()
        P.slimdp_linear_backward_weight(dy, x, dw, db, ws, accumulate=True)
        assert torch.equal(delta[1:-1], first[1:-1] * 2)               # the same sums again, and doubling is exact
        wide, flat = empty(n, k, torch.float32, 5, 1)
        P.slimdp_linear_backward_weight(dy, x, wide, None, ws)
        assert torch.equal(wide, first[1:1 + n * k].view(n, k)) and untouched(wide, flat)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_sums_stay_in_32_bits_over_a_long_axis(P, dtype):
    """A sum of 20000 products of one sign: 16-bit partial sums, or an accumulator that drops low bits, would show."""
    m, n, k = 24, 40, 20000
    g = gen(11)
    x, w = matrix(m, k, dtype, g).abs(), matrix(n, k, dtype, g).abs()
    y = torch.empty(m, n, device="cuda", dtype=dtype)
    P.slimdp_linear_forward(x, w, None, y, ws_of(P.linear_workspace_bytes(m, n, k, dtype)))
    ref, _ = R.product(x, w)
    # at most k / 16 truncations of 2^-23 in a row for 16-bit types, six times as many for fp32's parts
    chain = (6 if dtype == torch.float32 else 1) * (k / 16) * 2 * EPS
    close(y, ref, chain * ref + R.rounding(ref, dtype))
    dw = torch.empty(m, n, device="cuda")
    P.slimdp_linear_backward_weight(x.t().contiguous(), w.t().contiguous(), dw, None, ws_of(P.linear_workspace_bytes(k, m, n, dtype)))
    close(dw, ref, chain * ref + EPS * ref)


def test_linear_fp32_parts_keep_24_bits(P):
    """Operands whose low bits decide the result: (1 + 2^-20) - 1 and the like survive the split into parts."""
    m, n, k = 48, 80, 64
    g = gen(5)
    x = matrix(m, k, torch.float32, g)
    w = torch.zeros(n, k, device="cuda")
    w[:, 0] = 1.0
    x[:, 0] = 1.0 + torch.arange(m, device="cuda") * 2.0 ** -23
    y = torch.empty(m, n, device="cuda")
    P.slimdp_linear_forward(x, w, None, y, ws_of(P.linear_workspace_bytes(m, n, k, torch.float32)))
    assert torch.equal(y, x[:, :1].expand(m, n))               # one product with 1: exact
    for scale in (2.0 ** 100, 2.0 ** -100, 2.0 ** 60):
        a, b = matrix(m, k, torch.float32, g) * scale, matrix(n, k, torch.float32, g) * (1 / scale)
        P.slimdp_linear_forward(a, b, None, y, ws_of(P.linear_workspace_bytes(m, n, k, torch.float32)))
        ref, tol = R.product(a, b)
        close(y, ref, tol + EPS * ref.abs())


def test_linear_non_finite_values_stay_in_their_rows(P):
    for dtype in TYPES:
        m, n, k = 140, 96, 80
        g = gen(8)
        x, w = matrix(m, k, dtype, g), matrix(n, k, dtype, g, 0.1)
        x[3, 7], x[131, 2] = math.nan, math.inf
        y = torch.empty(m, n, device="cuda", dtype=dtype)
        P.slimdp_linear_forward(x, w, None, y, ws_of(P.linear_workspace_bytes(m, n, k, dtype)))
        assert y[3].isnan().all() and not y[131].isfinite().any()
        keep = [i for i in range(m) if i not in (3, 131)]
        ref, tol = R.product(x[keep], w)
        close(y[keep], ref, tol + R.rounding(ref, dtype))


def test_linear_of_no_rows(P):
    for dtype in TYPES:
        x, w = torch.empty(0, 24, device="cuda", dtype=dtype), torch.ones(40, 24, device="cuda", dtype=dtype)
        dy = torch.empty(0, 40, device="cuda", dtype=dtype)
        ws = ws_of(P.linear_workspace_bytes(0, 40, 24, dtype))
        P.slimdp_linear_forward(x, w, None, torch.empty_like(dy), ws)
        P.slimdp_linear_backward_input(dy, w, torch.empty_like(x), ws)
        dw, db = torch.full((40, 24), 3.0, device="cuda"), torch.full((40,), 3.0, device="cuda")
        P.slimdp_linear_backward_weight(dy, x, dw, db, ws, accumulate=True)
        assert (dw == 3).all() and (db == 3).all()
        P.slimdp_linear_backward_weight(dy, x, dw, db, ws)
        assert (dw == 0).all() and (db == 0).all()


def test_linear_results_do_not_depend_on_the_stream_or_the_run(P):
    m, n, k = 300, 500, 700
    for dtype in TYPES:
        x, w, dy, _, _ = linear_operands(m, n, k, dtype, 0, 3)
        ws = ws_of(P.linear_workspace_bytes(m, n, k, dtype))
        first = torch.empty(m, n, device="cuda", dtype=dtype)
        dw = torch.empty(n, k, device="cuda")
        P.slimdp_linear_forward(x, w, None, first, ws)
        P.slimdp_linear_backward_weight(dy, x, dw, None, ws)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        again, dw2 = torch.empty_like(first), torch.empty_like(dw)
        P.slimdp_linear_forward(x, w, None, again, ws, stream=side)
        P.slimdp_linear_backward_weight(dy, x, dw2, None, ws, stream=side)
        side.synchronize()
        assert torch.equal(first, again) and torch.equal(dw, dw2)


def test_linear_gradients_against_differences(P):
    m, n, k, step = 20, 24, 40, 2.0 ** -6
    f = torch.float32
    for act in ("gelu", "gelu_tanh", "silu"):
        z0, w, c, _, g = linear_operands(m, n, k, f, 0, 17)
        ws = ws_of(P.linear_workspace_bytes(m, n, k, f))
        bias = torch.randn(n, generator=g, device="cuda")

        def value(z0, w, bias):
            y = torch.empty(m, n, device="cuda")
            P.slimdp_linear_forward(R.act(z0.double(), act).float(), w, bias, y, ws)
            return (y.double() * c.double()).sum().item()

        dz, dw, db = torch.empty_like(z0), torch.empty_like(w), torch.empty_like(bias)
        P.slimdp_linear_backward_input(c, w, dz, ws, activation=act, z=z0)
        P.slimdp_linear_backward_weight(c, R.act(z0.double(), act).float(), dw, db, ws)
        scale = c.double().abs().sum().item()
        for at, grad in [(0, dz), (1, dw), (2, db)]:
            v = [z0, w, bias]
            u = torch.randn(v[at].shape, generator=g, device="cuda")
            plus, minus = list(v), list(v)
            plus[at], minus[at] = v[at] + step * u, v[at] - step * u
            diff = (value(*plus) - value(*minus)) / (2 * step)
            along = (grad.double() * u.double()).sum().item()
            # rounding of the sums over the step, and (for z0) a third derivative of at most 2 per unit
            assert abs(diff - along) <= 64 * EPS * scale * 4 / step + step ** 2 * scale


@pytest.mark.parametrize("dtype", TYPES)
def test_activation_backward(P, dtype):
    for m, n, pad in [(1, 1, 0), (3, 257, 2), (70, 1000, 8), (9, 20000, 0)]:
        g = gen(m + n)
        dy, z = matrix(m, n, dtype, g, 0.5, pad), matrix(m, n, dtype, g, 2.0, pad)
        for act in ACTS:
            dz, flat = empty(m, n, dtype, pad)
            P.slimdp_activation_backward(dy, z, dz, act)
            assert untouched(dz, flat)
            ref = dy.double() * R.act_slope(z.double(), act)
            close(dz, ref, R.rounding(ref, dtype) + 16 * EPS * dy.double().abs() * (2 + z.double().abs()), act)


@pytest.mark.parametrize("dtype", TYPES)
def test_activation_backward_in_place_and_without_z(P, dtype):
    for m, n, pad in [(5, 3, 0), (131, 264, 8), (40, 1000, 1)]:
        g = gen(m + 2 * n)
        dy, z = matrix(m, n, dtype, g, 0.5, pad), matrix(m, n, dtype, g, 2.0, pad)
        dz, _ = empty(m, n, dtype, pad)
        P.slimdp_activation_backward(dy, z, dz, "gelu")
        over = dy.clone()
        P.slimdp_activation_backward(over, z, over, "gelu")
        assert torch.equal(over, dz)
        P.slimdp_activation_backward(dy, z, dz, "none")
        assert torch.equal(dz, dy)


def test_activation_backward_of_more_rows_than_a_grid_covers(P):
    m, n = 8 * 65535 + 1003, 131
    g = gen(5)
    dy, z = matrix(m, n, torch.bfloat16, g), matrix(m, n, torch.bfloat16, g)
    dz = torch.full_like(dy, -77.0)
    P.slimdp_activation_backward(dy, z, dz, "relu")
    assert torch.equal(dz, torch.where(z > 0, dy, torch.zeros_like(dy)))


# ------------------------------------------------------------------------------------------ distillation

def distill(P, logits, idx, teacher, label=None, weight=None, T=1.0, kd=1.0, ce=0.0, pad=0, offset=0):
    rows, vocab = logits.shape
    loss = torch.full((rows,), -77.0, device="cuda")
    d, flat = empty(rows, vocab, logits.dtype, pad, offset)
    P.slimdp_distill(logits, idx, teacher, loss, d, label=label, row_weight=weight, temperature=T, kd_weight=kd,
                     ce_weight=ce)
    assert untouched(d, flat)
    alone = torch.full((rows,), -77.0, device="cuda")
    P.slimdp_distill(logits, idx, teacher, alone, None, label=label, row_weight=weight, temperature=T, kd_weight=kd,
                     ce_weight=ce)
    assert torch.equal(loss.isnan(), alone.isnan()) and torch.equal(loss.nan_to_num(), alone.nan_to_num())
    return loss, d


def distill_check(P, logits, idx, teacher, label=None, weight=None, T=1.0, kd=1.0, ce=0.0, pad=0, offset=0):
    loss, d = distill(P, logits, idx, teacher, label, weight, T, kd, ce, pad, offset)
    rl, tl, rd, td = R.distill(logits, idx, teacher, label, weight, T, kd, ce)
    close(loss, rl, tl + R.rounding(rl, torch.float32), "loss")
    close(d, rd, td + R.rounding(rd, logits.dtype), "dlogits")


def distill_inputs(rows, vocab, top, dtype, seed, pad=0, offset=0):
    g = gen(seed)
    logits = matrix(rows, vocab, dtype, g, 3.0, pad, offset)
    idx = torch.rand(rows, vocab, generator=g, device="cuda").argsort(1)[:, :top].to(torch.int32).contiguous()
    teacher = torch.randn(rows, top, generator=g, device="cuda") * 2
    label = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    weight = torch.rand(rows, generator=g, device="cuda")
    return logits, idx, teacher, label, weight


DISTILL_SHAPES = [(1, 1, 1), (3, 2, 2), (4, 7, 3), (2, 9, 9), (5, 100, 1), (9, 1000, 5), (4, 1003, 64), (6, 4099, 37),
                  (3, 32000, 128), (2, 50021, 700), (2, 131072, 64), (3, 140001, 16), (2, 300000, 8), (300, 500, 20)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,top", DISTILL_SHAPES)
def test_distill(P, dtype, rows, vocab, top):
    logits, idx, teacher, label, weight = distill_inputs(rows, vocab, top, dtype, rows + vocab)
    distill_check(P, logits, idx, teacher)
    distill_check(P, logits, idx, teacher, label, weight, 2.0, 0.7, 0.3)
    distill_check(P, logits, None, None, label, weight, 1.0, 1.0, 0.5)
    distill_check(P, logits, idx, teacher, label, None, 0.5, 0.0, 1.0)
    distill_check(P, logits, idx, teacher.to(torch.bfloat16), None, weight, 3.5, 1.0, 0.0)
    distill_check(P, logits, idx, teacher.to(torch.float16), label, weight, 1.0, 0.5, 0.5)


@pytest.mark.parametrize("rows,vocab,top,dtype", [(6000, 500, 6, torch.float32), (5000, 3001, 33, torch.bfloat16),
                                                  (3000, 4000, 12, torch.float32), (2500, 9000, 40, torch.bfloat16),
                                                  (700, 30001, 64, torch.float16), (260, 131072, 64, torch.bfloat16),
                                                  (150, 131072, 300, torch.float32), (90, 200000, 64, torch.bfloat16)])
def test_distill_of_many_more_rows_than_run_at_once(P, rows, vocab, top, dtype):
    """Rows follow one another through the same buffers; some have no term, so that neighbours are of different lengths."""
    g = gen(rows)
    logits = matrix(rows, vocab, dtype, g, 3.0)
    idx = torch.randint(0, vocab, (rows, top), generator=g, device="cuda").to(torch.int32)
    idx[::7] = -1
    teacher = torch.randn(rows, top, generator=g, device="cuda") * 2
    label = torch.randint(0, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    weight = torch.rand(rows, generator=g, device="cuda")
    weight[::5] = 0
    distill_check(P, logits, idx, teacher, None, weight, 2.0, 1.0, 0.0)
    distill_check(P, logits, idx, teacher, label, weight, 2.0, 0.5, 0.5)
    distill_check(P, logits, idx, teacher, label, weight, 3.0, 0.5, 0.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(8, 0), (0, 8), (3, 0), (0, 1), (5, 3)])
def test_distill_rows_of_any_alignment(P, dtype, pad, offset):
    for vocab in (5, 1000, 40009):
        a = distill_inputs(5, vocab, 4, dtype, vocab + pad, pad, offset)
        distill_check(P, *a, T=2.0, kd=0.5, ce=0.5, pad=pad, offset=offset)
        distill_check(P, *a, T=2.0, kd=0.5, ce=0.5)
        same = a[0]
        loss, d = distill(P, same, a[1], a[2], a[3], a[4], 2.0, 0.5, 0.5)
        inplace = torch.empty(5, device="cuda")
        P.slimdp_distill(same, a[1], a[2], inplace, same, label=a[3], row_weight=a[4], temperature=2.0, kd_weight=0.5,
                         ce_weight=0.5)
        assert torch.equal(inplace, loss) and torch.equal(same, d)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [40, 3001, 70000])
def test_distill_of_hard_rows(P, dtype, vocab):
    logits, idx, teacher, label, weight = distill_inputs(16, vocab, 6, dtype, vocab)
    low = torch.finfo(dtype).min
    idx[0] = -1                                  # no entry
    idx[1, 2:] = vocab + 5                       # entries outside the vocabulary
    idx[2] = torch.tensor([9, 3, 9, 9, 3, 1], dtype=torch.int32, device="cuda")   # entries that repeat an index
    label[2] = 9
    teacher[3] = -math.inf                       # a teacher with nothing to say
    teacher[4, 1:] = -math.inf                   # one that is certain
    logits[5] = -math.inf                        # nothing but masked logits
    logits[6] = low                              # masked by the type's lowest value
    logits[7, 1:] = -math.inf                    # one logit left
    idx[7] = torch.tensor([0, -1, -1, -1, -1, -1], dtype=torch.int32, device="cuda")
    label[7] = 0
    logits[8, ::2] = low
    label[9], label[10] = -100, vocab            # no label
    weight[11] = 0.0                             # a padded position ...
    logits[11, 0] = math.nan                     # ... whose content does not matter
    idx[12], label[12] = -1, -1                  # neither
    logits[13, idx[13, 0].long()] = -math.inf    # the teacher names what the student excludes: an infinite loss
    teacher[14, 0] = 60.0
    logits[15] *= 20
    for T, kd, ce in [(1.0, 1.0, 0.0), (2.0, 0.5, 0.5), (0.25, 1.0, 0.1), (1.0, 0.0, 1.0)]:
        distill_check(P, logits, idx, teacher, label, weight, T, kd, ce)
    loss, d = distill(P, logits, idx, teacher, label, weight, 2.0, 0.5, 0.5)
    for r in (5, 11, 12):
        assert loss[r] == 0 and (d[r] == 0).all()
    assert loss[13] == math.inf and d[13].isfinite().all()
    logits[1, 3], logits[2, 3], teacher[8, 0] = math.nan, math.inf, math.nan
    loss2, d2 = distill(P, logits, idx, teacher, label, weight, 2.0, 0.5, 0.5)
    for r in (1, 2, 8):
        assert loss2[r].isnan() and d2[r].isnan().any()
    keep = [0, 3, 4, 6, 7, 9, 10, 14, 15]
    assert torch.equal(loss2[keep], loss[keep]) and torch.equal(d2[keep], d[keep])


def test_distill_without_rows_or_entries(P):
    z = torch.empty(0, 10, device="cuda")
    P.slimdp_distill(z, None, None, torch.empty(0, device="cuda"), torch.empty_like(z))
    logits = matrix(4, 10, torch.float32, gen(1))
    none = torch.empty(4, 0, device="cuda")
    loss, d = distill(P, logits, none.to(torch.int32), none)
    assert (loss == 0).all() and (d == 0).all()


def test_distill_gradient_against_differences(P):
    rows, vocab, step = 5, 60, 2.0 ** -6
    logits, idx, teacher, label, weight = distill_inputs(rows, vocab, 7, torch.float32, 23)
    kw = dict(label=label, weight=weight, T=2.0, kd=0.8, ce=0.4)
    _, d = distill(P, logits, idx, teacher, **kw)
    u = torch.randn(rows, vocab, generator=gen(2), device="cuda")
    plus, minus = (distill(P, logits + s * step * u, idx, teacher, **kw)[0].double() for s in (1, -1))
    diff = (plus - minus) / (2 * step)
    along = (d.double() * u.double()).sum(1)
    # the loss is a sum of terms below 40 with a few roundings each; its third derivative along u is below |u|^3
    close(diff, along, 32 * EPS * 40 / step + step ** 2 * u.double().abs().amax(1) ** 3)


# ------------------------------------------------------------------------------------------ all of them

def test_offsets_beyond_32_bits(P):
    """Matrices of more than 2^32 elements: the last rows are where an offset of 32 bits would land elsewhere."""
    g = gen(77)
    vocab = 131072
    rows = (1 << 32) // vocab + 40
    logits = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)
    last = matrix(24, vocab, torch.bfloat16, g, 3.0)
    logits[-24:] = last
    idx = torch.randint(0, vocab, (rows, 5), generator=g, device="cuda").to(torch.int32)
    teacher = torch.randn(rows, 5, generator=g, device="cuda")
    loss = torch.empty(rows, device="cuda")
    P.slimdp_distill(logits, idx, teacher, loss, logits, temperature=2.0)
    rl, tl, rd, td = R.distill(last, idx[-24:], teacher[-24:], None, None, 2.0, 1.0, 0.0)
    close(loss[-24:], rl, tl + R.rounding(rl, torch.float32), "loss")
    close(logits[-24:], rd, td + R.rounding(rd, torch.bfloat16), "dlogits")
    del logits
    dim = 4096
    rows = (1 << 32) // dim + 100
    x = torch.zeros(rows, dim, device="cuda", dtype=torch.bfloat16)
    x[-50:] = matrix(50, dim, torch.bfloat16, g)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    P.slimdp_layernorm_forward(x, None, None, 1e-5, y, mean, rstd)
    ln_check(x[-50:], None, None, 1e-5, y[-50:], mean[-50:], rstd[-50:])
    dgamma, dbeta = torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    dy = y.zero_()                                  # only the last rows have a gradient
    dy[-50:] = matrix(50, dim, torch.bfloat16, g, 0.1)
    dx = torch.empty_like(x)
    P.slimdp_layernorm_backward(dy, x, None, mean, rstd, dx, dgamma, dbeta, ws_of(P.layernorm_workspace_bytes(rows, dim)))
    rdx, rdg, rdb, _, gg, r = R.layernorm_grad(dy[-50:], x[-50:], None, mean[-50:], rstd[-50:])
    assert ((dx[-50:].double() - rdx).norm() / rdx.norm()).item() < 2.0 ** -8
    assert ((dgamma.double() - rdg).norm() / rdg.norm()).item() < 1e-5
    assert ((dbeta.double() - rdb).norm() / rdb.norm()).item() < 1e-5
    del dx, dy, y
    w = matrix(72, dim, torch.bfloat16, g)
    out = torch.empty(rows, 72, device="cuda", dtype=torch.bfloat16)
    P.slimdp_linear_forward(x, w, None, out, ws_of(P.linear_workspace_bytes(rows, 72, dim, torch.bfloat16)))
    ref, tol = R.product(x[-50:], w)
    close(out[-50:], ref, tol + R.rounding(ref, torch.bfloat16))


def test_calls_can_be_captured_in_a_graph(P):
    """Every call is work on its stream alone: a captured step replays with what its buffers hold then."""
    m, n, k, vocab = 300, 200, 136, 9000
    g = gen(9)
    x, w, dy, _, _ = linear_operands(m, n, k, torch.bfloat16, 3, 4)              # padded rows: packed first
    ws = ws_of(P.linear_workspace_bytes(m, n, k, torch.bfloat16) + P.layernorm_workspace_bytes(m, k))
    logits, idx, teacher, label, weight = distill_inputs(60, vocab, 20, torch.bfloat16, 5)
    y, dx, dw, db = torch.empty_like(dy), torch.empty_like(x), torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    h, dh = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(m, device="cuda"), torch.empty(m, device="cuda")
    dg, dbeta = torch.empty(k, device="cuda"), torch.empty(k, device="cuda")
    loss, dl = torch.empty(60, device="cuda"), torch.empty_like(logits)

    def step():
        P.slimdp_layernorm_forward(x, None, None, 1e-5, h, mean, rstd)
        P.slimdp_linear_forward(h, w, None, y, ws, activation="silu")
        P.slimdp_linear_backward_input(dy, w, dx, ws)
        P.slimdp_linear_backward_weight(dy, h, dw, db, ws)
        P.slimdp_layernorm_backward(dx, x, None, mean, rstd, dh, dg, dbeta, ws)
        P.slimdp_distill(logits, idx, teacher, loss, dl, label=label, row_weight=weight, temperature=2.0, kd_weight=0.5,
                         ce_weight=0.5)

    outs = (h, y, dx, dw, db, dh, dg, dbeta, loss, dl)
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    x.copy_(matrix(m, k, torch.bfloat16, g, 2.0))
    logits.copy_(matrix(60, vocab, torch.bfloat16, g, 2.0))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in outs]
    step()
    for a, b in zip(got, outs):
        assert torch.equal(a, b)
    P.train_read_status()
