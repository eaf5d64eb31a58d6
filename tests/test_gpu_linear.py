"""The linear layer (hla_linear / hla_linear_bwd) against float64.

Tolerances, element by element, with u = 2^-24 and h = 2^-8 (bf16) or 2^-24 (fp32), half
a step of the result's type:

  z     (K + 3) u (sum |x||w| + |b|)                 fp32 sums of K exact products
  pre   E_z + h |z|
  y     1.13 E_z + 1e-6 |z| + (h + u) (|act| + |residual|)
        (slopes of the activations stay below 1.13; the bf16 kernel's normal distribution
        is within 3.1e-7, every exponential and reciprocal within 4 u)
  dz    |dy| 2e-6 (1 + |z|) + h |dz|                 z is the pre of the forward
        (rounded for the products; with no activation dz is dy, exact)
  dx    sum_f (E_dz + (F + 3) u |dz|) |w| + h |dx|
  dw    sum_t (E_dz + (T + 3) u |dz|) |x| + h |dw|
  db    sum_t (E_dz without its rounding + (T + 3) u |dz|) + h |db|

and 1% for the second order, with 1e-37 for underflow."""
import ctypes
import math

import pytest
import torch

import paper_2511_05832_amd as hla

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32
HALF = {BF: 2.0 ** -8, F32: U}


def act64(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z * 1


def slope64(z, act):
    z = z.clone().requires_grad_(True)
    return torch.autograd.grad(act64(z, act).sum(), z)[0]


def check(name, got, want, tol):
    over = (got.double().cpu() - want).abs() - 1.01 * tol - 1e-37
    worst = float(torch.nan_to_num(over, nan=math.inf).max())
    assert worst <= 0, f"{name}: {worst:.3e} over the tolerance"


def make(T, K, F, dtype, seed, std=None):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g) * std).to(dtype).cuda()
    return normal(T, K), normal(F, K, std=std or K ** -0.5), normal(F), normal(T, F), normal(T, F)


def check_forward(x, w, b, r, act, y, pre):
    h = HALF[x.dtype]
    X, W = x.double().cpu(), w.double().cpu()
    B = torch.zeros(w.shape[0]).double() if b is None else b.double().cpu()
    R = torch.zeros(y.shape).double() if r is None else r.double().cpu()
    z = X @ W.T + B
    ez = (X.shape[1] + 3) * U * (X.abs() @ W.abs().T + B.abs())
    a = act64(z, act)
    check("y", y, a + R, 1.13 * ez + 1e-6 * z.abs() + (h + U) * (a.abs() + R.abs()))
    if pre is not None:
        check("pre", pre, z, ez + h * z.abs())


def check_backward(x, w, dy, pre, act, dx, dw, db):
    h = HALF[x.dtype]
    X, W, G = x.double().cpu(), w.double().cpu(), dy.double().cpu()
    if act == "none":
        dz, e = G, torch.zeros_like(G)
        er = e
    else:
        Z = pre.double().cpu()
        dz = G * slope64(Z, act)
        e = G.abs() * 2e-6 * (1 + Z.abs())
        er = e + h * dz.abs()
    T, F = dz.shape
    if dx is not None:
        want = dz @ W
        check("dx", dx, want, (er + (F + 3) * U * dz.abs()) @ W.abs() + h * want.abs())
    if dw is not None:
        want = dz.T @ X
        check("dw", dw, want, (er + (T + 3) * U * dz.abs()).T @ X.abs() + h * want.abs())
    if db is not None:
        want = dz.sum(0)
        check("db", db, want, (e + (T + 3) * U * dz.abs()).sum(0) + h * want.abs())


# tokens: one, around the 16- and 64-token kernels, whole and ragged tiles; widths: the
# narrowest, whole tiles, ragged ones, contractions that end inside a stage
SIZES = [(1, 8, 8), (1, 200, 1032), (3, 72, 64), (16, 192, 40), (17, 64, 200), (64, 1032, 24), (65, 8, 136),
         (130, 192, 768), (257, 200, 520), (1000, 64, 64), (2100, 136, 8), (384, 512, 384)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(size, act, dtype):
    x, w, b, r, dy = make(*size, dtype, seed=sum(size))
    y, pre = hla.linear(x, w, b, act=act, residual=r, with_pre=True)
    check_forward(x, w, b, r, act, y, pre)
    assert torch.equal(hla.linear(x, w, b, act=act, residual=r), y)
    check_forward(x, w, None, None, act, hla.linear(x, w, act=act), None)
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act=act, with_bias=True)
    check_backward(x, w, dy, pre, act, dx, dw, db)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(70, 4096, 136), (200, 2056, 520), (513, 1032, 64)], ids=str)
def test_split_contraction_and_without_a_workspace(size, dtype):
    T, K, F = size
    x, w, b, r, _ = make(T, K, F, dtype, seed=7)
    n = ctypes.c_int64()
    assert hla.lib().hla_linear_workspace(T, K, F, 2, hla._dtype_code(x), 0, ctypes.byref(n)) == hla.HLA_OK
    assert n.value > 0
    y, pre = hla.linear(x, w, b, act="gelu", residual=r, with_pre=True)
    check_forward(x, w, b, r, "gelu", y, pre)
    for work in (0, n.value - 16):
        buf = torch.empty(max(work, 16), dtype=torch.uint8, device="cuda")
        y, pre = torch.empty_like(y), torch.empty_like(pre)
        st = hla.lib().hla_linear(*(t.data_ptr() for t in (x, w, b, r)), 2, y.data_ptr(), pre.data_ptr(), T, K, F,
                                  hla._dtype_code(x), buf.data_ptr() if work else 0, work, hla._stream(x))
        assert st == hla.HLA_OK
        check_forward(x, w, b, r, "gelu", y, pre)


# products large enough for the 256-wide tiles, ragged in every direction
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size", [(BF, (4200, 328, 3000)), (BF, (3000, 2600, 520)), (F32, (2000, 196, 1300)),
                                        (BF, (40000, 72, 104))], ids=str)
def test_large(size, dtype):
    x, w, b, r, dy = make(*size, dtype, seed=1)
    y, pre = hla.linear(x, w, b, act="gelu", residual=r, with_pre=True)
    check_forward(x, w, b, r, "gelu", y, pre)
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act="gelu", with_bias=True)
    check_backward(x, w, dy, pre, "gelu", dx, dw, db)


# tiles for every CU, the last of each row and column ragged: a short contraction (128 x
# 128), a longer one (256 x 256), and the same for dx
@pytest.mark.gpu
@pytest.mark.parametrize("size", [(33000, 72, 520), (7700, 264, 2040), (7700, 2040, 264)], ids=str)
def test_tiles_for_every_cu(size):
    x, w, b, r, dy = make(*size, BF, seed=8)
    y, pre = hla.linear(x, w, b, act="gelu", residual=r, with_pre=True)
    check_forward(x, w, b, r, "gelu", y, pre)
    check_forward(x, w, None, None, "silu", hla.linear(x, w, act="silu"), None)
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act="gelu", with_bias=True)
    check_backward(x, w, dy, pre, "gelu", dx, dw, db)


@pytest.mark.gpu
def test_weight_gradients_in_wide_tiles():
    """dw in 256 x 256 tiles that fill the CUs, the last column of them and the tokens
    ragged (as many tiles of 256 as there are CUs)."""
    x, w, b, r, dy = make(200, 4088, 4096, BF, seed=9)
    _, pre = hla.linear(x, w, b, act="gelu", with_pre=True)
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act="gelu", with_bias=True)
    check_backward(x, w, dy, pre, "gelu", dx, dw, db)


@pytest.mark.gpu
def test_weight_gradients_in_parts_of_wide_tiles():
    """dw in 256 x 256 tiles, the tokens in four parts, everything ragged. Rows of dx and of
    dw, each on its own, against float64."""
    T, K, F = 8200, 1016, 4088
    x, w, b, r, dy = make(T, K, F, BF, seed=10)
    n = ctypes.c_int64()
    assert hla.lib().hla_linear_workspace(T, K, F, 0, hla.HLA_BF16, 1, ctypes.byref(n)) == hla.HLA_OK
    tiles = ((K + 255) // 256) * ((F + 255) // 256)
    parts = torch.cuda.get_device_properties(0).multi_processor_count // tiles
    assert parts > 1 and parts * K * F * 4 <= n.value < (parts + 1) * K * F * 4
    y, pre = hla.linear(x, w, b, act="gelu", residual=r, with_pre=True)
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act="gelu", with_bias=True)
    ts = torch.cat([torch.arange(0, T, 97), torch.arange(T - 9, T)]).cuda()
    fs = torch.cat([torch.arange(0, F, 89), torch.arange(F - 9, F)]).cuda()
    check_forward(x[ts], w, b, r[ts], "gelu", y[ts], pre[ts])
    check_backward(x[ts], w, dy[ts], pre[ts], "gelu", dx[ts], None, None)
    check_backward(x, w[fs], dy[:, fs], pre[:, fs], "gelu", None, dw[fs], db[fs])
    assert all(bool(t.isfinite().all()) for t in (y, pre, dx, dw, db))


# dw in 128 x 128 tiles, whole; dx in 256 x 256 tiles, the features in parts
@pytest.mark.gpu
@pytest.mark.parametrize("size", [(304, 2000, 3000), (2050, 2040, 8200)], ids=str)
def test_gradients_in_tiles_of_other_shapes(size):
    T, K, F = size
    x, w, b, r, dy = make(*size, BF, seed=11)
    _, pre = hla.linear(x, w, b, act="silu", with_pre=True)
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act="silu", with_bias=True)
    ts = torch.cat([torch.arange(0, T, 31), torch.arange(T - 9, T)]).cuda()
    fs = torch.cat([torch.arange(0, F, 61), torch.arange(F - 9, F)]).cuda()
    check_backward(x[ts], w, dy[ts], pre[ts], "silu", dx[ts], None, None)
    check_backward(x, w[fs], dy[:, fs], pre[:, fs], "silu", None, dw[fs], db[fs])
    assert all(bool(t.isfinite().all()) for t in (dx, dw, db))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size,keep", [((150, 64, 4096), 0), ((4096, 64, 96), 1)], ids=["dx", "dw"])
def test_one_gradient_in_parts(size, keep, dtype):
    """dx or dw alone, its contraction in parts: the bits of the call for all three."""
    T, K, F = size
    x, w, b, r, dy = make(*size, dtype, seed=12)
    n, code = ctypes.c_int64(), hla._dtype_code(x)
    assert hla.lib().hla_linear_workspace(T, K, F, 0, code, 1, ctypes.byref(n)) == hla.HLA_OK
    want = hla.linear_bwd(x, w, dy)[keep]
    assert n.value >= 2 * want.numel() * 4, "parts"
    got, work = torch.full_like(want, 7.0), torch.empty(n.value, dtype=torch.uint8, device="cuda")
    args = [got.data_ptr() if i == keep else 0 for i in range(3)]
    st = hla.lib().hla_linear_bwd(x.data_ptr(), w.data_ptr(), 0, dy.data_ptr(), 0, *args, T, K, F, code,
                                  work.data_ptr(), n.value, hla._stream(x))
    assert st == hla.HLA_OK, hla.lib().hla_last_error()
    check_backward(x, w, dy, None, "none", got if keep == 0 else None, got if keep == 1 else None, None)
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("K,F", [(8, 8192), (8192, 8)])
def test_more_results_than_32_bits_count(K, F):
    """x or y of 4.9e9 elements: rows at the ends and around element 2^32."""
    T = 600000
    g = torch.Generator(device="cuda").manual_seed(13)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=BF, device="cuda").normal_(0, std, generator=g)
    x, w, b, dy = normal(T, K), normal(F, K, std=K ** -0.5), normal(F), normal(T, F)
    y, pre = hla.linear(x, w, b, act="silu", with_pre=True)
    mid = 2 ** 32 // max(K, F)
    ts = torch.cat([torch.arange(0, 9), torch.arange(mid - 5, mid + 5), torch.arange(T - 9, T)]).cuda()
    check_forward(x[ts], w, b, None, "silu", y[ts], pre[ts])
    dx, dw, db = hla.linear_bwd(x, w, dy, pre, act="silu", with_bias=True)
    check_backward(x[ts], w, dy[ts], pre[ts], "silu", dx[ts], None, None)
    fs, ks = torch.tensor([0, F // 2, F - 1]).cuda(), torch.tensor([0, K // 2 + 1, K - 1]).cuda()
    check_backward(x[:, ks], w[fs][:, ks], dy[:, fs], pre[:, fs], "silu", None, dw[fs][:, ks], db[fs])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_some_gradients_only(dtype):
    T, K, F = 150, 64, 96
    x, w, b, r, dy = make(T, K, F, dtype, seed=2)
    _, pre = hla.linear(x, w, b, act="silu", with_pre=True)
    full = hla.linear_bwd(x, w, dy, pre, act="silu", with_bias=True)
    n = ctypes.c_int64()
    code = hla._dtype_code(x)
    assert hla.lib().hla_linear_workspace(T, K, F, 4, code, 1, ctypes.byref(n)) == hla.HLA_OK
    for keep in ((0,), (1,), (2,), (0, 2)):
        outs = [torch.full_like(t, 7.0) for t in full]
        work = torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda")
        args = [outs[i].data_ptr() if i in keep else 0 for i in range(3)]
        st = hla.lib().hla_linear_bwd(x.data_ptr() if 1 in keep else 0, w.data_ptr() if 0 in keep else 0,
                                      pre.data_ptr(), dy.data_ptr(), 4, *args, T, K, F, code, work.data_ptr(),
                                      n.value, hla._stream(x))
        assert st == hla.HLA_OK, hla.lib().hla_last_error()
        for i in range(3):
            assert torch.equal(outs[i], full[i]) if i in keep else bool((outs[i] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 40, 300])
def test_leading_dimensions_and_residual_in_place(T):
    x, w, b, r, dy = make(2 * T, 64, 72, BF, seed=3)
    want = hla.linear(x, w, b, act="relu", residual=r)
    x3, r3 = x.view(2, T, 64), r.clone().view(2, T, 72)
    got = hla.linear(x3, w, b, act="relu", residual=r3, out=r3)
    assert got is r3 and torch.equal(got.view(-1, 72), want)
    dx, dw, _ = hla.linear_bwd(x3, w, dy.view(2, T, 72))
    assert dx.shape == x3.shape
    check_backward(x, w, dy, None, "none", dx.view(-1, 64), dw, None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
def test_activations_far_out(act, dtype):
    """Arguments from 2^-20 to 2^90 of either sign, through a layer that passes them on."""
    z = torch.cat([s * 2.0 ** torch.arange(-20, 91, 3).float() for s in (1, -1)])
    z = torch.cat([z, torch.tensor([0.0, -0.0, 5.25, -5.25, 9.0, -9.0])]).to(dtype).cuda()
    n = z.numel() // 8 * 8
    x, w = torch.zeros(n, 8, dtype=dtype, device="cuda"), torch.zeros(8, 8, dtype=dtype, device="cuda")
    x[:, 0] = z[:n]
    w[:, 0] = 1.0
    y, pre = hla.linear(x, w, act=act, with_pre=True)
    check_forward(x, w, None, None, act, y, pre)
    dy = torch.ones(n, 8, dtype=dtype, device="cuda")
    dx, _, _ = hla.linear_bwd(x, w, dy, pre, act=act)
    want = 8 * slope64(z[:n].double().cpu(), act)
    # slopes within 1e-6 (the density's argument z^2 / 2 is off by 2 u z^2 / 2, which
    # e^{-z^2 / 2} z outweighs), eight of them summed and rounded twice
    assert float((dx[:, 0].double().cpu() - want).abs().max()) < 8 * (2e-6 + 3 * HALF[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("T", [8, 72])
def test_infinite_arguments(T, act, dtype):
    """In either type: at inf an activation is inf, at -inf relu and gelu are 0 (the other
    two NaN), slopes are their limits at both, and NaN stays NaN."""
    inf, nan = math.inf, math.nan
    z = torch.tensor([inf, -inf, nan, 1.0] * (T // 4)).to(dtype).cuda()
    x, w = torch.zeros(T, 8, dtype=dtype, device="cuda"), torch.zeros(8, 8, dtype=dtype, device="cuda")
    x[:, 0] = z
    w[:, 0] = 1.0
    y, pre = hla.linear(x, w, act=act, with_pre=True)
    assert torch.equal(pre[0::4], torch.full_like(pre[0::4], inf)) and bool(pre[2::4].isnan().all())
    assert bool((y[0::4] == inf).all()) and bool(y[2::4].isnan().all())
    assert bool((y[1::4] == 0).all()) if act in ("relu", "gelu") else bool(y[1::4].isnan().all())
    assert bool(y[3::4].isfinite().all())
    dx, _, _ = hla.linear_bwd(torch.zeros_like(x), w, torch.ones_like(y), pre, act=act)
    assert bool((dx[0::4, 0] == 8).all()) and bool((dx[1::4, 0] == 0).all()) and bool(dx[3::4].isfinite().all())
    if act != "relu":
        assert bool(dx[2::4, 0].isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("T", [7, 200])
def test_nan_and_infinity_stay_in_their_rows(T):
    x, w, b, r, _ = make(T, 72, 40, BF, seed=4)
    want = hla.linear(x, w, b, act="gelu")
    x[3, 5], x[5, 70] = float("nan"), float("inf")
    y = hla.linear(x, w, b, act="gelu")
    rows = [i for i in range(T) if i not in (3, 5)]
    assert torch.equal(y[rows], want[rows]) and bool(y[3].isnan().all()) and not bool(y[5].isfinite().all())


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of <y, dy> in float64 at the fp32 inputs."""
    T, K, F = 6, 8, 12
    x, w, b, r, dy = make(T, K, F, F32, seed=5)
    for act in ("gelu", "gelu_tanh", "silu"):
        _, pre = hla.linear(x, w, b, act=act, with_pre=True)
        grads = hla.linear_bwd(x, w, dy, pre, act=act, with_bias=True)

        def value(ts):
            return float((act64(ts[0] @ ts[1].T + ts[2], act) * dy.double().cpu()).sum())
        step = 2.0 ** -12
        for which, (t, g) in enumerate(zip((x, w, b), grads)):
            for i in range(0, t.numel(), 5):
                ts = [v.double().cpu().clone() for v in (x, w, b)]
                ts[which].view(-1)[i] += step
                up = value(ts)
                ts[which].view(-1)[i] -= 2 * step
                diff = (up - value(ts)) / (2 * step)
                # third derivatives below 2, |x|, |w| < 4, |dy| < 4 over at most 12 terms:
                # step^2 / 6 * 2 * 64 * 4 * 12 = 6e-5; fp32's own 2e-5
                assert abs(diff - float(g.view(-1)[i])) < 6e-5 + 2e-5 * max(1.0, abs(diff)), (act, which, i)


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(5, 256, 512), (300, 256, 512)], ids=str)
def test_two_graphs_replayed_in_turn(size):
    x, w, b, r, dy = make(*size, BF, seed=6)
    x2 = x.flip(0).contiguous()

    def step(t):
        y, pre = hla.linear(t, w, b, act="gelu", residual=r, with_pre=True)
        return (y, pre, *hla.linear_bwd(t, w, dy, pre, act="gelu", with_bias=True))
    step(x)
    torch.cuda.synchronize()
    graphs = []
    for t in (x, x2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = step(t)
        graphs.append((g, res, t))
    for n in range(3):
        b.normal_()
        for g, _, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, res, t in graphs:
            for a, c in zip(res, step(t)):
                assert torch.equal(a, c), n


INV, UNS = hla.HLA_ERR_INVALID_ARG, hla.HLA_ERR_UNSUPPORTED
X, W, B, R, Y, P, G, DX, DW, DB, WK = (0x10000000 * i for i in range(1, 12))


@pytest.mark.parametrize("kw,status,text", [
    (dict(x=0), INV, "x is NULL"),
    (dict(w=0), INV, "w is NULL"),
    (dict(y=0), INV, "y is NULL"),
    (dict(T=0), INV, "positive"),
    (dict(K=0), INV, "positive"),
    (dict(K=36), UNS, "multiples of 8"),
    (dict(F=12), UNS, "multiples of 8"),
    (dict(F=10, dtype=hla.HLA_F32), UNS, "multiples of 4"),
    (dict(T=1 << 31), UNS, "2^30"),
    (dict(K=1 << 20), UNS, "2^20"),
    (dict(dtype=9), INV, "dtype"),
    (dict(act=9), INV, "activation"),
    (dict(x=X + 8), INV, "aligned"),
    (dict(bias=B + 2), INV, "aligned"),
    (dict(y=X), INV, "y overlaps x"),
    (dict(y=W), INV, "y overlaps w"),
    (dict(y=B), INV, "y overlaps bias"),
    (dict(y=R + 16), INV, "y overlaps residual"),
    (dict(pre=R), INV, "pre overlaps residual"),
    (dict(pre=Y + 64), INV, "pre overlaps y"),
    (dict(K=4096, work=X, bytes=1 << 24), INV, "work overlaps x"),
    (dict(K=4096, work=WK + 8, bytes=1 << 24), INV, "aligned"),
], ids=str)
def test_refusals_forward(kw, status, text):
    a = dict(x=X, w=W, bias=B, residual=R, act=2, y=Y, pre=P, T=128, K=64, F=64, dtype=hla.HLA_BF16, work=0,
             bytes=0)
    a.update(kw)
    st = hla.lib().hla_linear(*a.values(), None)
    assert st == status and text in hla.lib().hla_last_error().decode(), hla.lib().hla_last_error()


@pytest.mark.parametrize("kw,status,text", [
    (dict(dx=0, dw=0, db=0), INV, "all NULL"),
    (dict(dy=0), INV, "dy is NULL"),
    (dict(w=0), INV, "w is NULL"),
    (dict(x=0), INV, "x is NULL"),
    (dict(pre=0), INV, "pre is NULL"),
    (dict(T=-1), INV, "positive"),
    (dict(K=36), UNS, "multiples of 8"),
    (dict(work=0), INV, "work is NULL"),
    (dict(bytes=64), INV, "are needed"),
    (dict(work=WK + 8), INV, "aligned"),
    (dict(dx=X), INV, "dx overlaps x"),
    (dict(dx=DW), INV, "dw overlaps dx"),
    (dict(db=DW + 64), INV, "db overlaps dw"),
    (dict(dw=G), INV, "dw overlaps dy"),
    (dict(work=P), INV, "work overlaps pre"),
    (dict(work=DX), INV, "work overlaps dx"),
], ids=str)
def test_refusals_backward(kw, status, text):
    a = dict(x=X, w=W, pre=P, dy=G, act=2, dx=DX, dw=DW, db=DB, T=128, K=64, F=64, dtype=hla.HLA_BF16, work=WK,
             bytes=1 << 26)
    a.update(kw)
    st = hla.lib().hla_linear_bwd(*a.values(), None)
    assert st == status and text in hla.lib().hla_last_error().decode(), hla.lib().hla_last_error()


def test_tensors_are_checked_before_the_workspace():
    """The size of the workspace depends on the device, which is asked last."""
    st = hla.lib().hla_linear_bwd(X + 8, W, P, G, 2, DX, DW, DB, 128, 64, 64, hla.HLA_BF16, 0, 0, None)
    assert st == INV and "x is not 16-byte aligned" in hla.lib().hla_last_error().decode()
    st = hla.lib().hla_linear_bwd(X, W, P, G, 2, DX, DX, DB, 128, 64, 64, hla.HLA_BF16, 0, 0, None)
    assert st == INV and "dw overlaps dx" in hla.lib().hla_last_error().decode()


@pytest.mark.parametrize("T,K,F", [(1 << 30, 8, 8), (1 << 30, 8, 64), (1 << 26, 1024, 8), (1 << 26, 8, 1024)],
                         ids=str)
@pytest.mark.parametrize("dtype", [hla.HLA_BF16, hla.HLA_F32])
def test_more_workgroups_than_a_launch_holds(T, K, F, dtype):
    """A launch counts its threads in 32 bits: 2^24 workgroups of 256 are too many."""
    n = ctypes.c_int64()
    for backward in (0, 1):
        st = hla.lib().hla_linear_workspace(T, K, F, 2, dtype, backward, ctypes.byref(n))
        assert st == UNS and "2^36" in hla.lib().hla_last_error().decode()
    assert hla.lib().hla_linear_workspace((1 << 30) - 256, 8, 64, 2, dtype, 1, ctypes.byref(n)) == hla.HLA_OK
    wide = (1 << 20) - 8   # (the weights' gradient)
    for backward, want in ((0, hla.HLA_OK), (1, UNS)):
        assert hla.lib().hla_linear_workspace(128, wide, wide, 2, dtype, backward, ctypes.byref(n)) == want


def test_refusals_of_the_binding():
    x, w = torch.zeros(4, 8), torch.zeros(8, 8)
    with pytest.raises(hla.HLAError, match="GPU"):
        hla.linear(x, w)
