"""Rotary positions (hla_rope) against float64.

Tolerance: one rounding of the result to its type, half a step: 2^-8 (bf16) or 2^-24
(fp32) of the value, plus the fp32 arithmetic. A turned feature is x1 c - x2 s: sine and
cosine are each off by at most 4e-7 (the angle's rounding to fp32 as half-turns below 1,
pi * 2^-25 = 0.9e-7; float64 products at positions up to 2^28, 3 * 2^-25 = 0.9e-7; the
functions' own two ulps, 2.4e-7 at most), two products and a sum round three times, so
6e-7 (|x1| + |x2|) bounds it."""
import math

import pytest
import torch

import paper_2511_05832_amd as hla

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def reference(x, freqs, pos=None, grid_w=0, interleaved=False, magnitude=1.0, inverse=False):
    """float64, feature by feature. Returns (value, |x1| + |x2| of the pair)."""
    x = x.double().cpu()
    B, H, N, d = x.shape
    pos = torch.arange(N) if pos is None else pos.cpu().long()
    pos = pos.expand(B, N) if pos.dim() == 1 else pos
    f = freqs.double().cpu()
    P = f.numel()
    y, size = x.clone(), x.abs()
    for axis in range(2 if grid_w else 1):
        c = pos if not grid_w else (pos // grid_w if axis == 0 else pos % grid_w)
        for p in range(P):
            a = (c.double() * f[p])[:, None]
            cs, sn = torch.cos(a) * magnitude, torch.sin(a) * (-magnitude if inverse else magnitude)
            i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + P)
            i, j = i + axis * 2 * P, j + axis * 2 * P
            y[..., i] = x[..., i] * cs - x[..., j] * sn
            y[..., j] = x[..., j] * cs + x[..., i] * sn
            size[..., i] = size[..., j] = (x[..., i].abs() + x[..., j].abs()) * abs(magnitude)
    return y, size


def check(got, x, *args, **kw):
    want, size = reference(x, *args, **kw)
    err = (got.double().cpu() - want).abs()
    bar = HALF_STEP[got.dtype] * want.abs() + 6e-7 * size * (1 + HALF_STEP[got.dtype])
    worst = float((err - bar).max())
    assert worst <= 0, f"{worst:.3e} over the tolerance"


def normal(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("grid_w", [0, 7])
# pairs that fill chunks, that cross them, and a single one; all of a row or part of it
@pytest.mark.parametrize("d,turned", [(32, 32), (64, 32), (80, 80), (96, 20), (64, 4), (40, 36)])
def test_layouts(dtype, interleaved, grid_w, d, turned):
    pairs = turned // (4 if grid_w else 2)
    freqs, _ = hla.rope_freqs(pairs)
    x = normal((2, 3, 21, d), dtype, d + turned)
    k = normal((2, 1, 21, d), dtype, d + turned + 1)
    pos = torch.randperm(21, generator=torch.Generator().manual_seed(3)).to(torch.int32).cuda()
    args = dict(pos=pos, grid_w=grid_w, interleaved=interleaved)
    q2, k2 = hla.rope(x, freqs, k=k, **args)
    check(q2, x, freqs, **args)
    check(k2, k, freqs, **args)
    assert torch.equal(hla.rope(x, freqs, **args), q2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,heads,kv,N", [(1, 1, 1, 1), (5, 8, 2, 1), (3, 2, 2, 257), (1, 40, 8, 4096),
                                          (64, 12, 12, 33)])
def test_far_positions_of_each_batch_element(dtype, B, heads, kv, N):
    freqs, m = hla.rope_freqs(32, base=500000.0, factor=8.0, method="parts", length=8192)
    q, k = normal((B, heads, N, 64), dtype, 1), normal((B, kv, N, 64), dtype, 2)
    first = torch.tensor([(2 ** 28 - N - 1) // (b + 1) * (-1) ** b for b in range(B)])
    pos = (first[:, None] + torch.arange(N)).to(torch.int32).cuda()
    q2, k2 = hla.rope(q, freqs, k=k, pos=pos, magnitude=m)
    check(q2, q, freqs, pos=pos, magnitude=m)
    check(k2, k, freqs, pos=pos, magnitude=m)


@pytest.mark.gpu
def test_hilbert_order_gives_the_cells_rotations():
    """Rotating tokens in Hilbert order by the order's ids is rotating them in grid order
    and gathering."""
    H, W = 12, 20
    order, _ = hla.hilbert_perm(H, W)
    freqs, _ = hla.rope_freqs(8, base=100.0)
    x = normal((2, 2, H * W, 32), torch.bfloat16, 5)
    a = hla.rope(hla.gather(x, order), freqs, pos=order, grid_w=W)
    b = hla.gather(hla.rope(x, freqs, grid_w=W), order)
    assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_views_of_one_tensor_in_place(interleaved):
    """q and k inside a projection's [B, N, heads + 2 kv, d]; v is left as it was."""
    B, N, heads, kv, d = 2, 50, 4, 2, 64
    freqs, _ = hla.rope_freqs(20)
    t = normal((B, N, heads + 2 * kv, d), torch.bfloat16, 9)
    was = t.clone()
    q, k = t[:, :, :heads].transpose(1, 2), t[:, :, heads:heads + kv].transpose(1, 2)
    q0, k0 = q.contiguous(), k.contiguous()
    hla.rope(q, freqs, k=k, interleaved=interleaved, q_out=q, k_out=k)
    check(q, q0, freqs, interleaved=interleaved)
    check(k, k0, freqs, interleaved=interleaved)
    assert torch.equal(t[:, :, heads + kv:], was[:, :, heads + kv:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,pairs", [(256, 13), (512, 13), (520, 13), (1040, 6), (1040, 260)])
def test_long_rows(d, pairs, interleaved, dtype):
    """Rows of a wave's chunks, one more, and many; what is not turned keeps its bits."""
    freqs, _ = hla.rope_freqs(pairs)
    x = normal((2, 2, 37, d), dtype, d)
    x[0, 1, 5, 2 * pairs:2 * pairs + 3] = torch.tensor([float("nan"), float("inf"), -0.0])
    got = hla.rope(x, freqs, interleaved=interleaved)
    bits = torch.int16 if dtype is torch.bfloat16 else torch.int32
    assert torch.equal(got[..., 2 * pairs:].contiguous().view(bits), x[..., 2 * pairs:].contiguous().view(bits))
    check(got[..., :2 * pairs].contiguous(), x[..., :2 * pairs].contiguous(), freqs, interleaved=interleaved)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
# pairs that fill accesses, in halves and interleaved; chunks; pairs beside features to copy;
# rows too long for chunks, by the pair and by the access
@pytest.mark.parametrize("d,pairs,interleaved", [(64, 32, False), (64, 32, True), (64, 13, False), (64, 13, True),
                                                 (1032, 13, False), (1032, 64, False)], ids=str)
@pytest.mark.parametrize("where", ["shared", "per batch", "grid"])
def test_more_than_the_caches_hold(d, pairs, interleaved, dtype, where):
    """Calls that move more than 256 MB, with runs of heads that cross batch elements: the
    bits of calls on pieces of the sequence, and rows of them against float64."""
    B, heads, kv = 3, 11, 2
    N = (1 << 27) // (B * (heads + kv) * d * dtype.itemsize) + 13
    assert 2 * B * (heads + kv) * N * d * dtype.itemsize > 256 << 20
    g = torch.Generator(device="cuda").manual_seed(14)
    q, k = (torch.randn(B, h, N, d, generator=g, device="cuda").to(dtype) for h in (heads, kv))
    kw = dict(interleaved=interleaved, grid_w=0)
    pos = torch.randperm(N, generator=g, device="cuda").to(torch.int32)
    if where == "per batch":
        pos = torch.stack([pos, pos.flip(0), pos * 3])
    elif where == "grid":
        kw["grid_w"], pairs = 131, pairs // 2
    freqs, _ = hla.rope_freqs(pairs)
    q2, k2 = hla.rope(q, freqs, k=k, pos=pos, **kw)
    edges = [0, N // 3, N // 3 + 1, N - 8, N]
    for a, b in zip(edges, edges[1:]):
        q3, k3 = hla.rope(q[:, :, a:b], freqs, k=k[:, :, a:b], pos=pos[..., a:b].contiguous(), **kw)
        assert torch.equal(q2[:, :, a:b], q3) and torch.equal(k2[:, :, a:b], k3), (a, b)
    rows = torch.tensor([0, 1, N // 2, N - 2, N - 1], device="cuda")
    check(q2[:, :, rows], q[:, :, rows], freqs, pos=pos[..., rows], **kw)
    check(k2[:, :, rows], k[:, :, rows], freqs, pos=pos[..., rows], **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("pairs,interleaved", [(32, False), (13, False), (13, True)])
def test_rows_that_lie_far_apart(pairs, interleaved):
    """Rows 64 MiB apart, heads side by side: offsets past 32 bits; the bits of the dense call."""
    N, far = 150, 2 ** 25
    freqs, _ = hla.rope_freqs(pairs)
    q, k = normal((1, 3, N, 64), torch.bfloat16, 15), normal((1, 1, N, 64), torch.bfloat16, 16)
    want = hla.rope(q, freqs, k=k, interleaved=interleaved)
    t = torch.empty(N * far, dtype=torch.bfloat16, device="cuda")
    q2, k2, q3, k3 = (t[256 * i:].as_strided((1, h, N, 64), (N * far, 64, far, 1)) for i, h in enumerate((3, 1, 3, 1)))
    q2.copy_(q)
    k2.copy_(k)
    got = hla.rope(q2, freqs, k=k2, interleaved=interleaved, q_out=q3, k_out=k3)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_infinity_stays_in_its_pair(interleaved):
    freqs, _ = hla.rope_freqs(5)
    x = normal((1, 2, 30, 32), torch.bfloat16, 13)
    want = hla.rope(x, freqs, interleaved=interleaved)
    x[0, 1, 7, 3] = float("inf")
    got = hla.rope(x, freqs, interleaved=interleaved)
    pair = [2, 3] if interleaved else [3, 8]
    assert not bool(got[0, 1, 7, pair].isfinite().any())
    got[0, 1, 7, pair] = want[0, 1, 7, pair]
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_one_row_for_the_whole_batch():
    freqs, _ = hla.rope_freqs(16)
    x = normal((1, 2, 5, 32), torch.float32, 4)
    got = hla.rope(x.expand(3, 2, 5, 32), freqs)
    check(got, x.expand(3, 2, 5, 32), freqs)


@pytest.mark.gpu
def test_inverse_is_the_gradient():
    """<rope(x), g> differenced in x, against rope(g, inverse)."""
    freqs, _ = hla.rope_freqs(8)
    x, g = normal((1, 2, 9, 32), torch.float32, 6), normal((1, 2, 9, 32), torch.float32, 7)
    kw = dict(grid_w=3, magnitude=1.25)
    grad = hla.rope(g, freqs, inverse=True, **kw)
    check(grad, g, freqs, inverse=True, **kw)
    step = 0.5   # the map is linear: a difference of any length is exact but for rounding
    for i in range(0, x.numel(), 37):
        e = torch.zeros_like(x)
        e.view(-1)[i] = step
        up, down = hla.rope(x + e, freqs, **kw), hla.rope(x - e, freqs, **kw)
        diff = ((up.double() - down.double()) * g.double()).sum() / (2 * step)
        # each difference of 32-bit values below 8 is off by at most 8 * 2^-22, of which
        # the pair's two differ from zero, times |g| < 5
        assert abs(float(diff) - float(grad.view(-1)[i])) < 2 * 8 * 2.0 ** -22 * 5


@pytest.mark.gpu
def test_graph_replays():
    freqs, _ = hla.rope_freqs(16)
    x = normal((2, 3, 65, 32), torch.bfloat16, 11)
    pos = torch.zeros(2, 65, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    hla.rope(x, freqs, pos=pos, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hla.rope(x, freqs, pos=pos, q_out=out)
    for r in range(3):
        pos.copy_(torch.arange(130).view(2, 65) * (r + 1))
        x.normal_()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, hla.rope(x, freqs, pos=pos)), r


@pytest.mark.gpu
def test_another_stream():
    freqs, _ = hla.rope_freqs(16)
    x = normal((2, 3, 65, 32), torch.float32, 12)
    want = hla.rope(x, freqs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = hla.rope(x, freqs)
    s.synchronize()
    assert torch.equal(got, want)


def test_frequencies():
    f, m = hla.rope_freqs(4, base=10000.0, device="cpu")
    assert m == 1.0 and torch.allclose(f, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64))
    f4, _ = hla.rope_freqs(4, factor=4.0, device="cpu")
    assert torch.equal(f4, f / 4)
    fb, _ = hla.rope_freqs(4, factor=4.0, method="base", device="cpu")
    assert float(fb[0]) == 1.0 and math.isclose(float(fb[3]), float(f[3]) / 4)
    fp, m = hla.rope_freqs(4, factor=4.0, method="parts", length=6283, device="cpu")
    assert math.isclose(m, 1 + 0.1 * math.log(4.0))
    # 1000 and 100 turns: unchanged; 10 turns: 9 / 31 kept; 1 turn: divided
    assert torch.equal(fp[:2], f[:2]) and math.isclose(float(fp[3]), float(f[3]) / 4, rel_tol=1e-4)
    keep = (6283 * 0.01 / (2 * math.pi) - 1) / 31
    assert math.isclose(float(fp[2]), 0.01 * (keep + (1 - keep) / 4), rel_tol=1e-12)
    for bad in (dict(pairs=0), dict(pairs=4, factor=0.5), dict(pairs=4, method="x"),
                dict(pairs=4, method="parts")):
        with pytest.raises(hla.HLAError):
            hla.rope_freqs(device="cpu", **bad)


class Raw:
    """The C entry point on made-up addresses: every call here must be refused."""
    A, B, C, D, F, P = (0x10000000 * i for i in range(1, 7))

    def __init__(self):
        self.a = dict(q=(self.A, 4096, 2048, 64), k=None, q_out=(self.B, 4096, 2048, 64), k_out=None, pos=0,
                      pos_stride=0, freqs=self.F, B=2, heads=2, kv_heads=0, N=32, d=64, pairs=16,
                      grid_w=0, interleaved=0, inverse=0, magnitude=1.0, dtype=hla.HLA_BF16)

    def __call__(self, **kw):
        a = dict(self.a, **kw)
        for n in ("q", "k", "q_out", "k_out"):
            a[n] = None if a[n] is None else hla.View(*a[n])
        st = hla.lib().hla_rope(*a.values(), None)
        return st, hla.lib().hla_last_error().decode()


INV, UNS = hla.HLA_ERR_INVALID_ARG, hla.HLA_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,status,text", [
    (dict(q=None), INV, "NULL"),
    (dict(k=(Raw.C, 0, 0, 64)), INV, "k and k_out"),
    (dict(k=(Raw.C, 0, 0, 64), k_out=(Raw.D, 4096, 2048, 64)), INV, "positive"),
    (dict(N=0), INV, "positive"),
    (dict(pairs=0), INV, "positive"),
    (dict(pairs=33), INV, "features"),
    (dict(pairs=17, grid_w=8), INV, "features"),
    (dict(grid_w=-1), INV, "grid_w"),
    (dict(magnitude=float("nan")), INV, "finite"),
    (dict(d=36, pairs=4), UNS, "multiple of 16"),
    (dict(N=1 << 26, B=1, q=(Raw.A, 0, 0, 64)), UNS, "2^30"),
    (dict(freqs=0), INV, "freqs"),
    (dict(freqs=Raw.F + 4), INV, "aligned"),
    (dict(pos=Raw.P + 2), INV, "aligned"),
    (dict(pos=Raw.P, pos_stride=31), INV, "pos_stride"),
    (dict(pos=Raw.B + 8), INV, "overlaps pos"),
    (dict(freqs=Raw.B + 8), INV, "overlaps freqs"),
    (dict(q=(Raw.A + 8, 4096, 2048, 64)), INV, "aligned"),
    (dict(q=(Raw.A, 4096, 2048, 68)), INV, "stride"),
    (dict(q=(Raw.A, 4096, -2048, 64)), INV, "stride"),
    (dict(q_out=(Raw.B, 4096, 0, 64)), INV, "overlap each other"),
    (dict(q_out=(Raw.A + 128, 4096, 2048, 64)), INV, "overlaps q"),
    (dict(q_out=(Raw.A, 4096, 64, 128)), INV, "overlaps q"),
    # k_out in the rows of q_out
    (dict(k=(Raw.C, 4096, 2048, 64), k_out=(Raw.B, 4096, 2048, 64), kv_heads=2), INV, "k_out"),
    (dict(dtype=7), INV, "dtype"),
], ids=str)
def test_refusals(kw, status, text):
    st, msg = Raw()(**kw)
    assert st == status and text in msg, (st, msg)


def test_refusals_of_the_binding():
    x = torch.zeros(1, 1, 2, 32)
    with pytest.raises(hla.HLAError, match="GPU"):
        hla.rope(x, torch.ones(4, dtype=torch.float64))
