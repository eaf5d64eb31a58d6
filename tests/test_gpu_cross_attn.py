"""Cross attention (hla_cross_attn_fwd / hla_cross_attn_bwd) against float64.

Tolerances, element by element, from first-order error bounds with u = 2^-24 and, for
bf16, h = 2^-8 (half a step, relative to the value; 0 for fp32):

  scores    E_S = (d + 6) u scale sum |q||k| + 4 u |S|     (fp32 sums of d products)
  weights   e_P = 2 E_S + (M + 8) u, relative               (the row's sum is off too)
  out       sum_j P|v| (e_P + h + (M + 8) u) + (h + u) |out|
            (h: weights rounded to bf16 as operands; the result's own rounding)
  lse       E_S + (M + 8) u + 2 u |lse|
  dS        P (|dP - delta| (e_P + h + 4 u) + E_dP + E_delta), with
            E_dP = (d + 2) u sum |dout||v|, E_delta = sum |dout| E_out + (d + 2) u sum |dout||out|
  dq        scale sum_j (E_dS + M u |dS|) |k| + (h + u) |dq|
  dk        scale sum_r (E_dS + R u |dS|) |q| + (h + u) |dk|      (R: rows that share the key)
  dv        sum_r P (e_P + h + (R + 8) u) |dout| + (h + u) |dv|

and 2% for the second order, with 1e-30 for underflow."""
import ctypes

import pytest
import torch

import paper_2511_05832_amd as hla

U = 2.0 ** -24
BF, F32 = torch.bfloat16, torch.float32


def reference(q, k, v, lengths, scale, dout=None):
    """{name: (value, tolerance)} in float64 on the CPU."""
    h = 2.0 ** -8 if q.dtype == BF else 0.0
    q, k, v = (t.detach().double().cpu() for t in (q, k, v))
    B, H, N, d = q.shape
    kv, M = k.shape[1], k.shape[2]
    G = H // kv
    R = G * N
    res = {n: (torch.zeros(B, H, N, d).double(), torch.zeros(B, H, N, d).double()) for n in ("out", "dq")}
    res.update({n: (torch.zeros_like(k), torch.zeros_like(k)) for n in ("dk", "dv")})
    res["lse"] = (torch.full((B, H, N), -torch.inf).double(), torch.zeros(B, H, N).double())
    for b in range(B):
        n = M if lengths is None else max(0, min(M, int(lengths[b])))
        if n == 0:
            continue
        for hh in range(H):
            t = hh // G
            Q, K, V = q[b, hh], k[b, t, :n], v[b, t, :n]
            S = scale * (Q @ K.T)
            ES = (d + 6) * U * scale * (Q.abs() @ K.abs().T) + 4 * U * S.abs()
            lse = torch.logsumexp(S, 1)
            P = torch.exp(S - lse[:, None])
            es = ES.max(1, keepdim=True).values
            eP = 2 * es + (M + 8) * U
            out = P @ V
            eo = (P * (eP + h + (M + 8) * U)) @ V.abs() + (h + U) * out.abs()
            res["out"][0][b, hh], res["out"][1][b, hh] = out, eo
            res["lse"][0][b, hh] = lse
            res["lse"][1][b, hh] = es[:, 0] + (M + 8) * U + 2 * U * lse.abs()
            if dout is None:
                continue
            D = dout[b, hh].double().cpu()
            dP = D @ V.T
            delta = (P * dP).sum(1, keepdim=True)
            dS = P * (dP - delta)
            e_delta = (D.abs() * eo).sum(1, keepdim=True) + (d + 2) * U * (D.abs() * out.abs()).sum(1, keepdim=True)
            eS = P * ((dP - delta).abs() * (eP + h + 4 * U) + (d + 2) * U * (D.abs() @ V.abs().T) + e_delta)
            res["dq"][0][b, hh] = scale * dS @ K
            res["dq"][1][b, hh] = scale * (eS + M * U * dS.abs()) @ K.abs()
            res["dk"][0][b, t, :n] += scale * dS.T @ Q
            res["dk"][1][b, t, :n] += scale * (eS + R * U * dS.abs()).T @ Q.abs()
            res["dv"][0][b, t, :n] += P.T @ D
            res["dv"][1][b, t, :n] += (P * (eP + h + (R + 8) * U)).T @ D.abs()
    for n in ("dq", "dk", "dv"):
        res[n][1].add_((h + U) * res[n][0].abs())
    return res


def compare(name, got, ref):
    want, tol = ref[name]
    got = got.double().cpu()
    none = torch.isinf(want)
    assert torch.equal(got[none], want[none]), f"{name}: rows without a key"
    over = torch.where(none, 0.0, (got - want).abs() - 1.02 * tol - 1e-30)
    worst = float(torch.nan_to_num(over, nan=torch.inf).max())
    assert worst <= 0, f"{name}: {worst:.3e} over the tolerance"


def inputs(B, H, kv, N, M, d, dtype, seed, packed=False):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g).to(dtype).cuda()
    if packed:
        t = normal(B, M, 2, kv, d)
        k, v = t[:, :, 0].transpose(1, 2), t[:, :, 1].transpose(1, 2)
        return normal(B, N, H, d).transpose(1, 2), k, v, normal(B, N, H, d).transpose(1, 2)
    return normal(B, H, N, d), normal(B, kv, M, d), normal(B, kv, M, d), normal(B, H, N, d)


def lengths_of(B, M, kind):
    if kind == "all":
        return None
    ls = {"ends": [M, 0, 1, M - 1], "inside": [M // 2 + 1, 64, 32, 33], "past": [M + 7, -3, M, 1 << 30]}[kind]
    return torch.tensor([ls[b % 4] for b in range(B)], dtype=torch.int32, device="cuda")


SIZES = [  # B, heads, kv_heads, N, M, d
    (1, 1, 1, 1, 1, 32),
    (4, 4, 2, 1, 300, 64),
    (4, 6, 3, 65, 77, 32),
    (2, 2, 2, 33, 64, 64),
    (2, 8, 1, 5, 1000, 64),
    (1, 2, 1, 200, 129, 64),
    (1, 3, 3, 128, 128, 32),
    (3, 1, 1, 700, 31, 64),
    (1, 2, 2, 1500, 96, 32),
    (1, 4, 4, 16, 5000, 32),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kind", ["all", "ends", "inside", "past"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(size, kind, dtype):
    B, H, kv, N, M, d = size
    q, k, v, dout = inputs(*size, dtype, seed=sum(size))
    lengths = lengths_of(B, M, kind)
    ref = reference(q, k, v, lengths, d ** -0.5, dout)
    out, lse = hla.cross_attn_fwd(q, k, v, lengths)
    compare("out", out, ref)
    compare("lse", lse, ref)
    for name, g in zip(("dq", "dk", "dv"), hla.cross_attn_bwd(q, k, v, out, dout, lse, lengths)):
        compare(name, g, ref)


# the row splits of dk and dv go by what the lengths leave: most of it, little, one key,
# nothing; and over more batch elements than are looked at
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size,lengths", [
    ((5, 2, 1, 2000, 300, 32), [0, 300, 64, 1, 0]), ((5, 2, 1, 2000, 300, 32), [129, 0, 0, 0, 0]),
    ((5, 2, 1, 2000, 300, 32), [0] * 5), ((3, 2, 2, 4100, 100, 64), [100, 5, 70]),
    ((70, 1, 1, 1000, 40, 32), [b % 41 for b in range(70)])], ids=str)
def test_gradients_of_uneven_lengths(size, lengths, dtype):
    q, k, v, dout = inputs(*size, dtype, seed=9)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    ref = reference(q, k, v, n, size[-1] ** -0.5, dout)
    out, lse = hla.cross_attn_fwd(q, k, v, n)
    for name, got in zip(("dq", "dk", "dv"), hla.cross_attn_bwd(q, k, v, out, dout, lse, n)):
        compare(name, got, ref)


@pytest.mark.gpu
def test_replays_with_other_lengths():
    """A captured step whose lengths change between replays, row splits of dk and dv with them."""
    q, k, v, dout = inputs(5, 2, 1, 2000, 300, 32, BF, seed=10)
    n = torch.full((5,), 300, dtype=torch.int32, device="cuda")

    def step():
        out, lse = hla.cross_attn_fwd(q, k, v, n)
        return (out, lse, *hla.cross_attn_bwd(q, k, v, out, dout, lse, n))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for lengths in ([300, 0, 3, 128, 129], [0, 0, 64, 0, 0], [0] * 5, [300] * 5):
        n.copy_(torch.tensor(lengths, dtype=torch.int32))
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for t, want in zip(got, step()):
            assert torch.equal(t, want), lengths


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(2, 4, 2, 40, 77, 64), (4, 6, 6, 1, 200, 32)], ids=str)
def test_views_of_projections(size, dtype):
    """q as [B, N, heads, d], k and v inside one [B, M, 2, kv, d], gradients into the same
    layouts: the bits of the contiguous call, and nothing outside the rows written."""
    B, H, kv, N, M, d = size
    q, k, v, dout = inputs(*size, dtype, seed=5, packed=True)
    lengths = lengths_of(B, M, "inside")
    want, wl = hla.cross_attn_fwd(q.contiguous(), k.contiguous(), v.contiguous(), lengths)
    wg = hla.cross_attn_bwd(q.contiguous(), k.contiguous(), v.contiguous(), want, dout.contiguous(), wl, lengths)

    def spaced(*shape):   # a tensor with a guard row after every row
        t = torch.full((*shape[:-1], 2 * shape[-1]), 7.0, dtype=dtype, device="cuda")
        return t, t[..., :shape[-1]]
    raw_o, o = spaced(B, N, H, d)
    raw_q, dq = spaced(B, N, H, d)
    raw_kv, dkv = spaced(B, M, 2, kv, d)
    out, lse = hla.cross_attn_fwd(q, k, v, lengths, out=o.transpose(1, 2))
    grads = hla.cross_attn_bwd(q, k, v, out, dout, lse, lengths, dq=dq.transpose(1, 2),
                               dk=dkv[:, :, 0].transpose(1, 2), dv=dkv[:, :, 1].transpose(1, 2))
    assert torch.equal(out, want) and torch.equal(lse, wl)
    for a, b in zip(grads, wg):
        assert torch.equal(a, b)
    for raw in (raw_o, raw_q, raw_kv):
        assert bool((raw[..., d:] == 7.0).all())
    assert hla.cross_attn_fwd(q, k, v, lengths)[0].stride() == q.stride()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 50])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -3e38])
def test_unseen_states_reach_nothing(bad, N, dtype):
    B, H, kv, M, d = 4, 4, 2, 330, 64
    q, k, v, dout = inputs(B, H, kv, N, M, d, dtype, seed=8)
    lengths = torch.tensor([0, 1, 100, 320], dtype=torch.int32, device="cuda")
    want, lse = hla.cross_attn_fwd(q, k, v, lengths)
    grads = hla.cross_attn_bwd(q, k, v, want, dout, lse, lengths)
    for b, n in enumerate(lengths.tolist()):
        k[b, :, n:] = bad
        v[b, :, n:] = bad
    out, lse2 = hla.cross_attn_fwd(q, k, v, lengths)
    assert torch.equal(out, want) and torch.equal(lse, lse2)
    assert bool((out[0] == 0).all()) and bool((lse[0] == -torch.inf).all())
    for a, b in zip(hla.cross_attn_bwd(q, k, v, out, dout, lse, lengths), grads):
        assert torch.equal(a, b)
    assert all(bool((g[b, :, n:] == 0).all()) for g in grads[1:] for b, n in enumerate(lengths.tolist()))


# keys that stay in LDS; tiles of 128 rows; few rows
@pytest.mark.gpu
@pytest.mark.parametrize("N,M", [(300, 77), (2100, 200), (40, 200)])
def test_gradients_where_few_keys_are_seen(N, M):
    """dS = P (dP - delta) cancels where one to three keys share the weight; the rounding
    of out must not come through delta. What may: dS rounded as an operand and the result,
    each by half a step at most, uniformly: sqrt(2) 2^-8 / sqrt(3) = 3.2e-3 in the 2-norm
    (<dout, out> of the rounded out would leave 4.4e-3)."""
    B, H, kv, d = 4, 4, 4, 64
    q, k, v, dout = inputs(B, H, kv, N, M, d, BF, seed=2)
    lengths = torch.tensor([1, 2, 3, 3], dtype=torch.int32, device="cuda")
    out, lse = hla.cross_attn_fwd(q, k, v, lengths)
    ref = reference(q, k, v, lengths, d ** -0.5, dout)
    for name, g in zip(("dq", "dk", "dv"), hla.cross_attn_bwd(q, k, v, out, dout, lse, lengths)):
        want = ref[name][0]
        assert float((g.double().cpu() - want).norm() / want.norm()) < 3.2e-3, name


@pytest.mark.gpu
def test_large_scores():
    """Scores of several hundred, of either sign: the running maximum carries them."""
    B, H, kv, N, M, d = 2, 2, 2, 40, 200, 32
    q, k, v, dout = inputs(B, H, kv, N, M, d, F32, seed=3)
    q, scale = q * 20, 2.0
    ref = reference(q, k, v, None, scale, dout)
    out, lse = hla.cross_attn_fwd(q, k, v, scale=scale)
    compare("out", out, ref)
    compare("lse", lse, ref)
    for name, g in zip(("dq", "dk", "dv"), hla.cross_attn_bwd(q, k, v, out, dout, lse, scale=scale)):
        compare(name, g, ref)


@pytest.mark.gpu
def test_states_shared_by_the_batch():
    """k and v of one batch element expanded over all (stride 0)."""
    q, k, v, dout = inputs(3, 4, 2, 20, 90, 64, BF, seed=4)
    k, v = k[:1].expand(3, -1, -1, -1), v[:1].expand(3, -1, -1, -1)
    want, lse = hla.cross_attn_fwd(q, k.contiguous(), v.contiguous())
    out, _ = hla.cross_attn_fwd(q, k, v)
    assert torch.equal(out, want)
    dk, dv = torch.empty(3, 2, 90, 64, dtype=BF, device="cuda"), torch.empty(3, 2, 90, 64, dtype=BF, device="cuda")
    a = hla.cross_attn_bwd(q, k, v, out, dout, lse, dk=dk, dv=dv)
    b = hla.cross_attn_bwd(q, k.contiguous(), v.contiguous(), out, dout, lse)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.gpu
def test_gradients_against_differences():
    """Central differences of <out, dout> in float32 inputs. The float64 value of the same
    inputs stands in for the forward, whose own error is bounded above."""
    B, H, kv, N, M, d = 1, 2, 1, 5, 9, 32
    q, k, v, dout = inputs(B, H, kv, N, M, d, F32, seed=6)
    lengths = torch.tensor([7], dtype=torch.int32, device="cuda")
    out, lse = hla.cross_attn_fwd(q, k, v, lengths)
    grads = hla.cross_attn_bwd(q, k, v, out, dout, lse, lengths)
    D = dout.double().cpu()

    def value(ts):
        r = reference(*ts, lengths, d ** -0.5)
        return float((r["out"][0] * D).sum())
    step = 2.0 ** -12
    for which, (t, g) in enumerate(zip((q, k, v), grads)):
        for i in range(0, t.numel(), t.numel() // 11):
            ts = [x.detach().double().cpu().clone() for x in (q, k, v)]
            ts[which].view(-1)[i] += step
            up = value(ts)
            ts[which].view(-1)[i] -= 2 * step
            diff = (up - value(ts)) / (2 * step)
            # a third derivative of at most 10 times step^2 / 6, and float32's bound of 1e-5
            assert abs(diff - float(g.view(-1)[i])) < 10 * step ** 2 + 1e-5 * max(1.0, abs(diff))


@pytest.mark.gpu
@pytest.mark.parametrize("size", [(2, 4, 2, 1, 2000, 64), (2, 4, 2, 300, 77, 64)], ids=str)
def test_two_graphs_replayed_in_turn(size):
    """Two captured steps with workspaces of their own, replayed in turn with eager calls
    between, give the eager bits every time."""
    q, k, v, dout = inputs(*size, BF, seed=12)
    lengths = torch.full((size[0],), size[4], dtype=torch.int32, device="cuda")

    def step(qq):
        out, lse = hla.cross_attn_fwd(qq, k, v, lengths)
        return (out, lse, *hla.cross_attn_bwd(qq, k, v, out, dout, lse, lengths))
    q2 = q.flip(2).contiguous() * 2
    step(q)
    torch.cuda.synchronize()
    graphs = []
    for x in (q, q2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = step(x)
        graphs.append((g, r, x))
    for n in (size[4], 70, 0, 33):
        lengths.fill_(n)
        for g, _, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, r, x in graphs:
            for a, b in zip(r, step(x)):
                assert torch.equal(a, b), n


@pytest.mark.gpu
def test_streams_at_once():
    """Calls on two streams, each with its own workspace."""
    size = (2, 4, 2, 3, 3000, 64)
    sets = [inputs(*size, BF, seed=s) for s in (1, 2)]
    want = [hla.cross_attn_fwd(*s[:3])[0] for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = []
    for _ in range(3):
        for st, s in zip(streams, sets):
            with torch.cuda.stream(st):
                got.append(hla.cross_attn_fwd(*s[:3])[0])
    torch.cuda.synchronize()
    for i, t in enumerate(got):
        assert torch.equal(t, want[i % 2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
# keys that stay in LDS; few rows, without and with key splits; many rows
@pytest.mark.parametrize("size", [(1, 2, 2, 300, 77, 32), (2, 4, 2, 40, 300, 64), (2, 4, 2, 1, 3000, 64),
                                  (4, 2, 2, 4001, 321, 64)], ids=str)
def test_large_values(size, dtype):
    """Values of 2^101 under scores of 16: the results are in range, and no sum before the
    division by the row's weight may leave it (weights about a reference of 0, e^16 each,
    would take 30 of them to 2^129)."""
    q, k, v, _ = inputs(*size, dtype, seed=21)
    q, k = 1 + 0.05 * q, 1 + 0.05 * k
    v = 2.0 ** 101 * v.abs()
    scale = 16.0 / size[-1]
    out, lse = hla.cross_attn_fwd(q, k, v, scale=scale)
    ref = reference(q[:1, :1], k[:1, :1], v[:1, :1], None, scale)
    compare("out", out[:1, :1], ref)
    compare("lse", lse[:1, :1], ref)
    assert bool(out.isfinite().all())


def cus():
    return torch.cuda.get_device_properties(0).multi_processor_count


def work_bytes(size, dtype, backward):
    n = ctypes.c_int64()
    code = hla.HLA_BF16 if dtype is BF else hla.HLA_F32
    assert hla.lib().hla_cross_attn_workspace(*size, code, backward, ctypes.byref(n)) == hla.HLA_OK
    return n.value


def check_pairs(size, lengths, dtype, seed, pairs):
    """A step, with NaN in the states that are not seen: some (batch, key head) pairs, each
    on its own, against float64, and no other result NaN or infinite."""
    B, H, kv, N, M, d = size
    G = H // kv
    q, k, v, dout = inputs(*size, dtype, seed=seed)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for b, x in enumerate(lengths or ()):
        k[b, :, x:] = v[b, :, x:] = float("nan")
    out, lse = hla.cross_attn_fwd(q, k, v, n)
    grads = hla.cross_attn_bwd(q, k, v, out, dout, lse, n)
    for b, t in pairs:
        one, hs, ts = slice(b, b + 1), slice(t * G, t * G + G), slice(t, t + 1)
        ref = reference(q[one, hs], k[one, ts], v[one, ts], None if n is None else n[one], d ** -0.5, dout[one, hs])
        for name, got, heads in zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *grads), (hs, hs, hs, ts, ts)):
            compare(name, got[one, heads], ref)
    assert all(bool(g.isfinite().all()) for g in (out, *grads))
    assert torch.equal(lse.isfinite().all(2).all(1).cpu(),
                       torch.tensor([x > 0 for x in lengths] if lengths else [True] * B))


# Tiles of 128 rows (as many as there are CUs, and keys that do not stay in LDS), several
# key tiles, ragged at both ends: below, at and above the 256 keys up to which delta is put
# right, with elements that see none; shared heads; and dk and dv in tiles of 128 keys, the
# rows split (the first three) or not (the last)
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("size,lengths", [
    ((4, 2, 2, 4001, 321, 64), None), ((4, 2, 2, 4001, 321, 64), [321, 257, 256, 129]),
    ((4, 2, 2, 4001, 321, 32), [0, 1, 65, 320]), ((2, 8, 2, 2050, 700, 64), [700, 333]),
    ((2, 8, 2, 2050, 700, 32), None), ((8, 8, 8, 400, 300, 64), [300, 0, 1, 299, 128, 129, 257, 64]),
    ((8, 8, 8, 400, 300, 32), None)], ids=str)
def test_many_rows(size, lengths, dtype):
    B, H, kv, N, M, d = size
    rows = B * kv * ((H // kv * N + 127) // 128)
    assert M > 128 and rows >= cus(), "tiles of 128 rows"
    parts = 2 * B * kv * ((M + 127) // 128) <= cus()
    stats = 8 * B * kv * ((H // kv * N + 127) // 128 * 128)
    assert (work_bytes(size, dtype, 1) > stats) == parts and parts == (size[0] < 8)
    check_pairs(size, lengths, dtype, 31, [(0, 0), (1, kv - 1), (B - 2, 1), (B - 1, 0)])


@pytest.mark.gpu
@pytest.mark.parametrize("lengths", [None, [130, 1, 0, 129, 64, 128, 127, 130, 33, 0, 100]], ids=["all", "ragged"])
def test_two_workgroups_per_cu_for_dk_and_dv(lengths):
    """Heads of 32 in bf16 with rows enough that the splits of dk and dv take twice as many
    workgroups as there are CUs."""
    size = (11, 4, 4, 6000, 130, 32)
    assert work_bytes(size, BF, 1) == 8 * 44 * 6016 + 2 * cus() * 128 * 8 * 32
    check_pairs(size, lengths, BF, 32, [(0, 0), (3, 1), (5, 2), (10, 3)])


# a token and its key splits, few rows, keys that stay in LDS, many rows
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N,M", [(1, 1100), (70, 1100), (200, 100), (33000, 300)])
def test_rows_that_lie_far_apart(N, M, dtype):
    """States 16 MiB apart (in one tensor, heads side by side) and queries over some 8 GiB:
    offsets past 32 bits in every input and output; the bits of the dense call."""
    B, H, kv, d = 1, 2, 1, 64
    q, k, v, dout = inputs(B, H, kv, N, M, d, dtype, seed=41)
    n = torch.tensor([M - 3], dtype=torch.int32, device="cuda")
    want, lse = hla.cross_attn_fwd(q, k, v, n)
    grads = hla.cross_attn_bwd(q, k, v, want, dout, lse, n)
    far, near = 2 ** 24 // dtype.itemsize, min(2 ** 25, 2 ** 33 // N // dtype.itemsize // 1024 * 1024)
    states = torch.empty(M * far, dtype=dtype, device="cuda")
    rows = torch.empty(N * near, dtype=dtype, device="cuda")
    k2, v2, dk, dv = (states[256 * i:].as_strided((B, kv, M, d), (M * far, d, far, 1)) for i in range(4))
    q2, out, dout2, dq = (rows[256 * i:].as_strided((B, H, N, d), (N * near, d, near, 1)) for i in range(4))
    for to, t in ((q2, q), (k2, k), (v2, v), (dout2, dout)):
        to.copy_(t)
    got, lse2 = hla.cross_attn_fwd(q2, k2, v2, n, out=out)
    assert torch.equal(got, want) and torch.equal(lse2, lse)
    for a, b in zip(hla.cross_attn_bwd(q2, k2, v2, got, dout2, lse2, n, dq=dq, dk=dk, dv=dv), grads):
        assert torch.equal(a, b)


class Raw:
    """The C entries on made-up addresses: every call here must be refused."""
    Q, K, V, O, L, W, G, DQ, DK, DV, N = (0x10000000 * i for i in range(1, 12))

    def __init__(self):
        row = (64 * 64 * 4, 64 * 64, 64)
        self.fwd = dict(q=(self.Q, *row), k=(self.K, *row), v=(self.V, *row), lengths=0, out=(self.O, *row),
                        lse=self.L, B=2, heads=4, kv=4, N=64, M=64, d=64, dtype=hla.HLA_BF16, scale=0.125,
                        work=self.W, bytes=1 << 28)
        self.bwd = dict(q=(self.Q, *row), k=(self.K, *row), v=(self.V, *row), out=(self.O, *row),
                        dout=(self.G, *row), lse=self.L, lengths=0, dq=(self.DQ, *row), dk=(self.DK, *row),
                        dv=(self.DV, *row), B=2, heads=4, kv=4, N=64, M=64, d=64, dtype=hla.HLA_BF16,
                        scale=0.125, work=self.W, bytes=1 << 28)

    def __call__(self, backward, kw):
        a = dict(self.bwd if backward else self.fwd)
        a.update((n, x) for n, x in kw.items() if n in a)
        a = [None if n in VIEWS and x is None else (hla.View(*x) if n in VIEWS else x) for n, x in a.items()]
        st = (hla.lib().hla_cross_attn_bwd if backward else hla.lib().hla_cross_attn_fwd)(*a, None)
        return st, hla.lib().hla_last_error().decode()


VIEWS = {"q", "k", "v", "out", "dout", "dq", "dk", "dv"}
INV, UNS = hla.HLA_ERR_INVALID_ARG, hla.HLA_ERR_UNSUPPORTED
ROW = (64 * 64 * 4, 64 * 64, 64)


@pytest.mark.parametrize("kw,status,text", [
    (dict(q=None), INV, "NULL"),
    (dict(out=None), INV, "NULL"),
    (dict(N=0), INV, "positive"),
    (dict(M=0), INV, "positive"),
    (dict(kv=3), INV, "multiple of kv_heads"),
    (dict(d=48), UNS, "head_dim"),
    (dict(N=1 << 31), UNS, "2^30"),
    (dict(heads=1 << 21, N=1 << 20), UNS, "2^30"),
    (dict(dtype=5), INV, "dtype"),
    (dict(scale=0.0), INV, "scale"),
    (dict(scale=float("nan")), INV, "scale"),
    (dict(lse=Raw.L + 2), INV, "lse"),
    (dict(lengths=2), INV, "lengths"),
    (dict(q=(Raw.Q + 8, *ROW)), INV, "aligned"),
    (dict(k=(Raw.K, *ROW[:2], 60)), INV, "stride"),
    (dict(v=(Raw.V, *ROW[:2], -64)), INV, "stride"),
    (dict(k=(Raw.K, *ROW[:2], 1 << 24)), UNS, "2^25"),
    (dict(q=(Raw.Q, 1 << 45, 1 << 36, 64)), UNS, "2^36"),
    (dict(work=0, M=100000, N=64, B=1, heads=1, kv=1), INV, "work"),
    (dict(lse=Raw.W, N=1, M=4096, B=1, heads=1, kv=1), INV, "overlaps"),
], ids=str)
@pytest.mark.parametrize("backward", [0, 1])
def test_refusals(kw, status, text, backward):
    if kw.get("work") == 0 and not backward:
        kw = dict(kw, N=1)   # (needs a split)
    st, msg = Raw()(backward, kw)
    assert st == status and text in msg, (st, msg)


@pytest.mark.parametrize("backward,kw,text", [
    (0, dict(out=(Raw.Q + 64, *ROW)), "out overlaps q"),
    (0, dict(out=(Raw.V, *ROW)), "out overlaps v"),
    (0, dict(out=(Raw.O, ROW[0], 0, 64)), "overlap each other"),
    (0, dict(lse=Raw.O + 64), "out overlaps lse"),
    (0, dict(lse=Raw.K), "lse overlaps k"),
    (0, dict(N=1, M=4096, bytes=64), "are needed"),
    (0, dict(N=1, M=4096, work=Raw.Q), "work overlaps q"),
    (1, dict(lse=0), "lse is NULL"),
    (1, dict(work=0), "work is NULL"),
    (1, dict(work=Raw.W + 4), "aligned"),
    (1, dict(bytes=8), "are needed"),
    (1, dict(dq=(Raw.Q, *ROW)), "dq overlaps q"),
    (1, dict(dk=(Raw.DQ, *ROW)), "dk overlaps dq"),
    (1, dict(dv=(Raw.DK, *ROW)), "dv overlaps dk"),
    (1, dict(dk=(Raw.O, *ROW)), "dk overlaps out"),
    (1, dict(dv=(Raw.W, *ROW)), "dv overlaps work"),
    (1, dict(work=Raw.G), "work overlaps dout"),
], ids=str)
def test_refusals_of_overlaps(backward, kw, text):
    st, msg = Raw()(backward, kw)
    assert st == INV and text in msg, (st, msg)


@pytest.mark.parametrize("backward,kw,text", [
    (0, dict(q=(Raw.Q + 8, *ROW)), "q is not 16-byte aligned"),
    (0, dict(out=(Raw.V, *ROW)), "out overlaps v"),
    (1, dict(dk=(Raw.DQ, *ROW)), "dk overlaps dq"),
    (1, dict(lse=Raw.DV), "dv overlaps lse"),
], ids=str)
def test_tensors_are_checked_before_the_workspace(backward, kw, text):
    """The size of the workspace depends on the device, which is asked last."""
    st, msg = Raw()(backward, dict(kw, N=1, M=2048, B=1, heads=1, kv=1, work=0))
    assert st == INV and text in msg, (st, msg)


def test_more_workgroups_than_a_launch_holds():
    """A launch counts its threads in 32 bits: 2^24 workgroups of 256 are too many."""
    for B, kv, N in ((1 << 22, 4, 1), (3 << 20, 4, 129)):
        for backward in (0, 1):
            st, msg = Raw()(backward, dict(B=B, heads=kv, kv=kv, N=N, M=1))
            assert st == UNS and "2^24" in msg, (st, msg)
    n = ctypes.c_int64()
    L = hla.lib()
    for M, want in ((1 << 30, UNS), ((1 << 30) - (1 << 16), hla.HLA_OK)):   # keys of the backward only
        assert L.hla_cross_attn_workspace(1, 1, 1, 1, M, 64, hla.HLA_BF16, 1, ctypes.byref(n)) == want
        assert L.hla_cross_attn_workspace(1, 1, 1, 1, M, 64, hla.HLA_BF16, 0, ctypes.byref(n)) == hla.HLA_OK


def test_workspace_sizes():
    n = ctypes.c_int64()
    L = hla.lib()
    assert L.hla_cross_attn_workspace(2, 4, 4, 64, 64, 64, hla.HLA_BF16, 1, ctypes.byref(n)) == hla.HLA_OK
    assert n.value >= 2 * 4 * 64 * 8
    assert L.hla_cross_attn_workspace(2, 4, 3, 64, 64, 64, hla.HLA_BF16, 1, ctypes.byref(n)) == INV
    assert L.hla_cross_attn_workspace(2, 4, 4, 64, 64, 64, hla.HLA_BF16, 0, None) == INV


def test_refusals_of_the_binding():
    x = torch.zeros(1, 1, 2, 32)
    with pytest.raises(hla.HLAError, match="GPU"):
        hla.cross_attn_fwd(x, x, x)
