"""The operators of a transformer block on image tokens, run together as a program
would: Hilbert order, projections, rotary positions of the grid cells, local attention,
cross attention to ragged states, MLP, each with its residual; forward and the whole
chain of gradients.

fp32: against the same block in float64 with torch's autograd. A stage's result is off
by at most (n + 8) 2^-24 of its terms' magnitudes for sums of n <= 160 terms, 1e-5, and
the chain is 14 stages deep with gains near 1, so 2e-4 in the 2-norm bounds it.
bf16: against the fp32 run on the same (bf16) inputs. Each of the 14 stages rounds its
operands and result to half a step, 2^-8, at most twice; errors of independent roundings
add in squares: 2 sqrt(14) 2^-8 = 3e-2 in the 2-norm."""
import math

import pytest
import torch

import paper_2511_05832_amd as hla

H, W, B, HEADS, D, KV, M, CE, FF = 12, 20, 3, 4, 32, 2, 23, 48, 160
C, N = HEADS * D, H * W
PATTERN = ("hilbert_slide", H, W, 17, 0)
NAMES = ("x", "states", "w_qkv", "w_o", "w_q", "w_kv", "w_c", "w1", "b1", "w2", "b2")


def tensors(dtype, seed=0):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g) * std).to(torch.bfloat16).to(dtype)
    return dict(x=normal(B, N, C), states=normal(B, M, CE), w_qkv=normal(3 * C, C, std=C ** -0.5),
                w_o=normal(C, C, std=C ** -0.5), w_q=normal(C, C, std=C ** -0.5),
                w_kv=normal(2 * KV * D, CE, std=CE ** -0.5), w_c=normal(C, C, std=C ** -0.5),
                w1=normal(FF, C, std=C ** -0.5), b1=normal(FF, std=0.1), w2=normal(C, FF, std=FF ** -0.5),
                b2=normal(C, std=0.1), dy=normal(B, N, C))


LENGTHS = [M, 0, 9]


def heads_of(t, n):
    """[B, N, n * D] -> [B, n, N, D], a view."""
    return t.view(B, -1, n, D).transpose(1, 2)


def from_host():
    """What a program copies from the host once: frequencies, lengths."""
    return hla.rope_freqs(D // 4, base=100.0)[0], torch.tensor(LENGTHS, dtype=torch.int32, device="cuda")


def run(t, host=None):
    """The block and its gradients by the package's operators."""
    t = {n: v.cuda() for n, v in t.items()}
    freqs, lengths = host or from_host()
    order, _ = hla.hilbert_perm(H, W)
    mask = hla.build_block_mask(PATTERN, 64, 64, columns=True)
    rot = dict(pos=order, grid_w=W)
    # local attention, in Hilbert order
    xh = hla.gather(t["x"], order)
    qkv = hla.linear(xh, t["w_qkv"]).view(B, N, 3, HEADS, D)
    q, k = hla.rope(qkv[:, :, 0].transpose(1, 2), freqs, k=qkv[:, :, 1].transpose(1, 2), **rot)
    q, k, v = (x.contiguous() for x in (q, k, qkv[:, :, 2].transpose(1, 2)))
    o, lse = hla.attn_fwd(q, k, v, mask)
    om = o.transpose(1, 2).reshape(B, N, C)
    h1 = hla.linear(om, t["w_o"], residual=xh)
    # cross attention to the states
    qc = heads_of(hla.linear(h1, t["w_q"]), HEADS)
    kv = hla.linear(t["states"], t["w_kv"]).view(B, M, 2, KV, D)
    kc, vc = kv[:, :, 0].transpose(1, 2), kv[:, :, 1].transpose(1, 2)
    oc, lsec = hla.cross_attn_fwd(qc, kc, vc, lengths)
    ocm = oc.transpose(1, 2).reshape(B, N, C)
    h2 = hla.linear(ocm, t["w_c"], residual=h1)
    # MLP
    a, pre = hla.linear(h2, t["w1"], t["b1"], act="gelu", with_pre=True)
    y = hla.scatter(hla.linear(a, t["w2"], t["b2"], residual=h2), order)

    g = {}
    dy = hla.gather(t["dy"], order)
    da, g["w2"], g["b2"] = hla.linear_bwd(a, t["w2"], dy, with_bias=True)
    d, g["w1"], g["b1"] = hla.linear_bwd(h2, t["w1"], da, pre, act="gelu", with_bias=True)
    dh2 = dy + d
    docm, g["w_c"], _ = hla.linear_bwd(ocm, t["w_c"], dh2)
    dkv = torch.empty_like(kv)
    dqc, _, _ = hla.cross_attn_bwd(qc, kc, vc, oc, heads_of(docm, HEADS), lsec, lengths,
                                   dk=dkv[:, :, 0].transpose(1, 2), dv=dkv[:, :, 1].transpose(1, 2))
    g["states"], g["w_kv"], _ = hla.linear_bwd(t["states"], t["w_kv"], dkv.view(B, M, -1))
    d, g["w_q"], _ = hla.linear_bwd(h1, t["w_q"], dqc.transpose(1, 2).reshape(B, N, C))
    dh1 = dh2 + d
    dom, g["w_o"], _ = hla.linear_bwd(om, t["w_o"], dh1)
    dq, dk, dv = hla.attn_bwd(q, k, v, o, heads_of(dom, HEADS).contiguous(), lse, mask)
    dqkv = torch.empty(B, N, 3, HEADS, D, dtype=dy.dtype, device="cuda")
    dqkv[:, :, 2] = dv.transpose(1, 2)
    hla.rope(dq, freqs, k=dk, inverse=True, q_out=dqkv[:, :, 0].transpose(1, 2),
             k_out=dqkv[:, :, 1].transpose(1, 2), **rot)
    d, g["w_qkv"], _ = hla.linear_bwd(xh, t["w_qkv"], dqkv.view(B, N, 3 * C))
    g["x"] = hla.scatter(dh1 + d, order)
    return y, g


def reference(t):
    """The block in float64, tokens in grid order, and autograd's gradients."""
    from oracle import hilbert
    p = {n: t[n].double().requires_grad_(True) for n in NAMES}
    rank = torch.from_numpy(hilbert.hilbert_rank(H, W).copy()).long()
    pos = torch.arange(N)
    freqs = 100.0 ** (-torch.arange(D // 4, dtype=torch.float64) / (D // 4))

    def turn(x):   # [B, h, N, D]: rows turn the first half, columns the second
        parts = []
        for axis, c in enumerate((pos // W, pos % W)):
            a = c[:, None].double() * freqs
            u = x[..., axis * D // 2:(axis + 1) * D // 2]
            u1, u2 = u[..., :D // 4], u[..., D // 4:]
            parts += [u1 * a.cos() - u2 * a.sin(), u2 * a.cos() + u1 * a.sin()]
        return torch.cat(parts, dim=-1)

    def attend(q, k, v, seen):
        s = torch.where(seen, q @ k.transpose(-1, -2) / math.sqrt(D), -math.inf)
        top = s.amax(-1, keepdim=True).detach()
        e = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
        total = e.sum(-1, keepdim=True)
        return (e / torch.where(total > 0, total, 1.0)) @ v

    qkv = (p["x"] @ p["w_qkv"].T).view(B, N, 3, HEADS, D)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    near = (rank[:, None] - rank[None, :]).abs() <= PATTERN[3]
    o = attend(turn(q), turn(k), v, near)
    h1 = o.transpose(1, 2).reshape(B, N, C) @ p["w_o"].T + p["x"]
    qc = heads_of(h1 @ p["w_q"].T, HEADS)
    kv = (p["states"] @ p["w_kv"].T).view(B, M, 2, KV, D)
    kc, vc = (kv[:, :, i].transpose(1, 2).repeat_interleave(HEADS // KV, dim=1) for i in range(2))
    seen = torch.arange(M)[None, None, None] < torch.tensor(LENGTHS)[:, None, None, None]
    oc = attend(qc, kc, vc, seen)
    h2 = oc.transpose(1, 2).reshape(B, N, C) @ p["w_c"].T + h1
    z = h2 @ p["w1"].T + p["b1"]
    y = (z * 0.5 * torch.erfc(-z / math.sqrt(2))) @ p["w2"].T + p["b2"] + h2
    y.backward(t["dy"].double())
    return y.detach(), {n: p[n].grad for n in NAMES}


def far(a, b):
    b = b.double().cpu()
    return float((a.double().cpu() - b).norm() / b.norm())


@pytest.mark.gpu
def test_block_and_gradients_fp32():
    t = tensors(torch.float32)
    y, g = run(t)
    ry, rg = reference(t)
    offs = {"y": far(y, ry), **{n: far(g[n], rg[n]) for n in NAMES}}
    print(offs)
    assert all(v < 2e-4 for v in offs.values()), offs
    # (a batch element without states gets no gradient on them)
    assert bool((g["states"][1] == 0).all())


@pytest.mark.gpu
def test_block_and_gradients_bf16():
    y, g = run(tensors(torch.bfloat16))
    ry, rg = run(tensors(torch.float32))
    offs = {"y": far(y, ry), **{n: far(g[n], rg[n]) for n in NAMES}}
    print(offs)
    assert all(v < 3e-2 for v in offs.values()), offs


@pytest.mark.gpu
def test_block_replayed_from_a_graph():
    t = {n: v.cuda() for n, v in tensors(torch.bfloat16).items()}
    host = from_host()
    run(t, host)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, g = run(t, host)
    for r in range(3):
        t["x"].copy_(tensors(torch.bfloat16, seed=r)["x"])
        graph.replay()
        torch.cuda.synchronize()
        ey, eg = run(t, host)
        assert torch.equal(y, ey) and all(torch.equal(g[n], eg[n]) for n in NAMES), r
