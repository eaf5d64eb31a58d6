"""What the transformer-block operators around the local attention are timed on:
rotary positions (``rope``), cross attention to an encoder's states
(``cross_attn_fwd`` / ``cross_attn_bwd``) and the token-wise linear layer with bias,
activation and residual (``linear`` / ``linear_bwd``).

A case is one pass through one operator. ``run`` computes it in plain form from
elementary torch operations, in float32 (angles in float64), rounded once at the end;
with ``own`` set it makes the calls of this package instead.

    rope    q and k rotated by their positions (inverse: the gradient's way back)
    cross   attention forward, with ``train`` forward and backward
    linear  the layer forward, with ``train`` forward and backward
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ES = {"bf16": 2, "f32": 4}


def _rope(B, heads, kv_heads, N, d, rot, dtype, interleaved=False, grid_w=0, per_batch=False,
          inverse=False, base=10000.0, factor=1.0, far=0, name=None):
    c = dict(op="rope", B=B, heads=heads, kv_heads=kv_heads, N=N, d=d, rot=rot, dtype=dtype,
             interleaved=interleaved, grid_w=grid_w, per_batch=per_batch, inverse=inverse,
             base=base, factor=factor, far=far)
    if name:
        c["name"] = name
    return c


def _cross(B, heads, kv_heads, N, M, d, dtype, ragged=True, train=False, packed=False, name=None):
    c = dict(op="cross", B=B, heads=heads, kv_heads=kv_heads, N=N, M=M, d=d, dtype=dtype,
             ragged=ragged, train=train, packed=packed)
    if name:
        c["name"] = name
    return c


def _linear(T, K, F, dtype, act, bias=True, residual=False, train=False, name=None):
    c = dict(op="linear", T=T, K=K, F=F, dtype=dtype, act=act, bias=bias, residual=residual,
             train=train)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Serving, one new token per sequence of a long context: every batch element at
        # its own far position, fewer key heads than query heads. Latency.
        _rope(16, 16, 4, 1, 64, 64, "bf16", per_batch=True, far=131072, factor=8.0,
              name="rope_token"),
        # The 64x64 image layer (6 heads of 32, batch 16): row and column rotations of the
        # tokens in their reordered sequence.
        _rope(16, 6, 6, 4096, 32, 32, "bf16", interleaved=True, grid_w=64, name="rope_grid_64"),
        # Training in float32 at the longest sequence (256x256): the gradient's rotation of
        # half of each head, shared key heads.
        _rope(1, 8, 2, 65536, 64, 32, "f32", inverse=True, base=500000.0,
              name="rope_grad_f32_long"),
        # A decoder's single token against the states of a long input, ragged batch,
        # shared key heads: the states are read once.
        _cross(16, 16, 4, 1, 4096, 64, "bf16", name="cross_token"),
        # Image tokens of the 64x64 layer looking at a short text; q, k, v as the
        # projections leave them (token rows, heads inside), k and v in one tensor.
        _cross(16, 6, 6, 4096, 77, 32, "bf16", packed=True, name="cross_text_64"),
        # Training a 128x128 feature map on short texts, some of them empty.
        _cross(4, 8, 8, 16384, 77, 64, "bf16", train=True, name="cross_text_128_train"),
        # Training on another image's states: both sides long, shared key heads.
        _cross(2, 8, 2, 4096, 4096, 64, "bf16", train=True, name="cross_long_train"),
        # Training in float32 at a modest size with an odd number of states.
        _cross(2, 4, 4, 1024, 257, 32, "f32", train=True, name="cross_f32_train"),
        # An MLP's first layer for a few tokens: the weights' bytes.
        _linear(4, 2048, 8192, "bf16", "gelu_tanh", name="linear_token"),
        # The first MLP layer of the 64x64 image layer, whole batch: 192 -> 768.
        _linear(65536, 192, 768, "bf16", "gelu", name="linear_mlp_64"),
        # Training a wide layer: matrix-core work.
        _linear(16384, 1024, 4096, "bf16", "gelu", residual=True, train=True,
                name="linear_wide_train"),
        # Training in float32.
        _linear(4096, 192, 768, "f32", "silu", residual=True, train=True,
                name="linear_f32_train"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _draw_rope(rng):
    dtype = rng.choice(["bf16", "bf16", "f32"])
    kv = rng.choice([1, 2, 3, 4])
    heads = kv * rng.choice([1, 2, 4])
    B, d = _log(rng, 1, 16), rng.choice([32, 64, 80, 96, 128])
    room = 80_000_000 // (B * (heads + kv) * d * ES[dtype])
    N = _log(rng, 1, max(1, min(65536, room)))
    W = 0
    if rng.random() < 0.5:
        W = _log(rng, 1, N)
        N = W * max(1, N // W)
    rot = d if rng.random() < 0.5 else 4 * rng.randint(1, d // 4)
    return _rope(B, heads, kv, N, d, rot, dtype, interleaved=rng.random() < 0.5, grid_w=W,
                 per_batch=rng.random() < 0.3, inverse=rng.random() < 0.4,
                 base=rng.choice([10000.0, 500000.0]), factor=rng.choice([1.0, 4.0]),
                 far=0 if W else rng.choice([0, 0, 100000]))


def _draw_cross(rng):
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([32, 64])
    kv = rng.choice([1, 2, 4, 6])
    heads = kv * rng.choice([1, 1, 2, 4])
    B, train = _log(rng, 1, 16), rng.random() < 0.5
    # at most the work of the largest listed case (float32: of a fiftieth of it)
    room = 2 ** 28 // (1 if dtype == "bf16" else 50) // (B * heads) // (d // 32)
    M = _log(rng, 1, min(8192, max(1, room)))
    N = _log(rng, 1, max(1, min(16384, room // M)))
    return _cross(B, heads, kv, N, M, d, dtype, ragged=rng.random() < 0.7, train=train,
                  packed=rng.random() < 0.4)


def _draw_linear(rng):
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    K, F = 8 * _log(rng, 4, 512), 8 * _log(rng, 4, 512)
    room = 2 ** (36 if dtype == "bf16" else 31) // (K * F)
    T = _log(rng, 1, max(1, min(65536, room)))
    return _linear(T, K, F, dtype, rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                   bias=rng.random() < 0.8, residual=rng.random() < 0.4,
                   train=rng.random() < 0.5)


def draw(rng):
    return rng.choice([_draw_rope, _draw_cross, _draw_linear])(rng)


# ---------------------------------------------------------------------------
# Inputs

class _State:
    pass


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DT[c["dtype"]]

    def normal(*shape, std=1.0):
        x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
        return (x * std if std != 1.0 else x).to(dt)

    s = _State()
    s.c = c
    if c["op"] == "rope":
        B, N, d = c["B"], c["N"], c["d"]
        s.q = normal(B, c["heads"], N, d)
        s.k = normal(B, c["kv_heads"], N, d)
        # one frequency per rotated pair and axis; a longer context than the one trained
        # on divides them by its factor
        pairs = c["rot"] // (4 if c["grid_w"] else 2)
        i = torch.arange(pairs, device="cuda", dtype=torch.float64)
        s.freqs = c["base"] ** (-i / pairs) / c["factor"]
        rows = B if c["per_batch"] else 1
        if c["grid_w"]:     # cells of the grid, in the order of the sequence
            s.pos = torch.stack([torch.randperm(N, generator=g, device="cuda") for _ in range(rows)])
        else:
            first = torch.randint(0, c["far"] + 1, (rows, 1), generator=g, device="cuda")
            s.pos = first + torch.arange(N, device="cuda")
        s.pos = s.pos.to(torch.int32)
        if not c["per_batch"]:
            s.pos = s.pos[0]
    elif c["op"] == "cross":
        B, N, M, d, h, kv = c["B"], c["N"], c["M"], c["d"], c["heads"], c["kv_heads"]
        if c["packed"]:     # as token-wise projections leave them
            s.q = normal(B, N, h, d).transpose(1, 2)
            states = normal(B, M, 2, kv, d)
            s.k, s.v = states[:, :, 0].transpose(1, 2), states[:, :, 1].transpose(1, 2)
        else:
            s.q, s.k, s.v = normal(B, h, N, d), normal(B, kv, M, d), normal(B, kv, M, d)
        s.lengths = None
        if c["ragged"]:     # from nothing to all of the states, the longest all of them
            s.lengths = torch.randint(0, M + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            if N == 1:      # a decoder's inputs: the longer half
                s.lengths = (s.lengths + M + 1) // 2
            s.lengths[0] = M
        if c["train"]:
            s.dout = normal(B, h, N, d)
    else:
        T, K, F = c["T"], c["K"], c["F"]
        s.x = normal(T, K)
        s.w = normal(F, K, std=K ** -0.5)
        s.bias = normal(F, std=0.1) if c["bias"] else None
        s.residual = normal(T, F) if c["residual"] else None
        if c["train"]:
            s.dy = normal(T, F)
    return s


# ---------------------------------------------------------------------------
# Plain forms

def _angles(pos, freqs, grid_w):
    """float64 [1 or B, 1, N, pairs] (grid: the rows' pairs, then the columns')."""
    p = pos.to(torch.float64)
    p = p.reshape(-1, 1, p.shape[-1], 1)
    if not grid_w:
        return p * freqs
    r = torch.floor(p / grid_w)
    return torch.cat([r * freqs, (p - r * grid_w) * freqs], dim=-1)


def _pairs_of(x, axes, interleaved):
    """The two members of every pair of x [..., rot], each [..., axes * pairs]."""
    y = x.reshape(*x.shape[:-1], axes, -1)
    if interleaved:
        a, b = y[..., 0::2], y[..., 1::2]
    else:
        n = y.shape[-1] // 2
        a, b = y[..., :n], y[..., n:]
    return a.flatten(-2), b.flatten(-2)


def _pairs_back(a, b, axes, interleaved):
    a = a.reshape(*a.shape[:-1], axes, -1)
    b = b.reshape(*b.shape[:-1], axes, -1)
    if interleaved:
        return torch.stack([a, b], dim=-1).flatten(-3)
    return torch.cat([a, b], dim=-1).flatten(-2)


def _plain_rope(s):
    c = s.c
    ang = _angles(s.pos, s.freqs, c["grid_w"])
    cos, sin = torch.cos(ang).float(), torch.sin(ang).float()
    if c["inverse"]:
        sin = -sin
    axes = 2 if c["grid_w"] else 1

    def turn(x):
        y = x.float()
        a, b = _pairs_of(y[..., :c["rot"]], axes, c["interleaved"])
        z = _pairs_back(a * cos - b * sin, b * cos + a * sin, axes, c["interleaved"])
        return torch.cat([z, y[..., c["rot"]:]], dim=-1).to(x.dtype)

    return {"q": turn(s.q), "k": turn(s.k)}


def _plain_cross(s):
    c = s.c
    B, h, kv, M = c["B"], c["heads"], c["kv_heads"], c["M"]
    scale = c["d"] ** -0.5
    q, k, v = s.q.float().contiguous(), s.k.float(), s.v.float()
    g = h // kv
    kr, vr = k.repeat_interleave(g, dim=1), v.repeat_interleave(g, dim=1)
    S = torch.matmul(q, kr.transpose(-1, -2).contiguous()) * scale
    if s.lengths is not None:
        seen = torch.arange(M, device=q.device) < s.lengths.view(B, 1, 1, 1)
        S = torch.where(seen, S, -math.inf)
    top = S.amax(dim=-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    P = torch.exp(S - top)
    total = P.sum(dim=-1, keepdim=True)
    lse = top + torch.log(total)
    P = P / torch.where(total > 0, total, 1.0)
    out = torch.matmul(P, vr)
    r = {"out": out.to(s.q.dtype), "lse": lse.squeeze(-1)}
    if c["train"]:
        do = s.dout.float()
        dP = torch.matmul(do, vr.transpose(-1, -2).contiguous())
        dS = P * (dP - (do * out).sum(dim=-1, keepdim=True))
        dq = torch.matmul(dS, kr) * scale
        dk = torch.matmul(dS.transpose(-1, -2).contiguous(), q) * scale
        dv = torch.matmul(P.transpose(-1, -2).contiguous(), do)
        r["dq"] = dq.to(s.q.dtype)
        r["dk"] = dk.reshape(B, kv, g, M, -1).sum(dim=2).to(s.q.dtype)
        r["dv"] = dv.reshape(B, kv, g, M, -1).sum(dim=2).to(s.q.dtype)
    return r


def _act(z, kind):
    """The activation and its derivative, in z's type."""
    if kind == "none":
        return z, torch.ones_like(z)
    if kind == "relu":
        on = (z > 0).to(z.dtype)
        return z * on, on
    if kind == "silu":
        e = 1 / (1 + torch.exp(-z))
        return z * e, e * (1 + z * (1 - e))
    if kind == "gelu":
        cdf = 0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    u = math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)     # gelu_tanh
    t = torch.tanh(u)
    du = math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * du


def _linear_in(s, dt):
    c = s.c
    x, w = s.x.to(dt), s.w.to(dt)
    z = x @ w.T
    if s.bias is not None:
        z = z + s.bias.to(dt)
    a, da = _act(z, c["act"])
    y = a if s.residual is None else a + s.residual.to(dt)
    r = {"y": y}
    if c["train"]:
        dz = s.dy.to(dt) * da
        r["dx"] = dz @ w
        r["dw"] = dz.T @ x
        if s.bias is not None:
            r["db"] = dz.sum(dim=0)
    return r


def _plain_linear(s):
    return {n: t.to(s.x.dtype) for n, t in _linear_in(s, torch.float32).items()}


# ---------------------------------------------------------------------------
# This package's calls

def _own_rope(s):
    import paper_2511_05832_amd as hla
    c = s.c
    q, k = hla.rope(s.q, s.freqs, k=s.k, pos=s.pos, grid_w=c["grid_w"],
                    interleaved=c["interleaved"], inverse=c["inverse"])
    return {"q": q, "k": k}


def _own_cross(s):
    import paper_2511_05832_amd as hla
    out, lse = hla.cross_attn_fwd(s.q, s.k, s.v, lengths=s.lengths)
    r = {"out": out, "lse": lse}
    if s.c["train"]:
        r["dq"], r["dk"], r["dv"] = hla.cross_attn_bwd(s.q, s.k, s.v, out, s.dout, lse,
                                                       lengths=s.lengths)
    return r


def _own_linear(s):
    import paper_2511_05832_amd as hla
    c = s.c
    if not c["train"]:
        return {"y": hla.linear(s.x, s.w, s.bias, act=c["act"], residual=s.residual)}
    y, pre = hla.linear(s.x, s.w, s.bias, act=c["act"], residual=s.residual, with_pre=True)
    dx, dw, db = hla.linear_bwd(s.x, s.w, s.dy, pre=pre, act=c["act"],
                                with_bias=s.bias is not None)
    r = {"y": y, "dx": dx, "dw": dw}
    if db is not None:
        r["db"] = db
    return r


def run(state):
    op = state.c["op"]
    if own:
        return {"rope": _own_rope, "cross": _own_cross, "linear": _own_linear}[op](state)
    return {"rope": _plain_rope, "cross": _plain_cross, "linear": _plain_linear}[op](state)


# ---------------------------------------------------------------------------
# Costs and values from the definitions

def work(case):
    c = case
    es = ES[c["dtype"]]
    if c["op"] == "rope":
        n = c["B"] * (c["heads"] + c["kv_heads"]) * c["N"]
        return {"bytes": 2 * n * c["d"] * es + 4 * c["N"] * (c["B"] if c["per_batch"] else 1),
                "flops": 3 * n * c["rot"]}
    if c["op"] == "cross":
        B, N, M, d, h, kv = c["B"], c["N"], c["M"], c["d"], c["heads"], c["kv_heads"]
        # ragged: the longest batch element sees all, the others half on average (a
        # decoder's single token: three quarters)
        seen = B * M
        if c["ragged"]:
            seen = int(M * (1 + (B - 1) * (0.75 if N == 1 else 0.5)))
        rows, states = B * h * N * d * es, seen * kv * d * es
        byts, flops = 2 * rows + 2 * states + 4 * B * h * N, 4 * seen * h * N * d
        if c["train"]:
            # the backward reads q, out, dout, lse, k, v and writes dq and all of dk, dv
            byts += 4 * rows + 2 * states + 4 * B * h * N + 2 * B * M * kv * d * es
            flops += 10 * seen * h * N * d
        return {"bytes": byts, "flops": flops}
    T, K, F = c["T"], c["K"], c["F"]
    byts = es * (T * K + F * K + T * F * (2 if c["residual"] else 1))
    flops = 2 * T * K * F
    if c["train"]:
        # forward: z stored as well; backward: x, w, z, dy read, dx, dw written
        kept = c["act"] != "none"
        byts += es * (2 * T * K + 2 * F * K + T * F * (3 if kept else 1))
        flops += 4 * T * K * F
    return {"bytes": byts, "flops": flops}


def _exact_rope(s):
    c = s.c
    d, rot = c["d"], c["rot"]
    axes = 2 if c["grid_w"] else 1
    P = rot // (2 * axes)
    # feature e of the rotated part: its axis, pair, and whether it is the pair's second
    e = torch.arange(rot, device="cuda")
    axis, within = e // (2 * P), e % (2 * P)
    if c["interleaved"]:
        pair, second = within // 2, within % 2 == 1
        other = torch.where(second, e - 1, e + 1)
    else:
        pair, second = within % P, within >= P
        other = torch.where(second, e - P, e + P)
    pos = s.pos.reshape(-1, c["N"]).long()
    coord = torch.stack([pos // c["grid_w"], pos % c["grid_w"]]) if axes == 2 else pos[None]
    ang = coord[axis].permute(1, 2, 0).double() * s.freqs[pair]          # [rows, N, rot]
    cos = torch.cos(ang)[:, None]
    sin = (torch.sin(ang) * torch.where(second, 1.0, -1.0).double() * (-1 if c["inverse"] else 1))[:, None]

    def turn(x):
        y = x.double().clone()
        r = y[..., :rot]
        y[..., :rot] = r * cos + r[..., other] * sin
        return y

    return {"q": turn(s.q), "k": turn(s.k)}


def _exact_cross(s):
    c = s.c
    B, h, kv, N, M, d = c["B"], c["heads"], c["kv_heads"], c["N"], c["M"], c["d"]
    g, scale = h // kv, 1.0 / math.sqrt(d)
    q = s.q.double().reshape(B, kv, g * N, d)        # the rows that share a key head
    k, v = s.k.double().contiguous(), s.v.double().contiguous()
    r = {"out": torch.zeros(B, kv, g * N, d, device="cuda", dtype=torch.float64),
         "lse": torch.full((B, kv, g * N), -math.inf, device="cuda", dtype=torch.float64)}
    if c["train"]:
        do = s.dout.double().reshape(B, kv, g * N, d)
        r.update(dq=torch.zeros_like(q), dk=torch.zeros_like(k), dv=torch.zeros_like(v))
    for b in range(B):
        n = M if s.lengths is None else int(s.lengths[b])
        if n == 0:
            continue
        for j in range(kv):
            K, V = k[b, j, :n], v[b, j, :n]
            S = (q[b, j] @ K.T.contiguous()) * scale
            lse = torch.logsumexp(S, dim=1)
            P = torch.exp(S - lse[:, None])
            r["lse"][b, j], r["out"][b, j] = lse, P @ V
            if c["train"]:
                D = do[b, j]
                dP = D @ V.T.contiguous()
                dS = P * (dP - (P * dP).sum(dim=1, keepdim=True))
                r["dq"][b, j] = (dS @ K) * scale
                r["dk"][b, j, :n] = (dS.T.contiguous() @ q[b, j]) * scale
                r["dv"][b, j, :n] = P.T.contiguous() @ D
    for n in ("out", "dq"):
        if n in r:
            r[n] = r[n].reshape(B, h, N, d)
    r["lse"] = r["lse"].reshape(B, h, N)
    return r


def _exact_linear(s):
    c = s.c
    x, w = s.x.double(), s.w.double()
    z = torch.nn.functional.linear(x, w, None if s.bias is None else s.bias.double())
    z.requires_grad_(True)
    with torch.enable_grad():
        a = {"none": lambda t: t * 1, "relu": torch.relu, "silu": torch.nn.functional.silu,
             "gelu": torch.nn.functional.gelu,
             "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[c["act"]](z)
        r = {"y": a.detach() if s.residual is None else a.detach() + s.residual.double()}
        if c["train"]:
            dz, = torch.autograd.grad(a, z, s.dy.double())
            r["dx"], r["dw"] = dz @ w, dz.T.contiguous() @ x
            if s.bias is not None:
                r["db"] = dz.sum(dim=0)
    return r


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "cross": _exact_cross, "linear": _exact_linear}[case["op"]](s)
