"""What the performance of the operators around the quantized linear layer is measured on.

``fused``: the online linear (per-token INT8 activations, dual-scale INT8 or INT4 weights) whose epilogue applies the
activation, the gate of each group of tokens and the residual stream, ``Y = R + g * act(x W^T + b)``.
``heads``: RMS norm of queries and keys (for each head, or over a token's whole row) and the rotation by the token's positions
along up to three axes (time, height, width), in one pass over both.

Shapes are those of ``workloads.py`` (hidden 1536 / FFN 8960 with 12 heads of 128, hidden 5120 / FFN 13824 with 40, 4680 tokens
per chunk of three latent frames of 30 x 52, 32760 per clip) and ragged ones.  Activations are N(0, 1) with the outlier channels
fifteen times larger; weights are drawn as codes with their scales, the outlier columns' twenty-five times larger.
"""
import math

import torch

own = False

GROUPS_OF_TOKENS = 1560          # tokens of one latent frame: they share a gate
EPS = 1e-6
THETA = 10000.0


def listed():
    return [
        # attention's output projection of one chunk onto the residual stream, a gate for each of its three frames
        dict(name="out-proj", op="fused", M=4680, K=1536, N=1536, c=16, x="bf16", y="bf16", bits=8, act=False, residual=True, gates=3),
        # FFN down-projection of one chunk onto a residual stream that is kept in fp32
        dict(name="ffn-down", op="fused", M=4680, K=8960, N=1536, c=64, x="bf16", y="f32", bits=8, act=False, residual=True, gates=3),
        # FFN up-projection of one chunk with GELU, for a down-projection that quantizes by token
        dict(name="ffn-up-gelu", op="fused", M=4680, K=1536, N=8960, c=16, x="bf16", y="bf16", bits=8, act=True, residual=False, gates=0),
        # the larger model's FFN up-projection with its widest outlier block: the largest product
        dict(name="ffn-up-large", op="fused", M=4680, K=5120, N=13824, c=128, x="bf16", y="bf16", bits=8, act=True, residual=False, gates=0),
        # a single token through an INT4 down-projection: the weights are all the bytes
        dict(name="one-token-w4", op="fused", M=1, K=8960, N=1536, c=32, x="bf16", y="bf16", bits=4, act=False, residual=True, gates=1),
        # nothing divides anything, an outlier block wider than 128, all three endings, fp32
        dict(name="fused-ragged", op="fused", M=2251, K=2360, N=2252, c=150, x="f32", y="f32", bits=8, act=True, residual=True, gates=5),
        # queries and keys of one chunk: norm for each head, three axes
        dict(name="heads-chunk", op="heads", M=4680, hq=12, hk=12, d=128, axes="44,42,42", inter=True, norm="head", x="bf16", start=18, heads_first=False),
        # queries and keys of a whole clip, normed over the whole row: the most bytes
        dict(name="heads-clip", op="heads", M=32760, hq=12, hk=12, d=128, axes="44,42,42", inter=True, norm="row", x="bf16", start=0, heads_first=False),
        # the larger model's queries with shared keys in fp32, rotated in halves, written heads first for attention
        dict(name="heads-large", op="heads", M=4680, hq=40, hk=8, d=128, axes="44,42,42", inter=False, norm="head", x="f32", start=0, heads_first=True),
        # one frame, the rotation alone
        dict(name="rotation-frame", op="heads", M=1560, hq=12, hk=12, d=128, axes="44,42,42", inter=True, norm="none", x="bf16", start=500, heads_first=False),
        # a single token with one axis: launch and host work count
        dict(name="heads-one", op="heads", M=1, hq=12, hk=12, d=128, axes="128", inter=False, norm="head", x="bf16", start=30000, heads_first=False),
        # an odd head size of which part is rotated, shared keys, odd counts
        dict(name="heads-ragged", op="heads", M=1027, hq=10, hk=3, d=100, axes="20,22,18", inter=True, norm="head", x="f32", start=7, heads_first=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A channel count: half of them multiples of 64 as model widths are, a quarter multiples of 8, a quarter any."""
    v = _log_uniform(rng, lo, hi)
    step = rng.choice((64, 64, 8, 1))
    return max(step, v // step * step)


def _draw_fused(rng):
    M, K, N = _log_uniform(rng, 1, 4680), _width(rng, 64, 13824), _width(rng, 64, 13824)
    # the odd shapes run on slower kernels: a drawn case stays below the largest listed one in time too
    if M * K * N > 4680 * 5120 * 13824 // (1 if N % 8 == 0 and K % 4 == 0 else 8):
        return _draw_fused(rng)
    residual = rng.random() < 0.6
    return dict(op="fused", M=M, K=K, N=N, c=rng.choice((0, rng.randint(1, max(1, min(K // 60, 200))))), x=rng.choice(("f32", "bf16")),
                y=rng.choice(("bf16", "bf16", "f32")), bits=rng.choice((8, 8, 4)), act=not residual or rng.random() < 0.3, residual=residual,
                gates=rng.choice((0, 1, rng.randint(1, 6))) if residual else rng.choice((0, 0, 1)))


def _draw_heads(rng):
    d = rng.choice((64, 128, 128, 256, 8 * rng.randint(4, 32), rng.randint(16, 256)))
    hq = _log_uniform(rng, 1, 40)
    hk = rng.choice((hq, max(1, hq // rng.choice((2, 4, 5, 8)))))
    n_axes = rng.choice((1, 2, 3, 3))
    pairs = max(n_axes, rng.choice((d // 2, d // 2, d // 4)))
    cut = pairs // n_axes
    widths = [2 * cut] * (n_axes - 1) + [2 * (pairs - cut * (n_axes - 1))]
    most = 32760 * 24 * 128 // ((hq + hk) * d * 4)
    return dict(op="heads", M=_log_uniform(rng, 1, min(32760, most)), hq=hq, hk=hk, d=d, axes=",".join(map(str, widths)), inter=rng.random() < 0.5,
                norm=rng.choice(("head", "head", "row", "none")), x=rng.choice(("bf16", "bf16", "f32")), start=rng.choice((0, _log_uniform(rng, 1, 1000000))),
                heads_first=rng.random() < 0.3)


def draw(rng):
    return _draw_fused(rng) if rng.random() < 0.5 else _draw_heads(rng)


# ------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _outliers(case):
    """Channels of the outlier block: the planted ones, filled up to a multiple of 32."""
    return min(case["K"], (case["c"] + 31) // 32 * 32)


def _packed(codes, K_o, bits):
    """The layer's packed codes, [outlier | pad to 32 | normal | pad to 128] along K, two INT4 codes to a byte."""
    N, K = codes.shape
    off = (K_o + 31) // 32 * 32
    kp = (off + K - K_o + 127) // 128 * 128
    P = torch.zeros((N, kp + 128), dtype=torch.int8, device="cuda")
    P[:, :K_o] = codes[:, :K_o]
    P[:, off:off + K - K_o] = codes[:, K_o:]
    if bits == 8:
        return P
    g = (P.view(N, -1, 4, 4) & 15).to(torch.uint8)
    return torch.stack([g[:, :, 0] | (g[:, :, 1] << 4), g[:, :, 2] | (g[:, :, 3] << 4)], dim=2).reshape(N, -1).contiguous()


def _prepare_fused(case, seed):
    gen = _generator(seed)
    M, K, N, K_o = case["M"], case["K"], case["N"], _outliers(case)
    qmax = 127 if case["bits"] == 8 else 7
    order = torch.randperm(K, generator=gen, device="cuda")
    out, rest = order[:K_o].sort().values, order[K_o:].sort().values
    codes = (torch.randn((N, K), generator=gen, device="cuda") * (qmax / 3.5)).round_().clamp_(-qmax, qmax).to(torch.int8)
    X = torch.randn((M, K), generator=gen, device="cuda")
    X[:, out[:case["c"]]] *= 15.0
    spread = torch.rand((2, N), generator=gen, device="cuda") * 0.4 + 0.8
    y = _dtype(case["y"])
    st = dict(case=case, X=X.to(_dtype(case["x"])), codes=codes, Wq=_packed(codes, K_o, case["bits"]), perm=torch.cat([out, rest]).to(torch.int32),
              s_n=0.07 / qmax * spread[0], s_o=(1.75 / qmax if K_o else 0.0) * spread[1], bias=torch.randn(N, generator=gen, device="cuda") * 0.01,
              gate=None, rows=None, residual=None)
    if case["gates"]:
        st["gate"] = torch.randn((case["gates"], N), generator=gen, device="cuda") * 0.3
        st["rows"] = -(-M // case["gates"])                  # the last group may be shorter
    if case["residual"]:
        st["residual"] = (torch.randn((M, N), generator=gen, device="cuda") * 2.0).to(y)
    return st


def _axes(case):
    return tuple(int(a) for a in case["axes"].split(","))


def _frequencies(axes):
    return torch.cat([THETA ** (-torch.arange(0, a, 2, dtype=torch.float64, device="cuda") / a) for a in axes])


def _positions(case):
    """Position along each axis of the tokens of consecutive frames of 30 x 52 (two axes: of one image; one: of a text)."""
    m, n = torch.arange(case["M"], device="cuda"), len(_axes(case))
    if n == 1:
        p = [m + case["start"]]
    elif n == 2:
        p = [m // 52 + case["start"], m % 52]
    else:
        p = [m // GROUPS_OF_TOKENS + case["start"], m // 52 % 30, m % 52]
    return torch.stack(p, dim=1).to(torch.int32)


def _prepare_heads(case, seed):
    gen = _generator(seed)
    M, hq, hk, d = case["M"], case["hq"], case["hk"], case["d"]
    qkv = torch.randn((M, (hq + 2 * hk) * d), generator=gen, device="cuda") * 1.5        # the fused projection's output
    qkv[:, ::37] *= 6.0
    qkv = qkv.to(_dtype(case["x"]))
    n_q, n_k = (d, d) if case["norm"] == "head" else (hq * d, hk * d)
    weights = [None, None]
    if case["norm"] != "none":
        weights = [1.0 + 0.3 * torch.randn(n, generator=gen, device="cuda") for n in (n_q, n_k)]
    return dict(case=case, Q=qkv[:, :hq * d].unflatten(1, (hq, d)), K=qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d)), w_q=weights[0], w_k=weights[1],
                pos=_positions(case), freq=_frequencies(_axes(case)))


def prepare(case, seed):
    return _prepare_fused(case, seed) if case["op"] == "fused" else _prepare_heads(case, seed)


# ------------------------------------------------------------------------------------------- the operators

def _plain_fused(st):
    case, X = st["case"], st["X"].float()
    K_o = _outliers(case)
    most = X.abs().amax(dim=1, keepdim=True)
    s_x = most / torch.full_like(most, 127.0)                # a quotient: by a number torch multiplies with its reciprocal
    Xq = torch.where(s_x > 0, torch.clamp(torch.round(X / s_x), -127, 127), torch.zeros_like(X))[:, st["perm"].long()]
    W = st["codes"].float()
    Y = (Xq[:, K_o:] @ W[:, K_o:].t()) * st["s_n"]
    if K_o:
        Y = Y + (Xq[:, :K_o] @ W[:, :K_o].t()) * st["s_o"]
    Y = Y * s_x + st["bias"]
    if case["act"]:
        Y = 0.5 * Y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (Y + 0.044715 * Y * Y * Y)))
    if st["gate"] is not None:
        Y = Y * st["gate"].repeat_interleave(st["rows"], dim=0)[:case["M"]]
    if st["residual"] is not None:
        Y = st["residual"].float() + Y
    return Y.to(_dtype(case["y"]))


def _plain_norm(x, case, w):
    if case["norm"] == "head":
        return x * torch.rsqrt(x.square().mean(dim=2, keepdim=True) + EPS) * w
    if case["norm"] == "row":
        return x * torch.rsqrt(x.square().mean(dim=(1, 2), keepdim=True) + EPS) * w.view(x.shape[1], x.shape[2])
    return x


def _plain_rotate(x, cos, sin, case):
    r = 2 * cos.shape[1]
    cos, sin = cos[:, None], sin[:, None]
    a, b = (x[:, :, 0:r:2], x[:, :, 1:r:2]) if case["inter"] else (x[:, :, :r // 2], x[:, :, r // 2:r])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, v], dim=3).flatten(2) if case["inter"] else torch.cat([u, v], dim=2)
    return torch.cat([turned, x[:, :, r:]], dim=2)


def _plain_heads(st):
    case = st["case"]
    pairs = torch.tensor([a // 2 for a in _axes(case)], device="cuda")
    angle = torch.repeat_interleave(st["pos"].double(), pairs, dim=1) * st["freq"]       # far positions need the 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = [_plain_rotate(_plain_norm(x.float(), case, w), cos, sin, case).to(x.dtype) for x, w in ((st["Q"], st["w_q"]), (st["K"], st["w_k"]))]
    return [o.transpose(0, 1).contiguous() for o in out] if case["heads_first"] else out


def _own_fused(st):
    import paper_2605_21072_amd as q
    case = st["case"]
    w = q.DualScaleWeight(st["Wq"], st["s_n"], st["s_o"], st["perm"], _outliers(case), case["N"], case["K"], None, case["bits"])
    return q.w8a8_linear_fused(st["X"], w, st["bias"], act=q.ACT_GELU_TANH if case["act"] else q.ACT_NONE, gate=st["gate"], gate_rows=st["rows"],
                               residual=st["residual"], out_dtype=_dtype(case["y"]))


def _own_heads(st):
    import paper_2605_21072_amd as q
    case, Q, K = st["case"], st["Q"], st["K"]
    norm = {"none": q.NORM_NONE, "head": q.NORM_HEAD, "row": q.NORM_ROW}[case["norm"]]
    rope = q.Rope(_axes(case), st["freq"], case["inter"])
    if not case["heads_first"]:
        return list(q.qk_norm_rope(Q, K, norm, st["w_q"], st["w_k"], EPS, st["pos"], rope))
    out = [torch.empty((x.shape[1], x.shape[0], x.shape[2]), dtype=x.dtype, device=x.device) for x in (Q, K)]
    q.qk_norm_rope(Q, K, norm, st["w_q"], st["w_k"], EPS, st["pos"], rope, out_q=out[0].transpose(0, 1), out_k=out[1].transpose(0, 1))
    return out


def run(st):
    if st["case"]["op"] == "fused":
        return _own_fused(st) if own else _plain_fused(st)
    return _own_heads(st) if own else _plain_heads(st)


# ------------------------------------------------------------------------------------------- in 64 bits

def _exact_fused(st):
    """The definition: codes by the fp32 quotient that it asks for, everything behind them in 64 bits."""
    case, K_o = st["case"], _outliers(st["case"])
    X = st["X"].double()
    scale = (X.abs().max(dim=1).values / 127.0).float().double()             # an fp32 quotient rounded by way of fp64 is the fp32 quotient
    quotient = (X / torch.where(scale > 0, scale, torch.ones_like(scale)).unsqueeze(1)).float().double()
    weight = torch.zeros((case["N"], case["K"]), dtype=torch.float64, device="cuda")
    column = torch.cat([st["s_o"].double().unsqueeze(1).expand(-1, K_o), st["s_n"].double().unsqueeze(1).expand(-1, case["K"] - K_o)], dim=1)
    weight[:, st["perm"].long()] = st["codes"].double() * column
    y = torch.addmm(st["bias"].double(), quotient.round().clamp(-127, 127) * scale.unsqueeze(1), weight.t())
    if case["act"]:
        y = y / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))        # 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))
    if st["gate"] is not None:
        y = y * st["gate"].double()[torch.arange(case["M"], device="cuda") // st["rows"]]
    return y if st["residual"] is None else y + st["residual"].double()


def _exact_heads(st):
    case, out, at = st["case"], [], 0
    turns = []
    for axis, width in enumerate(_axes(case)):
        turns.append(st["pos"][:, axis].double().unsqueeze(1) * st["freq"][at:at + width // 2])
        at += width // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.cat(turns, dim=1)).unsqueeze(1)
    for x, w in ((st["Q"].double(), st["w_q"]), (st["K"].double(), st["w_k"])):
        if case["norm"] != "none":
            over = (2,) if case["norm"] == "head" else (1, 2)
            x = x / torch.sqrt((x * x).mean(dim=over, keepdim=True) + EPS) * w.double().reshape((-1, case["d"]))
        first = torch.arange(at, device="cuda") * (2 if case["inter"] else 1)
        second = first + (1 if case["inter"] else at)
        z = torch.complex(x[:, :, first], x[:, :, second]) * turn
        x = x.clone()
        x[:, :, first], x[:, :, second] = z.real, z.imag
        out.append(x.transpose(0, 1).contiguous() if case["heads_first"] else x)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_fused(st) if case["op"] == "fused" else _exact_heads(st)


def work(case):
    M = case["M"]
    xb = 4 if case["x"] == "f32" else 2
    if case["op"] == "heads":
        values = M * (case["hq"] + case["hk"]) * case["d"]
        weights = 0 if case["norm"] == "none" else 2 * case["d"] if case["norm"] == "head" else (case["hq"] + case["hk"]) * case["d"]
        pairs = sum(_axes(case)) // 2
        # in and out, positions, frequencies, norm weights; two operations a value for the sum of squares, two for the scaling,
        # three for the rotation, and an angle with its sine and cosine (counted as ten) for each token and pair
        return dict(bytes=2 * values * xb + 4 * M * len(_axes(case)) + 8 * pairs + 4 * weights,
                    flops=values * (3 + (0 if case["norm"] == "none" else 4)) + 10 * M * pairs)
    K, N = case["K"], case["N"]
    yb = 4 if case["y"] == "f32" else 2
    return dict(bytes=M * K * xb + N * K * case["bits"] // 8 + 12 * N + (4 * K if case["c"] else 0) + 4 * N * case["gates"] +
                M * N * yb * (2 if case["residual"] else 1), flops=2 * M * N * K)
