"""Head norms and rotation by position against the definition in 64 bits."""
import pytest
import torch

import paper_2605_21072_amd as q

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


def definition(x, norm, w, eps, pos, rope):
    """(value, bound on what fp32 may be off by before the result is rounded) in 64 bits, on the host."""
    x = x.detach().cpu().double()
    M, H, D = x.shape
    err = torch.zeros_like(x)
    if norm != q.NORM_NONE:
        over = (2,) if norm == q.NORM_HEAD else (1, 2)
        n = D if norm == q.NORM_HEAD else H * D
        x = x / torch.sqrt((x * x).mean(dim=over, keepdim=True) + eps)
        if w is not None:
            x = x * w.cpu().double().reshape(-1, D)
        # a sum of n squares in at most n / 64 + 64 dependent steps, half of its error in the root; division, root, two products
        err = x.abs() * U32 * ((n / 64 + 64) / 2 + 8)
    if rope is not None:
        R = sum(rope.axis_dims)
        col = torch.cat([torch.full((d // 2,), i) for i, d in enumerate(rope.axis_dims)])
        angle = pos.cpu().reshape(M, -1).double()[:, col] * rope.freq.cpu()
        c, s = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1)
        i = torch.arange(R // 2)
        a, b = (2 * i, 2 * i + 1) if rope.interleaved else (i, i + R // 2)
        u, v, eu, ev = x[:, :, a], x[:, :, b], err[:, :, a], err[:, :, b]
        x, err = x.clone(), err.clone()
        x[:, :, a], x[:, :, b] = u * c - v * s, u * s + v * c
        # sine and cosine within 4 steps and what the fp64 angle is off by; a product and a fused step
        t = 6 * U32 + angle.abs().unsqueeze(1) * 2.0 ** -51
        err[:, :, a] = err[:, :, b] = eu + ev + t * (u.abs() + v.abs())
    return x, err


def check(got, x, norm, w, eps, pos, rope, what=""):
    want, err = definition(x, norm, w, eps, pos, rope)
    bound = err + (2.0 ** -8 if got.dtype == torch.bfloat16 else U32) * (want.abs() + err) + 1e-37
    off = (got.cpu().double() - want).abs()
    assert bool((off <= bound).all()), "%s: off by %g of the bound" % (what, float((off / bound).max()))


def make(seed, M, hq, hk, D, dtype, axes, norm, interleaved, far=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (2 * torch.randn((M, (hq + 2 * hk) * D), generator=gen, device="cuda")).to(dtype)
    Q, K = qkv[:, :hq * D].unflatten(1, (hq, D)), qkv[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D))
    n = {q.NORM_NONE: lambda h: None, q.NORM_HEAD: lambda h: D, q.NORM_ROW: lambda h: h * D}[norm]
    wq, wk = (None if n(h) is None else torch.randn(n(h), generator=gen, device="cuda") for h in (hq, hk))
    if not axes:
        return qkv, Q, K, wq, wk, None, None
    pos = torch.randint(-50, 2000, (M, len(axes)), generator=gen, device="cuda", dtype=torch.int32) + far
    return qkv, Q, K, wq, wk, pos, q.Rope(axes, q.rope_frequencies(axes), interleaved)


NORMS = [q.NORM_NONE, q.NORM_HEAD, q.NORM_ROW]
#        M, heads, key heads, D, axes
SHAPES = [(1, 12, 12, 128, (44, 42, 42)), (37, 12, 12, 128, (44, 42, 42)), (5, 40, 8, 128, (128,)), (300, 3, 1, 64, (32, 32)), (9, 16, 16, 80, (40, 40)),
          (11, 10, 3, 100, (20, 22, 18)), (3, 2, 2, 512, (256, 128, 128)), (7, 5, 5, 8, (4, 2, 2)), (4, 1, 1, 2, (2,)), (6, 3, 2, 33, (16, 16)),
          (2, 2, 1, 1, ()), (13, 7, 7, 96, ()), (33, 4, 4, 72, (24, 24, 24)), (8, 6, 6, 256, (64,)), (1, 1, 1, 128, (16, 56, 56)), (21, 9, 2, 24, (8, 8)),
          (2, 72, 72, 128, (44, 42, 42)), (6, 33, 5, 104, (52, 52)), (2, 260, 3, 128, (44, 42, 42)), (3, 2, 2, 511, (20,)), (5, 50, 50, 256, (64, 96, 96)),
          (3, 64, 64, 512, (512,)), (500, 40, 8, 128, (44, 42, 42)), (1100, 40, 20, 100, (20, 22, 18)),
          (4100, 1, 2, 64, (32, 32)), (9001, 3, 1, 40, (40,)), (70001, 1, 1, 8, (4, 2, 2)), (8193, 2, 2, 33, (16, 16)), (20000, 1, 4, 100, (20, 22, 18)), (4500, 2, 1, 128, (128,)),
          (66000, 5, 1, 1, ()), (4500, 12, 1, 128, (44, 42, 42)), (2100, 10, 3, 100, (20, 22, 18)), (5000, 1, 17, 64, (64,)),
          (8203, 2, 1, 256, (64,)), (8211, 1, 1, 264, (88, 88, 88)), (16387, 1, 1, 33, (16, 16)), (40003, 1, 2, 40, (40,))]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("M,hq,hk,D,axes", SHAPES)
def test_norm_and_rotation(M, hq, hk, D, axes, interleaved, dtype):
    for norm in NORMS:
        qkv, Q, K, wq, wk, pos, rope = make(M * D + norm, M, hq, hk, D, dtype, axes, norm, interleaved)
        keep = qkv.clone()
        oq, ok = q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope)
        assert torch.equal(qkv, keep) and oq.is_contiguous() and ok.is_contiguous()
        check(oq, Q, norm, wq, 1e-6, pos, rope, "Q norm %d" % norm)
        check(ok, K, norm, wk, 1e-6, pos, rope, "K norm %d" % norm)
        # queries alone; in place, which leaves the values (and everything else) as they are
        only, none = q.qk_norm_rope(Q, None, norm, wq, None, 1e-6, pos, rope)
        assert none is None and torch.equal(only, oq)
        q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope, out_q=Q, out_k=K)
        assert torch.equal(Q, oq) and torch.equal(K, ok) and torch.equal(qkv[:, (hq + hk) * D:], keep[:, (hq + hk) * D:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,axes", [(128, (44, 42, 42)), (72, (24, 24, 24)), (50, (10, 20, 20))])
def test_orders_strides_and_alignment(D, axes, dtype):
    M, hq, hk = 19, 6, 2
    for norm in NORMS:
        for interleaved in (True, False):
            _, Q, K, wq, wk, pos, rope = make(norm, M, hq, hk, D, dtype, axes, norm, interleaved)
            # each layout may go to another kernel, which sums in another order: every result is held to the definition
            def held(got):
                check(got[0], Q, norm, wq, 1e-6, pos, rope)
                check(got[1], K, norm, wk, 1e-6, pos, rope)
            held(q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope))
            # heads first, in and out
            heads = [torch.full((h + 1, M + 1, D + 8), 3.0, dtype=dtype, device="cuda") for h in (hq, hk)]
            outs = [t[:h, :M, :D].transpose(0, 1) for t, h in zip(heads, (hq, hk))]
            q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope, out_q=outs[0], out_k=outs[1])
            held(outs)
            for t, h in zip(heads, (hq, hk)):
                t[:h, :M, :D] = 3.0
                assert bool((t == 3.0).all())
            ins = [t[:h, :M, :D].transpose(0, 1) for t, h in zip(heads, (hq, hk))]
            ins[0].copy_(Q), ins[1].copy_(K)
            held(q.qk_norm_rope(ins[0], ins[1], norm, wq, wk, 1e-6, pos, rope))
            # at odd addresses, positions as columns of a wider table
            flat = torch.empty(M * hq * D + 1, dtype=dtype, device="cuda")
            odd = flat[1:].view(M, hq, D).copy_(Q)
            table = torch.zeros((M, 5), dtype=torch.int32, device="cuda")
            table[:, 1:1 + len(axes)] = pos
            held(q.qk_norm_rope(odd, K, norm, wq, wk, 1e-6, table[:, 1:1 + len(axes)], rope))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hq,D", [(4, 128), (12, 128), (40, 128), (33, 100), (50, 256), (1, 64), (2, 72)])
def test_a_token_has_the_same_bits_in_any_batch(hq, D, dtype):
    """However many waves share a row, and however many tokens there are."""
    M = 4700 if hq > 2 else 40000
    for norm in NORMS:
        _, Q, _, wq, _, pos, rope = make(norm, M, hq, hq, D, dtype, (20, 22, 18), norm, True)
        whole, _ = q.qk_norm_rope(Q, None, norm, wq, None, 1e-6, pos, rope)
        for first, n in ((0, 1), (3, 40), (7, 300), (20, 1500), (0, 3000)):
            part, _ = q.qk_norm_rope(Q[first:first + n], None, norm, wq, None, 1e-6, pos[first:first + n], rope)
            assert torch.equal(part, whole[first:first + n]), (norm, first, n)


@pytest.mark.parametrize("far", [100_000, 30_000_000, 2**31 - 3000, -2**31 + 100])
def test_far_positions(far):
    for D, axes in ((128, (44, 42, 42)), (50, (10, 20, 20))):
        _, Q, K, wq, wk, pos, rope = make(1, 9, 3, 2, D, torch.float32, axes, q.NORM_HEAD, True, far)
        oq, ok = q.qk_norm_rope(Q, K, q.NORM_HEAD, wq, wk, 1e-6, pos, rope)
        check(oq, Q, q.NORM_HEAD, wq, 1e-6, pos, rope)
        check(ok, K, q.NORM_HEAD, wk, 1e-6, pos, rope)


def test_whole_turns_and_position_zero():
    """Quarter turns come out exactly; position 0 leaves what the norm gives."""
    freq = torch.full((64,), torch.pi / 2, dtype=torch.float64, device="cuda")
    Q = torch.randn((8, 4, 128), device="cuda")
    pos = torch.arange(-4, 4, dtype=torch.int32, device="cuda")
    out, _ = q.qk_norm_rope(Q, None, q.NORM_NONE, pos=pos, rope=q.Rope((128,), freq))
    a, b = Q[..., 0::2], Q[..., 1::2]
    for m in range(8):
        want = [(a, b), (-b, a), (-a, -b), (b, -a)][int(pos[m]) % 4]
        assert torch.allclose(out[m, :, 0::2], want[0][m], rtol=0, atol=2e-6) and torch.allclose(out[m, :, 1::2], want[1][m], rtol=0, atol=2e-6)
    assert torch.equal(out[4], Q[4])


@pytest.mark.parametrize("D", [128, 50])
def test_zero_rows_infinities_and_nan_stay_in_their_row(D):
    axes = (D // 2 // 2 * 2,)
    for norm in NORMS:
        for dtype in (torch.bfloat16, torch.float32):
            _, Q, K, wq, wk, pos, rope = make(2, 12, 3, 3, D, dtype, axes, norm, True)
            Q, K = Q.clone(), K.clone()
            want = q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope)
            Q[3], Q[5, 1, 7], K[7, 2, 0] = 0.0, float("nan"), float("inf")
            got = q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope)
            assert bool((got[0][3] == 0).all())
            assert bool(got[0][5, 1].isnan().any()) and not bool(got[1][7, 2].isfinite().all())
            for i, m, h in ((0, 5, 1), (1, 7, 2)):
                if norm == q.NORM_ROW:
                    got[i][m] = want[i][m]
                else:
                    got[i][m, h] = want[i][m, h]
            got[0][3] = want[0][3]
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    out, _ = q.qk_norm_rope(torch.zeros((2, 2, D), device="cuda"), None, q.NORM_HEAD, eps=0.0)
    assert bool(out.isnan().all())                      # 0 / 0, as the formula says


def test_without_weights_and_with_tiny_and_large_values():
    for D in (128, 50):
        x = torch.randn((6, 4, D), device="cuda")
        for scale in (1e-15, 1e-4, 1e4, 1e15):
            y = x * scale
            for norm in (q.NORM_HEAD, q.NORM_ROW):
                out, _ = q.qk_norm_rope(y, None, norm, eps=0.0)
                check(out, y, norm, None, 0.0, None, None, "scale %g" % scale)


def test_many_tokens_and_the_same_result_twice():
    for M, hq, hk, D, axes, norm in ((5000, 12, 12, 128, (44, 42, 42), q.NORM_ROW), (70000, 1, 1, 64, (64,), q.NORM_HEAD), (3001, 5, 2, 50, (10, 20), q.NORM_HEAD)):
        _, Q, K, wq, wk, pos, rope = make(4, M, hq, hk, D, torch.bfloat16, axes, norm, True)
        a, b = q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope), q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        at = torch.randperm(M)[:200].sort().values.cuda()
        at[0], at[-1] = 0, M - 1
        check(a[0][at], Q[at], norm, wq, 1e-6, pos[at], rope)
        check(a[1][at], K[at], norm, wk, 1e-6, pos[at], rope)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,hq,hk,D,extra", [(300, 4, 2, 64, 2 * 64), (1, 12, 12, 128, 12 * 128), (77, 3, 0, 40, 11), (130, 2, 2, 50, 0)])
def test_qkv_projection_is_the_linear_and_the_pass(M, hq, hk, D, extra, dtype, bits):
    K, N = 256, (hq + hk) * D + extra
    gen = torch.Generator(device="cuda").manual_seed(M + D)
    W = torch.randn((N, K), generator=gen, device="cuda") * 0.02
    W[:, 11] *= 30
    w = q.quantize_weight(W, bits=bits)
    X, bias = torch.randn((M, K), generator=gen, device="cuda"), torch.randn(N, generator=gen, device="cuda")
    wq, wk = (1 + 0.2 * torch.randn(D, generator=gen, device="cuda") for _ in range(2))
    axes = (D // 4 * 2, 2)
    rope, pos = q.Rope(axes, q.rope_frequencies(axes)), torch.randint(0, 99, (M, 2), generator=gen, device="cuda", dtype=torch.int32)
    want = q.w8a8_linear(X, w, bias, dtype)
    Q, Kk = want[:, :hq * D].unflatten(1, (hq, D)), want[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D)) if hk else None
    q.qk_norm_rope(Q, Kk, q.NORM_HEAD, wq, wk if hk else None, 1e-6, pos, rope, out_q=Q, out_k=Kk)
    Y = q.w8a8_linear_qkv(X, w, bias, hq, hk, D, q.NORM_HEAD, wq, wk if hk else None, 1e-6, pos, rope, dtype)
    assert torch.equal(Y, want)


def test_a_block_of_the_operators_together():
    """x -> q / k / v with norm and rotation -> attention -> projection onto the stream -> FFN onto the stream, captured and replayed."""
    M, C, H, D, F = 130, 256, 4, 64, 640
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")      # noqa: E731
    layers = [q.quantize_weight(rand(n, k) * 0.05) for n, k in ((3 * C, C), (C, C), (F, C), (C, F))]
    biases = [rand(w.N) * 0.1 for w in layers]
    wq, wk, gates = 1 + 0.1 * rand(D), 1 + 0.1 * rand(D), rand(2, 2, C) * 0.5
    axes = (24, 20, 20)
    rope = q.Rope(axes, q.rope_frequencies(axes))
    pos = torch.stack([torch.arange(M) // 65, torch.arange(M) // 13 % 5, torch.arange(M) % 13], dim=1).to(torch.int32).cuda()

    def block(x, linear, ending, heads):
        qkv = heads(x)
        Q, K, V = (t.unflatten(1, (H, D)).transpose(0, 1) for t in qkv.split(C, dim=1))
        P = torch.softmax((Q.float() @ K.float().transpose(1, 2).contiguous()) / D ** 0.5, dim=2)
        a = (P @ V.float()).transpose(0, 1).flatten(1).to(x.dtype)
        x = ending(a, 1, 0, gates[0], x)
        return ending(linear(x, 2), 3, 0, gates[1], x)

    fused = lambda x: block(                                                                                # noqa: E731
        x, lambda t, i: q.w8a8_linear_fused(t, layers[i], biases[i], act=q.ACT_GELU_TANH),
        lambda t, i, act, g, r: q.w8a8_linear_fused(t, layers[i], biases[i], gate=g, gate_rows=65, residual=r),
        lambda t: q.w8a8_linear_qkv(t, layers[0], biases[0], H, H, D, q.NORM_HEAD, wq, wk, 1e-6, pos, rope))

    def plain(x):
        def y32(t, i):
            return q.w8a8_linear(t, layers[i], biases[i], torch.float32).double()

        def heads(t):
            y = q.w8a8_linear(t, layers[0], biases[0])
            for c, w in ((0, wq), (C, wk)):
                y[:, c:c + C] = definition(y[:, c:c + C].unflatten(1, (H, D)), q.NORM_HEAD, w, 1e-6, pos, rope)[0].flatten(1).to(y.dtype).cuda()
            return y
        return block(x, lambda t, i: torch.nn.functional.gelu(y32(t, i), approximate="tanh").bfloat16(),
                     lambda t, i, act, g, r: (r.double() + g.double()[torch.arange(M, device="cuda") // 65] * y32(t, i)).bfloat16(), heads)

    x = rand(M, C).bfloat16()
    got, want = fused(x), plain(x)
    # A value next to a rounding boundary goes to the other side on one of the two ways, a step of 2^-7 of itself, and moves an INT8 code of the next
    # layer's input (1 / 254 of its row's largest value): both are small against the sum of a row's contributions.
    assert float((got.double() - want.double()).norm() / want.double().norm()) < 2.0 ** -7
    still = x.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = fused(still)
    for k in range(3):
        new = rand(M, C).bfloat16()
        still.copy_(new)
        want = fused(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_given_streams():
    _, Q, K, wq, wk, pos, rope = make(5, 700, 6, 6, 128, torch.bfloat16, (44, 42, 42), q.NORM_HEAD, True)
    want = q.qk_norm_rope(Q, K, q.NORM_HEAD, wq, wk, 1e-6, pos, rope)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s1):
        torch.cuda._sleep(2_000_000)
    got = [q.qk_norm_rope(Q, K, q.NORM_HEAD, wq, wk, 1e-6, pos, rope, stream=s) for s in (s1, s2, s1, s2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, want[0]) and torch.equal(b, want[1]) for a, b in got)
