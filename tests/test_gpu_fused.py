"""The GEMM's fused endings (activation, gate, residual) against the definition in 64 bits, on every kernel that can run the shape."""
import pytest
import torch

import paper_2605_21072_amd as q

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


def layer(seed, N, K, K_o, bits):
    """A layer given by its codes; rows of `Wq` in the packed layout."""
    gen = torch.Generator().manual_seed(seed)
    qmax = 127 if bits == 8 else 7
    codes = torch.randint(-qmax, qmax + 1, (N, K), generator=gen, dtype=torch.int8)
    off, kp = q.packed_normal_offset(K_o), q.packed_k(K, K_o)
    P = torch.zeros((N, kp + 128), dtype=torch.int8)
    P[:, :K_o], P[:, off:off + K - K_o] = codes[:, :K_o], codes[:, K_o:]
    if bits == 4:
        g = (P.view(N, -1, 4, 4) & 15).to(torch.uint8)
        P = torch.stack([g[:, :, 0] | (g[:, :, 1] << 4), g[:, :, 2] | (g[:, :, 3] << 4)], dim=2).reshape(N, -1).contiguous()
    s = torch.rand((2, N), generator=gen) * 1e-3 + 1e-4
    perm = torch.randperm(K, generator=gen).to(torch.int32)
    return q.DualScaleWeight(P.cuda(), s[0].cuda(), (s[1] * 30).cuda(), perm.cuda(), K_o, N, K, None, bits), codes


def definition(Xq, s_x, w, codes, bias):
    """(y, bound on what the kernel's fp32 may be off by), in 64 bits, from the packed codes of the activations."""
    off = q.packed_normal_offset(w.K_o)
    X = torch.cat([Xq[:, :w.K_o], Xq[:, off:off + w.K - w.K_o]], dim=1).cpu().double()
    W = codes.double()
    an, ao = X[:, w.K_o:] @ W[:, w.K_o:].t(), X[:, :w.K_o] @ W[:, :w.K_o].t()
    n, o = an * w.s_normal.cpu().double(), ao * w.s_outlier.cpu().double()
    s, b = s_x.cpu().double().unsqueeze(1), torch.zeros(w.N, dtype=torch.float64) if bias is None else bias.cpu().double()
    # conversion of each sum, the first product, two fused steps: every one off by at most U32 of what it rounds
    return s * (n + o) + b, 5 * U32 * (s * (n.abs() + o.abs()) + b.abs())


def gelu(y):
    return y / (1 + torch.exp(-2 * (2 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3)))


def check(Y, y, err, act, gate, rows, residual):
    if act:
        # the function's slope is at most 1.13; then what the header states of its evaluation
        y, err = gelu(y), 1.13 * err + 4e-7 + 2e-6 * gelu(y).abs()
    if gate is not None:
        g = gate.cpu().double().reshape(-1, y.shape[1])[torch.arange(y.shape[0]) // rows]
        y, err = y * g, err * g.abs()
    if residual is not None:
        y = y + residual.cpu().double()
    bound = err + U32 * y.abs()                                     # the one fused step that joins them
    if Y.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (y.abs() + bound)
    off = (Y.cpu().double() - y).abs()
    assert bool((off <= bound + 1e-37).all()), "off by %g of the bound" % float((off / (bound + 1e-37)).max())


def inputs(seed, M, K, N, dtype, act, gates, residual):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((M, K), generator=gen, device="cuda")
    bias = torch.randn(N, generator=gen, device="cuda")
    gate = torch.randn((gates, N), generator=gen, device="cuda") if gates else None
    R = (4 * torch.randn((M, N), generator=gen, device="cuda")).to(dtype) if residual else None
    return X, bias, gate, R


ENDINGS = [(1, 0, False), (0, 0, True), (0, 3, True), (1, 2, True), (0, 1, False), (1, 1, False), (0, 0, False)]     # act, gate rows, residual
#        M, N, K, K_o: one token; whole tiles; ragged rows; more tiles than CUs; any N; wide and odd outlier blocks; short K
SHAPES = [(1, 64, 128, 0), (256, 256, 256, 32), (300, 520, 1000, 96), (129, 1544, 384, 128), (2100, 1536, 256, 64), (77, 131, 200, 7),
          (70, 264, 640, 200), (1, 1, 1, 0), (17, 8, 96, 96), (65, 24, 33, 33),
          (140, 516, 256, 32), (1, 40, 5000, 0)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K,K_o", SHAPES)
def test_endings(M, N, K, K_o, dtype, bits):
    w, codes = layer(M + N + K, N, K, K_o, bits)
    for n, (act, gates, residual) in enumerate(ENDINGS):
        gates = min(gates, M)
        X, bias, gate, R = inputs(100 * n + M, M, K, N, dtype, act, gates, residual)
        rows = -(-M // gates) if gates else None
        Y = q.w8a8_linear_fused(X, w, bias, act=act, gate=gate, gate_rows=rows, residual=R, out_dtype=dtype)
        Xq, s_x = q.quant_act(X, w.perm if K_o else None, K_o)
        assert torch.equal(Y, q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=act, gate=gate, gate_rows=rows, residual=R, out_dtype=dtype))
        y, err = definition(Xq, s_x, w, codes, bias)
        check(Y, y, err, act, gate, rows, R)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,K,K_o", [(300, 520, 1000, 96), (700, 136, 200, 32), (77, 131, 200, 150)])
def test_every_kernel_by_number(M, N, K, K_o, dtype):
    ran = set()
    for bits in (8, 4):
        w, codes = layer(7 + bits, N, K, K_o, bits)
        for act, gates, residual in ((1, 0, False), (0, 4, True), (1, 7, True)):
            X, bias, gate, R = inputs(act + gates, M, K, N, dtype, act, gates, residual)
            rows = -(-M // gates) if gates else None
            Xq, s_x = q.quant_act(X, w.perm, K_o)
            y, err = definition(Xq, s_x, w, codes, bias)
            first = None
            for v in range(1, q.fused_gemm_num_variants() + 1):
                try:
                    Y = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=act, gate=gate, gate_rows=rows, residual=R, out_dtype=dtype, variant=v)
                except q.QarvdError as e:
                    assert e.status == -2
                    continue
                ran.add(v)
                check(Y, y, err, act, gate, rows, R)
                first = Y if first is None else first
                assert torch.equal(Y, first)         # sums are exact and the epilogue is the same: the same bits from every kernel
    assert len(ran) >= (8 if N % 8 == 0 else 6)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("N,K,K_o", [(8, 96, 96), (131, 1000, 7), (520, 4200, 160), (2056, 130, 0), (4104, 300, 64), (8200, 260, 33)])
def test_few_rows(N, K, K_o, bits):
    """Tokens from one to more than the kernels for few rows take, outputs on either side of what each of them takes."""
    w, codes = layer(N + K, N, K, K_o, bits)
    for M in (1, 2, 7, 8, 9, 16, 17, 32, 33):
        gates = min(M, 3)
        rows = -(-M // gates)
        for act, residual, dtype in ((0, True, torch.bfloat16), (1, False, torch.float32)):
            X, bias, gate, R = inputs(M, M, K, N, dtype, act, gates, residual)
            Xq, s_x = q.quant_act(X, w.perm if K_o else None, K_o)
            y, err = definition(Xq, s_x, w, codes, bias)
            Y = q.w8a8_linear_fused(X, w, bias, act=act, gate=gate, gate_rows=rows, residual=R, out_dtype=dtype)
            check(Y, y, err, act, gate, rows, R)
            for v in range(1, q.fused_gemm_num_variants() + 1):
                try:
                    got = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=act, gate=gate, gate_rows=rows, residual=R, out_dtype=dtype, variant=v)
                except q.QarvdError as e:
                    assert e.status == -2
                    continue
                assert torch.equal(got, Y), v


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("K,K_o", [(4, 0), (3, 3), (97, 33), (1536, 32), (2048, 1), (2047, 2047), (2048, 0), (2049, 64), (8960, 64), (10240, 0), (10239, 160),
                                   (10240, 10240), (10241, 32)])
def test_tokens_quantized_on_the_way(K, K_o, bits):
    """One row is quantized by the GEMM's own workgroups, up to 10240 channels: the codes and scales of quant_act, whatever the rows' sizes."""
    N = 72
    w, _ = layer(K, N, K, K_o, bits)
    gen = torch.Generator(device="cuda").manual_seed(K)
    scales = torch.tensor([1.0, 0.0, 1e-36, 3e34, 1e-30, 1.0, 1e-4, 1e4, 1.0, 0.0, 1.0, 1e-36, 1.0, 1.0, 3e34, 1.0, 1.0], device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        for M in (1, 2, 7, 8, 9, 16, 17):
            rows = torch.randn((M, K + 1), generator=gen, device="cuda")
            rows[:, ::7] *= 15
            for first in range(5 if M == 1 else 1):
                X = rows * scales[first:first + M, None]
                if M != 2:
                    X[M - 1] = torch.where(rows[M - 1] > 3, float("inf"), X[M - 1]) if first == 0 and M > 2 else X[M - 1]
                X = X.to(dtype)[:, 1:]                   # (an odd address, too)
                Xq, s_x = q.quant_act(X, w.perm if K_o else None, K_o)
                bias, R = torch.randn(N, generator=gen, device="cuda"), torch.randn((M, N), generator=gen, device="cuda")
                want = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, residual=R, out_dtype=torch.float32)
                got = q.w8a8_linear_fused(X, w, bias, residual=R, out_dtype=torch.float32)
                assert torch.equal(got.view(torch.int32), want.view(torch.int32)), (dtype, M, first)


@pytest.mark.parametrize("N", [2048, 2056, 4096, 4104])
def test_tokens_quantized_on_the_way_by_width(N):
    """Outputs on either side of what one round of workgroups holds."""
    K, K_o = 520, 40
    w, _ = layer(N, N, K, K_o, 8)
    for M in (1, 8, 9, 16):
        X, bias, gate, R = inputs(M, M, K, N, torch.bfloat16, 1, 1, True)
        Xq, s_x = q.quant_act(X, w.perm, K_o)
        want = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=1, gate=gate, residual=R)
        assert torch.equal(q.w8a8_linear_fused(X, w, bias, act=1, gate=gate, residual=R), want)


@pytest.mark.parametrize("M,rows", [(300, 1), (300, 7), (300, 100), (300, 255), (300, 256), (300, 299), (1100, 300), (1100, 520), (40, 40), (40, 1 << 30)])
def test_groups_of_tokens(M, rows):
    """Groups shorter than a row block, boundaries inside a tile and a wave's rows, one group; the result is the formula's, bit for bit."""
    N, K = 264, 128
    w, _ = layer(3, N, K, 32, 8)
    groups = -(-M // rows)
    X, bias, gate, R = inputs(rows % 1000, M, K, N, torch.float32, 0, groups, True)
    Xq, s_x = q.quant_act(X, w.perm, 32)
    y = q.w8a8_dual_gemm(Xq, s_x, w, bias, M, torch.float32).double()
    want = (y * gate.double()[torch.arange(M, device="cuda") // rows] + R.double()).float()       # the fp32 product is exact in 64 bits
    ran = 0
    for v in range(q.fused_gemm_num_variants() + 1):
        try:
            got = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, gate=gate, gate_rows=rows, residual=R, out_dtype=torch.float32, variant=v)
        except q.QarvdError as e:
            assert e.status == -2 and v > 0
            continue
        ran += 1
        assert torch.equal(got, want), v
    assert ran >= (9 if rows >= 255 or groups <= 2 else 5)         # (many short groups: the general kernels and the heuristic)


def test_without_an_ending_it_is_the_plain_linear():
    for bits in (8, 4):
        w, _ = layer(1, 520, 1000, 96, bits)
        X, bias, _, _ = inputs(2, 300, 1000, 520, torch.bfloat16, 0, 0, False)
        assert torch.equal(q.w8a8_linear_fused(X, w, bias), q.w8a8_linear(X, w, bias))
        assert torch.equal(q.w8a8_linear_fused(X, w, None, out_dtype=torch.float32), q.w8a8_linear(X, w, None, torch.float32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,shift", [(300, 520, 0), (300, 520, 1), (300, 520, 8), (77, 131, 3), (1, 520, 0)])
def test_strides_alignment_and_in_place(M, N, dtype, shift):
    """Y, residual and gate as parts of wider buffers, at aligned and odd places; Y on the residual itself; nothing else is written."""
    K = 256
    w, _ = layer(5, N, K, 32, 8)
    X, bias, gate, R = inputs(6, M, K, N, dtype, 1, 2 if M > 1 else 1, True)
    rows = -(-M // gate.shape[0])
    want = q.w8a8_linear_fused(X, w, bias, act=1, gate=gate, gate_rows=rows, residual=R, out_dtype=dtype)
    guard = torch.full((M + 2, N + 64), 7.0, dtype=dtype, device="cuda")
    wide_g = torch.full((gate.shape[0] + 1, N + 16), float("nan"), device="cuda")
    part, part_g = guard[1:M + 1, shift:shift + N], wide_g[:gate.shape[0], shift:shift + N]
    part.copy_(R)
    part_g.copy_(gate)
    Y = q.w8a8_linear_fused(X, w, bias, act=1, gate=part_g, gate_rows=rows, residual=part, out_dtype=dtype)
    assert torch.equal(Y, want)
    back = q.w8a8_linear_fused(X, w, bias, act=1, gate=part_g, gate_rows=rows, residual=part, Y=part)
    assert back is part and torch.equal(part, want)
    rest = guard.clone()
    rest[1:M + 1, shift:shift + N] = 7.0
    assert bool((rest == 7.0).all())


def test_strides_beyond_what_the_fast_kernels_address():
    M, N, K = 3, 16, 128
    w, _ = layer(8, N, K, 32, 8)
    X, bias, gate, R = inputs(9, M, K, N, torch.bfloat16, 1, 3, True)
    want = q.w8a8_linear_fused(X, w, bias, act=1, gate=gate, gate_rows=1, residual=R)
    Xq, s_x = q.quant_act(X, w.perm, 32)
    far = torch.zeros((M, (1 << 22) + 64), dtype=torch.int8, device="cuda")
    far[:, :Xq.shape[1]] = Xq
    assert torch.equal(q.w8a8_dual_gemm_fused(far, s_x, w, bias, M, act=1, gate=gate, gate_rows=1, residual=R), want)
    far_r = torch.zeros((M, (1 << 21) + 1), dtype=torch.bfloat16, device="cuda")
    far_g = torch.zeros((M, (1 << 21) + 1), device="cuda")
    far_r[:, :N], far_g[:, :N] = R, gate
    assert torch.equal(q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=1, gate=far_g[:, :N], gate_rows=1, residual=far_r[:, :N]), want)


@pytest.mark.parametrize("N", [264, 131])
def test_infinities_and_nan_stay_where_they_are(N):
    M, K = 130, 128
    w, _ = layer(11, N, K, 0, 8)
    X, bias, gate, R = inputs(12, M, K, N, torch.bfloat16, 0, 1, True)
    want = q.w8a8_linear_fused(X, w, bias, gate=gate, residual=R)
    R[3, 5], R[64, N - 1], R[M - 1, 0] = float("nan"), float("inf"), float("-inf")
    Y = q.w8a8_linear_fused(X, w, bias, gate=gate, residual=R)
    assert bool(Y[3, 5].isnan()) and float(Y[64, N - 1]) == float("inf") and float(Y[M - 1, 0]) == float("-inf")
    Y[3, 5], Y[64, N - 1], Y[M - 1, 0] = want[3, 5], want[64, N - 1], want[M - 1, 0]
    assert torch.equal(Y, want)
    X[7] = 0.0                                   # a token of zeros: its scale is 0, what is left is the bias
    Y = q.w8a8_linear_fused(X, w, bias, act=1, out_dtype=torch.float32)
    check(Y[7:8], bias.cpu().double().unsqueeze(0), torch.zeros((1, N), dtype=torch.float64), 1, None, None, None)


def test_without_outliers_their_scales_are_not_read():
    """No outlier block: what stands in s_outlier is of no matter, on any kernel."""
    for bits in (8, 4):
        for N, K in ((520, 256), (131, 300)):
            w, _ = layer(21, N, K, 0, bits)
            for M in (1, 5, 20, 300):
                X, bias, gate, R = inputs(22, M, K, N, torch.float32, 0, 1, True)
                want = q.w8a8_linear_fused(X, w, bias, gate=gate, residual=R, out_dtype=torch.float32)
                keep, w.s_outlier = w.s_outlier, torch.full_like(w.s_outlier, float("nan"))
                Xq, s_x = q.quant_act(X, None, 0)
                for v in range(q.fused_gemm_num_variants() + 1):
                    try:
                        got = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, gate=gate, residual=R, out_dtype=torch.float32, variant=v)
                    except q.QarvdError:
                        continue
                    assert torch.equal(got, want), v
                assert torch.equal(q.w8a8_linear_fused(X, w, bias, gate=gate, residual=R, out_dtype=torch.float32), want)
                w.s_outlier = keep


def test_gelu_far_from_zero():
    """A bias of any size through the activation: the tails are 0 and the value itself."""
    N, K = 512, 128
    w, codes = layer(13, N, K, 0, 8)
    X = torch.zeros((2, K), device="cuda")
    bias = torch.cat([torch.linspace(-12, 12, 400), torch.logspace(1, 38, 56), -torch.logspace(1, 38, 56)]).cuda()
    Y = q.w8a8_linear_fused(X, w, bias, act=1, out_dtype=torch.float32)
    y = bias.cpu().double().expand(2, N)
    want = torch.where(y < -20, torch.zeros_like(y), torch.where(y > 20, y, gelu(y.clamp(-20, 20))))
    assert bool(((Y.cpu().double() - want).abs() <= 4e-7 + 2e-6 * want.abs()).all())


def test_captured_and_replayed():
    M, N, K = 300, 520, 256
    w, _ = layer(15, N, K, 32, 8)
    X, bias, gate, R = inputs(16, M, K, N, torch.bfloat16, 0, 3, True)
    Y = torch.empty_like(R)
    call = lambda: q.w8a8_linear_fused(X, w, bias, gate=gate, residual=R, Y=Y)     # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        X2, _, g2, R2 = inputs(50 + seed, M, K, N, torch.bfloat16, 0, 3, True)
        X.copy_(X2), gate.copy_(g2), R.copy_(R2)
        want = q.w8a8_linear_fused(X2, w, bias, gate=g2, residual=R2)
        Y.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want)


def test_two_streams_at_once():
    M, N, K = 300, 520, 1000
    (w1, _), (w2, _) = layer(17, N, K, 96, 8), layer(18, N, K, 96, 4)
    a, b = inputs(19, M, K, N, torch.bfloat16, 0, 3, True), inputs(20, M, K, N, torch.bfloat16, 0, 3, True)
    run = lambda w, i, s=None: q.w8a8_linear_fused(i[0], w, i[1], act=1, gate=i[2], residual=i[3], stream=s)      # noqa: E731
    want = run(w1, a), run(w2, b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for s in (s1, s2):
        with torch.cuda.stream(s):
            torch.cuda._sleep(2_000_000)
    got = [(run(w1, a, s1), run(w2, b, s2)) for _ in range(6)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[0]) and torch.equal(y, want[1]) for x, y in got)
