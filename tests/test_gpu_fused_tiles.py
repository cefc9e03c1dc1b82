"""The fused endings where a workgroup has several tiles, where strides leave the fast kernels' range, and on a token that is not finite."""
import pytest
import torch

import paper_2605_21072_amd as q
from test_gpu_fused import U32, gelu, layer

pytestmark = pytest.mark.gpu

# kernels by number: what they need of a call (see qarvd_ending in the header), INT8 and INT4 weights
ALIGNED, ANY_WIDTH, ANY_STRIDE, FEW_TOKENS = (({1, 2, 3, 4, 5, 6}, {11, 12, 13}), ({7, 8, 9}, {14, 15}), ({10}, {16}), ({17, 18, 19}, {20, 21, 22}))
SHORTEST_GROUP = {1: 255, 2: 255, 5: 63, 6: 63, 11: 255, 12: 255}      # of more than two groups, on the aligned tiles of 256 and of 64 rows (128: 127)
GELU_ALONE = {1, 11}                                       # 256 x 256


def of(bits, *kinds):
    return set().union(*(k[0 if bits == 8 else 1] for k in kinds))


def tensors(seed, M, K, N, dtype, gates, residual):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    X = torch.randn((M, K), generator=gen, device="cuda")
    bias = torch.randn(N, generator=gen, device="cuda")
    gate = torch.randn((gates, N), generator=gen, device="cuda") if gates else None
    return X, bias, gate, (4 * torch.randn((M, N), generator=gen, device="cuda")).to(dtype) if residual else None


def product(Xq, s_x, w, codes, bias):
    """(y, bound on the kernel's fp32), in 64 bits."""
    off = q.packed_normal_offset(w.K_o)
    X = torch.cat([Xq[:, :w.K_o], Xq[:, off:off + w.K - w.K_o]], dim=1).double()
    Wt = codes.cuda().double().t().contiguous()
    n, o = (X[:, w.K_o:] @ Wt[w.K_o:]) * w.s_normal.double(), (X[:, :w.K_o] @ Wt[:w.K_o]) * w.s_outlier.double()
    s = s_x.double().unsqueeze(1)
    # conversion of each sum, the first product, two fused steps: every one off by at most U32 of what it rounds
    return s * (n + o) + bias.double(), 5 * U32 * (s * (n.abs() + o.abs()) + bias.double().abs())


def check(Y, y, err, act, gate, rows, residual):
    if act:
        a = gelu(y)
        y, err = a, 1.13 * err + 4e-7 + 2e-6 * a.abs()      # the slope is at most 1.13; then what the header states
    if gate is not None:
        g = gate.double()[torch.arange(y.shape[0], device="cuda") // rows]
        y, err = y * g, err * g.abs()
    if residual is not None:
        y = y + residual.double()
    bound = err + U32 * y.abs()
    if Y.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * (y.abs() + bound)
    off = (Y.double() - y).abs()
    assert bool((off <= bound + 1e-37).all()), "off by %g of the bound" % float((off / (bound + 1e-37)).max())


def run_all(call, expected):
    """Every kernel that takes the call, each with the same bits; the set of those that do is the expected one."""
    first, ran = call(0), set()
    for v in range(1, q.fused_gemm_num_variants() + 1):
        try:
            got = call(v)
        except q.QarvdError as e:
            assert e.status == -2
            continue
        ran.add(v)
        assert torch.equal(got, first), v
    assert ran == expected
    return first


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("N,K,K_o", [(2256, 200, 40), (2256, 1000, 0), (2256, 1000, 100), (2251, 200, 150), (2251, 1000, 40)])
def test_several_tiles_to_a_workgroup(N, K, K_o, bits):
    """On every kernel by number: scales, gates and residual of a workgroup's later tiles, K shorter and longer than the ring of stages, no outliers and
    such in one and in two k-steps, groups of tokens that end inside tiles, at their last row and within a wave's rows."""
    M = 9300
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    # more than two rounds of the tallest tiles with a residual, more than one of 256 x 256; the smaller tiles have more of both
    assert (M + 255) // 256 * ((N + 127) // 128) > 2 * cus and (M + 255) // 256 * ((N + 255) // 256) > cus
    aligned = N % 8 == 0 and q.packed_normal_offset(K_o) <= 128
    w, codes = layer(N + K + K_o, N, K, K_o, bits)
    X, bias, _, _ = tensors(1, M, K, N, torch.float32, 0, False)
    Xq, s_x = q.quant_act(X, w.perm if K_o else None, K_o)
    y, err = product(Xq, s_x, w, codes, bias)
    for dtype in (torch.bfloat16, torch.float32):
        fast = aligned or (dtype == torch.float32 and N % 4 == 0 and q.packed_normal_offset(K_o) <= 128)
        for act, rows, residual in ((1, 0, False), (0, 3100, True), (1, 300, True), (0, 0, True), (0, 127, True), (1, 100, False), (0, 7, True)):
            gates = -(-M // rows) if rows else 0
            _, _, gate, R = tensors(2 + rows, M, K, N, dtype, gates, residual)
            expected = of(bits, ANY_WIDTH, ANY_STRIDE, FEW_TOKENS)
            if fast:
                # two groups' gates at most stand beside an aligned tile's scales
                expected |= {v for v in of(bits, ALIGNED) if (not rows or gates <= 2 or rows >= SHORTEST_GROUP.get(v, 127)) and not (v in GELU_ALONE and (rows or residual))}
            Y = run_all(lambda v: q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=act, gate=gate, gate_rows=rows or None, residual=R, out_dtype=dtype,     # noqa: B023
                                                         variant=v), expected)
            check(Y, y, err, act, gate, rows, R)
            if residual:                                    # onto the residual itself
                into = R.clone()
                q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, act=act, gate=gate, gate_rows=rows or None, residual=into, Y=into)
                assert torch.equal(into, Y)


def wide(rows, columns, row_stride, dtype):
    return torch.zeros((rows, row_stride), dtype=dtype, device="cuda")[:, :columns]


@pytest.mark.parametrize("bits", [8, 4])
def test_far_strides_on_every_kernel(bits):
    """Strides beyond 2^22 bytes of codes, or 2^20 elements of residual, gate and output: who takes them, and the same bits."""
    M, N, K, K_o = 300, 520, 256, 32                        # (too many outputs for the kernels for few tokens to be chosen)
    w, codes = layer(8, N, K, K_o, bits)
    for dtype in (torch.bfloat16, torch.float32):
        X, bias, gate, R = tensors(9, M, K, N, dtype, 2, True)
        Xq, s_x = q.quant_act(X, w.perm, K_o)
        call = lambda v, Xq=Xq, w=w, **kw: q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, M, variant=v, **{**dict(act=1, gate=gate, gate_rows=150, residual=R, out_dtype=dtype), **kw})      # noqa: E731, E501
        want = call(0)
        check(want, *product(Xq, s_x, w, codes, bias), 1, gate, 150, R)

        def far(expected, **kw):
            assert torch.equal(run_all(lambda v: call(v, **kw), expected), want)

        any_stride = of(bits, ANY_STRIDE, FEW_TOKENS)
        far_x = wide(M, Xq.shape[1], (1 << 22) + 64, torch.int8)
        far_x.copy_(Xq)
        far(any_stride, Xq=far_x)
        del far_x
        far_w = wide(N, w.Wq.shape[1], (1 << 22) + 64, w.Wq.dtype)
        far_w.copy_(w.Wq)
        far(any_stride, w=q.DualScaleWeight(far_w, w.s_normal, w.s_outlier, w.perm, K_o, N, K, None, bits))
        del far_w
        any_width = any_stride | of(bits, ANY_WIDTH)
        far_r = wide(M, N, (1 << 20) + 16, dtype)
        far_r.copy_(R)
        far(any_width, residual=far_r)
        far_g = wide(2, N, (1 << 20) + 16, torch.float32)
        far_g.copy_(gate)
        far(any_width, gate=far_g)
        far(any_width, gate=far_g, residual=far_r)
        for v in sorted(any_width) + [0]:
            far_y = wide(M, N, (1 << 20) + 16, dtype)
            assert call(v, Y=far_y) is far_y and torch.equal(far_y, want)
            into = wide(M, N, (1 << 20) + 16, dtype)
            into.copy_(R)
            assert torch.equal(call(v, Y=into, residual=into), want)
        for v in of(bits, ALIGNED):
            with pytest.raises(q.QarvdError):
                call(v, Y=far_r)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("K,K_o", [(4, 0), (97, 33), (1536, 32), (2047, 2047), (2049, 64), (10240, 0), (10239, 160)])
def test_a_token_that_is_not_finite(K, K_o, bits):
    """One token quantized on the way with infinities and NaN, first and last channel among them: the codes and scale of quant_act."""
    N = 72
    w, _ = layer(K, N, K, K_o, bits)
    gen = torch.Generator(device="cuda").manual_seed(K)
    bias, R = torch.randn(N, generator=gen, device="cuda"), torch.randn((1, N), generator=gen, device="cuda")
    inf, nan = float("inf"), float("nan")
    finite = 0
    for dtype in (torch.float32, torch.bfloat16):
        for put in ({0: nan}, {K - 1: nan}, {0: nan, K // 2: nan, K - 1: nan}, {0: inf}, {K - 1: -inf}, {0: inf, K - 1: nan}, {K // 2: -inf, K - 1: inf}):
            x = torch.randn((1, K), generator=gen, device="cuda")
            for k, v in put.items():
                x[0, k] = v
            x = x.to(dtype)
            Xq, s_x = q.quant_act(x, w.perm if K_o else None, K_o)
            want = q.w8a8_dual_gemm_fused(Xq, s_x, w, bias, 1, residual=R, out_dtype=torch.float32)
            got = q.w8a8_linear_fused(x, w, bias, residual=R, out_dtype=torch.float32)
            assert torch.equal(got.isnan(), want.isnan()), (dtype, put)
            assert torch.equal(got.nan_to_num(nan=0.0).view(torch.int32), want.nan_to_num(nan=0.0).view(torch.int32)), (dtype, put)
            finite += int(got.isfinite().all())
    assert finite >= 2                                      # a NaN alone does not reach the scale: those rows compare codes
