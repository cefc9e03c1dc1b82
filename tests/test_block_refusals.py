"""What the fused endings and the head norms refuse, on the host and before anything is launched: no GPU needed."""
import ctypes as C
import types

import pytest
import torch

import paper_2605_21072_amd as q
from paper_2605_21072_amd import binding
from paper_2605_21072_amd.binding import _Ending, _Heads, _Rope

INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
P = 0x1000                      # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    if not q.lib_path().exists():
        from paper_2605_21072_amd import build
        build.build()
    return q.load_library()


def test_endings(lib):
    def call(variant=0, bits=8, Y=P, M=4, N=8, ydt=1, act=0, rows=2, gate=P, ldg=8, residual=P, ldr=8, ldwq=128):
        e = _Ending(act, rows, gate, ldg, residual, ldr)
        return lib.qarvd_dual_gemm_fused(P, 128, P, bits, P, ldwq, P, P, None, C.byref(e), M, N, 128, 0, Y, ydt, 8, variant, None)

    n = q.fused_gemm_num_variants()
    assert n >= 1
    assert call(variant=n + 1) == INVALID and call(variant=-1) == INVALID
    assert call(bits=16) == INVALID and call(Y=None) == INVALID and call(M=0) == INVALID
    assert call(act=2) == INVALID and call(act=-1) == INVALID
    assert call(rows=0) == INVALID and call(rows=-3) == INVALID                 # groups of no tokens
    assert call(ldg=7) == INVALID                                               # gate rows that overlap
    assert call(ldr=7) == INVALID                                               # residual rows that overlap
    assert call(gate=P + 2) == UNSUPPORTED and call(residual=P + 1) == UNSUPPORTED and call(ydt=0, residual=P + 2) == UNSUPPORTED
    assert call(ydt=5) == UNSUPPORTED
    # kernels by number: the other weight width; a residual that only the general tiles take
    taken = [[call(variant=v, bits=b, act=9) for v in range(1, n + 1)] for b in (8, 4)]
    assert all(s == INVALID for row in taken for s in row)                      # the ending is looked at first
    assert call(variant=1, bits=4, ldwq=64) == UNSUPPORTED and call(variant=1, residual=P + 2) == UNSUPPORTED
    assert call(variant=1, N=8, gate=P + 4) == UNSUPPORTED
    # one call with the quantizer: the ending and the workspace are checked before it
    e = _Ending(7, 1, None, 0, None, 0)
    args = [P, 0, 128, None, 8, P, 128, P, P, None, C.byref(e), 4, 8, 128, 0, P, 1, 8, P, 1 << 20, None]
    assert lib.qarvd_linear_fused(*args) == INVALID
    args[19] = 16
    assert lib.qarvd_linear_fused(*args) == WORKSPACE


def test_heads(lib):
    def call(q_=True, k=None, dt=1, M=4, D=64, norm=1, eps=1e-6, rope=None):
        return lib.qarvd_qk_norm_rope(C.byref(heads()) if q_ is True else q_ and C.byref(q_), k and C.byref(k), dt, M, D, norm, eps,
                                      rope and C.byref(rope), None)

    def heads(x=P, ld=128, hs=64, out=P, ld_out=128, hs_out=64, w=None, n=2):
        return _Heads(x, ld, hs, out, ld_out, hs_out, w, n)

    def rope(pos=P, ld=3, freq=P, n=3, dims=(24, 20, 20), inter=1):
        return _Rope(pos, ld, freq, n, (C.c_int32 * 3)(*dims), inter)

    assert call(q_=None) == INVALID
    assert call(M=0) == INVALID and call(D=0) == INVALID and call(D=513, q_=heads(ld=2000, hs=600, ld_out=2000, hs_out=600)) == UNSUPPORTED
    assert call(norm=3) == INVALID and call(norm=-1) == INVALID and call(dt=4) == UNSUPPORTED
    for eps in (-1e-6, float("nan"), float("inf")):
        assert call(eps=eps) == INVALID
    for bad in (dict(x=None), dict(out=None), dict(n=0), dict(hs=63), dict(hs_out=63), dict(ld=127), dict(ld_out=127), dict(ld=0), dict(ld_out=-128),
                dict(ld_out=1 << 41)):
        assert call(q_=heads(**bad)) == INVALID, bad
        assert call(k=heads(**bad)) == INVALID, bad
    for bad in (dict(x=P + 1), dict(out=P + 1), dict(w=P + 2)):
        assert call(q_=heads(**bad)) == UNSUPPORTED and call(k=heads(**bad)) == UNSUPPORTED
    assert call(dt=0, q_=heads(x=P + 2)) == UNSUPPORTED
    for bad in (dict(pos=None), dict(freq=None), dict(n=0), dict(n=4), dict(ld=2), dict(dims=(24, 20, 22)), dict(dims=(24, 0, 20)), dict(dims=(23, 21, 20)),
                dict(dims=(-2, 20, 20)), dict(inter=2)):
        assert call(rope=rope(**bad)) == INVALID, bad
    assert call(rope=rope(pos=P + 2)) == UNSUPPORTED and call(rope=rope(freq=P + 4)) == UNSUPPORTED
    # the projection with its heads: more columns than the layer has; nothing of the linear runs before the heads are checked
    qkv = [P, 0, 128, None, 8, P, 128, P, P, None, 4, 192, 128, 0, 2, 1, 64, 1, None, None, 1e-6, None, P, 1, 192, P, 1 << 20, None]
    for i, v in ((14, 0), (15, -1), (15, 2), (16, 0), (17, 5), (20, -1.0), (22, None), (24, 191)):
        a = list(qkv)
        a[i] = v
        assert lib.qarvd_linear_qkv(*a) == INVALID, (i, v)


class Fake(torch.Tensor):
    """A host tensor that says it is on the device, for the Python path's own checks."""
    is_cuda = True


def bad_endings(put):
    M, N, K = 4, 8, 128
    X, Xq = put(torch.zeros(M, K)), put(torch.zeros((M, 256), dtype=torch.int8))
    w = q.DualScaleWeight(put(torch.zeros((N, 256), dtype=torch.int8)), put(torch.ones(N)), put(torch.ones(N)), None, 0, N, K)
    f, b, z = put(torch.zeros(M, N)), put(torch.zeros(M, N, dtype=torch.bfloat16)), lambda *s, **k: put(torch.zeros(*s, **k))
    for bad, err in ((dict(gate=z(N, dtype=torch.bfloat16)), TypeError), (dict(gate=z(N + 1)), ValueError),
                     (dict(gate=z(3, N)), ValueError), (dict(gate=z(2, N), gate_rows=1), ValueError),
                     (dict(gate=z(2, N), gate_rows=0), ValueError), (dict(gate=z(2, N), gate_rows=-4), ValueError), (dict(gate=z(0, N)), ValueError),
                     (dict(gate=z(0, N), gate_rows=4), ValueError), (dict(gate=z(N, 4).t()[:1]), ValueError), (dict(gate_rows=2), ValueError),
                     (dict(gate=z(2, 2, N)), ValueError), (dict(act=5), q.QarvdError),
                     (dict(residual=f), TypeError), (dict(residual=b[:3]), ValueError), (dict(residual=b[:, :7]), ValueError),
                     (dict(residual=z(N, M, dtype=torch.bfloat16).t()), ValueError), (dict(residual=b, out_dtype=torch.float32), TypeError),
                     (dict(Y=b[:2]), ValueError), (dict(Y=z(N, M).t()), ValueError), (dict(out_dtype=torch.float16), TypeError)):
        yield lambda s, bad=bad: q.w8a8_linear_fused(X, w, None, stream=s, **bad), err
        yield lambda s, bad=bad: q.w8a8_dual_gemm_fused(Xq, put(torch.ones(M)), w, None, M, stream=s, **bad), err
    for bias, err in ((z(N, dtype=torch.bfloat16), TypeError), (z(N - 1), ValueError), (z(N, 2)[:, 0], ValueError)):
        yield lambda s, bias=bias: q.w8a8_linear_fused(X, w, bias, stream=s), err
        yield lambda s, bias=bias: q.w8a8_dual_gemm_fused(Xq, put(torch.ones(M)), w, bias, M, stream=s), err
    yield lambda s: q.w8a8_linear_fused(put(torch.zeros(M, K - 1)), w, None, stream=s), ValueError
    yield lambda s: q.w8a8_linear_fused(torch.zeros(M, K), w, None, stream=s), ValueError              # not on the device
    yield lambda s: q.w8a8_dual_gemm_fused(Xq, put(torch.ones(9)), w, None, M + 1, stream=s), ValueError


def bad_heads(put):
    M, H, D = 4, 2, 64
    z = lambda *s, **k: put(torch.zeros(*s, **k))       # noqa: E731
    Q, K = z(M, H, D), z(M, 1, D)
    pos, freq = z((M, 2), dtype=torch.int32), z(32, dtype=torch.float64)
    rope = q.Rope((32, 32), freq)
    for args, err in ((dict(Q=torch.zeros(M, H, D)), ValueError), (dict(Q=Q[0]), ValueError), (dict(Q=z(M, D, H).transpose(1, 2)), ValueError),
                      (dict(K=z(M + 1, 1, D)), ValueError), (dict(K=z(M, 1, D - 2)), ValueError), (dict(K=K.bfloat16()), ValueError),
                      (dict(Q=Q.half(), K=K.half()), TypeError),
                      (dict(K=None, out_k=Q), ValueError), (dict(K=None, weight_k=z(D)), ValueError),
                      (dict(weight_q=z(D - 1)), ValueError), (dict(weight_q=z(2 * D)), ValueError),
                      (dict(weight_q=z(D), norm=q.NORM_ROW), ValueError), (dict(weight_q=z(D), norm=q.NORM_NONE), ValueError),
                      (dict(weight_k=z(D, dtype=torch.float64)), TypeError), (dict(weight_q=z(2 * D)[::2]), ValueError),
                      (dict(out_q=K), ValueError), (dict(out_q=Q.bfloat16()), ValueError), (dict(out_q=torch.zeros(M, H, D)), ValueError),
                      (dict(norm=3), q.QarvdError), (dict(eps=-1.0), q.QarvdError), (dict(Q=Q[:, :, :0], K=None), q.QarvdError),
                      (dict(Q=Q.expand(M, H, D)[:, :1].expand(M, 2, D)), q.QarvdError),                 # heads on top of each other
                      (dict(pos=pos), ValueError), (dict(rope=rope), TypeError), (dict(rope=rope, pos=pos.long()), TypeError),
                      (dict(rope=rope, pos=pos[:3]), ValueError), (dict(rope=rope, pos=pos[:, :1]), ValueError),
                      (dict(rope=q.Rope((64,), freq), pos=pos), ValueError), (dict(rope=q.Rope((32, 32), freq.float()), pos=pos), TypeError),
                      (dict(rope=q.Rope((32, 30), freq), pos=pos), ValueError), (dict(rope=q.Rope((), freq), pos=pos), ValueError),
                      (dict(rope=q.Rope((65, -1), freq), pos=pos), q.QarvdError), (dict(rope=q.Rope((16, 16, 16, 16), freq), pos=pos), ValueError)):
        yield lambda s, a={**dict(Q=Q, K=K), **args}: q.qk_norm_rope(stream=s, **a), err
    w = q.DualScaleWeight(z((192, 256), dtype=torch.int8), put(torch.ones(192)), put(torch.ones(192)), None, 0, 192, 128)
    X = z(M, 128)
    for args, err in ((dict(heads_q=4), q.QarvdError), (dict(heads_q=0), q.QarvdError), (dict(weight_q=z(63)), ValueError), (dict(pos=pos), ValueError),
                      (dict(norm=7), q.QarvdError), (dict(eps=-1.0), q.QarvdError), (dict(out_dtype=torch.float16), TypeError)):
        yield lambda s, a={**dict(heads_q=2, heads_k=1, head_dim=64), **args}: q.w8a8_linear_qkv(X, w, None, stream=s, **a), err


@pytest.mark.parametrize("calls", [bad_endings, bad_heads])
def test_the_binding_refuses(lib, monkeypatch, calls):
    monkeypatch.setattr(binding, "_native", lambda lib, stream: None)
    monkeypatch.setattr(binding, "_on_call_device", lambda *a: None)
    monkeypatch.setattr(binding, "_stream", lambda s: 0)
    for call, err in calls(lambda t: t.as_subclass(Fake)):
        with pytest.raises(err):
            call(None)


@pytest.mark.gpu
@pytest.mark.parametrize("calls", [bad_endings, bad_heads])
def test_both_marshallings_refuse_the_same(calls):
    s = torch.cuda.Stream()
    for call, err in calls(lambda t: t.cuda()):
        for stream in (None, s):
            with pytest.raises(err):
                call(stream)


def test_tensors_of_another_device_are_refused(lib, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)

    class On:
        def __init__(self, n):
            self.n, self.device = n, "cuda:%d" % n

        def get_device(self):
            return self.n

    binding._on_call_device(None, On(1), None, On(1))
    with pytest.raises(ValueError):
        binding._on_call_device(None, On(1), On(0))

    binding._on_call_device(types.SimpleNamespace(cuda_stream=0), On(1))        # a stream that is a handle: the current device

    class Stream:
        device_index = 0

    binding._on_call_device(Stream(), On(0))
    with pytest.raises(ValueError):
        binding._on_call_device(Stream(), On(1))


def test_frequencies():
    f = q.rope_frequencies((8, 4), 100.0, "cpu")
    assert f.dtype == torch.float64 and torch.allclose(f, torch.tensor([1, 100 ** -0.25, 100 ** -0.5, 100 ** -0.75, 1, 0.1], dtype=torch.float64))
