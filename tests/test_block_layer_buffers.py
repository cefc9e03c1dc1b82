"""A layer whose buffers are not what its sizes say, or that lie elsewhere, is refused by the fused calls before anything is launched."""
import dataclasses
import types

import pytest
import torch

import paper_2605_21072_amd as q
from paper_2605_21072_amd import binding

M, N, K, K_o = 4, 16, 128, 32
CALLS = ("linear", "gemm", "qkv")


class Fake(torch.Tensor):
    """A host tensor that says it is on the device, for the Python path's own checks."""
    is_cuda = True


def parts(put):
    w = q.DualScaleWeight(put(torch.zeros((N, 256), dtype=torch.int8)), put(torch.ones(N)), put(torch.ones(N)),
                          put(torch.arange(K, dtype=torch.int32)), K_o, N, K)
    return dict(w=w, X=put(torch.ones(M, K)), Xq=put(torch.zeros((M, 256), dtype=torch.int8)), s_x=put(torch.ones(M)))


def call(kind, p, stream=None):
    if kind == "linear":
        return q.w8a8_linear_fused(p["X"], p["w"], None, act=1, stream=stream)
    if kind == "qkv":
        return q.w8a8_linear_qkv(p["X"], p["w"], None, 1, 1, 8, stream=stream)
    return q.w8a8_dual_gemm_fused(p["Xq"], p["s_x"], p["w"], None, M, act=1, stream=stream)


def bad(put):
    """(calls that refuse it, error, the replaced parts)."""
    def layer(**k):
        p = parts(put)
        p["w"] = dataclasses.replace(p["w"], **k)
        return p
    for name in ("s_normal", "s_outlier"):
        for t, err in ((torch.ones(N - 1), ValueError), (torch.ones(N).double(), TypeError), (torch.ones(2 * N)[::2], ValueError)):
            yield CALLS, err, layer(**{name: put(t)})
    for t, err in ((torch.arange(K), TypeError), (torch.arange(K - 1, dtype=torch.int32), ValueError), (torch.arange(2 * K, dtype=torch.int32)[::2], ValueError)):
        yield ("linear", "qkv"), err, layer(perm=put(t))
    yield CALLS, ValueError, layer(Wq=put(torch.zeros((N - 1, 256), dtype=torch.int8)))
    yield CALLS, ValueError, layer(Wq=put(torch.zeros((256, N), dtype=torch.int8).t()))
    yield CALLS, ValueError, layer(Wq=put(torch.zeros(N * 256, dtype=torch.int8)))
    for k, t, err in (("s_x", torch.ones(M - 1), ValueError), ("s_x", torch.ones(M).bfloat16(), TypeError), ("s_x", torch.ones(2 * M)[::2], ValueError),
                      ("Xq", torch.zeros((256, M), dtype=torch.int8).t(), ValueError), ("Xq", torch.zeros(M * 256, dtype=torch.int8), ValueError)):
        yield ("gemm",), err, {**parts(put), k: put(t)}


@pytest.fixture
def python_path(monkeypatch):
    if not q.lib_path().exists():
        from paper_2605_21072_amd import build
        build.build()
    monkeypatch.setattr(binding, "_native", lambda lib, stream: None)
    monkeypatch.setattr(binding, "_stream", lambda s: 0)


def test_the_binding_refuses(python_path, monkeypatch):
    monkeypatch.setattr(binding, "_on_call_device", lambda *a: None)
    for kinds, err, p in bad(lambda t: t.as_subclass(Fake)):
        for kind in kinds:
            with pytest.raises(err):
                call(kind, p)


def test_every_tensor_of_a_call_is_looked_up(python_path, monkeypatch):
    """All that a kernel reads is among what the device check gets; without outliers the permutation is not read."""
    class Seen(Exception):
        pass

    def stop(stream, *tensors):
        raise Seen(*tensors)

    monkeypatch.setattr(binding, "_on_call_device", stop)
    for kind, names in (("linear", ("X", "Wq", "s_normal", "s_outlier", "perm")), ("qkv", ("X", "Wq", "s_normal", "s_outlier", "perm")),
                        ("gemm", ("Xq", "s_x", "Wq", "s_normal", "s_outlier"))):
        p = parts(lambda t: t.as_subclass(Fake))
        every = {**p, **{f.name: getattr(p["w"], f.name) for f in dataclasses.fields(p["w"])}}
        with pytest.raises(Seen) as e:
            call(kind, p)
        for n in names:
            assert any(t is every[n] for t in e.value.args), (kind, n)
        p["w"].K_o = 0
        with pytest.raises(Seen) as e:
            call(kind, p)
        assert not any(t is p["w"].perm for t in e.value.args)


def test_the_native_marshalling_refuses(python_path):
    """Its GEMM call on host tensors (device -1), which never gets to the entry point."""
    host = binding._load_host(q.load_library())

    def gemm(p, device=-1):
        w = p["w"]
        return host.gemm_fused(p["Xq"], p["s_x"], 8, w.Wq, w.s_normal, w.s_outlier, None, M, N, K, K_o, 1, None, None, None, torch.bfloat16, None, 0, 0, device)

    for kinds, err, p in bad(lambda t: t):
        if "gemm" in kinds:
            with pytest.raises(err):
                gemm(p)
    with pytest.raises(ValueError):
        gemm(parts(lambda t: t), device=0)


def on_device(t):
    """The same strides, too."""
    return t.cuda() if t.is_contiguous() else torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device="cuda").copy_(t)


@pytest.mark.gpu
def test_both_marshallings_refuse_the_same():
    s = torch.cuda.Stream()
    for kinds, err, p in bad(on_device):
        for kind in kinds:
            for stream in (None, s):
                with pytest.raises(err):
                    call(kind, p, stream)
    for name in ("s_normal", "s_outlier", "perm", "s_x"):   # on the host
        for kind in CALLS:
            p = parts(lambda t: t.cuda())
            holder = p["w"] if name != "s_x" else types.SimpleNamespace()
            setattr(holder, name, (torch.arange(K, dtype=torch.int32) if name == "perm" else torch.ones(N)))
            if name == "s_x":
                p["s_x"] = holder.s_x[:M]
            if (name == "s_x" and kind != "gemm") or (name == "perm" and kind == "gemm"):
                continue
            for stream in (None, s):
                with pytest.raises(ValueError):
                    call(kind, p, stream)


@pytest.mark.gpu
def test_larger_buffers_serve_a_smaller_layer():
    """As quantize_weight_static leaves them: buffers for more outputs and channels than the layer has."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    W = torch.randn((40, 200), generator=gen, device="cuda") * 0.02
    W[:, 5] *= 40
    big = q.DualScaleWeight(torch.empty((64, 512), dtype=torch.int8, device="cuda"), *(torch.empty(64, device="cuda") for _ in range(2)),
                            torch.empty(300, dtype=torch.int32, device="cuda"), 0, 0, 0)
    w, own = q.quantize_weight_static(W, big), q.quantize_weight(W)
    assert w.K_o == own.K_o > 0
    X = torch.randn((3, 200), generator=gen, device="cuda")
    for stream in (None, torch.cuda.Stream()):
        torch.cuda.synchronize()
        a, b = (q.w8a8_linear_fused(X, v, None, act=1, stream=stream) for v in (w, own))
        torch.cuda.synchronize()
        assert torch.equal(a, b)
