"""out_dtype=None means torch's default type in the fused calls, on the current stream and on a given one."""
import pytest
import torch

import paper_2605_21072_amd as q
from paper_2605_21072_amd import binding
from test_block_layer_buffers import CALLS, Fake, parts


def call(kind, p, stream=None, **kw):
    if kind == "linear":
        return q.w8a8_linear_fused(p["X"], p["w"], None, act=1, out_dtype=None, stream=stream, **kw)
    if kind == "qkv":
        return q.w8a8_linear_qkv(p["X"], p["w"], None, 1, 1, 8, out_dtype=None, stream=stream)
    return q.w8a8_dual_gemm_fused(p["Xq"], p["s_x"], p["w"], None, p["X"].shape[0], act=1, out_dtype=None, stream=stream, **kw)


def test_the_python_path_takes_it(monkeypatch):
    """As far as the device check, which stands behind those of the types."""
    if not q.lib_path().exists():
        from paper_2605_21072_amd import build
        build.build()

    class Reached(Exception):
        pass

    def stop(*a):
        raise Reached

    monkeypatch.setattr(binding, "_native", lambda lib, stream: None)
    monkeypatch.setattr(binding, "_on_call_device", stop)
    p = parts(lambda t: t.as_subclass(Fake))
    R = torch.zeros(p["X"].shape[0], p["w"].N).as_subclass(Fake)
    for kind in CALLS:
        with pytest.raises(Reached):
            call(kind, p, **({} if kind == "qkv" else dict(residual=R)))


@pytest.mark.gpu
def test_both_marshallings_give_the_default_type():
    p = parts(lambda t: t.cuda())
    for kind in CALLS:
        for stream in (None, torch.cuda.Stream()):
            torch.cuda.synchronize()
            assert call(kind, p, stream).dtype == torch.get_default_dtype() == torch.float32
