"""A fused linear with more outputs than the kernels for few tokens have work-items for in one launch."""
import pytest
import torch

import paper_2605_21072_amd as q

pytestmark = pytest.mark.gpu


def test_more_work_items_than_a_launch_has():
    """16 work-items an output on INT4 weights from 2^28 outputs on.  One token of ones: an output is the sum of its row's codes."""
    N, K = (1 << 28) + 40, 32
    Wq = torch.zeros((N, 64), dtype=torch.uint8, device="cuda")
    at = torch.tensor([0, 1, 31, 32, 640, 1 << 27, (1 << 28) - 1, 1 << 28, N - 2, N - 1], device="cuda")
    Wq[at, 0] = torch.arange(1, 1 + len(at), device="cuda", dtype=torch.uint8) % 8          # the low half byte: one code, the others 0
    ones = torch.ones(N, device="cuda")
    w = q.DualScaleWeight(Wq, ones, ones, None, 0, N, K, None, 4)
    X = torch.ones((1, K), device="cuda")
    Y = torch.full((1, N), -1.0, dtype=torch.bfloat16, device="cuda")
    gate = torch.full((N,), 2.0, device="cuda")
    q.w8a8_linear_fused(X, w, None, gate=gate, Y=Y)
    # X's codes are 127 at a scale of 1 / 127, so that a code of 1 adds 1 within a step of bf16's
    want = 2.0 * (torch.arange(1, 1 + len(at), device="cuda") % 8)
    assert bool(((Y[0, at].float() - want).abs() <= 2.0 ** -8 * want).all())
    Y[0, at] = 0.0
    assert bool((Y == 0).all())                              # written, all of them
    Xq, s_x = q.quant_act(X, None, 0)
    few_tokens = [v for v in range(20, 23)]                  # (of INT4 weights)
    for v in few_tokens:
        with pytest.raises(q.QarvdError) as e:
            q.w8a8_dual_gemm_fused(Xq, s_x, w, None, 1, gate=gate, Y=Y, variant=v)
        assert e.value.status == -2
