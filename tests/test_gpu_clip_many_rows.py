"""The percentile-clip weight step over more rows than one launch has work-items for, against the same rows by themselves."""
import numpy as np
import pytest
import torch

import paper_2605_21072_amd as q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 4])
def test_more_rows_than_a_launch_has_work_items_for(bits):
    N, K = (1 << 24) + 5, 8                                  # 256 work-items a row
    at = torch.tensor([0, 1, 4, 5, (1 << 22) - 1, 1 << 22, (1 << 23) + 1, (1 << 24) - 1, 1 << 24, N - 1], device="cuda")
    rows = torch.randn((len(at), K), generator=torch.Generator(device="cuda").manual_seed(bits), device="cuda")
    W = torch.zeros((N, K), device="cuda")
    W[at] = rows
    mask = np.array([0, 1, 0, 0, 1, 0, 0, 0], dtype=np.uint8)
    w = q.quantize_weight(W, forced_mask=mask, clip_search=True, want_norms=False, bits=bits)
    few = q.quantize_weight(rows, forced_mask=mask, clip_search=True, want_norms=False, bits=bits)
    assert w.K_o == few.K_o == 2 and torch.equal(w.perm, few.perm)
    assert bool((few.s_normal > 0).all()) and torch.equal(w.s_normal[at], few.s_normal) and torch.equal(w.s_outlier[at], few.s_outlier)
    extent = w.kp * bits // 8
    assert torch.equal(w.Wq[at, :extent], few.Wq[:, :extent])
    w.s_normal[at] = w.s_outlier[at] = 0.0
    assert bool((w.s_normal == 0).all()) and bool((w.s_outlier == 0).all())
