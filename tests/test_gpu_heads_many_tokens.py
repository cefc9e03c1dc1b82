"""Norm and rotation over more tokens than one launch has work-items for, against the same call on a part of them."""
import pytest
import torch

import paper_2605_21072_amd as q

pytestmark = pytest.mark.gpu


def around(M, *borders):
    """Tokens at both ends and on either side of each border."""
    at = [0, 1, M - 2, M - 1] + [b + i for b in borders for i in (-1, 0, 1) if 0 <= b + i < M]
    return torch.tensor(sorted(set(at)), device="cuda")


# 64 lanes a token from 2^26 tokens on, 256 where a head needs more lanes than a wave has, from 2^24 on; what was not computed stays at 1
@pytest.mark.parametrize("M,H,D,axes,interleaved", [((1 << 26) + 5, 64, 1, (), True), ((1 << 24) + 5, 1, 512, (500,), False)])
def test_more_work_items_than_a_launch_has(M, H, D, axes, interleaved):
    x = torch.ones((M, H, D), dtype=torch.bfloat16, device="cuda")
    at = around(M, 1 << 21, 1 << 22, 1 << 24, 1 << 26)
    gen = torch.Generator(device="cuda").manual_seed(D)
    x[at] = torch.randn((len(at), H, D), generator=gen, device="cuda").bfloat16()
    pos = rope = None
    if axes:
        pos, rope = torch.arange(M, dtype=torch.int32, device="cuda").unsqueeze(1), q.Rope(axes, q.rope_frequencies(axes), interleaved)
    w = 3 + torch.rand(D, generator=gen, device="cuda")             # (a token of ones comes out above 2)
    part, _ = q.qk_norm_rope(x[at], None, q.NORM_HEAD, w, None, 1e-6, None if pos is None else pos[at], rope)
    out, _ = q.qk_norm_rope(x, None, q.NORM_HEAD, w, None, 1e-6, pos, rope, out_q=x)
    assert out is x and torch.equal(x[at], part)
    x[at] = 4.0
    last = x[:, 0, D - 1]                                           # (not rotated)
    assert bool((last > 2).all())


def test_two_launches_of_queries_and_keys():
    """A border between launches inside both tensors: strided parts of one buffer, positions in a wider table, heads first on the way out."""
    M, hq, hk, D, axes = (1 << 21) + 37, 3, 1, 8, (4, 2, 2)
    gen = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((M, 5 * D), generator=gen, device="cuda")
    Q, K = qkv[:, :hq * D].unflatten(1, (hq, D)), qkv[:, hq * D:(hq + hk) * D].unflatten(1, (hk, D))
    table = torch.randint(0, 4000, (M, 5), generator=gen, device="cuda", dtype=torch.int32)
    pos, rope = table[:, 1:4], q.Rope(axes, q.rope_frequencies(axes))
    at = around(M, 1 << 21)
    for norm in (q.NORM_NONE, q.NORM_HEAD, q.NORM_ROW):
        wq, wk = ((torch.randn(h * D if norm == q.NORM_ROW else D, generator=gen, device="cuda") if norm else None) for h in (hq, hk))
        want = q.qk_norm_rope(Q[at], K[at], norm, wq, wk, 1e-6, pos[at], rope)
        outs = [torch.zeros((h, M, D), device="cuda").transpose(0, 1) for h in (hq, hk)]
        q.qk_norm_rope(Q, K, norm, wq, wk, 1e-6, pos, rope, out_q=outs[0], out_k=outs[1])
        alone, _ = q.qk_norm_rope(Q, None, norm, wq, None, 1e-6, pos, rope)
        for got, x in ((outs[0], want[0]), (outs[1], want[1]), (alone, want[0])):
            assert torch.equal(got[at], x)
            assert bool((got != 0).flatten(1).any(1).all())         # every token was written
