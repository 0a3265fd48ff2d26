"""Attention over packed sequences on the GPU at sizes and layouts where its kernels' grids, forms and strides end: against the definitions
in 64 bits (tests/attention_reference.py derives the bounds)."""
import pytest
import torch

from paper_2501_17086_amd import binding as B
from tests import attention_reference as R
from tests.test_gpu_attention_ops import normal

pytestmark = pytest.mark.gpu


def test_more_workgroups_than_one_dimension_of_a_grid_holds():
    """A million sequences of one token, 16 heads, fp32: 17 million workgroups of 256 threads.  Each row is its own key's value: the weight
    is the exponential of a rounding of its score.  Roundings, f = 2^-24: the score (dh + 3) f sum |q k| scale, in the weight's
    exponent with f |lse| of its product and of the stored statistic; weights, sums and results 8 f; dout v and D, two sums of dh
    terms that cancel, (dh + 4) f sum |dout v| each, and what the weight's error makes of their difference."""
    n, H, D = 1 << 20, 16, 8
    q, k, v, do = (normal((n, H, D), torch.float32, s) for s in (1, 2, 3, 4))
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    a = B.make_attention(q, k, v, q_offsets=off, k_offsets=off)
    for t in (a.o, a.lse, a.dq, a.dk, a.dv):
        t.fill_(12345.0)
    B.hbp_attention_forward(a)
    B.hbp_attention_backward(a, do)
    scale = D ** -0.5
    for i in range(0, n, 1 << 17):
        r = slice(i, i + (1 << 17))
        qd, kd, vd, gd = (t[r].double() for t in (q, k, v, do))
        s, off_s = (qd * kd).sum(-1) * scale, (D + 3) * R.F * (qd * kd).abs().sum(-1) * scale
        lse = s * R.LOG2E
        R.assert_within(a.lse[r], lse, off_s * R.LOG2E * 1.01 + 4 * R.F * lse.abs() + 1e-37, "lse")
        R.assert_within(a.o[r], vd, vd.abs() * 8 * R.F + 1e-37, "o")
        rel = (off_s + 4 * R.F * s.abs() + 8 * R.F)[..., None] * 1.01
        R.assert_within(a.dv[r], gd, gd.abs() * rel + 1e-37, "dv")
        ds = (2 * (D + 4) + 10) * R.F * (gd * vd).abs().sum(-1, keepdim=True) * 1.01 * scale
        R.assert_within(a.dq[r], torch.zeros_like(qd), ds * kd.abs() + 1e-37, "dq")
        R.assert_within(a.dk[r], torch.zeros_like(kd), ds * qd.abs() + 1e-37, "dk")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_heads_close_behind_one_another_are_no_overlap(dtype):
    """Head after head, with room between rows and none behind a head's last row: written as any other layout."""
    n, H, D = 37, 3, 64
    row, head = D + 8, (n - 1) * (D + 8) + D
    place = lambda: torch.full(((H - 1) * head + (n - 1) * row + D,), 12345.0, dtype=dtype, device="cuda")
    x = normal((n, H, D), dtype, 5)
    want, memory = torch.empty_like(x), place()
    out = memory.as_strided((n, H, D), (row, head, 1))
    rot = B.make_rotary(D)
    B.hbp_rotary(rot, x, want)
    B.hbp_rotary(rot, x, out)
    assert torch.equal(out, want)
    out.fill_(12345.0)
    assert bool((memory == 12345.0).all())
    q, k, v, do = (normal((n, H, D), dtype, s) for s in (6, 7, 8, 9))
    a, b = B.make_attention(q, k, v), B.make_attention(q, k, v)
    for name in ("o", "dq", "dk", "dv"):
        setattr(b, name, place().as_strided((n, H, D), (row, head, 1)))
    for t in (a, b):
        B.hbp_attention_forward(t)
        B.hbp_attention_backward(t, do)
    for name in ("o", "lse", "dq", "dk", "dv"):
        assert torch.equal(getattr(a, name), getattr(b, name)), name


def test_heads_that_do_overlap_are_refused():
    memory = torch.zeros(4096, device="cuda")
    x = normal((5, 3, 64), torch.float32, 5)
    for strides in ((72, 72 * 4 + 56, 1), (56, 512, 1), (64, 64, 1), (200, 72, 1), (0, 64, 1)):
        with pytest.raises(B.HbpError):
            B.hbp_rotary(B.make_rotary(64), x, memory.as_strided((5, 3, 64), strides))
