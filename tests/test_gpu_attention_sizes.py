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
